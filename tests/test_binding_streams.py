"""Where the binding takes the memory of a call's own tensors from when the call names a stream (CPU: allocations, streams and the
library's entry points are stood in for; nothing is launched)."""
import contextlib

import numpy as np
import pytest
import torch

from paper_2605_28115_amd import binding as bd

GRID = (1, 4, 4, 2, 2, 1, 2, 8)                            # frames, height, width, cells, floors, budget
HERE, THERE = "the current stream", 0x5150


class Device:
    """Memory by the stream that was current when it was asked for, and what the entry points were given."""

    def __init__(self, monkeypatch):
        self.stream, self.owner, self.kept, self.recorded, self.given = HERE, {}, [], {}, None
        empty = torch.empty

        def recording_empty(*a, **kw):
            t = empty(*a, **kw)
            self.kept.append(t)
            self.owner[t.data_ptr()] = self.stream
            return t

        @contextlib.contextmanager
        def on(stream):
            before, self.stream = self.stream, stream
            yield
            self.stream = before

        monkeypatch.setattr(torch, "empty", recording_empty)
        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: handle)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda: self.stream)
        monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: self.recorded.setdefault(t.data_ptr(), []).append(s), raising=False)
        monkeypatch.setattr(bd, "_mx_placed", lambda *a: None)
        monkeypatch.setattr(bd, "_raw_stream", lambda device: 0)
        monkeypatch.setattr(bd, "_current_device", lambda: 0)
        for name in bd.EXPORTS:
            if not name.endswith(("_bytes", "_count", "_offsets")):
                monkeypatch.setattr(bd.lib, name, self.entry)

    def entry(self, *args):
        self.given = args
        return bd.CIVIC_OK


def rand(*shape, dtype=torch.bfloat16):
    return torch.randn(shape).to(dtype)


def calls():
    b, s, hq, hkv, d = 2, 40, 8, 2, 64
    hidden, ids, anchor = rand(b, 20, 64), torch.zeros(3, b, 20, dtype=torch.int32), torch.randn(64)
    q, k = rand(b, s, hq, d), rand(b, s, hkv, d)
    table = torch.randn(b, s, d // 2, 2)
    kc = rand(b, hkv, 2048, d)
    cache = bd.civic_mx_cache(b, hkv, 4096, d, 4, device="cpu")
    pk, pv = rand(b * s, hkv, d), rand(b * s, hkv, d)
    off = np.array([0, s, 2 * s], np.int64)
    return {
        "score": lambda st: bd.civic_score(hidden, anchor, stream=st),
        "score_visual": lambda st: bd.civic_score_visual(hidden, GRID, [2], anchor, stream=st),
        "select": lambda st: bd.civic_select(torch.randn(b, 16), GRID, want_flags=True, stream=st),
        "compact": lambda st: bd.civic_compact(hidden, ids, GRID, [2], torch.zeros(b, 8, dtype=torch.int32), stream=st),
        "compact_prefill": lambda st: bd.civic_compact_prefill(hidden, ids, GRID, [2], anchor, stream=st),
        "compact_prefill_ragged": lambda st: bd.civic_compact_prefill_ragged(rand(40, 64), torch.zeros(3, 40, dtype=torch.int32), [20, 20], [GRID, GRID],
                                                                             [[2], [2]], anchor, stream=st),
        "prefill_attn": lambda st: bd.civic_prefill_attn(q, k, k, stream=st),
        "prefill_attn_kv": lambda st: bd.civic_prefill_attn_kv(q, k, k, kc, kc, stream=st),
        "prefill_attn_rope": lambda st: bd.civic_prefill_attn_rope(q, k, k, table, stream=st),
        "prefill_attn_ragged": lambda st: bd.civic_prefill_attn_ragged(rand(b * s, hq, d), pk, pv, off, stream=st),
        "decode_attn": lambda st: bd.civic_decode_attn(rand(b, hq, d), kc, kc, 2000, stream=st),
        "decode_attn_ragged": lambda st: bd.civic_decode_attn_ragged(rand(b, hq, d), kc, kc, [2000, 9], stream=st),
        "mrope_table": lambda st: bd.civic_mrope_table(ids, np.zeros(32), np.ones(32), stream=st),
        "mrope_apply": lambda st: bd.civic_mrope_apply(q, table, stream=st),
        "anchor_aggregate": lambda st: bd.civic_anchor_aggregate(hidden, rand(16, 64), want_token_weight=True, stream=st),
        "kv_compress": lambda st: bd.civic_kv_compress(k, k, torch.rand(s, 8), stream=st),
        "kv_compress_ragged": lambda st: bd.civic_kv_compress_ragged(pk, pv, torch.rand(2 * s, 8), off, stream=st),
        "cross_attn": lambda st: bd.civic_cross_attn(q, k, k, stream=st),
        "cross_attn_ragged": lambda st: bd.civic_cross_attn_ragged(rand(b * s, hq, d), k, k, off, stream=st),
        "decode_attn_mx": lambda st: bd.civic_decode_attn_mx(rand(b, hq, d), cache, 4096, stream=st),
        "prefill_attn_mx": lambda st: bd.civic_prefill_attn_mx(rand(b, 5, hq, d), cache, 4096, stream=st),
    }


@pytest.mark.parametrize("name", list(calls()))
@pytest.mark.parametrize("stream", [None, THERE], ids=["unnamed", "named"])
def test_a_calls_own_tensors_come_from_the_stream_that_it_runs_on(monkeypatch, name, stream):
    call = calls()[name]
    device = Device(monkeypatch)
    result = call(stream)
    own = [p for p in device.given if isinstance(p, int) and p in device.owner]
    assert own and device.given[-1] == (0 if stream is None else stream)
    assert {device.owner[p] for p in own} == {HERE if stream is None else stream}
    # what outlives the call is not handed on before the caller's stream is through with it either; a workspace is the call's alone
    results = {t.data_ptr() for t in (result if isinstance(result, tuple) else (result,)) if t is not None}
    for p in own:
        assert device.recorded.get(p, []) == ([HERE] if stream is not None and p in results else [])


def test_the_calls_with_a_workspace_were_given_one(monkeypatch):
    """Contexts above are long enough that the attention over them is split."""
    for name in ("decode_attn", "decode_attn_ragged", "decode_attn_mx", "prefill_attn_mx", "anchor_aggregate", "kv_compress", "kv_compress_ragged"):
        call = calls()[name]
        with monkeypatch.context() as m:
            device = Device(m)
            result = call(THERE)
            results = {t.data_ptr() for t in (result if isinstance(result, tuple) else (result,))}
            assert any(isinstance(p, int) and p in device.owner and p not in results for p in device.given), name
