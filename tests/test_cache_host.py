"""Host side of the calls that weigh, evict and share cache rows: refusals before any launch, workspace sizes, streams, and the oracle's
functions against closed forms (no call reaches the GPU)."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle
from paper_2605_28115_amd import binding as bd
from test_binding_streams import HERE, THERE, Device, rand

F, ODD, F2, F3 = C.c_void_p(1 << 40), C.c_void_p((1 << 40) + 2), C.c_void_p(2 << 40), C.c_void_p(3 << 40)
I, W, X = bd.ERR_INVALID_ARG, bd.ERR_WORKSPACE, bd.ERR_UNSUPPORTED


def strides(*s):
    return (C.c_int64 * 3)(*s)


def weights(q=F, k=F, base=None, out=F2, dt=1, b=2, t=3, hq=8, hkv=2, d=64, qs=(1536, 512, 64), s_max=100, n=90, ctx=None, scale=0.0, ws=None, wsb=0):
    return bd.lib.civic_attn_weights(q, k, base, out, dt, b, t, hq, hkv, d, None if qs is None else strides(*qs), s_max, n, ctx, 1, C.c_float(scale), ws, wsb, None)


def decode(q=F, k=F, v=F, out=F, base=None, w=F2, dt=1, b=2, hq=8, hkv=2, d=64, s_max=100, n=90, ctx=None, scale=0.0, ws=None, wsb=0):
    return bd.lib.civic_decode_attn_weights(q, k, v, out, base, w, dt, b, hq, hkv, d, s_max, n, ctx, C.c_float(scale), ws, wsb, None)


def evict(k=F, v=F2, w=F3, dt=1, b=2, hkv=2, d=64, s_max=100, n=90, ctx=None, keep=40, first=4, recent=8, ko=C.c_void_p(4 << 40), vo=C.c_void_p(5 << 40),
          wo=C.c_void_p(6 << 40), idx=C.c_void_p(7 << 40), co=None, s_out=50, ws=None, wsb=0):
    return bd.lib.civic_kv_evict(k, v, w, dt, b, hkv, d, s_max, n, ctx, keep, first, recent, ko, vo, wo, idx, co, s_out, ws, wsb, None)


def shared(q=F, kp=F, vp=F, k=F, v=F, out=F, dt=1, b=2, t=3, hq=8, hkv=2, d=64, qs=(1536, 512, 64), os=(1536, 512, 64), sp=100, n_p=90, pc=None, s_max=100,
           n=90, ctx=None, scale=0.0, ws=None, wsb=0):
    return bd.lib.civic_prefill_attn_shared(q, kp, vp, k, v, out, dt, b, t, hq, hkv, d, None if qs is None else strides(*qs), None if os is None else strides(*os),
                                            sp, n_p, pc, s_max, n, ctx, 1, C.c_float(scale), ws, wsb, None)


SIZES = [dict(dt=7), dict(b=-1), dict(hkv=0), dict(d=0), dict(d=60), dict(n=-1), dict(n=101), dict(s_max=-1)]
ATTENTION = [dict(hq=7), dict(hq=0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(k=None), dict(q=ODD), dict(k=ODD), dict(ws=ODD), dict(ctx=ODD)]


@pytest.mark.parametrize("bad", SIZES + ATTENTION + [dict(t=-1), dict(out=None), dict(out=ODD), dict(base=ODD), dict(qs=None), dict(qs=(1536, 512, 60)),
                                                      dict(qs=(1536, -512, 64)), dict(qs=(1536, 512, 56)), dict(base=C.c_void_p((2 << 40) + 4))], ids=str)
def test_weights_refuses(bad):
    assert weights(**bad) == I


@pytest.mark.parametrize("bad", SIZES + ATTENTION + [dict(v=None), dict(out=None), dict(w=None), dict(out=ODD), dict(v=ODD), dict(w=ODD), dict(base=ODD),
                                                      dict(base=C.c_void_p((2 << 40) + 1596))], ids=str)
def test_decode_that_weighs_refuses(bad):
    assert decode(**bad) == I


@pytest.mark.parametrize("bad", SIZES + [
    dict(k=None), dict(v=None), dict(w=None), dict(ko=None), dict(vo=None), dict(idx=None), dict(k=ODD), dict(ko=ODD), dict(w=ODD), dict(wo=ODD), dict(idx=ODD),
    dict(ctx=ODD), dict(co=ODD), dict(ws=ODD), dict(keep=-1), dict(first=-1), dict(recent=-1), dict(first=33), dict(recent=2 ** 62), dict(s_out=39), dict(s_out=-1),
    dict(ko=F), dict(ko=F, s_out=100), dict(ko=F, vo=F, s_out=100), dict(ko=F2, vo=F, s_out=100), dict(ko=F, vo=F2), dict(ko=C.c_void_p((1 << 40) + 16)),
    dict(vo=C.c_void_p((2 << 40) + 100 * 4 * 128 - 16)), dict(ko=C.c_void_p(5 << 40)), dict(wo=F3), dict(wo=C.c_void_p((3 << 40) + 4)),
    dict(ctx=F, co=C.c_void_p((1 << 40) + 4))], ids=str)
def test_evict_refuses(bad):
    assert evict(**bad) == I


@pytest.mark.parametrize("bad", SIZES + ATTENTION + [
    dict(t=-1), dict(v=None), dict(kp=None), dict(vp=None), dict(out=None), dict(kp=ODD), dict(vp=ODD), dict(v=ODD), dict(out=ODD), dict(pc=ODD), dict(n_p=-1),
    dict(n_p=101), dict(sp=-1), dict(qs=None), dict(os=None), dict(qs=(1536, 512, 60)), dict(os=(1536, 512, 56)), dict(os=(0, 512, 64)), dict(os=(1536, 0, 64)),
    dict(os=(1536, 448, 64)), dict(os=(512, 512, 64)), dict(os=(2 ** 62, 2 ** 62, 64))], ids=str)
def test_shared_refuses(bad):
    assert shared(**bad) == I


def test_what_is_not_covered():
    wide = dict(d=264, qs=(8000, 2112, 264))
    assert weights(**wide) == X and shared(**wide, os=(8000, 2112, 264)) == X and decode(d=264) == X
    for call in (weights, decode, shared):
        assert call(s_max=(1 << 22) + 1) == X
    assert evict(d=264) == X and evict(s_max=(1 << 22) + 1) == X and evict(s_out=(1 << 22) + 1) == X
    assert shared(sp=(1 << 22) + 1) == X
    assert weights(b=1 << 23) == X and weights(b=1 << 19, s_max=1 << 22, n=1 << 22) == W and decode(b=1 << 21) == X and shared(b=1 << 21) == X and evict(b=1 << 21) == X
    assert evict(b=1 << 19, n=100, keep=4000, s_out=4000, s_max=4000) == W


@pytest.mark.parametrize("dt,d", [(1, 8), (1, 64), (1, 128), (1, 256), (0, 256)])
def test_as_many_pairs_as_are_covered(dt, d):
    """Into other arrays 2^21 pairs of any width and 2^23 chunks of 64 rows; in place the rows' width counts, the chunks do not."""
    far = dict(dt=dt, d=d, hkv=1, s_max=100, n=90, first=0, recent=0, v=C.c_void_p(1 << 50), w=C.c_void_p(2 << 50), ko=C.c_void_p(3 << 50), vo=C.c_void_p(4 << 50),
               wo=C.c_void_p(5 << 50), idx=C.c_void_p(6 << 50))
    assert evict(**far, b=1 << 21, keep=1) == W and evict(**far, b=(1 << 21) + 1, keep=1) == X
    many = dict(far, s_max=4000, n=4000, s_out=4000)
    assert evict(**many, b=1 << 17, keep=4000) == W and evict(**many, b=(1 << 23) // 63 + 1, keep=4000) == X
    most = ((1 << 21) - 1) // -(-d * (2 if dt else 4) // 128)
    here = dict(far, k=F, ko=F, vo=far["v"], s_out=100)
    assert evict(**here, b=most, keep=1) == W and evict(**here, b=most + 1, keep=1) == X
    here = dict(many, k=F, ko=F, vo=far["v"], s_out=4000)
    assert evict(**here, b=min(most, (1 << 23) // 63 + 1), keep=4000) == W


def test_a_missing_or_small_workspace_is_refused():
    need = bd.civic_attn_weights_workspace_bytes(torch.bfloat16, 2, 3, 8, 2, 64, 90)
    assert need > 0 and weights() == W and weights(ws=F3, wsb=need - 1) == W
    need = bd.civic_decode_attn_weights_workspace_bytes(torch.bfloat16, 2, 8, 2, 64, 90)
    assert need > 0 and decode() == W and decode(ws=F3, wsb=need - 1) == W
    need = bd.civic_kv_evict_workspace_bytes(2, 2, 90)
    assert need > 0 and evict() == W and evict(ws=C.c_void_p(8 << 40), wsb=need - 1) == W
    assert evict(ko=F, vo=F2, wo=F3, s_out=100) == W          # in place, and no other fault
    need = bd.civic_attn_shared_workspace_bytes(torch.bfloat16, 2, 3, 8, 2, 64, 9000, 90)
    long = dict(sp=9000, n_p=9000)
    assert need > 0 and shared(**long) == W and shared(**long, ws=F3, wsb=need - 1) == W


def at(n, by=0):
    return C.c_void_p((n << 40) + by)


def test_written_memory_is_shared_with_nothing():
    """Each pair of arrays of which a call writes one, where their first or last 16 bytes meet."""
    big = 1 << 30                                              # bytes of workspace that are there
    k, sums = 4 * 100 * 128, 4 * 100 * 4                       # bytes of 4 x 100 rows of 64 bf16 channels, of their weights

    good = dict(q=at(1), k=at(2), out=at(3), base=at(4), ctx=at(5), ws=at(6), wsb=big)
    size = dict(q=6144, k=k, out=sums, base=sums, ctx=8, ws=bd.civic_attn_weights_workspace_bytes(torch.bfloat16, 2, 3, 8, 2, 64, 90))
    names = list(size)
    for i, written in enumerate(names):
        for j, other in enumerate(names):
            if i == j or written not in ("out", "ws") or {written, other} == {"out", "base"}:
                continue
            for by in (0, (size[other] - 1) // 16 * 16):
                assert weights(**dict(good, **{written: at(j + 1, by)})) == I, (written, other, by)
    assert weights(**dict(good, qs=(2 ** 62, 2 ** 62, 64), b=4, out=at(1, 1 << 20))) == I   # (a reach that no 64 bits hold)

    good = dict(q=at(1), k=at(2), v=at(3), out=at(4), w=at(5), base=at(6), ctx=at(7), ws=at(8), wsb=big)
    size = dict(q=2048, k=k, v=k, out=2048, w=sums, base=sums, ctx=8, ws=bd.civic_decode_attn_weights_workspace_bytes(torch.bfloat16, 2, 8, 2, 64, 90))
    names = list(size)
    for i, written in enumerate(names):
        for j, other in enumerate(names):
            if i == j or written not in ("out", "w", "ws") or (written, other) == ("w", "base"):
                continue
            for by in (0, (size[other] - 1) // 16 * 16):
                if (written, other, by) != ("out", "q", 0):
                    assert decode(**dict(good, **{written: at(j + 1, by)})) == I, (written, other, by)

    good = dict(k=at(1), v=at(2), w=at(3), ko=at(4), vo=at(5), wo=at(6), idx=at(7), co=at(8), ctx=at(9), ws=at(10), wsb=big)
    size = dict(k=k, v=k, w=sums, ko=4 * 50 * 128, vo=4 * 50 * 128, wo=4 * 50 * 4, idx=4 * 40 * 4, co=8, ctx=8, ws=bd.civic_kv_evict_workspace_bytes(2, 2, 90))
    names = list(size)
    for i, written in enumerate(names):
        for j, other in enumerate(names):
            if i == j or written in ("k", "v", "w", "ctx"):
                continue
            for by in (0, (size[other] - 1) // 16 * 16):
                if (written, other, by) != ("co", "ctx", 0):
                    assert evict(**dict(good, **{written: at(j + 1, by)})) == I, (written, other, by)
    good = dict(q=at(1), kp=at(2), vp=at(3), k=at(4), v=at(5), out=at(6), ctx=at(7), pc=at(8), ws=at(9), wsb=big, sp=9000, n_p=9000)
    size = dict(q=6144, kp=2 * 9000 * 128, vp=2 * 9000 * 128, k=k, v=k, out=6144, ctx=8, pc=4, ws=bd.civic_attn_shared_workspace_bytes(torch.bfloat16, 2, 3, 8, 2, 64, 9000, 90))
    names = list(size)
    for i, written in enumerate(names):
        for j, other in enumerate(names):
            if i == j or written not in ("out", "ws") or (written, other) == ("out", "q"):
                continue
            for by in (0, (size[other] - 1) // 16 * 16):
                assert shared(**dict(good, **{written: at(j + 1, by)})) == I, (written, other, by)

    good = dict(k=at(1), v=at(2), w=at(3), ko=at(4), vo=at(5), wo=at(6), idx=at(7), co=at(8), ctx=at(9), ws=at(10), wsb=big)
    # in place, and a workspace that is too small: no other fault
    assert evict(**dict(good, ko=at(1), vo=at(2), wo=at(3), co=at(9), s_out=100, wsb=0)) == W


def test_calls_without_work_launch_nothing():
    assert weights(b=0, q=None, k=None, out=None) == bd.CIVIC_OK and weights(s_max=0, n=0, out=None, k=None) == bd.CIVIC_OK
    assert decode(b=0, q=None, k=None, v=None, out=None, w=None) == bd.CIVIC_OK
    assert evict(b=0, k=None, v=None, w=None, ko=None, vo=None, wo=None, idx=None) == bd.CIVIC_OK
    assert shared(b=0, q=None, out=None) == bd.CIVIC_OK and shared(t=0, q=None, out=None) == bd.CIVIC_OK


def test_types_that_are_not_there():
    for call, sizes in ((bd.civic_attn_weights_workspace_bytes, (1, 1, 2, 2, 8, 1)), (bd.civic_decode_attn_weights_workspace_bytes, (1, 2, 2, 8, 1)),
                        (bd.civic_attn_shared_workspace_bytes, (1, 1, 2, 2, 8, 1, 1))):
        with pytest.raises(TypeError):
            call(torch.float16, *sizes)


def test_bytes_of_sizes_out_of_range_are_none():
    L = bd.lib
    assert L.civic_attn_weights_workspace_bytes(9, 1, 1, 1, 1, 8, 1) == 0 and L.civic_attn_weights_workspace_bytes(1, 1, 1, 3, 2, 8, 1) == 0
    assert L.civic_decode_attn_weights_workspace_bytes(1, 1, 1, 1, 264, 1) == 0 and L.civic_kv_evict_workspace_bytes(-1, 1, 1) == 0
    assert L.civic_attn_shared_workspace_bytes(1, 1, 1, 1, 1, 8, -1, 1) == 0 and L.civic_attn_shared_workspace_bytes(1, 1, 0, 1, 1, 8, 1, 1) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("sizes", [(1, 1, 4, 2, 64), (4, 1, 16, 8, 128), (64, 1, 32, 8, 128), (16, 61, 28, 4, 128), (1, 300, 8, 2, 128), (3, 5, 16, 8, 96),
                                   (2, 40, 8, 2, 256), (2, 64, 16, 2, 128), (9, 1, 34, 2, 96), (28, 46, 32, 4, 256), (16, 4, 16, 8, 256), (12, 1, 32, 2, 256)], ids=str)
def test_a_workspace_for_a_length_serves_the_shorter_ones(dtype, sizes):
    b, t, hq, hkv, d = sizes
    around = sorted({max(m + k, 0) for m in range(0, 9000, 64) for k in (-1, 0, 1)} | {1 << 16, 100000, 1 << 20, 1 << 22})
    prefixes = (0, 1, 33, 500, 8001, 1 << 22)
    last, last_d, last_s = 0, 0, {}
    for n in around:
        need = bd.civic_attn_weights_workspace_bytes(dtype, b, t, hq, hkv, d, n)
        assert need >= last, n
        last = need
        need = bd.civic_decode_attn_weights_workspace_bytes(dtype, b, hq, hkv, d, n)
        assert need >= last_d, n
        last_d = need
        row = [bd.civic_attn_shared_workspace_bytes(dtype, b, t, hq, hkv, d, p, n) for p in prefixes]
        assert row == sorted(row) and all(x >= last_s.get(p, 0) for p, x in zip(prefixes, row)), n
        last_s = dict(zip(prefixes, row))
    row = [bd.civic_attn_shared_workspace_bytes(dtype, b, t, hq, hkv, d, p, 100) for p in around]
    assert row == sorted(row)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("sizes", [
    (16, 8192, 32, 8, 128, 8192, 8192), (16, 8192, 32, 8, 80, 8192, 8192), (1, 32768, 32, 8, 80, 0, 32768), (64, 8192, 64, 8, 8, 8192, 0),
    (4, 2000, 16, 4, 256, 70, 2000), (1, 1 << 22, 8, 1, 8, 1 << 22, 1 << 22), (2, 100, 32, 8, 192, 1 << 20, 100), (1024, 40, 32, 8, 72, 0, 60000),
    (1, 33, 1, 1, 248, 1 << 22, 0)], ids=str)
def test_pieces_of_prompts_do_not_grow_with_rows_times_keys(dtype, sizes):
    """More than 32 rows a KV head: a grid that fills the chip is not cut (its launch has fewer than 2^32 threads, and no workspace), one that does not
    makes 3840 pieces of 32 rows at most."""
    b, t, hq, hkv, d, prefix, n = sizes
    most = 3840 * 32 * (d + 2) * 4 + 16
    assert bd.civic_attn_shared_workspace_bytes(dtype, b, t, hq, hkv, d, prefix, n) <= most
    if b * hkv * (t * (hq // hkv) // 32) >= 3840:
        assert bd.civic_attn_shared_workspace_bytes(dtype, b, t, hq, hkv, d, prefix, n) == 0


def calls():
    b, hq, hkv, d = 2, 8, 2, 64
    kc, q, w = rand(b, hkv, 3000, d), rand(b, 5, hq, d), torch.rand(b, hkv, 3000)
    return {
        "weights": lambda st: bd.civic_attn_weights(q, kc, 2900, stream=st),
        "decode": lambda st: bd.civic_decode_attn_weights(rand(b, hq, d), kc, kc, 2900, stream=st),
        "evict": lambda st: bd.civic_kv_evict(kc, kc, w, 500, 2900, stream=st),
        "decode_shared": lambda st: bd.civic_decode_attn_shared(rand(b, hq, d), kc[0], kc[0], kc, kc, 2900, stream=st),
        "prefill_shared": lambda st: bd.civic_prefill_attn_shared(q, kc[0], kc[0], kc, kc, 2900, stream=st),
    }


@pytest.mark.parametrize("name", list(calls()))
@pytest.mark.parametrize("stream", [None, THERE], ids=["unnamed", "named"])
def test_a_calls_own_tensors_come_from_the_stream_that_it_runs_on(monkeypatch, name, stream):
    call = calls()[name]
    device = Device(monkeypatch)
    monkeypatch.setattr(bd, "_placed", lambda *a: None)
    result = call(stream)
    own = [p for p in device.given if isinstance(p, int) and p in device.owner]
    assert own and device.given[-1] == (0 if stream is None else stream)
    assert {device.owner[p] for p in own} == {HERE if stream is None else stream}
    results = {t.data_ptr() for t in (result if isinstance(result, tuple) else (result,))}
    assert any(p not in results for p in own)                 # a workspace among them
    for p in own:
        assert device.recorded.get(p, []) == ([HERE] if stream is not None and p in results else [])


def test_the_binding_checks_shapes_types_and_places(monkeypatch):
    b, hq, hkv, d = 2, 8, 2, 64
    q, kc, w = torch.zeros(b, 3, hq, d), torch.zeros(b, hkv, 50, d), torch.zeros(b, hkv, 50)
    bad = [
        lambda: bd.civic_attn_weights(q.to(torch.bfloat16), kc, 50), lambda: bd.civic_attn_weights(q[:1], kc, 50), lambda: bd.civic_attn_weights(q[:, 0], kc, 50),
        lambda: bd.civic_attn_weights(q, kc[:, :, ::2], 25), lambda: bd.civic_attn_weights(q, kc, 50, base=w.double()), lambda: bd.civic_attn_weights(q, kc, 50, weights=w[..., :40]),
        lambda: bd.civic_decode_attn_weights(q, kc, kc, 50), lambda: bd.civic_decode_attn_weights(q[:, 0], kc, kc, 50), lambda: bd.civic_decode_attn_weights(q[:, 0].contiguous(), kc, kc[..., :40, :], 50),
        lambda: bd.civic_kv_evict(kc, kc, w, 10, 50, k_out=kc), lambda: bd.civic_kv_evict(kc, kc, w.half(), 10, 50), lambda: bd.civic_kv_evict(kc, kc, w, 10, 50, kept_idx=torch.zeros(b, hkv, 9, dtype=torch.int32)),
        lambda: bd.civic_kv_evict(kc, kc, w, 10, 50, k_out=kc.half(), v_out=kc.half()), lambda: bd.civic_prefill_attn_shared(q, kc[0, :1], kc[0, :1], kc, kc, 50),
        lambda: bd.civic_prefill_attn_shared(q, kc[0], kc[0], kc, kc, 50, prefix_ctx=torch.zeros(2, dtype=torch.int32)), lambda: bd.civic_prefill_attn_shared(q, kc[0].half(), kc[0], kc, kc, 50),
        lambda: bd.civic_decode_attn_shared(q[:, 0], kc[0], kc[0], kc, kc, 50), lambda: bd.civic_prefill_attn_shared(q, kc[0], kc[0], kc, kc, 50, out=q[:, :2]),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: bd.civic_attn_weights(q, kc, 50), lambda: bd.civic_kv_evict(kc, kc.clone(), w, 10, 50), lambda: bd.civic_prefill_attn_shared(q, kc[0], kc[0], kc, kc, 50)):
        with pytest.raises(ValueError, match="device"):        # host tensors
            call()
    monkeypatch.setattr(bd, "_placed", lambda *a: None)
    monkeypatch.setattr(bd, "_stream", lambda stream: 0)
    with pytest.raises(ValueError):                            # one int32 a sample
        bd.civic_attn_weights(q, kc, 50, ctx=torch.zeros(2, dtype=torch.int64))
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(64, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            bd.civic_attn_weights(q, kc, 50, workspace=ws)


# --------------------------------------------------------------------------------------------------------------- oracle
def test_oracle_weights_of_a_token_add_up_to_one():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 4, 6, 8)).astype(np.float32), rng.standard_normal((2, 2, 9, 8)).astype(np.float32)
    for causal in (False, True):
        w, _ = oracle.attention_weights(q, k, [9, 2], causal)
        total = w.sum(axis=-1)
        assert np.allclose(total[0], 1) and np.allclose(total[1], [[1 if not causal or 2 - (3 - i) > 0 else 0] * 6 for i in range(4)])
        assert not w[1, :, :, 2:].any()
    # equal keys: the mean over what a token sees; against attention over one-hot values
    w, _ = oracle.attention_weights(q, np.ones_like(k), [9, 9], True)
    assert np.allclose(w[0, 1, 0, :7], 1 / 7) and not w[0, 1, 0, 7:].any()
    one_hot = np.broadcast_to(np.eye(9, 8, dtype=np.float32), (2, 2, 9, 8)).copy()
    w, _ = oracle.attention_weights(q, k, [9, 9], True)
    assert np.allclose(oracle.cache_attention(q, k, one_hot, [9, 9], True)[0], w[..., :8])


def test_oracle_evict_by_hand():
    w = np.array([[[5, 1, 1, 9, 0, 7, 1, 2]]], np.float32)
    assert oracle.evict(w, [8], 4, 1, 1) == [[[0, 3, 5, 7]]]
    assert oracle.evict(w, [8], 5, 1, 1) == [[[0, 1, 3, 5, 7]]]              # of three equal ones the lowest
    assert oracle.evict(w, [7], 4, 0, 2) == [[[0, 3, 5, 6]]] and oracle.evict(w, [3], 4, 1, 1) == [[[0, 1, 2]]]
    assert oracle.evict(np.array([[[np.nan, -1, -0.0, 0.0]]]), [4], 2, 0, 0) == [[[2, 3]]] and oracle.evict(w, [8], 0, 0, 0) == [[[]]]


def test_oracle_shared_is_one_long_cache():
    rng = np.random.default_rng(1)
    mk = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    q, kp, vp, k, v = mk(2, 5, 4, 8), mk(2, 7, 8), mk(2, 7, 8), mk(2, 2, 6, 8), mk(2, 2, 6, 8)
    both = [np.concatenate((np.broadcast_to(p, (2,) + p.shape), c), axis=2) for p, c in ((kp, k), (vp, v))]
    for causal in (False, True):
        out, _, _ = oracle.shared_attention(q, kp, vp, k, v, [6, 6], causal)
        assert np.allclose(out, oracle.cache_attention(q, *both, [13, 13], causal)[0])
    # a sample with fewer rows than tokens: the first ones see the prefix alone
    out, _, _ = oracle.shared_attention(q, kp, vp, k, v, [6, 2], True)
    assert np.allclose(out[1, :3], oracle.cache_attention(q[1:, :3], kp[None], vp[None], [7], False)[0])
    assert not oracle.shared_attention(q, kp[:, :0], vp[:, :0], k, v, [6, 2], True)[0][1, :3].any()
