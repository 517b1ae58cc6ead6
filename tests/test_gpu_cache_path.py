"""The run of them together: a prompt in a cache, the weights of its last tokens, what stays of it as the prefix of several questions, their
answers token by token, and a long conversation that forgets in place; each step against the oracle."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_attn_shared import tolerance
from test_gpu_attn_weights import TYPES, bd, group_sums, host, sums_tolerance  # noqa: F401  (bd: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("seq", [1, 20, 60, 300])
def test_caches_without_rows(bd, dtype, seq):  # noqa: F811
    """n_ctx = 0: the caches may be missing; totals are what they were, outputs zeros."""
    import ctypes as C
    esz, at = (2 if dtype else 4), lambda t: None if t is None else C.c_void_p(t.data_ptr())  # noqa: E731
    q = torch.ones((2, seq, 4, 64), dtype=torch.bfloat16 if dtype else torch.float32, device="cuda")
    some = torch.ones((2, 2, 50, 64), dtype=q.dtype, device="cuda")
    out, base, w = torch.full_like(q, 3.0), torch.rand((2, 2, 50), device="cuda"), torch.full((2, 2, 50), 3.0, device="cuda")
    strides = (C.c_int64 * 3)(seq * 256, 256, 64)
    assert esz * q.numel() == q.nbytes
    ws = torch.empty(max(bd.lib.civic_attn_weights_workspace_bytes(dtype, 2, seq, 4, 2, 64, 0), 16), dtype=torch.uint8, device="cuda")
    assert bd.lib.civic_attn_weights(at(q), None, at(base), at(w), dtype, 2, seq, 4, 2, 64, strides, 50, 0, None, 1, C.c_float(0), at(ws), ws.numel(), None) == bd.CIVIC_OK
    assert torch.equal(w, base)
    w.fill_(3.0)                                              # no tokens: the same
    assert bd.lib.civic_attn_weights(None, at(some), at(base), at(w), dtype, 2, 0, 4, 2, 64, strides, 50, 50, None, 1, C.c_float(0), None, 0, None) == bd.CIVIC_OK
    assert torch.equal(w, base)
    assert bd.lib.civic_prefill_attn_shared(at(q), None, None, None, None, at(out), dtype, 2, seq, 4, 2, 64, strides, strides, 0, 0, None, 50, 0, None, 1, C.c_float(0),
                                            None, 0, None) == bd.CIVIC_OK
    assert not out.any()
    if seq == 1:
        out.fill_(3.0), w.fill_(3.0)
        assert bd.lib.civic_decode_attn_weights(at(q), None, None, at(out), None, at(w), dtype, 2, 4, 2, 64, 50, 0, None, C.c_float(0), None, 0, None) == bd.CIVIC_OK
        assert not out.any() and not w.any()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_prompt_its_questions_and_answers(bd, dtype):  # noqa: F811
    hq, hkv, d, n, keep, batch = 8, 2, 64, 500, 180, 3
    g = torch.Generator(device="cuda").manual_seed(0)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(TYPES[dtype])  # noqa: E731
    q, k, v = mk(1, n, hq, d), mk(1, n, hkv, d), mk(1, n, hkv, d)
    axis, inv = np.arange(d // 2) % 3, (1e4 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)

    def table(b, first, seq):
        ids = (first + torch.arange(seq, device="cuda", dtype=torch.int32)).expand(3, b, seq).contiguous()
        return bd.civic_mrope_table(ids, axis, inv)

    cs = table(1, 0, n)
    kc, vc = torch.zeros((1, hkv, 512, d), dtype=k.dtype, device="cuda"), torch.zeros((1, hkv, 512, d), dtype=k.dtype, device="cuda")
    bd.civic_kv_write_rope(k, v, cs, kc, vc)
    q = bd.civic_mrope_apply(q, cs)
    # the last 48 tokens look back
    w = bd.civic_attn_weights(q[:, -48:], kc, n)
    ref_w, size = oracle.attention_weights(host(q[:, -48:]), host(kc), [n], True)
    assert (np.abs(host(w) - group_sums(ref_w, hkv)) <= sums_tolerance(ref_w, size, hkv, d, np.zeros(1))).all()
    kp, vp, wp, idx, held = bd.civic_kv_evict(kc, vc, w, keep, n, first=4, recent=48)
    kept = oracle.evict(w.cpu().numpy(), [n], keep, 4, 48)[0]
    assert [idx[0, h].tolist() for h in range(hkv)] == kept and held.tolist() == [keep]
    # questions of 11 tokens, then tokens one by one, at the positions behind the whole prompt
    own_k, own_v = (torch.full((batch, hkv, 32, d), float("nan"), dtype=k.dtype, device="cuda") for _ in range(2))
    rows = 0
    for seq in (11, 1, 1):
        q, k, v = mk(batch, seq, hq, d), mk(batch, seq, hkv, d), mk(batch, seq, hkv, d)
        cs = table(batch, n + rows, seq)
        bd.civic_kv_write_rope(k, v, cs, own_k, own_v, rows)
        q = bd.civic_mrope_apply(q, cs)
        rows += seq
        if seq > 1:
            out = bd.civic_prefill_attn_shared(q, kp[0], vp[0], own_k, own_v, rows, prefix_ctx=held)
        else:
            out = bd.civic_decode_attn_shared(q[:, 0], kp[0], vp[0], own_k, own_v, rows, prefix_ctx=held)[:, None]
        ref, wa, la = oracle.shared_attention(host(q), host(kp[0]), host(vp[0]), np.nan_to_num(host(own_k)), np.nan_to_num(host(own_v)), [rows] * batch, True)
        assert (np.abs(host(out) - ref) <= tolerance(ref, wa, la, d, keep + rows, dtype, True)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_conversation_that_forgets_in_place(bd, dtype):  # noqa: F811
    """200 tokens through a cache of 64 rows: every step adds a row and its weights, every 16 or so the cache goes back to 48 rows."""
    batch, hq, hkv, d, room, keep = 2, 4, 2, 64, 64, 48
    g = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(TYPES[dtype])  # noqa: E731
    kc, vc = (torch.zeros((batch, hkv, room, d), dtype=TYPES[dtype], device="cuda") for _ in range(2))
    w = torch.zeros((batch, hkv, room), device="cuda")
    seen, n = [], 0                                            # every token's K and V; rows held
    rows = np.zeros((batch, hkv, 0), np.int64)                 # the tokens that the rows are
    for step in range(200):
        k, v, q = mk(batch, 1, hkv, d), mk(batch, 1, hkv, d), mk(batch, hq, d)
        bd.civic_kv_write(k, v, kc, vc, n)
        seen.append((host(k)[:, 0], host(v)[:, 0]))
        rows = np.concatenate((rows, np.full((batch, hkv, 1), step)), axis=2)
        n += 1
        before = host(w)
        out, _ = bd.civic_decode_attn_weights(q, kc, vc, n, base=w, weights=w)
        if step % 7 == 0 or n == room:
            kh, vh = (np.stack([[np.stack([seen[t][x][b, h] for t in rows[b, h]]) for h in range(hkv)] for b in range(batch)]) for x in range(2))
            ref, wa, la = oracle.cache_attention(host(q)[:, None], kh, vh, [n] * batch, False)
            assert (np.abs(host(out) - ref[:, 0]) <= tolerance(ref, wa, la, d, n, dtype, False)[:, 0]).all()
            ref_w, size = oracle.attention_weights(host(q)[:, None], kh, [n] * batch, False)
            got = host(w)
            assert (np.abs(got[..., :n] - before[..., :n] - group_sums(ref_w, hkv)) <= sums_tolerance(ref_w, size, hkv, d, got[..., :n]) + np.abs(got[..., :n]) * 2.0 ** -24).all()
            assert not got[..., n:].any()
        if n == room:
            kept = oracle.evict(w.cpu().numpy(), [n] * batch, keep, 4, 8)
            bd.civic_kv_evict(kc, vc, w, keep, n, first=4, recent=8, k_out=kc, v_out=vc, weights_out=w)
            rows = np.stack([[rows[b, h][kept[b][h]] for h in range(hkv)] for b in range(batch)])
            n = keep
