"""civic_kv_evict on the GPU, through the C ABI, against the oracle: rows, weights and numbers to the bit."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_parity import log

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def bd():
    from paper_2605_28115_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return binding


def caches(seed, dtype, batch, hkv, s_max, d):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((batch, hkv, s_max, d), generator=g, device="cuda").to(TYPES[dtype]) for _ in range(2))
    return k, v, torch.exp(3.0 * torch.randn((batch, hkv, s_max), generator=g, device="cuda"))


def check(got, k, v, weights, ctx, keep, first, recent, before=None):
    """`before`: what k_out and v_out held (rows behind the kept ones are left as they were)."""
    k_out, v_out, w_out, idx, ctx_out = got
    kept = oracle.evict(weights.cpu().numpy(), ctx, keep, first, recent)
    assert ctx_out.tolist() == [min(n, keep) for n in ctx]
    idx_h, w_h, w = idx.cpu().numpy(), w_out.cpu().numpy(), weights.cpu().numpy()
    for b, heads in enumerate(kept):
        for g, rows in enumerate(heads):
            m = len(rows)
            assert idx_h[b, g, :m].tolist() == rows and (idx_h[b, g, m:] == -1).all()
            assert np.array_equal(w_h[b, g, :m], w[b, g, rows], equal_nan=True) and not w_h[b, g, m:].any()
            at = torch.tensor(rows, dtype=torch.long, device="cuda")
            for out, src, old in ((k_out, k, before[0] if before else None), (v_out, v, before[1] if before else None)):
                assert torch.equal(out[b, g, :m].view(torch.uint8), src[b, g, at].view(torch.uint8))
                if old is not None:
                    assert torch.equal(out[b, g, m:].view(torch.uint8), old[b, g, m:].view(torch.uint8))


CASES = [
    # batch, H_kv, head_dim, contexts, s_max, keep, first, recent
    (1, 8, 128, [469], 512, 156, 4, 32),
    (1, 1, 8, [1], 1, 1, 0, 0),
    (1, 2, 64, [117], 128, 117, 0, 0),
    (3, 2, 64, [0, 5, 90], 90, 17, 3, 4),
    (2, 3, 40, [33, 64], 65, 32, 32, 0),                       # the first rows alone
    (2, 3, 72, [33, 64], 65, 32, 0, 32),                       # the latest alone
    (2, 2, 96, [200, 199], 201, 1, 0, 0),
    (2, 2, 136, [1024, 1025], 1025, 1024, 0, 0),               # one row goes
    (1, 2, 256, [3000], 3001, 1777, 16, 100),
    (5, 4, 128, [700, 1, 3584, 2048, 2049], 3584, 1024, 4, 128),
    (1, 1, 64, [70001], 70001, 30011, 5, 6),
    (2, 2, 128, [50, 60], 64, 0, 0, 0),                        # nothing stays
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", CASES, ids=str)
def test_rows_that_stay(bd, dtype, case):
    batch, hkv, d, ctx, s_max, keep, first, recent = case
    log("kv_evict", dtype, case)
    k, v, w = caches(len(str(case)), dtype, batch, hkv, s_max, d)
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    check(bd.civic_kv_evict(k, v, w, keep, max(ctx), ctx=lens, first=first, recent=recent), k, v, w, ctx, keep, first, recent)
    # into larger caches, which keep what lies behind
    k2, v2, w2 = caches(1, dtype, batch, hkv, max(keep, 1) + 5, d)
    old = k2.clone(), v2.clone()
    check(bd.civic_kv_evict(k, v, w, keep, max(ctx), ctx=lens, first=first, recent=recent, k_out=k2, v_out=v2, weights_out=w2), k, v, w, ctx, keep,
          first, recent, old)
    # in place: caches, weights and lengths
    if keep <= s_max:
        ki, vi, wi, li = k.clone(), v.clone(), w.clone(), lens.clone()
        got = bd.civic_kv_evict(ki, vi, wi, keep, max(ctx), ctx=li, first=first, recent=recent, k_out=ki, v_out=vi, weights_out=wi, ctx_out=li)
        assert got[0] is ki and got[2] is wi and got[4] is li
        check(got, k, v, w, ctx, keep, first, recent, (k, v))


LONG = [
    # (caches that are selected from in pieces)
    (3, 2, 64, [16385, 4096, 0], 16385, 4095, 4, 32),
    (2, 1, 8, [40960, 8193], 40961, 8192, 1, 1),
    (1, 3, 40, [20481], 20490, 20480, 0, 0),                   # one row goes
    (4, 1, 16, [33000, 20000, 12289, 17], 33000, 9000, 4500, 4500),   # the ends alone
    (2, 2, 8, [300001, 131073], 300001, 70000, 5, 9000),
    (260, 2, 8, [16390 - 70 * i if i < 3 else i for i in range(260)], 16400, 100, 1, 2),   # more pairs than units: a piece each
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", LONG, ids=lambda c: str(c)[:60])
def test_rows_of_long_caches_that_stay(bd, dtype, case):
    test_rows_that_stay(bd, dtype, case)


@pytest.mark.parametrize("in_place", [False, True])
def test_equal_weights_of_long_caches(bd, in_place):
    """Ties that lie in several pieces, weights that are all equal, NaN, infinities, numbers below the normal ones."""
    n = 40000
    k, v, w = caches(4, "bf16", 6, 1, n, 8)
    rng = np.random.default_rng(0)
    w[0] = 0.0
    w[1] = torch.from_numpy(rng.integers(0, 4, (1, n)).astype(np.float32)).cuda()
    w[2, :, ::3], w[2, :, 1::3] = 0.0, -0.0
    w[3, :, ::2] = float("nan")
    w[4, :, :15000], w[4, :, 15000:20000] = float("inf"), float("-inf")
    w[5] = torch.from_numpy(rng.integers(0, 50, (1, n)).astype(np.float32) * np.float32(1e-45)).cuda()
    ctx = [n, n - 1, n, 30000, n, 25000]
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    ki, vi, wi = (x.clone() for x in (k, v, w))
    kw = dict(k_out=ki, v_out=vi, weights_out=wi) if in_place else {}
    check(bd.civic_kv_evict(ki, vi, wi, 21000, n, ctx=lens, first=2, recent=33, **kw), k, v, w, ctx, 21000, 2, 33)


def test_a_long_cache_forgets_in_a_graph(bd):
    k, v, w = caches(9, "bf16", 2, 2, 30000, 16)
    lens = torch.tensor([30000, 20000], dtype=torch.int32, device="cuda")
    idx = torch.empty((2, 2, 9000), dtype=torch.int32, device="cuda")
    ws = torch.empty(bd.civic_kv_evict_workspace_bytes(2, 2, 30000) + 4, dtype=torch.uint8, device="cuda")[4:]
    first = [x.clone() for x in (k, v, w, lens)]
    step = lambda: bd.civic_kv_evict(k, v, w, 9000, 30000, ctx=lens, first=4, recent=20, k_out=k, v_out=v, weights_out=w, kept_idx=idx, ctx_out=lens, workspace=ws)  # noqa: E731
    step()
    for x, y in zip((k, v, w, lens), first):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for ctx in ([30000, 20000], [9001, 5], [30000, 30000]):
        lens.copy_(torch.tensor(ctx, dtype=torch.int32))
        w.copy_(first[2].roll(sum(ctx), dims=2))
        old = [x.clone() for x in (k, v, w)]
        graph.replay()
        torch.cuda.synchronize()
        check((k, v, w, idx, lens), *old, ctx, 9000, 4, 20, old[:2])


@pytest.mark.parametrize("n", [90, 20000])
def test_nothing_stays_of_caches_that_are_not_there(bd, n):
    """keep = 0: no cache, weight or number is read or written, and they may be missing; the lengths are 0."""
    import ctypes as C
    out, lens = torch.full((2, 1, 40), 3.0, device="cuda"), torch.full((2,), 7, dtype=torch.int32, device="cuda")
    ws = torch.empty(bd.civic_kv_evict_workspace_bytes(2, 1, n), dtype=torch.uint8, device="cuda")
    rc = bd.lib.civic_kv_evict(None, None, None, 1, 2, 1, 64, n, n, None, 0, 0, 0, None, None, C.c_void_p(out.data_ptr()), None, C.c_void_p(lens.data_ptr()), 40,
                               C.c_void_p(ws.data_ptr()), ws.numel(), None)
    torch.cuda.synchronize()
    assert rc == bd.CIVIC_OK and not out.any() and not lens.any()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", [c for c in CASES if c[5] <= c[4]], ids=str)
def test_in_place_with_lengths_of_their_own(bd, dtype, case):
    """The new lengths beside the old ones, which stay; no weights out."""
    batch, hkv, d, ctx, s_max, keep, first, recent = case
    log("kv_evict in place", dtype, case)
    k, v, w = caches(len(str(case)) + 1, dtype, batch, hkv, s_max, d)
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    ki, vi, wi = k.clone(), v.clone(), w.clone()
    got = bd.civic_kv_evict(ki, vi, wi, keep, max(ctx), ctx=lens, first=first, recent=recent, k_out=ki, v_out=vi, weights_out=wi)
    check(got, k, v, w, ctx, keep, first, recent, (k, v))
    assert lens.tolist() == ctx


@pytest.mark.parametrize("in_place", [False, True])
def test_equal_weights_and_odd_ones(bd, in_place):
    """Weights that are equal (all, or at the border), zeros of both signs, infinities, NaN, numbers below the normal ones."""
    k, v, w = caches(4, "bf16", 8, 2, 3000, 64)
    rng = np.random.default_rng(0)
    w[0] = 0.0
    w[1] = torch.from_numpy(rng.integers(0, 4, (2, 3000)).astype(np.float32)).cuda()
    w[2, :, ::3], w[2, :, 1::3] = 0.0, -0.0
    w[3, :, ::2] = float("nan")
    w[4, :, :1500], w[4, :, 1500:2000] = float("inf"), float("-inf")
    w[5] = torch.from_numpy(rng.integers(0, 50, (2, 3000)).astype(np.float32) * np.float32(1e-45)).cuda()
    w[6] = -w[6]
    w[7] = float("nan")
    ctx = [3000, 2999, 3000, 3000, 3000, 1200, 3000, 3000]
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    ki, vi, wi = (x.clone() for x in (k, v, w))
    kw = dict(k_out=ki, v_out=vi, weights_out=wi) if in_place else {}
    check(bd.civic_kv_evict(ki, vi, wi, 1100, 3000, ctx=lens, first=2, recent=33, **kw), k, v, w, ctx, 1100, 2, 33)


def test_one_length_for_all_and_lengths_out_of_range(bd):
    k, v, w = caches(5, "fp32", 2, 2, 100, 64)
    check(bd.civic_kv_evict(k, v, w, 40, 90, first=1, recent=2), k, v, w, [90, 90], 40, 1, 2)
    lens = torch.tensor([1000, -3], dtype=torch.int32, device="cuda")
    check(bd.civic_kv_evict(k, v, w, 40, 90, ctx=lens, first=1, recent=2), k, v, w, [90, 0], 40, 1, 2)


def test_rows_beyond_32_bits(bd):
    hkv, s_max, d = 2, 1 << 22, 256
    k = torch.empty((2, hkv, s_max, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    kk, vv, ww = caches(6, "bf16", 2, hkv, 500, d)
    w = torch.zeros((2, hkv, s_max), device="cuda")
    # few rows at the far end of the last head are what is kept
    far = s_max - 500
    k[:, :, far:], v[:, :, far:], w[:, :, far:] = kk, vv, ww
    got = bd.civic_kv_evict(k, v, w, 300, s_max)
    kept = oracle.evict(ww.cpu().numpy(), [500, 500], 300, 0, 0)
    for b in range(2):
        for g in range(hkv):
            assert got[3][b, g].tolist() == [far + r for r in kept[b][g]]
            assert torch.equal(got[0][b, g], kk[b, g, kept[b][g]]) and torch.equal(got[1][b, g], vv[b, g, kept[b][g]])
    k_first = k[1, 1, far:].clone()
    bd.civic_kv_evict(k, v, w, 300, s_max, k_out=k, v_out=v, weights_out=w)
    assert torch.equal(k[1, 1, :300], got[0][1, 1]) and torch.equal(v[1, 1, :300], got[1][1, 1]) and torch.equal(k[1, 1, far:], k_first)


def test_in_a_graph_into_other_caches(bd):
    """Short rows, captured: selected and moved in one launch."""
    k, v, w = caches(8, "bf16", 3, 2, 400, 64)
    lens = torch.tensor([400, 100, 0], dtype=torch.int32, device="cuda")
    out = dict(k_out=torch.zeros((3, 2, 70, 64), dtype=torch.bfloat16, device="cuda"), v_out=torch.zeros((3, 2, 70, 64), dtype=torch.bfloat16, device="cuda"),
               weights_out=torch.zeros((3, 2, 70), device="cuda"), kept_idx=torch.empty((3, 2, 64), dtype=torch.int32, device="cuda"),
               ctx_out=torch.empty(3, dtype=torch.int32, device="cuda"))
    ws = torch.empty(bd.civic_kv_evict_workspace_bytes(3, 2, 400), dtype=torch.uint8, device="cuda")
    step = lambda: bd.civic_kv_evict(k, v, w, 64, 400, ctx=lens, first=4, recent=20, workspace=ws, **out)  # noqa: E731
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for ctx in ([400, 100, 0], [64, 65, 63], [399, 1, 400]):
        lens.copy_(torch.tensor(ctx, dtype=torch.int32))
        w.copy_(w.roll(sum(ctx), dims=2))
        old = out["k_out"].clone(), out["v_out"].clone()
        graph.replay()
        torch.cuda.synchronize()
        check(got, k, v, w, ctx, 64, 4, 20, old)


def test_in_a_graph_a_cache_forgets_again_and_again(bd):
    """Captured in place, replayed on what the last replay left."""
    k, v, w = caches(7, "bf16", 3, 2, 600, 128)
    lens = torch.tensor([600, 500, 40], dtype=torch.int32, device="cuda")
    idx = torch.empty((3, 2, 350), dtype=torch.int32, device="cuda")
    ws = torch.empty(bd.civic_kv_evict_workspace_bytes(3, 2, 600), dtype=torch.uint8, device="cuda")
    first = [x.clone() for x in (k, v, w, lens)]

    def step():
        return bd.civic_kv_evict(k, v, w, 350, 600, ctx=lens, first=4, recent=20, k_out=k, v_out=v, weights_out=w, kept_idx=idx, ctx_out=lens, workspace=ws)

    step()                                                    # (loads the library's code)
    for x, y in zip((k, v, w, lens), first):
        x.copy_(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for ctx in ([600, 500, 40], [351, 350, 599], [600, 600, 600]):
        lens.copy_(torch.tensor(ctx, dtype=torch.int32))
        w.copy_(first[2].roll(sum(ctx), dims=2))
        old = [x.clone() for x in (k, v, w)]
        graph.replay()
        torch.cuda.synchronize()
        check((k, v, w, idx, lens), *old, ctx, 350, 4, 20, old[:2])


@pytest.mark.parametrize("lengths_too", [False, True], ids=["", "lengths in place"])
def test_as_many_pairs_as_are_covered(bd, lengths_too):
    """2^21 pairs into other arrays, in one launch and (where the lengths are changed in place) in two."""
    pairs = 1 << 21
    log("kv_evict", pairs, lengths_too)
    k, v, w = caches(21, "bf16", pairs, 1, 2, 8)
    lens = torch.full((pairs,), 2, dtype=torch.int32, device="cuda")
    k_out, v_out, w_out, idx, ctx_out = bd.civic_kv_evict(k, v, w, 1, 2, ctx=lens, ctx_out=lens if lengths_too else None)
    want = (w[:, 0, 1] > w[:, 0, 0]).to(torch.int32)
    at = torch.arange(pairs, device="cuda"), torch.zeros(pairs, dtype=torch.long, device="cuda"), want.long()
    assert torch.equal(idx[:, 0, 0], want) and (ctx_out == 1).all() and torch.equal(w_out[:, 0, 0], w[at])
    assert torch.equal(k_out[:, 0, 0].view(torch.int16), k[at].view(torch.int16)) and torch.equal(v_out[:, 0, 0].view(torch.int16), v[at].view(torch.int16))


@pytest.mark.parametrize("in_place", [False, True], ids=["", "in place"])
@pytest.mark.parametrize("ctx,keep,s_out", [([469, 3], 156, 469 + 1024), ([469, 3], 156, 469 + 1025), ([469, 469], 156, 70001), ([9000, 2000], 3000, 40000), ([9000, 2000], 6000, 7001),
                                            ([17000, 9], 500, 70001), ([17000, 16999], 500, 17001), ([0, 0], 9, 9000), ([5], 2, (1 << 22) - 1), ([20000], 7000, 1 << 21)], ids=str)
def test_room_behind_the_rows(bd, in_place, ctx, keep, s_out):
    """weights_out is cleared behind the kept rows to the end of its memory and not beyond, whoever does it."""
    n, hkv = max(ctx), 3
    if in_place and s_out < n:
        return
    log("kv_evict room", ctx, keep, s_out, in_place)
    k, v, w = caches(31, "bf16", len(ctx), hkv, max(n, 1), 8)
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    want = bd.civic_kv_evict(k, v, w, keep, n, ctx=lens, first=1, recent=1)
    check(want, k, v, w, ctx, keep, 1, 1)
    kk, vv = (torch.zeros((len(ctx), hkv, s_out, 8), dtype=k.dtype, device="cuda") for _ in range(2))
    held = torch.full((len(ctx) * hkv * s_out + 64,), 3.0, device="cuda")
    ww = held[32:-32].view(len(ctx), hkv, s_out)
    if in_place:
        kk[:, :, :n], vv[:, :, :n], ww[:, :, :n] = k[:, :, :n], v[:, :, :n], w[:, :, :n]
        got = bd.civic_kv_evict(kk, vv, ww, keep, n, ctx=lens, first=1, recent=1, k_out=kk, v_out=vv, weights_out=ww)
    else:
        got = bd.civic_kv_evict(k, v, w, keep, n, ctx=lens, first=1, recent=1, k_out=kk, v_out=vv, weights_out=ww)
    most = min(keep, n)
    assert (held[:32] == 3.0).all() and (held[-32:] == 3.0).all() and not ww[:, :, most:].any()
    assert torch.equal(ww[:, :, :most], want[2][:, :, :most]) and torch.equal(got[3], want[3]) and torch.equal(got[4], want[4])
    for i, m in enumerate(min(x, keep) for x in ctx):
        assert torch.equal(kk[i, :, :m], want[0][i, :, :m]) and torch.equal(vv[i, :, :m], want[1][i, :, :m])
