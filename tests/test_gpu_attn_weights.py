"""civic_attn_weights and civic_decode_attn_weights on the GPU, through the C ABI, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_parity import log

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def bd():
    from paper_2605_28115_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return binding


def host(t):
    return np.ascontiguousarray(t.detach().float().cpu().numpy())


def group_sums(w, hkv):
    """Weights [batch, seq, H_q, s_max] -> per KV head [batch, H_kv, s_max]."""
    b, t, hq, n = w.shape
    return w.reshape(b, t, hkv, hq // hkv, n).sum(axis=(1, 3))


def sums_tolerance(w, size, hkv, d, base):
    """With u = 2^-24, Z = max_j |scale| sum |q k_j| of a softmax row: a logit is off by (d + 6) u Z (d products, the scale, what is taken off,
    the rounding of their difference), a weight by twice that relative (itself and the sum it is divided by) and 8 u for its exponential and the
    quotient.  A lane adds at most n / 16 of a row's n exponentials one by one, and the lanes' sums meet in at most 64 more additions, joined by
    exact powers of two: (n / 16 + 64) u.  Weights of r = seq * group rows are added up the same way: (r / 16 + 64) u of the total, and base u."""
    b, t, hq, n = w.shape
    off = 2 * (d + 6) * U * size[..., None] + (8 + n / 16 + 64) * U
    total = group_sums(w, hkv)
    return group_sums(w * off, hkv) + total * (t * (hq // hkv) / 16 + 64) * U + (np.abs(base) + total) * U + 1e-37


def inputs(seed, dtype, batch, seq, hq, hkv, d, s_max, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return (mk(batch, seq, hq, d) * size).to(TYPES[dtype]), mk(batch, hkv, s_max, d).to(TYPES[dtype]), mk(batch, hkv, s_max, d).to(TYPES[dtype]), mk(batch, hkv, s_max).abs()


CASES = [
    # batch, seq, H_q, H_kv, head_dim, contexts, s_max, causal
    (1, 1, 4, 2, 64, [117], 128, True),
    (1, 1, 1, 1, 8, [1], 1, True),
    (2, 5, 8, 8, 40, [5, 3], 9, True),                        # the second sample's first tokens see nothing
    (3, 7, 16, 8, 128, [0, 7, 33], 40, True),
    (3, 7, 16, 8, 128, [0, 7, 33], 33, False),
    (2, 32, 16, 8, 128, [469, 300], 471, True),
    (1, 61, 28, 4, 128, [1001], 1024, True),
    (1, 300, 8, 2, 96, [300], 301, True),
    (2, 33, 12, 4, 72, [200, 31], 200, True),
    (1, 700, 8, 2, 64, [901], 920, True),                     # more query rows than are in LDS at a time
    (2, 600, 8, 2, 64, [600, 17], 600, False),
    (1, 3, 17, 1, 128, [2500], 2600, True),                   # keys in pieces
    (1, 40, 8, 2, 256, [777], 800, True),
    (2, 9, 6, 2, 136, [64, 65], 66, True),
    (1, 130, 4, 4, 248, [131], 144, True),
    (65, 2, 2, 1, 64, list(range(65)), 64 + 5, True),
    (1, 2, 2, 2, 128, [9000], 9001, False),
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", CASES, ids=str)
def test_weights_of_rows(bd, dtype, case):
    batch, seq, hq, hkv, d, ctx, s_max, causal = case
    log("attn_weights", dtype, case)
    q, k, _, base = inputs(len(str(case)), dtype, batch, seq, hq, hkv, d, s_max)
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    for i, n in enumerate(ctx):
        k[i, :, n:] = float("nan")                            # rows behind a context have no influence
    got = bd.civic_attn_weights(q, k, max(ctx), ctx=lens, causal=causal, base=base)
    w, size = oracle.attention_weights(host(q), np.nan_to_num(host(k)), ctx, causal)
    ref = group_sums(w, hkv) + host(base)
    assert (np.abs(host(got) - ref) <= sums_tolerance(w, size, hkv, d, host(base))).all()
    # without a base, and onto the base itself: the same sums, in the same order
    none = bd.civic_attn_weights(q, k, max(ctx), ctx=lens, causal=causal, weights=torch.full_like(base, float("nan")))
    assert torch.equal(got, base + none)
    here = base.clone()
    assert bd.civic_attn_weights(q, k, max(ctx), ctx=lens, causal=causal, base=here, weights=here) is here and torch.equal(here, got)
    for i, n in enumerate(ctx):
        assert torch.equal(got[i, :, n:], base[i, :, n:]) and not none[i, :, n:].any()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", [c for c in CASES if c[2] // c[3] <= 17][:9] + [
    (2, 1, 70, 1, 64, [333, 20], 340, True),                  # more heads of a group than a round takes
    (3, 1, 40, 2, 128, [1500, 0, 64], 1500, True),
    (1, 1, 8, 2, 128, [20001], 20010, True),
    (1, 1, 8, 8, 256, [5000], 5000, True),
    (70, 1, 28, 4, 128, [(37 * i) % 700 for i in range(70)], 700, True),
], ids=str)
def test_decode_that_weighs(bd, dtype, case):
    from test_gpu_mx import tolerance
    batch, _, hq, hkv, d, ctx, s_max, _ = case
    log("decode_attn_weights", dtype, case)
    q, k, v, base = inputs(len(str(case)) + 7, dtype, batch, 1, hq, hkv, d, s_max)
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    for i, n in enumerate(ctx):
        k[i, :, n:], v[i, :, n:] = float("nan"), float("inf")
    out, got = bd.civic_decode_attn_weights(q[:, 0], k, v, max(ctx), ctx=lens, base=base)
    kh, vh = (np.nan_to_num(host(x), posinf=0.0) for x in (k, v))
    w, size = oracle.attention_weights(host(q), kh, ctx, False)
    assert (np.abs(host(got) - group_sums(w, hkv) - host(base)) <= sums_tolerance(w, size, hkv, d, host(base))).all()
    ref, wa, la = oracle.cache_attention(host(q), kh, vh, ctx, False)
    assert (np.abs(host(out) - ref[:, 0]) <= tolerance(ref, wa, la, d, s_max, dtype)[:, 0]).all()
    here = base.clone()
    again, _ = bd.civic_decode_attn_weights(q[:, 0], k, v, max(ctx), ctx=lens, base=here, weights=here)
    assert torch.equal(here, got) and torch.equal(again, out)
    _, none = bd.civic_decode_attn_weights(q[:, 0], k, v, max(ctx), ctx=lens)
    for i, n in enumerate(ctx):
        assert torch.equal(got[i, :, n:], base[i, :, n:]) and not none[i, :, n:].any()


BORDERS = [
    # (query rows of a KV head / keys: where one kernel takes over from another)
    (2, 4, 8, 2, 128, [250, 3], 260, True), (2, 4, 8, 2, 128, [251, 4], 260, True), (2, 4, 8, 2, 128, [1024, 250], 1030, True),
    (2, 4, 8, 2, 128, [1025, 17], 1030, False), (3, 1, 16, 1, 64, [5000, 0, 63], 5000, True), (2, 2, 14, 2, 96, [4100, 4000], 4100, True),
    (2, 16, 2, 2, 256, [300, 15], 300, True), (2, 5, 6, 2, 136, [2000, 1999], 2000, True), (3, 3, 8, 2, 40, [1500, 2, 700], 1501, True),
    (2, 17, 1, 1, 128, [1024, 16], 1024, True), (2, 8, 8, 2, 128, [1024, 9], 1024, True), (2, 8, 8, 2, 128, [1025, 9], 1025, True),
    (2, 33, 1, 1, 128, [512, 40], 513, True), (2, 33, 1, 1, 128, [513, 40], 513, True), (2, 16, 8, 2, 64, [512, 16], 512, False),
    (2, 65, 1, 1, 128, [512, 64], 512, True), (2, 96, 1, 1, 96, [700, 95], 700, True), (2, 97, 1, 1, 96, [700, 95], 700, True),
    (2, 300, 4, 1, 128, [9000, 8000], 9000, True),            # many pieces of keys, several of rows
    (2, 300, 4, 1, 64, [4500, 10], 4500, False),
    (512, 2, 8, 1, 64, [(37 * i) % 1500 for i in range(512)], 1500, True),   # logits that leave in rounds, rows in one piece
    (300, 1, 7, 1, 128, [(53 * i) % 500 for i in range(300)], 500, True),
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", BORDERS, ids=lambda c: str(c)[:60])
def test_weights_at_the_borders_of_the_kernels(bd, dtype, case):
    test_weights_of_rows(bd, dtype, case)


STAY = [
    # (many keys of query rows that fit LDS: 100, 256, 500, 128 of them)
    (8, 25, 32, 8, 128, [8700, 1, 8000, 7000, 5000, 100, 24, 0], 8710, True),
    (8, 64, 32, 8, 72, [8200, 8192, 8193, 63, 0, 300, 4000, 257], 8210, True),
    (4, 100, 80, 16, 64, [8300, 40, 8001, 100], 8300, True),
    (8, 32, 32, 8, 128, [8300, 256, 255, 1, 0, 8299, 8193, 8192], 8300, False),
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", STAY, ids=lambda c: str(c)[:60])
def test_many_keys_of_some_query_rows(bd, dtype, case):
    batch, seq, hq, hkv, d, ctx, s_max, causal = case
    log("attn_weights", dtype, case)
    q, k, _, base = inputs(len(str(case)), dtype, batch, seq, hq, hkv, d, s_max)
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    for i, n in enumerate(ctx):
        k[i, :, n:] = float("nan")
    got = bd.civic_attn_weights(q, k, max(ctx), ctx=lens, causal=causal, base=base)
    here = base.clone()
    assert torch.equal(bd.civic_attn_weights(q, k, max(ctx), ctx=lens, causal=causal, base=here, weights=here), got)
    for i, n in enumerate(ctx):
        assert torch.equal(got[i, :, n:], base[i, :, n:])
        for g in (0, hkv - 1):                                # (some heads: the rest of the cost is the oracle's)
            heads = slice(g * (hq // hkv), (g + 1) * (hq // hkv))
            w, size = oracle.attention_weights(host(q[i:i + 1, :, heads]), np.nan_to_num(host(k[i:i + 1, g:g + 1])), [n], causal)
            b = host(base[i:i + 1, g:g + 1])
            assert (np.abs(host(got[i:i + 1, g:g + 1]) - group_sums(w, 1) - b) <= sums_tolerance(w, size, 1, d, b)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", [
    (512, 1, 16, 1, 64, [(37 * i) % 1500 for i in range(512)], 1500, True), (257, 1, 34, 2, 128, [(37 * i) % 400 for i in range(257)], 400, True),
    (3, 1, 20, 1, 96, [700, 0, 64], 700, True), (2, 1, 32, 1, 256, [1100, 33], 1100, True), (2, 1, 5, 1, 200, [641, 640], 700, True)], ids=lambda c: str(c)[:60])
def test_decode_at_the_borders_of_the_kernels(bd, dtype, case):
    test_decode_that_weighs(bd, dtype, case)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("seq,n", [(4, 60), (4, 1000), (4, 1500), (4, 9000), (14, 900), (20, 400), (20, 1000), (100, 700), (100, 270000)])
def test_what_is_lost_with_a_nan(bd, dtype, seq, n):
    """A NaN query takes the rows that it sees with it, a NaN key the rows that the tokens see which see it; nothing else changes."""
    q, k, _, base = inputs(12, dtype, 2, seq, 4, 2, 64, n + 9)
    lens = torch.tensor([n, n - 7], dtype=torch.int32, device="cuda")
    clean = host(bd.civic_attn_weights(q, k, n, ctx=lens, base=base))
    q[0, 0, 3, 1] = float("nan")                              # (KV head 1: sees n - seq + 1 rows)
    got = host(bd.civic_attn_weights(q, k, n, ctx=lens, base=base))
    assert np.isnan(got[0, 1, :n - seq + 1]).all() and np.isfinite(got[0, 1, n - seq + 1:]).all()
    assert np.array_equal(got[0, 0], clean[0, 0]) and np.array_equal(got[1], clean[1])
    q[0, 0, 3, 1] = 0.0
    k[1, 0, n - 8, 5] = float("nan")                          # the last row of sample 1, which its last token alone sees
    got = host(bd.civic_attn_weights(q, k, n, ctx=lens, base=base))
    assert np.isnan(got[1, 0, :n - 7]).all() and np.array_equal(got[1, 0, n - 7:], clean[1, 0, n - 7:])
    assert np.array_equal(got[1, 1], clean[1, 1]) and np.array_equal(got[0, 0], clean[0, 0])
    part = host(bd.civic_attn_weights(q[1:, :-1], k[1:], n - 8, base=base[1:]))
    assert np.isfinite(part).all()


def test_one_length_for_all(bd):
    q, k, v, _ = inputs(3, "bf16", 2, 4, 8, 2, 64, 100)
    lens = torch.full((2,), 57, dtype=torch.int32, device="cuda")
    assert torch.equal(bd.civic_attn_weights(q, k, 57), bd.civic_attn_weights(q, k, 57, ctx=lens))
    # lengths beyond n_ctx are taken as n_ctx, below 0 as 0
    odd = torch.tensor([1 << 30, -5], dtype=torch.int32, device="cuda")
    got = bd.civic_attn_weights(q, k, 57, ctx=odd)
    assert torch.equal(got[0], bd.civic_attn_weights(q, k, 57)[0]) and not got[1].any()
    out, w = bd.civic_decode_attn_weights(q[:, 0].contiguous(), k, v, 57, ctx=odd)
    assert not out[1].any() and not w[1].any() and torch.equal(w[0], bd.civic_decode_attn_weights(q[:, 0].contiguous(), k, v, 57)[1][0])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("scale", [-0.3, 1e-30, 40.0])
def test_scales(bd, dtype, scale):
    """Negative, next to nothing, and so large that one row takes all."""
    from test_gpu_mx import tolerance
    q, k, v, _ = inputs(5, dtype, 2, 3, 8, 2, 64, 200)
    ctx = [200, 77]
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    w, size = oracle.attention_weights(host(q), host(k), ctx, True, scale)
    got = bd.civic_attn_weights(q, k, 200, ctx=lens, softmax_scale=scale)
    assert (np.abs(host(got) - group_sums(w, 2)) <= sums_tolerance(w, size, 2, 64, np.zeros(1))).all()
    out, got = bd.civic_decode_attn_weights(q[:, 2].contiguous(), k, v, 200, ctx=lens, softmax_scale=scale)
    w, size = oracle.attention_weights(host(q)[:, 2:], host(k), ctx, False, scale)
    assert (np.abs(host(got) - group_sums(w, 2)) <= sums_tolerance(w, size, 2, 64, np.zeros(1))).all()
    ref, wa, la = oracle.cache_attention(host(q)[:, 2:], host(k), host(v), ctx, False, scale)
    assert (np.abs(host(out) - ref[:, 0]) <= tolerance(ref, wa, la, 64, 200, dtype)[:, 0]).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_queries_of_a_projection(bd, dtype):
    """Q as a part of wider rows, heads outermost, and shared by the batch (a stride of 0)."""
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = torch.randn((2, 9, 24, 64), generator=g, device="cuda").to(TYPES[dtype])
    k = torch.randn((2, 4, 50, 64), generator=g, device="cuda").to(TYPES[dtype])
    for q in (rows[:, :, 3:11], rows[:, :, :8].transpose(1, 2).contiguous().transpose(1, 2), rows[:1, :, :8].expand(2, -1, -1, -1)):
        assert torch.equal(bd.civic_attn_weights(q, k, 50), bd.civic_attn_weights(q.contiguous(), k, 50))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_nan_and_infinities(bd, dtype):
    """A key that is NaN or infinite takes the tokens that see it with it, and no others; so does a query."""
    q, k, v, base = inputs(6, dtype, 1, 40, 4, 2, 64, 64)
    k[0, 0, 50, 3], k[0, 1, 60, 5] = float("nan"), float("inf")
    q[0, 30, 3, 1] = float("nan")                             # (KV head 1)
    got = host(bd.civic_attn_weights(q, k, 64))[0]
    kh = np.nan_to_num(host(k), posinf=0.0)
    # head 0: tokens 26 .. 39 see row 50, and with them all rows are lost; what only the first 26 would have given is lost with them
    assert np.isnan(got[0]).sum() == 64 and np.isnan(got[1]).sum() == 64
    # with the odd tokens out of the call nothing is
    w, size = oracle.attention_weights(host(q)[:, :26], kh[:, :, :50], [50], True)
    part = host(bd.civic_attn_weights(q[:, :26], k, 50))
    assert (np.abs(part[..., :50] - group_sums(w, 2)) <= sums_tolerance(w, size, 2, 64, np.zeros(1))).all()
    # rows that only later tokens see are theirs alone: the NaN query's token sees rows below 55
    k2 = inputs(6, dtype, 1, 40, 4, 2, 64, 64)[1]
    got = host(bd.civic_attn_weights(q, k2, 64))[0, 1]
    assert np.isnan(got[:55]).all() and np.isfinite(got[55:]).all()
    # V: the heads that read it
    v[0, 1, 7, 9] = float("-inf")
    out, w = bd.civic_decode_attn_weights(q[:, 0].contiguous(), k2, v, 64)
    out = host(out)[0]
    assert np.isfinite(out[:2]).all() and (out[2:, 9] == -np.inf).all() and np.isfinite(np.delete(out[2:], 9, axis=1)).all()
    assert torch.isfinite(w).all()


def test_far_logits(bd):
    """Logits of tens of thousands, the largest of them first, last and in between: the weights still add up to one for every row."""
    q, k, _, _ = inputs(8, "fp32", 1, 16, 4, 2, 64, 3000, size=4000.0)
    w, size = oracle.attention_weights(host(q), host(k), [3000], False)
    got = host(bd.civic_attn_weights(q, k, 3000, causal=False))
    assert (np.abs(got - group_sums(w, 2)) <= sums_tolerance(w, size, 2, 64, np.zeros(1))).all()
    assert abs(got.sum() - 16 * 4) <= 64 * (3000 / 16 + 200) * U * 2


def test_caches_beyond_32_bits(bd):
    """Rows whose byte offsets pass 2^32."""
    hkv, s_max, d, n = 2, 1 << 22, 256, 300
    k = torch.empty((2, hkv, s_max, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    q, kk, vv, _ = inputs(9, "bf16", 2, 1, 4, hkv, d, n)
    k[:, :, :n], v[:, :, :n] = kk, vv
    want_out, want = bd.civic_decode_attn_weights(q[:, 0], kk, vv, n)
    out, got = bd.civic_decode_attn_weights(q[:, 0], k, v, n)
    assert torch.equal(out, want_out) and torch.equal(got[..., :n], want) and not got[..., n:].any()
    got = bd.civic_attn_weights(q, k, n)
    assert torch.equal(got[..., :n], bd.civic_attn_weights(q, kk, n)) and not got[..., n:].any()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("seq", [1, 3])
def test_few_rows_of_a_long_cache_in_a_graph(bd, dtype, seq):
    """Rows in pieces, their logits in the workspace, which a second graph shares."""
    q, k, _, base = inputs(13, dtype, 2, seq, 8, 2, 128, 6000)
    lens = torch.tensor([6000, 5000], dtype=torch.int32, device="cuda")
    ws = torch.empty(bd.civic_attn_weights_workspace_bytes(q.dtype, 2, seq, 8, 2, 128, 6000), dtype=torch.uint8, device="cuda")
    sums = [torch.zeros_like(base), torch.zeros_like(base)]
    steps = [lambda: bd.civic_attn_weights(q, k, 6000, ctx=lens, base=base, weights=sums[0], workspace=ws),
             lambda: bd.civic_attn_weights(q, k, 6000, ctx=lens, causal=False, weights=sums[1], workspace=ws)]
    want = []
    for sizes in ([6000, 5000], [2, 1500], [0, 6000]):
        lens.copy_(torch.tensor(sizes, dtype=torch.int32))
        for step in steps:
            step()
        want.append([x.clone() for x in sums])
    graphs = [torch.cuda.CUDAGraph() for _ in steps]
    for graph, step in zip(graphs, steps):
        with torch.cuda.graph(graph):
            step()
    for i, sizes in ((0, [6000, 5000]), (2, [0, 6000]), (1, [2, 1500]), (0, [6000, 5000])):
        lens.copy_(torch.tensor(sizes, dtype=torch.int32))
        for x in sums:
            x.fill_(5.0)
        for graph in graphs:
            graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(sums, want[i]))


def test_on_another_stream_and_in_a_graph(bd):
    q, k, v, base = inputs(11, "bf16", 3, 6, 8, 2, 128, 700)
    lens = torch.tensor([700, 400, 9], dtype=torch.int32, device="cuda")
    q1 = q[:, 0].contiguous()
    need = [bd.civic_attn_weights_workspace_bytes(q.dtype, 3, 6, 8, 2, 128, 700), bd.civic_decode_attn_weights_workspace_bytes(q.dtype, 3, 8, 2, 128, 700)]
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in need]
    sums, out = torch.zeros_like(base), torch.empty_like(q1)

    def step():
        bd.civic_attn_weights(q, k, 700, ctx=lens, base=base, weights=sums, workspace=ws[0])
        bd.civic_decode_attn_weights(q1, k, v, 700, ctx=lens, base=sums, weights=sums, out=out, workspace=ws[1])

    step()
    want = [(sums.clone(), out.clone())]
    lens.copy_(torch.tensor([1, 0, 650], dtype=torch.int32))
    step()
    want.append((sums.clone(), out.clone()))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for i in (0, 1, 1, 0):
        lens.copy_(torch.tensor([[700, 400, 9], [1, 0, 650]][i], dtype=torch.int32))
        sums.fill_(7.0)
        graph.replay()
        assert torch.equal(sums, want[i][0]) and torch.equal(out, want[i][1])
        torch.cuda.synchronize()
    lens.copy_(torch.tensor([700, 400, 9], dtype=torch.int32))
    torch.cuda.synchronize()
    got = bd.civic_attn_weights(q, k, 700, ctx=lens, base=base, stream=side)
    o, w = bd.civic_decode_attn_weights(q1, k, v, 700, ctx=lens, base=got, stream=side)
    side.synchronize()
    assert torch.equal(w, want[0][0]) and torch.equal(o, want[0][1])


@pytest.mark.parametrize("case", [
    (3, 100, 4, 4, 128, 700),                                 # query rows in tiles, keys in pieces
    (4, 300, 8, 2, 64, 300),                                  # rows in pieces, whose totals are added up
    (8, 25, 32, 8, 128, 8700),                                # query rows that stay in LDS
    (8, 64, 16, 8, 72, 8200),
    (3, 20, 4, 2, 128, 700), (2, 90, 1, 1, 96, 700), (3, 3, 4, 2, 128, 9000),
], ids=str)
def test_far_logits_of_bf16_rows_add_up_to_one(bd, case):
    """Logits of some 40000, whole numbers and so exact in the product: what is taken off a row's exponents must not be rounded at their size, 2^-8 there
    (a weight would be off by up to 1.4e-3).  The first sample's keys are equal, every weight 1 / n; the others' logits fall by one from key to key, sixteen of them in turn.  With
    u = 2^-24 a weight's exponent is at most 64 below the base: 64 ln 2 u for its rounding, 8 u as in sums_tolerance for the exponential and the quotient, and
    sums over n keys and r rows by (n / 16 + 64 + r / 16 + 64) u."""
    batch, seq, hq, hkv, d, n = case
    log("attn_weights far", case)
    q = torch.zeros((batch, seq, hq, d), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((batch, hkv, n, d), dtype=torch.bfloat16, device="cuda")
    near = torch.arange(n, device="cuda")
    for b in range(batch):
        q[b, :, :, 0], k[b, :, :, 0] = 200.0 + 2 * b, 201.0 - b    # about 40200, another fraction of a power of two in each
        q[b, :, :, 1] = 1.0
        k[b, :, :, 1] = -(near % 16).float() if b else 0.0
    got = host(bd.civic_attn_weights(q, k, n, causal=False, softmax_scale=1.0))
    rows = seq * (hq // hkv)
    off = (64 * np.log(2) + 8 + n / 16 + 64 + rows / 16 + 64) * U
    assert np.abs(got.astype(np.float64).sum(axis=-1) - rows).max() <= rows * off
    z = -(np.arange(n) % 16).astype(np.float64)
    for b in range(batch):
        w = np.exp(z) / np.exp(z).sum() if b else np.full(n, 1.0 / n)
        # (c = log2 e in fp32 is off by u / 2 of it: 2 u |z| of a weight)
        assert (np.abs(got[b] - rows * w) <= rows * w * (off + 2 * U * np.abs(z))).all(), b


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", [
    # batch, seq, H_q, H_kv, head_dim, contexts, s_max: room behind the contexts, by the pairs' workgroups or by some of their own
    (2, 1, 8, 2, 64, [469, 17], 469 + 1024), (2, 1, 8, 2, 64, [469, 0], 469 + 1025), (1, 1, 4, 1, 128, [100], 70001), (3, 9, 8, 2, 64, [469, 30, 1], 5003),
    (2, 4, 4, 2, 128, [1000, 77], 1 << 16), (2, 40, 4, 2, 64, [300, 41], 4101), (2, 40, 4, 2, 256, [300, 41], 9000), (2, 100, 4, 2, 64, [300, 41], 40003),
    (4100, 2, 1, 1, 8, [9] * 4100, 1300), (4095, 2, 1, 1, 8, [9] * 4095, 1300), (1, 1, 2, 2, 8, [1], (1 << 22) - 1)], ids=lambda c: f"{c[:5]} {c[5][:3]} {c[6]}")
def test_room_behind_the_contexts(bd, dtype, case):
    """Rows behind a context become base's, or 0, or stay as they are, to the end of the cache and not beyond; the rows before are those of a cache without room."""
    batch, seq, hq, hkv, d, ctx, s_max = case
    log("attn_weights room", dtype, case[:5], s_max)
    n = max(ctx)
    q, k, v, _ = inputs(15, dtype, batch, seq, hq, hkv, d, n)
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    kk, vv = (torch.empty((batch, hkv, s_max, d), dtype=q.dtype, device="cuda") for _ in range(2))
    kk[:, :, :n], vv[:, :, :n] = k, v
    base = torch.rand((batch, hkv, s_max), device="cuda")
    held = torch.full((base.numel() + 64,), 3.0, device="cuda")
    q1 = q[:, 0].contiguous()
    near = base[:, :, :n].contiguous()
    for call, short in ((lambda **kw: bd.civic_attn_weights(q, kk, n, ctx=lens, **kw), bd.civic_attn_weights(q, k, n, ctx=lens, base=near)),
                        (lambda **kw: bd.civic_decode_attn_weights(q1, kk, vv, n, ctx=lens, **kw)[1], bd.civic_decode_attn_weights(q1, k, v, n, ctx=lens, base=near)[1])):
        for kind in ("other", "none", "same"):
            got = held.fill_(3.0)[32:-32].view(base.shape)
            if kind == "same":
                got.copy_(base)
            call(base=base if kind == "other" else got if kind == "same" else None, weights=got)
            assert (held[:32] == 3.0).all() and (held[-32:] == 3.0).all()
            if kind == "none":
                assert not got[:, :, n:].any() and all(not got[i, :, ctx[i]:].any() for i in range(min(batch, 5)))
            else:
                assert torch.equal(got[:, :, n:], base[:, :, n:]) and torch.equal(got[:, :, :n], short)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", [(2, 8, 2, 64, 300), (1, 8, 2, 128, 9000), (3, 70, 1, 64, 700), (1, 4, 4, 256, 5000)], ids=str)
def test_outputs_over_the_queries(bd, dtype, case):
    """out may be q: in one launch, in pieces, and with more heads of a group than a workgroup takes."""
    batch, hq, hkv, d, n = case
    q, k, v, base = inputs(17, dtype, batch, 1, hq, hkv, d, n)
    q = q[:, 0].contiguous()
    want = bd.civic_decode_attn_weights(q, k, v, n, base=base)
    got = bd.civic_decode_attn_weights(q, k, v, n, base=base, out=q)
    assert got[0] is q and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", [(2, 1, 8, 2, 64, 300), (2, 3, 8, 2, 128, 9000), (2, 16, 4, 2, 64, 500), (2, 40, 4, 2, 64, 700), (2, 40, 4, 2, 256, 300), (2, 100, 4, 2, 128, 700),
                                  (8, 25, 32, 8, 64, 8300)], ids=str)
def test_logits_of_minus_infinity(bd, dtype, case):
    """An infinite key against queries of one sign: its weight is 0, the others are those of a row without it; a row of nothing else adds nothing."""
    batch, seq, hq, hkv, d, n = case
    log("attn_weights infinity", dtype, case)
    q, k, v, _ = inputs(19, dtype, batch, seq, hq, hkv, d, n)
    q[..., 3] = q[..., 3].abs() + 0.5
    at = [0, 1, n // 2, n - seq]
    clean = k.clone()
    k[:, :, at, 3] = -float("inf")
    k[1, 1, :, 3] = -float("inf")                             # nothing else
    got = host(bd.civic_attn_weights(q, k, n, causal=False))
    assert not got[:, :, at].any() and not got[1, 1].any()
    heads = hq // hkv
    for g in range(min(hkv, 2)):                              # (sample 0: as if the rows were not there)
        rest = np.setdiff1d(np.arange(n), at)
        w, size = oracle.attention_weights(host(q[:1, :, g * heads:(g + 1) * heads]), host(clean[:1, g:g + 1, rest]), [len(rest)], False)
        assert (np.abs(got[0, g][rest] - group_sums(w, 1)[0, 0]) <= sums_tolerance(w, size, 1, d, np.zeros(1))[0, 0]).all()
    out, w = bd.civic_decode_attn_weights(q[:, 0].contiguous(), k, v, n)
    assert not w[:, :, at].any() and not w[1, 1].any() and not out[1, heads:2 * heads].any() and torch.isfinite(out.float()).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", [
    # (fp32 of up to 16 pairs and more than 384 keys: two launches)
    (2, 16, 32, 8, 64, [384, 17], 390, True), (2, 16, 32, 8, 64, [385, 17], 390, True), (17, 20, 1, 1, 40, [385 - i for i in range(17)], 385, True),
    (16, 20, 1, 1, 40, [1024 - 60 * i for i in range(16)], 1024, True), (17, 20, 1, 1, 64, [1024 - 60 * i for i in range(17)], 1024, False)], ids=lambda c: str(c)[:60])
def test_weights_where_one_launch_gives_way_to_two(bd, dtype, case):
    test_weights_of_rows(bd, dtype, case)
