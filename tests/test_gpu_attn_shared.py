"""civic_decode_attn_shared and civic_prefill_attn_shared on the GPU, through the C ABI, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_attn_weights import TYPES, U, bd, host  # noqa: F401  (bd: the fixture)
from test_gpu_parity import log

pytestmark = pytest.mark.gpu


def tolerance(ref, weight_abs, logit_abs, d, n, dtype, once):
    """Per row, with w the weights, A = sum w max|v|, Z = max |scale| sum |q k|, u = 2^-24 and n the keys: a weight is off by 2 (d + 6) u Z + 8 u
    relative (its logit and the sum it is divided by; exponential, quotient), sums of n weights and of n products with V by (n / 16 + 64) u each
    (a lane adds at most n / 16 of them one by one).  bf16: a weight as two bf16 terms leaves 2^-16 of it, the output is rounded by half a step,
    2^-8 of it; fp32: u.  `once`: bf16 weights of many rows may be rounded to bf16 once, by at most 2^-8 of a weight: 2^-8 (A + |out|)."""
    a = weight_abs[..., None]
    off = a * (2 * (d + 6) * U * logit_abs[..., None] + 8 * U + 2 * (n / 16 + 64) * U + (2.0 ** -16 if dtype == "bf16" else U))
    own = np.abs(ref) * (2.0 ** -8 if dtype == "bf16" else U)
    if once and dtype == "bf16":
        own = own + 2.0 ** -8 * (a + np.abs(ref)) * (1 + 2.0 ** -7)
    return off + own


def inputs(seed, dtype, batch, seq, hq, hkv, d, s_prefix, s_max):
    g = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(TYPES[dtype])  # noqa: E731
    return mk(batch, seq, hq, d), mk(hkv, s_prefix, d), mk(hkv, s_prefix, d), mk(batch, hkv, s_max, d), mk(batch, hkv, s_max, d)


CASES = [
    # batch, seq, H_q, H_kv, head_dim, prefix rows, contexts, s_max, causal
    (1, 1, 4, 2, 64, 117, [3], 8, True),
    (4, 1, 16, 8, 128, 469, [1, 23, 7, 0], 64, True),
    (1, 1, 1, 1, 8, 1, [0], 1, True),
    (3, 1, 8, 8, 40, 5, [0, 1, 2], 3, True),
    (3, 1, 28, 4, 128, 33, [40, 0, 64], 64, True),
    (2, 1, 8, 2, 64, 0, [70, 0], 71, True),                    # no prefix
    (65, 1, 8, 2, 128, 1000, list(range(65)), 65, True),
    (9, 1, 34, 2, 96, 300, [31, 32, 33, 0, 1, 2, 500, 64, 65], 500, True),   # 17 heads a group
    (2, 1, 70, 1, 256, 129, [300, 10], 300, True),             # more than 32 rows of a sample
    (5, 5, 16, 8, 128, 600, [5, 9, 3, 0, 100], 100, True),     # drafted tokens; some see none of their own rows
    (5, 5, 16, 8, 128, 600, [5, 9, 3, 0, 100], 100, False),
    (3, 61, 28, 4, 128, 401, [61, 200, 70], 201, True),
    (2, 100, 8, 2, 64, 257, [100, 50], 100, True),
    (2, 130, 4, 4, 96, 64, [131, 130], 144, False),
    (1, 300, 8, 2, 128, 1000, [700], 700, True),
    (2, 33, 12, 4, 72, 63, [40, 33], 40, True),
    (2, 17, 8, 2, 256, 200, [64, 17], 64, True),
    (2, 200, 8, 8, 128, 0, [200, 317], 317, True),             # a chunk over plain caches
    (2, 40, 6, 2, 136, 100, [0, 41], 41, True),                # a sample without rows of its own
    (1, 7, 4, 2, 64, 9000, [7], 7, True),
    (2, 64, 16, 2, 128, 3000, [64, 100], 100, True),
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", CASES, ids=str)
def test_behind_a_shared_prefix(bd, dtype, case):  # noqa: F811
    batch, seq, hq, hkv, d, prefix, ctx, s_max, causal = case
    log("attn_shared", dtype, case)
    q, kp, vp, kc, vc = inputs(len(str(case)), dtype, batch, seq, hq, hkv, d, prefix + 3, s_max)
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    kp[:, prefix:], vp[:, prefix:] = float("nan"), float("inf")   # rows behind a length have no influence
    for i, n in enumerate(ctx):
        kc[i, :, n:], vc[i, :, n:] = float("inf"), float("nan")
    kw = dict(ctx=lens, n_prefix=prefix)
    if seq == 1:
        out = bd.civic_decode_attn_shared(q[:, 0], kp, vp, kc, vc, max(ctx), **kw)[:, None]
        long = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, max(ctx), causal=causal, **kw)
        assert torch.equal(out, long)
    else:
        out = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, max(ctx), causal=causal, **kw)
    clean = [np.nan_to_num(host(x), posinf=0.0) for x in (kp[:, :prefix], vp[:, :prefix], kc, vc)]
    ref, wa, la = oracle.shared_attention(host(q), *clean, ctx, causal)
    rows = seq * (hq // hkv)
    assert (np.abs(host(out) - ref) <= tolerance(ref, wa, la, d, prefix + s_max, dtype, rows > 32 or batch * rows > 32)).all()
    # the prefix's length on the device, in longer memory
    count = torch.tensor([prefix], dtype=torch.int32, device="cuda")
    same = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, s_max, ctx=lens, causal=causal, prefix_ctx=count)
    assert (np.abs(host(same) - ref) <= tolerance(ref, wa, la, d, prefix + s_max, dtype, rows > 32 or batch * rows > 32)).all()


LONG = [
    # (prefixes whose workgroups serve all samples: longer than 2048 rows, or behind more than 256 pairs)
    (5, 1, 16, 8, 128, 2500, [1, 0, 33, 64, 7], 64, True),     # 10 rows a KV head
    (9, 1, 16, 8, 128, 2500, [1, 0, 33, 64, 7, 500, 31, 32, 2], 500, True),   # 18
    (65, 1, 8, 2, 128, 2500, list(range(65)), 65, True),       # 260
    (20, 1, 16, 2, 64, 2100, [(29 * i) % 100 for i in range(20)], 100, True),
    (20, 1, 8, 2, 96, 2049, [(29 * i) % 100 for i in range(20)], 100, True),
    (3, 1, 34, 2, 96, 2600, [1000, 0, 5], 1000, True),         # 17 of a sample
    (4, 8, 8, 2, 64, 3000, [100, 8, 7, 0], 100, True),         # 32 of a sample, some of which see none of their own
    (3, 16, 4, 2, 128, 2500, [40, 16, 300], 300, False),
    (2, 17, 4, 2, 128, 2500, [40, 16], 300, True),             # 34
    (40, 1, 16, 8, 128, 100, [(29 * i) % 64 for i in range(40)], 64, True),   # 320 pairs
    (150, 2, 8, 2, 64, 33, [(29 * i) % 40 for i in range(150)], 40, True),
    (6, 1, 12, 4, 72, 2200, [1, 0, 33, 64, 7, 70], 70, True),
    (6, 2, 8, 2, 256, 2200, [1, 0, 33, 64, 7, 70], 70, True),
    (12, 2, 8, 2, 40, 2200, [(29 * i) % 64 for i in range(12)], 64, True),
    (4, 1, 8, 2, 64, 20000, [3000, 1, 0, 64], 3000, True),
    (6, 8, 8, 2, 256, 2200, [1, 0, 33, 64, 7, 70], 70, True),  # 32 rows of 256 channels, 192 together
    (20, 1, 16, 8, 256, 2100, [(29 * i) % 100 for i in range(20)], 100, True),
    (3, 100, 8, 2, 256, 300, [100, 333, 99], 333, True),       # 400
    (24, 4, 16, 8, 256, 3500, [(29 * i) % 100 for i in range(24)], 100, True),   # 256 channels with much work: the prefix by many rows at a time
    (12, 8, 16, 4, 256, 4000, [8 + i for i in range(12)], 20, False),
    (4, 100, 16, 4, 256, 700, [100, 333, 99, 0], 333, True),
    (2, 160, 16, 4, 256, 0, [1000, 64], 1000, False),
    (1, 130, 16, 2, 256, 3000, [200], 200, True),
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", LONG, ids=lambda c: str(c)[:60])
def test_behind_a_long_prefix(bd, dtype, case):  # noqa: F811
    test_behind_a_shared_prefix(bd, dtype, case)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("scale", [-0.2, 1e-30, 30.0])
@pytest.mark.parametrize("sizes", [(3, 1, 8, 2, 64), (2, 70, 4, 2, 128)], ids=str)
def test_scales(bd, dtype, scale, sizes):  # noqa: F811
    batch, seq, hq, hkv, d = sizes
    q, kp, vp, kc, vc = inputs(2, dtype, *sizes, 150, 90)
    out = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 90, softmax_scale=scale)
    ref, wa, la = oracle.shared_attention(host(q), host(kp), host(vp), host(kc), host(vc), [90] * batch, True, scale)
    assert (np.abs(host(out) - ref) <= tolerance(ref, wa, la, d, 240, dtype, True)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_far_logits(bd, dtype):  # noqa: F811
    """Logits of thousands whose largest lies in the prefix for some rows and in their own cache for others."""
    for batch, seq, prefix in ((5, 1, 700), (2, 50, 700), (3, 1, 2200), (5, 4, 2200)):
        q, kp, vp, kc, vc = inputs(3, dtype, batch, seq, 8, 2, 64, prefix, 200)
        q = (q.float() * 800).to(q.dtype)
        out = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 200)
        ref, wa, la = oracle.shared_attention(host(q), host(kp), host(vp), host(kc), host(vc), [200] * batch, True)
        assert (np.abs(host(out) - ref) <= tolerance(ref, wa, la, 64, prefix + 200, dtype, True)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("sizes", [(3, 1, 8, 2, 64), (3, 4, 8, 2, 128), (2, 70, 4, 2, 128), (2, 70, 4, 2, 64), (2, 40, 4, 2, 72), (2, 40, 4, 2, 256)], ids=str)
def test_infinities_and_nan_reach_who_sees_them(bd, dtype, sizes):  # noqa: F811
    reach(bd, dtype, sizes, 100)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("sizes", [(3, 1, 8, 2, 64), (9, 1, 8, 2, 128), (9, 4, 8, 2, 96), (4, 16, 4, 2, 64), (4, 16, 4, 2, 128), (5, 9, 4, 2, 96), (40, 4, 16, 8, 256), (4, 150, 16, 4, 256), (3, 3, 8, 2, 72),
                                   (3, 3, 8, 2, 256)], ids=str)
def test_infinities_and_nan_behind_a_long_prefix(bd, dtype, sizes):  # noqa: F811
    reach(bd, dtype, sizes, 2300)


def reach(bd, dtype, sizes, prefix):  # noqa: F811
    batch, seq, hq, hkv, d = sizes
    q, kp, vp, kc, vc = inputs(4, dtype, *sizes, prefix, 128)
    n = [128, 90]
    lens = torch.tensor((n * batch)[:batch], dtype=torch.int32, device="cuda")
    want = host(bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 128, ctx=lens))
    others = [i for i in range(batch) if i != 1]
    at = 90 - (seq + 1) // 2                                   # of sample 1: seen by the later half of its tokens
    vc[1, 0, at, 5], vc[1, 1, at, 3] = float("inf"), float("nan")
    vc[1, :, 90:] = float("nan")
    out = host(bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 128, ctx=lens))
    group = hq // hkv
    sees = np.array([at < 90 - (seq - 1 - i) for i in range(seq)])
    hit = np.zeros(out.shape, bool)
    hit[1, sees, :group, 5] = True
    assert (out[hit] == np.inf).all()
    nan = np.zeros(out.shape, bool)
    nan[1, sees, group:2 * group, 3] = True                   # (KV head 1)
    assert np.isnan(out[nan]).all()
    # everything else is what it was, but for the roundings of a sum made another way
    rest = ~(hit | nan)
    ref, wa, la = oracle.shared_attention(host(q), host(kp), host(vp), host(kc), np.nan_to_num(host(vc), posinf=0.0), lens.tolist(), True)
    assert (np.abs(out - want)[rest] <= 2 * tolerance(ref, wa, la, d, prefix + 128, dtype, True)[rest]).all()
    # a NaN key: the softmax rows that see it
    kc[1, 1, at, 0] = float("nan")
    out = host(bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 128, ctx=lens))
    assert np.isnan(out[1, sees, group:2 * group]).all() and np.isfinite(out[1, ~sees]).all() and np.isfinite(out[others]).all()
    # in the prefix: everyone
    vp[0, 50, 7] = float("-inf")
    out = host(bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 128, ctx=lens))
    assert (out[:, :, :group, 7] == -np.inf).all() and np.isfinite(out[others][:, :, group:]).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_strided_queries_and_outputs(bd, dtype):  # noqa: F811
    for seq, prefix in ((1, 90), (5, 90), (80, 90), (1, 2100), (5, 2100)):
        q, kp, vp, kc, vc = inputs(5, dtype, 2, seq, 8, 2, 64, prefix, 100)
        want = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 100)
        wide = torch.full((2, seq, 20, 64), 7.0, device="cuda", dtype=q.dtype)
        wide[:, :, 3:11] = q
        out = torch.full((2, 8, seq + 2, 64), 9.0, device="cuda", dtype=q.dtype)
        got = bd.civic_prefill_attn_shared(wide[:, :, 3:11], kp, vp, kc, vc, 100, out=out[:, :, 1:-1].transpose(1, 2))
        assert torch.equal(got, want) and (out[:, :, 0] == 9.0).all() and (out[:, :, -1] == 9.0).all()


def test_lengths_out_of_range(bd):  # noqa: F811
    q, kp, vp, kc, vc = inputs(6, "bf16", 2, 3, 8, 2, 64, 90, 100)
    want = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 60, n_prefix=50)
    lens = torch.tensor([1 << 30, 60], dtype=torch.int32, device="cuda")
    assert torch.equal(bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 60, ctx=lens, n_prefix=50, prefix_ctx=torch.tensor([77], dtype=torch.int32, device="cuda")), want)
    none = torch.tensor([-1, 0], dtype=torch.int32, device="cuda")
    out = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 60, ctx=none, n_prefix=50, prefix_ctx=torch.tensor([-3], dtype=torch.int32, device="cuda"))
    assert not out.any()


def test_the_same_on_every_call_in_a_graph_and_on_another_stream(bd):  # noqa: F811
    for batch, seq, prefix in ((6, 1, 2000), (3, 40, 2000), (3, 1, 4000), (6, 5, 4000)):
        q, kp, vp, kc, vc = inputs(7, "bf16", batch, seq, 16, 4, 128, prefix, 300)
        lens = torch.full((batch,), 300, dtype=torch.int32, device="cuda")
        count = torch.tensor([prefix], dtype=torch.int32, device="cuda")
        ws = torch.empty(bd.civic_attn_shared_workspace_bytes(q.dtype, batch, seq, 16, 4, 128, prefix, 300), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        step = lambda: bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 300, ctx=lens, prefix_ctx=count, out=out, workspace=ws)  # noqa: E731
        sizes = [(300, prefix), (41, 1), (0, 0), (299, prefix - 1)]
        want = []
        for n, p in sizes:
            lens.fill_(n), count.fill_(p)
            want.append(step().clone())
            assert torch.equal(step(), want[-1])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        for i in (0, 1, 2, 3, 0):
            lens.fill_(sizes[i][0]), count.fill_(sizes[i][1])
            out.fill_(3.0)
            graph.replay()
            assert torch.equal(out, want[i])
        torch.cuda.synchronize()
        got = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 300, ctx=lens, prefix_ctx=count, stream=side)
        side.synchronize()
        assert torch.equal(got, want[0])


def test_caches_beyond_32_bits(bd):  # noqa: F811
    hkv, rows, d = 3, 1 << 22, 256
    kc = torch.empty((2, hkv, rows, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    for seq in (1, 40):
        q, kp, vp, kk, vv = inputs(8, "bf16", 2, seq, 6, hkv, d, 200, 100)
        kc[:, :, :100], vc[:, :, :100] = kk, vv
        want = bd.civic_prefill_attn_shared(q, kp, vp, kk, vv, 100)
        assert torch.equal(bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 100), want)
        big_k, big_v = kc[0], vc[0]                            # (as a prefix)
        big_k[:, :200], big_v[:, :200] = kp, vp
        assert torch.equal(bd.civic_prefill_attn_shared(q, big_k, big_v, kk, vv, 100, n_prefix=200), want)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("sizes", [(3, 1, 8, 2, 64, 700), (2, 70, 4, 2, 128, 700), (2, 70, 4, 2, 64, 0), (5, 9, 4, 2, 96, 2300), (9, 4, 8, 2, 128, 2300), (2, 40, 4, 2, 72, 700),
                                   (4, 150, 16, 4, 256, 1100), (24, 4, 16, 8, 256, 3500)], ids=str)
def test_large_values_behind_weights_that_grow(bd, dtype, sizes):  # noqa: F811
    """A key whose weight is 2^18 of what a row has seen before it, and values of 2^112: finite, since 2^9 times the sum over V is 2^125 at most."""
    batch, seq, hq, hkv, d, prefix = sizes
    log("attn_shared large", dtype, sizes)
    q, kp, vp, kc, vc = (torch.zeros_like(x) for x in inputs(9, dtype, batch, seq, hq, hkv, d, prefix, 700))
    q[..., 0] = 1.0
    for k, v in ((kp, vp), (kc, vc)):
        k[..., 499::512, 0] = 18.0                             # (the last tiles of runs of eight steps of 64)
        v[..., 499::512, :] = 2.0 ** 112
        v[..., 3:5, :] = -2.0 ** 112
    out = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 700, causal=False, softmax_scale=float(np.log(2.0)))
    ref, wa, la = oracle.shared_attention(host(q), host(kp), host(vp), host(kc), host(vc), [700] * batch, False, float(np.log(2.0)))
    assert (np.abs(host(out) - ref) <= tolerance(ref, wa, la, d, prefix + 700, dtype, True)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("sizes", [(3, 1, 8, 2, 64, 100), (9, 1, 8, 2, 128, 2300), (2, 70, 4, 2, 128, 100), (5, 9, 4, 2, 96, 2300), (2, 40, 4, 2, 72, 100), (4, 150, 16, 4, 256, 1100)], ids=str)
def test_logits_of_minus_infinity(bd, dtype, sizes):  # noqa: F811
    """An infinite key of the prefix and one of a sample against queries of one sign: weights of 0; a token that sees nothing else gives zeros."""
    batch, seq, hq, hkv, d, prefix = sizes
    log("attn_shared infinity", dtype, sizes)
    q, kp, vp, kc, vc = inputs(10, dtype, batch, seq, hq, hkv, d, prefix, 90)
    q[..., 2] = q[..., 2].abs() + 0.5
    clean = [host(x) for x in (kp, vp, kc, vc)]
    kp[:, [0, prefix // 2], 2] = -float("inf")
    kc[:, :, [5, 89], 2] = -float("inf")
    out = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 90, causal=False)
    p, o = np.setdiff1d(np.arange(prefix), [0, prefix // 2]), np.setdiff1d(np.arange(90), [5, 89])
    ref, wa, la = oracle.shared_attention(host(q), clean[0][:, p], clean[1][:, p], clean[2][:, :, o], clean[3][:, :, o], [88] * batch, False)
    assert (np.abs(host(out) - ref) <= tolerance(ref, wa, la, d, prefix + 90, dtype, True)).all()
    kp[1, :, 2] = -float("inf")
    kc[1, 1, :, 2] = -float("inf")
    out = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 90, causal=False)
    assert not out[1, :, hq // hkv:2 * (hq // hkv)].any() and torch.isfinite(out.float()).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("sizes", [(3, 1, 8, 2, 64, 100), (9, 1, 8, 2, 128, 2300), (2, 70, 4, 2, 128, 100), (1, 40, 4, 2, 128, 9000), (5, 9, 4, 2, 96, 2300), (2, 40, 4, 2, 72, 3000),
                                   (4, 150, 16, 4, 256, 1100), (1, 3, 4, 2, 64, 9000)], ids=str)
def test_outputs_over_the_queries(bd, dtype, sizes):  # noqa: F811
    """out may be q, also as a part of wider rows whose next part holds the outputs of another call."""
    batch, seq, hq, hkv, d, prefix = sizes
    q, kp, vp, kc, vc = inputs(11, dtype, batch, seq, hq, hkv, d, prefix, 150)
    want = bd.civic_prefill_attn_shared(q, kp, vp, kc, vc, 150)
    wide = torch.cat((q, torch.full_like(q, 7.0)), dim=2)
    part, rest = wide[:, :, :hq], wide[:, :, hq:]
    assert torch.equal(bd.civic_prefill_attn_shared(part, kp, vp, kc, vc, 150, out=rest), want) and torch.equal(rest, want) and torch.equal(part, q)
    assert torch.equal(bd.civic_prefill_attn_shared(part, kp, vp, kc, vc, 150, out=part), want) and torch.equal(part, want) and torch.equal(rest, want)
