"""The KV cache in 8 or 4 bits on the GPU, through the C ABI, against the oracle: writes and reads to the byte, attention within a
bound on its roundings (tolerance below), and the run of them together as a serving program makes it."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_28115_amd import workloads as wl
from test_gpu_parity import log, to_dev, to_host, widen

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def bd():
    from paper_2605_28115_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return binding


def tolerance(ref, weight_abs, logit_abs, d, n, dtype, rows=1):
    """Per row, with w the weights, A = sum w max|v| and Z = max |scale| sum |q k|, u = 2^-24:
    a logit is off by (d + 4) u Z (d products, the scale, the maximum taken off), a weight by twice that (itself and the sum it is
    divided by) plus 4 u for the exponential and its argument's rounding; sums of n weights by n u, products with V by n u.
    bf16, up to 32 query rows a KV head: a weight is held as two bf16 terms, each rounding at most 2^-8 relative: 2^-16; the output by
    half a step, 2^-8 of it.
    bf16, more rows: a weight is rounded to bf16 once, p (1 + e) with |e| <= 2^-8, in the products and in their sum alike: the output
    sum p (1 + e) v / sum p (1 + e) is off by sum w e (v - out), at most 2^-8 (A + |out|) / (1 - 2^-8), before its own rounding.
    fp32 rows: three terms leave 2^-24 of a query's channel (d u Z covers it) and of a weight; the output u."""
    u = 2.0 ** -24
    off = weight_abs * (2 * (d + 4) * u * logit_abs * (1 if dtype == "bf16" else 2) + 8 * u + 2 * (n + 64) * u + (2.0 ** -16 if dtype == "bf16" else u))
    own = np.abs(ref) * (2.0 ** -8 if dtype == "bf16" else u)
    if dtype == "bf16" and rows > 32:
        own = own + 2.0 ** -8 * (weight_abs[..., None] + np.abs(ref)) / (1 - 2.0 ** -8)
    return off[..., None] + own


def cache_of(bd, k, v, bits):
    """Host rows [batch, H_kv, s_max, d] as a cache on the device (the oracle's bytes), and the values it holds."""
    (kc, ks), (vc, vs) = oracle.mx_encode(k, bits), oracle.mx_encode(v, bits)
    dev = [torch.from_numpy(x).cuda() for x in (kc, ks, vc, vs)]
    return bd.MxCache(*dev, bits), oracle.mx_decode(kc, ks, bits), oracle.mx_decode(vc, vs, bits)


def spoil(cache, ctx):
    """NaN in every row at or behind a sample's context: codes of any bits, scales 255."""
    for b, n in enumerate(ctx):
        for codes, scales in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
            codes[b, :, n:] = 0x7F
            scales[b, :, n:] = 255


def rows_with_oddities(rng, shape, dtype):
    x = (rng.standard_normal(shape) * np.exp(rng.uniform(-3, 3, shape[:-1] + (1,)))).astype(np.float32)
    flat = x.reshape(-1, shape[-1])
    special = [0.0, 3.38e38, 1e-38, 2.0 ** -100, 2.0 ** -104, np.inf, np.nan, -np.inf, -0.0, 1e-40, 7.0, 464.0]
    for i, s in enumerate(special[:len(flat)]):
        flat[i, (5 * i) % shape[-1]] = s
    if len(flat) > 14:
        flat[12] = 0.0
        flat[13] = 3.38e38
        flat[14] = np.arange(shape[-1]) * 0.25 - 4               # ties
    return _quantize_odd(x, dtype)


def _quantize_odd(x, dtype):
    if dtype == "fp32":
        return x
    bits = wl.f32_to_bf16_bits(np.where(np.isfinite(x), x, 0).astype(np.float32))
    bits[np.isnan(x)] = 0x7FC0
    bits[np.isposinf(x)] = 0x7F80
    bits[np.isneginf(x)] = 0xFF80
    return bits


# ------------------------------------------------------------------------------------------------- write and read
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 32), (2, 3, 2, 64), (3, 37, 8, 128), (1, 300, 3, 96), (2, 17, 5, 256), (1, 130, 1, 160), (5, 65, 4, 224)], ids=str)
def test_write_gives_the_oracles_bytes_and_read_its_values(bd, bits, dtype, shape):
    b, seq, h, d = shape
    rng = np.random.default_rng(b * seq + d)
    k, v = (rows_with_oddities(rng, shape, dtype) for _ in range(2))
    first = 3
    pos = rng.integers(0, 20, b).astype(np.int32)
    cache = bd.civic_mx_cache(b, h, first + 20 + seq, d, bits)
    for t in cache[:4]:
        t.fill_(0xA5)
    want = [t.cpu().numpy().copy() for t in cache[:4]]
    for i, x in enumerate((k, v)):
        codes, scales = oracle.mx_encode(widen(x), bits)
        for s in range(b):
            at = slice(first + pos[s], first + pos[s] + seq)
            want[2 * i][s, :, at] = codes[s].transpose(1, 0, 2)
            want[2 * i + 1][s, :, at] = scales[s].transpose(1, 0, 2)
    # K and V of a token side by side, as a projection leaves them
    both = torch.stack((to_dev(k), to_dev(v)), dim=2)
    d_pos = torch.from_numpy(pos).cuda()
    bd.civic_kv_write_mx(both[:, :, 0], both[:, :, 1], cache, first, pos=d_pos)
    for name, t, w in zip(cache._fields, cache[:4], want):
        assert np.array_equal(t.cpu().numpy(), w), name
    back = torch.full((b, seq + 2, 2, h, d), 7.0, dtype=TYPES[dtype], device="cuda")
    bd.civic_kv_read_mx(cache, back[:, :seq, 0], back[:, :seq, 1], first, pos=d_pos)
    for i, x in enumerate((k, v)):
        ref = oracle.mx_decode(*oracle.mx_encode(widen(x), bits), bits)
        assert np.array_equal(widen(to_host(back[:, :seq, i])), ref, equal_nan=True)
    assert (back[:, seq:] == 7.0).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_read_of_every_code_and_scale(bd, bits):
    rng = np.random.default_rng(bits)
    s_max = 512
    scales = np.repeat(np.arange(256, dtype=np.uint8), 2)[None, None, :, None]
    codes = rng.integers(0, 256, (1, 1, s_max, 32 * bits // 8)).astype(np.uint8)
    codes[0, 0, :, 0] = np.arange(s_max) & 255
    dev = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (codes, scales, codes, scales)]
    ref = oracle.mx_decode(codes, scales, bits).transpose(0, 2, 1, 3)
    for dtype in ("fp32", "bf16"):
        k, v = (torch.empty((1, s_max, 1, 32), dtype=TYPES[dtype], device="cuda") for _ in range(2))
        bd.civic_kv_read_mx(bd.MxCache(*dev, bits), k, v)
        got = widen(to_host(k))
        # inside the range of normal numbers every value is exact; below it may become 0, beyond it is infinite
        fine = np.isnan(ref) | ((np.abs(ref) >= 2.0 ** -126) & (np.abs(ref) < 2.0 ** 127)) | (ref == 0)
        assert fine.mean() > 0.9 and np.array_equal(got[fine], ref[fine], equal_nan=True)
        assert (np.abs(got[np.abs(ref) < 2.0 ** -126]) <= 2.0 ** -126).all()
        assert torch.equal(k.view(torch.uint8), v.view(torch.uint8))


@pytest.mark.parametrize("bits", [4, 8])
def test_rows_outside_the_cache_are_left_out(bd, bits):
    b, seq, h, d, s_max = 4, 9, 2, 64, 32
    rng = np.random.default_rng(1)
    k = rng.standard_normal((b, seq, h, d)).astype(np.float32)
    pos = torch.tensor([-4, 28, 32, -2 ** 31], dtype=torch.int32, device="cuda")
    cache = bd.civic_mx_cache(b, h, s_max, d, bits)
    bd.civic_kv_write_mx(to_dev(k), to_dev(k), cache, 0, pos=pos)
    codes, scales = oracle.mx_encode(k, bits)
    want = np.zeros((b, h, s_max, d // 32), np.uint8)
    want[0, :, 0:5] = scales[0, 4:].transpose(1, 0, 2)
    want[1, :, 28:32] = scales[1, :4].transpose(1, 0, 2)
    assert np.array_equal(cache.k_scales.cpu().numpy(), want) and np.array_equal(cache.v_scales.cpu().numpy(), want)
    out = torch.full((2, b, seq, h, d), 5.0, device="cuda")
    bd.civic_kv_read_mx(cache, out[0], out[1], 0, pos=pos)
    ref = oracle.mx_decode(codes, scales, bits)
    inside = np.zeros((b, seq), bool)
    inside[0, 4:], inside[1, :4] = True, True
    for x in out.cpu().numpy():
        assert np.array_equal(x[inside], ref[inside]) and (x[~inside] == 5.0).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 256])
def test_rotated_write_is_rotation_then_write(bd, bits, dtype, d):
    b, seq, h = 2, 45, 3
    gen = torch.Generator(device="cuda").manual_seed(d)
    k, v = (torch.randn((b, seq, h, d), device="cuda", generator=gen).to(TYPES[dtype]) for _ in range(2))
    ids = torch.randint(0, 5000, (3, b, seq), dtype=torch.int32, device="cuda", generator=gen)
    table = bd.civic_mrope_table(ids, np.arange(d // 2) % 3, 1e4 ** (-np.arange(d // 2) / (d // 2)))
    one, two = (bd.civic_mx_cache(b, h, 64, d, bits) for _ in range(2))
    bd.civic_kv_write_mx(k, v, one, 7, cos_sin=table)
    bd.civic_kv_write_mx(bd.civic_mrope_apply(k, table), v, two, 7)
    for x, y in zip(one[:4], two[:4]):
        assert torch.equal(x, y)
    assert one.k_codes.any()


@pytest.mark.parametrize("lens", [[1], [5, 0, 17, 64, 3], [7] * 130], ids=["one", "some", "groups"])
@pytest.mark.parametrize("bits,dtype,rope", [(4, "bf16", True), (8, "fp32", True), (4, "fp32", False), (8, "bf16", False)])
def test_ragged_write_is_the_write_of_each_sample(bd, lens, bits, dtype, rope):
    h, d = 2, 64
    gen = torch.Generator(device="cuda").manual_seed(len(lens))
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    k, v = (torch.randn((int(off[-1]), h, d), device="cuda", generator=gen).to(TYPES[dtype]) for _ in range(2))
    angle = torch.rand((int(off[-1]), d // 2), device="cuda", generator=gen) * 6
    table = torch.stack((angle.cos(), angle.sin()), dim=-1) if rope else None
    pos = torch.tensor([(3 * i) % 11 for i in range(len(lens))], dtype=torch.int32, device="cuda")
    one, two = (bd.civic_mx_cache(len(lens), h, 96, d, bits) for _ in range(2))
    bd.civic_kv_write_mx_ragged(k, v, one, off, 2, pos=pos, cos_sin=table)
    for b, n in enumerate(lens):
        at = slice(int(off[b]), int(off[b + 1]))
        single = bd.MxCache(*[t[b:b + 1] for t in two[:4]], bits)
        bd.civic_kv_write_mx(k[None, at], v[None, at], single, 2, pos=pos[b:b + 1], cos_sin=None if table is None else table[None, at].contiguous())
    for x, y in zip(one[:4], two[:4]):
        assert torch.equal(x, y)


# ------------------------------------------------------------------------------------------------------ attention
def check(bd, q, cache, kv, ctx, causal=False, scale=0.0, n_ctx=None, decode=False, dtype="bf16", by_number=False):
    """One call against the oracle; q [batch, seq, H_q, d] host storage."""
    n_ctx = max(ctx) if n_ctx is None else n_ctx
    d_ctx = None if by_number else torch.tensor(ctx, dtype=torch.int32, device="cuda")
    b, seq, hq, d = q.shape
    need = bd.civic_attn_mx_workspace_bytes(TYPES[dtype], cache.format, b, seq, hq, kv[0].shape[1], d, n_ctx)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")              # NaN: it needs no values
    if decode:
        out = bd.civic_decode_attn_mx(to_dev(q)[:, 0], cache, n_ctx, ctx=d_ctx, softmax_scale=scale, workspace=ws)[:, None]
    else:
        out = bd.civic_prefill_attn_mx(to_dev(q), cache, n_ctx, ctx=d_ctx, causal=causal, softmax_scale=scale, workspace=ws)
    got = widen(to_host(out)).astype(np.float64)
    ref, wa, la = oracle.cache_attention(widen(q), *kv, ctx, causal, None if scale == 0.0 else scale)
    tol = tolerance(ref, wa, la, d, max(ctx), dtype, seq * hq // kv[0].shape[1])
    worst = float((np.abs(got - ref) / np.maximum(tol, 1e-300)).max()) if got.size else 0.0
    log("   worst error / tolerance", worst, "abs", float(np.abs(got - ref).max()))
    assert np.isfinite(got).all() and worst <= 1.0
    return out


def inputs(bd, seed, b, seq, hq, hkv, d, s_max, bits, dtype, loud=1.0):
    rng = np.random.default_rng(seed)
    q = wl.quantize((rng.standard_normal((b, seq, hq, d)) * loud).astype(np.float32), dtype)[0]
    k, v = (rng.standard_normal((b, hkv, s_max, d)).astype(np.float32) for _ in range(2))
    k[..., : d // 8] *= 4.0
    cache, kf, vf = cache_of(bd, k, v, bits)
    return q, cache, (kf, vf)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [
    # batch, H_q, H_kv, d, s_max, contexts
    (1, 4, 4, 128, 32, [1]), (2, 8, 2, 128, 64, [33, 0]), (1, 32, 8, 128, 960, [938]), (3, 6, 2, 64, 320, [257, 31, 32]), (2, 12, 4, 96, 160, [129, 128]),
    (1, 8, 1, 128, 4128, [4097]), (1, 2, 2, 256, 704, [513]), (2, 3, 1, 32, 64, [64, 63]), (1, 64, 2, 128, 608, [511]), (9, 8, 8, 64, 224, [0, 1, 2, 31, 65, 127, 129, 200, 224]),
    (2, 5, 1, 160, 288, [1, 270]), (1, 16, 16, 224, 96, [95]), (1, 20, 1, 128, 2016, [2000]),
], ids=str)
def test_decode_matches_the_oracle(bd, bits, dtype, shape):
    b, hq, hkv, d, s_max, ctx = shape
    log("decode", bits, dtype, shape)
    q, cache, kv = inputs(bd, d + s_max, b, 1, hq, hkv, d, s_max, bits, dtype)
    spoil(cache, ctx)
    check(bd, q, cache, kv, ctx, decode=True, dtype=dtype)
    check(bd, q, cache, kv, ctx, decode=True, dtype=dtype, n_ctx=s_max, scale=0.2)          # a bound that no sample reaches
    check(bd, q, cache, kv, [min(ctx)] * b, decode=True, dtype=dtype, by_number=True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", [
    # batch, tokens, H_q, H_kv, d, s_max, contexts
    (1, 2, 4, 2, 64, 64, [40]), (2, 5, 16, 8, 128, 1056, [1000, 37]), (3, 7, 8, 2, 96, 160, [3, 0, 150]), (1, 128, 8, 2, 128, 640, [600]),
    (2, 33, 28, 4, 128, 320, [33, 300]), (1, 300, 4, 1, 64, 320, [300]), (16, 40, 8, 8, 128, 96, [5 * i for i in range(16)]), (1, 19, 2, 2, 256, 96, [80]),
    (4, 70, 16, 2, 32, 96, [96, 70, 69, 1]), (40, 90, 4, 2, 64, 192, [4 * i + 30 for i in range(40)]),
], ids=str)
def test_prefill_matches_the_oracle(bd, bits, dtype, causal, shape):
    b, seq, hq, hkv, d, s_max, ctx = shape
    log("prefill", bits, dtype, causal, shape)
    q, cache, kv = inputs(bd, d + seq, b, seq, hq, hkv, d, s_max, bits, dtype)
    spoil(cache, ctx)
    check(bd, q, cache, kv, ctx, causal=causal, dtype=dtype)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("shape", [
    # batch, tokens, H_q, H_kv, d, s_max, contexts: many samples and heads of 256 rows; long chunks over long contexts, in splits and whole
    (32, 256, 8, 8, 64, 320, [280 + i for i in range(32)]), (20, 130, 16, 8, 128, 192, [130 + 3 * i for i in range(20)]),
    (1, 1024, 28, 4, 128, 4544, [4501]), (8, 512, 16, 4, 96, 1024, [520 + 60 * i for i in range(8)]), (2, 300, 16, 4, 256, 1504, [1500, 301]),
    (1, 2000, 4, 1, 64, 2016, [2000]), (1, 3, 64, 1, 128, 20000, [19999]),
], ids=lambda s: str(s[:6]))
def test_long_chunks_match_the_oracle_at_their_ends_and_middle(bd, bits, shape):
    """Whole chunks on the GPU; the oracle takes tokens of it with the context that they end: token i of a chunk that ends at row n is the
    last token of a context of n - (seq - 1 - i) rows."""
    b, seq, hq, hkv, d, s_max, ctx = shape
    log("long chunk", bits, shape[:6])
    q, cache, kv = inputs(bd, seq + d, b, seq, hq, hkv, d, s_max, bits, "bf16")
    spoil(cache, ctx)
    out = widen(to_host(bd.civic_prefill_attn_mx(to_dev(q), cache, max(ctx), ctx=torch.tensor(ctx, dtype=torch.int32, device="cuda"))))
    assert np.isfinite(out).all()
    for at in sorted({0, 1, seq // 2 - 1, seq // 2, seq - 1}):
        few = np.linspace(0, b - 1, min(b, 5)).astype(int)
        part = [max(ctx[i] - (seq - 1 - at), 0) for i in few]
        ref, wa, la = oracle.cache_attention(widen(q[few, at:at + 1]), kv[0][few], kv[1][few], part, False)
        tol = tolerance(ref, wa, la, d, max(part), "bf16", seq * hq // hkv)
        assert (np.abs(out[few, at:at + 1] - ref) <= tol).all(), at


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_contexts_around_the_tiles(bd, bits, causal, d):
    """Chunks of 40 tokens whose contexts end at, before and behind multiples of 64 and 128 rows, under one bound for all of them."""
    ctx = [0, 1, 39, 40, 41, 63, 64, 65, 103, 104, 127, 128, 129, 167, 191, 192, 193, 255, 256, 257, 319, 321, 383, 384]
    q, cache, kv = inputs(bd, 5, len(ctx), 40, 8, 4, d, 384, bits, "bf16")
    spoil(cache, ctx)
    log("tiles", bits, causal, d)
    check(bd, q, cache, kv, ctx, causal=causal)
    check(bd, q, cache, kv, ctx, causal=causal, scale=-0.3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_random_shapes(bd, dtype):
    rng = np.random.default_rng(99)
    for it in range(60):
        bits, d, hkv = int(rng.choice([4, 8])), int(rng.choice([32, 64, 96, 128, 128, 160, 192, 256])), int(rng.choice([1, 2, 3, 8]))
        hq, b = hkv * int(rng.choice([1, 2, 3, 4, 7, 16])), int(rng.choice([1, 2, 5]))
        seq = int(rng.choice([1, 1, 2, 3, 8, 17, 33, 60]))
        top = int(rng.choice([1, 31, 32, 33, 64, 65, 128, 300, 700, 1300]))
        ctx = [int(x) for x in rng.integers(0, top + 1, b)]
        ctx[0] = top
        s_max = -(-top // 32) * 32
        causal, scale = bool(rng.integers(0, 2)), float(rng.choice([0.0, 0.0, -0.15, 0.4]))
        log("random", it, bits, dtype, (b, seq, hq, hkv, d, s_max, ctx), causal, scale)
        q, cache, kv = inputs(bd, it, b, seq, hq, hkv, d, s_max, bits, dtype)
        spoil(cache, ctx)
        check(bd, q, cache, kv, ctx, causal=causal, dtype=dtype, scale=scale)


def test_scales_of_any_size(bd):
    """A scale so small that all weights are one: the mean of V; one so large that one key has all of it."""
    q, cache, (kf, vf) = inputs(bd, 21, 1, 2, 4, 2, 64, 64, 8, "fp32")
    mean = bd.civic_prefill_attn_mx(to_dev(q), cache, 50, causal=False, softmax_scale=1e-42)
    want = torch.from_numpy(vf[:, :, :50].mean(axis=2)).cuda().repeat_interleave(2, dim=1)
    assert (mean - want[:, None]).abs().max() <= 1e-5
    for scale in (1e30, -1e30, 3e38):
        one = bd.civic_prefill_attn_mx(to_dev(q), cache, 50, causal=False, softmax_scale=scale)
        z = np.einsum("bthd,bhnd->bthn", q.astype(np.float64), np.repeat(kf[:, :, :50], 2, axis=1).astype(np.float64)) * np.sign(scale)
        pick = z.argmax(axis=3)
        want = np.stack([[[vf[0, h // 2, pick[0, t, h]] for h in range(4)] for t in range(2)]])
        good = torch.isfinite(one).all(dim=3)                                                # (a logit beyond fp32 is infinite: NaN)
        assert good.any() or scale == 3e38
        assert (one.cpu().numpy() == want)[good.cpu().numpy()].all()


def test_attention_of_strided_queries_and_outputs(bd):
    b, seq, hq, hkv, d, s_max = 2, 21, 8, 2, 128, 160
    q, cache, kv = inputs(bd, 2, b, seq, hq, hkv, d, s_max, 4, "bf16")
    ctx = torch.tensor([150, 90], dtype=torch.int32, device="cuda")
    plain = bd.civic_prefill_attn_mx(to_dev(q), cache, 160, ctx=ctx)
    wide = torch.full((b, seq, 3, hq, d), 9.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :, 1] = to_dev(q)
    heads_first = torch.full((b, hq, seq + 1, d), 9.0, dtype=torch.bfloat16, device="cuda")
    bd.civic_prefill_attn_mx(wide[:, :, 1], cache, 160, ctx=ctx, out=heads_first[:, :, :seq].transpose(1, 2))
    assert torch.equal(heads_first[:, :, :seq].transpose(1, 2), plain) and (heads_first[:, :, seq:] == 9.0).all()
    # one token through the strided call is the decode call
    a = bd.civic_prefill_attn_mx(wide[:, -1:, 1], cache, 160, ctx=ctx)
    assert torch.equal(a[:, 0], bd.civic_decode_attn_mx(to_dev(q)[:, -1].contiguous(), cache, 160, ctx=ctx))


def test_contexts_out_of_range_are_taken_at_their_ends(bd):
    q, cache, kv = inputs(bd, 3, 4, 1, 8, 2, 64, 128, 8, "bf16")
    far = torch.tensor([-5, 1000, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    near = torch.tensor([0, 100, 100, 0], dtype=torch.int32, device="cuda")
    x, y = (bd.civic_decode_attn_mx(to_dev(q)[:, 0], cache, 100, ctx=c) for c in (far, near))
    assert torch.equal(x, y) and (x[0] == 0).all() and (x[3] == 0).all() and x[1].any()
    empty = bd.civic_decode_attn_mx(to_dev(q)[:, 0], cache, 0)
    assert (empty == 0).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_key_per_query_and_large_logits(bd, bits, dtype):
    """Every head attends to one row (out = that V row at full size); logits that grow or fall along the context, far apart between
    wavefronts and splits."""
    rng = np.random.default_rng(31)
    b, hq, hkv, d, n = 2, 8, 2, 128, 1500
    k, v = (rng.standard_normal((b, hkv, 1504, d)).astype(np.float32) for _ in range(2))
    cache, kf, vf = cache_of(bd, k, v, bits)
    pick = rng.integers(0, n, (b, hq))
    q = np.stack([np.stack([4.0 * kf[i, h // 4, pick[i, h]] for h in range(hq)]) for i in range(b)])[:, None]
    q = wl.quantize(q.astype(np.float32), dtype)[0]
    out = widen(to_host(check(bd, q, cache, (kf, vf), [n] * b, decode=True, dtype=dtype)))
    for i in range(b):
        for h in range(hq):
            assert np.abs(out[i, 0, h] - vf[i, h // 4, pick[i, h]]).max() < 0.05 * np.abs(vf).max()
    for sign in (1.0, -1.0):
        k2 = rng.standard_normal(k.shape).astype(np.float32) * 0.5
        k2[..., :32] = 0.0
        k2[..., 0] = sign * np.arange(1504, dtype=np.float32)[None, None]
        q2 = np.zeros((b, 3, hq, d), np.float32)
        q2[..., 0] = 8.0
        cache2, kf2, vf2 = cache_of(bd, k2, v, bits)
        check(bd, wl.quantize(q2, dtype)[0], cache2, (kf2, vf2), [n, 700], causal=True, dtype=dtype)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("shape", [(1, 9, 8, 2, 128, 512, 500), (16, 80, 8, 4, 64, 128, 120), (1, 3, 4, 1, 256, 96, 90), (2, 6, 4, 2, 96, 64, 60),
                                   (2, 40, 16, 8, 128, 384, 380), (1, 300, 28, 4, 128, 1056, 1050)], ids=str)
def test_a_nan_of_the_cache_reaches_the_tokens_that_see_it(bd, bits, shape):
    b, seq, hq, hkv, d, s_max, n = shape
    q, cache, (kf, vf) = inputs(bd, 8, b, seq, hq, hkv, d, s_max, bits, "bf16")
    ctx = torch.full((b,), n, dtype=torch.int32, device="cuda")
    clean = bd.civic_prefill_attn_mx(to_dev(q), cache, n, ctx=ctx)
    at = n - seq + 2                                           # seen from the chunk's token 2 on
    head, block = hkv - 1, d // 32 - 1
    group = hq // hkv
    mine = torch.arange(hq, device="cuda") // group == head
    # a block of V: these channels of the tokens that see it
    cache.v_scales[0, head, at, block] = 255
    out = bd.civic_prefill_attn_mx(to_dev(q), cache, n, ctx=ctx)
    hit = torch.zeros_like(clean, dtype=torch.bool)
    hit[0, 2:, mine, 32 * block:32 * block + 32] = True
    assert torch.equal(out.isnan(), hit)
    # what it does not reach is what a row without that block's values gives
    assert torch.equal(out[:1, :2], clean[:1, :2]) and torch.equal(out[:, :, ~mine], clean[:, :, ~mine]) and torch.equal(out[1:], clean[1:])
    assert (out[~hit].float() - clean[~hit].float()).abs().max() <= 2.0 ** -6 * max(1.0, float(clean.float().abs().max()))
    # a block of K: every channel of the tokens that see it
    cache.v_scales[0, head, at, block] = 127
    cache.k_scales[0, head, at, 0] = 255
    out = bd.civic_prefill_attn_mx(to_dev(q), cache, n, ctx=ctx)
    hit[0, 2:, mine] = True
    assert torch.equal(out.isnan(), hit) and torch.equal(out[:1, :2], clean[:1, :2])
    # a row of NaN as the write makes it of an infinity, past the chunk's own rows
    cache.k_scales[0, head, at, 0] = 127
    bad = torch.full((b, 1, hkv, d), float("inf"), dtype=torch.bfloat16, device="cuda")
    bd.civic_kv_write_mx(bad, bad, cache, n)
    assert not bd.civic_prefill_attn_mx(to_dev(q), cache, n, ctx=ctx).isnan().any()
    assert bd.civic_prefill_attn_mx(to_dev(q), cache, n + 1)[:, -1].isnan().all()


def test_queries_of_nan_or_infinity_stay_in_their_rows(bd):
    q, cache, kv = inputs(bd, 9, 2, 6, 8, 2, 64, 96, 4, "bf16")
    clean = bd.civic_prefill_attn_mx(to_dev(q), cache, 90)
    dq = to_dev(q)
    dq[0, 3, 2, 5], dq[1, 0, 7, 0] = float("nan"), float("inf")
    out = bd.civic_prefill_attn_mx(dq, cache, 90)
    rows = torch.ones((2, 6, 8), dtype=torch.bool, device="cuda")
    rows[0, 3, 2], rows[1, 0, 7] = False, False
    assert torch.equal(out[rows], clean[rows]) and out[0, 3, 2].isnan().all()


def test_offsets_past_32_bits(bd):
    """A cache of 4.3 GB a tensor: the last rows of the last head, written, read and attended."""
    b, h, d, s_max = 2, 8, 256, 1 << 20
    cache = bd.civic_mx_cache(b, h, s_max, d, 8)
    gen = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn((b, 50, h, d), device="cuda", generator=gen) for _ in range(2))
    at = s_max - 50
    bd.civic_kv_write_mx(k, v, cache, at)
    back = bd.civic_kv_read_mx(cache, torch.empty_like(k), torch.empty_like(v), at)
    for x, y in zip(back, (k, v)):
        assert np.array_equal(x.cpu().numpy(), oracle.mx_decode(*oracle.mx_encode(y.cpu().numpy(), 8), 8))
    # a key that outweighs the zeros in front of it
    q = (k[:, 49] * 2.0).contiguous()
    out = bd.civic_decode_attn_mx(q, cache, s_max)
    z = (q[:, :, None].double() * back[0].double().transpose(1, 2)).sum(-1) / 16.0
    p = torch.exp(z)
    ref = (p[..., None] * back[1].double().transpose(1, 2)).sum(2) / (p.sum(-1) + (s_max - 50))[..., None]
    assert (out.double() - ref).abs().max() <= 1e-4 * ref.abs().max()


# ----------------------------------------------------------------------------------------------- the run of them
@pytest.mark.parametrize("bits", [4, 8])
def test_a_conversation_of_a_ragged_batch(bd, bits):
    """Packed prompts attended and written rotated, a follow-up question, then tokens one by one: every attention against the
    oracle on the values that the cache holds."""
    lens, hq, hkv, d, dtype = [27, 120, 64], 8, 2, 64, "bf16"
    b, t, steps = len(lens), 10, 4
    gen = torch.Generator(device="cuda").manual_seed(bits)
    new = lambda *s: torch.randn(s, device="cuda", generator=gen).bfloat16()  # noqa: E731
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    cache = bd.civic_mx_cache(b, hkv, 160, d, bits)
    angle = torch.rand((int(off[-1]), d // 2), device="cuda", generator=gen) * 6
    table = torch.stack((angle.cos(), angle.sin()), dim=-1)
    k, v = new(int(off[-1]), hkv, d), new(int(off[-1]), hkv, d)
    bd.civic_kv_write_mx_ragged(k, v, cache, off, cos_sin=table)
    ctx = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def held():
        kf, vf = (torch.empty((b, 160, hkv, d), device="cuda") for _ in range(2))
        return [np.ascontiguousarray(x.cpu().numpy().transpose(0, 2, 1, 3)) for x in bd.civic_kv_read_mx(cache, kf, vf)]

    rotated = bd.civic_mrope_apply(k[None], table[None].contiguous())[0].float().cpu().numpy()
    kf, _ = held()
    for i, n in enumerate(lens):
        want = oracle.mx_decode(*oracle.mx_encode(rotated[off[i]:off[i + 1]], bits), bits)
        assert np.array_equal(kf[i, :, :n], want.transpose(1, 0, 2))
    for seq in (t, *[1] * steps):
        q, k, v = new(b, seq, hq, d), new(b, seq, hkv, d), new(b, seq, hkv, d)
        bd.civic_kv_write_mx(k, v, cache, pos=ctx)
        ctx = ctx + seq
        if seq > 1:
            out = bd.civic_prefill_attn_mx(q, cache, 160, ctx=ctx)
        else:
            out = bd.civic_decode_attn_mx(q[:, 0], cache, 160, ctx=ctx)[:, None]
        ref, wa, la = oracle.cache_attention(q.float().cpu().numpy(), *held(), ctx.cpu().numpy(), True)
        assert (np.abs(out.float().cpu().numpy() - ref) <= tolerance(ref, wa, la, d, 160, dtype, seq * hq // hkv)).all()
    assert ctx.tolist() == [n + t + steps for n in lens]


def test_decode_over_the_values_is_the_decode_of_a_wide_cache(bd):
    """The same values in bf16, through civic_decode_attn: both within their roundings of one another."""
    q, cache, (kf, vf) = inputs(bd, 12, 4, 1, 32, 8, 128, 960, 4, "bf16")
    kc, vc = (torch.from_numpy(x).cuda().bfloat16() for x in (kf, vf))
    a = bd.civic_decode_attn_mx(to_dev(q)[:, 0], cache, 938).float()
    c = bd.civic_decode_attn(to_dev(q)[:, 0].contiguous(), kc, vc, 938).float()
    assert (a - c).abs().max() <= 2.0 ** -7 * float(c.abs().max())


def test_a_captured_step_follows_positions_and_contexts(bd):
    """Write, decode and the advance of the positions as one graph: every replay against the eager calls."""
    b, hq, hkv, d, s_max = 3, 8, 2, 128, 2080
    gen = torch.Generator(device="cuda").manual_seed(6)
    start = torch.tensor([0, 700, 2000], dtype=torch.int32, device="cuda")
    one, two = (bd.civic_mx_cache(b, hkv, s_max, d, 4) for _ in range(2))
    fill = torch.randn((b, 2000, hkv, d), device="cuda", generator=gen).bfloat16()
    for c in (one, two):
        bd.civic_kv_write_mx(fill, fill, c)
    q, k, v = (torch.empty((b, 1, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    pos, out = start.clone(), torch.empty((b, hq, d), dtype=torch.bfloat16, device="cuda")
    need = bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 4, b, 1, hq, hkv, d, s_max)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def step():
        bd.civic_kv_write_mx(k, v, one, pos=pos)
        pos.add_(1)
        bd.civic_decode_attn_mx(q[:, 0], one, s_max, ctx=pos, out=out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    pos.copy_(start)
    for i in range(5):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda", generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        at = start + i
        bd.civic_kv_write_mx(k, v, two, pos=at)
        ref = bd.civic_decode_attn_mx(q[:, 0], two, s_max, ctx=at + 1)
        assert torch.equal(pos, at + 1) and torch.equal(out, ref), i
        rows = [(one.k_codes[j, :, :int(at[j]) + 1], two.k_codes[j, :, :int(at[j]) + 1]) for j in range(b)]
        assert all(torch.equal(x, y) for x, y in rows)


def test_calls_on_two_streams_with_workspaces_of_their_own(bd):
    q, cache, kv = inputs(bd, 14, 2, 1, 16, 4, 128, 3008, 4, "bf16")
    dq = to_dev(q)[:, 0].contiguous()
    ref = [bd.civic_decode_attn_mx(dq, cache, n) for n in (3000, 1777)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    for i, (s, n) in enumerate(zip(streams, (3000, 1777))):
        with torch.cuda.stream(s):
            outs[i] = [bd.civic_decode_attn_mx(dq, cache, n) for _ in range(10)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, r) for o, r in zip(outs, ref) for x in o)
    other = bd.civic_decode_attn_mx(dq, cache, 3000, stream=streams[0])
    streams[0].synchronize()
    assert torch.equal(other, ref[0])
