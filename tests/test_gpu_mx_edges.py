"""The cache in 8 or 4 bits where its calls meet odd values, other streams, growing contexts and the rest of the path."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_mx import TYPES, bd, cache_of, inputs, spoil, tolerance  # noqa: F401  (bd: the fixture)
from test_gpu_parity import log, to_dev, to_host, widen

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------- NaN blocks and their cost
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", [
    # batch, tokens, H_q, H_kv, d, s_max, contexts: a token over splits; 32 rows; chunks of more, whole and in splits, of every width
    (2, 1, 8, 2, 128, 2016, [2000, 731]), (1, 1, 4, 2, 64, 160, [131]), (2, 6, 8, 2, 128, 1024, [1000, 77]), (1, 7, 4, 1, 96, 320, [301]),
    (1, 300, 14, 2, 128, 1056, [1050]), (9, 140, 8, 4, 128, 320, [140 + 20 * i for i in range(9)]), (3, 90, 4, 2, 64, 640, [600, 90, 400]),
    (2, 60, 4, 2, 96, 512, [500, 61]), (1, 50, 4, 2, 160, 352, [340]), (2, 40, 2, 1, 256, 288, [280, 41]),
], ids=str)
def test_nan_blocks_reach_exactly_the_tokens_that_see_them(bd, bits, dtype, causal, shape):
    b, seq, hq, hkv, d, s_max, ctx = shape
    log("nan blocks", bits, dtype, causal, shape)
    q, cache, (kf, vf) = inputs(bd, 40 + d, b, seq, hq, hkv, d, s_max, bits, dtype)
    rng = np.random.default_rng(s_max + bits)
    for n, back in zip((0, 3, 30, 64, 100), (0, 1, 2, 3, 4)):
        i = int(rng.integers(b))
        # among the rows that only some of the chunk's tokens see, and in front of them
        key = max(ctx[i] - 1 - (n if n < seq else int(rng.integers(ctx[i]))), 0)
        head, block = int(rng.integers(hkv)), (int(rng.integers(d // 32)) + back) % (d // 32)
        cache.v_scales[i, head, key, block] = 255
        vf[i, head, key, 32 * block:32 * block + 32] = np.nan
    spoil(cache, ctx)
    out = bd.civic_prefill_attn_mx(to_dev(q), cache, max(ctx), ctx=torch.tensor(ctx, dtype=torch.int32, device="cuda"), causal=causal)
    got = widen(to_host(out)).astype(np.float64)
    ref, wa, la = oracle.cache_attention(widen(q), kf, vf, ctx, causal)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.isnan(ref).any()
    fine = ~np.isnan(ref)
    tol = tolerance(np.where(fine, ref, 0.0), wa, la, d, max(ctx), dtype, seq * hq // hkv)
    assert (np.abs(got - ref)[fine] <= tol[fine]).all()


def microseconds(call):
    """The shortest of a few calls on the GPU."""
    call()
    best = float("inf")
    for _ in range(6):
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        call()
        stop.record()
        stop.synchronize()
        best = min(best, 1000.0 * start.elapsed_time(stop))
    return best


@pytest.mark.parametrize("shape", [
    # batch, tokens, H_q, H_kv, d, s_max, context, bits
    (1, 1024, 28, 4, 128, 9024, 9001, 8), (1, 1024, 28, 4, 128, 9024, 9001, 4), (2, 256, 16, 4, 96, 6016, 6000, 4), (8, 1, 32, 8, 128, 32768, 32700, 8),
    (64, 1, 32, 8, 128, 3584, 3550, 4), (16, 5, 32, 8, 128, 4096, 4000, 4),
], ids=str)
def test_a_value_that_is_not_finite_costs_about_another_pass(bd, shape):
    """An element of a query, or a block of the cache, that is NaN has a workgroup go over its keys once more; with what it then looks
    up that is to stay below four passes (and a launch), however long the context is."""
    b, seq, hq, hkv, d, s_max, n, bits = shape
    gen = torch.Generator(device="cuda").manual_seed(n)
    cache = bd.civic_mx_cache(b, hkv, s_max, d, bits)
    for t in cache[:4]:
        t.copy_(torch.randint(0, 120, t.shape, dtype=torch.uint8, device="cuda", generator=gen))
    cache.k_scales.fill_(120), cache.v_scales.fill_(120)
    q = torch.randn((b, seq, hq, d), device="cuda", generator=gen).bfloat16()
    ws = torch.empty(max(bd.civic_attn_mx_workspace_bytes(torch.bfloat16, bits, b, seq, hq, hkv, d, n), 16), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    call = lambda: bd.civic_prefill_attn_mx(q, cache, n, out=out, workspace=ws)  # noqa: E731
    clean = microseconds(call)
    assert out.isfinite().all()
    q[0, seq - 1, 0, 3] = float("nan")
    query = microseconds(call)
    assert out[0, seq - 1, 0].isnan().all() and int(out.isnan().sum()) == d
    q[0, seq - 1, 0, 3] = 0.0
    cache.v_scales[:, :, n // 2, 0] = 255
    block = microseconds(call)
    assert int(out.isnan().sum()) == b * seq * hq * 32
    log("   us clean, NaN query, NaN blocks", clean, query, block)
    assert max(query, block) <= 4 * clean + 20


# ------------------------------------------------------------------------------------------------------ named streams
@pytest.mark.parametrize("form", ["object", "handle"])
@pytest.mark.parametrize("seq", [1, 5])
def test_a_named_streams_calls_share_no_memory_with_the_current_one(bd, form, seq):
    """The call's result and workspace are neither memory that queued work of the current stream still writes, nor handed to the current
    stream while the call's kernels wait on theirs."""
    b, hq, hkv, d, n = 2, 16, 4, 128, 3000
    q, cache, kv = inputs(bd, 15, b, seq, hq, hkv, d, 3008, 4, "bf16")
    dq = to_dev(q)
    need = bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 4, b, seq, hq, hkv, d, n)
    assert need > 0

    def call(stream):
        if seq == 1:
            return bd.civic_decode_attn_mx(dq[:, 0], cache, n, stream=stream)
        return bd.civic_prefill_attn_mx(dq, cache, n, stream=stream)

    ref = call(None)
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    stream = side if form == "object" else side.cuda_stream
    busy = torch.randn((4096, 4096), device="cuda")
    sizes = (need, ref.nbytes)
    for _ in range(3):
        # the current stream's memory, free again while its writes are still to come
        torch.cuda.synchronize()
        torch.mm(busy, busy)
        old = [torch.empty(s, dtype=torch.uint8, device="cuda") for s in sizes for _ in range(4)]
        for t in old:
            t.fill_(0xFF)
        del old, t
        first = call(stream)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(first, ref)
        # the call's, while its kernels are still to come
        side.wait_stream(here)
        with torch.cuda.stream(side):
            torch.mm(busy, busy)
        second = call(stream)
        new = [torch.full((s,), 0xFF, dtype=torch.uint8, device="cuda") for s in sizes for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(second, ref) and all((t == 0xFF).all() for t in new)
        del new, first, second
    # the default stream by its handle
    torch.cuda.synchronize()
    assert torch.equal(call(torch.cuda.default_stream().cuda_stream), ref)


# ---------------------------------------------------------------------------------------------------------- workspaces
@pytest.mark.parametrize("shape", [(4, 1, 32, 8, 128), (1, 1, 8, 4, 64), (1, 40, 8, 2, 128), (1, 130, 4, 1, 64), (2, 9, 16, 8, 256)], ids=str)
def test_one_workspace_serves_a_growing_context(bd, shape):
    """Sized once for the cache, with guard bytes behind it: every shorter context is taken, gives what a workspace of its own gives, and
    leaves the bytes behind alone."""
    b, seq, hq, hkv, d = shape
    s_max = 4480
    q, cache, kv = inputs(bd, 17, b, seq, hq, hkv, d, s_max, 4, "bf16")
    dq = to_dev(q)
    need = bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 4, b, seq, hq, hkv, d, s_max)
    assert need > 0
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    for n in (1, 130, 640, 641, 768, 769, 1025, 2048, 2049, 4096, 4097, 4224, 4225, 4480):
        log("context", n, shape)
        a = bd.civic_prefill_attn_mx(dq, cache, n, workspace=ws[:need])
        assert torch.equal(a, bd.civic_prefill_attn_mx(dq, cache, n)) and a.isfinite().all()
    assert (ws[need:] == 0xFF).all()


# ---------------------------------------------------------------------------------------------------------- large logits
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", [(1, 2, 4, 2, 64, 704, 700), (2, 1, 8, 2, 128, 1504, 1500), (32, 1, 16, 8, 64, 704, 700), (1, 20, 4, 1, 96, 480, 470)], ids=str)
def test_large_logits_that_lie_close_keep_their_weights(bd, bits, causal, shape):
    """Logits of some 20000 to 44000, exact in fp32 and a few units apart, whose largest differ between the steps, wavefronts and splits that
    meet.  With s the fp32 scale times log2(e), a logit z in the part taken against m has the weight 2^(s z - s m) up to: the argument's
    rounding (|s (z - m)| <= 12: 2^-21) and the exponential's (2^-23); what joins the parts (renewals, wavefronts, splits: at most 8 factors of
    the like): below 2^-17 in all; s itself is off by 2^-24 of 12.  Sums of n weights and products are off by (n + 64) 2^-24 each, values
    by 2^-24.  Weights of 20000 times 2^-24 of rounding left in a part would be 1e-3."""
    b, seq, hq, hkv, d, s_max, n = shape
    rng = np.random.default_rng(d + n)
    values = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    k = np.zeros((b, hkv, s_max, d), np.float32)
    k[..., 0] = 1.0
    # the largest logit of 32 consecutive keys is one of the values; that of all 6
    most = rng.integers(3, 8, (b, hkv, s_max // 32)).repeat(32, axis=2)
    k[..., 1] = values[(rng.random((b, hkv, s_max)) * (most + 1)).astype(int)]
    k[..., 2] = 6.0                                                                          # the block's scale; no query looks at it
    v = (rng.choice([-1.0, 1.0], (b, hkv, s_max // 32, d)).repeat(32, axis=2) * rng.choice([2.0, 3.0, 4.0, 6.0], (b, hkv, s_max, d))).astype(np.float32)
    cache, kf, vf = cache_of(bd, k, v, bits)
    assert np.array_equal(kf, k) and np.array_equal(vf, v)
    q = np.zeros((b, seq, hq, d), np.float32)
    q[..., 0] = rng.integers(20000, 44000, (b, seq, hq))
    q[..., 1] = 1.0
    spoil(cache, [n] * b)
    got = bd.civic_prefill_attn_mx(to_dev(q), cache, n, causal=causal, softmax_scale=1.0).cpu().numpy().astype(np.float64)
    z = np.repeat(k[:, :, :n, 1], hq // hkv, axis=1)[:, None].astype(np.float64)              # the constant of a row falls out
    sees = np.arange(n) < (n - (seq - 1 - np.arange(seq)) if causal else np.full(seq, n))[:, None]
    w = np.where(sees[None, :, None], np.exp(z - 6.0), 0.0)
    w /= w.sum(-1, keepdims=True)
    ref = np.einsum("bthn,bhnd->bthd", w, np.repeat(vf[:, :, :n], hq // hkv, axis=1).astype(np.float64))
    tol = 6.0 * (2.0 * (n + 64) * 2.0 ** -24 + 2.0 ** -17 + 2.0 ** -24)
    log("   off by", np.abs(got - ref).max(), "of", tol)
    assert np.abs(got - ref).max() <= tol


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("seq", [1, 20])
def test_queries_up_to_the_largest_fp32_number(bd, bits, seq):
    """A query at the end of fp32's range against keys as small: logits of a few units, which its bf16 terms have to be finite for."""
    b, hq, hkv, d, n = 1, 4, 2, 64, 300
    rng = np.random.default_rng(bits)
    k = (rng.choice([0.5, 1.0, 2.0, 6.0], (b, hkv, 320, d)) * 2.0 ** -90).astype(np.float32)
    k[..., 1:8] *= 0
    v = rng.standard_normal((b, hkv, 320, d)).astype(np.float32)
    cache, kf, vf = cache_of(bd, k, v, bits)
    q = np.zeros((b, seq, hq, d), np.float32)
    q[..., 0] = rng.choice(np.array([3.4028235e38, 3.4e38, 3.397e38, 3.39e38, -3.4028235e38], np.float32), (b, seq, hq))
    q[..., 8] = rng.standard_normal((b, seq, hq)) * 1e38
    scale = 2.0 ** -38                                        # logits q k scale: up to 2^128 6 2^-90 2^-38
    out = bd.civic_prefill_attn_mx(to_dev(q), cache, n, softmax_scale=scale).cpu().numpy().astype(np.float64)
    ref, wa, la = oracle.cache_attention(q, kf, vf, [n], True, scale)
    assert np.isfinite(out).all() and (np.abs(out - ref) <= tolerance(ref, wa, la, d, n, "fp32", seq * 2)).all()
    # and an infinity stays one: the rows that hold it are NaN, no others
    q[0, 0, 1, 9] = np.inf
    again = bd.civic_prefill_attn_mx(to_dev(q), cache, n, softmax_scale=scale).cpu().numpy()
    hit = np.zeros(again.shape[:3], bool)
    hit[0, 0, 1] = True
    assert np.isnan(again[hit]).all() and np.array_equal(again[~hit], out[~hit].astype(np.float32))
