"""A KV cache held in 8 or 4 bits: what is measured of its write, its read back and the attention over it.

The cache is in the OCP microscaling formats.  Every 32 consecutive channels of a head row share one scale, a power of
two held in a byte s (2^(s - 127)); an element is an e2m1 number (format 4: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
negatives, two in a byte, the even channel in the low half) or an e4m3 number (format 8).  A block's exponent is the
least e for which its largest magnitude is at most 7 * 2^e (e2m1) or 464 * 2^e (e4m3), held within [-100, 125] and
[-100, 119]; an element is the code nearest to x * 2^-e, ties to the even code.  A block that holds a NaN or an infinity
has s = 255 and reads back as NaN.

Four kinds of pass, each a public call of paper_2605_28115_amd.binding (the write followed by the read back of its rows,
so that what the cache now holds is there as values):

  write    K and V rows of new tokens into the cache, K rotated on its way where the case says so
  read     cache rows back as K and V rows
  decode   one new token's attention over the cache
  prefill  a chunk of new tokens' attention over a cache that holds them and what came before

`run` computes the same with elementary torch operations in 32 bits where `own` is false.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 32
#: per format: the largest magnitude that a scale of 1 takes, the largest exponent, the largest element
TAKES, TOP, LARGEST = {4: 7.0, 8: 464.0}, {4: 125, 8: 119}, {4: 6.0, 8: 448.0}
BOTTOM = -100


# ------------------------------------------------------------------------------------------------------ the cases
def listed():
    large, small = dict(q_heads=32, kv_heads=8, head_dim=128), dict(q_heads=16, kv_heads=8, head_dim=128)
    return [
        # one generated token of one conversation enters its cache: a few kilobytes, launches are everything
        dict(name="write-token", kind="write", format=4, dtype="bf16", batch=1, seq=1, pos0=469, s_max=512, spread=0, rope=False, **small),
        # the compact prompts of four two-image conversations, keys rotated on the way
        dict(name="write-prompts", kind="write", format=4, dtype="bf16", batch=4, seq=938, pos0=0, s_max=1024, spread=0, rope=True, **large),
        # sixteen long prompts in full precision into eight bits, each behind what its sample holds already
        dict(name="write-long", kind="write", format=8, dtype="fp32", batch=16, seq=4001, pos0=5, s_max=4096, spread=33, rope=False, **large),
        # one image prompt's rows back, for a check or a move to another place
        dict(name="read-prompt", kind="read", format=8, dtype="bf16", batch=1, seq=469, pos0=0, s_max=480, spread=0, **small),
        # a serving batch's whole cache back in 16 bits
        dict(name="read-serve", kind="read", format=4, dtype="bf16", batch=64, seq=3550, pos0=17, s_max=3584, spread=9, **large),
        # the next token of the smallest configuration, in full precision
        dict(name="decode-tiny", kind="decode", format=8, dtype="fp32", batch=1, ctx="117", s_max=128, q_heads=4, kv_heads=2, head_dim=64),
        # the next token of a single conversation
        dict(name="decode-one", kind="decode", format=4, dtype="bf16", batch=1, ctx="469", s_max=512, **small),
        # the next token of a serving batch of 64 conversations, every one at a length of its own
        dict(name="decode-serve", kind="decode", format=4, dtype="bf16", batch=64, ctx="117..3584", s_max=3584, **large),
        # the next token of eight conversations about hours of video
        dict(name="decode-long", kind="decode", format=8, dtype="bf16", batch=8, ctx="65000", s_max=65536, **large),
        # five drafted tokens of sixteen conversations, checked in one pass
        dict(name="prefill-draft", kind="prefill", format=4, dtype="bf16", batch=16, seq=5, ctx="1000..4000", s_max=4096, causal=True, **small),
        # a follow-up question of 128 tokens to four compact prompts
        dict(name="prefill-question", kind="prefill", format=4, dtype="bf16", batch=4, seq=128, ctx="1066", s_max=1088, causal=True, **large),
        # a chunk of a long document behind eight thousand tokens
        dict(name="prefill-chunk", kind="prefill", format=8, dtype="bf16", batch=1, seq=1024, ctx="9001", s_max=9024, causal=True,
             q_heads=28, kv_heads=4, head_dim=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    most = {k: max(work(c)["bytes"] for c in listed() if c["kind"] == k) for k in ("write", "read", "decode", "prefill")}
    busiest = max(work(c)["flops"] for c in listed())
    while True:
        q, kv = rng.choice([(4, 2), (8, 8), (16, 8), (16, 16), (16, 4), (32, 8), (32, 8), (32, 4), (28, 4), (24, 2), (64, 4)])
        c = dict(kind=rng.choice(["write", "read", "decode", "decode", "prefill", "prefill"]), format=rng.choice([4, 4, 8]),
                 dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]), batch=_log(rng, 1, 64), q_heads=q, kv_heads=kv,
                 head_dim=rng.choice([64, 96, 128, 128, 128, 256]))
        if c["kind"] in ("write", "read"):
            c["seq"], c["pos0"], c["spread"] = _log(rng, 1, 8000), rng.choice([0, 0, _log(rng, 1, 900)]), rng.choice([0, _log(rng, 1, 200)])
            c["s_max"] = _whole(c["pos0"] + c["spread"] + c["seq"] + _log(rng, 1, 100))
            if c["kind"] == "write":
                c["rope"] = rng.random() < 0.5
        else:
            top = _log(rng, 1, 100000)
            c["ctx"] = "%d" % top if rng.random() < 0.5 else "%d..%d" % (top // rng.choice([2, 8, 30]), top)
            c["s_max"] = _whole(top + _log(rng, 1, 500))
            if c["kind"] == "prefill":
                c["seq"], c["causal"] = min(_log(rng, 2, 2000), top), rng.random() < 0.8
        w = work(c)
        # no dearer than the listed ones of its kind; in full precision a chunk of at most a tenth of their products
        if w["bytes"] <= most[c["kind"]] and w["flops"] <= busiest * (0.1 if c["dtype"] == "fp32" else 1.0):
            return c


def _whole(rows):
    return -(-rows // BLOCK) * BLOCK


def _contexts(c):
    """Rows that every sample's cache holds: one number, or spread evenly over lo..hi in a fixed shuffled order."""
    n = c["batch"]
    if ".." not in c["ctx"]:
        return [int(c["ctx"])] * n
    lo, hi = (int(x) for x in c["ctx"].split(".."))
    at = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    step = next(s for s in (37, 41, 43, 47) if math.gcd(s, n) == 1)
    return [at[i * step % n] for i in range(n)]


def _firsts(c):
    """The cache row of every sample's first token, counted from pos0: 0, or up to `spread` in a fixed order."""
    return [(11 * i) % (c["spread"] + 1) for i in range(c["batch"])]


def work(case):
    c, d, e = case, case["head_dim"], 2 if case["dtype"] == "bf16" else 4
    held = c["format"] / 8 + 1 / BLOCK                                      # bytes of an element in the cache, scale included
    if c["kind"] in ("write", "read"):
        n = 2 * c["batch"] * c["seq"] * c["kv_heads"] * d
        table = c["batch"] * c["seq"] * d * 4 if c.get("rope") else 0
        # the rows read, the codes written; and for their values the codes read, the rows written
        passes = 2 if c["kind"] == "write" else 1
        return {"bytes": int(n * (held + e) * passes) + table, "flops": 8 * n * passes}
    ctx, t = _contexts(c), c.get("seq", 1)
    pairs = 0
    for n in ctx:
        # token i of the chunk sees rows below n - t + 1 + i
        pairs += sum(max(0, n - t + 1 + i) for i in range(t)) if c.get("causal") else n * t
    return {"bytes": int(2 * c["kv_heads"] * d * held * sum(ctx)) + 2 * c["batch"] * t * c["q_heads"] * d * e, "flops": 4 * c["q_heads"] * d * pairs}


# ----------------------------------------------------------------------------------------------------- plain form
def _two(e):
    """2^e in fp32 for whole e in [-126, 127], by its bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _exponents(x, fmt):
    """Of blocks of fp32 values [..., 32]: the exponents [..., 1] as whole numbers."""
    amax = x.abs().amax(dim=-1, keepdim=True)
    m, ex = torch.frexp(amax)                                               # amax = m * 2^ex, m in [0.5, 1)
    m7, ex7 = math.frexp(TAKES[fmt])
    e = (ex - ex7 + (m > m7).int()).clamp(BOTTOM, TOP[fmt])
    return torch.where(amax == 0, torch.full_like(e, BOTTOM), e)


def _rounded(y, fmt):
    """fp32 values to the nearest element of the format, ties to the even code, saturating."""
    lowest, bits = (0, 1) if fmt == 4 else (-6, 3)                         # exponent of the smallest normal element, mantissa bits
    _, ex = torch.frexp(y)
    step = _two((ex - 1).clamp_min(lowest) - bits)
    return (torch.round(y / step) * step).clamp(-LARGEST[fmt], LARGEST[fmt])


def _quantised(x, fmt):
    """fp32 rows [..., d] -> the elements [..., d] (fp32 values) and the blocks' exponents [..., d / 32]; NaN blocks hold NaN."""
    b = x.unflatten(-1, (-1, BLOCK))
    odd = ~torch.isfinite(b).all(dim=-1, keepdim=True)
    b = torch.where(odd, torch.zeros_like(b), b)
    e = _exponents(b, fmt)
    y = _rounded(b * _two(-e), fmt)
    return torch.where(odd, torch.full_like(y, math.nan), y).flatten(-2), e.squeeze(-1)


def _values(codes, scales, fmt):
    """Codes and scales of cache rows -> fp32 values."""
    c = codes.int()
    if fmt == 4:
        c = torch.stack((c & 15, c >> 4), dim=-1).flatten(-2)
        sign, e, m, bits, bias = c >> 3, (c >> 1) & 3, c & 1, 1, 1
    else:
        sign, e, m, bits, bias = c >> 7, (c >> 3) & 15, c & 7, 3, 7
    mag = (m + torch.where(e > 0, 1 << bits, 0)).float() * _two(e.clamp_min(1) - bias - bits)
    x = torch.where(sign > 0, -mag, mag).unflatten(-1, (-1, BLOCK))
    s = scales.int().unsqueeze(-1)
    return torch.where(s == 255, torch.full_like(x, math.nan), x * _two(s - 127)).flatten(-2)


def _rotated(k, cos_sin):
    """Rotary pairs (i, i + d/2) of fp32 rows [batch, seq, heads, d]; the product and sum as a fused multiply-add rounds them."""
    x0, x1 = k.chunk(2, dim=-1)
    c, s = cos_sin[:, :, None, :, 0], cos_sin[:, :, None, :, 1]
    y0 = (x0.double() * c.double() - (x1 * s).double()).float()
    y1 = (x1.double() * c.double() + (x0 * s).double()).float()
    return torch.cat((y0, y1), dim=-1)


def _rows(s):
    """Cache rows of every sample's tokens, [batch, 1, seq, 1]."""
    at = s["pos0"] + torch.arange(s["seq"], device="cuda")
    return (at if s["pos"] is None else at + s["pos"][:, None]).expand(s["batch"], s["seq"])[:, None, :, None].long()


def _plain_write(s):
    k, v, fmt, dt = s["k"].float(), s["v"].float(), s["format"], s["k"].dtype
    if s["cos_sin"] is not None:
        k = _rotated(k, s["cos_sin"]).to(dt).float()
    (ky, ke), (vy, ve) = _quantised(k, fmt), _quantised(v, fmt)
    return [(y * _two(e).repeat_interleave(BLOCK, dim=-1)).to(dt) for y, e in ((ky, ke), (vy, ve))]


def _plain_read(s):
    at = _rows(s)
    take = lambda t: t.gather(2, at.expand(-1, t.shape[1], -1, t.shape[3]))  # noqa: E731
    return [_values(take(c), take(x), s["format"]).transpose(1, 2).contiguous().to(s["dtype"])
            for c, x in ((s["k_codes"], s["k_scales"]), (s["v_codes"], s["v_scales"]))]


def _plain_attention(s):
    q, n = s["q"], s["n_ctx"]
    b, t, hq, d = q.shape
    kv = s["k_codes"].shape[1]
    k = _values(s["k_codes"][:, :, :n], s["k_scales"][:, :, :n], s["format"])
    v = _values(s["v_codes"][:, :, :n], s["v_scales"][:, :, :n], s["format"])
    # queries of a KV head as rows (token, head of the group)
    rows = q.float().unflatten(2, (kv, hq // kv)).permute(0, 2, 1, 3, 4).reshape(b, kv, t * (hq // kv), d)
    z = torch.matmul(rows, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    sees = s["ctx"][:, None].expand(b, t)
    if s["causal"]:
        sees = sees - (t - 1) + torch.arange(t, device="cuda")
    sees = sees.repeat_interleave(hq // kv, dim=1)[:, None, :, None]
    there = torch.arange(n, device="cuda") < sees
    z = torch.where(there, z, torch.full_like(z, -math.inf))
    top = z.amax(dim=-1, keepdim=True) if n else z.new_zeros(())
    p = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.reshape(b, kv, t, hq // kv, d).permute(0, 2, 1, 3, 4).reshape(b, t, hq, d).to(q.dtype)


# --------------------------------------------------------------------------------------------------- inputs, passes
def _packed(y, e, fmt):
    """Elements and exponents as a cache holds them: bytes [..., d / 2] or [..., d], scales [..., d / 32]."""
    a = y.abs()
    if fmt == 4:
        code = torch.bucketize(a, torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=y.device)).to(torch.uint8)
        code += 8 * (y < 0).to(torch.uint8)
        code = code[..., 0::2] | (code[..., 1::2] << 4)
    else:
        code = y.to(torch.float8_e4m3fn).view(torch.uint8)
    return code, (e + 127).to(torch.uint8)


def prepare(case, seed):
    c, d, fmt, dt = case, case["head_dim"], case["format"], DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    kv, b, rows = c["kv_heads"], c["batch"], c["s_max"]
    # keys have channels of a size of their own, as trained ones do
    loud = 1.0 + 3.0 * (torch.rand((kv, d), generator=g, device="cuda") < 0.05).float()
    s = {"kind": c["kind"], "format": fmt, "dtype": dt, "batch": b, "causal": c.get("causal", False)}
    if c["kind"] in ("write", "read"):
        s.update(seq=c["seq"], pos0=c["pos0"], pos=torch.tensor(_firsts(c), dtype=torch.int32, device="cuda") if c["spread"] else None)
    if c["kind"] == "write":
        # as a projection leaves them: K and V of a token side by side in one row
        both = randn(b, c["seq"], 2, kv, d)
        both[:, :, 0] *= loud
        both = both.to(dt)
        s.update(k=both[:, :, 0], v=both[:, :, 1], cos_sin=None)
        if c["rope"]:
            at = (c["pos0"] + torch.arange(c["seq"], device="cuda", dtype=torch.float64))[:, None] * (1.0e6 ** (-torch.arange(d // 2, device="cuda", dtype=torch.float64) / (d // 2)))
            s["cos_sin"] = torch.stack((at.cos(), at.sin()), dim=-1).float().expand(b, -1, -1, -1).contiguous()
    else:
        for name, size in (("k", loud), ("v", torch.ones_like(loud))):
            codes = torch.empty((b, kv, rows, d * fmt // 8), dtype=torch.uint8, device="cuda")
            scales = torch.empty((b, kv, rows, d // BLOCK), dtype=torch.uint8, device="cuda")
            for i in range(b):
                codes[i], scales[i] = _packed(*_quantised(randn(kv, rows, d) * size[:, None], fmt), fmt)
            s[name + "_codes"], s[name + "_scales"] = codes, scales
    if c["kind"] in ("decode", "prefill"):
        ctx = _contexts(c)
        s.update(q=randn(b, c.get("seq", 1), c["q_heads"], d).to(dt), n_ctx=max(ctx), ctx=torch.tensor(ctx, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2605_28115_amd import binding as bd
        if c["kind"] == "write":
            s["cache"] = bd.civic_mx_cache(b, kv, rows, d, fmt)
        else:
            s["cache"] = bd.MxCache(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], fmt)
        if c["kind"] in ("write", "read"):
            s["back"] = tuple(torch.empty((b, c["seq"], kv, d), dtype=dt, device="cuda") for _ in range(2))
        else:
            s["out"] = torch.empty_like(s["q"])
            need = bd.civic_attn_mx_workspace_bytes(dt, fmt, b, c.get("seq", 1), c["q_heads"], kv, d, s["n_ctx"])
            s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


def run(state):
    s = state
    if not own:
        if s["kind"] in ("write", "read"):
            return (_plain_write if s["kind"] == "write" else _plain_read)(s)
        return [_plain_attention(s)]
    from paper_2605_28115_amd import binding as bd
    if s["kind"] == "write":
        bd.civic_kv_write_mx(s["k"], s["v"], s["cache"], s["pos0"], pos=s["pos"], cos_sin=s["cos_sin"])
    if s["kind"] in ("write", "read"):
        return list(bd.civic_kv_read_mx(s["cache"], *s["back"], s["pos0"], pos=s["pos"]))
    if s["kind"] == "decode":
        bd.civic_decode_attn_mx(s["q"][:, 0], s["cache"], s["n_ctx"], ctx=s["ctx"], out=s["out"][:, 0], workspace=s["workspace"])
    else:
        bd.civic_prefill_attn_mx(s["q"], s["cache"], s["n_ctx"], ctx=s["ctx"], causal=s["causal"], out=s["out"], workspace=s["workspace"])
    return [s["out"]]


# -------------------------------------------------------------------------------------------------------- 64 bits
def _elements(fmt):
    """The format's magnitudes in the order of their codes, in 64 bits."""
    if fmt == 4:
        return [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return [((m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10)) for e in range(16) for m in range(8)][:127]


def _power(e):
    """2^e in 64 bits for whole e, by its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(codes, scales, fmt):
    table = _elements(fmt) + ([0.0] if fmt == 8 else [])
    table = torch.tensor(table + [-x for x in table], dtype=torch.float64, device=codes.device)
    index = codes.long() if fmt == 8 else torch.stack((codes.long() % 16, codes.long() // 16), dim=-1).flatten(-2)
    return table[index] * _power(scales.long() - 127).repeat_interleave(BLOCK, dim=-1)


def _exact_quantised(x, fmt):
    """Rows in 64 bits -> the values that the cache holds for them: the nearest element by search, ties to the even one."""
    el = torch.tensor(_elements(fmt), dtype=torch.float64, device=x.device)
    b = x.unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(dim=-1, keepdim=True)
    e = torch.ceil(torch.log2(amax / TAKES[fmt])).clamp(BOTTOM, TOP[fmt])
    e = torch.where((amax <= TAKES[fmt] * _power(e - 1)) & (e > BOTTOM), e - 1, e)     # the logarithm may be a rounding off
    e = torch.where((amax > TAKES[fmt] * _power(e)) & (e < TOP[fmt]), e + 1, e)
    y = (b.abs() / _power(e)).contiguous()
    below = (torch.searchsorted(el, y, right=True) - 1).clamp_max(len(el) - 2)
    lo, hi = el[below], el[below + 1]
    up = (y - lo > hi - y) | ((y - lo == hi - y) & (below % 2 == 1))
    return (torch.where(up, hi, lo) * torch.sign(b) * _power(e)).flatten(-2)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    fmt, n = c["format"], case["batch"]
    if c["kind"] == "write":
        k, v = s["k"].double(), s["v"].double()
        if s["cos_sin"] is not None:
            turn = torch.view_as_complex(s["cos_sin"].double())[:, :, None]
            half = k.shape[-1] // 2
            z = torch.complex(k[..., :half], k[..., half:]) * turn
            k = torch.cat((z.real, z.imag), dim=-1).to(s["dtype"]).double()           # rotated keys are held in the rows' type
        return [torch.cat([_exact_quantised(x[i:i + 1], fmt) for i in range(n)]) for x in (k, v)]
    if c["kind"] == "read":
        out = []
        for name in ("k", "v"):
            first = [c["pos0"] + f for f in _firsts(c)]
            out.append(torch.stack([_exact_values(s[name + "_codes"][i, :, f:f + c["seq"]], s[name + "_scales"][i, :, f:f + c["seq"]], fmt).transpose(0, 1)
                                    for i, f in enumerate(first)]))
        return out
    q = s["q"].double()
    t, hq, d = q.shape[1:]
    group = hq // c["kv_heads"]
    out = torch.zeros_like(q)
    for i, held in enumerate(_contexts(c)):
        for g in range(c["kv_heads"] if held else 0):
            k = _exact_values(s["k_codes"][i, g, :held], s["k_scales"][i, g, :held], fmt)
            v = _exact_values(s["v_codes"][i, g, :held], s["v_scales"][i, g, :held], fmt)
            z = torch.einsum("thd,nd->htn", q[i, :, g * group:(g + 1) * group], k) / math.sqrt(d)
            if c.get("causal"):
                late = torch.arange(held, device="cuda")[None] > torch.arange(t, device="cuda")[:, None] + (held - t)
                z = z.masked_fill(late, -math.inf)
            p = torch.softmax(z, dim=-1).nan_to_num(0.0)                               # a token that sees no row: zeros
            out[i, :, g * group:(g + 1) * group] = torch.einsum("htn,nd->thd", p, v)
    return [out]
