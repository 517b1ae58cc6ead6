"""A cache that forgets and a prefix that is shared: what is measured of four kinds of pass over a KV cache, each a public call of
paper_2605_28115_amd.binding.

  weights  how much attention every cache row has received from the last `seq` tokens: the sum of their softmax weights over the
           tokens and over the query heads of the row's KV head
  decode   one new token's attention over the cache, with those sums as a second output
  evict    of every KV head the rows with the largest sums, with the first and the latest ones, moved together in their order
  shared   new tokens' attention over a prefix that the whole batch shares and, behind it, their sample's own cache rows

The caches are [batch, kv_heads, s_max, head_dim] (the prefix without the batch).  Sample b holds ctx[b] rows, the new tokens' own
rows the last of them; token i of seq sees the rows j < ctx[b] - (seq - 1 - i) where causal.  A token that sees no row has no weights,
and an output of zeros.

`run` computes the same with elementary torch operations in 32 bits where `own` is false.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
ESZ = {"fp32": 4, "bf16": 2}


# ------------------------------------------------------------------------------------------------------ the cases
def listed():
    large, small = dict(q_heads=32, kv_heads=8, head_dim=128), dict(q_heads=16, kv_heads=8, head_dim=128)
    return [
        # the last words of one compact prompt look back at it, before the first eviction: launches are everything
        dict(name="weights-window", kind="weights", dtype="bf16", batch=1, seq=32, ctx="469", s_max=512, causal=True, base=False, **small),
        # four whole compact prompts weigh their own rows
        dict(name="weights-prompts", kind="weights", dtype="bf16", batch=4, seq=938, ctx="938", s_max=1024, causal=True, base=False, **large),
        # a question of 61 tokens about hours of video adds to what the rows have gathered
        dict(name="weights-video", kind="weights", dtype="bf16", batch=2, seq=61, ctx="41000..65000", s_max=65536, causal=True, base=True, **large),
        # the next token of the smallest configuration, in full precision
        dict(name="decode-tiny", kind="decode", dtype="fp32", batch=1, ctx="117", s_max=128, base=True, q_heads=4, kv_heads=2, head_dim=64),
        # the next token of a serving batch of 64 conversations, every one at a length of its own
        dict(name="decode-serve", kind="decode", dtype="bf16", batch=64, ctx="117..3584", s_max=3584, base=True, **large),
        # the next token of eight conversations about hours of video
        dict(name="decode-long", kind="decode", dtype="bf16", batch=8, ctx="65000", s_max=65536, base=True, **large),
        # one prompt's cache to a third of its rows, as the visual tokens before it
        dict(name="evict-prompt", kind="evict", dtype="bf16", batch=1, ctx="469", s_max=512, keep=156, first=4, recent=32, **small),
        # a serving batch's caches to at most 1024 rows; some samples hold fewer
        dict(name="evict-serve", kind="evict", dtype="bf16", batch=64, ctx="700..3584", s_max=3584, keep=1024, first=4, recent=128, **large),
        # two conversations about hours of video, in full precision
        dict(name="evict-long", kind="evict", dtype="fp32", batch=2, ctx="65000", s_max=65536, keep=16001, first=16, recent=512, **large),
        # the next token of four answers about one image prompt
        dict(name="shared-few", kind="shared", dtype="bf16", batch=4, seq=1, prefix=469, ctx="1..23", s_max=64, causal=True, **small),
        # the next token of 64 conversations that began with the same long document
        dict(name="shared-serve", kind="shared", dtype="bf16", batch=64, seq=1, prefix=8001, ctx="117..900", s_max=1024, causal=True, **large),
        # sixteen questions about one video, asked in one pass
        dict(name="shared-questions", kind="shared", dtype="bf16", batch=16, seq=61, prefix=4001, ctx="61..200", s_max=256, causal=True,
             q_heads=28, kv_heads=4, head_dim=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    kinds = ("weights", "decode", "evict", "shared")
    most = {k: max(work(c)["bytes"] for c in listed() if c["kind"] == k) for k in kinds}
    busiest = {k: max(work(c)["flops"] for c in listed() if c["kind"] == k) for k in kinds}
    while True:
        q, kv = rng.choice([(4, 2), (8, 8), (16, 8), (16, 16), (16, 4), (32, 8), (32, 8), (32, 4), (28, 4), (24, 2), (64, 4)])
        c = dict(kind=rng.choice(["weights", "decode", "evict", "shared", "shared"]), dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]),
                 batch=_log(rng, 1, 64), q_heads=q, kv_heads=kv, head_dim=rng.choice([64, 96, 128, 128, 128, 256]))
        top = _log(rng, 1, 2000 if c["kind"] == "shared" else 100000)
        c["ctx"] = "%d" % top if rng.random() < 0.5 else "%d..%d" % (top // rng.choice([2, 8, 30]), top)
        c["s_max"] = top + _log(rng, 1, 500)
        if c["kind"] in ("weights", "decode"):
            c["base"] = rng.random() < 0.5
        if c["kind"] in ("weights", "shared"):
            c["causal"] = rng.random() < 0.8
            c["seq"] = 1 if c["kind"] == "shared" and rng.random() < 0.4 else min(_log(rng, 1, 2000), top)
        if c["kind"] == "shared":
            c["prefix"] = _log(rng, 1, 40000)
        if c["kind"] == "evict":
            c["first"], c["recent"] = rng.choice([0, 4, _log(rng, 1, 100)]), rng.choice([0, 32, _log(rng, 1, 1000)])
            c["keep"] = c["first"] + c["recent"] + _log(rng, 1, max(top, 2))
        w = work(c)
        # no dearer than the listed ones of its kind; in full precision at most a tenth of their products
        if w["bytes"] <= most[c["kind"]] and w["flops"] <= busiest[c["kind"]] * (0.1 if c["dtype"] == "fp32" else 1.0) + 1e6:
            return c


def _contexts(c):
    """Rows that every sample's cache holds: one number, or spread evenly over lo..hi in a fixed shuffled order."""
    n = c["batch"]
    if ".." not in c["ctx"]:
        return [int(c["ctx"])] * n
    lo, hi = (int(x) for x in c["ctx"].split(".."))
    at = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    step = next(s for s in (37, 41, 43, 47) if math.gcd(s, n) == 1)
    return [at[i * step % n] for i in range(n)]


def _pairs(c):
    """(token, own cache row) pairs of the batch."""
    t = c.get("seq", 1)
    if c.get("causal"):
        return sum(sum(max(0, n - t + 1 + i) for i in range(t)) for n in _contexts(c))
    return sum(_contexts(c)) * t


def work(case):
    c, d, e, b = case, case["head_dim"], ESZ[case["dtype"]], case["batch"]
    row, hq, hkv, held = d * e, case["q_heads"], case["kv_heads"], sum(_contexts(case))
    sums = 4 * hkv * (b * c["s_max"] + (held if c.get("base") else 0))                # written; those added to, read
    if c["kind"] == "weights":
        return {"bytes": hkv * row * held + b * c["seq"] * hq * row + sums, "flops": 2 * hq * d * _pairs(c)}
    if c["kind"] == "decode":
        return {"bytes": 2 * hkv * row * held + 2 * b * hq * row + sums, "flops": 4 * hq * d * held}
    if c["kind"] == "evict":
        kept = sum(min(n, c["keep"]) for n in _contexts(c))
        return {"bytes": hkv * (4 * held + 2 * 2 * row * kept + b * 8 * c["keep"]), "flops": hkv * held}
    return {"bytes": 2 * hkv * row * (held + c["prefix"]) + 2 * b * c["seq"] * hq * row,
            "flops": 4 * hq * d * (_pairs(c) + b * c["seq"] * c["prefix"])}


# ----------------------------------------------------------------------------------------------------- plain form
def _sees(s, n, device):
    """[batch, seq, n]: whether a token sees a row of its sample's cache."""
    sees = s["ctx"][:, None].expand(s["batch"], s["seq"])
    if s["causal"]:
        sees = sees - (s["seq"] - 1) + torch.arange(s["seq"], device=device)
    return torch.arange(n, device=device) < sees[:, :, None]


def _by_group(q, kv):
    """[seq, heads, d] -> [kv, seq * group, d] in fp32: the queries of a KV head as rows (token, head of the group)."""
    t, hq, d = q.shape
    return q.float().unflatten(1, (kv, hq // kv)).transpose(0, 1).reshape(kv, t * (hq // kv), d)


def _from_groups(o, t, hq):
    """The reverse."""
    kv, _, d = o.shape
    return o.reshape(kv, t, hq // kv, d).transpose(0, 1).reshape(t, hq, d)


def _softmax(z, seen):
    """Weights over the last axis where seen; none where nothing is."""
    z = torch.where(seen, z, torch.full_like(z, -math.inf))
    top = z.amax(dim=-1, keepdim=True) if z.shape[-1] else z.new_zeros(z.shape[:-1] + (1,))
    p = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(dim=-1, keepdim=True)
    return p / torch.where(total > 0, total, torch.ones_like(total))


def _plain_attention(s):
    """weights, decode: the sums, and for decode the output."""
    q, n = s["q"], s["n_ctx"]
    b, t, hq, d = q.shape
    kv, s_max = s["k"].shape[1:3]
    sums = torch.zeros((b, kv, s_max), dtype=torch.float32, device=q.device) if s["base"] is None else s["base"].clone()
    out = torch.empty_like(q)
    sees = _sees(s, n, q.device)
    for i in range(b):
        rows = _by_group(q[i], kv)
        seen = sees[i].repeat_interleave(hq // kv, dim=0)
        for g in range(kv):
            z = torch.matmul(rows[g], s["k"][i, g, :n].float().t()) * (1.0 / math.sqrt(d))
            p = _softmax(z, seen)
            sums[i, g, :n] += p.sum(dim=0)
            if s["kind"] == "decode":
                out[i, :, g * (hq // kv):(g + 1) * (hq // kv)] = torch.matmul(p, s["v"][i, g, :n].float()).reshape(t, hq // kv, d).to(q.dtype)
    return [sums] if s["kind"] == "weights" else [out, sums]


def _plain_shared(s):
    q, n = s["q"], s["n_ctx"]
    b, t, hq, d = q.shape
    kv = s["k"].shape[1]
    kp, vp = s["k_prefix"].float(), s["v_prefix"].float()
    sees = _sees(s, n, q.device)
    whole = torch.ones((t, kp.shape[1]), dtype=torch.bool, device=q.device)
    out = torch.empty_like(q)
    for i in range(b):
        rows = _by_group(q[i], kv)
        k, v = torch.cat((kp, s["k"][i, :, :n].float()), dim=1), torch.cat((vp, s["v"][i, :, :n].float()), dim=1)
        seen = torch.cat((whole, sees[i]), dim=1).repeat_interleave(hq // kv, dim=0)
        p = _softmax(torch.matmul(rows, k.transpose(1, 2)) * (1.0 / math.sqrt(d)), seen[None])
        out[i] = _from_groups(torch.matmul(p, v), t, hq).to(q.dtype)
    return [out]


def _plain_evict(s):
    k, v, w, keep = s["k"], s["v"], s["weights"], s["keep"]
    b, kv, s_max, d = k.shape
    n = s["ctx"].long()[:, None, None]
    at = torch.arange(s_max, device=k.device)
    held = (at < n).expand(b, kv, s_max)
    fixed = held & ((at < s["first"]) | (at >= n - s["recent"]))
    # an order of all rows: those that stay whatever they weigh, by falling sums (the lower row first where equal), what is not held
    score = torch.where(fixed, torch.full_like(w, math.inf), torch.where(held, w, torch.full_like(w, -math.inf)))
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :keep]
    if keep > s_max:
        order = torch.nn.functional.pad(order, (0, keep - s_max))
    kept = n.clamp_max(keep)
    there = (torch.arange(keep, device=k.device) < kept).expand(b, kv, keep)
    idx = torch.where(there, order, torch.full_like(order, s_max)).sort(dim=-1).values   # rising, what is not there last
    take = idx.clamp_max(s_max - 1)

    def rows(x):
        r = x.gather(2, take[..., None].expand(-1, -1, -1, d))
        return torch.where(there[..., None], r, torch.zeros_like(r))

    kept_w = torch.where(there, w.gather(2, take), torch.zeros_like(w[:, :, :1]))
    return [rows(k), rows(v), kept_w, torch.where(there, idx, torch.full_like(idx, -1)).int(), kept[:, 0, 0].int()]


# --------------------------------------------------------------------------------------------------- inputs, passes
def prepare(case, seed):
    c, d, dt, b = case, case["head_dim"], DTYPES[case["dtype"]], case["batch"]
    hq, kv, s_max = c["q_heads"], c["kv_heads"], c["s_max"]
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    # keys have channels of a size of their own, as trained ones do
    loud = 1.0 + 3.0 * (torch.rand((kv, 1, d), generator=g, device="cuda") < 0.05).float()

    def cache(rows, size, batch=None):
        if batch is None:
            return (randn(kv, rows, d) * size).to(dt)
        x = torch.empty((batch, kv, rows, d), dtype=dt, device="cuda")
        for i in range(batch):
            x[i] = randn(kv, rows, d) * size
        return x

    ctx = _contexts(c)
    s = {"kind": c["kind"], "batch": b, "seq": c.get("seq", 1), "causal": c.get("causal", False), "n_ctx": max(ctx),
         "ctx": torch.tensor(ctx, dtype=torch.int32, device="cuda"), "k": cache(s_max, loud, b)}
    if c["kind"] != "weights":
        s["v"] = cache(s_max, 1.0, b)
    if c["kind"] != "evict":
        s["q"] = randn(b, s["seq"], hq, d).to(dt)
    if c["kind"] in ("weights", "decode"):
        # what the rows have gathered so far, and nothing behind a sample's rows
        s["base"] = None
        if c["base"]:
            s["base"] = torch.exp(2.0 * randn(b, kv, s_max)) * (torch.arange(s_max, device="cuda") < s["ctx"][:, None, None])
    elif c["kind"] == "evict":
        # sums as they come about: over many orders of magnitude, none at all for some rows, and equal ones
        w = torch.exp(3.0 * randn(b, kv, s_max) - 4.0)
        none = torch.rand((b, kv, s_max), generator=g, device="cuda") < 0.1
        s["weights"] = torch.where(none, torch.zeros_like(w), torch.where(w > 1.0, torch.round(w * 8.0) / 8.0, w))
        s.update(keep=c["keep"], first=c["first"], recent=c["recent"])
    elif c["kind"] == "shared":
        s["k_prefix"], s["v_prefix"] = cache(c["prefix"], loud), cache(c["prefix"], 1.0)
    if own:
        from paper_2605_28115_amd import binding as bd
        need = 0
        if c["kind"] in ("weights", "decode"):
            s["sums"] = torch.empty((b, kv, s_max), dtype=torch.float32, device="cuda")
        if c["kind"] in ("decode", "shared"):
            s["out"] = torch.empty_like(s["q"])
        if c["kind"] == "weights":
            need = bd.civic_attn_weights_workspace_bytes(dt, b, s["seq"], hq, kv, d, s["n_ctx"])
        elif c["kind"] == "decode":
            need = bd.civic_decode_attn_weights_workspace_bytes(dt, b, hq, kv, d, s["n_ctx"])
        elif c["kind"] == "shared":
            need = bd.civic_attn_shared_workspace_bytes(dt, b, s["seq"], hq, kv, d, c["prefix"], s["n_ctx"])
        else:
            need = bd.civic_kv_evict_workspace_bytes(b, kv, s["n_ctx"])
            s["kept"] = [torch.zeros((b, kv, c["keep"], d), dtype=dt, device="cuda") for _ in range(2)] + [
                torch.zeros((b, kv, c["keep"]), dtype=torch.float32, device="cuda"), torch.zeros((b, kv, c["keep"]), dtype=torch.int32, device="cuda"),
                torch.zeros(b, dtype=torch.int32, device="cuda")]
        s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


def run(state):
    s = state
    if not own:
        return {"evict": _plain_evict, "shared": _plain_shared}.get(s["kind"], _plain_attention)(s)
    from paper_2605_28115_amd import binding as bd
    if s["kind"] == "weights":
        bd.civic_attn_weights(s["q"], s["k"], s["n_ctx"], ctx=s["ctx"], causal=s["causal"], base=s["base"], weights=s["sums"], workspace=s["workspace"])
        return [s["sums"]]
    if s["kind"] == "decode":
        bd.civic_decode_attn_weights(s["q"][:, 0], s["k"], s["v"], s["n_ctx"], ctx=s["ctx"], base=s["base"], weights=s["sums"], out=s["out"][:, 0],
                                     workspace=s["workspace"])
        return [s["out"], s["sums"]]
    if s["kind"] == "evict":
        k, v, w, idx, ctx = s["kept"]
        bd.civic_kv_evict(s["k"], s["v"], s["weights"], s["keep"], s["n_ctx"], ctx=s["ctx"], first=s["first"], recent=s["recent"], k_out=k, v_out=v,
                          weights_out=w, kept_idx=idx, ctx_out=ctx, workspace=s["workspace"])
        return list(s["kept"])
    if s["seq"] == 1:
        bd.civic_decode_attn_shared(s["q"][:, 0], s["k_prefix"], s["v_prefix"], s["k"], s["v"], s["n_ctx"], ctx=s["ctx"], out=s["out"][:, 0],
                                    workspace=s["workspace"])
    else:
        bd.civic_prefill_attn_shared(s["q"], s["k_prefix"], s["v_prefix"], s["k"], s["v"], s["n_ctx"], ctx=s["ctx"], causal=s["causal"], out=s["out"],
                                     workspace=s["workspace"])
    return [s["out"]]


# -------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    ctx, kv, t = _contexts(c), c["kv_heads"], c.get("seq", 1)
    if c["kind"] == "evict":
        k, v, w = (torch.zeros_like(x[:, :, :1]).expand(-1, -1, c["keep"], *x.shape[3:]).double().contiguous() for x in (s["k"], s["v"], s["weights"]))
        idx = torch.full((c["batch"], kv, c["keep"]), -1, dtype=torch.int32, device="cuda")
        for i, n in enumerate(ctx):
            m = min(n, c["keep"])
            lo, hi = c["first"], n - c["recent"]
            for g in range(kv):
                if m == n:
                    rows = torch.arange(n, device="cuda")
                else:
                    among = s["weights"][i, g, lo:hi]
                    # the least of the sums that stay, then as many of the equal ones as there is room for, from the first
                    room = m - c["first"] - c["recent"]
                    border = among.kthvalue(hi - lo - room + 1).values if room else among.new_tensor(math.inf)
                    stays, equal = among > border, (among == border).nonzero().flatten()
                    stays[equal[:room - int(stays.sum())]] = room > 0
                    rows = torch.cat((torch.arange(lo, device="cuda"), lo + stays.nonzero().flatten(), torch.arange(hi, n, device="cuda")))
                idx[i, g, :m] = rows.int()
                k[i, g, :m], v[i, g, :m], w[i, g, :m] = s["k"][i, g, rows].double(), s["v"][i, g, rows].double(), s["weights"][i, g, rows].double()
        return [k, v, w, idx, torch.tensor([min(n, c["keep"]) for n in ctx], dtype=torch.int32, device="cuda")]
    hq, d = s["q"].shape[2:]
    group = hq // kv
    # twice the time of the listed ones would be too long
    if 4 * hq * d * (_pairs(c) + c["batch"] * t * c.get("prefix", 0)) > 1.5e12:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    sums = torch.zeros((c["batch"], kv, c["s_max"]), dtype=torch.float64, device="cuda")
    if s.get("base") is not None:
        sums += s["base"].double()
    for i, held in enumerate(ctx):
        for g in range(kv):
            k = s["k"][i, g, :held].double()
            if c["kind"] == "shared":
                k = torch.cat((s["k_prefix"][g].double(), k))
            if k.shape[0] == 0:
                continue
            v = None
            if c["kind"] != "weights":
                v = s["v"][i, g, :held].double()
                if c["kind"] == "shared":
                    v = torch.cat((s["v_prefix"][g].double(), v))
            for h in range(g * group, (g + 1) * group):
                z = (s["q"][i, :, h].double() @ k.t()) / math.sqrt(d)
                if c.get("causal"):
                    row = torch.arange(k.shape[0], device="cuda")[None] - c.get("prefix", 0)
                    z = z.masked_fill(row > torch.arange(t, device="cuda")[:, None] + (held - t), -math.inf)
                p = torch.softmax(z, dim=-1).nan_to_num(0.0)                           # a token that sees no row
                if c["kind"] != "shared":
                    sums[i, g, :held] += p.sum(dim=0)
                if v is not None:
                    out[i, :, h] = p @ v
    return {"weights": [sums], "decode": [out, sums], "shared": [out]}[c["kind"]]
