"""The path into a cache in 8 or 4 bits: compact prompts of different length and grid, their compact positions, attention over the
prompts, the cache they enter rotated, and the questions and tokens that follow, each step against the oracle."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_mx import bd, tolerance  # noqa: F401  (bd: the fixture)
from test_gpu_parity import attn_tol, log
from test_gpu_ragged_path import layout
from test_gpu_rope import rope_tol

pytestmark = pytest.mark.gpu


def host(t):
    return np.ascontiguousarray(t.float().cpu().numpy())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_compact_prompts_their_questions_and_answers(bd, bits, dtype):
    grids = [(1, 8, 8, 4, 4, 2, 0, 20), (2, 6, 5, 2, 2, 1, 3, 31), (1, 16, 16, 4, 4, 1, 0, 85)]
    b, dim, hq, hkv, d, s_max = len(grids), 128, 8, 2, 64, 192
    name = "bf16" if dtype == torch.bfloat16 else "fp32"
    rng = np.random.default_rng(bits)
    gen = torch.Generator(device="cuda").manual_seed(bits)
    starts, lens = layout(rng, grids, 9)
    total = int(sum(lens))
    hidden = torch.randn((total, dim), device="cuda", generator=gen).to(dtype)
    ids = torch.from_numpy(np.stack([np.concatenate([np.arange(n) for n in lens])] * 3).astype(np.int32)).cuda()
    anchor = torch.from_numpy(bd.civic_anchor_normalize(rng.standard_normal(dim).astype(np.float32))).cuda()
    log("path", bits, name, lens)
    _, _, rows, pos, _ = bd.civic_compact_prefill_ragged(hidden, ids, lens, grids, starts, anchor)
    _, _, _, off = bd.civic_ragged_offsets(lens, grids)
    weights = [torch.randn((dim, h * d), device="cuda", generator=gen) * dim ** -0.5 for h in (hq, hkv, hkv)]
    project = lambda x: [torch.mm(x.float(), w).to(dtype).view(x.shape[0], -1, d) for w in weights]  # noqa: E731
    axis, inv = np.arange(d // 2) % 3, (1e4 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)

    # the prompts: rotated, attended, written
    q, k, v = project(rows)
    table = bd.civic_mrope_table(pos[:, None].contiguous(), axis, inv)
    turned = [bd.civic_mrope_apply(x[None], table)[0] for x in (q, k)]
    out = bd.civic_prefill_attn_ragged(*turned, v, off)
    cache = bd.civic_mx_cache(b, hkv, s_max, d, bits)
    bd.civic_kv_write_mx_ragged(k, v, cache, off, cos_sin=table[0])
    want = [np.zeros((b, hkv, s_max, d), np.float32) for _ in range(2)]
    ids_h, table_h = pos.cpu().numpy(), oracle.mrope_table(pos[:, None].cpu().numpy(), axis, inv)
    for i in range(b):
        at = slice(int(off[i]), int(off[i + 1]))
        qi, ki, vi = (host(x[at])[None] for x in (*turned, v))
        # the angles are those of the compact positions
        ref_k = oracle.mrope_apply(host(k[at])[None], table_h[:, at])
        assert np.abs(ki - ref_k).max() <= rope_tol(ref_k, name) and ids_h[:, at].max() < lens[i]
        ref = oracle.attention(qi, ki, vi, True)
        assert np.abs(host(out[at]) - ref[0]).max() <= attn_tol(ref, name)
        for w, x in zip(want, (ki[0], vi[0])):
            w[i, :, :at.stop - at.start] = oracle.mx_decode(*oracle.mx_encode(x.transpose(1, 0, 2), bits), bits)
    ctx = torch.from_numpy(np.diff(off).astype(np.int32)).cuda()

    def held():
        kf, vf = (torch.empty((b, s_max, hkv, d), device="cuda") for _ in range(2))
        return [np.ascontiguousarray(x.cpu().numpy().transpose(0, 2, 1, 3)) for x in bd.civic_kv_read_mx(cache, kf, vf)]

    for x, w in zip(held(), want):
        assert np.array_equal(x, w)

    # a question (more than 32 rows a KV head), a short one, then tokens one by one, at the ids behind the prompts' last
    last = torch.tensor([int(ids_h[:, off[i]:off[i + 1]].max()) for i in range(b)], dtype=torch.int32, device="cuda")
    for seq in (11, 3, 1, 1):
        q, k, v = (x.view(b, seq, -1, d) for x in project(torch.randn((b * seq, dim), device="cuda", generator=gen).to(dtype)))
        new = (last[:, None] + 1 + torch.arange(seq, device="cuda", dtype=torch.int32)).expand(3, b, seq).contiguous()
        table = bd.civic_mrope_table(new, axis, inv)
        bd.civic_kv_write_mx(k, v, cache, pos=ctx, cos_sin=table)
        ctx, last = ctx + seq, last + seq
        q = bd.civic_mrope_apply(q, table)
        if seq > 1:
            out = bd.civic_prefill_attn_mx(q, cache, s_max, ctx=ctx)
        else:
            out = bd.civic_decode_attn_mx(q[:, 0], cache, s_max, ctx=ctx)[:, None]
        ref, wa, la = oracle.cache_attention(host(q), *held(), ctx.cpu().numpy(), True)
        assert (np.abs(host(out) - ref) <= tolerance(ref, wa, la, d, s_max, name, seq * hq // hkv)).all()
    assert ctx.tolist() == [int(n) + 16 for n in np.diff(off)]
