"""The microscaled cache on the CPU: the oracle against closed forms and against torch's own 8-bit type, the plain forms of
perf/operators.py against both, and every refusal of the C entry points (no call reaches the GPU)."""
import ctypes as C
import itertools

import numpy as np
import pytest
import torch

import oracle

FAKE = C.c_void_p(0x1000)


@pytest.fixture(scope="module")
def bd():
    from paper_2605_28115_amd import binding
    return binding


def rows(seed, n=600, d=96):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((n, d)) * np.exp(rng.uniform(-30, 30, (n, 1)))).astype(np.float32)
    x[::3] = torch.from_numpy(x[::3]).bfloat16().float().numpy()      # few bits: ties are common
    x[0], x[1], x[2] = 0.0, 3.4e38, 1e-38
    x[3] = np.arange(d) * 2.0 ** -102
    return x


@pytest.mark.parametrize("bits", [4, 8])
def test_oracle_rounds_to_the_nearest_element_of_the_least_scale(bits):
    x = rows(bits)
    codes, scales = oracle.mx_encode(x, bits)
    y = oracle.mx_decode(codes, scales, bits).astype(np.float64)
    e = np.repeat(scales.astype(np.int64) - 127, 32, axis=1)
    amax = np.abs(x.astype(np.float64)).reshape(len(x), -1, 32).max(axis=2)
    most, top, bottom = (7.0, 125, -100) if bits == 4 else (464.0, 119, -100)
    se = scales.astype(np.int64) - 127
    assert ((amax <= most * 2.0 ** se) | (se == top)).all() and ((amax > most * 2.0 ** (se - 1)) | (se == bottom)).all()
    # half a step: 2^-2 (e2m1) or 2^-4 (e4m3) of the value, and of the smallest normal element
    step = np.maximum(np.abs(x), (1.0 if bits == 4 else 2.0 ** -6) * 2.0 ** e)
    inside = se < top
    off = np.abs(y - x) / step
    assert off.reshape(len(x), -1, 32)[inside].max() <= (2.0 ** -2 if bits == 4 else 2.0 ** -4)
    assert np.isfinite(y).all()


def test_oracle_elements_are_torchs_eight_bit_type():
    codes = np.arange(256, dtype=np.uint8).reshape(8, 32)
    y = oracle.mx_decode(codes, np.full((8, 1), 127, np.uint8), 8)
    t = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(np.isnan(y), np.isnan(t)) and np.array_equal(y[~np.isnan(y)], t[~np.isnan(t)])
    x = np.random.default_rng(1).uniform(-448, 448, (64, 32)).astype(np.float32)
    x[:, 0] = 448.0                                                    # scale 1
    assert np.array_equal(oracle.mx_encode(x, 8)[0], torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("x,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (-5.0, 14), (7.0, 7), (-7.0, 15), (0.26, 1)])
def test_oracle_ties_of_the_four_bit_element(x, code):
    v = np.zeros((1, 32), np.float32)
    v[0, 0], v[0, 1] = 6.0, x                                          # scale 1
    codes, scales = oracle.mx_encode(v, 4)
    assert scales[0, 0] == 127 and codes[0, 0] >> 4 == code


@pytest.mark.parametrize("bits", [4, 8])
def test_oracle_keeps_odd_blocks_apart(bits):
    x = np.random.default_rng(3).standard_normal((4, 64)).astype(np.float32)
    x[1, 40], x[2, 3], x[3, 0] = np.nan, -np.inf, np.inf
    codes, scales = oracle.mx_encode(x, bits)
    assert (scales == 255).tolist() == [[False, False], [False, True], [True, False], [True, False]]
    y = oracle.mx_decode(codes, scales, bits)
    assert np.array_equal(np.isnan(y).reshape(4, 2, 32).all(axis=2), scales == 255) and np.isnan(y).sum() == 96


@pytest.mark.parametrize("bits", [4, 8])
def test_plain_forms_agree_with_the_oracle(bits):
    import perf.operators as op
    x = rows(10 + bits)
    y, e = op._quantised(torch.from_numpy(x), bits)
    codes, scales = oracle.mx_encode(x, bits)
    assert np.array_equal(e.numpy() + 127, scales)
    pc, ps = op._packed(y, e, bits)
    got = op._values(pc, ps, bits).numpy()
    assert np.array_equal(got, oracle.mx_decode(codes, scales, bits)) and np.array_equal(ps.numpy(), scales)
    assert np.array_equal(op._exact_quantised(torch.from_numpy(x).double(), bits).numpy(), got)
    assert np.array_equal(op._exact_values(pc, ps, bits).numpy(), got)


def test_oracle_cache_attention_is_the_decode_and_the_prefill_oracle():
    rng = np.random.default_rng(5)
    b, t, hq, hkv, d, n = 2, 6, 4, 2, 32, 64
    q = rng.standard_normal((b, t, hq, d)).astype(np.float32)
    k, v = (rng.standard_normal((b, hkv, n, d)).astype(np.float32) for _ in range(2))
    one, _, _ = oracle.cache_attention(q[:, :1], k, v, [40, 40], False)
    assert np.abs(one[:, 0] - oracle.decode_attention(q[:, 0], k, v, 40)).max() < 1e-14
    # the chunk is the whole context: causal prefill
    kp, vp = (np.ascontiguousarray(x[:, :, :t].transpose(0, 2, 1, 3)) for x in (k, v))
    all_, _, _ = oracle.cache_attention(q, k, v, [t, t], True)
    assert np.abs(all_ - oracle.attention(q, kp, vp, True)).max() < 1e-14
    # shorter than the chunk: its first tokens see nothing; the last one sees what a decode step does
    some, size, _ = oracle.cache_attention(q, k, v, [2, 0], True)
    assert (some[0, :4] == 0).all() and (some[1] == 0).all() and (size[0, :4] == 0).all()
    assert np.abs(some[0, 5] - oracle.decode_attention(q[:1, 5], k[:1], v[:1], 2)[0]).max() < 1e-14


# ------------------------------------------------------------------------------------------------------- refusals
def _write(bd, ragged=False, **kw):
    a = dict(k=FAKE, v=FAKE, strides=(4096, 1024, 128), dtype=1, cos=None, fmt=4, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, batch=2, seq=3,
             off=(0, 3, 6), hkv=8, d=128, s_max=64, pos0=0, pos=None)
    a.update(kw)
    st = (C.c_int64 * 3)(*a["strides"]) if a["strides"] else None
    head = [a["k"], a["v"], st, a["dtype"], a["cos"], a["fmt"], a["kc"], a["ks"], a["vc"], a["vs"], a["batch"]]
    tail = [a["hkv"], a["d"], a["s_max"], a["pos0"], a["pos"], None]
    if ragged:
        off = (C.c_int64 * len(a["off"]))(*a["off"]) if a["off"] else None
        return bd.lib.civic_kv_write_mx_ragged(*head, off, *tail)
    return bd.lib.civic_kv_write_mx(*head, a["seq"], *tail)


def _read(bd, **kw):
    a = dict(k=FAKE, v=FAKE, strides=(4096, 1024, 128), dtype=1, fmt=4, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, batch=2, seq=3, hkv=8, d=128,
             s_max=64, pos0=0, pos=None)
    a.update(kw)
    st = (C.c_int64 * 3)(*a["strides"]) if a["strides"] else None
    return bd.lib.civic_kv_read_mx(a["kc"], a["ks"], a["vc"], a["vs"], a["fmt"], a["k"], a["v"], st, a["dtype"], a["batch"], a["seq"], a["hkv"],
                                   a["d"], a["s_max"], a["pos0"], a["pos"], None)


ROWS_BAD = [dict(k=None), dict(v=None), dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None), dict(strides=None), dict(dtype=2), dict(fmt=6),
            dict(fmt=0), dict(batch=-1), dict(hkv=0), dict(d=0), dict(d=72), dict(d=-32), dict(s_max=65), dict(s_max=-32),
            dict(pos0=-1), dict(pos0=62), dict(pos0=65, pos=FAKE), dict(k=C.c_void_p(0x1008)), dict(kc=C.c_void_p(0x1004)),
            dict(vs=C.c_void_p(0x1001)), dict(pos=C.c_void_p(0x1002)), dict(strides=(4096, 1024, 64)), dict(strides=(4096, -1024, 128)),
            dict(strides=(4096, 1028, 128))]
ROWS_LARGE = [dict(d=288, strides=(9216, 2304, 288)), dict(batch=65536, off=[0] * 65536 + [3]), dict(hkv=40000), dict(s_max=(1 << 22) + 32)]


@pytest.mark.parametrize("call", ["write", "ragged", "read"])
@pytest.mark.parametrize("kw", ROWS_BAD, ids=str)
def test_row_calls_refuse_bad_arguments(bd, call, kw):
    f = {"write": _write, "ragged": lambda bd, **k: _write(bd, True, **k), "read": _read}[call]
    assert f(bd, **kw) == bd.ERR_INVALID_ARG


@pytest.mark.parametrize("call", ["write", "ragged", "read"])
@pytest.mark.parametrize("kw", ROWS_LARGE, ids=lambda k: str(sorted(k)))
def test_row_calls_refuse_what_they_do_not_cover(bd, call, kw):
    f = {"write": _write, "ragged": lambda bd, **k: _write(bd, True, **k), "read": _read}[call]
    assert f(bd, **kw) == bd.ERR_UNSUPPORTED


def test_row_calls_with_nothing_to_do(bd):
    none = dict(k=None, v=None, kc=None, ks=None, vc=None, vs=None)
    assert _write(bd, seq=0, **none) == bd.CIVIC_OK and _write(bd, batch=0, **none) == bd.CIVIC_OK and _read(bd, seq=0, **none) == bd.CIVIC_OK
    assert _write(bd, True, off=(0, 0, 0), **none) == bd.CIVIC_OK
    assert _write(bd, seq=-1) == bd.ERR_INVALID_ARG and _read(bd, seq=-1) == bd.ERR_INVALID_ARG
    assert _write(bd, cos=C.c_void_p(0x1008)) == bd.ERR_INVALID_ARG
    for off in (None, (1, 3, 6), (0, 4, 3), (0, 3, 68)):
        assert _write(bd, True, off=off) == bd.ERR_INVALID_ARG
    assert _write(bd, True, off=(0, 3, 3 + (1 << 27)), s_max=1 << 27, pos=FAKE) == bd.ERR_UNSUPPORTED
    many = (1 << 25) + 1                                                                     # tokens, all but a few outside the cache
    assert _write(bd, seq=many, pos=FAKE) == bd.ERR_UNSUPPORTED and _read(bd, seq=many, pos=FAKE) == bd.ERR_UNSUPPORTED
    assert _write(bd, True, off=(0, 3, 3 + many), pos=FAKE) == bd.ERR_UNSUPPORTED


def _attn(bd, decode=False, **kw):
    a = dict(q=FAKE, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, out=FAKE, dtype=1, fmt=4, batch=2, seq=5, hq=8, hkv=2, d=128, qs=(5120, 1024, 128),
             os=(5120, 1024, 128), s_max=4096, n_ctx=4096, ctx=None, causal=1, scale=0.0, ws=None, ws_bytes=0)
    a.update(kw)
    qs, os_ = ((C.c_int64 * 3)(*a[x]) if a[x] else None for x in ("qs", "os"))
    head = [a["q"], a["kc"], a["ks"], a["vc"], a["vs"], a["out"], a["dtype"], a["fmt"], a["batch"]]
    tail = [C.c_float(a["scale"]), a["ws"], a["ws_bytes"], None]
    if decode:
        return bd.lib.civic_decode_attn_mx(*head, a["hq"], a["hkv"], a["d"], a["s_max"], a["n_ctx"], a["ctx"], *tail)
    return bd.lib.civic_prefill_attn_mx(*head, a["seq"], a["hq"], a["hkv"], a["d"], qs, os_, a["s_max"], a["n_ctx"], a["ctx"], a["causal"], *tail)


ATTN_BAD = [dict(q=None), dict(out=None), dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None), dict(dtype=7), dict(fmt=5), dict(batch=-1),
            dict(hq=0), dict(hkv=0), dict(hq=7), dict(d=0), dict(d=80), dict(s_max=4100), dict(s_max=2048), dict(n_ctx=-1),
            dict(scale=float("nan")), dict(scale=float("inf")), dict(q=C.c_void_p(0x1008)), dict(ks=C.c_void_p(0x1002)),
            dict(out=C.c_void_p(0x1004)), dict(ctx=C.c_void_p(0x1001)), dict(ws=C.c_void_p(0x1004), ws_bytes=1 << 30)]


@pytest.mark.parametrize("decode", [True, False], ids=["decode", "prefill"])
@pytest.mark.parametrize("kw", ATTN_BAD, ids=str)
def test_attention_refuses_bad_arguments(bd, decode, kw):
    assert _attn(bd, decode, **kw) == bd.ERR_INVALID_ARG


def test_attention_refuses_bad_strides_and_what_it_does_not_cover(bd):
    for kw in (dict(qs=None), dict(os=None), dict(seq=-1), dict(qs=(5120, 1024, 64)), dict(os=(5120, 1024, 64)), dict(qs=(5120, 1028, 128)),
               dict(os=(-5120, 1024, 128))):
        assert _attn(bd, **kw) == bd.ERR_INVALID_ARG, kw
    for kw in (dict(d=288, qs=(11520, 2304, 288), os=(11520, 2304, 288)), dict(batch=65536), dict(s_max=(1 << 22) + 32), dict(seq=1 << 20)):
        assert _attn(bd, **kw) == bd.ERR_UNSUPPORTED, kw
    for kw in (dict(batch=0), dict(seq=0)):
        assert _attn(bd, q=None, out=None, **kw) == bd.CIVIC_OK


def test_attention_refuses_a_missing_workspace(bd):
    for decode, seq in ((True, 1), (False, 5)):
        need = bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 4, 2, seq, 8, 2, 128, 4096)
        assert need > 0
        assert _attn(bd, decode) == bd.ERR_WORKSPACE and _attn(bd, decode, ws=FAKE, ws_bytes=need - 1) == bd.ERR_WORKSPACE
    assert bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 4, 0, 1, 8, 2, 128, 4096) == 0
    assert bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 5, 2, 1, 8, 2, 128, 4096) == 0
    # more context, batch or heads never takes a size that overflows
    for b, n in itertools.product((1, 1000, 65535), (1, 100, 1 << 22)):
        assert 0 <= bd.civic_attn_mx_workspace_bytes(torch.float32, 8, b, 1, 64, 8, 256, n) < 1 << 40


def test_binding_refuses_what_does_not_fit(bd):
    cache = bd.civic_mx_cache(2, 4, 33, 64, 4, device="cpu")
    assert cache.k_codes.shape == (2, 4, 64, 32) and cache.k_scales.shape == (2, 4, 64, 2)
    for bad in (dict(format=5), dict(head_dim=48)):
        with pytest.raises(ValueError):
            bd.civic_mx_cache(**dict(dict(batch=1, n_kv_heads=1, rows=1, head_dim=64, format=4, device="cpu"), **bad))
    k = torch.zeros(2, 3, 4, 64)
    for cache2, k2, v2, kw in ((cache, k, k[:, :2], {}), (cache, k.double(), k, {}), (cache, torch.zeros(2, 3, 4, 32), torch.zeros(2, 3, 4, 32), {}),
                               (cache, k, k, dict(cos_sin=torch.zeros(2, 3, 31, 2))), (cache, k, k, {})):   # the last: not on a device
        with pytest.raises((ValueError, TypeError)):
            bd.civic_kv_write_mx(k2, v2, cache2, **kw)
    for kw in (dict(format=8), dict(k_codes=cache.k_codes.float()), dict(v_scales=cache.v_scales[:1]), dict(k_scales=cache.k_scales.transpose(0, 1))):
        with pytest.raises(ValueError):
            cache._replace(**kw)
    with pytest.raises(ValueError):
        bd.civic_decode_attn_mx(torch.zeros(2, 8, 32), cache, 5)
    with pytest.raises(ValueError):
        bd.civic_prefill_attn_mx(torch.zeros(3, 1, 8, 64), cache, 5)
