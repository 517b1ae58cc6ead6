"""Host side of the calls on a cache in 8 or 4 bits: workspace sizes and argument conversion (no call reaches the GPU)."""
import ctypes as C

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def bd():
    from paper_2605_28115_amd import binding
    return binding


# ---------------------------------------------------------------------------------------------------------- workspaces
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("sizes", [
    # batch, tokens, H_q, H_kv, head_dim
    (4, 1, 32, 8, 128), (1, 1, 16, 8, 128), (1, 1, 4, 2, 64), (16, 5, 16, 8, 128), (3, 5, 16, 4, 256), (1, 5, 28, 4, 128), (1, 10, 28, 4, 128),
    (4, 128, 32, 8, 128), (1, 1024, 28, 4, 128), (1, 300, 4, 1, 64), (2, 40, 16, 2, 96), (1, 60, 8, 2, 256), (8, 512, 32, 8, 128),
], ids=str)
def test_a_workspace_for_a_context_serves_the_shorter_ones(bd, dtype, sizes):
    """The bytes never fall with n_ctx: around every multiple of the steps of 64 and 128 rows, and at a cache's size."""
    b, seq, hq, hkv, d = sizes
    around = sorted({max(m + k, 0) for m in range(0, 20000, 64) for k in (-1, 0, 1)} | {1 << 16, 100000, 1 << 20, 1 << 22})
    for fmt in (4, 8):
        last = 0
        for n in around:
            need = bd.civic_attn_mx_workspace_bytes(dtype, fmt, b, seq, hq, hkv, d, n)
            assert need >= last, n
            last = need


def test_a_workspace_for_no_context_is_none(bd):
    for seq in (1, 5, 200):
        assert bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 4, 2, seq, 8, 2, 128, 0) == 0
        assert bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 4, 2, seq, 8, 2, 128, 31) == 0


# ----------------------------------------------------------------------------------------------------------- arguments
def test_numbers_of_numpy_and_torch_are_taken_as_the_other_calls_take_them(bd, monkeypatch):
    """Lengths, positions and scales as a program computes them; the batch is empty, so that nothing is launched."""
    monkeypatch.setattr(bd, "_mx_placed", lambda *a: None)
    monkeypatch.setattr(bd, "_stream", lambda stream: 0)
    cache = bd.civic_mx_cache(0, 2, 64, 64, 8, device="cpu")
    k, q = torch.zeros(0, 3, 2, 64), torch.zeros(0, 3, 4, 64)
    for n, scale in ((np.int64(5), np.float32(0.5)), (np.int32(5), np.float64(0.5)), (torch.tensor(5), torch.tensor(0.5)), (5, 1)):
        bd.civic_kv_write_mx(k, k, cache, n)
        bd.civic_kv_read_mx(cache, k, k, n)
        bd.civic_kv_write_mx_ragged(torch.zeros(0, 2, 64), torch.zeros(0, 2, 64), cache, [0], n)
        assert bd.civic_decode_attn_mx(q[:, 0], cache, n, softmax_scale=scale).shape == (0, 4, 64)
        assert bd.civic_prefill_attn_mx(q, cache, n, softmax_scale=scale).shape == q.shape
        assert bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 8, n, n, n, n, 64, n) == bd.civic_attn_mx_workspace_bytes(torch.bfloat16, 8, 5, 5, 5, 5, 64, 5)
        assert bd.civic_decode_attn_workspace_bytes(torch.bfloat16, n, n, n, 64, n) == bd.civic_decode_attn_workspace_bytes(torch.bfloat16, 5, 5, 5, 64, 5)


FAKE = C.c_void_p(0x1000)


def read_into(bd, strides, batch=2, seq=5, hkv=8, d=128):
    return bd.lib.civic_kv_read_mx(FAKE, FAKE, FAKE, FAKE, 4, FAKE, FAKE, (C.c_int64 * 3)(*strides), 1, batch, seq, hkv, d, 64, 0, None, None)


def attend_into(bd, strides, batch=2, seq=5, hq=8, d=128):
    """With a workspace that is missing, so that what the strides do not refuse is refused behind them."""
    qs = (C.c_int64 * 3)(seq * hq * d, hq * d, d)
    return bd.lib.civic_prefill_attn_mx(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1, 4, batch, seq, hq, 2, d, qs, (C.c_int64 * 3)(*strides), 4096, 4096, None, 1,
                                        C.c_float(0.0), None, 0, None)


@pytest.mark.parametrize("strides", [(0, 1024, 128), (5120, 0, 128), (5120, 1024, 136), (1024, 1024, 128), (5120, 896, 128), (128, 1024, 128), (4096, 1024, 128),
                                     (2 ** 62, 2 ** 62, 128), (256, 512, 384)], ids=str)
def test_rows_that_are_written_lie_apart(bd, strides):
    assert read_into(bd, strides) == bd.ERR_INVALID_ARG and attend_into(bd, strides) == bd.ERR_INVALID_ARG


@pytest.mark.parametrize("strides", [(5120, 1024, 128), (8192, 1024, 128), (5120, 128, 640), (1024, 2048, 128), (128, 256, 1280), (10240, 2048, 136),
                                     (2 ** 40, 2 ** 30, 2 ** 20)], ids=str)
def test_rows_in_any_order_and_at_any_distance_are_taken(bd, strides):
    assert attend_into(bd, strides) == bd.ERR_WORKSPACE


def test_strides_of_axes_of_one_do_not_count(bd):
    assert attend_into(bd, (0, 1024, 128), batch=1) == bd.ERR_WORKSPACE
    assert attend_into(bd, (1024, 0, 128), seq=1) == bd.ERR_WORKSPACE


def test_a_workspace_of_repeated_memory_is_refused(bd, monkeypatch):
    """An expanded tensor has the bytes of all its elements and the memory of one."""
    monkeypatch.setattr(bd, "_mx_placed", lambda *a: None)
    monkeypatch.setattr(bd, "_stream", lambda stream: 0)
    cache, q = bd.civic_mx_cache(0, 2, 64, 64, 8, device="cpu"), torch.zeros(0, 3, 4, 64)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(64, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            bd.civic_prefill_attn_mx(q, cache, 64, workspace=ws)
        with pytest.raises(ValueError):
            bd.civic_decode_attn_mx(q[:, 0], cache, 64, workspace=ws)
