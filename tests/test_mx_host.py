"""Host side of the calls on a cache in 8 or 4 bits: workspace sizes and argument conversion (no call reaches the GPU)."""
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
