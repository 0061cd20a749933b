"""Strides that a cache in 8 bits may have and one in bf16 may not: the workspace's size is that of any other strides."""
import pytest

from paper_2604_05438_amd import binding as B


def config(stride_tok, kv_dtype=B.TKPHI_BF16):
    return B.tkphi_paged_config(8, 2, 64, kv_dtype, 0.125, 32, 32 * stride_tok, 64, stride_tok, 0, 64, 0, 16, 1, 2, 8, 0)


STEP = B.tkphi_step(4096, 4096, 3, 10, 20, 12, 300, 0)


@pytest.mark.parametrize("stride", [128, (1 << 27) - 16, 1 << 27, (1 << 28) - 16])
def test_tokens_far_apart(stride):
    size = B.tkphi_paged_workspace_bytes(config(128), STEP)
    assert size > 0 and B.tkphi_paged_workspace_bytes(config(stride), STEP) == size, B.tkphi_last_error()
    pool, rows = B.tkphi_quant_pool(4096, 8192, 12288, 16384, 40, 0), B.tkphi_attention_rows(4096, 8192, 4096, 512, 64, 512, 64)
    # the call takes the config too: what it refuses is a workspace that is a byte short
    assert B.lib().tkphi_quant_block_attention(config(stride), STEP, pool, rows, 4096, size - 1, None) == B.TKPHI_EWORKSPACE


def test_refused_by_both():
    assert B.tkphi_paged_workspace_bytes(config(1 << 28), STEP) == 0 and "stride_tok" in B.tkphi_last_error()
    assert B.tkphi_paged_workspace_bytes(config(1 << 27, B.TKPHI_F32), STEP) == 0 and "stride_tok" in B.tkphi_last_error()
    assert B.tkphi_paged_workspace_bytes(config(120), STEP) == B.tkphi_paged_workspace_bytes(config(128), STEP)      # (bf16 rows of 240 bytes)
    assert B.tkphi_paged_workspace_bytes(config(124), STEP) == 0 and "stride" in B.tkphi_last_error()
    pool, rows = B.tkphi_kv_pool(4096, 8192, 16384, 40, 0), B.tkphi_attention_rows(4096, 8192, 4096, 512, 64, 512, 64)
    assert B.lib().tkphi_block_attention(config(1 << 27), STEP, pool, rows, 4096, 1 << 40, None) == B.TKPHI_ESHAPE
