"""Sizes that the block norms and the 4-bit calls refuse before they look at a pointer."""
import pytest

from paper_2605_11005_amd import binding as B

EUNSUPPORTED = 2


def call(name, *args):
    return getattr(B.load_library(), name)(*args)


@pytest.mark.parametrize("batch,n,K", [(1, 0x7FFFFE10, 32), (1, 16, 0x7FFFFE20), (1 << 20, 1 << 20, 512), (1, 16, 48), (1 << 30, 16, 1024)])
def test_tiles_beyond_32_bits(batch, n, K):
    assert call("moe_mx4_quantize", None, B.MOE_BF16, batch, n, K, 0, None, None, None) == EUNSUPPORTED
    assert call("moe_mx4_quantize", None, B.MOE_BF16, batch, K, n, 1, None, None, None) == EUNSUPPORTED
    assert call("moe_mx4_dequantize", None, None, batch, n, K, None, B.MOE_F32, None) == EUNSUPPORTED


def test_rows_near_the_end_of_32_bits():
    T = 0x7FFF0001
    assert call("moe_block_norm_fwd", None, None, None, 0, None, None, B.MOE_BF16, B.MOE_BF16, T, 64, 1.0, 1.0, 1e-5, None, None, None, None, None) == EUNSUPPORTED
    assert call("moe_block_norm_bwd", None, None, None, 0, None, None, None, None, None, None, B.MOE_BF16, B.MOE_BF16, T, 64, 1.0, 1.0, None, None, None,
                None, None, 0, None, 0, None) == EUNSUPPORTED


def test_the_norms_workspace_grows_with_the_rows():
    for d in (8, 512, 1024, 2048, 8192, 16384):
        sizes = [B.moe_workspace_bytes(B.WS_BLOCK_NORM, 0, T, 0, d, 0, 0, 0) for T in (0, 1, 5, 511, 512, 513, 2048, 4096, 8191, 8192, 1 << 20)]
        assert sizes == sorted(sizes)
