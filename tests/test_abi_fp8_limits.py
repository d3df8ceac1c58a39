"""Sizes at the limits of the 8-bit entry points, on the CPU.  No call here reaches the GPU."""
import pytest

from paper_2509_15965_amd import rl_decode as R
from test_abi_fp8 import gemm, quantise


@pytest.mark.parametrize("form", [0, 1, 2])
@pytest.mark.parametrize("dtype", [0, 1])
def test_quantise_refuses_blocks_whose_launch_cannot_be_counted(form, dtype):
    """617093 rows of 435 blocks are 2^28 - 1: 2^24 workgroups of 256 threads in fp32, one more than 32 bits count."""
    assert quantise(form=form, n=617093, k=435 * 128, dtype=dtype) == R.RL_ERR_UNSUPPORTED


@pytest.mark.parametrize("dt", [0, 1])
def test_product_refuses_tiles_whose_launch_cannot_be_counted(dt):
    """4096 x 4096 tiles and more, of 256 threads each."""
    for m, n in ((1 << 20, 1 << 20), (1 << 19, 1 << 19)):
        assert gemm(m=m, n=n, k=128, ldo=n, dt=dt) == R.RL_ERR_UNSUPPORTED


def test_cache_bytes_of_counts_past_32_bits():
    for bad in (((1 << 32) + 1, 32, 1, 64), (1, (1 << 32) + 32, 1, 64), (1, 32, (1 << 32) + 1, 64), (1, 32, 1, (1 << 32) + 64)):
        assert R.kv_quant_bytes(*bad) == 0, bad
    assert R.kv_quant_bytes(1, 32, 1, 64) == 4352
