"""Sums of the 8-bit product keep fp32's 24 bits, whatever the output's type (needs an MI355X).

Inputs are chosen so that a sum in fewer bits shows through the rounding to bf16 behind it: large terms that cancel beside
small ones that are left.
"""
import pytest
import torch

import fp8_plain as F
from paper_2509_15965_amd import rl_decode as R
from test_gpu_fp8 import BF, DEV, F32, gen, room

pytestmark = pytest.mark.gpu


def cancelling(m, n, k, seed):
    """Codes of a [m][k] and w [n][k] whose large products, 2^16 each, cancel in pairs half a block apart and leave a sum of
    products of -9 .. 9: every partial sum is a whole number, at most 2^16 k / 8 + 9 k, below 2^24 for k = 1920 and less."""
    g = gen(seed)
    half = lambda rows: torch.randint(-3, 4, (rows, k // 128, 2, 64), generator=g, device=DEV).float()
    a, w = half(m), half(n)
    big = torch.randperm(64, generator=g, device=DEV)[:16]                   # of 64 places, in all rows
    sign = torch.randint(0, 2, (m, k // 128, 16), generator=g, device=DEV).float() * 512 - 256
    a[:, :, 0, big], a[:, :, 1, big] = sign, -sign
    w[:, :, :, big] = 256.0
    return a.view(m, k), w.view(n, k)


@pytest.mark.parametrize("m,n,k", [(1, 300, 896), (20, 1000, 1920), (33, 300, 896), (64, 129, 1024), (130, 700, 384), (300, 260, 1920), (512, 4608, 1024),
                                   (700, 9300, 256), (2100, 4301, 128), (40, 66000, 384)])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_products_beside_larger_ones_that_cancel(m, n, k, dtype):
    """Every sum is exact in fp32, so the output is the whole number that is left, rounded once."""
    a, w = cancelling(m, n, k, m + n)
    A, W = room(m, k), room(n, k, True)
    R.quantise(a, *A)
    R.quantise(w, *W, form="tiles")
    assert torch.equal(F.matrix(*A), a.double()) and torch.equal(F.matrix(*W, True), w.double())
    out = torch.empty(m, n, dtype=dtype, device=DEV)
    R.gemm_quant(*A, *W, out)
    want = a.double() @ w.double().t()
    assert torch.equal(out, want.to(dtype)), (out.double() - want).abs().max()
