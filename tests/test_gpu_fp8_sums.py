"""Sums of the 8-bit product and of the attention over the 8-bit cache keep fp32's 24 bits, whatever the output's type (needs an
MI355X).

Inputs are chosen so that a sum in fewer bits shows through the rounding to bf16 behind it: large terms that cancel beside
small ones that are left.
"""
import pytest
import torch

import fp8_plain as F
from paper_2509_15965_amd import rl_decode as R
from test_gpu_fp8 import BF, DEV, F32, U, Cache, attend, gen, packed, room

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


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d,page", [(64, 32), (128, 64)])
def test_softmax_weights_keep_24_bits(dtype, d, page):
    """Three positions, of scores 0, -s and -s + r 2^-12 (s < 1/2; exact sums of exact products) and values 0, v and -v: the
    output is v (p1 - p2) / (1 + p1 + p2), and its terms' sum is 2^11 times as large and more.

    Error of that sum, relative to it: a score times log2(e), less than 0.73, is off by two roundings (2 u of it), the difference
    to the largest, 0, by none, the exponential by 2 u: 4 u in all.  A weight split into three bf16 numbers loses 2^-27 of it.
    Their products with v are exact and are added in three instructions of two terms, 2 u (a cut instead of a rounding) a term:
    12 u.  What follows is relative to the small output: sum of weights, division and rounding to the type."""
    n, heads, group = 96, 2, 4
    g = gen(3)
    c = Cache([3] * n, page, heads, d, 1)
    seqs, pos = packed([3] * n, [0] * n)
    k, v = (torch.zeros(3 * n, heads, d, device=DEV) for _ in range(2))
    k[pos > 0, :, 0] = -1.0
    k[pos == 2, :, 1] = 1.0
    x = torch.randint(8, 16, (n, heads, d), generator=g, device=DEV).float()
    v[pos == 1], v[pos == 2] = x, -x
    c.append(seqs, pos, k, v)
    q = torch.zeros(n, heads * group, d, device=DEV)
    q[..., 0] = torch.randint(8, 128, q.shape[:2], generator=g, device=DEV) / 256.0
    q[..., 1] = torch.randint(1, 4, q.shape[:2], generator=g, device=DEV) / 4096.0
    q = q.to(dtype)
    o = attend(c, q, [3] * n, scale=1.0)
    step = U if dtype == F32 else 2.0 ** -8
    worst = 0.0
    for i in range(n):
        want, size, _ = F.attention(q[i], *c.numbers(i, 3), 1.0)
        assert (want.abs() * 256 <= size).all() and (want.abs() > 0).all()
        tol = (4 + 12 + 0.125) * U * size + (8 * U + step) * want.abs()
        worst = max(worst, ((o[i].double() - want).abs() / tol).max().item())
    assert worst <= 1.0, worst
