"""The 8-bit operators at the far ends of their arguments (needs an MI355X)."""
import pytest
import torch

import fp8_plain as F
from paper_2509_15965_amd import rl_decode as R
from test_gpu_fp8 import BF, DEV, F32, INF, NAN, U, check_codes, check_outside, gen, room

pytestmark = pytest.mark.gpu


def far_gates():
    """(g, u): e^-g passes fp32 from |g| = 88.7 on, e^g is below its normal numbers from 87.3 on, and g e^g u is a normal one
    for the u given here."""
    return [(-80.5, 1.0), (-87.0, 1.0), (-87.5, -3.0), (-88.5, 1.0), (-89.0, 7.0), (-90.0, 1.0), (-90.0, 1e30), (-95.0, 1e10), (-100.0, -1e38), (-104.0, 1e20),
            (-120.0, 1e30), (-140.0, -3e38), (-150.0, 1e38), (-172.0, 3e38), (-174.5, 3e38), (-176.0, 3e38), (-178.0, -3e38)]


@pytest.mark.parametrize("dtype", [F32, BF])
def test_swiglu_of_gates_far_below_zero(dtype):
    """delta: the exponential's argument is within 1 u where it is split off a whole number (|f| <= 1/2), the exponential within two
    steps, 2 u each of its smallest; 1 + e^g, reciprocal (two steps) and the products: 6 u.  A row each, so that each has a scale of
    its own."""
    pairs = torch.tensor(far_gates(), device=DEV).to(dtype)
    codes, scales = room(len(pairs), 1)
    R.quantise(pairs, codes, scales, form="swiglu")
    g, u = pairs[:, :1].double(), pairs[:, 1:].double()
    v = g * torch.exp(g) / (1 + torch.exp(g)) * u
    assert (v.abs() > 2.0 ** -126).all()
    check_codes(codes, scales, v, 12 * U)
    check_outside(codes, scales, 1)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_swiglu_of_near_and_far_gates_in_a_row(dtype):
    """Rows whose gates lie on both sides of where the way of computing them changes; products of all sizes.  delta as above."""
    n, k = 40, 300
    r = gen(5)
    g = (torch.rand(n, k, generator=r, device=DEV) * 110 - 100).to(dtype)
    u = (torch.randn(n, k, generator=r, device=DEV) * 1e4 * torch.exp((-g.float()).clamp(min=0, max=70))).to(dtype)
    x = torch.cat([g, u], 1)
    codes, scales = room(n, k)
    R.quantise(x, codes, scales, form="swiglu")
    g, u = g.double(), u.double()
    check_codes(codes, scales, g * torch.sigmoid(g) * u, 12 * U)
    check_outside(codes, scales, k)


def test_swiglu_of_gates_without_a_finite_exponential():
    """A gate so low that g e^g u is below every code's step is 0; infinite and absent ones are NaN, as in the formula."""
    g = torch.tensor([-400.0, -1e30, -3e38, -400.0, -INF, -INF, NAN, -100.0, -100.0], device=DEV)
    u = torch.tensor([3e38, -3e38, 1.0, 0.0, 1.0, 0.0, 1.0, INF, NAN], device=DEV)
    codes, scales = room(9, 1)
    R.quantise(torch.stack([g, u], 1), codes, scales, form="swiglu")
    v = F.matrix(codes, scales)[:, 0]
    assert (v[:4] == 0).all() and (scales[:4, 0] == 127).all() and torch.isnan(v[4:]).all()


def test_binding_refuses_counts_past_32_bits():
    """Counts that C takes in 32 bits: none may come out as another."""
    pool = torch.zeros(R.kv_quant_bytes(2, 32, 2, 64), dtype=torch.uint8, device=DEV)
    table, ln = torch.zeros(1, 2, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    q = torch.zeros(1, 2, 64, device=DEV)
    call = lambda **kw: R.attention_quant(pool, table, q, ln, torch.empty_like(q), scale=1.0, **dict(dict(page_size=32, n_kv_heads=2, max_length=4), **kw))
    call()
    for more in (dict(max_length=(1 << 32) + 4), dict(max_length=-(1 << 32)), dict(page_size=(1 << 32) + 32), dict(n_kv_heads=(1 << 32) + 2)):
        with pytest.raises(ValueError):
            call(**more)
    with pytest.raises(ValueError):
        R.kv_quant_append(pool, table, ln, ln, q, q, page_size=(1 << 32) + 32)
