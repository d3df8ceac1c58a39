"""Log-probabilities, their gradient and the policy loss from logits far from
ordinary ranges: small temperatures and large logits (needs an MI355X).

Tolerances as in test_gpu_losses.py.  The forms here take the difference to
the row's largest logit before dividing by the temperature: ln n is lost next
to 1e10.
"""
import math

import pytest
import torch

from paper_2509_15965_amd import rl_decode as R
from test_gpu_losses import BF, DEV, F32, U, forward, gen, gradient, gradient_tol, near, rel

pytestmark = pytest.mark.gpu


def formula(z, y, T):
    """log p, log-probabilities of y and entropies in 64 bits."""
    z = z.double()
    t = (z - z.max(1, keepdim=True).values) / T
    q = t - t.exp().sum(1, keepdim=True).log()
    return q, q.gather(1, y.long()[:, None])[:, 0], torch.special.entr(q.exp()).sum(1)


FAR = [1e6, 3e7, 1e8, 1e9, 4e9, 1e10, 1e12, 1e20, 1e30, 1e35, 1e37, 1e38]


def far_rows(V, dtype, seed):
    """Rows of +-v alone, of v and values a few of the type's steps below, and of ordinary values with v at two places."""
    g = gen(seed)
    randn = lambda: torch.randn(V, generator=g, device=DEV)
    step = torch.finfo(dtype).eps
    rows = []
    for v in FAR:
        rows += [torch.full((V,), v, device=DEV), torch.full((V,), -v, device=DEV)]
        rows.append(-v * (1 + step * torch.randint(0, 4, (V,), generator=g, device=DEV).float()))
        r = 3 * randn()
        r[torch.randint(0, V, (2,), generator=g, device=DEV)] = v
        rows.append(r)
    return torch.stack(rows).to(dtype).clamp(torch.finfo(dtype).min, torch.finfo(dtype).max)


CASES = [("rows", T) for T in (1.0, 0.7)] + [("ordinary", T) for T in (1e-6, 1e-7, 1e-8, 3e-9, 1e-9, 1e-12, 1e-30, 1e30)]


def inputs(kind, V, dtype, seed):
    z = far_rows(V, dtype, seed) if kind == "rows" else (3 * torch.randn(40, V, generator=gen(seed), device=DEV)).to(dtype)
    y = torch.randint(0, V, (z.shape[0],), generator=gen(seed + 1), device=DEV, dtype=torch.int32)
    y[::2] = z[::2].float().argmax(1).int()
    return z, y


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [9, 5000, 70001])
@pytest.mark.parametrize("kind,T", CASES)
def test_logprobs(kind, T, V, dtype):
    z, y = inputs(kind, V, dtype, V)
    q, want, H = formula(z, y, T)
    lp, ent, st = forward(z, y, T)
    near(lp, want, 4 * rel(V), 2 * U)
    near(ent, H, 6 * rel(V) * (1 + math.log(V)), 2 * U)
    only, _, _ = forward(z, y, T, entropy=False)
    near(only, want, 4 * rel(V), 2 * U)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [9, 5000, 70001])
def test_entries_far_below_a_row(V, dtype):
    """Ordinary rows some of whose entries are masked by a large negative number, 10^9 to 10^11."""
    n = 100
    z, y = inputs("ordinary", V, dtype, 5)
    z = z.repeat(3, 1)[:n]
    mask = torch.rand(n, V, generator=gen(6), device=DEV) < 0.4
    mask[:, V // 2] = False
    z = torch.where(mask, -torch.logspace(9, 11, n, device=DEV)[:, None].to(dtype), z)
    y = torch.full((n,), V // 2, device=DEV, dtype=torch.int32)
    q, want, H = formula(z, y, 1.0)
    for entropy in (True, False):
        lp, ent, st = forward(z, y, 1.0, entropy)
        near(lp, want, 4 * rel(V), 2 * U)
        if entropy:
            near(ent, H, 6 * rel(V) * (1 + math.log(V)), 2 * U)


def check_gradient(dz, q, H, y, g, ge, T, dtype, V, more=0.0):
    """`more`: what the caller allows g to be off, relative."""
    err, step = gradient_tol(q, H, g, ge, T, dtype, V)
    if ge is not None:      # the entropy's own error is in the formula
        err = err + q.exp() * (ge.double().abs() / T * 6 * rel(V) * (1 + math.log(V)))[:, None]
    near(dz, gradient(q, H, y, g, ge, T), err + (g.double().abs() / T * 2 * U)[:, None], step + 4 * U + more)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [9, 5000, 70001])
@pytest.mark.parametrize("kind,T", CASES)
def test_gradient(kind, T, V, dtype):
    z, y = inputs(kind, V, dtype, V)
    n = z.shape[0]
    q, _, H = formula(z, y, T)
    _, ent, st = forward(z, y, T)
    g, ge = torch.randn(n, generator=gen(1), device=DEV), torch.randn(n, generator=gen(2), device=DEV)
    for e in (ge, None):
        dz = torch.full_like(z, 9.0)
        R.token_logprobs_backward(z, y, st, g, dz, entropy=None if e is None else ent, d_entropy=e, temperature=T)
        assert dz.isfinite().all()
        check_gradient(dz, q, H, y, g, e, T, dtype, V)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [9, 5000, 70001])      # rows in registers, and (70001) cut over the chip
@pytest.mark.parametrize("kind,T", CASES)
def test_policy_loss_from_logits(kind, T, V, dtype):
    z, _ = inputs(kind, V, dtype, V)
    n = z.shape[0]
    y = z.float().argmax(1).int()
    q, lp, H = formula(z, y, T)
    old = (lp + 0.3 * torch.randn(n, generator=gen(3), device=DEV)).float()
    adv = torch.randn(n, generator=gen(4), device=DEV)
    for coef in (0.0, 0.02):
        out, olp, ent = torch.empty(8, device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        dz = torch.full_like(z, 9.0)
        R.policy_loss_logits(z, y, old, adv, out, olp, dz, out_entropy=ent, token_advantages=True, aggregate="sum",
                             clip_low=0.9, clip_high=20.0, entropy_coef=coef, temperature=T)
        assert out.isfinite().all() and dz.isfinite().all()
        near(olp, lp, 4 * rel(V), 2 * U)
        g = -adv.double() * (lp - old.double()).exp()
        # the log-probability in the ratio is within 4 rel(V)
        check_gradient(dz, q, H, y, g, torch.full_like(g, -coef) if coef else None, T, dtype, V, 4 * rel(V))
