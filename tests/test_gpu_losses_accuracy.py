"""How near log-probabilities, entropies and the loss from logits come to 64
bits over many rows (needs an MI355X).

Limits.  log p = (z_y - max) / T - ln s is worked out in 64 bits from an fp32
sum s and rounded to fp32.
- Rounding: half a step at most, step / sqrt(12) in the mean square.
- ln s: an exponential is within one step, 2^-23, were they all off the same
  way.  Their arguments (half a step of |t| < 32, weighted by the
  probability) and a lane's some 80 additions (2.9 u in the mean square) are
  independent from entry to entry and from lane to lane: less than as much
  again.  2^-22 bounds the mean and the mean square.
- The mean over n rows of what has no sign adds four standard errors.
- Without entropies, the correction for the rounding of log2(e) / T (6e-8 of
  it at most) takes a lane's entries for its largest: 1.5 nats too high for
  593 values of N(0, 1/2), under 1e-7.
- Entropies are ln s - ln 2 u / s, with u a sum of entries times exponents t
  relative to a reference d off the largest: |t| + |d| stay under 46 = 32 /
  ln 2 here, and a few roundings of 2^-24 each, half of them the same way:
  32 x 2^-23 = 2^-18.
"""
import math

import pytest
import torch

from paper_2509_15965_amd import rl_decode as R
from test_gpu_losses import BF, DEV, F32, U, forward, gen, near

pytestmark = pytest.mark.gpu

# log2(e) / T lies nearly half a step above 1, where rounding it to fp32 moves it the most
BENT = 1.4426950408889634 / (1.0 + 0.98 * 2.0 ** -24)


def formula(z, y, T):
    """log p of y and entropies in 64 bits, some rows at a time."""
    lp, H = torch.empty(z.shape[0], dtype=torch.double, device=DEV), torch.empty(z.shape[0], dtype=torch.double, device=DEV)
    for a in range(0, z.shape[0], 128):
        x = z[a:a + 128].double() / T
        q = x - torch.logsumexp(x, 1, keepdim=True)
        lp[a:a + 128] = q.gather(1, y[a:a + 128].long()[:, None])[:, 0]
        H[a:a + 128] = torch.special.entr(q.exp()).sum(1)
    return lp, H


def step_of(x):
    """The fp32 step at x."""
    return torch.exp2(torch.floor(torch.log2(x.abs())) - 23)


def values(path, z, y, T):
    """Log-probabilities and entropies by the forward kernel, cut over the chip, or by the loss from logits."""
    n = z.shape[0]
    if path == "forward":
        return forward(z, y, T)[:2]
    if path == "no entropy":
        return forward(z, y, T, entropy=False)[0], None
    if path == "cut":
        parts = [forward(z[a:a + 100], y[a:a + 100], T)[:2] for a in range(0, n, 100)]
        return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
    f = lambda *s: torch.empty(*s, device=DEV)
    out, lp, ent, dz = f(8), f(n), f(n), torch.empty_like(z)
    R.policy_loss_logits(z, y, torch.zeros(n, device=DEV), torch.ones(1, device=DEV), out, lp, dz, out_entropy=ent, temperature=T)
    return lp, ent


PATHS = [("forward", BF, 1024, 152064), ("forward", F32, 1024, 80000), ("forward", BF, 2048, 32000), ("no entropy", BF, 1024, 152064),
         ("no entropy", F32, 1024, 80000), ("cut", BF, 800, 152064), ("loss", BF, 1024, 152064), ("loss", F32, 1024, 80000),
         ("loss", BF, 2048, 32000), ("loss", BF, 600, 170001)]


@pytest.mark.parametrize("path,dtype,n,V", PATHS)
@pytest.mark.parametrize("T", [1.0, 0.6, BENT])
def test_logprobs_over_many_rows(path, dtype, n, V, T):
    g = gen(V + n)
    z = torch.randn(n, V, generator=g, device=DEV)
    y = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    if T == BENT:          # entries some 10 nats below the largest hold most of the probability
        z *= 0.5
        z.scatter_(1, torch.randint(0, V, (n, 1), generator=g, device=DEV), 10.0 + torch.rand(n, 1, generator=g, device=DEV))
    else:
        z *= 3.0
    z = z.to(dtype)
    want, H = formula(z, y, T)
    lp, ent = values(path, z, y, T)
    d = lp.double() - want
    square = float((step_of(want) ** 2).mean() / 12)
    mean, rms = float(d.mean()), math.sqrt(float((d * d).mean()))
    ln_s = 2.0 ** -22
    print(f"{path} {dtype} {n} x {V}, T = {T:.6g}: mean {mean:.3g}, mean square {rms:.3g}, rounding alone {math.sqrt(square):.3g}")
    assert abs(mean) <= ln_s + 4 * math.sqrt((square + ln_s ** 2) / n)
    assert rms <= math.sqrt(square + ln_s ** 2) * (1 + 4 / math.sqrt(2 * n))
    if ent is not None:
        e = ent.double() - H
        print(f"   entropies: mean {float(e.mean()):.3g}, mean square {math.sqrt(float((e * e).mean())):.3g}")
        assert math.sqrt(float((e * e).mean())) <= 2.0 ** -18


# rows in registers, and the three kernels: one row alone, and one that counts among many
@pytest.mark.parametrize("n,V,dtype", [(1, 4096, F32), (1, 70001, BF), (1, 170001, F32), (200, 152064, BF), (200, 32000, F32)])
def test_loss_is_of_logprobs_before_rounding(n, V, dtype):
    """Tokens of log p near -100, where an fp32 step is 7.6e-6: the ratio to a log-probability of fp32 is within what ln s is
    off (2^-22, twice for one row), and the loss is rounded once."""
    T = 0.7
    for seed in range(12):
        g = gen(seed)
        z = (3 * torch.randn(n, V, generator=g, device=DEV))
        at = n // 2
        y = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
        z[at, y[at].long()] = -50.0 - seed
        z = z.to(dtype)
        mask = torch.zeros(n, device=DEV, dtype=torch.bool)
        mask[at] = True
        lp, _ = formula(z[at:at + 1], y[at:at + 1], T)
        assert 64 < -lp < 128
        old = torch.full((n,), float(lp.float()), device=DEV)
        out, olp, dz = torch.empty(8, device=DEV), torch.empty(n, device=DEV), torch.empty_like(z)
        R.policy_loss_logits(z, y, old, torch.ones(1, device=DEV), out, olp, dz, mask=mask, temperature=T)
        ratio = (lp - old[at].double()).exp()
        near(-out[0], ratio[0], 2.0 ** -21, 2 * U)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,V", [(3, 4000), (300, 32000), (20, 70001), (100, 100003)])
def test_tokens_that_are_nearly_certain(n, V, dtype):
    """The target 25 to 40 nats above its neighbours and far behind a lane's first entries, so that the lane's sum is relative
    to one of those: its own term is 2^t 2^-t, each within a step of 2^-23, and two roundings; the others sum to at most
    V e^-25 (below 1.5e-6)."""
    g = gen(n)
    z = torch.rand(n, V, generator=g, device=DEV)
    y = torch.randint(V - 200, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    z.scatter_(1, y.long()[:, None], 26.0 + 14 * torch.rand(n, 1, generator=g, device=DEV))
    z = z.to(dtype)
    want, _ = formula(z, y, 1.0)
    off = 4 * 2.0 ** -23
    lp, ent, st = forward(z, y, 1.0)
    near(lp, want, off)
    d = torch.randn(n, generator=g, device=DEV)
    dz = torch.empty_like(z)
    R.token_logprobs_backward(z, y, st, d, dz)
    own = dz.gather(1, y.long()[:, None])[:, 0]
    true = -d.double() * torch.expm1(want)
    near(own, true, d.abs().double() * off, 2.0 ** -8 if dtype == BF else 2 * U)
    out, olp = torch.empty(8, device=DEV), torch.empty(n, device=DEV)
    R.policy_loss_logits(z, y, want.float(), d, out, olp, dz, token_advantages=True, aggregate="sum")
    near(olp, want, off)
    own = dz.gather(1, y.long()[:, None])[:, 0]
    near(own, true * -1, d.abs().double() * (off * 1.01), 2.0 ** -8 if dtype == BF else 4 * U)
