"""The preference loss of answers that hold a token of probability 0 (needs an MI355X)."""

import pytest
import torch

from paper_2509_15965_amd import rl_decode as R
from test_gpu_losses import DEV, U, gen, near

pytestmark = pytest.mark.gpu
INF = float("inf")


# one workgroup for all, a workgroup a pair, pairs cut over the chip
@pytest.mark.parametrize("pairs,each", [(3, 50), (40, 50), (2, 20000)])
@pytest.mark.parametrize("form", ["sigmoid", "hinge"])
@pytest.mark.parametrize("average", [False, True])
def test_answers_of_probability_0(pairs, each, form, average):
    """A log-probability of -inf in a rejected answer makes its margin inf: loss and gradient of the pair are 0 without
    label smoothing.  In a chosen one the loss is inf, and the gradient -beta (1 - s) / pairs."""
    n, beta = 2 * pairs * each, 0.5
    offs = torch.arange(0, n + 1, each, device=DEV, dtype=torch.int32)
    lp = -4 * torch.rand(n, generator=gen(pairs), device=DEV) / each
    plain = [(lp.double().view(2 * pairs, each)[i].sum() / (each if average else 1)) * beta for i in range(2 * pairs)]
    h = torch.stack([plain[2 * i] - plain[2 * i + 1] for i in range(pairs)])
    d = -torch.sigmoid(-h) if form == "sigmoid" else -(h < 1).double()
    loss = torch.nn.functional.softplus(-h) if form == "sigmoid" else (1 - h).clamp(min=0)
    per = beta / pairs / (each if average else 1)

    def run(lp, **more):
        out, g, rew = torch.empty(8, device=DEV), torch.empty(n, device=DEV), torch.empty(2 * pairs, device=DEV)
        R.preference_loss(lp, offs, out, g, out_rewards=rew, beta=beta, form=form, average=average, **more)
        return out, g.view(pairs, 2, each), rew

    rejected = lp.clone()
    rejected[each + each // 2] = -INF                 # pair 0's
    out, g, rew = run(rejected)
    near(out[0], loss[1:].sum() / pairs, 1e-12, 2 * U)
    assert not g[0].any() and rew[1] == -INF and out[2] == -INF and out[3] == INF
    near(g[1:, 0], (d[1:] * per)[:, None].expand(-1, each), 1e-13, 2 * U)
    near(g[1:, 1], (-d[1:] * per)[:, None].expand(-1, each), 1e-13, 2 * U)
    chosen = lp.clone()
    chosen[each // 2] = -INF
    out, g, rew = run(chosen)
    assert out[0] == INF and rew[0] == -INF
    near(g[0, 0], torch.full((each,), -per, device=DEV), 0.0, 2 * U)
    near(g[0, 1], torch.full((each,), per, device=DEV), 0.0, 2 * U)
    if form == "sigmoid":
        s = 0.25
        out, g, rew = run(rejected, label_smoothing=s)
        assert out[0] == INF
        near(g[0, 0], torch.full((each,), s * per, device=DEV), 0.0, 2 * U)
        out, g, rew = run(chosen, label_smoothing=s)
        assert out[0] == INF
        near(g[0, 0], torch.full((each,), -(1 - s) * per, device=DEV), 0.0, 2 * U)
