"""Token log-probabilities, the policy loss and the preference loss against
plain 64-bit forms (needs an MI355X).

Tolerances.  u = 2^-24 is half a step of fp32.  A row's sum of k exponentials
in any order is within k u of itself and each exponential within
(|t| + 4) 2 u (its argument has two roundings, the hardware's exponential one
step), where e^-|t| |t| <= 0.37: REL(V) = (V / 64 + 64) u bounds the sum for
every split of a row over at least 64 lanes, join included.
"""
import math

import pytest
import torch

from paper_2509_15965_amd import rl_decode as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")


def rel(V):
    return (V / 64 + 64) * U


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def make(n, V, dtype, seed, pad=0, shift=0, spread=3.0):
    """Logits [n][V] in a buffer of rows V + pad that starts `shift` elements past 16 bytes, and targets."""
    g = gen(seed)
    buf = (torch.randn(n * (V + pad) + shift + 8, generator=g, device=DEV) * spread).to(dtype)
    z = buf[shift:shift + n * (V + pad)].view(n, V + pad)[:, :V]
    y = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    return z, y


def formula(z, y, T):
    """log p, log-probabilities and entropies in 64 bits."""
    x = z.double() / (T or 1.0)
    q = x - torch.logsumexp(x, 1, keepdim=True)
    p = q.exp()
    return q, q.gather(1, y.long().clamp(0, z.shape[1] - 1)[:, None])[:, 0], torch.special.entr(p).sum(1)


def gradient(q, H, y, g, ge, T):
    p = q.exp()
    d = -p * g.double()[:, None]
    d.scatter_add_(1, y.long()[:, None], g.double()[:, None])
    if ge is not None:
        d += ge.double()[:, None] * (torch.special.entr(p) - p * H[:, None])
    return d / (T or 1.0)


def gradient_tol(q, H, g, ge, T, dtype, V):
    """p's relative error is REL + (|q| + |t| + 8) 2 u, that of the factor the same; then one rounding to dtype."""
    p, a = q.exp(), q.clamp(min=-200).abs()
    f = g.double().abs()[:, None]
    if ge is not None:
        f = f + ge.double().abs()[:, None] * (a + H.abs()[:, None] + 1)
    err = p * f / (T or 1.0) * (2 * rel(V) + (4 * a + 16) * 2 * U)
    return err, 2.0 ** -8 if dtype == BF else 2 * U


def forward(z, y, T, entropy=True):
    n = z.shape[0]
    lp, ent, st = torch.full((n,), 7.0, device=DEV), torch.full((n,), 7.0, device=DEV), torch.full((n, 2), 7.0, device=DEV)
    R.token_logprobs(z, y, lp, out_entropy=ent if entropy else None, out_stats=st, temperature=T)
    return lp, ent, st


def near(got, want, atol, rtol=0.0):
    got, want = got.double(), want.double()
    tol = atol + rtol * want.abs() + 1e-37
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()), float(((got - want).abs() / tol).max()))


SHAPES = [(1, 1, 0, 0), (2, 2, 0, 0), (5, 3, 1, 1), (3, 7, 0, 0), (4, 8, 0, 0), (3, 63, 2, 3), (2, 257, 0, 1), (300, 1000, 0, 0),
          (17, 2047, 1, 0), (9, 2049, 0, 5), (6, 4096, 0, 0), (2, 50001, 0, 0), (1, 152064, 0, 0), (3, 151936, 8, 0),
          (1025, 2500, 3, 0)]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,V,pad,shift", SHAPES)
@pytest.mark.parametrize("T", [1.0, 0.6])
def test_logprobs_and_gradient(n, V, pad, shift, T, dtype):
    z, y = make(n, V, dtype, n * V + shift, pad, shift)
    q, want, H = formula(z, y, T)
    lp, ent, st = forward(z, y, T)
    near(lp, want, 4 * rel(V), 2 * U)
    assert (lp <= 0).all() and (ent >= 0).all()
    near(ent, H, 6 * rel(V) * (1 + math.log(V)), 2 * U)
    g = torch.randn(n, generator=gen(1), device=DEV)
    ge = torch.randn(n, generator=gen(2), device=DEV)
    if n > 2:
        g[1] = ge[1] = 0
    for e in (ge, None):
        store = torch.full((n, V + pad + 1), 5.0, device=DEV, dtype=dtype)
        dz = store[:, :V]
        R.token_logprobs_backward(z, y, st, g, dz, entropy=None if e is None else ent, d_entropy=e, temperature=T)
        err, step = gradient_tol(q, H, g, e, T, dtype, V)
        near(dz, gradient(q, H, y, g, e, T), err + (g.double().abs() / T * 2 * U)[:, None], step)
        assert (store[:, V:] == 5.0).all()          # entries behind a row stay
        if n > 2:
            assert not dz[1].any()
    # in place, and again: the same bits
    kept = dz.clone()
    z2 = z.clone() if pad == 0 and shift == 0 else torch.empty(n, V + 3, device=DEV, dtype=dtype)[:, :V].copy_(z)
    lp2, ent2, st2 = forward(z2, y, T)
    R.token_logprobs_backward(z2, y, st2, g, z2, temperature=T)
    if z2.stride(0) % 8 == z.stride(0) % 8:
        assert torch.equal(lp2, lp) and torch.equal(ent2, ent) and torch.equal(st2, st)
    near(z2, kept, 2 * err, step * 2)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [5, 1000, 40000])
def test_rows_that_are_not_ordinary(V, dtype):
    low = torch.finfo(dtype).min
    z, y = make(12, V, dtype, V)
    z[0] = -INF
    z[1] = -INF
    z[1, V // 2] = 3.0
    y[1] = V // 2
    z[2] = low                                   # a mask of the type's lowest value everywhere
    z[3, 1:] = low
    y[3] = 0
    z[4, V - 1] = INF
    z[5, 0] = NAN
    z[6] = 0.0
    y[7], y[8] = -1, V
    z[9] = -INF
    z[9, :2] = torch.tensor([1.0, 1.0], dtype=dtype)
    y[9] = V - 1                                 # a token that the distribution does not hold
    z[10, 0], z[10, 1] = -low, low               # the type's whole range in one row
    y[10] = 0
    z[11] *= 1000.0
    lp, ent, st = forward(z, y, 1.0)
    q, want, H = formula(z, y, 1.0)
    assert lp[[0, 4, 5, 7, 8]].isnan().all() and ent[[0, 4, 5]].isnan().all()
    for i in (1, 3, 10):
        assert lp[i] == 0 and ent[i] == 0, i
    for i in (2, 6):
        near(lp[i], torch.tensor(-math.log(V), device=DEV), 4 * rel(V), 2 * U)
        near(ent[i], torch.tensor(math.log(V), device=DEV), 6 * rel(V) * (1 + math.log(V)), 2 * U)
    assert lp[9] == -INF
    near(ent[9], torch.tensor(math.log(2.0), device=DEV), 6 * rel(V), 2 * U)
    near(lp[11], want[11], 4 * rel(V), 4 * U)    # |z| in the thousands: the difference to the largest is rounded
    near(ent[[7, 8, 11]], H[[7, 8, 11]], 6 * rel(V) * (1 + math.log(V)), 4 * U)
    g = torch.ones(12, device=DEV)
    ge = torch.full((12,), 0.5, device=DEV)
    dz = torch.full_like(z, 9.0)
    R.token_logprobs_backward(z, y, st, g, dz, entropy=ent, d_entropy=ge)
    assert dz[[0, 4, 5]].isnan().any(1).all()
    ok = [1, 2, 3, 6, 9, 10]
    assert dz[ok].isfinite().all() and not dz[1].any() and not dz[3].any() and not dz[10].any()
    near(dz[6], gradient(q[6:7], H[6:7], y[6:7], g[6:7], ge[6:7], 1.0)[0], 40 * rel(V) / V, 2.0 ** -8)
    # a target outside the vocabulary has no log-probability to differentiate
    qq = q[7:9]
    err, step = gradient_tol(qq, H[7:9], 0 * g[7:9], ge[7:9], 1.0, dtype, V)
    near(dz[7:9], gradient(qq, H[7:9], 0 * y[7:9], 0 * g[7:9], ge[7:9], 1.0), err, step)
    # rows without a gradient are zeros whatever they hold
    R.token_logprobs_backward(z, y, st, 0 * g, dz, entropy=ent, d_entropy=0 * ge)
    assert not dz.any()
    R.token_logprobs_backward(z, y, st, 0 * g, z)
    assert not z.any()


def test_offsets_past_32_bits():
    """30000 rows of 152064 bf16 logits: 4.6e9 entries, 9.1 GB."""
    n, V, rows = 30000, 152064, [0, 14121, 14122, 14123, 28243, 28245, 29999]
    z = torch.zeros(n, V, device=DEV, dtype=BF)
    y = torch.randint(0, V, (n,), generator=gen(5), device=DEV, dtype=torch.int32)
    z[rows] = (torch.randn(len(rows), V, generator=gen(4), device=DEV) * 3).to(BF)
    lp, ent, st = forward(z, y, 1.0)
    q, want, H = formula(z[rows], y[rows], 1.0)
    near(lp[rows], want, 4 * rel(V), 2 * U)
    near(lp[1:14000], torch.full((13999,), -math.log(V), device=DEV), 4 * rel(V), 2 * U)
    g = torch.randn(n, generator=gen(1), device=DEV)
    R.token_logprobs_backward(z, y, st, g, z)
    err, step = gradient_tol(q, H, g[rows], None, 1.0, BF, V)
    near(z[rows], gradient(q, H, y[rows], g[rows], None, 1.0), err + (g[rows].double().abs() * 2 * U)[:, None], step)
    del z
    torch.cuda.empty_cache()


def test_gradient_against_differences():
    """d (sum g logp + ge H) / dz by central differences: with h = 2^-5 the quotient is off by the third derivative,
    under (|g| + |ge| (ln V + 3)) h^2, and by the rounding of fp32 log-probabilities and entropies,
    (4 rel + 2 u ln V) / h."""
    V, h = 11, 2.0 ** -5
    z, y = make(1, V, F32, 3, spread=1.0)
    g, ge = torch.tensor([0.7], device=DEV), torch.tensor([-0.4], device=DEV)
    lp, ent, st = forward(z, y, 0.8)
    dz = torch.empty_like(z)
    R.token_logprobs_backward(z, y, st, g, dz, entropy=ent, d_entropy=ge, temperature=0.8)
    zz = z.repeat(2 * V, 1)
    i = torch.arange(V, device=DEV)
    zz[2 * i, i] += h
    zz[2 * i + 1, i] -= h
    lps, ents, _ = forward(zz, y.repeat(2 * V), 0.8)
    f = g * lps.double() + ge * ents.double()
    tol = (0.7 + 0.4 * (math.log(V) + 3)) * h * h / 0.8 ** 3 + 1.1 * (8 * rel(V) + 2 * U * 4) / h
    near(dz[0], (f[0::2] - f[1::2]) / (2 * h), tol)


# ------------------------------------------------------------------------------------------------ policy loss

def policy_formula(lp, old, ref, adv, ent, offs, live, *, clip_low, clip_high, dual_clip, kl, kl_coef, entropy_coef,
                   aggregate, scale, token_advantages):
    """Loss, its terms and gradients in 64 bits, token by token on the host."""
    n, k = lp.numel(), offs.numel() - 1
    h = lambda t: None if t is None else t.double().cpu().tolist()
    lp, old, ref, adv, ent = h(lp), h(old), h(ref), h(adv), h(ent)
    offs, live = offs.tolist(), live.tolist()
    seq = [-1] * n
    for s in range(k):
        for i in range(offs[s], offs[s + 1]):
            seq[i] = s
    live = [live[i] and seq[i] >= 0 for i in range(n)]
    counts = [sum(live[offs[s]:offs[s + 1]]) for s in range(k)]
    total, some = sum(counts), sum(c > 0 for c in counts)
    t = dict(pg=[], kl=[], h=[], clip=0, dual=0, diff=[])
    g, ge = [0.0] * n, [0.0] * n
    for i in range(n):
        if not live[i]:
            continue
        w = {"token_mean": 1 / total, "sequence_mean": 1 / (counts[seq[i]] * some), "sum": 1.0}[aggregate]
        A = adv[i if token_advantages else seq[i]]
        lr = lp[i] - old[i]
        r = math.exp(min(20.0, max(-20.0, lr)))
        rc = min(1 + clip_high, max(1 - clip_low, r))
        pg = max(-A * r, -A * rc)
        stopped = -A * rc > -A * r
        dual = dual_clip > 0 and A < 0 and r > dual_clip
        if dual:
            pg = -A * dual_clip
        d = 0.0 if stopped or dual or abs(lr) > 20 else -A * r
        kv = 0.0
        if ref is not None:
            raw = ref[i] - lp[i]
            x = min(20.0, max(-20.0, raw))
            kv, dk = {"k1": (-x, 1.0), "k2": (x * x / 2, -x), "k3": (math.expm1(x) - x, -math.expm1(x))}[kl]
            if abs(raw) <= 20:
                d += kl_coef * dk
        t["pg"].append(w * pg)
        t["kl"].append(w * kv)
        t["h"].append(0.0 if ent is None else w * ent[i])
        t["clip"] += stopped
        t["dual"] += dual
        t["diff"].append(-lr)
        g[i] = scale * w * d
        ge[i] = -scale * w * entropy_coef
    pg, kv, hh = math.fsum(t["pg"]), math.fsum(t["kl"]), math.fsum(t["h"])
    m = max(1, total)
    out = [scale * (pg + kl_coef * kv - entropy_coef * hh), pg, kv, hh, t["clip"] / m, t["dual"] / m, math.fsum(t["diff"]) / m, total]
    size = sum(abs(v) for k2 in ("pg", "kl", "h") for v in t[k2]) + sum(map(abs, t["diff"])) / m
    return out, g, ge, size


def check_policy(out, g, ge, want):
    """fp64 sums of n terms, then one rounding to fp32."""
    w, wg, wge, size = want
    dev = lambda a: torch.tensor(a, device=DEV, dtype=torch.double)
    near(out, dev(w), 1e-12 * (1 + size), 2 * U)
    near(g, dev(wg), 1e-13, 2 * U)
    if ge is not None:
        near(ge, dev(wge), 1e-13, 2 * U)


DEFAULT = dict(clip_low=0.2, clip_high=0.28, dual_clip=0.0, kl="k3", kl_coef=0.05, entropy_coef=0.0, aggregate="token_mean",
               scale=1.0, token_advantages=False)


def batch(lens, seed, masked=0.0, before=0, behind=0, spread=0.3, token=False):
    g = gen(seed)
    offs = torch.tensor([before] + lens).cumsum(0)
    n = int(offs[-1]) + behind
    lp = -4 * torch.rand(n, generator=g, device=DEV)
    old = lp + spread * torch.randn(n, generator=g, device=DEV)
    ref = lp + spread * torch.randn(n, generator=g, device=DEV)
    ent = 3 * torch.rand(n, generator=g, device=DEV)
    adv = torch.randn(n if token else len(lens), generator=g, device=DEV)
    mask = (torch.rand(n, generator=g, device=DEV) >= masked).to(torch.uint8)
    return dict(lp=lp, old=old, ref=ref, ent=ent, adv=adv, mask=mask, offs=offs.to(torch.int32).to(DEV), n=n)


def run_policy(b, opts, use_ref=True, use_ent=True, use_mask=True, use_offs=True, **more):
    o = DEFAULT | opts
    n = b["n"]
    out, g, ge = torch.full((8,), 3.0, device=DEV), torch.full((n,), 3.0, device=DEV), torch.full((n,), 3.0, device=DEV)
    R.policy_loss(b["lp"], b["old"], b["adv"], out, g, seq_offsets=b["offs"] if use_offs else None,
                  ref_logp=b["ref"] if use_ref else None, entropy=b["ent"] if use_ent else None,
                  mask=b["mask"] if use_mask else None, d_entropy=ge, **o, **more)
    live = b["mask"].bool() if use_mask else torch.ones(n, dtype=torch.bool)
    want = policy_formula(b["lp"], b["old"], b["ref"] if use_ref else None, b["adv"], b["ent"] if use_ent else None,
                          b["offs"], live, **o)
    return out, g, ge, want


LENS = [[1], [3, 1, 2], [0, 5, 0], [1500], [700, 0, 1, 900, 64], [1023, 1, 1], [1024], [1, 1024, 1025, 3, 0],
        [2] * 300, [37] * 150 + [0] * 20, [4000, 5000, 3]]


@pytest.mark.parametrize("lens", LENS, ids=lambda l: f"{len(l)}x{sum(l)}")
@pytest.mark.parametrize("aggregate", ["token_mean", "sequence_mean", "sum"])
def test_policy_loss_lengths(lens, aggregate):
    token = len(lens) % 2 == 1
    b = batch(lens, sum(lens), masked=0.3, before=len(lens) % 3, behind=len(lens) % 2 * 5, token=token)
    check_policy(*run_policy(b, dict(aggregate=aggregate, token_advantages=token, entropy_coef=0.01, dual_clip=3.0)))
    check_policy(*run_policy(b, dict(aggregate=aggregate, token_advantages=token, scale=-2.5), use_mask=False))


@pytest.mark.parametrize("kl", ["k1", "k2", "k3"])
@pytest.mark.parametrize("dual", [0.0, 1.5])
def test_policy_loss_terms(kl, dual):
    b = batch([50, 3, 200], 7, masked=0.2, spread=0.8)
    b["adv"][1] = 0.0
    b["lp"][:6] = torch.tensor([0.0, -1e-3, -30.0, -60.0, -1.0, -2.0])
    b["old"][:6] = torch.tensor([0.0, -40.0, -1.0, -1.0, -1.0, -2.0 - math.log(1.28)])   # equal, and past the clamps
    b["ref"][:6] = torch.tensor([0.0, -50.0, -2.0, -1.0, -INF, -2.0])
    b["mask"][:6] = 1
    for ref in (True, False):
        check_policy(*run_policy(b, dict(kl=kl, dual_clip=dual, kl_coef=0.3 if ref else 0.0), use_ref=ref))
    check_policy(*run_policy(b, dict(kl=kl, dual_clip=dual, clip_low=0.0, clip_high=0.0), use_ent=False))


def test_policy_loss_looks_only_at_counted_tokens():
    b = batch([40, 30, 20], 9, masked=0.4, before=3, behind=4)
    b["mask"][3:43] = 0                                    # a sequence without a counted token
    live = b["mask"].bool()
    live[:3] = live[-4:] = False
    want = run_policy(b, dict(aggregate="sequence_mean", entropy_coef=0.1))
    for k, bad in (("lp", NAN), ("old", INF), ("ref", -INF), ("ent", NAN)):
        b[k][~live] = bad
    b["adv"][0] = NAN
    got = run_policy(b, dict(aggregate="sequence_mean", entropy_coef=0.1))
    for x, y in zip(got[:3], want[:3]):
        assert torch.equal(x, y)
    b["mask"][:] = 0
    out, g, ge, _ = run_policy(b, dict(entropy_coef=0.1))
    assert not out.any() and not g.any() and not ge.any()
    b["mask"][50] = 1
    b["lp"][50] = NAN
    out, g, _, _ = run_policy(b, dict(entropy_coef=0.1))
    assert out[0].isnan() and g[50].isnan() and out[7] == 1 and int(g.isnan().sum()) == 1


def test_policy_loss_without_tokens():
    e = torch.empty(0, device=DEV)
    out = torch.full((8,), 3.0, device=DEV)
    R.policy_loss(e, e, torch.ones(1, device=DEV), out, e)
    assert not out.any()
    out.fill_(3.0)
    R.policy_loss_logits(torch.empty(0, 50, device=DEV), torch.empty(0, device=DEV, dtype=torch.int32), e,
                         torch.ones(1, device=DEV), out, e, torch.empty(0, 50, device=DEV))
    assert not out.any()


def test_policy_loss_one_sequence_without_offsets_and_bool_mask():
    b = batch([333], 2, masked=0.5)
    got = run_policy(b, {}, use_offs=False)
    check_policy(*got)
    out, g = torch.empty(8, device=DEV), torch.empty(333, device=DEV)
    R.policy_loss(b["lp"], b["old"], b["adv"], out, g, ref_logp=b["ref"], mask=b["mask"].bool(), **(DEFAULT | {"entropy_coef": 0.0}))
    assert torch.equal(g, got[1]) and torch.equal(out[:3], got[0][:3])


def test_policy_loss_many_tokens_and_sequences():
    """Past one workgroup's share of tokens and sequences, against torch's sums in 64 bits."""
    n, k = 700001, 5000
    g = gen(3)
    cut = torch.randint(0, n + 1, (k - 1,), generator=g, device=DEV).sort().values
    offs = torch.cat([cut.new_zeros(1), cut, cut.new_full((1,), n)]).int()
    lp = -4 * torch.rand(n, generator=g, device=DEV)
    old = lp + 0.05 * torch.randn(n, generator=g, device=DEV)
    adv = torch.randn(k, generator=g, device=DEV)
    out, d = torch.empty(8, device=DEV), torch.empty(n, device=DEV)
    R.policy_loss(lp, old, adv, out, d, seq_offsets=offs, clip_low=0.9, clip_high=9.0, aggregate="sequence_mean")
    seq = torch.searchsorted(offs[1:].long(), torch.arange(n, device=DEV), right=True)
    lens = (offs[1:] - offs[:-1]).double()
    w = 1 / (lens[seq] * (lens > 0).sum())
    pg = -adv.double()[seq] * (lp.double() - old.double()).exp() * w
    near(out[0], pg.sum(), 1e-11 * pg.abs().sum(), 2 * U)
    near(d, pg, 1e-15, 2 * U)
    assert int(out[7]) == n and out[4] == 0


def test_policy_gradient_against_differences():
    """h = 2^-8: third derivatives of the terms are at most 2 |A| e^|lr| w here, the loss has a rounding of 2 u |loss|."""
    b = batch([6, 5], 12, spread=0.1)
    o = dict(clip_low=0.9, clip_high=4.0, kl="k3", kl_coef=0.2, entropy_coef=0.05, aggregate="sequence_mean")
    base, g, ge, _ = run_policy(b, o)
    h = 2.0 ** -8
    for key, grad in (("lp", g), ("ent", ge)):
        for i in range(11):
            v = []
            for sgn in (1, -1):
                c = dict(b, **{key: b[key].clone()})
                c[key][i] += sgn * h
                step = float(c[key][i].double() - b[key][i].double())
                v.append((float(run_policy(c, o)[0][0].double()), step))
            quotient = (v[0][0] - v[1][0]) / (v[0][1] - v[1][1])
            tol = 4 * float(b["adv"].abs().max()) * h * h + 2 * U * (abs(v[0][0]) + 1) / h
            assert abs(quotient - float(grad[i])) <= tol, (key, i)


# ------------------------------------------------------------------------------------- from logits in one call

@pytest.mark.parametrize("n,V,dtype,lens,inplace", [
    (1, 1, F32, [1], False), (1, 50001, BF, [1], True), (7, 33, BF, [2, 0, 5], False), (24, 151936, BF, [20, 4], False),
    (300, 4096, F32, [100, 150, 50], True), (256, 4095, F32, [256], False), (600, 2051, BF, [1] * 600, True),
    (700, 32000, BF, [300, 100, 290], False), (260, 152064, BF, [30] * 8 + [20], True), (270, 152065, BF, [270], False),
    (257, 81921, F32, [200, 57], False), (300, 170001, BF, [300], True), (1030, 517, F32, [515, 515], False)])
@pytest.mark.parametrize("T,ent", [(1.0, 0.0), (0.7, 0.02)])
def test_policy_loss_logits(n, V, dtype, lens, inplace, T, ent):
    before = (n - sum(lens))
    b = batch(lens, n, masked=0.25, before=before, token=True)
    z, y = make(n, V, dtype, n + V, pad=n % 3, shift=n % 2)
    q, lp, H = formula(z, y, T)
    # old log-probabilities near the new ones, none of them within 1e-3 of a clip border of its ratio
    d = 0.3 * torch.randn(n, generator=gen(8), device=DEV)
    for r in (0.8, 1.28, 2.0):
        d = torch.where((d + math.log(r)).abs() < 1e-3, d + 3e-3, d)
    old, ref = (lp + d).float(), (lp + 0.1 * torch.randn(n, generator=gen(6), device=DEV)).float()
    o = DEFAULT | dict(entropy_coef=ent, dual_clip=2.0, aggregate="sequence_mean", token_advantages=True, scale=3.0)
    mask = b["mask"]
    if n > 4:
        mask[2] = 0
        z[2] = NAN                                    # padding
    dead = ~mask.bool()
    dead[:before] = True
    store = torch.full((n, V + n % 3), 9.0, device=DEV, dtype=dtype)
    dz = z if inplace else store[:, :V]
    out, out_lp = torch.empty(8, device=DEV), torch.empty(n, device=DEV)
    out_ent = torch.empty(n, device=DEV) if ent or V % 2 else None
    R.policy_loss_logits(z, y, old, b["adv"], out, out_lp, dz, seq_offsets=b["offs"], ref_logp=ref, mask=mask,
                         out_entropy=out_ent, temperature=T, **o)
    near(out_lp, torch.where(dead, 0.0, lp), 4 * rel(V), 2 * U)
    if out_ent is not None:
        near(out_ent, torch.where(dead, 0.0, H), 6 * rel(V) * (1 + math.log(V)), 2 * U)
    # the loss and the tokens' gradients of the log-probabilities that came out
    # (theirs before rounding, at most x = U |lp| away.  A token's pg moves by |pg| x, its KL by |exp(d) - 1| x < x, since
    # |d| < 0.7 here; weights sum to 1.  A gradient moves by |g| x, and kl_coef exp(d) w x < 0.11 w x for its KL)
    want = policy_formula(out_lp, old, ref, b["adv"], out_ent, b["offs"], ~dead, **o)
    w, wg, wge, size = want
    dev = lambda a: torch.tensor(a, device=DEV, dtype=torch.double)
    x = U * torch.where(dead, 0.0, lp).abs()
    near(out, dev(w), 1e-12 * (1 + size) + o["scale"] * (size + 1) * float(x.max()), 2 * U)
    g, ge = dev(wg), dev(wge) if ent else None
    err, step = gradient_tol(q, H, g, ge, T, dtype, V)
    full = gradient(q, H, y, g, ge, T)
    full[dead], err[dead] = 0.0, 0.0
    moved = (g.abs() + 0.11 * o["scale"]) * x / T
    near(dz, full, err + (g.abs() / T * 4 * U + moved)[:, None], step + 4 * U)
    if not inplace:
        assert (store[:, V:] == 9.0).all()


def test_policy_loss_logits_entropy_output_changes_nothing_else():
    n, V = 400, 3001
    z, y = make(n, V, BF, 1)
    b = batch([200, 200], 4)
    o = dict(seq_offsets=b["offs"], ref_logp=b["ref"][:n], kl_coef=0.1)
    res = []
    for ent in (None, torch.empty(n, device=DEV)):
        out, lp, dz = torch.empty(8, device=DEV), torch.empty(n, device=DEV), torch.empty_like(z)
        R.policy_loss_logits(z, y, b["old"], b["adv"], out, lp, dz, out_entropy=ent, **o)
        res.append((out[:3].clone(), lp, dz))
    near(res[0][1], res[1][1], 4 * rel(V), 2 * U)
    near(res[0][0], res[1][0], 40 * rel(V), 2 * U)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [5, 1000, 9001, 70001])
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_policy_loss_logits_rows_that_are_not_ordinary(V, dtype, T):
    """The same twelve rows among many and alone: what is no number, of one value or out of range gives the same either way,
    and other rows do not notice."""
    low = torch.finfo(dtype).min
    n, k, at = 1100, 12, 40
    z, y = make(n, V, dtype, V, spread=1.0)
    odd = z[at:at + k]
    odd[0] = -INF
    odd[1] = -INF
    odd[1, V // 2] = 3.0
    odd[2] = low
    odd[3, 1:] = low
    odd[4, V - 1] = INF
    odd[5, 0] = NAN
    odd[6] = 0.0
    odd[9] = -INF
    odd[9, :2] = 1.0
    odd[10, 0], odd[10, 1] = -low, low
    odd[11] = -low
    y[at:at + k] = torch.tensor([0, V // 2, 1, 0, 0, 0, 2, -1, V, V - 1, 0, 3], dtype=torch.int32)
    q, lp, H = formula(z, y, T)
    old = torch.where(lp.isfinite(), lp, -1.0).clamp(min=-30).float()
    adv = torch.linspace(-1.0, 2.0, n, device=DEV)
    o = dict(clip_low=0.5, clip_high=8.0, token_advantages=True, aggregate="sum", entropy_coef=0.02)
    res = []
    for a, b in ((0, n), (at, at + k)):
        out, olp, ent = torch.empty(8, device=DEV), torch.empty(b - a, device=DEV), torch.empty(b - a, device=DEV)
        dz = torch.full((b - a, V), 9.0, device=DEV, dtype=dtype)
        R.policy_loss_logits(z[a:b], y[a:b], old[a:b], adv[a:b], out, olp, dz, out_entropy=ent, temperature=T, **o)
        assert out[0].isnan()
        res.append((olp, ent, dz))
    (olp, ent, dz), (olp2, ent2, dz2) = res
    rows = [i for i in range(k) if i not in (0, 4, 5)]
    i = torch.tensor(rows, device=DEV)
    assert ent[at + i].isfinite().all() and olp[at + torch.tensor([0, 4, 5, 7, 8], device=DEV)].isnan().all()
    assert dz[at + torch.tensor([0, 4, 5], device=DEV)].isnan().any(1).all()
    assert dz[at + i].isfinite().all() and not dz[at + 1].any() and not dz[at + 10].any()
    # both ways are within the bounds of the formula, so twice those apart
    near(ent[at + i], ent2[i], 12 * rel(V) * (1 + math.log(V)), 4 * U)
    j = torch.tensor([1, 2, 3, 6, 10, 11], device=DEV)
    near(olp[at + j], olp2[j], 8 * rel(V), 4 * U)
    assert olp[at + 9] == -INF and olp2[9] == -INF
    for r in rows:
        g = adv[at + r].abs().double() + 0.02 * (2 + math.log(V))
        near(dz[at + r], dz2[r], g / T * 40 * rel(V), 2.0 ** -7 if dtype == BF else 40 * rel(V))
    # ordinary rows against the formula; ratios are 1, inside the clip
    plain = torch.ones(n, dtype=torch.bool, device=DEV)
    plain[at:at + k] = False
    near(olp[plain], lp[plain], 4 * rel(V), 2 * U)
    g = (-adv.double() * (olp.double() - old.double()).exp())[plain]
    ge = torch.full_like(g, -0.02)
    err, step = gradient_tol(q[plain], H[plain], g, ge, T, dtype, V)
    err += q[plain].exp() * 0.02 / T * 6 * rel(V) * (1 + math.log(V))      # of the entropy in the formula
    # g is of log-probabilities before rounding: U |lp| of it
    near(dz[plain], gradient(q[plain], H[plain], y[plain], g, ge, T),
         err + (g.abs() / T * (4 + lp[plain].abs()) * U)[:, None], step + 4 * U)


@pytest.mark.parametrize("n", [191, 192, 1023, 1025, 2500])
@pytest.mark.parametrize("offs", [None, "none", "ends"])
def test_policy_loss_logits_rows_without_a_token(n, offs):
    """Runs of rows that do not count, at every place of a workgroup's rows, without offsets, with none that count, and
    with rows before the first and behind the last sequence."""
    V = 300
    z, y = make(n, V, BF, n)
    mask = (torch.arange(n, device=DEV) // 7 % 3 != 0) if offs is None else torch.ones(n, device=DEV, dtype=torch.bool)
    dead = ~mask
    so = None
    if offs == "none":
        mask[:] = False
        dead[:] = True
    elif offs == "ends":
        so = torch.tensor([60, 60, n - 90], device=DEV, dtype=torch.int32)
        dead[:60] = dead[n - 90:] = True
        mask = None
    z[dead] = NAN
    y[dead] = -7
    q, lp, H = formula(z, y, 1.0)
    old = torch.where(dead, NAN, lp).float()
    adv = torch.full((n,), 1.5, device=DEV)
    adv[dead] = NAN
    out, olp = torch.full((8,), 3.0, device=DEV), torch.full((n,), 3.0, device=DEV)
    dz = torch.full_like(z, 9.0)
    R.policy_loss_logits(z, y, old, adv, out, olp, dz, mask=mask, seq_offsets=so, token_advantages=True, clip_high=4.0)
    live = int((~dead).sum())
    assert not dz[dead].any() and not olp[dead].any() and float(out[7]) == live
    if not live:
        assert not out.any()
        return
    near(olp[~dead], lp[~dead], 4 * rel(V), 2 * U)
    near(out[0], torch.tensor(-1.5, device=DEV), 1.5 * 8 * rel(V), 2 * U)
    g = (-1.5 / live) * (olp.double() - old.double()).exp()[~dead]
    qd, yd = q[~dead], y[~dead]
    err, step = gradient_tol(qd, H[~dead], g, None, 1.0, BF, V)
    # g is of log-probabilities before rounding: U |lp| of it
    near(dz[~dead], gradient(qd, H[~dead], yd, g, None, 1.0), err + (g.abs() * (4 + lp[~dead].abs()) * U)[:, None], step + 4 * U)


def test_policy_loss_counts_in_long_sequences():
    """Masks counted by a wave, a workgroup and a wide one: sequences of every length among others of it, odd starts."""
    for lens in ([40] * 300 + [1, 0, 17], [1500, 3000, 1, 0, 2047], [50001, 1, 16385, 30000], [70001]):
        b = batch(lens, len(lens), masked=0.3, before=3, behind=2)
        for aggregate in ("token_mean", "sequence_mean"):
            check_policy(*run_policy(b, dict(aggregate=aggregate)))


# -------------------------------------------------------------------------------------------- preference loss

def preference_formula(lp, ref, offs, live, *, form, average, beta, label_smoothing, margin, scale):
    h = lambda t: None if t is None else t.double().cpu().tolist()
    lp, ref, offs, live = h(lp), h(ref), offs.tolist(), live.tolist()
    P = (len(offs) - 1) // 2
    grad, rewards, sums, losses = [0.0] * len(lp), [], [], []
    per, size = [], 0.0
    for s in range(2 * P):
        at = [i for i in range(offs[s], offs[s + 1]) if live[i]]
        per.append(1 / max(1, len(at)) if average else 1.0)
        sums.append(math.fsum(lp[i] for i in at) * per[s])
        rewards.append(beta * per[s] * math.fsum(v for i in at for v in ((lp[i],) if ref is None else (lp[i], -ref[i]))))
        size += sum(abs(lp[i]) for i in at)
    for p in range(P):
        x = rewards[2 * p] - rewards[2 * p + 1] - margin
        softplus = lambda v: max(v, 0.0) + math.log1p(math.exp(-abs(v)))
        sig = lambda v: math.exp(-softplus(-v))
        if form == "sigmoid":
            losses.append((1 - label_smoothing) * softplus(-x) + label_smoothing * softplus(x))
            d = label_smoothing * sig(x) - (1 - label_smoothing) * sig(-x)
        elif form == "hinge":
            losses.append(max(0.0, 1 - x))
            d = -1.0 if x < 1 else 0.0
        else:
            losses.append(((x - 0.5) / beta) ** 2)
            d = 2 * (x - 0.5) / beta ** 2
        for s, sign in ((2 * p, 1), (2 * p + 1, -1)):
            for i in range(offs[s], offs[s + 1]):
                if live[i]:
                    grad[i] = sign * scale * beta * d * per[s] / P
    c, r = rewards[0::2], rewards[1::2]
    mean = lambda v: math.fsum(v) / P
    out = [scale * mean(losses), mean(c), mean(r), mean(c) - mean(r), mean([float(a > b) for a, b in zip(c, r)]),
           mean(sums[0::2]), mean(sums[1::2]), P]
    return out, grad, rewards, size


def run_preference(b, use_ref=True, use_mask=True, **opts):
    o = dict(form="sigmoid", average=False, beta=0.1, label_smoothing=0.0, margin=0.0, scale=1.0) | opts
    n, P = b["n"], (b["offs"].numel() - 1) // 2
    out, g, rew = torch.full((8,), 3.0, device=DEV), torch.full((n,), 3.0, device=DEV), torch.full((2 * P,), 3.0, device=DEV)
    ref, mask = b["ref"] if use_ref else None, b["mask"] if use_mask else None
    R.preference_loss(b["lp"], b["offs"], out, g, ref_logp=ref, mask=mask, out_rewards=rew, **o)
    live = b["mask"].bool() if use_mask else torch.ones(n, dtype=torch.bool)
    w, wg, wr, size = preference_formula(b["lp"], ref, b["offs"], live, **o)
    dev = lambda a: torch.tensor(a, device=DEV, dtype=torch.double)
    s = max(1.0, 1 / o["beta"]) ** 2
    near(out, dev(w), 1e-12 * s * (1 + size) ** 2, 2 * U)
    near(g, dev(wg), 1e-12 * s * (1 + size), 2 * U)
    near(rew, dev(wr), 1e-12 * (1 + size), 2 * U)
    return out, g, rew


PAIRS = [[1, 1], [3, 0], [0, 0], [1, 2, 0, 7], [255, 257], [1500, 900], [5000, 4], [64] * 40, [33000, 30001], [1, 2] * 700,
         [20000, 17000, 3, 90], [700, 2500, 1, 0] * 20]


@pytest.mark.parametrize("lens", PAIRS, ids=lambda l: f"{len(l)}x{sum(l)}")
@pytest.mark.parametrize("form", ["sigmoid", "hinge", "squared"])
def test_preference_loss(lens, form):
    b = batch(lens, sum(lens) + 1, masked=0.3, before=len(lens) % 5, behind=sum(lens) % 7, spread=0.05)
    run_preference(b, form=form, average=True, beta=0.7, margin=0.2)
    run_preference(b, form=form, beta=0.05, scale=-4.0, use_mask=False)
    run_preference(b, form=form, use_ref=False, beta=1e-3)
    if form == "sigmoid":
        run_preference(b, label_smoothing=0.1, beta=0.5)


def test_preference_loss_far_margins_and_padding():
    b = batch([4, 4, 4, 4, 6, 6], 3, masked=0.0, behind=3)
    b["lp"][:4], b["lp"][4:8] = 0.0, -500.0            # beta 5: a margin of 10000 either way
    b["lp"][8:12], b["lp"][12:16] = -500.0, 0.0
    b["ref"][:16] = 0.0
    b["mask"][18], b["lp"][18], b["ref"][18] = 0, NAN, INF
    b["lp"][-3:] = NAN
    for form in ("sigmoid", "hinge", "squared"):
        out, g, rew = run_preference(b, form=form, beta=5.0)
        assert out.isfinite().all() and g.isfinite().all() and g[18] == 0 and not g[-3:].any()
    same = batch([50, 50], 1)
    same["lp"][50:] = same["lp"][:50]
    same["ref"][50:] = same["ref"][:50]
    out, g, rew = run_preference(same)
    assert out[4] == 0 and rew[0] == rew[1]              # equal rewards: no winner


def test_preference_gradient_against_differences():
    """h = 2^-4 on one token: h^2 beta^3 / 6 of the third derivative (at most 1/6), and 2 u loss / h of rounding."""
    b = batch([5, 4, 3, 6], 21, masked=0.2)
    o = dict(beta=0.6, label_smoothing=0.1, margin=0.1)
    out, g, _ = run_preference(b, **o)
    h = 2.0 ** -4
    for i in range(b["n"]):
        v = []
        for sgn in (1, -1):
            c = dict(b, lp=b["lp"].clone())
            c["lp"][i] += sgn * h
            v.append((float(run_preference(c, **o)[0][0].double()), float(c["lp"][i].double() - b["lp"][i].double())))
        assert abs((v[0][0] - v[1][0]) / (v[0][1] - v[1][1]) - float(g[i])) <= h * h * 0.6 ** 3 / 6 + 4 * U * 2 / h, i


# ------------------------------------------------------------------------------- together, streams and graphs

def chain(z, y, b, bufs, T=0.9):
    """Log-probabilities, preference loss, gradient of the logits; then the policy loss from the same logits."""
    R.token_logprobs(z, y, bufs["lp"], out_entropy=bufs["ent"], out_stats=bufs["st"], temperature=T, workspace=bufs["w0"])
    R.preference_loss(bufs["lp"], b["offs"], bufs["out"], bufs["g"], ref_logp=b["ref"], mask=b["mask"], workspace=bufs["w1"])
    R.token_logprobs_backward(z, y, bufs["st"], bufs["g"], bufs["dz"], temperature=T)
    R.policy_loss(bufs["lp"], b["old"], b["adv"], bufs["out3"], bufs["g3"], seq_offsets=b["offs"], ref_logp=b["ref"],
                  mask=b["mask"], kl_coef=0.1, aggregate="sequence_mean", workspace=bufs["w3"])
    R.policy_loss_logits(z, y, b["old"], b["adv"], bufs["out2"], bufs["lp2"], bufs["dz2"], seq_offsets=b["offs"],
                         ref_logp=b["ref"], mask=b["mask"], out_entropy=bufs["ent2"], temperature=T, kl_coef=0.1,
                         entropy_coef=0.01, workspace=bufs["w2"])


def buffers(n, V, k, dtype):
    L = R.lib()
    f = lambda *s: torch.zeros(*s, device=DEV)
    ws = lambda nb: torch.full((nb,), 255, dtype=torch.uint8, device=DEV)     # NaN patterns, were they read
    return dict(lp=f(n), ent=f(n), st=f(n, 2), out=f(8), g=f(n), dz=torch.zeros(n, V, device=DEV, dtype=dtype),
                out2=f(8), lp2=f(n), ent2=f(n), dz2=torch.zeros(n, V, device=DEV, dtype=dtype), out3=f(8), g3=f(n),
                w0=ws(L.rl_logprob_workspace_bytes(n, V)), w1=ws(L.rl_preference_workspace_bytes(n, k // 2)),
                w2=ws(L.rl_policy_logits_workspace_bytes(n, k, V)), w3=ws(L.rl_policy_workspace_bytes(n, k)))


NAMES = ("lp", "ent", "st", "out", "g", "dz", "out2", "lp2", "ent2", "dz2", "out3", "g3")


@pytest.mark.parametrize("lens,V,dtype", [([9, 4, 6, 5], 50000, BF), ([200, 100, 150, 62], 3000, F32)])
def test_streams_and_graph_replays(lens, V, dtype):
    n = sum(lens)
    b = batch(lens, 5, masked=0.2)
    inputs = [make(n, V, dtype, 40 + i) for i in range(3)]
    eager = []
    for z, y in inputs:
        e = buffers(n, V, 4, dtype)
        chain(z, y, b, e)
        eager.append(e)
    torch.cuda.synchronize()
    # two streams at once, each with buffers of its own
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    b1, b2 = buffers(n, V, 4, dtype), buffers(n, V, 4, dtype)
    torch.cuda.synchronize()
    for _ in range(3):
        for st, bf, (z, y) in ((s1, b1, inputs[0]), (s2, b2, inputs[1])):
            with torch.cuda.stream(st):
                chain(z, y, b, bf)
    torch.cuda.synchronize()
    for got, want in ((b1, eager[0]), (b2, eager[1])):
        for k in NAMES:
            assert torch.equal(got[k], want[k]), k
    # a stream by argument, workspace made by the call
    lp = torch.empty(n, device=DEV)
    R.token_logprobs(*inputs[0], lp, temperature=0.9, stream=s1)
    s1.synchronize()
    near(lp, eager[0]["lp"], 8 * rel(V), 2 * U)
    # captured once, replayed on other inputs with eager work between
    z, y = inputs[0][0].clone(), inputs[0][1].clone()
    cap = buffers(n, V, 4, dtype)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(z, y, b, cap)
        with torch.cuda.graph(graph, stream=side):
            chain(z, y, b, cap)
    torch.cuda.synchronize()
    for i in (1, 2, 0, 1):
        z.copy_(inputs[i][0])
        y.copy_(inputs[i][1])
        other = buffers(n, V, 4, dtype)
        chain(*inputs[(i + 1) % 3], b, other)
        graph.replay()
        torch.cuda.synchronize()
        for k in NAMES:
            assert torch.equal(cap[k], eager[i][k]), (i, k)
            assert torch.equal(other[k], eager[(i + 1) % 3][k]), (i, k)


def test_workspace_of_a_call_on_another_stream():
    """What the current stream has freed and still uses is no workspace of a call on another stream."""
    n, V = 400, 3001
    z, y = make(n, V, F32, 3)
    b = batch([n], 3)
    f = lambda *s: torch.empty(*s, device=DEV)
    want, got = (f(8), f(n), f(n, V)), (f(8), f(n), f(n, V))
    R.policy_loss_logits(z, y, b["old"], b["adv"], *want, aggregate="sequence_mean", mask=b["mask"])
    x = torch.randn(4096, 4096, device=DEV)
    nbytes = R.lib().rl_policy_logits_workspace_bytes(n, 1, V)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(8):
        x = x @ x * 1e-3
    held = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(4)]
    for h in held:
        h.fill_(255)                  # when the products are done
    del held, h
    R.policy_loss_logits(z, y, b["old"], b["adv"], *got, aggregate="sequence_mean", mask=b["mask"], stream=side)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_temperatures_out_of_range():
    z, y = make(2, 9, F32, 1)
    for T in (1e-50, -1e-50, 1e-31, 2e30, INF, NAN):
        with pytest.raises(R.RLError):
            R.token_logprobs(z, y, torch.empty(2, device=DEV), temperature=T)
    lp = torch.empty(2, device=DEV)
    R.token_logprobs(z, y, lp, temperature=0)
    near(lp, formula(z, y, 1.0)[1], 4 * rel(9), 2 * U)
    for T in (1e-30, 1e30):       # |z| < 16, so log-probabilities are within 32e30, which fp32 holds
        R.token_logprobs(z, y, lp, temperature=T)
        near(lp, formula(z, y, T)[1], 4 * rel(9), 2 * U)


def test_binding_refusals():
    n, V = 4, 16
    z, y = make(n, V, BF, 1)
    f = lambda k=n: torch.zeros(k, device=DEV)
    i32 = lambda k: torch.zeros(k, device=DEV, dtype=torch.int32)
    bad = [lambda: R.token_logprobs(z.half(), y, f()), lambda: R.token_logprobs(z[0], y, f()),
           lambda: R.token_logprobs(z.t(), y, f()), lambda: R.token_logprobs(z, y.long(), f()),
           lambda: R.token_logprobs(z, y[:3], f()), lambda: R.token_logprobs(z, y, f().cpu()),
           lambda: R.token_logprobs(z, y, f(8)[::2]), lambda: R.token_logprobs(z, y, f(), out_stats=f(4)),
           lambda: R.token_logprobs(z, y, f(), workspace=f(64)),
           lambda: R.token_logprobs(z[:1].expand(4, V), y, f()),
           lambda: R.token_logprobs_backward(z, y, f(8), f(), z.float()),
           lambda: R.token_logprobs_backward(z, y, f(8), f(), z[:, :8]),
           lambda: R.policy_loss(f(), f(), f(2), f(8), f()), lambda: R.policy_loss(f(), f(), f(1), f(7), f()),
           lambda: R.policy_loss(f(), f(), f(1), f(8), f(), kl="k4"),
           lambda: R.policy_loss(f(), f(), f(1), f(8), f(), aggregate="mean"),
           lambda: R.policy_loss(f(), f(), f(1), f(8), f(), seq_offsets=i32(0)),
           lambda: R.policy_loss(f(), f(), f(1), f(8), f(), mask=f()),
           lambda: R.policy_loss(f().double(), f(), f(1), f(8), f()),
           lambda: R.preference_loss(f(), i32(4), f(8), f()), lambda: R.preference_loss(f(), i32(3), f(8), f(), form="x"),
           lambda: R.preference_loss(f(), i32(3), f(8), f(3))]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was not refused")
    refused = [lambda: R.token_logprobs(z, y, f(), temperature=-1.0),
               lambda: R.policy_loss(f(), f(), f(1), f(8), f(), kl_coef=0.1),
               lambda: R.policy_loss(f(), f(), f(1), f(8), f(), entropy_coef=0.1),
               lambda: R.policy_loss(f(), f(), f(1), f(8), f(), dual_clip=0.5),
               lambda: R.preference_loss(f(), i32(1), f(8), f()),
               lambda: R.preference_loss(f(), i32(3), f(8), f(), beta=0.0),
               # a gradient that begins inside the logits
               lambda: R.token_logprobs_backward(z, y, f(8), f(), torch.as_strided(z, (n, V), (V, 1), 2))]
    for k, call in enumerate(refused):
        with pytest.raises(R.RLError) as e:
            call()
        assert e.value.status == R.RL_ERR_INVALID_ARG, k


def test_sizes_past_32_bits_are_refused():
    f = lambda k: torch.zeros(k, device=DEV)
    y = torch.zeros(1, device=DEV, dtype=torch.int32)
    big = torch.empty(1, (1 << 32) + 5, device=DEV, dtype=BF)     # 5 to a 32-bit argument
    with pytest.raises(ValueError):
        R.token_logprobs(big, y, f(1))
    many = big.view(-1)[:(1 << 32)].view(torch.float32)           # 2^31 entries
    with pytest.raises(ValueError):
        R.policy_loss(many, many, f(1), f(8), many)
    with pytest.raises(ValueError):
        R.preference_loss(many, torch.zeros(3, device=DEV, dtype=torch.int32), f(8), many)


def test_lying_offsets_through_rows_stay_in_bounds():
    n, V = 400, 24
    z, y = make(n, V, F32, 2)
    old, adv = torch.zeros(n, device=DEV), torch.ones(2, device=DEV)
    for offs in ([-5, 30, 400], [0, 900, 400], [50, 10, 400], [0, 0, 1 << 30], [400, 400, 400], [-9, -3, -1]):
        o = torch.tensor(offs, dtype=torch.int32, device=DEV)
        big, lps = torch.full((n + 64, V), 4.0, device=DEV), torch.full((n + 64,), 4.0, device=DEV)
        for aggregate in ("token_mean", "sequence_mean"):
            R.policy_loss_logits(z, y, old, adv, torch.empty(8, device=DEV), lps[32:32 + n], big[32:32 + n], seq_offsets=o,
                                 aggregate=aggregate)
        for t in (big, lps):
            assert (t[:32] == 4.0).all() and (t[32 + n:] == 4.0).all()


def test_offsets_that_lie_stay_in_bounds():
    """Offsets that fall or leave the tokens: results are nobody's, but neighbours of every buffer stay."""
    n, V = 64, 40
    for offs in ([-5, 30, 64], [0, 90, 64], [50, 10, 64], [0, 0, 1 << 30], [64, 64, 64], [-9, -3, -1]):
        o = torch.tensor(offs, dtype=torch.int32, device=DEV)
        big = torch.full((n + 512,), 4.0, device=DEV)
        g = big[256:256 + n]
        b = batch([n], 1)
        adv = torch.ones(2, device=DEV)
        R.policy_loss(b["lp"], b["old"], adv, torch.empty(8, device=DEV), g, seq_offsets=o, aggregate="sequence_mean")
        R.preference_loss(b["lp"], o, torch.empty(8, device=DEV), g)
        z, y = make(n, V, F32, 2)
        zb = torch.full((n + 64, V), 4.0, device=DEV)
        R.policy_loss_logits(z, y, b["old"], adv, torch.empty(8, device=DEV), torch.empty(n, device=DEV), zb[32:32 + n],
                             seq_offsets=o, aggregate="sequence_mean")
        assert (big[:256] == 4.0).all() and (big[256 + n:] == 4.0).all()
        assert (zb[:32] == 4.0).all() and (zb[32 + n:] == 4.0).all()


def test_rollout_to_gradient():
    """What the engine samples, scored by these operators: logits of the responses' positions (one forced pass), their
    log-probabilities equal the rollout's, and the policy loss of the fresh policy has ratio 1 everywhere."""
    from paper_2509_15965_amd.configs import ModelShape
    from paper_2509_15965_amd.inputs import make_weights
    shape = ModelShape(2, 256, 4, 2, 64, 512, 4096, 1e-6, 1e4, "fp32")
    w = make_weights(shape, 3, device=DEV, init="normal")
    P, G, m, plen = 2, 3, 5, 7
    S, T = P * G, 0.8
    eng = R.Engine(shape, w, max_seqs=S, max_ctx=32, max_prefill_tokens=128)
    try:
        slots, uids = list(range(S)), list(range(100, 100 + S))
        offs = [0, plen, 2 * plen]
        ptok = torch.randint(0, 4096, (2 * plen,), generator=gen(1), device=DEV, dtype=torch.int32)
        tok, lps = torch.empty(m, S, device=DEV, dtype=torch.int32), torch.empty(m, S, device=DEV)
        eng.prefill(slots, uids, offs, ptok, tok[0], lps[0], group=G, seed=5, temperature=T)
        for t in range(1, m):
            eng.step(slots, uids, tok[t - 1], tok[t], lps[t], seed=5, temperature=T)
        # the actor's pass: logits of every response position
        logits, scratch, sl = torch.empty(m, S, 4096, device=DEV), torch.empty(S, device=DEV, dtype=torch.int32), torch.empty(S, device=DEV)
        eng.release(slots)
        first = torch.empty(P, 4096, device=DEV)
        eng.prefill(slots, uids, offs, ptok, scratch, sl, group=G, seed=5, temperature=T, out_logits=first)
        logits[0] = first.repeat_interleave(G, 0)
        for t in range(1, m):
            eng.step(slots, uids, tok[t - 1], scratch, sl, seed=5, temperature=T, out_logits=logits[t])
        # packed tokens, sequence after sequence; the reference policy's values by scoring
        z = logits.transpose(0, 1).reshape(S * m, 4096).contiguous()
        y, old = tok.t().reshape(-1).contiguous(), lps.t().reshape(-1).contiguous()
        so = torch.arange(0, S * m + 1, m, device=DEV, dtype=torch.int32)
        ref = torch.empty(S * m, device=DEV)
        eng.release(slots)
        eng.score(slots, offs, ptok, so.cpu().numpy(), y, ref, group=G, temperature=T)
        lp, ent, st = forward(z, y, T)
        # fp32 logits of two kernels' summation orders: |z| of a few units, 512 products
        near(lp, old, 1e-4)
        near(lp, ref, 1e-4)
        adv = torch.tensor([1.0, -0.5, -0.5, 0.3, -1.0, 0.7], device=DEV)
        out, dz = torch.empty(8, device=DEV), torch.empty_like(z)
        R.policy_loss_logits(z, y, old, adv, out, lp, dz, seq_offsets=so, ref_logp=ref, temperature=T, kl_coef=0.1,
                             aggregate="sequence_mean")
        near(out[0], -adv.mean(), 1e-4 * 2)
        assert out[4] == 0 and out[7] == S * m and abs(float(out[2])) < 1e-7
        q, _, H = formula(z, y, T)
        g = -adv.double().repeat_interleave(m) / (m * S)
        near(dz, gradient(q, H, y, g, None, T), 2e-4 * float(g.abs().max()) / T)
        # and pairs made of a group's best and worst response
        d = torch.empty(S * m, device=DEV)
        R.preference_loss(lp, so, out, d, ref_logp=ref)
        near(out[0], torch.tensor(math.log(2.0), device=DEV), 1e-4)
        R.token_logprobs_backward(z, y, st, d, dz, temperature=T)
        near(dz, gradient(q, H, y, d, None, T), 1e-5, 1e-5)
    finally:
        eng.close()


@pytest.mark.parametrize("dtype", [F32, BF])
def test_most_rows_and_sequences(dtype):
    """2^20 rows, every one a sequence of its own, through every call that takes rows."""
    n, V = 1 << 20, 5
    z, y = make(n, V, dtype, 1)
    q, want, H = formula(z, y, 1.0)
    lp, ent, st = forward(z, y, 1.0)
    near(lp, want, 4 * rel(V), 2 * U)
    near(ent, H, 6 * rel(V) * (1 + math.log(V)), 2 * U)
    g = torch.randn(n, generator=gen(2), device=DEV)
    dz = torch.full_like(z, 9.0)
    R.token_logprobs_backward(z, y, st, g, dz)
    err, step = gradient_tol(q, H, g, None, 1.0, dtype, V)
    near(dz, gradient(q, H, y, g, None, 1.0), err + (g.double().abs() * 2 * U)[:, None], step)
    offs = torch.arange(n + 1, device=DEV, dtype=torch.int32)
    mask = torch.ones(n, device=DEV, dtype=torch.bool)
    mask[-1] = False
    for m in (None, mask):
        out = torch.empty(8, device=DEV)
        R.policy_loss_logits(z, y, lp, g, out, lp.clone(), dz, seq_offsets=offs, aggregate="sequence_mean", mask=m)
        live = n if m is None else n - 1
        assert float(out[7]) == live
        # ratios are within U |lp| of 1
        w = -g.double()[:live]
        near(out[0], w.mean(), w.abs().mean() * U * float(lp.abs().max()) + 1e-9 * w.abs().mean(), 2 * U)
        err, step = gradient_tol(q[:live], H[:live], w / live, None, 1.0, dtype, V)
        near(dz[:live], gradient(q[:live], H[:live], y[:live], w / live, None, 1.0),
             err + ((w / live).abs() * (4 + lp[:live].abs()) * U)[:, None], step + 4 * U)
        assert m is None or not dz[-1].any()


def test_calls_without_rows():
    f = lambda *k: torch.full(k, 3.0, device=DEV)
    z, y = torch.empty(0, 7, device=DEV), torch.empty(0, device=DEV, dtype=torch.int32)
    R.token_logprobs(z, y, f(0), out_entropy=f(0), out_stats=f(0, 2))
    R.token_logprobs_backward(z, y, f(0, 2), f(0), torch.empty_like(z))
    for so in (None, torch.zeros(4, device=DEV, dtype=torch.int32)):
        out = f(8)
        R.policy_loss_logits(z, y, f(0), f(1 if so is None else 3), out, f(0), torch.empty_like(z), seq_offsets=so)
        assert not out.any()


def test_captured_call_makes_its_own_workspace():
    n, V = 300, 3000
    inputs = [make(n, V, BF, i) for i in range(3)]
    b = batch([100, 0, 200], 4, masked=0.2)
    f = lambda *k: torch.empty(*k, device=DEV)
    z, y = inputs[0][0].clone(), inputs[0][1].clone()

    def call(z, y, out, lp, dz):
        R.policy_loss_logits(z, y, b["old"], b["adv"], out, lp, dz, seq_offsets=b["offs"], mask=b["mask"],
                             aggregate="sequence_mean")
    want = []
    for zi, yi in inputs:
        o = (f(8), f(n), torch.empty_like(zi))
        call(zi, yi, *o)
        want.append(o)
    got = (f(8), f(n), torch.empty_like(z))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call(z, y, *got)
    for i in (1, 2, 0, 1):
        z.copy_(inputs[i][0])
        y.copy_(inputs[i][1])
        scratch = torch.full((1 << 20,), NAN, device=DEV)      # eager work between replays
        graph.replay()
        o = (f(8), f(n), torch.empty_like(z))
        call(*inputs[i], *o)
        torch.cuda.synchronize()
        for a, e, w in zip(got, o, want[i]):
            assert torch.equal(a, w) and torch.equal(e, w)
        del scratch


def test_most_tokens_and_pairs():
    n, pairs = 1 << 24, 1 << 19
    g = gen(7)
    lp = -4 * torch.rand(n, generator=g, device=DEV)
    old = lp + 0.05 * torch.randn(n, generator=g, device=DEV)
    mask = torch.rand(n, generator=g, device=DEV) < 0.7
    out, d = torch.empty(8, device=DEV), torch.empty(n, device=DEV)
    live = mask.double()
    for aggregate in ("token_mean", "sequence_mean"):       # one sequence: the same
        R.policy_loss(lp, old, torch.full((1,), -0.5, device=DEV), out, d, mask=mask, clip_low=0.9, clip_high=9.0,
                      aggregate=aggregate)
        pg = 0.5 * (lp.double() - old.double()).exp() * live / live.sum()
        near(out[0], pg.sum(), 1e-11, 2 * U)
        near(d, pg, 1e-18, 2 * U)
        assert float(out[7]) == float(live.sum())
    # pairs of 16 and 16 tokens
    offs = torch.arange(0, n + 1, 16, device=DEV, dtype=torch.int32)
    r = torch.empty(2 * pairs, device=DEV)
    R.preference_loss(lp, offs, out, d, ref_logp=old, mask=mask, out_rewards=r, beta=0.3)
    s = ((lp.double() - old.double()) * live).view(pairs, 2, 16).sum(2)
    near(r.view(pairs, 2), 0.3 * s, 1e-12, 2 * U)
    h = 0.3 * (s[:, 0] - s[:, 1])
    near(out[0], torch.nn.functional.softplus(-h).mean(), 1e-11, 2 * U)
    w = -0.3 * torch.sigmoid(-h) / pairs
    want = (torch.stack([w, -w], 1)[:, :, None] * live.view(pairs, 2, 16)).view(n)
    near(d, want, 1e-18, 2 * U)
