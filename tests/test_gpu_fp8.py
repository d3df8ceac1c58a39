"""The 8-bit operators against their definitions in 64 bits (needs an MI355X).

Tolerances.  u = 2^-24 is half a step of fp32.
Codes of given numbers are exact: a scale is a power of two, so nothing is rounded but the code.  Codes of computed numbers
(norm, SwiGLU) are those of a number within (1 + delta) of the formula's: the scale byte and, under it, the code lie between
those of the numbers at either end.
A product of codes is exact in fp32; a sum of k of them, added one after the other with at most one step (2 u) lost each, is
within 2 k u sum |a w|.  Where the output is bf16 the matrix instruction may add eight products with 14 bits counted from the
leading bit of the largest: each loses less than 2^-13 of that, eight together less than 2^-10 of the eight's sum |a w|.
"""
import math

import pytest
import torch

import fp8_plain as F
from paper_2509_15965_amd import rl_decode as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")
EIGHTS = {F32: 0.0, BF: 2.0 ** -10}


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rows(n, k, dtype, seed, pad=0, shift=0, by=1.0):
    """[n][k] of numbers of uneven size, rows k + pad apart, `shift` entries past 16 bytes; the room between is NaN."""
    g = gen(seed)
    buf = torch.full((n * (k + pad) + shift + 8,), NAN, dtype=dtype, device=DEV)
    x = buf[shift:shift + n * (k + pad)].view(n, k + pad)[:, :k]
    x.copy_(torch.randn(n, k, generator=g, device=DEV) * torch.exp(2 * torch.randn(n, k, generator=g, device=DEV)) * by)
    return x


def room(n, k, weight=False, extra=0):
    """Codes and scales full of 0xA5, rows of codes `extra` blocks wider than needed."""
    kb = R.fp8_blocks(k)
    codes = torch.full((n, 128 * (kb + extra)), 0xA5, dtype=torch.uint8, device=DEV)
    scales = torch.full((R.fp8_blocks(n) if weight else n, (kb + 3) // 4 * 4 + 4 * extra), 0xA5, dtype=torch.uint8, device=DEV)
    return codes, scales


def check_outside(codes, scales, k):
    kb = R.fp8_blocks(k)
    assert (codes[:, 128 * kb:] == 0xA5).all() and (scales[:, kb:] == 0xA5).all()
    assert (codes[:, k:128 * kb] & 0x7F == 0).all()


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=1e9), torch.nan_to_num(b, nan=1e9))


def check_codes(codes, scales, v, delta):
    """codes, scales of v [n][k] (64 bits) when every number may be off by a factor 1 + delta."""
    k = v.shape[1]
    kb = R.fp8_blocks(k)
    a = F.finite_max(F.row_blocks(v), (2,))
    b = scales[:, :kb].int()
    lo, hi = F.scale_bytes(a * (1 - delta)), F.scale_bytes(a * (1 + delta))
    assert ((b == lo) | (b == hi)).all()
    got = F.code_values(codes[:, :128 * kb]).view(-1, kb, 128)
    x = F.row_blocks(v)
    p, q = (torch.nan_to_num(F.encode(x * f, b[..., None]).clamp(-448, 448), nan=1e9) for f in (1 - delta, 1 + delta))
    got = torch.nan_to_num(got, nan=1e9)
    assert ((got >= torch.minimum(p, q)) & (got <= torch.maximum(p, q))).all()


# ------------------------------------------------------------------------------------------------ quantiser


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,k,pad,shift", [(1, 1, 0, 0), (3, 127, 1, 0), (2, 128, 0, 3), (5, 129, 7, 1), (8, 256, 8, 0), (33, 688, 0, 0),
                                           (7, 1000, 3, 5), (513, 3584, 0, 0), (1, 131072, 0, 0), (2, 18944, 16, 8)])
def test_rows_are_exact(dtype, n, k, pad, shift):
    x = rows(n, k, dtype, n + k, pad, shift)
    codes, scales = room(n, k, extra=n % 2)
    R.quantise(x, codes, scales)
    check_codes(codes, scales, x.double(), 0.0)
    check_outside(codes, scales, k)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,k,pad,shift", [(1, 1, 0, 0), (127, 129, 1, 0), (128, 128, 0, 1), (129, 640, 0, 0), (300, 1000, 8, 0), (3584, 1536, 0, 0),
                                           (4608, 688, 0, 8), (1, 131072, 0, 0)])
def test_tiles_are_exact(dtype, n, k, pad, shift):
    x = rows(n, k, dtype, n + k, pad, shift)
    codes, scales = room(n, k, True, extra=n % 2)
    R.quantise(x, codes, scales, form="tiles")
    t = F.tile_blocks(x.double())
    want = F.scale_bytes(t.abs().amax((1, 3)))
    kb = R.fp8_blocks(k)
    assert torch.equal(scales[:, :kb].int(), want.int())
    vals = F.encode(t, want[:, None, :, None]).reshape(-1, 128 * kb)[:n]
    assert torch.equal(F.code_values(codes[:, :128 * kb]), vals)
    check_outside(codes, scales, k)


def special():
    """Blocks at the borders of the format, one a row."""
    r = torch.zeros(14, 128, dtype=torch.float32)
    r[1, 5] = 448.0                                         # scale 1, the largest code
    r[2, 5] = math.nextafter(448.0, 449.0) + 2 ** -15       # the next scale
    r[3, :16] = torch.arange(16) * 2.0 ** -10               # ties of subnormal codes beside 448
    r[3, 127] = -448.0
    r[4] = 3.4028234e38                                     # the largest number
    r[5, 7] = 2.0 ** -149                                   # the smallest
    r[6, 3] = 1.1754942e-38                                 # subnormal
    r[6, 4] = -(2.0 ** -130)
    r[7, 0], r[7, 1], r[7, 2], r[7, 3] = NAN, INF, -INF, 3.0
    r[8] = NAN
    r[9, 64] = -INF
    r[10] = torch.tensor([1.0, 1.0625, 1.1875, -1.3125] * 32)      # ties
    r[11, 1], r[11, 2] = 3e38, 1e-40                        # far apart
    r[12] = -0.0
    r[13, 0], r[13, 1] = 2.0 ** -118 * 1.75, 2.0 ** -118 * 1.7500002    # where the smallest scale begins
    return r


@pytest.mark.parametrize("form", ["rows", "tiles"])
def test_borders_of_the_format(form):
    for r in special().to(DEV):
        codes, scales = room(1, 128, form == "tiles")
        R.quantise(r[None].contiguous(), codes, scales, form=form)
        v = r[None].double()
        b = F.scale_bytes(F.finite_max(v, (1,)))[:, None]
        assert scales[0, 0].item() == b.item(), (r, scales[0, 0])
        assert same(F.code_values(codes), F.encode(v, b)), r


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n,k,pad,shift", [(1, 1, 0, 0), (3, 100, 0, 0), (2, 128, 5, 1), (5, 129, 0, 0), (65, 688, 0, 0), (9, 1001, 1, 0),
                                           (64, 8960, 0, 0), (512, 18944, 0, 0)])
def test_swiglu(dtype, n, k, pad, shift):
    """delta: e^-g within 2 steps (and |g| u where g log2(e) is rounded: 2 |g| u bounds it, |g| <= 100 before it is 0 or 1
    beside it), then four roundings: (2 * 100 + 10) u at most; where e^-g passes fp32 both are 0."""
    x = rows(n, 2 * k, dtype, n + k, pad, shift, 0.5).clamp_(-60, 60)
    codes, scales = room(n, k)
    R.quantise(x, codes, scales, form="swiglu")
    g, u = x[:, :k].double(), x[:, k:].double()
    check_codes(codes, scales, g * torch.sigmoid(g) * u, 210 * U)
    check_outside(codes, scales, k)


def test_swiglu_of_far_numbers():
    g = torch.tensor([[-200.0, 200.0, INF, -INF, NAN, 0.0, -90.0, 1e30]], device=DEV)
    u = torch.tensor([[2.0, 3.0, 1.0, 1.0, 1.0, INF, 1.0, 1e30]], device=DEV)
    codes, scales = room(1, 8)
    R.quantise(torch.cat([g, u], 1), codes, scales, form="swiglu")
    v = F.matrix(codes, scales)[0, :8]
    assert v[0].abs() < 1e-30 and abs(v[1].item() - 600.0) <= 600.0 * 2.0 ** -4
    assert torch.isnan(v[[2, 3, 4, 5, 7]]).all()


# ------------------------------------------------------------------------------------------------ norm


NORMS = [(1, 1, 0, 0), (3, 100, 0, 0), (8, 256, 0, 0), (5, 512, 1, 0), (7, 1000, 0, 3), (65, 1536, 0, 0), (4, 2048, 8, 0), (513, 3584, 0, 0),
         (3, 4096, 0, 8), (2, 4097, 0, 0), (9, 5120, 0, 0), (2, 8192, 0, 0), (3, 8193, 7, 0), (2, 32768, 0, 0),
         (37, 64, 0, 0), (33, 128, 3, 1), (70, 127, 0, 0), (6, 200, 0, 2), (3, 12288, 0, 0), (2, 16385, 0, 0), (2, 20000, 5, 0)]


@pytest.mark.parametrize("n,h,pad,shift", NORMS)
@pytest.mark.parametrize("dtype,add_dtype,w_dtype", [(F32, F32, F32), (F32, BF, BF), (BF, BF, BF), (BF, F32, F32), (F32, None, BF), (BF, None, F32)])
def test_norm(n, h, pad, shift, dtype, add_dtype, w_dtype):
    """delta: the sum of squares is of positive terms, a chain of at most 128 in a lane (two steps a term: product and sum) and
    9 joins: 265 u, its root half of that; division, root, reciprocal and two products: 6 u more."""
    x = rows(n, h, dtype, n + h, pad, shift)
    add = rows(n, h, add_dtype, n + h + 1, pad, 0) if add_dtype else None
    w = rows(1, h, w_dtype, 7, 0, shift)[0]
    total = torch.full((n, h + pad), NAN, dtype=dtype, device=DEV)[:, :h]
    codes, scales = room(n, h, extra=n % 2)
    R.rmsnorm_quant(x, w, codes, scales, add=add, out_sum=total, eps=1e-5)
    s = (x.float() + add.float()).to(dtype) if add_dtype else x
    assert torch.equal(total, s)
    s = s.double()
    y = s / torch.sqrt(s.square().mean(1, keepdim=True) + float(torch.tensor(1e-5))) * w.double()
    check_codes(codes, scales, y, (265 / 2 + 6) * U)
    check_outside(codes, scales, h)


@pytest.mark.parametrize("which", ["x", "add"])
def test_norm_sum_in_place(which):
    x, add = rows(6, 700, BF, 1, 4), rows(6, 700, BF, 2, 4)
    w = rows(1, 700, BF, 3)[0]
    want = room(6, 700)
    total = torch.empty_like(x)
    R.rmsnorm_quant(x, w, *want, add=add, out_sum=total)
    got = room(6, 700)
    to = x if which == "x" else add
    R.rmsnorm_quant(x, w, *got, add=add, out_sum=to)
    assert torch.equal(to, total) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def norm_64(s, w, eps):
    s = s.double()
    return s / torch.sqrt(s.square().mean(1, keepdim=True) + eps) * w.double()


@pytest.mark.parametrize("n,h", [(300, 64), (65, 130), (128, 896), (64, 3584), (32, 9000), (16, 32768)])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_norm_is_rounded_once(n, h, dtype):
    """Codes and scales are those of the formula in 64 bits: a number within 2^-48 of a border between two codes, where the two
    could differ, is one in 2^43 or fewer."""
    x, a = rows(n, h, dtype, 7), rows(n, h, BF, 8)
    w = rows(1, h, F32, 9)[0]
    s = torch.empty(n, h, dtype=dtype, device=DEV)
    codes, scales = room(n, h)
    R.rmsnorm_quant(x, w, codes, scales, add=a, out_sum=s, eps=1e-5)
    y = norm_64(s, w, 1e-5)
    kb = F.blocks(h)
    b = F.scale_bytes(F.finite_max(F.row_blocks(y), (2,)))
    assert torch.equal(scales[:, :kb].int(), b.int())
    assert torch.equal(F.code_values(codes).view(n, kb, 128), F.encode(F.row_blocks(y), b[..., None]))


def test_norm_of_rows_whose_squares_pass_fp32():
    x = torch.full((4, 300), 1e19, device=DEV)
    x[0] = 3e38
    x[1] = 1.0
    x[1, 7] = -2e19
    x[2, 299] = INF
    x[3] = 1e-30
    codes, scales = room(4, 300)
    w = torch.ones(300, device=DEV)
    R.rmsnorm_quant(x, w, codes, scales, eps=1e-40)
    v = F.matrix(codes, scales)[:, :300]
    y = norm_64(x, w, float(torch.tensor(1e-40, dtype=torch.float64)))
    keep = [0, 1, 3]
    b = F.scale_bytes(F.finite_max(F.row_blocks(y[keep]), (2,)))
    assert torch.equal(v[keep], (F.encode(F.row_blocks(y[keep]), b[..., None]) * F.factor(b.to(torch.uint8))[..., None]).flatten(1)[:, :300])
    assert (v[2, :299] == 0).all() and torch.isnan(v[2, 299])


def test_norm_of_rows_that_are_zero_or_not_finite():
    x = rows(5, 300, F32, 4)
    x[1] = 0.0
    x[2, 7] = NAN
    x[3, 9] = INF
    w = torch.ones(300, device=DEV)
    codes, scales = room(5, 300)
    R.rmsnorm_quant(x, w, codes, scales)
    v = F.matrix(codes, scales)[:, :300]
    assert (v[1] == 0).all() and (scales[1, :3] == 127).all()
    assert torch.isnan(v[2]).all()
    assert torch.isnan(v[3, 9]) and (v[3, :9] == 0).all() and (v[3, 10:] == 0).all()
    check_outside(codes, scales, 300)
    alone = room(1, 300)
    R.rmsnorm_quant(x[4:5], w, *alone)
    assert torch.equal(alone[0][0], codes[4]) and torch.isfinite(v[[0, 4]]).all()


# ------------------------------------------------------------------------------------------------ product


def whole_matrix(n, k, weight, seed):
    """Codes of whole numbers -3 .. 3 under scales 2^-2 .. 2^2: every sum is exact in fp32 up to k = 2^17."""
    kb = R.fp8_blocks(k)
    g = gen(seed)
    codes, scales = room(n, k, weight, extra=n % 2)
    v = torch.zeros(n, 128 * kb, device=DEV)
    v[:, :k] = torch.randint(-3, 4, (n, k), generator=g, device=DEV).float()
    codes[:, :128 * kb] = v.to(F.E4M3).view(torch.uint8)
    scales[:, :kb] = torch.randint(125, 130, (scales.shape[0], kb), generator=g, device=DEV).to(torch.uint8)
    return codes, scales


GEMMS = [(1, 1, 1), (1, 16, 128), (1, 2048, 1536), (1, 4097, 300), (2, 130, 18944), (3, 64, 129), (7, 200, 1000), (8, 3584, 3584), (15, 31, 640),
         (16, 1000, 256), (17, 4608, 3584), (24, 5000, 3584), (31, 129, 4096), (32, 256, 1280), (33, 300, 2048), (48, 513, 896), (64, 1000, 8960),
         (65, 129, 512), (100, 1000, 1536), (128, 256, 18944), (129, 385, 640), (200, 600, 8192), (255, 256, 384), (256, 512, 128), (257, 257, 257),
         (300, 4096, 1536), (512, 3584, 2048), (1000, 700, 1000), (1024, 1024, 3584), (2049, 1027, 896), (5, 40000, 256), (4100, 70, 3000),
         # more than 512 tiles of 128 x 128: large tiles, whole and with a last round cut into four, and small ones for few rows
         (1000, 9300, 300), (2100, 4301, 896), (512, 33001, 640), (770, 24600, 128), (40, 66000, 384),
         # up to 16 tokens, 16 and 32 weights a workgroup
         (12, 5003, 1000), (16, 8192, 384), (9, 8193, 384), (16, 12289, 200), (1, 65537, 130)]


@pytest.mark.parametrize("m,n,k", GEMMS)
def test_product_of_whole_numbers_is_exact(m, n, k):
    """|sums| <= 9 2^4 k and every term a multiple of 2^-4: within 24 bits up to k = 7281, where 2^-4 of 2^20 is left; above,
    the reference's own fp32 rounding is allowed, 2 k u of the terms' sum (see above)."""
    a, sa = whole_matrix(m, k, False, m + n)
    w, sw = whole_matrix(n, k, True, k + 1)
    kb = R.fp8_blocks(k)
    A, W = F.matrix(a[:, :128 * kb], sa), F.matrix(w[:, :128 * kb], sw, True)
    want = A @ W.t()
    for dtype in (F32, BF):
        pad = 3 if m % 2 else 0
        out = torch.full((m, n + pad), NAN, dtype=dtype, device=DEV)
        R.gemm_quant(a[:, :128 * kb], sa, w[:, :128 * kb], sw, out[:, :n])
        got = out[:, :n]
        if dtype == F32 and k <= 7281:
            assert torch.equal(got.double(), want), (got.double() - want).abs().max()
        elif k <= 7281:
            assert torch.equal(got, want.to(BF))
        else:
            tol = (2 * k * U + EIGHTS[dtype]) * (A.abs() @ W.abs().t()) + (want.abs() * 2.0 ** -8 if dtype == BF else 0)
            assert ((got.double() - want).abs() <= tol).all()
        assert torch.isnan(out[:, n:]).all()


@pytest.mark.parametrize("m,n,k", [(1, 500, 3584), (24, 1000, 3584), (64, 300, 2048), (130, 400, 8960), (700, 900, 4096)])
def test_product(m, n, k):
    x, y = rows(m, k, F32, 1), rows(n, k, F32, 2)
    a, w = room(m, k), room(n, k, True)
    R.quantise(x, *a)
    R.quantise(y, *w, form="tiles")
    A, W = F.matrix(*a), F.matrix(*w, True)
    want, size = A @ W.t(), A.abs() @ W.abs().t()
    for dtype, step in ((F32, 2.0 ** -24), (BF, 2.0 ** -8)):
        out = torch.empty(m, n, dtype=dtype, device=DEV)
        R.gemm_quant(*a, *w, out)
        assert ((out.double() - want).abs() <= (2 * k * U + EIGHTS[dtype]) * size + step * want.abs()).all()
        # the mean error is far below that bound: a rounding of a sum to fp32 a block, at most
        if dtype == F32:
            assert ((out.double() - want).norm() <= 2 * U * math.sqrt(k / 16) * size.norm())


@pytest.mark.parametrize("m", [1, 20, 200])
def test_product_of_scales_far_apart_and_nan(m):
    k, n = 640, 260
    a, sa = whole_matrix(m, k, False, 3)
    w, sw = whole_matrix(n, k, True, 4)
    a, w = a[:, :k].contiguous(), w[:, :k].contiguous()
    sa[0, :5] = torch.tensor([1, 60, 127, 190, 247], dtype=torch.uint8)
    sw[1, :5] = torch.tensor([247, 190, 127, 60, 1], dtype=torch.uint8)     # 2^-6 .. 2^-4 each: sums are exact in fp32
    w[5, 300] = 0x7F
    if m > 1:
        a[1, 600] = 0xFF
    want = F.matrix(a, sa) @ F.matrix(w, sw, True).t()
    out = torch.empty(m, n, dtype=F32, device=DEV)
    R.gemm_quant(a, sa, w, sw, out)
    assert torch.isnan(out[:, 5]).all() and (m == 1 or torch.isnan(out[1]).all())
    fine = torch.isfinite(want)
    fine[0, :128] = False      # 2^120 beside 2^-126: not exact
    fine[0, 256:] = False
    fine[1:, 128:256] = False
    assert torch.equal(out.double()[fine], want[fine])
    assert torch.isfinite(out[0, 128:256]).all() and torch.equal(out[0, 128:256].double(), want[0, 128:256])


def test_no_rows():
    a, w = room(0, 128), room(5, 128, True)
    R.gemm_quant(*a, *w, torch.empty(0, 5, device=DEV))
    x = torch.empty(0, 128, device=DEV)
    R.quantise(x, *a)
    R.rmsnorm_quant(x, torch.ones(128, device=DEV), *a)


# ------------------------------------------------------------------------------------------------ cache


class Cache:
    """A pool full of 0xFF (codes and scales that are no numbers) and a table of pages in random order."""

    def __init__(self, lens, page, heads, d, seed, spare=3):
        self.page, self.heads, self.d = page, heads, d
        need = [(n + page - 1) // page for n in lens]
        self.n_pages = sum(need) + spare
        perm = torch.randperm(self.n_pages, generator=gen(seed), device=DEV).int()
        self.table = torch.full((len(lens), max(need + [1])), -1, dtype=torch.int32, device=DEV)
        at = 0
        for i, k in enumerate(need):
            self.table[i, :k] = perm[at:at + k]
            at += k
        self.pool = torch.full((R.kv_quant_bytes(self.n_pages, page, heads, d),), 0xFF, dtype=torch.uint8, device=DEV)

    def append(self, seqs, pos, k, v, **kw):
        R.kv_quant_append(self.pool, self.table, seqs, pos, k, v, page_size=self.page, **kw)

    def numbers(self, seq, n):
        pos = torch.arange(n, device=DEV)
        a, b, c, e = F.places(self.page, self.heads, self.d, self.table, torch.full_like(pos, seq), pos)
        return F.cache_numbers(self.pool, a, c), F.cache_numbers(self.pool, b, e)


def packed(lens, starts):
    seqs = [i for i, n in enumerate(lens) for _ in range(n)]
    pos = [s + t for n, s in zip(lens, starts) for t in range(n)]
    return torch.tensor(seqs, dtype=torch.int32, device=DEV), torch.tensor(pos, dtype=torch.int32, device=DEV)


def kv(n, heads, d, dtype, seed, pad=0, shift=0):
    x = rows(n, 3 * heads * d, dtype, seed, pad, shift)
    return x[:, heads * d:2 * heads * d].unflatten(1, (heads, d)), x[:, 2 * heads * d:].unflatten(1, (heads, d))


CACHES = [([1], [0], 32, 1, 128, 0, 0), ([5, 1, 0, 40], [0, 31, 3, 9], 32, 2, 64, 0, 0), ([33, 100, 64], [0, 0, 128], 64, 4, 128, 0, 0),
          ([7, 8, 9, 16], [1, 8, 0, 7], 32, 3, 128, 3, 1), ([300], [5], 256, 8, 64, 0, 0), ([1] * 70, list(range(70)), 64, 4, 128, 0, 0),
          ([513, 2], [0, 4095], 4096, 2, 128, 8, 0), ([20, 30], [100, 3], 64, 5, 128, 0, 4)]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("lens,starts,page,heads,d,pad,shift", CACHES)
def test_cache_is_exact(dtype, lens, starts, page, heads, d, pad, shift):
    seqs, pos = packed(lens, starts)
    n = seqs.numel()
    c = Cache([s + k for s, k in zip(starts, lens)], page, heads, d, n)
    k, v = kv(n, heads, d, dtype, n, pad, shift)
    before = c.pool.clone()
    c.append(seqs, pos, k, v)
    touched = torch.zeros_like(c.pool, dtype=torch.bool)
    for x, at, sat in zip((k, v), F.places(page, heads, d, c.table, seqs, pos)[:2], F.places(page, heads, d, c.table, seqs, pos)[2:]):
        b = F.scale_bytes(x.double().abs().amax(2))
        assert torch.equal(c.pool[sat].int(), b.int())
        assert torch.equal(F.code_values(c.pool[at]), F.encode(x.double(), b[..., None]))
        touched[at] = True
        touched[sat] = True
    assert torch.equal(c.pool[~touched], before[~touched])
    order = torch.randperm(n, generator=gen(1), device=DEV)
    order = torch.cat([order, order[:3]])                       # the same place twice
    out = [torch.full((order.numel(), heads, d), NAN, dtype=dtype, device=DEV) for _ in range(2)]
    R.kv_quant_read(c.pool, c.table, seqs[order], pos[order], *out, page_size=page)
    for x, o in zip((k, v), out):
        b = F.scale_bytes(x.double().abs().amax(2))
        want = F.encode(x.double(), b[..., None]) * F.factor(b.to(torch.uint8))[..., None]
        assert torch.equal(o.double(), want[order])


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("order", ["single", "eights", "many"])
def test_cache_read_of_every_code_under_every_scale(dtype, order):
    """Numbers that the type does not hold are rounded to it: of bf16 below 2^-133, of either from 2^128 on."""
    n, page, heads, d = 508, 512, 33 if order == "many" else 1, 128
    c = Cache([n], page, heads, d, 0, 0)
    block = c.pool.view(1, -1)[0]
    i = torch.arange(n, device=DEV)
    seqs, pos = packed([n], [0])
    a, b, e, f = F.places(page, heads, d, c.table, seqs, pos)
    code = (128 * (i % 2)[:, None] + torch.arange(d, device=DEV)).to(torch.uint8)[:, None]
    block[a], block[b] = code, code
    block[e] = block[f] = (i // 2 + 1).to(torch.uint8)[:, None]
    if order == "single":
        pos, seqs = pos.flip(0), seqs
    out = [torch.empty(n, heads, d, dtype=dtype, device=DEV) for _ in range(2)]
    R.kv_quant_read(c.pool, c.table, seqs, pos, *out, page_size=page)
    for o, w in zip(out, c.numbers(0, n)):
        assert same(o.flip(0) if order == "single" else o, w.to(dtype))


def test_cache_tokens_in_any_order_and_one_by_one():
    lens, page, heads, d = [50, 41], 32, 2, 128
    seqs, pos = packed(lens, [0, 0])
    n = seqs.numel()
    k, v = kv(n, heads, d, BF, 5)
    whole = Cache(lens, page, heads, d, 9)
    whole.append(seqs, pos, k, v)
    mixed = Cache(lens, page, heads, d, 9)
    order = torch.randperm(n, generator=gen(2), device=DEV)
    mixed.append(seqs[order], pos[order], k[order], v[order])
    assert torch.equal(whole.pool, mixed.pool)
    single = Cache(lens, page, heads, d, 9)
    for i in range(n):
        single.append(seqs[i:i + 1], pos[i:i + 1], k[i:i + 1], v[i:i + 1])
    assert torch.equal(whole.pool, single.pool)


# (lengths, starts, page, heads, d, pad, shift): at least 16384 pairs of a token and a head
MANY = [([33, 100, 64, 1, 7, 8, 9, 16, 1, 1], [0, 0, 128, 5, 1, 8, 0, 7, 8, 15], 64, 96, 128, 0, 0), ([300, 1, 4], [5, 0, 28], 32, 64, 64, 3, 1),
        ([1] * 131, list(range(131)), 32, 128, 128, 0, 0), ([2100], [0], 4096, 8, 128, 8, 0), ([2047, 6], [4090, 2], 64, 8, 64, 0, 4),
        ([9, 15, 17, 23] * 40, [0, 7, 8, 1] * 40, 256, 7, 128, 1, 0)]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("lens,starts,page,heads,d,pad,shift", MANY)
def test_cache_of_many_tokens(dtype, lens, starts, page, heads, d, pad, shift):
    """In order, shuffled in parts, with tokens in between that have no place."""
    seqs, pos = packed(lens, starts)
    n = seqs.numel()
    assert n * heads >= 16384
    k, v = kv(n, heads, d, dtype, n, pad, shift)
    want = []
    for x in (k, v):
        b = F.scale_bytes(x.double().abs().amax(2))
        want.append(F.encode(x.double(), b[..., None]) * F.factor(b.to(torch.uint8))[..., None])
    some = torch.arange(n, device=DEV)
    some = torch.cat([some[:n // 3], some[n // 3:n // 2].flip(0), some[n // 2:]])
    gone = torch.zeros(n, dtype=torch.bool, device=DEV)
    gone[[n // 5, n - 1]] = True
    gone[n // 4:n // 4 + 9] = True
    for order, lost in ((torch.arange(n, device=DEV), None), (some, None), (torch.arange(n, device=DEV), gone)):
        c = Cache([s + m for s, m in zip(starts, lens)], page, heads, d, n)
        before = c.pool.clone()
        sq, ps = seqs[order], pos[order]
        ok = torch.ones(n, dtype=torch.bool, device=DEV)
        if lost is not None:
            sq, ps = torch.where(lost, -1, sq), torch.where(lost & (order % 2 == 0), -ps, ps)
            ok = ~lost
        kk, vv = (rows(n, 3 * heads * d, dtype, 0, pad, shift)[:, i * heads * d:(i + 1) * heads * d].unflatten(1, (heads, d)) for i in (1, 2))
        kk.copy_(k[order]), vv.copy_(v[order])
        c.append(sq, ps, kk, vv)
        a, b, e, f = F.places(page, heads, d, c.table, sq[ok], ps[ok])
        for w, at, sat in zip(want, (a, b), (e, f)):
            assert torch.equal(F.cache_numbers(c.pool, at, sat), w[order][ok])
            before[at], before[sat] = c.pool[at], c.pool[sat]
        assert torch.equal(c.pool, before)
        out = [torch.full((n, heads, d), NAN, dtype=dtype, device=DEV) for _ in range(2)]
        R.kv_quant_read(c.pool, c.table, sq, ps, *out, page_size=page)
        for w, o in zip(want, out):
            assert torch.equal(o.double(), torch.where(ok[:, None, None], w[order], 0.0))


def test_cache_of_many_tokens_past_the_pages():
    """A prompt of which a page in the middle is not there: nothing is written for it, and zeros are read."""
    n, page, heads, d = 2048, 64, 8, 128
    c = Cache([n], page, heads, d, 1, 0)
    c.table[0, 7], c.table[0, 20] = -1, c.n_pages
    seqs, pos = packed([n], [0])
    k, v = kv(n, heads, d, BF, 3)
    c.append(seqs, pos, k, v)
    ok = ((pos // page) != 7) & ((pos // page) != 20)
    a, b, e, f = F.places(page, heads, d, c.table, seqs[ok], pos[ok])
    written = torch.zeros_like(c.pool, dtype=torch.bool)
    for at in (a, b, e, f):
        written[at] = True
    assert (c.pool[~written] == 0xFF).all()
    out = [torch.full((n, heads, d), NAN, device=DEV) for _ in range(2)]
    R.kv_quant_read(c.pool, c.table, seqs, pos, *out, page_size=page)
    for o, at, sat in zip(out, (a, b), (e, f)):
        assert torch.equal(o[ok].double(), F.cache_numbers(c.pool, at, sat)) and (o[~ok] == 0).all() and (o[ok] != 0).any()


def test_cache_tokens_without_a_place():
    c = Cache([64, 64], 32, 2, 64, 1)
    c.table[1, 1] = c.n_pages            # no such page
    before = c.pool.clone()
    seqs = torch.tensor([-1, 2, 0, 0, 1, 0], dtype=torch.int32, device=DEV)
    pos = torch.tensor([0, 0, -1, 64, 40, 7], dtype=torch.int32, device=DEV)
    k, v = kv(6, 2, 64, F32, 3)
    c.append(seqs, pos, k, v)
    at = torch.cat([t.flatten() for t in F.places(32, 2, 64, c.table, seqs[5:], pos[5:])])
    changed = (c.pool != before).nonzero().flatten()
    assert torch.isin(changed, at).all() and changed.numel() > 0
    out = [torch.full((6, 2, 64), NAN, device=DEV) for _ in range(2)]
    R.kv_quant_read(c.pool, c.table, seqs, pos, *out, page_size=32)
    assert all((o[:5] == 0).all() and torch.isfinite(o[5]).all() and (o[5] != 0).any() for o in out)


# ------------------------------------------------------------------------------------------------ attention


def attend(c, q, lens, longest=None, seqs=None, **kw):
    out = torch.full((q.shape[0], q.shape[1], q.shape[2] + 8), NAN, dtype=q.dtype, device=DEV).flatten(1)
    o = out[:, :q.shape[1] * q.shape[2]].unflatten(1, q.shape[1:])
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    R.attention_quant(c.pool, c.table, q, ln, o, page_size=c.page, n_kv_heads=c.heads, scale=kw.pop("scale", q.shape[2] ** -0.5),
                      max_length=max(lens + [0]) if longest is None else longest, seqs=seqs, **kw)
    assert torch.isnan(out[:, q.shape[1] * q.shape[2]:]).all()
    return o


def check_attention(o, q, k, v, scale):
    """One row.  A score is a sum of d exact products (fp32 queries: of d times three, 2^-24 of a query lost), scaled and
    multiplied by log2(e): within (2 (3 d + 2) + 4) u of the terms' sum, at most `big`; a weight is within that, twice with the
    denominator's, and its own error: exponential (2 steps and the argument's rounding, inside the term above), sums over n positions
    (n / 128 + 64 steps), and 2^-16 (bf16) or 2^-23 (fp32) where it is split for the product with V.  What fp32 cannot hold is lost: a weight, or the rest of one, below 2^-126 may be
    0, which moves the result by at most 4 2^-126 n times the largest |v| (with one value the sum of them is that small itself)."""
    want, size, big = F.attention(q, k, v, scale)
    n, d = k.shape[0], q.shape[1]
    delta = 2 * ((2 * (3 * d + 2) + 4) * U * big + (n / 128 + 64) * 2 * U) + (2.0 ** -16 if q.dtype == BF else 2.0 ** -23)
    tol = size * (torch.exp(delta) - 1) + want.abs() * (2.0 ** -8 if q.dtype == BF else U) + 4 * 2.0 ** -126 * n * v.abs().max()
    err = (o.double() - want).abs()
    assert (err <= tol).all(), (err / tol).max()


ATTENTION = [([1], 32, 1, 1, 128), ([0, 1, 2, 31, 32, 33], 32, 2, 4, 64), ([63, 64, 65, 127, 128, 129, 0], 64, 2, 7, 128), ([500, 3], 256, 1, 16, 128),
             ([255, 256, 257, 1000], 32, 4, 5, 128), ([1023, 1024, 1025], 64, 8, 1, 64), ([3000, 17, 5000], 64, 2, 8, 128), ([40] * 40, 32, 4, 7, 128),
             ([9000], 4096, 1, 6, 64), ([300, 40], 64, 32, 1, 128)]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("lens,page,heads,group,d", ATTENTION)
def test_attention(dtype, lens, page, heads, group, d):
    c = Cache(lens, page, heads, d, len(lens))
    seqs, pos = packed(lens, [0] * len(lens))
    k, v = kv(seqs.numel(), heads, d, BF, 3)
    if seqs.numel():
        c.append(seqs, pos, k * 0.2, v)
    q = rows(len(lens), heads * group * d, dtype, 4, 3, 1, 0.3).unflatten(1, (heads * group, d))
    for longest in (None, c.table.shape[1] * page):
        o = attend(c, q, lens, longest)
        for i, n in enumerate(lens):
            if n == 0:
                assert (o[i] == 0).all()
            else:
                check_attention(o[i], q[i], *c.numbers(i, n), d ** -0.5)


def test_attention_rows_of_one_sequence():
    """Drafted tokens: rows of the same sequence, each with the length it sees; sequences that are not there."""
    heads, group, d, page = 2, 4, 128, 32
    c = Cache([200, 77], page, heads, d, 1)
    seqs, pos = packed([200, 77], [0, 0])
    c.append(seqs, pos, *kv(seqs.numel(), heads, d, BF, 3))
    rs = torch.tensor([0, 0, 1, 0, -1, 2, 1], dtype=torch.int32, device=DEV)
    lens = [197, 198, 77, 1, 5, 5, -3]
    q = rows(7, heads * group * d, BF, 4, 0, 0, 0.05).unflatten(1, (heads * group, d))
    o = attend(c, q, lens, seqs=rs)
    for i in range(4):
        check_attention(o[i], q[i], *c.numbers(int(rs[i]), lens[i]), d ** -0.5)
    assert (o[4:] == 0).all()


def test_attention_pages_that_are_not_there():
    heads, group, d, page = 2, 2, 64, 32
    c = Cache([160], page, heads, d, 1)
    seqs, pos = packed([160], [0])
    c.append(seqs, pos, *kv(160, heads, d, BF, 3))
    q = rows(1, heads * group * d, F32, 4, 0, 0, 0.3).unflatten(1, (heads * group, d))
    k, v = c.numbers(0, 160)
    gone = c.table.clone()
    c.table[0, 1], c.table[0, 3] = -1, c.n_pages
    o = attend(c, q, [150])
    keep = torch.cat([torch.arange(0, 32), torch.arange(64, 96), torch.arange(128, 150)]).to(DEV)
    check_attention(o[0], q[0], k[keep], v[keep], d ** -0.5)
    c.table[:] = -1
    assert (attend(c, q, [150]) == 0).all()
    c.table.copy_(gone)
    assert (attend(c, q, [150], 0) == 0).all()
    check_attention(attend(c, q, [150], 70)[0], q[0], k[:70], v[:70], d ** -0.5)      # taken as long as max_length


def test_attention_of_large_and_equal_scores():
    """Scores of several hundred, where all but the largest vanish, and scores that are all the same."""
    heads, group, d, page = 1, 8, 128, 64
    c = Cache([700], page, heads, d, 1)
    seqs, pos = packed([700], [0])
    k, v = kv(700, heads, d, BF, 3)
    c.append(seqs, pos, k.clamp(-4, 4), v)
    q = rows(1, heads * group * d, BF, 4, 0, 0, 1.0).unflatten(1, (group, d)).clamp(-8, 8)
    check_attention(attend(c, q, [700])[0], q[0], *c.numbers(0, 700), d ** -0.5)
    check_attention(attend(c, q, [700], scale=-0.3)[0], q[0], *c.numbers(0, 700), -0.3)
    check_attention(attend(c, q * 0, [700])[0], q[0] * 0, *c.numbers(0, 700), d ** -0.5)


def test_attention_of_nan():
    heads, group, d, page = 2, 3, 128, 32
    c = Cache([100], page, heads, d, 1)
    seqs, pos = packed([100], [0])
    k, v = kv(100, heads, d, BF, 3)
    k, v = k.clone(), v.clone()
    v[50, 1, 7] = NAN
    c.append(seqs, pos, k * 0.1, v)
    q = rows(1, heads * group * d, BF, 4, 0, 0, 0.3).unflatten(1, (heads * group, d)).clone()
    o = attend(c, q, [100])
    bad = torch.isnan(o[0])
    assert bad[3:, 7].all() and bad.sum() == 3
    assert not torch.isnan(attend(c, q, [50])).any()             # behind the row
    q[0, 1, 3] = NAN
    bad = torch.isnan(attend(c, q, [50]))[0]
    assert bad[1].all() and bad.sum() == d
    k[20, 0] = INF
    c.append(seqs, pos, k * 0.1, v)
    bad = torch.isnan(attend(c, q, [50]))[0]
    assert bad[:3].all() and not bad[3:].any()


def test_attention_past_two_gib():
    """A pool of over 4 GiB whose last pages hold the sequence."""
    heads, group, d, page = 8, 4, 128, 256
    block = F.block_bytes(page, d)
    n_pages = (9 << 29) // (heads * block) + 1
    pool = torch.full((n_pages * heads * block,), 0xFF, dtype=torch.uint8, device=DEV)
    c = Cache([600], page, heads, d, 1)
    c.pool, c.n_pages = pool, n_pages
    c.table[0] = torch.tensor([n_pages - 1, 0, n_pages - 2], dtype=torch.int32)
    seqs, pos = packed([600], [0])
    k, v = kv(600, heads, d, BF, 3)
    c.append(seqs, pos, k * 0.2, v)
    q = rows(1, heads * group * d, BF, 4, 0, 0, 0.3).unflatten(1, (heads * group, d))
    check_attention(attend(c, q, [600])[0], q[0], *c.numbers(0, 600), d ** -0.5)
    out = [torch.empty(600, heads, d, device=DEV) for _ in range(2)]
    R.kv_quant_read(c.pool, c.table, seqs, pos, *out, page_size=page)
    assert all(torch.equal(o.double(), w) for o, w in zip(out, c.numbers(0, 600)))


def test_attention_of_the_longest_row():
    """A row of nearly 2^31 positions in pages of 32, of which only the last three pages are there."""
    heads, group, d, page = 1, 2, 64, 32
    c = Cache([96], page, heads, d, 1)
    pages = c.table[0].clone()
    n_pages = (1 << 26) - 1
    c.table = torch.full((1, n_pages), -1, dtype=torch.int32, device=DEV)
    c.table[0, -3:] = pages
    seqs, pos = packed([96], [page * (n_pages - 3)])
    c.append(seqs, pos, *kv(96, heads, d, BF, 3))
    a, b, e, f = F.places(page, heads, d, c.table, seqs, pos)
    k, v = F.cache_numbers(c.pool, a, e), F.cache_numbers(c.pool, b, f)
    q = rows(1, group * d, BF, 4, 0, 0, 0.3).unflatten(1, (group, d))
    for gone in (0, 31, 70):
        check_attention(attend(c, q, [page * n_pages - gone], page * n_pages)[0], q[0], k[:96 - gone], v[:96 - gone], d ** -0.5)


# ------------------------------------------------------------------------------------------------ together


def rope(x, pos):
    """Rotate-half RoPE of [n][heads][d] in fp32 (theta 1e4)."""
    d = x.shape[2]
    a = pos.double()[:, None] * 1e4 ** (-torch.arange(0, d, 2, device=x.device).double() / d)
    c, s = a.cos().float()[:, None], a.sin().float()[:, None]
    p, q = x[..., :d // 2].float(), x[..., d // 2:].float()
    return torch.cat([p * c - q * s, q * c + p * s], 2).to(x.dtype)


class Layer:
    """One decoder layer in 8 bits on a batch of single tokens, with the buffers that it keeps."""

    def __init__(self, n, H, hq, hkv, d, ffn, lens, seed):
        self.n, self.H, self.hq, self.hkv, self.d, self.ffn, self.lens = n, H, hq, hkv, d, ffn, lens
        self.w = {}
        for i, (name, shape) in enumerate({"qkv": ((hq + 2 * hkv) * d, H), "o": (H, hq * d), "gate_up": (2 * ffn, H), "down": (H, ffn)}.items()):
            w = torch.randn(shape, generator=gen(seed + i), device=DEV, dtype=F32).div(math.sqrt(shape[1])).to(BF)
            self.w[name] = room(*shape, True)
            R.quantise(w, *self.w[name], form="tiles")
        self.norms = [rows(1, H, BF, seed + 9 + i, by=0.01)[0] + 1 for i in range(2)]
        self.cache = Cache([t + 1 for t in lens], 32, hkv, d, seed)
        seqs, pos = packed(lens, [0] * n)
        k, v = kv(seqs.numel(), hkv, d, BF, seed)
        self.cache.append(seqs, pos, k * 0.2, v * 0.2)
        self.seqs = torch.arange(n, dtype=torch.int32, device=DEV)
        self.pos = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.after = self.pos + 1
        e = lambda *s, t=BF: torch.empty(*s, dtype=t, device=DEV)
        self.qkv, self.att, self.branch, self.gate_up, self.down = e(n, (hq + 2 * hkv) * d), e(n, hq, d), e(n, H), e(n, 2 * ffn), e(n, H)
        self.a1, self.a2, self.a3, self.a4 = room(n, H), room(n, hq * d), room(n, H), room(n, ffn)
        self.sum = e(n, H, t=F32)
        need = max(R.lib().rl_gemm_quant_workspace_bytes(n, *s) for s in (((hq + 2 * hkv) * d, H), (H, hq * d), (2 * ffn, H), (H, ffn)))
        need = max(need, R.lib().rl_attention_quant_workspace_bytes(n, hkv, hq, d, max(lens) + 1), 1)
        self.ws = torch.empty(need, dtype=torch.uint8, device=DEV)

    def run(self, x):
        n, hq, hkv, d = self.n, self.hq, self.hkv, self.d
        R.rmsnorm_quant(x, self.norms[0], *self.a1)
        R.gemm_quant(*self.a1, *self.w["qkv"], self.qkv, workspace=self.ws)
        h = self.qkv.view(n, hq + 2 * hkv, d)
        self.q, self.k = rope(h[:, :hq], self.pos), rope(h[:, hq:hq + hkv], self.pos)
        R.kv_quant_append(self.cache.pool, self.cache.table, self.seqs, self.pos, self.k, h[:, hq + hkv:].contiguous(), page_size=32)
        R.attention_quant(self.cache.pool, self.cache.table, self.q, self.after, self.att, page_size=32, n_kv_heads=hkv, scale=d ** -0.5,
                          max_length=max(self.lens) + 1, workspace=self.ws)
        R.quantise(self.att.flatten(1), *self.a2)
        R.gemm_quant(*self.a2, *self.w["o"], self.branch, workspace=self.ws)
        R.rmsnorm_quant(x, self.norms[1], *self.a3, add=self.branch, out_sum=self.sum)
        R.gemm_quant(*self.a3, *self.w["gate_up"], self.gate_up, workspace=self.ws)
        R.quantise(self.gate_up, *self.a4, form="swiglu")
        R.gemm_quant(*self.a4, *self.w["down"], self.down, workspace=self.ws)
        return self.sum + self.down.float()


LAYERS = [(3, 256, 4, 2, 64, 688, [32, 0, 45]), (1, 1536, 12, 2, 128, 2240, [700]), (40, 512, 8, 1, 64, 1000, list(range(40)))]


@pytest.mark.parametrize("shape", LAYERS)
def test_a_layer(shape):
    """Every operator of the layer against its definition on the inputs that it was given there."""
    L = Layer(*shape, 5)
    x = rows(L.n, L.H, F32, 6, by=0.2)
    L.run(x)
    prod = lambda a, w: (F.matrix(*a) @ F.matrix(*L.w[w], True).t(), F.matrix(*a).abs() @ F.matrix(*L.w[w], True).abs().t())
    eps = float(torch.tensor(1e-6))
    normed = lambda s, w: s.double() / torch.sqrt(s.double().square().mean(1, keepdim=True) + eps) * w.double()
    check_codes(*L.a1, normed(x, L.norms[0]), 140 * U)
    for a, w, got, k in ((L.a1, "qkv", L.qkv, L.H), (L.a2, "o", L.branch, L.hq * L.d), (L.a3, "gate_up", L.gate_up, L.H), (L.a4, "down", L.down, L.ffn)):
        want, size = prod(a, w)
        assert ((got.double() - want).abs() <= (2 * k * U + EIGHTS[BF]) * size + 2.0 ** -8 * want.abs()).all(), w
    for i in range(L.n):
        check_attention(L.att[i], L.q[i], *L.cache.numbers(i, L.lens[i] + 1), L.d ** -0.5)
    check_codes(*L.a2, L.att.flatten(1).double(), 0.0)
    assert torch.equal(L.sum, x + L.branch.float())
    check_codes(*L.a3, normed(L.sum, L.norms[1]), 140 * U)
    g, u = L.gate_up[:, :L.ffn].double(), L.gate_up[:, L.ffn:].double()
    check_codes(*L.a4, g * torch.sigmoid(g) * u, 210 * U)


def test_a_layer_captured_and_on_another_stream():
    L = Layer(*LAYERS[1], 5)
    xs = [rows(L.n, L.H, F32, 6 + i, by=0.2) for i in range(4)]
    want = [L.run(x).clone() for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [L.run(x).clone() for x in xs]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    x = xs[0].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = L.run(x)
    for _ in range(2):
        for i in (2, 0, 3, 1):
            x.copy_(xs[i])
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[i])
            assert torch.equal(L.run(xs[(i + 1) % 4]), want[(i + 1) % 4])


def test_stream_argument_and_given_workspace():
    a, w = room(2, 8960), room(2048, 8960, True)
    R.quantise(rows(2, 8960, BF, 1), *a)
    R.quantise(rows(2048, 8960, BF, 2), *w, form="tiles")
    want = torch.empty(2, 2048, device=DEV)
    R.gemm_quant(*a, *w, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = torch.empty_like(want)
    R.gemm_quant(*a, *w, got, stream=side)
    need = R.lib().rl_gemm_quant_workspace_bytes(2, 2048, 8960)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    mine = torch.empty_like(want)
    R.gemm_quant(*a, *w, mine, workspace=ws[:need])
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(mine, want) and (ws[need:] == 0xFF).all()
    if need:
        with pytest.raises(R.RLError):
            R.gemm_quant(*a, *w, mine, workspace=ws[:need - 256])


def test_binding_refuses_wrong_tensors():
    x = torch.zeros(2, 256, device=DEV)
    c, s = R.empty_fp8(2, 256)
    w, sw = R.empty_fp8(5, 256, weight=True)
    table, pool = torch.zeros(1, 2, dtype=torch.int32, device=DEV), torch.zeros(R.kv_quant_bytes(2, 32, 2, 64), dtype=torch.uint8, device=DEV)
    i32 = torch.zeros(2, dtype=torch.int32, device=DEV)
    k = torch.zeros(2, 2, 64, device=DEV)
    R.kv_quant_append(pool, table, i32, torch.tensor([0, 1], dtype=torch.int32, device=DEV), k, k, page_size=32)
    for f in (lambda: R.quantise(x.half(), c, s), lambda: R.quantise(x, c[:1], s), lambda: R.quantise(x, c[:, :128], s), lambda: R.quantise(x, c, s[:, :1]),
              lambda: R.quantise(x, c.float(), s), lambda: R.quantise(x, c.cpu(), s), lambda: R.quantise(x[:, :255], c, s, form="swiglu"),
              lambda: R.quantise(x.t(), c, s), lambda: R.rmsnorm_quant(x, x[0, :200], c, s), lambda: R.rmsnorm_quant(x, x[0], c, s, add=x[:1]),
              lambda: R.rmsnorm_quant(x, x[0], c, s, out_sum=x.to(BF)), lambda: R.rmsnorm_quant(x, x[0].half(), c, s),
              lambda: R.gemm_quant(c, s, w, sw, torch.zeros(2, 4, device=DEV)), lambda: R.gemm_quant(c, s, w[:, :128], sw, torch.zeros(2, 5, device=DEV)),
              lambda: R.gemm_quant(c[:, :100], s, w, sw, torch.zeros(2, 5, device=DEV)), lambda: R.gemm_quant(c, s, w, sw, torch.zeros(5, 2, device=DEV).t()),
              lambda: R.kv_quant_append(pool, table, i32, i32[:1], k, k, page_size=32), lambda: R.kv_quant_append(pool, table, i32, i32, k, k[:1], page_size=32),
              lambda: R.kv_quant_append(pool, table, i32, i32, k, k, page_size=33), lambda: R.kv_quant_append(pool[:100], table, i32, i32, k, k, page_size=32),
              lambda: R.kv_quant_append(pool, table[0], i32, i32, k, k, page_size=32), lambda: R.kv_quant_append(pool, table, i32.long(), i32, k, k, page_size=32),
              lambda: R.kv_quant_read(pool, table, i32, i32, k.transpose(0, 1), k, page_size=32),
              lambda: R.attention_quant(pool, table, k, i32[:1], k, page_size=32, n_kv_heads=2, scale=1.0, max_length=4),
              lambda: R.attention_quant(pool, table, k, i32, k.to(BF), page_size=32, n_kv_heads=2, scale=1.0, max_length=4)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: R.attention_quant(pool, table, k, i32, k.clone(), page_size=32, n_kv_heads=2, scale=1.0, max_length=4),     # two rows, one sequence
              lambda: R.attention_quant(pool, table, k, i32, k.clone(), page_size=32, n_kv_heads=2, scale=1.0, max_length=65, seqs=i32),
              lambda: R.attention_quant(pool, table, k, i32, k.clone(), page_size=32, n_kv_heads=2, scale=NAN, max_length=4, seqs=i32),
              lambda: R.rmsnorm_quant(x, x[0], c, s, eps=0.0)):
        with pytest.raises(R.RLError):
            f()
