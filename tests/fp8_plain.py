"""The 8-bit format and its operators in 64 bits, from their definitions (tests only; on any device)."""
import math

import torch

E4M3 = torch.float8_e4m3fn


def power(e):
    """2^e in 64 bits, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def scale_bytes(a):
    """Scale byte of blocks of largest finite magnitude a (fp64)."""
    m, e = torch.frexp(a)                     # a = m 2^e, m in [1/2, 1); 448 = 0.875 2^9
    b = e - 9 + (m > 0.875).int() + 127
    return torch.where(a > 0, b.clamp(min=1), torch.full_like(b, 127))


def round_e4m3(x):
    """Nearest e4m3 numbers, ties to even, of |x| <= 448; NaN stays."""
    _, e = torch.frexp(torch.where(torch.isfinite(x), x, 0.0))
    step = power((e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def code_values(codes):
    """Numbers that codes stand for, from their bits: sign, four bits of exponent, three of significand."""
    c = codes.view(torch.uint8).long()
    s, e, f = c >> 7, (c >> 3) & 15, c & 7
    v = torch.where(e > 0, (8 + f).double() * power(e - 10), f.double() * 2.0 ** -9)
    v = torch.where((e == 15) & (f == 7), math.nan, v)
    return torch.where(s > 0, -v, v)


def factor(scales):
    return power(scales.view(torch.uint8).int() - 127)


def finite_max(v, dims):
    return torch.where(torch.isfinite(v), v, 0.0).abs().amax(dims)


def blocks(k):
    return (k + 127) // 128


def row_blocks(v):
    n, k = v.shape
    return torch.nn.functional.pad(v, (0, 128 * blocks(k) - k)).view(n, blocks(k), 128)


def tile_blocks(v):
    """[n][k] as [row tiles][128][blocks][128], padded with 0."""
    n, k = v.shape
    nb, kb = blocks(n), blocks(k)
    return torch.nn.functional.pad(v, (0, 128 * kb - k, 0, 128 * nb - n)).view(nb, 128, kb, 128)


def encode(v, bytes_):
    """Code values of v under scale bytes that broadcast to it; what is not finite is NaN."""
    return round_e4m3(torch.where(torch.isfinite(v), v / factor(bytes_.to(torch.uint8)), math.nan))


def matrix(codes, scales, weight=False):
    """The numbers of a matrix in 8 bits."""
    n, kb = codes.shape[0], codes.shape[1] // 128
    f = factor(scales[:, :kb])
    if weight:
        f = f.repeat_interleave(128, 0)[:n]
    return (code_values(codes).view(n, kb, 128) * f[:, :, None]).flatten(1)


def block_bytes(page, d):
    return (2 * page * (d + 1) + 255) // 256 * 256


def places(page, heads, d, table, seqs, pos):
    """Byte offsets in the pool: K codes, V codes [n][heads][d], K scales, V scales [n][heads]."""
    t = (pos.long() % page)[:, None]
    at = (table.long()[seqs.long(), pos.long() // page][:, None] * heads + torch.arange(heads, device=pos.device)) * block_bytes(page, d)
    i = torch.arange(d, device=pos.device)
    return ((at + t * d)[..., None] + i, (at + page * d + (t // 8) * 8 * d + t % 8)[..., None] + 8 * i,
            at + 2 * page * d + t, at + 2 * page * d + page + t)


def cache_numbers(pool, at, sat):
    return code_values(pool[at]) * factor(pool[sat])[..., None]


def attention(q, k, v, scale):
    """(out, weights' sum of |v|, largest sum of |q k|) of q [Hq][d] over k, v [n][Hkv][d] in 64 bits."""
    hq, d = q.shape
    hkv = k.shape[1]
    q = q.double().view(hkv, hq // hkv, d)
    k, v = k.transpose(0, 1).contiguous(), v.transpose(0, 1).contiguous()
    p = torch.softmax(scale * torch.matmul(q, k.transpose(1, 2).contiguous()), 2)
    big = torch.matmul(q.abs(), k.abs().transpose(1, 2).contiguous()).amax(2, keepdim=True) * abs(scale)
    return (torch.matmul(p, v).reshape(hq, d), torch.matmul(p, v.abs()).reshape(hq, d),
            big.expand(-1, -1, d).reshape(hq, d))
