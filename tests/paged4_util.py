"""The position rotation and the 4-bit cache in plain float64 on the CPU, from
the definitions in include/glide.h, and a 4-bit cache for the tests."""
import math

import torch

from paper_2607_24788_amd import paged4

from .paged_util import EPS16, EPS32, Ref, tables

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def rotate(x, pos, freqs, interleaved, dtype):
    """x [T][H][d] at positions pos [T]: the rotated rows in 64 bits, and how
    far the library's may be off: half a step of dtype, and in fp32 the
    fraction of a turn (half a step of a number up to 1/2, times 2 pi: 1.6 half
    steps of 1), sine and cosine (2 units in the last place: 4 half steps), two
    products and their sum (2); the turns themselves are fp64, three roundings."""
    x = x.double()
    tol = torch.zeros_like(x)
    if freqs is None:
        return x, tol
    f = freqs.double()
    a = pos.double()[:, None] * f
    # the angle's part of a turn, apart from a whole number of them: sine and cosine of it are exact enough at any
    # position that fp64 holds the product for (2^31 * a 24-bit frequency: 2 bits lost of 2^-53)
    cos, sin = a.cos()[:, None], a.sin()[:, None]
    r, y = 2 * f.numel(), x.clone()
    if interleaved:
        u, v = slice(0, r, 2), slice(1, r, 2)
    else:
        u, v = slice(0, r // 2), slice(r // 2, r)
    y[..., u] = x[..., u] * cos - x[..., v] * sin
    y[..., v] = x[..., v] * cos + x[..., u] * sin
    size = x[..., u].abs() + x[..., v].abs()
    off = size * (8 * EPS32 + 4 * 2.0 ** -53 * a.abs()[:, None])
    tol[..., u] = off
    tol[..., v] = off
    return y, tol


def rounding(y, dtype):
    return (EPS16 if dtype == torch.bfloat16 else EPS32) * y.abs()


def exponents(amax):
    """The least e in [-124, 125] with amax <= 7 * 2^e."""
    e = torch.full(amax.shape, -124, dtype=torch.int64)
    for k in range(-124, 125):
        e[amax > 7 * math.ldexp(1.0, k)] = k + 1
    return e


def levels(a):
    """Places in LEVELS nearest to a >= 0, ties to the even place."""
    d = (a[..., None] - LEVELS).abs()
    best = d.min(-1, keepdim=True).values
    near = d == best
    near[a == math.inf] = torch.arange(8) == 7
    place = torch.arange(8).expand(near.shape)
    odd = torch.where(near, place % 2, 9)
    even = (odd == odd.min(-1, keepdim=True).values) & near
    return torch.where(even, place, 99).min(-1).values


def quantise(x):
    """x [..][d] (any type) -> codes [..][d/2], scales [..][d/32] (uint8)."""
    g = x.double().unflatten(-1, (-1, 32))
    g = torch.where(g.isnan(), 0.0, g)
    e = exponents(g.abs().amax(-1))
    code = levels(g.abs() * torch.exp2(-e.double())[..., None]) + 8 * (g < 0)
    code = code.flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), (e + 127).to(torch.uint8)


def values(codes, scales):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    x = torch.where(c >= 8, -LEVELS[c % 8], LEVELS[c % 8])
    s = scales.long().clamp(3, 252).double() - 127
    return x * torch.exp2(s).repeat_interleave(32, -1)


class Case4:
    """A layer over a 4-bit cache on the device: slots without a token hold
    random bytes (scales out of range among them), pages in mixed order."""

    def __init__(self, B, Hq, Hkv, d, page, lens, window=None, sinks=0, dtype=torch.bfloat16, seed=0, extra_pages=1,
                 scale=1.0, sm_scale=None):
        self.gen = torch.Generator().manual_seed(900 + seed)
        counts = [-(-n // page) for n in lens]
        wide = max(max(counts), 1) + extra_pages
        n_pages = sum(counts) + 3
        self.g = g = paged4.Paged4(B, Hq, Hkv, d, page, n_pages, wide, window=window, n_sinks=sinks, dtype=dtype,
                                   sm_scale=sm_scale)
        self.lens_host, self.dtype, self.scale = list(lens), dtype, scale
        self.table = tables(self.gen, B, wide, counts, n_pages)
        pools = []
        for _ in range(2):
            codes = torch.randint(0, 256, (n_pages, Hkv, page, d // 2), generator=self.gen, dtype=torch.uint8)
            scales = torch.randint(0, 256, (n_pages, Hkv, page, d // 32), generator=self.gen, dtype=torch.uint8)
            scales[torch.rand(scales.shape, generator=self.gen) < 0.3] = 255
            for b, n in enumerate(lens):
                for i in range(counts[b]):
                    m, p = min(page, n - i * page), int(self.table[b, i])
                    codes[p, :, :m], scales[p, :, :m] = quantise(torch.randn((Hkv, m, d), generator=self.gen) * scale)
            pools.append((codes.cuda(), scales.cuda()))
        self.k, self.v = pools
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.dev_table = self.table.cuda()
        self.cache = g.cache(self.k, self.v, self.dev_table, self.lens)

    def normal(self, *shape):
        return (torch.randn(shape, generator=self.gen) * self.scale).to(self.dtype)

    def ref(self):
        k, v = (values(*(t.cpu() for t in pool)) for pool in (self.k, self.v))
        return Ref4(self.g, k, v, self.dev_table, self.lens)


class Ref4(Ref):
    """Ref with the error bounds of the 4-bit cache's rows.  In fp32 queries
    and weights go in as three parts: three times the additions."""

    def row(self, b, t, q, score=False):
        g = self.g
        G, d = g.n_q_heads // g.n_kv_heads, g.head_dim
        out, lse, tol, ztol = super().row(b, t, q, False)
        if g.torch_dtype == torch.bfloat16 or not lse.isfinite().any():
            return out, lse, tol, ztol
        seen = [j for j in range(min(t + 1, self.lens[b])) if j > t - g.window or j < g.n_sinks]
        pg, sl = torch.tensor([x for x in (self.slot(b, j) for j in seen) if x is not None]).T
        k, v = self.k[pg, :, sl], self.v[pg, :, sl]
        q = q.double().view(g.n_kv_heads, G, d)
        s = torch.einsum("hgd,nhd->hgn", q, k) * g.sm_scale
        size = torch.einsum("hgd,nhd->hgn", q.abs(), k.abs()) * abs(g.sm_scale)
        p = torch.exp(s - lse.view(g.n_kv_heads, G, 1))
        dl = ((3 * d + 4) * EPS32 * size.amax(-1)).view(-1) + (3 * len(pg) + 16) * EPS32
        part = torch.einsum("hgn,nhd->hgd", p, v.abs()).reshape(g.n_q_heads, d)
        return out, lse, part * (2 * dl)[:, None] + EPS32 * out.abs(), dl + 4 * EPS32 * (1 + lse.abs())
