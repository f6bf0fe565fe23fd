"""A paged cache for the tests, and its operators in plain float64 on the CPU
(from the definition in include/glide.h: one token at a time is looked up
through the block table, and every sum runs over the visible tokens only)."""
import math

import torch

from paper_2607_24788_amd import paged

EPS32 = 2.0 ** -24   # half a step of fp32, relative
EPS16 = 2.0 ** -8    # of bf16


def seen(t, n, W, ns):
    """Positions that the query at t sees, of n cached tokens."""
    return [j for j in range(min(t + 1, n)) if j > t - W or j < ns]


class Ref:
    """float64 copies of one layer's pools, and the operators on them."""

    def __init__(self, g, k, v, table, lens, w=None):
        self.g, self.table, self.lens = g, table.cpu().long(), [int(x) for x in lens.cpu()]
        self.k, self.v = k.cpu().double().contiguous(), v.cpu().double().contiguous()
        self.w = None if w is None else w.cpu().double()
        self.cap = g.max_pages * g.page_size
        self.lens = [min(max(x, 0), self.cap) for x in self.lens]

    def slot(self, b, j, table=None):
        p = int((self.table if table is None else table)[b, j // self.g.page_size])
        return (p, j % self.g.page_size) if 0 <= p < self.g.n_pages else None

    def append(self, b, j, k, v):
        at = self.slot(b, j) if j >= 0 else None
        if at is None:
            return
        p, s = at
        self.k[p, :, s], self.v[p, :, s] = k.double(), v.double()
        if self.w is not None:
            self.w[p, :, s] = 0.0

    def row(self, b, t, q, score):
        """The query at position t of sequence b: out [Hq][d], lse [Hq], and
        the bounds of their errors; score: its weights are added up."""
        g = self.g
        G, d = g.n_q_heads // g.n_kv_heads, g.head_dim
        at = [x for x in (self.slot(b, j) for j in seen(t, self.lens[b], g.window, g.n_sinks)) if x is not None] \
            if t >= 0 else []
        if not at:
            z = torch.zeros(g.n_q_heads, d, dtype=torch.float64)
            return z, torch.full((g.n_q_heads,), -math.inf, dtype=torch.float64), z, torch.zeros(g.n_q_heads)
        pg, sl = torch.tensor(at).T
        k, v = self.k[pg, :, sl], self.v[pg, :, sl]              # [n][Hkv][d]
        q = q.double().view(g.n_kv_heads, G, d)
        s = torch.einsum("hgd,nhd->hgn", q, k) * g.sm_scale
        size = torch.einsum("hgd,nhd->hgn", q.abs(), k.abs()) * abs(g.sm_scale)
        lse = torch.logsumexp(s, -1)
        p = torch.exp(s - lse[..., None])
        out = torch.einsum("hgn,nhd->hgd", p, v)
        if score:
            self.w[pg, :, sl] += p.sum(1).T
        # a score: d products and sums rounded in fp32, and its scaling
        ds = ((d + 4) * EPS32 * size.amax(-1)).view(-1)
        # a sum over n weights in fp32, each through one exponential
        dl = ds + (len(at) + 16) * EPS32
        part = torch.einsum("hgn,nhd->hgd", p, v.abs()).reshape(g.n_q_heads, d)
        out = out.reshape(g.n_q_heads, d)
        tol = part * (2 * dl)[:, None]
        if g.torch_dtype == torch.bfloat16:      # the weights and the output rounded to bf16
            tol = tol + EPS16 * part + EPS16 * out.abs()
        else:
            tol = tol + EPS32 * out.abs()
        # log of the sum, in the log2 domain and back
        return out, lse.reshape(-1), tol, dl + 4 * EPS32 * (1 + lse.reshape(-1).abs())

    def evict(self, budget, recent, dst=None):
        """Kept positions [B][Hkv][budget], new lens; moves the rows."""
        g = self.g
        kept = torch.full((g.batch, g.n_kv_heads, budget), -1, dtype=torch.int32)
        k, v, w = self.k.clone(), self.v.clone(), self.w.clone()
        for b, n in enumerate(self.lens):
            m = min(n, budget)
            for h in range(g.n_kv_heads):
                fixed = {j for j in range(n) if j < g.n_sinks or j >= n - recent}

                def rank(j):
                    at = self.slot(b, j)
                    x = float(w[at[0], h, at[1]]) if at else math.nan
                    return (2, 0.0) if math.isnan(x) else (1, -x)
                free = sorted((j for j in range(n) if j not in fixed), key=lambda j: (rank(j), j))
                keep = list(range(n)) if n <= budget else sorted(sorted(fixed) + free[:m - len(fixed)])
                for i, j in enumerate(keep):
                    kept[b, h, i] = j
                    src, to = self.slot(b, j), self.slot(b, i, dst)
                    if to is None:
                        continue
                    self.k[to[0], h, to[1]] = k[src[0], h, src[1]] if src else 0.0
                    self.v[to[0], h, to[1]] = v[src[0], h, src[1]] if src else 0.0
                    self.w[to[0], h, to[1]] = w[src[0], h, src[1]] if src else 0.0
        self.lens = [min(n, budget) for n in self.lens]
        if dst is not None:
            self.table = dst
        return kept, torch.tensor(self.lens, dtype=torch.int32)


def tables(gen, B, max_pages, counts, n_pages, first=0):
    """[B][max_pages] of distinct pages in mixed order, -1 behind the last."""
    ids = torch.randperm(n_pages - first, generator=gen)[:sum(counts)] + first
    t = torch.full((B, max_pages), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(counts):
        t[b, :n] = ids[at:at + n].int()
        at += n
    return t


class Case:
    """A layer on the device: pools whose unused slots hold NaN, a block table
    in mixed order, lens, and weights if asked for."""

    def __init__(self, B, Hq, Hkv, d, page, lens, window=None, sinks=0, dtype=torch.bfloat16, weights=False, seed=0,
                 extra_pages=1, scale=1.0, order="hnd", sm_scale=None):
        self.gen = torch.Generator().manual_seed(100 + seed)
        counts = [-(-n // page) for n in lens]
        wide = max(max(counts), 1) + extra_pages
        n_pages = sum(counts) + 3
        self.g = g = paged.Paged(B, Hq, Hkv, d, page, n_pages, wide, window=window, n_sinks=sinks, dtype=dtype,
                                 sm_scale=sm_scale)
        self.lens_host, self.dtype, self.scale = list(lens), dtype, scale
        self.table = tables(self.gen, B, wide, counts, n_pages)
        k, v = (torch.full((n_pages, Hkv, page, d), math.nan, dtype=dtype) for _ in range(2))
        w = torch.full((n_pages, Hkv, page), math.nan) if weights else None
        for b, n in enumerate(lens):
            for i in range(counts[b]):
                m = min(page, n - i * page)
                p = int(self.table[b, i])
                k[p, :, :m] = self.normal(Hkv, m, d)
                v[p, :, :m] = self.normal(Hkv, m, d)
                if weights:
                    w[p, :, :m] = torch.rand(Hkv, m, generator=self.gen)
        if order == "nhd":      # a pool stored [page][slot][head][d], seen as [page][head][slot][d]
            k, v = (x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (k, v))
        elif order == "joined":  # K and V of a page side by side
            kv = torch.stack([k, v], 1).cuda()
            k, v = kv[:, 0], kv[:, 1]
        else:
            k, v = k.cuda(), v.cuda()
        self.k, self.v, self.w = k, v, None if w is None else w.cuda()
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.dev_table = self.table.cuda()
        self.cache = g.cache(self.k, self.v, self.dev_table, self.lens, self.w)

    def normal(self, *shape):
        return (torch.randn(shape, generator=self.gen) * self.scale).to(self.dtype)

    def ref(self):
        return Ref(self.g, self.k, self.v, self.dev_table, self.lens, self.w)

    def pools_equal(self, ref):
        """K and V of the device against the reference's, bit for bit (NaN slots too)."""
        for name, x, y in (("K", self.k, ref.k), ("V", self.v, ref.v)):
            x = x.cpu().double()
            same = (x == y) | (x.isnan() & y.isnan())
            assert same.all(), f"{name} pool: {int((~same).sum())} elements differ"

    def weights_close(self, ref, rel=0.0):
        x, y = self.w.cpu().double(), ref.w
        assert torch.equal(x.isnan(), y.isnan()), "weights written where no token is, or not written"
        bad = ((x - y).abs() > rel * y.abs() + 1e-7).logical_and(~y.isnan())
        assert not bad.any(), f"weights: {int(bad.sum())} off, most {float((x - y).nan_to_num().abs().max()):.3e}"


def check_rows(got, lse, want):
    """Device rows against (out, lse, tol, lse tol) of the reference."""
    got, lse = got.cpu().double(), lse.cpu().double()
    for i, (o, z, tol, ztol) in enumerate(want):
        bad = (got[i] - o).abs() > tol + 1e-30
        assert torch.isfinite(got[i]).all(), f"row {i}: not finite"
        assert not bad.any(), (f"row {i}: off by {float((got[i] - o).abs().max()):.3e}, "
                               f"allowed {float(tol.max()):.3e}")
        none = z == -math.inf
        assert (lse[i][none] == -math.inf).all(), f"row {i}: lse of an empty row"
        assert ((lse[i] - z)[~none].abs() <= ztol[~none]).all(), \
            f"row {i}: lse off by {float((lse[i] - z)[~none].abs().max()):.3e}, allowed {float(ztol[~none].max()):.3e}"
