"""Pools whose offsets pass 32 bits: the same rows at their start and behind 4
GiB give the same bits."""
import pytest
import torch

from paper_2607_24788_amd import paged, paged4

from .test_gpu_append import frequencies
from .test_gpu_paged import nan_like

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
LENS, NEW = [130, 77], [70, 9]


def tables(first, count):
    t = torch.full((2, 10), -1, dtype=torch.int32)
    ids = torch.arange(count, dtype=torch.int32) + first
    t[0, :9], t[1, :5] = ids[:9].flip(0), ids[9:14]
    return t.cuda()


def rows(dtype):
    gen = torch.Generator().manual_seed(7)
    T = sum(NEW)
    return [torch.randn((T, h, 128), generator=gen).to(dtype).cuda() for h in (8, 2, 2)]


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_4_bit_cache(dtype):
    """Codes of 4.3 GB, 2^26 rows of 64 bytes and more."""
    P, Hkv, near = 16, 2, 16
    n_pages = (1 << 32) // (P * Hkv * 64) + near
    q, k, v = rows(dtype)
    got = []
    pools = None
    for first in (0, n_pages - 14):
        g = paged4.Paged4(2, 8, Hkv, 128, P, n_pages, 10, window=60, n_sinks=3, dtype=dtype)
        if pools is None:
            pools = g.new_pools()
        for codes, scales in pools:                # what is cached already, in the order of the table's pages
            gen = torch.Generator().manual_seed(8)
            codes[first:first + 14] = torch.randint(0, 256, (14, *codes.shape[1:]), generator=gen, dtype=torch.uint8).cuda()
            scales[first:first + 14] = torch.randint(120, 130, (14, *scales.shape[1:]), generator=gen, dtype=torch.uint8).cuda()
        c = g.cache(*pools, tables(first, 14), torch.tensor(LENS, dtype=torch.int32, device="cuda"))
        cu, ws, T = [0, NEW[0], sum(NEW)], g.new_workspace(sum(NEW)), sum(NEW)
        qo, out, one = nan_like(T, 8, 128, dtype=dtype), nan_like(T, 8, 128, dtype=dtype), nan_like(2, 8, 128, dtype=dtype)
        lse, ko, vo = nan_like(T, 8, dtype=FP32), nan_like(T, Hkv, 128, dtype=dtype), nan_like(T, Hkv, 128, dtype=dtype)
        g.append(c, k, v, cu, q=q, q_out=qo, freqs=frequencies(128).cuda())
        g.read(c, cu, ko, vo)
        g.prefill(c, qo, cu, out, ws, lse=lse)
        g.decode(c, qo[:2].contiguous(), one, ws)
        got.append([x.clone() for x in (qo, out, one, lse, ko, vo)] + [t[first:first + 14].clone() for p in pools for t in p])
    for x, y in zip(*got):
        assert torch.equal(x, y) and x.float().isfinite().all()


def test_bounds_and_sparse():
    """Pages of one token of 2^24 pages: bounds of 8 GiB, pools of 4."""
    P, Hkv, n_pages = 1, 2, (1 << 23) + 300
    dtype = BF16
    q, k, v = rows(dtype)
    got = []
    tensors = None
    for first in (0, n_pages - 250):
        g = paged.Paged(2, 8, Hkv, 128, P, n_pages, 140, dtype=dtype)
        if tensors is None:
            tensors = g.new_pools()[:2] + (g.new_bounds(),)
        kp, vp, bounds = tensors
        gen = torch.Generator().manual_seed(9)
        for pool in (kp, vp):
            pool[first:first + 250] = torch.randn((250, *pool.shape[1:]), generator=gen).to(dtype).cuda()
        table = torch.full((2, 140), -1, dtype=torch.int32)
        table[0, :130] = torch.arange(130) + first
        table[1, :77] = torch.arange(77) + first + 140
        c = g.cache(kp, vp, table.cuda(), torch.tensor(LENS, dtype=torch.int32, device="cuda"))
        cu, T = [0, NEW[0], sum(NEW)], sum(NEW)
        g.page_bounds(c, bounds)
        g.append(c, k, v, cu, bounds=bounds)
        out, lse = nan_like(T, 8, 128, dtype=dtype), nan_like(T, 8, dtype=FP32)
        sel = torch.full((T, Hkv, 20), 77, dtype=torch.int32, device="cuda")
        g.sparse(c, bounds, q, cu, 20, sel, out, g.new_sparse_workspace(T, 20), lse=lse)
        used = torch.cat([torch.arange(130), torch.arange(77) + 140]).cuda() + first
        got.append([x.clone() for x in (out, lse, sel)] + [x[used].clone() for x in (kp, vp, bounds)])
    for x, y in zip(*got):
        assert torch.equal(x, y) and x.float().isfinite().all()


def test_pages_of_one_token_by_the_million():
    """An append that keeps bounds has a workgroup for every page and KV head:
    2^24 of them, 2^32 threads, over several launches."""
    Hkv, T, n_seq = 16, 1 << 18, 4
    g = paged.Paged(n_seq, Hkv, Hkv, 64, 1, T * n_seq, T, dtype=BF16)
    kp, vp, _ = g.new_pools()
    bounds = g.new_bounds()
    table = torch.arange(T * n_seq, dtype=torch.int32, device="cuda").view(n_seq, T)
    c = g.cache(kp, vp, table, torch.full((n_seq,), T, dtype=torch.int32, device="cuda"))
    gen = torch.Generator(device="cuda").manual_seed(3)
    k = torch.empty((T * n_seq, Hkv, 64), dtype=BF16, device="cuda").normal_(generator=gen)
    for x in (kp, vp, bounds):
        x.fill_(float("nan"))
    g.append(c, k, k, [T * i for i in range(n_seq + 1)], bounds=bounds)
    assert torch.equal(kp.view_as(k), k) and torch.equal(vp.view_as(k), k)
    assert torch.equal(bounds[:, :, 0], k) and torch.equal(bounds[:, :, 1], k)


def test_sparse_rows_by_the_million():
    """2^24 rows of queries and KV heads, of which all but the last see nothing."""
    Hkv, T, P, lens = 8, 1 << 20, 256, [256, 77]
    g = paged.Paged(2, Hkv, Hkv, 64, P, 2, 1, dtype=BF16)
    gen = torch.Generator(device="cuda").manual_seed(4)
    kp, vp, _ = g.new_pools()
    for x in (kp, vp):
        x.normal_(generator=gen)
    c = g.cache(kp, vp, torch.tensor([[1], [0]], dtype=torch.int32, device="cuda"),
                torch.tensor(lens, dtype=torch.int32, device="cuda"))
    bounds = g.new_bounds()
    g.page_bounds(c, bounds)
    q = torch.empty((2 * T, Hkv, 64), dtype=BF16, device="cuda").normal_(generator=gen)
    out, lse = torch.full_like(q, float("nan")), torch.full((2 * T, Hkv), float("nan"), device="cuda")
    sel = torch.full((2 * T, Hkv, 1), 77, dtype=torch.int32, device="cuda")
    g.sparse(c, bounds, q, [0, T, 2 * T], 1, sel, out, g.new_sparse_workspace(2 * T, 1), n_first=0, lse=lse)
    for b, n in enumerate(lens):
        blind, seen = slice(b * T, (b + 1) * T - n), slice((b + 1) * T - n, (b + 1) * T)
        assert (sel[blind] == -1).all() and (out[blind] == 0).all() and (lse[blind] == float("-inf")).all()
        assert (sel[seen] == 0).all()
        # the rows that see something, by a call of their own
        few = [0, n if b == 0 else 0, n]
        o, l = torch.empty_like(q[seen]), torch.empty_like(lse[seen])
        s = torch.empty((n, Hkv, 1), dtype=torch.int32, device="cuda")
        g.sparse(c, bounds, q[seen].contiguous(), few, 1, s, o, g.new_sparse_workspace(n, 1), n_first=0, lse=l)
        scores = (q[seen].float().unsqueeze(1) * kp[1 - b, :, :n].float().transpose(0, 1)).sum(-1) / 8
        scores = scores.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1).unsqueeze(-1), float("-inf"))
        want = scores.double().logsumexp(1)
        # (fp32 sums of 64 products, 80 in all: 64 * 80 * 2^-24 / 8 each; outputs: weights and result, of both calls)
        assert (lse[seen].double() - want).abs().max() < 1e-4 and (l.double() - want).abs().max() < 1e-4
        assert out[seen].isfinite().all() and (out[seen].float() - o.float()).abs().max() < 4 * 2 ** -8 * 6
