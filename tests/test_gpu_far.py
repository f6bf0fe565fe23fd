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
