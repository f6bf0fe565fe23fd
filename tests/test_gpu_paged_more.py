"""Calls of the paged softmax cache beside tests/test_gpu_paged.py's, against
the same float64 definition (tests/paged_util.py)."""
import math

import pytest
import torch

from .paged_util import EPS16, EPS32, Case
from .test_gpu_paged import nan_like, run_decode, run_evict, run_prefill

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("call", ["prefill", "decode"])
def test_tokens_written_by_the_caller(dtype, call):
    """Rows that a caller writes into new pools itself: their weights add up
    from new_pools' zeros, on memory that held NaN before."""
    case = Case(2, 8, 2, 128, 16, [200, 90], 70, 2, dtype=dtype, weights=True, seed=120)
    g = case.g
    size = case.k.numel()
    del case.cache
    held = torch.full((4 * size,), float("nan"), device="cuda")      # for the allocator to give out again
    del held
    k, v, w = g.new_pools(weights=True)
    k.copy_(case.k)
    v.copy_(case.v)
    case.k, case.v, case.w = k, v, w
    case.cache = g.cache(k, v, case.dev_table, case.lens, w)
    if call == "prefill":
        run_prefill(case, [33, 90], 20, append=False)
    else:
        run_decode(case, False)
    assert case.w.isfinite().all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("sinks,recent,budget", [(20, 0, 90), (0, 30, 60), (0, 0, 150), (4, 8, 500)])
def test_kept_tokens_on_missing_pages(dtype, sinks, recent, budget):
    """Sinks, newest tokens or all of a budget on pages that are not
    allocated: rows of zeros where they move, which the next query sees with a
    score of 0; tokens that stay where they are stay missing."""
    case = Case(2, 8, 2, 128, 16, [160, 100], None, sinks, dtype=dtype, weights=True, seed=121)
    for i in (1, 4, 9):
        case.table[0, i] = -1
    case.table[1, 5] = case.g.n_pages
    case.dev_table.copy_(case.table)
    ref = run_evict(case, budget, recent, alias=True)
    case.lens_host = list(ref.lens)
    run_decode(case, False)


@pytest.mark.parametrize("dtype,page,Hq,Hkv,new,hist,W", [
    (BF16, 16, 8, 2, 0, 2100, None), (FP32, 16, 8, 2, 0, 2100, None), (BF16, 1, 4, 4, 0, 700, 500),   # decode
    (BF16, 16, 8, 2, 7, 2100, None), (BF16, 32, 8, 2, 150, 200, 70),      # attend_tiles
    (FP32, 16, 8, 2, 7, 1500, None), (FP32, 16, 4, 2, 40, 61, 30),        # attend_rows
    (BF16, 4, 4, 2, 33, 600, None),
    (FP32, 64, 32, 16, 450, 100, 300), (BF16, 8, 32, 16, 450, 0, None)])  # attend_shared
@pytest.mark.parametrize("hint", [True, False])
def test_nonfinite_values_of_underflowed_weight(dtype, page, Hq, Hkv, new, hist, W, hint):
    """Infinite and NaN values of tokens that a row sees at a score far below
    its largest (2^-185 of its weight): their elements are not finite, however
    a row is split and whatever its tiles hold beside them; all others have
    what the definition gives."""
    d, n = 64, hist + max(new, 1)
    case = Case(1, Hq, Hkv, d, page, [n], W, 3, dtype=dtype, seed=122)
    T = max(new, 1)
    q = torch.full((T, Hq, d), 2.0, dtype=dtype)
    k, v = (case.normal(T, Hkv, d) for _ in range(2))
    k.mul_(0.01)

    def put(j, key=None, at=0, value=0.0):
        """Token j: a key of one value, a value element; in the pool or among the new tokens."""
        for pool, fresh, x in ((case.k, k, key), (case.v, v, value)):
            row = pool[int(case.table[0, j // page]), :, j % page] if j < hist else fresh[j - hist]
            if pool is case.k and x is not None:
                row[:] = x
            elif pool is case.v:
                row[:, at] = x
    for j in range(hist):
        case.k[int(case.table[0, j // page]), :, j % page] *= 0.01
    put(2, key=8.0)                       # a sink with a score of 128
    bad = {(hist - 40, 5, math.inf), (hist - 3, 9, math.nan), (hist + new // 2, 17, -math.inf), (n - 2, 30, math.inf),
           (n // 2, 33, math.nan), (n // 3, 41, math.inf)}
    for j, at, x in bad:
        if j > 2:
            put(j, at=at, value=x)
    ref = case.ref()
    for i in range(T):
        ref.append(0, n - T + i, k[i], v[i])
    want = [ref.row(0, n - T + i, q[i], False) for i in range(T)]
    out, lse = nan_like(T, Hq, d, dtype=dtype), nan_like(T, Hq, dtype=FP32)
    ws = case.g.new_workspace(T).fill_(0xff)
    kw = dict(k=k.cuda(), v=v.cuda(), lse=lse, max_len=n if hint else 1)
    if new:
        case.g.prefill(case.cache, q.cuda(), [0, T], out, ws, **kw)
    else:
        case.g.decode(case.cache, q.cuda(), out, ws, **kw)
    got, lse = out.cpu().double(), lse.cpu().double()
    lost = 0
    for i, (o, z, tol, ztol) in enumerate(want):
        fine = o.isfinite()
        lost += int((~fine).sum())
        assert torch.equal(got[i].isfinite(), fine), f"row {i}"
        # a weight below 2^-126 of the row's largest is 0 in fp32: n of them, of values below 8, are less than
        # 2^12 * 2^-126 * 2^3 = 2^-111 (element 0 of the sink's value is 0: that row element holds nothing else)
        off = (got[i] - o).abs()[fine] > tol[fine] + 2.0 ** -111
        assert not off.any(), f"row {i}: {int(off.sum())} elements"
        seen = z.isfinite()
        assert ((lse[i] - z).abs()[seen] <= ztol[seen]).all(), f"row {i}: lse"
    assert lost > 0
    case.pools_equal(ref)


@pytest.mark.parametrize("past", [0, 8])
def test_rows_of_a_page_far_apart(past):
    """Pools stored [slot][page][head][d] whose slots are 2^26 elements apart,
    the most that a prefill's 32-bit offsets within a page take (15 rows:
    15 * 2^27 bytes and a row, below 2^31), and 8 more: another kernel."""
    case = Case(2, 8, 2, 128, 16, [150, 77], 90, 3, weights=True, seed=123)
    g, S = case.g, (1 << 26) + past
    shape = case.k.shape
    pools = []
    for x in (case.k, case.v):
        far = torch.empty(15 * S + shape[0] * shape[1] * shape[3], dtype=BF16, device="cuda").as_strided(
            shape, (shape[1] * shape[3], shape[3], S, 1))
        far.copy_(x)
        pools.append(far)
    case.k, case.v = pools
    case.cache = g.cache(*pools, case.dev_table, case.lens, case.w)
    run_prefill(case, [70, 33], 9)
    run_decode(case, True)
    run_evict(case, 60, 20)


@pytest.mark.parametrize("dtype,page,Hq,Hkv,new,hist", [
    (BF16, 16, 8, 2, 0, 700), (FP32, 16, 8, 2, 0, 700),                              # decode
    (BF16, 16, 8, 2, 150, 90), (FP32, 16, 4, 2, 40, 61), (FP32, 64, 32, 16, 450, 0)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_2_to_28(dtype, page, Hq, Hkv, new, hist, sign):
    """Scores near the ends of their range: one token that carries all the
    weight, or equal scores far below 0.  q, k and their products are powers
    of two, so scores carry no error but the scale's (tau log2(e), rounded)."""
    d, T = 64, max(new, 1)
    n = hist + T
    case = Case(1, Hq, Hkv, d, page, [n], None, 0, dtype=dtype, seed=124)
    q = torch.full((T, Hq, d), 2.0 ** 11, dtype=dtype)
    k = torch.zeros(T, Hkv, d, dtype=dtype)
    v = case.normal(T, Hkv, d)
    case.k.zero_()
    hot = 1 if hist else 0
    if sign > 0:
        (case.k[int(case.table[0, 0]), :, 1] if hist else k[0])[:] = 2.0 ** 14
    else:
        case.k.fill_(-2.0 ** 14)
        k.fill_(-2.0 ** 14)
    out, lse = nan_like(T, Hq, d, dtype=dtype), nan_like(T, Hq, dtype=FP32)
    kw = dict(k=k.cuda(), v=v.cuda(), lse=lse)
    if new:
        case.g.prefill(case.cache, q.cuda(), [0, T], out, case.g.new_workspace(T), **kw)
    else:
        case.g.decode(case.cache, q.cuda(), out, case.g.new_workspace(T), **kw)
    ref = case.ref()
    vs = torch.stack([ref.v[ref.slot(0, j)[0], :, ref.slot(0, j)[1]] for j in range(n)])     # [n][Hkv][d]
    G = Hq // Hkv
    for i in range(T):
        m = hist + i + 1
        seen = vs[hot:hot + 1] if sign > 0 else vs[:m]
        want, size = seen.mean(0).repeat_interleave(G, 0), seen.abs().mean(0).repeat_interleave(G, 0)
        # sums of m products in fp32, exponentials and a division; in bf16 two roundings (weights, output) more
        tol = size * ((m + 16) * EPS32 + (2 * EPS16 * (1 + EPS16) if dtype == BF16 else 0.0))
        assert ((out[i].cpu().double() - want).abs() <= tol).all(), f"row {i}"
        z = sign * 2.0 ** 28 + (0.0 if sign > 0 else math.log(m))
        # tau and tau log2(e) rounded, the score, the sum with the logarithm, and ln 2 and its product: 8 half steps
        assert ((lse[i].cpu().double() - z).abs() <= 8 * EPS32 * abs(z)).all(), f"row {i}: lse"
