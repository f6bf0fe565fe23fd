"""The paged softmax cache against its float64 definition (tests/paged_util.py):
decode, prefill, attention weights, eviction, and all of them in a row."""
import math
import random

import pytest
import torch

from paper_2607_24788_amd import glide, paged

from .paged_util import EPS32, Case, check_rows, tables

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def nan_like(*shape, dtype):
    return torch.full(shape, math.nan, dtype=dtype, device="cuda")


def weight_tol(case, n_scored):
    """Relative error of a sum of n_scored * G weights e^{s - lse}: scores and
    lse as bounded in Ref.row (|q||k| of these inputs below 4 d scale^2)."""
    g = case.g
    ds = (g.head_dim + 4) * EPS32 * 4 * g.head_dim * case.scale ** 2 * abs(g.sm_scale)
    return 2 * ds + (max(case.lens_host) + 16 + n_scored * 16) * EPS32


def run_decode(case, append, max_len=0, ws=None):
    g, B = case.g, case.g.batch
    q = case.normal(B, g.n_q_heads, g.head_dim)
    k, v = (case.normal(B, g.n_kv_heads, g.head_dim) for _ in range(2))
    ref = case.ref()
    want = []
    for b, n in enumerate(ref.lens):
        if append:
            ref.append(b, n - 1, k[b], v[b])
        want.append(ref.row(b, n - 1, q[b], ref.w is not None))
    out = nan_like(B, g.n_q_heads, g.head_dim, dtype=case.dtype)
    lse = nan_like(B, g.n_q_heads, dtype=FP32)
    if ws is None:
        ws = g.new_workspace(weights=case.w is not None).fill_(0xff)
    g.decode(case.cache, q.cuda(), out, ws, k=k.cuda() if append else None, v=v.cuda() if append else None, lse=lse,
             max_len=max_len)
    torch.cuda.synchronize()
    check_rows(out, lse, want)
    case.pools_equal(ref)
    if case.w is not None:
        case.weights_close(ref, weight_tol(case, 1))
    return out


DECODE = [
    # B, Hq, Hkv, d, page, lens, window, sinks
    (1, 4, 4, 64, 16, [1], None, 0),
    (3, 8, 2, 128, 16, [0, 1, 33], None, 0),
    (2, 32, 8, 128, 64, [700, 129], None, 0),
    (2, 32, 8, 128, 64, [700, 129], 100, 4),
    (3, 6, 2, 128, 32, [517, 64, 65], 64, 0),        # three heads per group, window at a page's edge
    (2, 16, 1, 128, 128, [1500, 31], 1, 1),          # sixteen heads; itself and one sink
    (2, 8, 8, 64, 1, [130, 77], 31, 70),             # pages of one token, more sinks than the window
    (2, 5, 1, 64, 256, [300, 2], 0, 3),              # sinks alone
    (1, 64, 8, 128, 64, [5003], 4095, 5),
    (1, 8, 2, 64, 1024, [2047], None, 0),
]


@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("i", range(len(DECODE)))
def test_decode(i, dtype, append):
    B, Hq, Hkv, d, page, lens, W, ns = DECODE[i]
    run_decode(Case(B, Hq, Hkv, d, page, lens, W, ns, dtype=dtype, weights=append, seed=i), append)


@pytest.mark.parametrize("max_len", [1, 600, 2100, 1 << 20])
def test_decode_length_hint_changes_no_result(max_len):
    """A bound of the lengths that is too small, right or far too large."""
    run_decode(Case(2, 8, 2, 128, 16, [2100, 600], dtype=FP32, weights=True, seed=3), True, max_len)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_decode_over_many_pieces(dtype):
    """A long sequence of one KV head: as many pieces as a join takes."""
    run_decode(Case(1, 4, 1, 64, 64, [40001], None, 0, dtype=dtype, weights=True, seed=8), True, 40001)


@pytest.mark.parametrize("order", ["nhd", "joined"])
def test_decode_strided_pools(order):
    run_decode(Case(2, 8, 2, 128, 32, [300, 77], 200, 2, seed=4, order=order, weights=True), True)


def test_decode_large_scores():
    """Scores of several hundred: a few tokens carry all the weight."""
    run_decode(Case(2, 8, 2, 64, 16, [400, 33], dtype=FP32, seed=5, scale=8.0), True)
    run_decode(Case(2, 8, 2, 64, 16, [400, 33], dtype=FP32, seed=5, sm_scale=-0.3), True)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_decode_missing_pages(dtype):
    """Pages that are not allocated, below zero or past the pool, among those
    of a sequence, the newest token's too; lens below 0 and past the table."""
    case = Case(5, 8, 2, 128, 16, [100, 64, 90, 48, 16], dtype=dtype, weights=True, seed=6)
    case.table[0, 2], case.table[1, 0], case.table[2, 5] = -1, case.g.n_pages, -7
    case.table[4, :] = -1
    case.dev_table.copy_(case.table)
    case.lens.copy_(torch.tensor([100, 64, 90, -3, 16]))
    case.lens_host = [100, 64, 90, 0, 16]
    run_decode(case, True)
    over = Case(1, 4, 2, 64, 16, [64], dtype=dtype, seed=7, extra_pages=0)
    over.lens.fill_(1 << 30)
    run_decode(over, False)


def run_prefill(case, new, observe=0, append=True, max_len=0):
    g = case.g
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    T = cu[-1]
    q = case.normal(T, g.n_q_heads, g.head_dim)
    k, v = (case.normal(T, g.n_kv_heads, g.head_dim) for _ in range(2))
    ref = case.ref()
    want = []
    for b, n in enumerate(new):
        p0 = ref.lens[b] - n
        if append:
            for i in range(n):
                ref.append(b, p0 + i, k[cu[b] + i], v[cu[b] + i])
        for i in range(n):
            want.append(ref.row(b, p0 + i, q[cu[b] + i], i >= n - observe))
    out = nan_like(T + 1, g.n_q_heads, g.head_dim, dtype=case.dtype)
    lse = nan_like(T + 1, g.n_q_heads, dtype=FP32)
    ws = g.new_workspace(T, weights=observe > 0).fill_(0xff)
    g.prefill(case.cache, q.cuda(), cu, out, ws, k=k.cuda() if append else None, v=v.cuda() if append else None,
              lse=lse, n_observe=observe, max_len=max_len)
    torch.cuda.synchronize()
    check_rows(out[:T], lse[:T], want)
    assert out[T:].isnan().all() and lse[T:].isnan().all(), "rows behind the last sequence"
    case.pools_equal(ref)
    if case.w is not None:
        case.weights_close(ref, weight_tol(case, observe))


PREFILL = [
    # B, Hq, Hkv, d, page, lens, new, window, sinks, observe
    (1, 4, 4, 64, 16, [1], [1], None, 0, 1),
    (1, 8, 2, 128, 64, [200], [200], None, 0, 0),
    (3, 8, 2, 128, 16, [70, 0, 133], [70, 0, 133], None, 0, 40),
    (4, 8, 2, 128, 32, [300, 65, 129, 40], [45, 65, 1, 0], None, 0, 500),
    (2, 32, 8, 128, 64, [330, 190], [130, 67], 100, 4, 32),
    (2, 6, 2, 128, 16, [257, 511], [257, 64], 64, 0, 0),      # three heads per group
    (2, 16, 1, 64, 128, [150, 340], [150, 20], 33, 70, 16),   # sixteen heads, more sinks than the window
    (2, 8, 8, 64, 1, [130, 77], [130, 7], 31, 3, 9),          # pages of one token
    (2, 5, 1, 64, 256, [300, 2], [299, 2], 0, 3, 5),          # sinks alone
    (1, 7, 7, 128, 64, [450], [450], 1, 0, 450),              # itself alone
    (2, 8, 2, 64, 1024, [1100, 900], [3, 5], None, 0, 4),     # few rows over a long cache: pieces joined
    (2, 8, 2, 128, 32, [2100, 1700], [40, 33], None, 0, 7),   # more rows, pieces joined
    (2, 8, 2, 64, 16, [1100, 1300], [70, 64], 700, 300, 64),  # the window's and the sinks' tiles overlap, or not
    (1, 4, 1, 128, 8, [260], [200], 90, 0, 3),                # pages smaller than a wave's rows
]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("i", range(len(PREFILL)))
def test_prefill(i, dtype):
    B, Hq, Hkv, d, page, lens, new, W, ns, obs = PREFILL[i]
    run_prefill(Case(B, Hq, Hkv, d, page, lens, W, ns, dtype=dtype, weights=obs > 0, seed=50 + i), new, obs)


@pytest.mark.parametrize("max_len", [1, 900, 1 << 20])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prefill_length_hint_changes_no_result(dtype, max_len):
    run_prefill(Case(2, 8, 2, 64, 16, [900, 700], 600, 4, dtype=dtype, weights=True, seed=69), [40, 9], 12,
                max_len=max_len)


@pytest.mark.parametrize("dtype,page,d,W,ns,hist", [(FP32, 16, 128, None, 0, 0), (FP32, 64, 64, 200, 70, 90),
                                                    (BF16, 8, 128, 333, 4, 50), (BF16, 1, 64, None, 0, 0)])
def test_prefill_rows_shared(dtype, page, d, W, ns, hist):
    """fp32, and bf16 on small pages, with rows enough for 64-row tiles."""
    new = [900, 0, 141]
    case = Case(3, 32, 16, d, page, [n + (hist if n else 0) for n in new], W, ns, dtype=dtype, weights=True, seed=67)
    case.table[0, 3] = -1
    case.dev_table.copy_(case.table)
    run_prefill(case, new, 7)


@pytest.mark.parametrize("values", ["k", "v"])
@pytest.mark.parametrize("dtype,page,Hq,Hkv,d,new,hist,W", [
    (BF16, 16, 8, 2, 128, [150, 70], 90, 40), (BF16, 32, 4, 4, 64, [200, 33], 100, None),
    (FP32, 16, 4, 2, 128, [50, 37], 61, 30), (FP32, 16, 4, 2, 64, [40, 7], 90, None), (BF16, 4, 4, 2, 128, [60, 9], 70, 25),
    (FP32, 64, 32, 16, 64, [600, 450], 100, 300), (BF16, 8, 32, 16, 128, [600, 450], 0, None),
    (FP32, 16, 4, 2, 128, [40, 7], 90, None), (FP32, 8, 4, 1, 128, [21, 40], 200, 170),
    (BF16, 4, 4, 2, 128, [60, 9], 200, None), (BF16, 8, 4, 2, 64, [40, 7], 210, 180)])
def test_nan_and_infinity_in_unseen_places(dtype, page, Hq, Hkv, d, new, hist, W, values):
    """Keys or values that are not finite, among the new tokens and the cached
    ones: rows that see them have what the definition gives, all others are as
    if they were not there."""
    case = Case(2, Hq, Hkv, d, page, [n + hist for n in new], W, 2, dtype=dtype, seed=65)
    g = case.g
    cu = [0, new[0], sum(new)]
    q, k, v = (case.normal(cu[-1], h, d) for h in (Hq, Hkv, Hkv))
    x = k if values == "k" else v
    for i, y in ((0, math.nan), (1, math.inf), (17, math.nan), (new[0] - 1, -math.inf), (new[0] - 2, math.nan)):
        x[i, i % Hkv, 3 * i % d] = y
    if hist:      # in the cache: before the window, at its edge, in the sinks
        pool = case.k if values == "k" else case.v
        for j in (1, 5, hist - 30, hist - 1):
            pool[int(case.table[0, j // page]), 0, j % page, j % d] = math.nan
    ref = case.ref()
    want = []
    for b, n in enumerate(new):
        for i in range(n):
            ref.append(b, hist + i, k[cu[b] + i], v[cu[b] + i])
        for i in range(n):
            want.append(ref.row(b, hist + i, q[cu[b] + i], False))
    out, lse = nan_like(cu[-1], Hq, d, dtype=dtype), nan_like(cu[-1], Hq, dtype=FP32)
    g.prefill(case.cache, q.cuda(), cu, out, g.new_workspace(cu[-1]), k=k.cuda(), v=v.cuda(), lse=lse,
              max_len=max(new) + hist)
    got, lse = out.cpu().double(), lse.cpu().double()
    clean = 0
    for i, (o, z, tol, ztol) in enumerate(want):
        fine = o.isfinite()
        clean += int(fine.all())
        assert torch.equal(got[i].isnan(), o.isnan()) and torch.equal(got[i][o.isinf()], o[o.isinf()]), f"row {i}"
        assert ((got[i] - o).abs()[fine] <= tol[fine]).all(), f"row {i}"
        assert torch.equal(lse[i].isfinite(), z.isfinite()) and ((lse[i] - z).abs()[z.isfinite()]
                                                                <= ztol[z.isfinite()]).all(), f"row {i}: lse"
    assert clean > 0
    case.pools_equal(ref)


def test_prefill_rows_shared_in_pieces():
    run_prefill(Case(1, 64, 64, 64, 32, [1503], None, 0, dtype=FP32, seed=66), [260], append=False, max_len=1503)


def test_prefill_many_rows_in_pieces():
    """Row tiles that do not fill the card over a long cache: each in pieces,
    rows that begin and end inside tiles, new rows inside a group of 16."""
    run_prefill(Case(1, 8, 1, 128, 64, [2777], None, 0, dtype=BF16, weights=True, seed=68), [100], 100, max_len=2777)


@pytest.mark.parametrize("seed", range(24))
def test_drawn(seed):
    """Calls of every kind, drawn: sizes, windows, sinks, pages, missing pages."""
    r = random.Random(1000 + seed)
    dtype = r.choice([BF16, BF16, FP32])
    Hkv, G, d = r.choice([1, 2, 3]), r.choice([1, 2, 3, 4, 7, 8]), r.choice([64, 128])
    page = r.choice([1, 2, 8, 16, 16, 32, 64, 128])
    B = r.randint(1, 4)
    new = [r.choice([0, 1, 2, r.randint(1, 130)]) for _ in range(B)]
    lens = [n + r.choice([0, 0, r.randint(0, 40), r.randint(0, 400)]) for n in new]
    W = r.choice([None, 1, r.randint(1, 64), r.randint(1, 300), 0])
    ns = r.choice([0, 1, 4, r.randint(1, 150)])
    if W == 0 and ns == 0:
        ns = 2
    case = Case(B, Hkv * G, Hkv, d, page, lens, W, ns, dtype=dtype, weights=True, seed=200 + seed,
                scale=r.choice([0.5, 1.0, 2.0]), order=r.choice(["hnd", "nhd", "joined"]))
    if r.random() < 0.4 and case.table.shape[1] > 2:
        case.table[r.randrange(B), r.randrange(case.table.shape[1] - 1)] = r.choice([-1, case.g.n_pages])
        case.dev_table.copy_(case.table)
    if sum(new):
        run_prefill(case, new, r.choice([0, 1, 20, 1000]), append=r.random() < 0.7, max_len=r.choice([0, max(lens)]))
    run_decode(case, r.random() < 0.7, r.choice([0, max(lens)]))
    recent = r.randint(0, 30)
    run_evict(case, min(ns, 200) + 1 + recent + r.randint(0, 60) if ns <= 200 else 400 + recent, recent,
              alias=r.random() < 0.5)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prefill_of_cached_tokens(dtype):
    """Without k and v: the tokens are in the cache, their weights kept."""
    run_prefill(Case(2, 8, 2, 128, 16, [200, 90], 50, 2, dtype=dtype, weights=True, seed=70), [33, 90], 20,
                append=False)


@pytest.mark.parametrize("order", ["nhd", "joined"])
def test_prefill_strided_pools(order):
    run_prefill(Case(2, 8, 2, 64, 32, [150, 77], None, 0, seed=71, order=order, weights=True), [90, 77], 8)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prefill_missing_pages(dtype):
    """Pages that are not allocated; more new tokens than lens says."""
    case = Case(3, 8, 2, 128, 16, [150, 140, 60], None, 2, dtype=dtype, weights=True, seed=72)
    case.table[0, 3], case.table[1, 0], case.table[1, 8] = -1, case.g.n_pages, 1 << 30
    case.dev_table.copy_(case.table)
    case.lens.copy_(torch.tensor([150, 140, 50]))
    case.lens_host = [150, 140, 50]
    run_prefill(case, [70, 140, 60], 30)


def test_many_sequences():
    """More sequences than one launch takes."""
    new = [(7 * i) % 5 for i in range(300)]
    run_prefill(Case(300, 4, 2, 64, 16, [n + i % 19 for i, n in enumerate(new)], 9, 1, seed=73, weights=True), new, 2)


def run_evict(case, budget, recent, dst=None, alias=False):
    g = case.g
    ref = case.ref()
    want, want_lens = ref.evict(budget, recent, None if dst is None else dst.long())
    kept = torch.full((g.batch, g.n_kv_heads, budget), 77, dtype=torch.int32, device="cuda")
    new_lens = case.lens if alias else torch.full((g.batch,), 77, dtype=torch.int32, device="cuda")
    ws = g.new_workspace(weights=True).fill_(0xff)
    g.evict(case.cache, budget, recent, kept, new_lens, ws, dst_table=None if dst is None else dst.cuda())
    torch.cuda.synchronize()
    assert torch.equal(new_lens.cpu(), want_lens)
    assert torch.equal(kept.cpu(), want)
    case.pools_equal(ref)
    case.weights_close(ref)
    return ref


EVICT = [
    # B, Hkv, d, page, lens, sinks, budget, recent
    (1, 2, 64, 16, [1], 0, 1, 0),
    (3, 2, 128, 16, [0, 40, 41], 0, 40, 0),
    (2, 4, 128, 64, [700, 129], 4, 100, 20),
    (2, 1, 64, 32, [2500, 513], 0, 512, 512),       # the newest alone
    (2, 2, 64, 1, [1300, 90], 7, 64, 0),
    (1, 8, 128, 256, [3001], 4, 1030, 100),
    (2, 2, 64, 16, [300, 200], 250, 260, 10),       # the sinks fill it, more of them than tokens
]


@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("i", range(len(EVICT)))
def test_evict(i, dtype, fresh):
    B, Hkv, d, page, lens, ns, budget, recent = EVICT[i]
    counts = [-(-min(n, budget) // page) for n in lens]
    case = Case(B, 2 * Hkv, Hkv, d, page, lens, None, ns, dtype=dtype, weights=True, seed=80 + i)
    dst = None
    if fresh:  # pages of their own at the pool's end
        old = case
        n0 = old.g.n_pages
        g = paged.Paged(B, 2 * Hkv, Hkv, d, page, n0 + sum(counts), old.g.max_pages, n_sinks=ns, dtype=dtype)
        pad = lambda x: torch.cat([x, torch.full((sum(counts), *x.shape[1:]), math.nan, dtype=x.dtype,  # noqa: E731
                                                 device="cuda")])
        case.k, case.v, case.w, case.g = pad(old.k), pad(old.v), pad(old.w), g
        case.cache = g.cache(case.k, case.v, case.dev_table, case.lens, case.w)
        dst = tables(case.gen, B, g.max_pages, counts, g.n_pages, first=n0)
    run_evict(case, budget, recent, dst, alias=i % 2 == 1)


def test_evict_equal_and_special_weights():
    """Equal weights, zeros of both signs, infinities and NaN."""
    case = Case(2, 4, 2, 64, 16, [900, 333], None, 2, dtype=FP32, weights=True, seed=90)
    w = case.w.cpu()
    pick = torch.randint(0, 9, w.shape, generator=case.gen)
    for i, x in enumerate([0.0, -0.0, 1.0, 1.0, math.inf, -math.inf, math.nan, 1e-42, -1e-42]):
        w[pick == i] = x
    w[case.w.cpu().isnan()] = math.nan
    case.w.copy_(w)
    g, ref = case.g, case.ref()
    want, _ = ref.evict(200, 10)
    kept = torch.empty((2, 2, 200), dtype=torch.int32, device="cuda")
    g.evict(case.cache, 200, 10, kept, case.lens, g.new_workspace(weights=True))
    assert torch.equal(kept.cpu(), want)
    x, y = case.w.cpu().double(), ref.w
    assert ((x == y) | (x.isnan() & y.isnan())).all()
    case.pools_equal(ref)


@pytest.mark.parametrize("n", [4096, 4097, 33000, 70003])
def test_evict_long(n):
    """Keys that fill LDS, and more than it holds."""
    run_evict(Case(1, 2, 1, 64, 64, [n], 4, 0, dtype=BF16, weights=True, seed=92, extra_pages=0), n // 3, n // 10)


def test_evict_missing_pages():
    """Tokens on pages that are not allocated go first; rows whose new place is
    not allocated are dropped."""
    case = Case(2, 4, 2, 128, 16, [200, 100], weights=True, seed=91)
    case.table[0, 4], case.table[0, 9], case.table[1, 0] = -1, case.g.n_pages + 5, -1
    case.dev_table.copy_(case.table)
    run_evict(case, 70, 20)


def test_prefill_decode_evict_in_a_row():
    """A session: the prompt, tokens one by one, an eviction in place, more
    tokens, each against the reference's own state."""
    case = Case(2, 8, 2, 128, 16, [150, 90], 80, 4, dtype=FP32, weights=True, seed=95, extra_pages=4)
    spare = [p for p in range(case.g.n_pages) if p not in case.table]
    case.table[0, 10], case.table[1, 6] = spare[0], spare[1]
    case.dev_table.copy_(case.table)
    run_prefill(case, [150, 90], 16)
    for step in range(12):
        if step == 6:
            ref = run_evict(case, 60, 20, alias=True)
            case.lens_host = list(ref.lens)
        case.lens += 1
        case.lens_host = [n + 1 for n in case.lens_host]
        run_decode(case, True)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_same_as_a_layer_without_its_linear_part(dtype):
    """The same window as a GLIDE layer's softmax part alone."""
    B, Hq, Hkv, d, W, lens = 2, 8, 2, 128, 70, [200, 133]
    case = Case(B, Hq, Hkv, d, 16, lens, W, 0, dtype=dtype, seed=96)
    cu = [0, lens[0], sum(lens)]
    q, k, v = (case.normal(cu[-1], h, d).cuda() for h in (Hq, Hkv, Hkv))
    got, want = torch.empty_like(q), torch.empty_like(q)
    case.g.prefill(case.cache, q, cu, got, case.g.new_workspace(cu[-1]), k=k, v=v)
    g = glide.Glide(1, B, Hq, Hkv, d, 64, [W], dtype=dtype, linear=False)
    st = g.new_state()
    g.state_init(st)
    g.prefill(st, torch.zeros(d, 64, dtype=dtype, device="cuda"), q, k, v, cu, want, g.new_workspace(cu[-1]))
    scale = v.float().abs().max().item()
    # both within their own bound of the same values: twice two roundings of
    # weights and output (bf16), or the scores' fp32 error
    tol = scale * (4 * 2 ** -8 if dtype == BF16 else 4 * (d + 4) * EPS32 * 4 * d ** 0.5)
    assert (got.float() - want.float()).abs().max().item() <= tol


def test_offsets_past_32_bits():
    """Pools of more than 4 GiB, the sequence's pages at their ends."""
    Hkv, d, page, n = 8, 128, 64, 40000
    g = paged.Paged(1, 16, Hkv, d, page, n, 8, window=300, n_sinks=70)
    k, v, w = g.new_pools(weights=True)
    assert k.numel() * 2 > 1 << 32
    case = Case(1, 16, Hkv, d, page, [400], 300, 70, weights=True, seed=97)
    table = torch.full((1, 8), -1, dtype=torch.int32, device="cuda")
    for i in range(7):
        p, q = n - 1 - 2 * i, int(case.table[0, i])
        table[0, i] = p
        k[p], v[p], w[p] = case.k[q], case.v[q], case.w[q]
    lens = torch.tensor([400], dtype=torch.int32, device="cuda")
    cache = g.cache(k, v, table, lens, w)
    x = [case.normal(30, h, d).cuda() for h in (16, Hkv, Hkv)]
    outs = []
    for gg, c in ((g, cache), (case.g, case.cache)):
        o, z = torch.empty_like(x[0]), torch.empty(30, 16, device="cuda")
        ws = gg.new_workspace(30, weights=True)
        gg.prefill(c, x[0], [0, 30], o, ws, k=x[1], v=x[2], lse=z, n_observe=9)
        kept, nl = torch.empty((1, Hkv, 128), dtype=torch.int32, device="cuda"), torch.empty_like(lens)
        gg.evict(c, 128, 20, kept, nl, ws)
        o2 = torch.empty((1, 16, d), dtype=BF16, device="cuda")
        gg.decode(c, x[0][:1], o2, ws)
        outs.append((o, z, kept, nl, o2))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_binding_refusals():
    case = Case(2, 8, 2, 64, 16, [50, 20], weights=True, seed=98)
    g, ws = case.g, case.g.new_workspace(8, weights=True)
    q = torch.zeros(2, 8, 64, dtype=BF16, device="cuda")
    kv = torch.zeros(2, 2, 64, dtype=BF16, device="cuda")
    out = torch.empty_like(q)
    for bad in (q.cpu(), q.float(), q[:1], q.transpose(0, 1)):
        with pytest.raises(ValueError):
            g.decode(case.cache, bad, out, ws)
        with pytest.raises(ValueError):
            g.decode(case.cache, q, bad, ws)
    with pytest.raises(ValueError, match="together"):
        g.decode(case.cache, q, out, ws, k=kv)
    with pytest.raises(ValueError):
        g.decode(case.cache, q, out, ws, lse=torch.empty(2, 8, dtype=BF16, device="cuda"))
    with pytest.raises(glide.GlideError, match="SIZE"):
        g.decode(case.cache, q, out, ws[:256])
    with pytest.raises(glide.GlideError, match="INVALID"):
        g.decode(case.cache, q, out, ws, max_len=-1)
    bare = g.cache(case.k, case.v, case.dev_table, case.lens)
    with pytest.raises(ValueError, match="weights"):
        g.prefill(bare, q, [0, 1, 2], out, ws, n_observe=1)
    kept, nl = torch.empty(2, 2, 30, dtype=torch.int32, device="cuda"), torch.empty_like(case.lens)
    with pytest.raises(ValueError, match="weights"):
        g.evict(bare, 30, 2, kept, nl, ws)
    with pytest.raises(ValueError, match="kept"):
        g.evict(case.cache, 31, 2, kept, nl, ws)
    with pytest.raises(ValueError, match="dst_table"):
        g.evict(case.cache, 30, 2, kept, nl, ws, dst_table=case.dev_table[:1])
    with pytest.raises(glide.GlideError, match="INVALID"):
        g.evict(case.cache, 0, 0, kept, nl, ws)
    for k in (case.k.float(), case.k[1:], case.k.transpose(2, 3), case.k.expand(*case.k.shape)[:, :1].expand(case.k.shape),
              case.k.cpu()):
        with pytest.raises(ValueError):
            g.cache(k, case.v, case.dev_table, case.lens)
    with pytest.raises(ValueError, match="lens"):
        g.cache(case.k, case.v, case.dev_table, case.lens.long())
    with pytest.raises(ValueError, match="block_table"):
        g.cache(case.k, case.v, case.dev_table[:, :1].contiguous(), case.lens)
    with pytest.raises(ValueError, match="weights"):
        g.cache(case.k, case.v, case.dev_table, case.lens, case.w[1:])


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_captured_calls(dtype):
    """Prefill with scored queries, decode steps and an eviction captured
    together, replayed on restored state and inputs, with eager work between,
    against the eager calls; two graphs share one workspace."""
    case = Case(2, 16, 2, 64, 16, [1300, 500], 900, 4, dtype=dtype, weights=True, seed=99)
    g = case.g
    new, steps = [40, 13], 3
    cu = [0, 40, 53]
    spare = [p for p in range(g.n_pages) if p not in case.table]
    case.table[0, 82], case.table[1, 32] = spare[0], spare[1]
    case.dev_table.copy_(case.table)
    q, k, v = (case.normal(53 + 2 * steps, h, 64).cuda() for h in (16, 2, 2))
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    kept = torch.empty((2, 2, 200), dtype=torch.int32, device="cuda")
    ws = g.new_workspace(53, weights=True)
    bufs = [case.k, case.v, case.w, case.lens]
    snap = [x.clone() for x in bufs]

    def calls():
        g.prefill(case.cache, q, cu, out, ws, k=k, v=v, lse=lse, n_observe=20, max_len=1300)
        for s in range(steps):
            case.lens.add_(1)
            i = 53 + 2 * s
            g.decode(case.cache, q[i:i + 2], out[i:i + 2], ws, k=k[i:i + 2], v=v[i:i + 2], lse=lse[i:i + 2],
                     max_len=1400)
        g.evict(case.cache, 200, 30, kept, case.lens, ws)

    def results():
        torch.cuda.synchronize()
        return [x.clone() for x in (out, lse, kept, *bufs)]

    def restore():
        for x, y in zip(bufs, snap):
            x.copy_(y)
        out.fill_(math.nan)
        ws.fill_(0xff)

    calls()
    want = results()
    graphs = []
    side = torch.cuda.Stream()
    for _ in range(2):
        restore()
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls()
        torch.cuda.synchronize()
        graphs.append(graph)
    same = lambda a, b: torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))  # noqa: E731
    for rep in range(4):
        restore()
        graphs[rep % 2].replay()
        assert all(same(a, b) for a, b in zip(results(), want)), f"replay {rep}"
        restore()
        calls()
        assert all(same(a, b) for a, b in zip(results(), want)), f"eager after replay {rep}"


def test_other_stream():
    """Two streams at once, each with its own cache and workspace."""
    cases = [Case(2, 8, 2, 128, 16, [700, 300], 500, 4, weights=True, seed=110 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    q = [c.normal(2, 8, 128).cuda() for c in cases]
    ws = [c.g.new_workspace(weights=True) for c in cases]
    want = [torch.empty_like(x) for x in q]
    for c, x, o, w in zip(cases, q, want, ws):
        c.g.decode(c.cache, x, o, w)
    torch.cuda.synchronize()
    outs = [[torch.empty_like(x) for _ in range(20)] for x in q]
    for i in range(20):
        for c, x, o, w, s in zip(cases, q, outs, ws, streams):
            c.g.decode(c.cache, x, o[i], w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for os_, w in zip(outs, want) for o in os_)
