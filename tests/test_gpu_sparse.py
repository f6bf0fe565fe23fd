"""Attention over selected pages against float64 on the CPU: which pages are
selected (equal to the last one), and the rows over them."""
import math
import random

import pytest
import torch

from . import paged_util
from .paged_util import Case, check_rows
from .test_gpu_append import cu_of, frequencies
from .test_gpu_paged import nan_like

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def made_bounds(case):
    b = nan_like(*case.k.shape[:2], 2, case.g.head_dim, dtype=case.dtype)
    case.g.page_bounds(case.cache, b)
    return b


def pages_of(case, b, t, q, bounds, n_select, first, recent):
    """The definition: pages selected for the row at t of sequence b, by KV head."""
    g, P = case.g, case.g.page_size
    G = g.n_q_heads // g.n_kv_heads
    mine = t // P
    there = [i for i in range(mine + 1) if 0 <= int(case.table[b, i]) < g.n_pages] if t >= 0 else []
    x = q.double().view(g.n_kv_heads, G, -1)
    x = -x if g.sm_scale < 0 else x
    up, down = x.clamp_min(0).sum(1), x.clamp_max(0).sum(1)      # (NaN stays NaN)
    rows = []
    for h in range(g.n_kv_heads):
        always = [i for i in there if i < first or i > mine - recent]
        rest = [i for i in there if i not in always]
        kb = bounds[[int(case.table[b, i]) for i in rest], h] if rest else None
        # (sums of one row alike for every row, which a matrix product's are not at its edges)
        score = (kb[:, 1] * up[h] + kb[:, 0] * down[h]).sum(-1).tolist() if rest else []
        order = sorted(range(len(rest)), key=lambda i: (math.isnan(score[i]), -score[i] if score[i] == score[i] else 0,
                                                        rest[i]))
        rows.append(sorted(always + [rest[i] for i in order[:n_select - len(always)]]))
    return rows


def run_sparse(case, new, n_select, first=1, recent=1, max_len=0, bounds=None, q=None):
    g, cu, T = case.g, cu_of(new), sum(new)
    d, G = g.head_dim, g.n_q_heads // g.n_kv_heads
    if q is None:
        q = case.normal(T, g.n_q_heads, d)
    dev_bounds = made_bounds(case) if bounds is None else bounds
    kb = dev_bounds.cpu().double()
    ref = case.ref()
    want, chosen = [], torch.full((T, g.n_kv_heads, n_select), -1, dtype=torch.int32)
    for b, n in enumerate(new):
        for i in range(n):
            t = ref.lens[b] - n + i
            pages = pages_of(case, b, t, q[cu[b] + i], kb, n_select, first, recent)
            parts = []
            for h, mine in enumerate(pages):
                chosen[cu[b] + i, h, :len(mine)] = torch.tensor(mine, dtype=torch.int32)
                # a row over these tokens alone: a sequence of its own of one KV head
                over = [j for p in mine for j in range(p * g.page_size, min(t + 1, (p + 1) * g.page_size))]
                parts.append(over_tokens(ref, b, h, over, q[cu[b] + i, h * G:(h + 1) * G]))
            want.append([torch.cat([x[k] for x in parts]) for k in range(4)])
    out, lse = nan_like(T + 1, g.n_q_heads, d, dtype=case.dtype), nan_like(T + 1, g.n_q_heads, dtype=FP32)
    sel = torch.full((T + 1, g.n_kv_heads, n_select), 77, dtype=torch.int32, device="cuda")
    ws = g.new_sparse_workspace(T, n_select).fill_(0xff)
    g.sparse(case.cache, dev_bounds, q.cuda(), cu, n_select, sel, out, ws, n_first=first, n_recent=recent, lse=lse,
             max_len=max_len)
    torch.cuda.synchronize()
    assert torch.equal(sel[:T].cpu(), chosen), "selected pages"
    check_rows(out[:T], lse[:T], want)
    assert out[T:].isnan().all() and lse[T:].isnan().all() and (sel[T:] == 77).all(), "rows behind the last sequence"
    case.pools_equal(ref)
    return chosen


class _Layer:
    def __init__(self, g, G):
        self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim = 1, G, 1, g.head_dim
        self.sm_scale, self.torch_dtype, self.window, self.n_sinks = g.sm_scale, g.torch_dtype, 1 << 30, 0


def over_tokens(ref, b, h, over, q):
    """Ref.row of head h's group over the tokens `over` of sequence b."""
    r = object.__new__(paged_util.Ref)
    r.g, r.w, r.lens = _Layer(ref.g, q.shape[0]), None, [len(over)]
    r.k, r.v = ref.k[:, h:h + 1], ref.v[:, h:h + 1]
    at = [ref.slot(b, j) for j in over]
    r.slot = lambda _, j: at[j]
    return r.row(0, len(over) - 1, q, False)


SHAPES = [
    # B, Hq, Hkv, d, page, lens, new, select, first, recent
    (1, 4, 4, 64, 16, [1], [1], 1, 0, 1),
    (1, 8, 2, 128, 16, [700], [1], 8, 1, 2),
    (3, 8, 2, 128, 16, [300, 5, 0], [1, 1, 0], 30, 0, 1),          # fewer pages than are selected
    (3, 32, 8, 64, 32, [900, 333, 1200], [9, 1, 3], 6, 2, 3),      # drafts
    (2, 16, 1, 128, 64, [900, 260], [130, 17], 3, 0, 1),           # a page's end inside the rows
    (2, 6, 2, 64, 1, [300, 90], [5, 90], 40, 3, 4),                # pages of one token
    (1, 5, 5, 128, 256, [2000], [2], 4, 4, 0 + 1),                 # (5 of 4 fixed: see below)
    (1, 8, 2, 64, 16, [20000], [1], 100, 1, 4),                    # more pages than 4 keys a thread
    (1, 2, 1, 64, 1, [5000], [2], 64, 1, 4),                       # more than 16 keys a thread
    (140, 2, 1, 64, 16, [40 + i for i in range(140)], [i % 3 for i in range(140)], 2, 0, 1),   # two launches
]
SHAPES[6] = (1, 5, 5, 128, 256, [2000], [2], 5, 4, 1)              # none left to select


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_sparse(dtype, i):
    B, Hq, Hkv, d, page, lens, new, select, first, recent = SHAPES[i]
    case = Case(B, Hq, Hkv, d, page, lens, dtype=dtype, seed=400 + i)
    run_sparse(case, new, select, first, recent, max_len=0 if i % 2 else max(lens))


@pytest.mark.parametrize("max_len", [1, 600, 1 << 20])
def test_length_hint_changes_no_result(max_len):
    run_sparse(Case(2, 8, 2, 128, 16, [1400, 600], dtype=FP32, seed=420), [2, 1], 12, max_len=max_len)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("pages", [90, 1500, 4500])
def test_equal_scores(dtype, pages):
    """Pages with the same bounds: the first of them; all in all, in part, and
    beside larger and smaller ones (a query of zeros scores all alike)."""
    case = Case(1, 4, 2, 64, 1, [pages], dtype=dtype, seed=421)
    keys = case.normal(5, 2, 64).cuda()
    which = torch.randint(0, 5, (pages,), generator=case.gen)
    rows = case.table[0, :pages].long().cuda()
    case.k[rows, :, 0] = keys[which.cuda()]
    for n in (7, pages // 5, pages // 2, pages - 1):
        run_sparse(case, [1], n, 0, 1)
    run_sparse(case, [1], 33, 1, 2, q=torch.zeros(1, 4, 64, dtype=dtype))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_missing_pages(dtype):
    """Pages that are not allocated are not selected, the row's own, the first
    and the last ones too; rows of lens below their number see nothing."""
    case = Case(4, 8, 2, 128, 16, [300, 260, 64, 40], dtype=dtype, seed=422)
    case.table[0, 0], case.table[0, 7], case.table[1, 16], case.table[2, :] = -1, case.g.n_pages, -5, -1
    case.dev_table.copy_(case.table)
    case.lens.copy_(torch.tensor([300, 260, 64, 2]))
    case.lens_host = [300, 260, 64, 2]
    run_sparse(case, [3, 2, 1, 5], 6, 2, 2)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_scale_below_zero(dtype):
    run_sparse(Case(1, 8, 2, 64, 16, [500], dtype=dtype, seed=423, sm_scale=-0.2), [3], 5)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_not_finite(dtype):
    """NaN and infinite keys and values of pages that a row does not select,
    and of slots behind its position; infinite and NaN scores in order."""
    case = Case(1, 4, 1, 64, 16, [480], dtype=dtype, seed=424)
    q = case.normal(3, 4, 64)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5        # of one sign: an infinite key has a score
    q[:, :, 1] = 0.0
    case.v[int(case.table[0, 4])] = math.nan
    case.v[int(case.table[0, 5])] = math.inf
    bounds = made_bounds(case)
    bounds[int(case.table[0, 4]), :, 1, 0] = -math.inf   # the least score but NaN
    bounds[int(case.table[0, 4]), :, 0, 0] = -math.inf
    bounds[int(case.table[0, 5]), :, 0, 1] = math.inf    # 0 * inf: NaN
    case.k[int(case.table[0, 29]), :, 15] = math.nan     # behind the first two rows
    case.v[int(case.table[0, 29]), :, 15] = math.inf
    case.lens.fill_(479)
    case.lens_host = [479]
    chosen = run_sparse(case, [3], 28, 1, 1, bounds=bounds, q=q)
    assert not (chosen == 4).any() and not (chosen == 5).any()


@pytest.mark.parametrize("Hkv,G,page,select,scale", [
    (64, 2, 32, 3, 1.0), (32, 1, 64, 2, 1.0), (32, 4, 128, 2, -1.0), (96, 8, 32, 4, 1.0), (64, 5, 32, 9, 1.0),
    (64, 2, 16, 14, 1.0), (96, 1, 16, 9, -1.0)])
def test_rows_that_share_a_wave(Hkv, G, page, select, scale):
    """Rows of a sequence together: ragged ends, missing pages, rows that see
    nothing, lists of different lengths."""
    new = [150 + 900 // Hkv, 1, 0, 23, 7]
    lens = [new[0] + 101, 1, 9, 20, 300]
    R = 16 // G
    assert Hkv * sum(-(-n // R) for n in new) >= 1024 or G == 1
    case = Case(5, Hkv * G, Hkv, 64 if Hkv > 32 else 128, page, lens, seed=480, sm_scale=scale * 0.15)
    if page < 100:
        case.table[0, 1] = -1
        case.dev_table.copy_(case.table)
    run_sparse(case, new, select, 0, 1, max_len=max(lens))


@pytest.mark.parametrize("new", [150, 530])
@pytest.mark.parametrize("where", ["k", "v"])
def test_not_finite_in_shared_pages(new, where):
    """Keys or values that are not finite in pages that some rows of a wave
    select and others do not, and at positions that some see and others do not:
    every row has what the definition gives of what it sees."""
    Hkv, G, d, page, hist = (64, 2, 64, 32, 100) if new == 150 else (16, 4, 128, 32, 70)
    assert Hkv * -(-new // (16 // G)) >= 1024
    case = Case(1, Hkv * G, Hkv, d, page, [hist + new], seed=490 + new)
    bounds = made_bounds(case)             # of finite keys
    pool = case.k if where == "k" else case.v
    for j, e, x in ((5, 3, math.nan), (33, 7, math.inf), (70, 9, -math.inf), (hist + 80, 11, math.nan),
                    (hist + 81, 12, math.inf), (hist + new - 9, 13, math.nan), (hist + new - 1, 14, math.inf)):
        pool[int(case.table[0, j // page]), ::3, j % page, e] = x
    g, select, T = case.g, 3, new
    q = case.normal(T, Hkv * G, d)
    kb, ref = bounds.cpu().double(), case.ref()
    out, lse = nan_like(T, Hkv * G, d, dtype=BF16), nan_like(T, Hkv * G, dtype=FP32)
    sel = torch.full((T, Hkv, select), 77, dtype=torch.int32, device="cuda")
    g.sparse(case.cache, bounds, q.cuda(), [0, T], select, sel, out, g.new_sparse_workspace(T, select), n_first=0, lse=lse)
    got, z = out.cpu().double(), lse.cpu().double()
    clean = lost = 0
    for i in list(range(0, T, 13)) + list(range(T - 12, T)) + list(range(76, 92)):
        t = hist + i
        pages = pages_of(case, 0, t, q[i], kb, select, 0, 1)
        for h in (0, 1, 2, 3, Hkv - 1):
            assert sel[i, h].tolist() == pages[h] + [-1] * (select - len(pages[h]))
            over = [j for p in pages[h] for j in range(p * page, min(t + 1, (p + 1) * page))]
            o, zl, tol, ztol = over_tokens(ref, 0, h, over, q[i, h * G:(h + 1) * G])
            x, y = got[i, h * G:(h + 1) * G], z[i, h * G:(h + 1) * G]
            fine = o.isfinite()
            clean, lost = clean + int(fine.all()), lost + int((~fine).sum())
            assert torch.equal(x.isfinite(), fine), (i, h)
            assert ((x - o).abs()[fine] <= tol[fine] + 1e-30).all(), (i, h)
            ok = zl.isfinite()
            assert torch.equal(y.isfinite(), ok) and ((y - zl).abs()[ok] <= ztol[ok]).all(), (i, h)
    assert clean > 0 and lost > 0


def test_rows_in_several_launches():
    """More rows than the scores of one launch hold: a table of 2^17 pages,
    256 MiB / (8 * 2 * 2^17 * ..) rows to a launch."""
    case = Case(2, 4, 2, 64, 1, [500, 300], seed=425, extra_pages=(1 << 17))
    assert case.g.max_pages > 1 << 17
    run_sparse(case, [170, 9], 6, 1, 1, max_len=500)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d,Hkv,G,page,sm_scale", [(128, 16, 3, 16, None), (64, 8, 16, 32, -0.3), (128, 32, 1, 1, None)])
def test_many_units(dtype, d, Hkv, G, page, sm_scale):
    """As many (row, KV head) units as have a wave each: ragged lengths, empty
    rows, missing pages, more pages than are selected and fewer."""
    new = [2100 // Hkv, 3, 0, 9]
    lens = [new[0] + 90, 3, 40, 5]
    case = Case(4, Hkv * G, Hkv, d, page, lens, dtype=dtype, seed=470, sm_scale=sm_scale, order="joined")
    case.table[0, 2] = -1
    case.dev_table.copy_(case.table)
    assert sum(new) * Hkv >= 2048
    run_sparse(case, new, 5, 1, 1)


def test_strided_pools_and_another_stream():
    case = Case(2, 8, 2, 128, 32, [500, 260], order="nhd", seed=426)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run_sparse(case, [2, 1], 4)


@pytest.mark.parametrize("seed", range(16))
def test_drawn(seed):
    r = random.Random(3000 + seed)
    dtype = r.choice([BF16, BF16, FP32])
    Hkv, G, d = r.choice([1, 2, 3]), r.choice([1, 2, 3, 4, 7, 16]), r.choice([64, 128])
    page = r.choice([1, 2, 8, 16, 16, 32, 64, 128])
    B = r.randint(1, 4)
    new = [r.choice([0, 1, 2, r.randint(1, 60)]) for _ in range(B)]
    new[0] = max(1, new[0])
    lens = [n + r.choice([0, r.randint(0, 40), r.randint(0, 900)]) for n in new]
    first, recent = r.randint(0, 3), r.randint(1, 4)
    case = Case(B, Hkv * G, Hkv, d, page, lens, 5, 1, dtype=dtype, seed=430 + seed, scale=r.choice([0.5, 1.0, 2.0]),
                order=r.choice(["hnd", "nhd", "joined"]))
    if r.random() < 0.4 and case.table.shape[1] > 2:
        case.table[r.randrange(B), r.randrange(case.table.shape[1] - 1)] = r.choice([-1, case.g.n_pages])
        case.dev_table.copy_(case.table)
    run_sparse(case, new, first + recent + r.choice([0, 1, r.randint(0, 30)]), first, recent,
               r.choice([0, max(lens)]))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_session(dtype):
    """As a program uses it: a prompt appended with its bounds, then tokens one
    by one, each read out over the pages it selects; the bounds kept are those
    of the cache."""
    case = Case(2, 8, 2, 128, 16, [330, 200], dtype=dtype, seed=450)
    g, f = case.g, frequencies(128).cuda()
    bounds = nan_like(*case.k.shape[:2], 2, 128, dtype=dtype)
    lens = [0, 0]
    for new in ([300, 180], [1, 1], [1, 1], [5, 0], [1, 1]):
        lens = [n + m for n, m in zip(lens, new)]
        case.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        case.lens_host = lens
        T = sum(new)
        q, k, v = (case.normal(T, h, 128).cuda() for h in (8, 2, 2))
        g.append(case.cache, k, v, cu_of(new), q=q, q_out=q, freqs=f, bounds=bounds)
        want = made_bounds(case)
        for b, n in enumerate(lens):
            for i in range(-(-n // 16)):
                p = int(case.table[b, i])
                assert torch.equal(bounds[p], want[p]), (b, i)
        if T < 100:
            run_sparse(case, new, 6, 1, 2, bounds=bounds, q=q.cpu(), max_len=max(lens))


def test_captured():
    case = Case(2, 8, 2, 128, 16, [900, 600], seed=451)
    g = case.g
    bounds = made_bounds(case)
    q = case.normal(2, 8, 128).cuda()
    out, lse = torch.empty_like(q), torch.empty(2, 8, device="cuda")
    sel = torch.empty(2, 2, 9, dtype=torch.int32, device="cuda")
    ws = g.new_sparse_workspace(2, 9)
    call = lambda: g.sparse(case.cache, bounds, q, [0, 1, 2], 9, sel, out, ws, lse=lse, max_len=900)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in range(4):
        q.copy_(case.normal(2, 8, 128))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, sel)]
        for t in (out, lse, sel):
            t.zero_()
        call()
        for x, y in zip(got, (out, lse, sel)):
            assert torch.equal(x, y), n
