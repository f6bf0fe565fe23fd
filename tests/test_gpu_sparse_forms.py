"""Rows that share a wave over selected pages, against float64 on the CPU: each
call asserts the kernel that it is planned for."""
import pytest
import torch

from .paged_util import Case, check_rows
from .test_gpu_append import cu_of
from .test_gpu_paged import nan_like
from .test_gpu_sparse import made_bounds, over_tokens, pages_of, run_sparse
from .test_planning import TILES, WAVES, sparse_form

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def sampled_sparse(case, new, n_select, rows, heads, first=0, recent=1, max_len=0):
    """As run_sparse, of some packed rows and KV heads."""
    g, cu, T, G = case.g, cu_of(new), sum(new), case.g.n_q_heads // case.g.n_kv_heads
    q, bounds = case.normal(T, g.n_q_heads, g.head_dim), made_bounds(case)
    out, lse = nan_like(T + 1, g.n_q_heads, g.head_dim, dtype=case.dtype), nan_like(T + 1, g.n_q_heads, dtype=FP32)
    sel = torch.full((T + 1, g.n_kv_heads, n_select), 77, dtype=torch.int32, device="cuda")
    g.sparse(case.cache, bounds, q.cuda(), cu, n_select, sel, out, g.new_sparse_workspace(T, n_select).fill_(0xff),
             n_first=first, n_recent=recent, lse=lse, max_len=max_len)
    kb, ref = bounds.cpu().double(), case.ref()
    for r in rows:
        b = next(b for b in range(len(new)) if cu[b] <= r < cu[b + 1])
        t = ref.lens[b] - new[b] + r - cu[b]
        pages = pages_of(case, b, t, q[r], kb, n_select, first, recent)
        for h in heads:
            assert sel[r, h].tolist() == pages[h] + [-1] * (n_select - len(pages[h])), (r, h)
            over = [j for p in pages[h] for j in range(p * g.page_size, min(t + 1, (p + 1) * g.page_size))]
            mine = slice(h * G, (h + 1) * G)
            check_rows(out[r:r + 1, mine], lse[r:r + 1, mine], [over_tokens(ref, b, h, over, q[r, mine])])
    assert out[:T].isfinite().all()
    assert out[T:].isnan().all() and lse[T:].isnan().all() and (sel[T:] == 77).all(), "rows behind the last sequence"


@pytest.mark.parametrize("G,page,d,select,scale", [(8, 32, 128, 4, 1.0), (7, 64, 64, 3, 1.0), (6, 128, 128, 2, -1.0),
                                                   (8, 256, 64, 2, 1.0)])
def test_two_rows_to_a_wave(G, page, d, select, scale):
    """Odd numbers of rows, a missing page, rows that see nothing."""
    Hkv, new = 64, [37, 1, 0, 9]
    lens = [new[0] + 3 * page + 5, 1, 9, 7]
    case = Case(4, Hkv * G, Hkv, d, page, lens, seed=630 + G + d, sm_scale=scale * 0.15)
    case.table[0, 1] = -1
    case.dev_table.copy_(case.table)
    assert sparse_form(case.g, new, select, max(lens)) == TILES
    run_sparse(case, new, select, 0, 1, max_len=max(lens))


@pytest.mark.parametrize("Hkv,G,page,d,select,form", [
    (32, 1, 64, 128, 4, TILES), (16, 2, 32, 128, 7, TILES), (8, 8, 128, 128, 3, TILES), (16, 5, 1024, 64, 2, TILES),
    (16, 3, 16, 128, 36, TILES), (32, 1, 16, 64, 20, TILES),          # pages of 16 tokens: by how many rows select one
    (16, 3, 16, 128, 18, WAVES), (32, 1, 16, 64, 12, WAVES)])
def test_many_rows_to_a_wave(Hkv, G, page, d, select, form):
    new, R = [700, 0, 431], 16 // G
    lens = [new[0] + 333, 5, new[2]]
    case = Case(3, Hkv * G, Hkv, d, page, lens, seed=640 + G + page)
    if page < 300:
        case.table[0, 2], case.table[2, 0] = -1, case.g.n_pages
        case.dev_table.copy_(case.table)
    assert sparse_form(case.g, new, select, max(lens)) == form
    rows = {0, 1, R - 1, R, 333 % 700, 699, 700, 701, 1129, 1130, *range(5, 1131, 83)}
    sampled_sparse(case, new, select, sorted(rows), (0, Hkv - 1), max_len=max(lens))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("new", [[1, 1], [3, 9], [600, 40]])
def test_weights_are_left_as_they_are(dtype, new):
    """On a cache with weights nothing is added to them, in any of the forms."""
    lens = [n + 200 for n in new]
    case = Case(2, 32, 8, 64, 32, lens, dtype=dtype, weights=True, seed=660)
    before = case.w.clone()
    sampled_sparse(case, new, 4, sorted({0, sum(new) - 1, sum(new) // 2}), (0, 7), max_len=max(lens))
    assert torch.equal(case.w.isnan(), before.isnan()) and torch.equal(case.w.nan_to_num(), before.nan_to_num())


@pytest.mark.parametrize("order", ["nhd", "joined"])
@pytest.mark.parametrize("G,d,page", [(4, 128, 64), (8, 64, 32)])
def test_shared_waves_over_strided_pools(order, G, d, page):
    """Rows at other strides, first and last pages kept, a scale below 0."""
    new, lens = [301, 77], [301 + 500, 77 + 9]
    case = Case(2, 16 * G, 16, d, page, lens, seed=670 + G, order=order, sm_scale=-0.1)
    assert sparse_form(case.g, new, 6, max(lens)) == TILES
    sampled_sparse(case, new, 6, [0, 1, 150, 299, 300, 301, 320, 377], (0, 5, 15), first=2, recent=3, max_len=max(lens))


@pytest.mark.parametrize("Hkv,G,new,form", [(16, 4, [300, 45], TILES), (8, 4, [400, 45], WAVES), (4, 4, [30, 1], 0)])
def test_captured(Hkv, G, new, form):
    """Each form captured into a graph, without lse, and replayed after other
    inputs came in, with eager work between: the bits of the eager call."""
    dtype = FP32 if form == WAVES else BF16
    lens, T = [n + 400 for n in new], sum(new)
    case = Case(2, Hkv * G, Hkv, 128, 32, lens, dtype=dtype, seed=680 + Hkv)
    g, bounds, q = case.g, made_bounds(case), case.normal(T, Hkv * G, 128).cuda()
    assert sparse_form(g, new, 5, max(lens)) == form
    out, sel = torch.empty_like(q), torch.empty(T, Hkv, 5, dtype=torch.int32, device="cuda")
    ws = g.new_sparse_workspace(T, 5)
    call = lambda: g.sparse(case.cache, bounds, q, cu_of(new), 5, sel, out, ws, max_len=max(lens))  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in range(3):
        q.copy_(case.normal(*q.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), sel.clone()
        out.zero_(), sel.zero_(), ws.fill_(0xff)
        call()
        assert torch.equal(got[0], out) and torch.equal(got[1], sel) and out.isfinite().all(), n
