"""Attention over a 4-bit paged cache against float64 on the CPU: decode and
prefill, windows and sinks, missing pages, drawn calls, streams and graphs."""
import math
import random

import pytest
import torch

from .paged4_util import Case4
from .paged_util import check_rows
from .test_gpu_append import check_four, cu_of
from .test_gpu_paged import DECODE, PREFILL, nan_like

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def run_decode4(case, max_len=0, q=None):
    g, B = case.g, case.g.batch
    if q is None:
        q = case.normal(B, g.n_q_heads, g.head_dim)
    ref = case.ref()
    want = [ref.row(b, n - 1, q[b]) for b, n in enumerate(ref.lens)]
    out, lse = nan_like(B + 1, g.n_q_heads, g.head_dim, dtype=case.dtype), nan_like(B + 1, g.n_q_heads, dtype=FP32)
    ws = g.new_workspace().fill_(0xff)
    g.decode(case.cache, q.cuda(), out, ws, lse=lse, max_len=max_len)
    torch.cuda.synchronize()
    check_rows(out[:B], lse[:B], want)
    assert out[B:].isnan().all() and lse[B:].isnan().all(), "rows behind the last sequence"
    return out


def run_prefill4(case, new, max_len=0):
    g, cu, T = case.g, cu_of(new), sum(new)
    q = case.normal(T, g.n_q_heads, g.head_dim)
    ref = case.ref()
    want = [ref.row(b, ref.lens[b] - n + i, q[cu[b] + i]) for b, n in enumerate(new) for i in range(n)]
    out, lse = nan_like(T + 1, g.n_q_heads, g.head_dim, dtype=case.dtype), nan_like(T + 1, g.n_q_heads, dtype=FP32)
    ws = g.new_workspace(T).fill_(0xff)
    g.prefill(case.cache, q.cuda(), cu, out, ws, lse=lse, max_len=max_len)
    torch.cuda.synchronize()
    check_rows(out[:T], lse[:T], want)
    assert out[T:].isnan().all() and lse[T:].isnan().all(), "rows behind the last sequence"


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("i", range(len(DECODE)))
def test_decode(i, dtype):
    B, Hq, Hkv, d, page, lens, W, ns = DECODE[i]
    run_decode4(Case4(B, Hq, Hkv, d, page, lens, W, ns, dtype=dtype, seed=i))


@pytest.mark.parametrize("max_len", [1, 600, 2100, 1 << 20])
def test_decode_length_hint_changes_no_result(max_len):
    run_decode4(Case4(2, 8, 2, 128, 16, [2100, 600], dtype=FP32, seed=31), max_len)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_over_many_pieces(dtype, d):
    run_decode4(Case4(1, 4, 1, d, 64, [20001], None, 0, dtype=dtype, seed=32), 20001)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_decode_large_scores(dtype):
    """Scores of several hundred: a few tokens carry all the weight; a scale below 0."""
    run_decode4(Case4(2, 8, 2, 64, 16, [400, 33], dtype=dtype, seed=33, scale=8.0))
    run_decode4(Case4(2, 8, 2, 64, 16, [400, 33], dtype=dtype, seed=33, sm_scale=-0.3))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_decode_missing_pages(dtype):
    case = Case4(5, 8, 2, 128, 16, [100, 64, 90, 48, 16], dtype=dtype, seed=34)
    case.table[0, 2], case.table[1, 0], case.table[2, 5] = -1, case.g.n_pages, -7
    case.table[4, :] = -1
    case.dev_table.copy_(case.table)
    case.lens.copy_(torch.tensor([100, 64, 90, -3, 16]))
    case.lens_host = [100, 64, 90, 0, 16]
    run_decode4(case)
    over = Case4(1, 4, 2, 64, 16, [64], dtype=dtype, seed=35, extra_pages=0)
    over.lens.fill_(1 << 30)
    run_decode4(over)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("i", range(len(PREFILL)))
def test_prefill(i, dtype):
    B, Hq, Hkv, d, page, lens, new, W, ns, _ = PREFILL[i]
    run_prefill4(Case4(B, Hq, Hkv, d, page, lens, W, ns, dtype=dtype, seed=50 + i), new)


@pytest.mark.parametrize("max_len", [1, 900, 1 << 20])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prefill_length_hint_changes_no_result(dtype, max_len):
    run_prefill4(Case4(2, 8, 2, 64, 16, [900, 700], 600, 4, dtype=dtype, seed=69), [40, 9], max_len)


@pytest.mark.parametrize("dtype,page,d,W,ns,hist", [(FP32, 16, 128, None, 0, 0), (FP32, 64, 64, 200, 70, 90),
                                                    (BF16, 8, 128, 333, 4, 50), (BF16, 64, 64, None, 0, 0)])
def test_prefill_many_rows(dtype, page, d, W, ns, hist):
    new = [500, 0, 141]
    case = Case4(3, 16, 8, d, page, [n + (hist if n else 0) for n in new], W, ns, dtype=dtype, seed=67)
    case.table[0, 3] = -1
    case.dev_table.copy_(case.table)
    run_prefill4(case, new)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prefill_many_rows_in_pieces(dtype):
    run_prefill4(Case4(1, 8, 1, 128, 64, [2777], None, 0, dtype=dtype, seed=68), [100], max_len=2777)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prefill_missing_pages(dtype):
    """Pages that are not allocated; more queries than lens says."""
    case = Case4(3, 8, 2, 128, 16, [150, 140, 60], None, 2, dtype=dtype, seed=72)
    case.table[0, 3], case.table[1, 0], case.table[1, 8] = -1, case.g.n_pages, 1 << 30
    case.dev_table.copy_(case.table)
    case.lens.copy_(torch.tensor([150, 140, 50]))
    case.lens_host = [150, 140, 50]
    run_prefill4(case, [70, 140, 60])


def test_many_sequences():
    """More sequences than one launch takes."""
    new = [(7 * i) % 5 for i in range(300)]
    run_prefill4(Case4(300, 4, 2, 64, 16, [n + i % 19 for i, n in enumerate(new)], 9, 1, seed=73), new)


@pytest.mark.parametrize("seed", range(24))
def test_drawn(seed):
    r = random.Random(2000 + seed)
    dtype = r.choice([BF16, BF16, FP32])
    Hkv, G, d = r.choice([1, 2, 3]), r.choice([1, 2, 3, 4, 7, 8, 16]), r.choice([64, 128])
    page = r.choice([1, 2, 8, 16, 16, 32, 64, 128])
    B = r.randint(1, 4)
    new = [r.choice([0, 1, 2, r.randint(1, 130)]) for _ in range(B)]
    lens = [n + r.choice([0, 0, r.randint(0, 40), r.randint(0, 400)]) for n in new]
    W = r.choice([None, 1, r.randint(1, 64), r.randint(1, 300), 0])
    ns = r.choice([0, 1, 4, r.randint(1, 150)])
    if W == 0 and ns == 0:
        ns = 2
    case = Case4(B, Hkv * G, Hkv, d, page, lens, W, ns, dtype=dtype, seed=200 + seed, scale=r.choice([0.5, 1.0, 2.0]))
    if r.random() < 0.4 and case.table.shape[1] > 2:
        case.table[r.randrange(B), r.randrange(case.table.shape[1] - 1)] = r.choice([-1, case.g.n_pages])
        case.dev_table.copy_(case.table)
    if sum(new):
        check_four(case, new, r.choice([0, 64]))
        run_prefill4(case, new, r.choice([0, max(lens)]))
    run_decode4(case, r.choice([0, max(lens)]))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_query_that_is_not_finite(dtype):
    """Its rows are NaN; the others, of the same group, are not touched."""
    case = Case4(1, 8, 2, 128, 16, [90], dtype=dtype, seed=74)
    q = case.normal(1, 8, 128)
    clean = run_decode4(case, q=q).clone()
    q[0, 1, 5], q[0, 6, 0] = math.nan, math.inf
    out = torch.empty_like(clean[:1])
    case.g.decode(case.cache, q.cuda(), out, case.g.new_workspace())
    for h in range(8):
        if h in (1, 6):
            assert not out[0, h].isfinite().any()
        else:
            assert torch.equal(out[0, h], clean[0, h])


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_session(dtype):
    """As a program uses it: a prompt appended and read out, tokens one by one,
    a few at once; on a stream of its own, with a window and sinks."""
    case = Case4(2, 8, 2, 128, 16, [150, 150], 70, 4, dtype=dtype, seed=75)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for at, new in (([90, 60], [90, 60]), ([91, 61], [1, 1]), ([92, 62], [1, 1]), ([99, 62], [7, 0])):
            case.lens.copy_(torch.tensor(at, dtype=torch.int32))
            case.lens_host = at
            check_four(case, new, 128)
            if max(new) == 1:
                run_decode4(case, max(at))
            else:
                run_prefill4(case, new, max(at))


def test_captured():
    """A step captured into a graph (append, prefill, decode) and replayed with
    eager work between; two graphs share a workspace."""
    case = Case4(2, 8, 2, 128, 16, [300, 140], seed=76)
    g, cu = case.g, [0, 20, 33]
    f = (10000.0 ** (-torch.arange(0, 128, 2).double() / 128)).float().cuda()
    q, k, v = (case.normal(33, h, 128).cuda() for h in (8, 2, 2))
    out, lse, one = torch.empty_like(q), torch.empty(33, 8, device="cuda"), torch.empty_like(q[:2])
    ws = g.new_workspace(33)

    def prompt():
        g.append(case.cache, k, v, cu, q=q, q_out=out, freqs=f)
        g.prefill(case.cache, q, cu, out, ws, lse=lse)

    def token():
        g.decode(case.cache, q[:2], one, ws)
    prompt()
    token()
    torch.cuda.synchronize()
    graphs = []
    for call in (prompt, token):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    for n in range(3):
        q.mul_(1.25)
        k.add_(0.25)
        for x in graphs:
            x.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, one, *case.k, *case.v)]
        for t in (out, lse, one):
            t.fill_(math.nan)
        prompt()
        token()
        for x, y in zip(got, (out, lse, one, *case.k, *case.v)):
            assert torch.equal(x, y), n
