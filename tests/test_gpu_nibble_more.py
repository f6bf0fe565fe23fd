"""Attention over a 4-bit paged cache against float64 on the CPU: queries at the
ends of fp32's range."""
import pytest
import torch

from .paged4_util import Case4
from .paged_util import check_rows
from .test_gpu_append import cu_of
from .test_gpu_nibble import run_decode4, run_prefill4
from .test_gpu_paged import nan_like

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def sampled_prefill4(case, new, rows, max_len=0, q=None):
    """A prefill of which the given packed rows are compared."""
    g, cu, T = case.g, cu_of(new), sum(new)
    if q is None:
        q = case.normal(T, g.n_q_heads, g.head_dim)
    out, lse = nan_like(T + 1, g.n_q_heads, g.head_dim, dtype=case.dtype), nan_like(T + 1, g.n_q_heads, dtype=FP32)
    g.prefill(case.cache, q.cuda(), cu, out, g.new_workspace(T).fill_(0xff), lse=lse, max_len=max_len)
    torch.cuda.synchronize()
    ref = case.ref()
    at = [next(b for b in range(len(new)) if cu[b] <= r < cu[b + 1]) for r in rows]
    want = [ref.row(b, ref.lens[b] - new[b] + r - cu[b], q[r]) for b, r in zip(at, rows)]
    check_rows(out[list(rows)], lse[list(rows)], want)
    assert out[:T].isfinite().all(), "rows that are not compared"
    assert out[T:].isnan().all() and lse[T:].isnan().all(), "rows behind the last sequence"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 9, 1500])
def test_queries_past_the_largest_bf16_number(d, T):
    """fp32 numbers go on where bf16's end (from 0x7f7f8000 on they round to
    infinity): queries of 3.39e38 .. 3.4e38 on a group of keys small enough that
    their scores are ordinary, and zeros among those keys."""
    case = Case4(1, 8, 4, d, 16, [T + 40], dtype=FP32, seed=80 + T, sm_scale=0.02)
    for codes, scales in (case.k,):
        scales[..., 0] = torch.randint(3, 6, scales[..., 0].shape, generator=case.gen, dtype=torch.uint8).cuda()
        codes[..., 2] = 0
    q = case.normal(T, 8, d)
    top = torch.randint(0x7f7f8000, 0x7f800000, (T, 8, 16), generator=case.gen, dtype=torch.int32).view(FP32)
    q[..., :16] = torch.where(torch.rand(top.shape, generator=case.gen) < 0.5, top, -top)
    assert q.isfinite().all() and (q[..., :16].abs() > 3.389e38).all()
    if T == 1:
        run_decode4(case, q=q)
    sampled_prefill4(case, [T], sorted({*range(0, T, 97), *range(max(0, T - 40), T)}), q=q)


@pytest.mark.parametrize("T", [1, 9, 1500])
def test_queries_among_the_smallest_numbers(T):
    """Queries of 2^-120 and of 2^-127 on keys of 2^100 and more: their bits
    down to 2^-133 count (what lies below has no place in a bf16 number: off by
    2^-133 of each key element at most, once for each)."""
    case = Case4(1, 8, 4, 64, 16, [T + 40], dtype=FP32, seed=90 + T, sm_scale=1.0)
    codes, scales = case.k
    scales.copy_(torch.randint(227, 230, scales.shape, generator=case.gen, dtype=torch.uint8))
    q = case.normal(T, 8, 64)
    q[..., :32] *= 2.0 ** -104
    q[..., 32:] *= 2.0 ** -126
    lost = 64 * 2.0 ** -133 * 6 * 2.0 ** 102
    assert lost < 2.0 ** -20          # far below the tolerance of the rows' scores, 2^-18 and more
    sampled_prefill4(case, [T], sorted({*range(0, T, 97), *range(max(0, T - 40), T)}), q=q)
