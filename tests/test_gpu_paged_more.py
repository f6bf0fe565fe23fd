"""Calls of the paged softmax cache beside tests/test_gpu_paged.py's, against
the same float64 definition (tests/paged_util.py)."""
import pytest
import torch

from .paged_util import Case
from .test_gpu_paged import run_decode, run_evict, run_prefill

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
