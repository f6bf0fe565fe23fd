"""Page bounds where tokens were taken back, and after an eviction."""
import pytest
import torch

from .paged_util import Case
from .test_gpu_append import check_plain, slot
from .test_gpu_paged import nan_like, run_evict

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def bounds_equal_the_pool(case, bounds):
    held, got, P = case.k.cpu().double(), bounds.cpu().double(), case.g.page_size
    for b, n in enumerate(case.lens.tolist()):
        for i in range(-(-n // P)):
            s = slot(case, b, i * P)
            if s is not None:
                x = held[s[0], :, :min(P, n - i * P)]
                assert torch.equal(got[s[0], :, 0], x.amin(1)) and torch.equal(got[s[0], :, 1], x.amax(1)), (b, i)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("G,page,new", [(4, 256, [60, 45]), (4, 64, [130, 40]), (1, 16, [20, 3]), (2, 64, [1, 1])])
def test_wider_bounds_stay(dtype, G, page, new):
    """Bounds that span more than a page's tokens (keys of tokens that were
    taken back) are joined to, whichever kernel keeps them: the first two calls
    take them by a launch of their own."""
    case = Case(2, 2 * G, 2, 128, page, [new[0] + page // 2, new[1] + page - 3], dtype=dtype, seed=600 + page + G)
    b = nan_like(*case.k.shape[:2], 2, 128, dtype=dtype)
    for s in range(2):
        at = int(case.table[s, (case.lens_host[s] - new[s]) // page])
        wide = case.normal(2, 128).abs() * 3
        b[at, :, 0], b[at, :, 1] = -wide.cuda(), wide.cuda()
    check_plain(case, new, 128, bounds=b)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_tokens_taken_back(dtype):
    """Drafts rejected and others appended in their place, in one call or token
    by token: the same bounds, those of all keys that were there; made anew,
    those of the keys that are."""
    got = []
    for step in (50, 1):
        case = Case(1, 8, 2, 128, 256, [150], dtype=dtype, seed=610)
        bounds = nan_like(*case.k.shape[:2], 2, 128, dtype=dtype)
        case.g.page_bounds(case.cache, bounds)
        first = case.k.cpu().double()[int(case.table[0, 0]), :, :150]
        k = (case.normal(50, 2, 128) * 0.5).to(dtype)
        for at in range(0, 50, step):
            case.lens.fill_(100 + at + step)
            x = k[at:at + step].contiguous().cuda()
            case.g.append(case.cache, x, x, [0, step], bounds=bounds)
        p = int(case.table[0, 0])
        every = torch.cat([first, k.double().transpose(0, 1)], 1)
        assert torch.equal(bounds[p, :, 0].cpu().double(), every.amin(1))
        assert torch.equal(bounds[p, :, 1].cpu().double(), every.amax(1))
        got.append(bounds[p].clone())
        case.g.page_bounds(case.cache, bounds)
        bounds_equal_the_pool(case, bounds)
        assert not torch.equal(bounds[p], got[-1])
    assert torch.equal(*got)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_after_an_eviction(dtype):
    case = Case(2, 8, 2, 128, 16, [90, 40], 64, 4, dtype=dtype, weights=True, seed=611)
    run_evict(case, 30, 10, alias=True)
    bounds = nan_like(*case.k.shape[:2], 2, 128, dtype=dtype)
    case.g.page_bounds(case.cache, bounds)
    assert case.lens.tolist() == [30, 30]
    bounds_equal_the_pool(case, bounds)
