"""What the paged cache's binding refuses before the library is called, on the
CPU: caches of another geometry, numbers that 32 bits do not hold."""
import pytest
import torch

from paper_2607_24788_amd import paged

SIZES = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=12, max_pages=5)


def layer(**kw):
    return paged.Paged(**{**SIZES, **kw})


def calls(g, cache, weights=True):
    """Every entry point with `cache`, and no tensor that it could follow."""
    yield lambda: g.prefill(cache, None, [0] * g.batch + [1], None, None, n_observe=1 if weights else 0)
    yield lambda: g.decode(cache, None, None, None)
    yield lambda: g.evict(cache, 40, 2, None, None, None)


@pytest.fixture
def cache_of(monkeypatch):
    """Caches of host tensors, which nothing here follows."""
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)

    def make(g):
        k, v, w = g.new_pools(weights=True, device="cpu")
        return g.cache(k, v, torch.zeros(g.batch, g.max_pages, dtype=torch.int32),
                       torch.zeros(g.batch, dtype=torch.int32), w)
    return make


OTHER = [dict(batch=3), dict(n_kv_heads=4), dict(head_dim=128), dict(page_size=32), dict(n_pages=13), dict(max_pages=6),
         dict(dtype=torch.float32)]


@pytest.mark.parametrize("i", range(len(OTHER)))
def test_caches_of_another_geometry(cache_of, i):
    name = next(iter(OTHER[i]))
    a, b = layer(), layer(**OTHER[i])
    for g, other in ((a, b), (b, a)):
        for call in calls(g, cache_of(other)):
            with pytest.raises(ValueError, match=f"cache was made for.*{name}"):
                call()


@pytest.mark.parametrize("kw", [dict(), dict(window=33), dict(n_sinks=3), dict(n_q_heads=16), dict(sm_scale=0.5)])
def test_layers_that_share_a_cache(cache_of, kw):
    """A layer of the same geometry takes the cache: the next argument is refused."""
    for call in calls(layer(**kw), cache_of(layer())):
        with pytest.raises(ValueError, match="(q|kept) must be a torch tensor"):
            call()


def test_not_a_cache():
    g = layer()
    for call in calls(g, object()):
        with pytest.raises(ValueError, match="Paged.cache"):
            call()
