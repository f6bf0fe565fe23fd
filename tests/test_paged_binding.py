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


# the 32 bits that are left of it: another number, in range or out of it
BIG = [1 << 32, (1 << 32) + 3, (1 << 31) + 16, -(1 << 32) + 2]


@pytest.mark.parametrize("x", BIG)
@pytest.mark.parametrize("name", [*SIZES, "window", "n_sinks"])
def test_sizes_past_32_bits(name, x):
    with pytest.raises(ValueError, match=f"{name} = {x} is not a 32-bit"):
        layer(**{"window": 64, "n_sinks": 4, name: x})


def test_a_window_in_range_is_the_library_s():
    for w in (None, 1, 1 << 30):
        g = layer(window=w)
        assert g.window == g.cfg.window == (paged.FULL if w is None else w)


@pytest.mark.parametrize("x", BIG)
def test_arguments_past_32_bits(cache_of, x):
    g = layer()
    c = cache_of(g)
    with pytest.raises(ValueError, match="n_observe.*32-bit"):
        g.prefill(c, None, [0, 1, 2], None, None, n_observe=x)
    for cu in ([0, x, 2], [0, 1, x]):
        with pytest.raises(ValueError, match="cu_seqlens.*32-bit"):
            g.prefill(c, None, cu, None, None)
    with pytest.raises(ValueError, match="n_recent.*32-bit"):
        g.evict(c, 40, x, None, None, None)
    with pytest.raises(ValueError, match="budget.*32-bit"):
        g.evict(c, x, 2, None, None, None)


@pytest.mark.parametrize("x", [1 << 64, (1 << 63) + 5])
def test_arguments_past_64_bits(cache_of, x):
    g = layer()
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    ws = g.new_workspace(2, device="cpu")
    with pytest.raises(ValueError, match="max_len.*64-bit"):
        g.prefill(cache_of(g), q, [0, 1, 2], q, ws, max_len=x)
    with pytest.raises(ValueError, match="max_len.*64-bit"):
        g.decode(cache_of(g), q, q, ws, max_len=x)
    with pytest.raises(ValueError, match="max_total_tokens.*64-bit"):
        g.new_workspace(x, device="cpu")


def test_sizes_are_whole_numbers():
    for kw in (dict(window=64.0), dict(batch="2"), dict(n_sinks=1.5)):
        with pytest.raises(TypeError):
            layer(**kw)


@pytest.fixture
def empty_is_nan():
    """torch.empty gives NaN, as memory of an earlier use may."""
    torch.use_deterministic_algorithms(True)
    yield
    torch.use_deterministic_algorithms(False)


def test_new_weights_are_zero(empty_is_nan):
    """Tokens that a caller writes itself into new pools add up from 0."""
    k, v, w = layer().new_pools(weights=True, device="cpu")
    assert k.isnan().all()      # (the fixture's doing)
    assert torch.equal(w, torch.zeros(12, 2, 16))
    assert layer().new_pools(device="cpu")[2] is None
