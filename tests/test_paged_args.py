"""Refusals of the paged cache's entry points that need no GPU: every argument
error is reported before any HIP call, by the library or by its binding.  The
pointers below are never followed."""
import ctypes

import pytest
import torch

from paper_2607_24788_amd import glide, paged

OK, NULL, INVALID, UNSUPPORTED, ALIGN, SIZE = 0, -1, -2, -3, -4, -5
P = 1 << 20          # an aligned address
BIG = 1 << 40        # a workspace size that is never too small


def cfg(**kw):
    c = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=glide.BF16, page_size=16, n_pages=40, max_pages=10,
             window=64, n_sinks=4, sm_scale=0.1)
    c.update(kw)
    return glide.PagedConfig(*[c[n] for n, _ in glide.PagedConfig._fields_])


def cache(**kw):
    a = glide.PagedCacheArg()
    a.k, a.v, a.weights, a.block_table, a.lens = (kw.get(n, P) for n in ("k", "v", "weights", "block_table", "lens"))
    for i in range(3):
        a.k_strides[i], a.v_strides[i] = kw.get("ks", (4096, 2048, 128))[i], kw.get("vs", (4096, 2048, 128))[i]
    return a


@pytest.fixture(scope="module")
def lib():
    return glide.load_library()


def prefill(lib, c=None, k=None, cu=(0, 3, 5), T=None, **kw):
    a = dict(q=P, kn=P, vn=P, observe=1, max_len=0, out=P, lse=P, ws=P, n=BIG)
    a.update(kw)
    arr = None if cu is None else (ctypes.c_int32 * len(cu))(*cu)
    return lib.glide_paged_prefill(None if c == "null" else ctypes.byref(c or cfg()),
                                   None if k == "null" else ctypes.byref(k or cache()), a["q"], a["kn"], a["vn"], arr,
                                   (cu[-1] if cu else 5) if T is None else T, a["observe"], a["max_len"], a["out"],
                                   a["lse"], a["ws"], a["n"], None)


def decode(lib, c=None, k=None, **kw):
    a = dict(q=P, kn=P, vn=P, max_len=0, out=P, lse=P, ws=P, n=BIG)
    a.update(kw)
    return lib.glide_paged_decode(None if c == "null" else ctypes.byref(c or cfg()),
                                  None if k == "null" else ctypes.byref(k or cache()), a["q"], a["kn"], a["vn"],
                                  a["max_len"], a["out"], a["lse"], a["ws"], a["n"], None)


def evict(lib, c=None, k=None, **kw):
    a = dict(budget=40, recent=8, dst=None, kept=P, lens=P, ws=P, n=BIG)
    a.update(kw)
    return lib.glide_paged_evict(None if c == "null" else ctypes.byref(c or cfg()),
                                 None if k == "null" else ctypes.byref(k or cache()), a["budget"], a["recent"],
                                 a["dst"], a["kept"], a["lens"], a["ws"], a["n"], None)


BAD_CFG = [
    (dict(batch=0), INVALID), (dict(n_q_heads=7), INVALID), (dict(n_kv_heads=0), INVALID), (dict(dtype=2), INVALID),
    (dict(page_size=0), INVALID), (dict(page_size=24), INVALID), (dict(page_size=2048), INVALID),
    (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=1 << 27), INVALID),
    (dict(window=-1), INVALID), (dict(window=(1 << 30) + 1), INVALID), (dict(n_sinks=-1), INVALID),
    (dict(window=0, n_sinks=0), INVALID), (dict(sm_scale=float("inf")), INVALID), (dict(sm_scale=float("nan")), INVALID),
    (dict(head_dim=96), UNSUPPORTED), (dict(n_q_heads=34), UNSUPPORTED), (dict(head_dim=0), INVALID),
    (dict(batch=1 << 20), UNSUPPORTED),
]


@pytest.mark.parametrize("i", range(len(BAD_CFG)))
def test_bad_configs(lib, i):
    kw, status = BAD_CFG[i]
    c = cfg(**kw)
    assert lib.glide_paged_workspace_bytes(ctypes.byref(c), 10, 1) == 0
    cu = (0, 3, 5) if c.batch < 3 else (0,) * c.batch + (5,)
    assert prefill(lib, c, cu=cu) == status
    assert decode(lib, c) == status
    assert evict(lib, c) == status


def test_null_arguments(lib):
    for call in (prefill, decode, evict):
        assert call(lib, c="null") == NULL
        assert call(lib, k="null") == NULL
        for name in ("k", "v", "block_table", "lens"):
            assert call(lib, k=cache(**{name: None})) == NULL
        assert call(lib, ws=None) == NULL
    for call in (prefill, decode):
        for name in ("q", "out", "kn", "vn"):      # k and v go together
            assert call(lib, **{name: None}) == NULL
    assert prefill(lib, cu=None) == NULL
    assert prefill(lib, k=cache(weights=None)) == NULL       # scored queries without weights
    assert evict(lib, k=cache(weights=None)) == NULL
    assert evict(lib, kept=None) == NULL and evict(lib, lens=None) == NULL
    assert lib.glide_paged_workspace_bytes(None, 0, 0) == 0


def test_alignment(lib):
    for call in (prefill, decode, evict):
        for kw in (dict(k=P + 8), dict(v=P + 2), dict(weights=P + 2), dict(block_table=P + 1), dict(lens=P + 2),
                   dict(ks=(4096, 2048, 124)), dict(vs=(4100, 2048, 128))):
            assert call(lib, k=cache(**kw)) == ALIGN
        assert call(lib, ws=P + 16) == ALIGN
    for call in (prefill, decode):
        for name in ("q", "kn", "vn", "out"):
            assert call(lib, **{name: P + 8}) == ALIGN
        assert call(lib, lse=P + 2) == ALIGN
    for name in ("dst", "kept", "lens"):
        assert evict(lib, **{name: P + 2}) == ALIGN


def test_ranges(lib):
    for call in (prefill, decode, evict):
        assert call(lib, k=cache(ks=(-4096, 2048, 128))) == INVALID
        assert call(lib, k=cache(vs=(1 << 60, 2048, 128))) == INVALID
    assert prefill(lib, max_len=-1) == INVALID and decode(lib, max_len=-1) == INVALID
    assert prefill(lib, observe=-1) == INVALID
    assert prefill(lib, cu=(1, 3, 5)) == INVALID and prefill(lib, cu=(0, 6, 5)) == INVALID
    assert prefill(lib, cu=(0, 3, 5), T=6) == INVALID and prefill(lib, cu=(0, 0, 0), T=-1) == INVALID
    assert prefill(lib, cu=(0, 0, 1 << 21)) == UNSUPPORTED   # 2^21 tokens of 2 KiB
    assert evict(lib, budget=0, recent=0) == INVALID and evict(lib, recent=-1) == INVALID
    assert evict(lib, budget=11, recent=8) == INVALID        # 4 sinks and 8 newest do not fit
    assert evict(lib, budget=(1 << 30) + 1) == INVALID
    assert lib.glide_paged_workspace_bytes(ctypes.byref(cfg()), (1 << 31) + 1, 0) == 0


def test_small_workspaces(lib):
    n = lib.glide_paged_workspace_bytes(ctypes.byref(cfg()), 5, 1)
    assert n > 256 and prefill(lib, n=n - 1) == SIZE
    n = lib.glide_paged_workspace_bytes(ctypes.byref(cfg()), 0, 1)
    assert n > 256 and decode(lib, n=n - 1) == SIZE
    assert evict(lib, n=255) == SIZE


def test_nothing_to_do(lib):
    """No token: no launch, and q, out need not be there."""
    assert prefill(lib, cu=(0, 0, 0), q=None, out=None, ws=None, n=0) == OK


@pytest.mark.parametrize("weights", [0, 1])
def test_workspace_serves_smaller_calls(lib, weights):
    """A size made for T tokens is enough for every smaller T and length."""
    for kw in (dict(), dict(batch=64, n_q_heads=32, n_kv_heads=8), dict(n_q_heads=16, n_kv_heads=1, head_dim=64)):
        c = ctypes.byref(cfg(**kw))
        sizes = [lib.glide_paged_workspace_bytes(c, t, weights)
                 for t in (0, 1, 2, 7, 31, 100, 500, 1000, 4000, 20000, 100000)]
        assert sizes == sorted(sizes) and sizes[0] >= 256
        assert lib.glide_paged_workspace_bytes(c, -1, weights) == 0


def make(**kw):
    a = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=40, max_pages=10)
    a.update(kw)
    return paged.Paged(**a)


def test_binding_refuses_bad_configs():
    for kw in (dict(page_size=3), dict(window=0), dict(dtype=torch.float16), dict(head_dim=80)):
        with pytest.raises(glide.GlideError):
            make(**kw)
    g = make(window=None)
    assert g.window == paged.FULL
    with pytest.raises(glide.GlideError):
        g.new_workspace(-1, device="cpu")


def test_binding_refuses_host_tensors():
    g = make()
    k, v, w = g.new_pools(weights=True, device="cpu")
    table, lens = torch.zeros(2, 10, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        g.cache(k, v, table, lens, w)
    with pytest.raises(ValueError, match="Paged.cache"):
        g.decode(None, None, None, None)
    with pytest.raises(ValueError, match="Paged.cache"):
        g.evict(None, 1, 0, None, None, None)
    with pytest.raises(ValueError, match="batch"):
        g.prefill(None, None, [0, 1], None, None)
