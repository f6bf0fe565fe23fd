"""Refusals of the calls that fill a paged cache, of the 4-bit cache and of the
attention over selected pages: by the library before any HIP call, or by the
binding.  The pointers below are never followed."""
import ctypes

import pytest
import torch

from paper_2607_24788_amd import glide, paged, paged4

from .test_paged_args import ALIGN, BAD_CFG, BIG, INVALID, NULL, OK, P, SIZE, UNSUPPORTED, cache, cfg


@pytest.fixture(scope="module")
def lib():
    return glide.load_library()


def cache4(**kw):
    names = [n for n, _ in glide.Paged4CacheArg._fields_]
    return glide.Paged4CacheArg(*(kw.get(n, P) for n in names))


def rotation(freqs=P, positions=None, rot_dim=128, interleaved=0):
    return glide.Rotation(freqs, positions, rot_dim, interleaved)


def ref(x):
    return None if x is None or x == "null" else ctypes.byref(x)


def cu_of(cu):
    return None if cu is None else (ctypes.c_int32 * len(cu))(*cu)


def append(lib, c=None, k=None, four=False, rot="default", cu=(0, 3, 5), T=None, **kw):
    a = dict(q=P, kn=P, vn=P, q_out=P, bounds=None)
    a.update(kw)
    f = lib.glide_nibble_append if four else lib.glide_paged_append
    args = [ref(c or cfg()), ref(k or (cache4() if four else cache())), ref(rotation() if rot == "default" else rot),
            a["q"], a["kn"], a["vn"], cu_of(cu), (cu[-1] if cu else 5) if T is None else T, a["q_out"]]
    return f(*args, None) if four else f(*args, a["bounds"], None)


def bounds(lib, c=None, k=None, max_len=0, b=P):
    return lib.glide_paged_bounds(ref(c or cfg()), ref(k or cache()), max_len, b, None)


def read(lib, c=None, k=None, cu=(0, 3, 5), T=None, ko=P, vo=P):
    return lib.glide_nibble_read(ref(c or cfg()), ref(k or cache4()), cu_of(cu),
                                 (cu[-1] if cu else 5) if T is None else T, ko, vo, None)


def prefill4(lib, c=None, k=None, cu=(0, 3, 5), T=None, **kw):
    a = dict(q=P, max_len=0, out=P, lse=P, ws=P, n=BIG)
    a.update(kw)
    return lib.glide_nibble_prefill(ref(c or cfg()), ref(k or cache4()), a["q"], cu_of(cu),
                                    (cu[-1] if cu else 5) if T is None else T, a["max_len"], a["out"], a["lse"],
                                    a["ws"], a["n"], None)


def decode4(lib, c=None, k=None, **kw):
    a = dict(q=P, max_len=0, out=P, lse=P, ws=P, n=BIG)
    a.update(kw)
    return lib.glide_nibble_decode(ref(c or cfg()), ref(k or cache4()), a["q"], a["max_len"], a["out"], a["lse"],
                                   a["ws"], a["n"], None)


def sparse(lib, c=None, k=None, cu=(0, 3, 5), T=None, **kw):
    a = dict(bounds=P, q=P, select=8, first=1, recent=1, max_len=0, selected=P, out=P, lse=P, ws=P, n=BIG)
    a.update(kw)
    return lib.glide_paged_sparse(ref(c or cfg()), ref(k or cache()), a["bounds"], a["q"], cu_of(cu),
                                  (cu[-1] if cu else 5) if T is None else T, a["select"], a["first"], a["recent"],
                                  a["max_len"], a["selected"], a["out"], a["lse"], a["ws"], a["n"], None)


def append4(lib, **kw):
    return append(lib, four=True, **kw)


ROWS = [append, append4, read, prefill4, sparse]      # calls over packed rows
ALL = ROWS + [bounds, decode4]
FOUR = [append4, read, prefill4, decode4]


@pytest.mark.parametrize("i", range(len(BAD_CFG)))
def test_bad_configs(lib, i):
    kw, status = BAD_CFG[i]
    c = cfg(**kw)
    cu = (0, 3, 5) if c.batch < 3 else (0,) * c.batch + (5,)
    for call in ALL:
        assert call(lib, c=c, **(dict(cu=cu) if call in ROWS else {})) == status, call
    assert lib.glide_nibble_workspace_bytes(ctypes.byref(c), 10) == 0
    assert lib.glide_paged_sparse_workspace_bytes(ctypes.byref(c), 10, 4) == 0


def test_null_arguments(lib):
    for call in ALL:
        assert call(lib, c="null") == NULL and call(lib, k="null") == NULL
        names = ("k_codes", "k_scales", "v_codes", "v_scales", "block_table", "lens") if call in FOUR else \
            ("k", "v", "block_table", "lens")
        for name in names:
            assert call(lib, k=(cache4 if call in FOUR else cache)(**{name: None})) == NULL, (call, name)
    for call in ROWS:
        assert call(lib, cu=None) == NULL
    for call in (append, append4):
        for name in ("q", "q_out", "kn", "vn"):        # q and q_out go together
            assert call(lib, **{name: None}) == NULL
        assert call(lib, rot=rotation(freqs=None)) == NULL
    for call in (prefill4, decode4, sparse):
        for name in ("q", "out", "ws"):
            assert call(lib, **{name: None}) == NULL
    for name in ("bounds", "selected"):
        assert sparse(lib, **{name: None}) == NULL
    assert bounds(lib, b=None) == NULL and read(lib, ko=None) == NULL and read(lib, vo=None) == NULL


def test_alignment(lib):
    for call in ALL:
        k4 = call in FOUR
        for name, at in (("k_codes" if k4 else "k", P + 8), ("v_scales" if k4 else "v", P + 4), ("block_table", P + 1),
                         ("lens", P + 2)):
            assert call(lib, k=(cache4 if k4 else cache)(**{name: at})) == ALIGN, (call, name)
    for call in (append, append4):
        for name in ("q", "q_out", "kn", "vn"):
            assert call(lib, **{name: P + 8}) == ALIGN
        assert call(lib, rot=rotation(freqs=P + 4)) == ALIGN and call(lib, rot=rotation(positions=P + 2)) == ALIGN
    assert append(lib, bounds=P + 8) == ALIGN and bounds(lib, b=P + 4) == ALIGN
    assert read(lib, ko=P + 8) == ALIGN and read(lib, vo=P + 2) == ALIGN
    for call in (prefill4, decode4, sparse):
        for name, at in (("q", P + 8), ("out", P + 8), ("lse", P + 2), ("ws", P + 16)):
            assert call(lib, **{name: at}) == ALIGN
    assert sparse(lib, bounds=P + 8) == ALIGN and sparse(lib, selected=P + 2) == ALIGN


def test_rows(lib):
    for call in ROWS:
        for cu, T in (((0, 3, 2), None), ((1, 3, 5), None), ((0, 3, 5), 4), ((0, 3, 5), -1), ((0, -1, 5), None)):
            assert call(lib, cu=cu, T=T) == INVALID, call
        far = 2 ** 31 // (8 * 128 * 2)        # rows of a sequence that span 2 GiB
        assert call(lib, cu=(0, far, far)) == UNSUPPORTED
        assert call(lib, cu=(0, 0, 0)) == OK
    # nothing to do needs no tensor
    assert append(lib, cu=(0, 0, 0), q=None, kn=None, vn=None) == OK
    assert sparse(lib, cu=(0, 0, 0), q=None, out=None, ws=None, selected=None) == OK


def test_ranges(lib):
    for rot_dim in (-16, 8, 130, 144):
        for call in (append, append4):
            assert call(lib, rot=rotation(rot_dim=rot_dim)) == INVALID
    assert append(lib, rot=rotation(interleaved=2)) == INVALID
    for rot_dim in (16, 32, 96, 112):         # pairs across groups of 32
        assert append4(lib, rot=rotation(rot_dim=rot_dim)) == UNSUPPORTED
    for call in (bounds, prefill4, decode4, sparse):
        assert call(lib, max_len=-1) == INVALID
    for kw in (dict(select=0), dict(select=-4), dict(select=(1 << 26) + 1), dict(first=-1), dict(recent=0),
               dict(first=4, recent=5), dict(first=(1 << 31) - 1, recent=(1 << 31) - 1)):
        assert sparse(lib, **kw) == INVALID, kw
    # rows of a 4-bit cache are numbered in 32 bits
    most = cfg(n_pages=1 << 27, n_kv_heads=2, page_size=16)
    over = cfg(n_pages=(1 << 27) + 1, n_kv_heads=2, page_size=16)
    for call in FOUR:
        assert call(lib, c=over) == UNSUPPORTED
    for call in (prefill4, decode4):
        assert call(lib, c=most, n=0) == SIZE


def test_small_workspaces(lib):
    c = cfg(batch=2, max_pages=1000, window=1 << 20)
    size = lib.glide_nibble_workspace_bytes(ctypes.byref(c), 5)
    assert prefill4(lib, c=c, n=size - 1) == SIZE
    assert decode4(lib, c=c, n=lib.glide_nibble_workspace_bytes(ctypes.byref(c), 0) - 1) == SIZE
    assert sparse(lib, c=c, n=lib.glide_paged_sparse_workspace_bytes(ctypes.byref(c), 5, 8) - 1) == SIZE
    for n, k in ((-1, 8), ((1 << 31) + 1, 8), (5, 0), (5, (1 << 26) + 1)):
        assert lib.glide_paged_sparse_workspace_bytes(ctypes.byref(c), n, k) == 0


def test_sparse_workspace_never_falls(lib):
    for kw in (dict(), dict(max_pages=1 << 20, page_size=1), dict(n_q_heads=64, n_kv_heads=64, max_pages=5000)):
        c = cfg(**kw)
        f = lambda n: lib.glide_paged_sparse_workspace_bytes(ctypes.byref(c), n, 20)  # noqa: E731
        sizes = [f(n) for n in (0, 1, 2, 7, 31, 32, 33, 500, 5000, 100000)]
        assert sizes == sorted(sizes) and sizes[-1] < 1 << 30


# -- the binding -------------------------------------------------------------

SIZES = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=12, max_pages=5)


@pytest.fixture
def on_host(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)

    def make(g):
        t = torch.zeros(g.batch, g.max_pages, dtype=torch.int32)
        n = torch.zeros(g.batch, dtype=torch.int32)
        if isinstance(g, paged4.Paged4):
            return g.cache(*g.new_pools(device="cpu"), t, n)
        k, v, w = g.new_pools(device="cpu")
        return g.cache(k, v, t, n)
    return make


def layers(**kw):
    return paged.Paged(**{**SIZES, **kw}), paged4.Paged4(**{**SIZES, **kw})


def binding_calls(g, c, T=3):
    cu = [0, T, T]
    z = lambda *s: torch.zeros(s, dtype=g.torch_dtype)  # noqa: E731
    yield lambda: g.append(c, z(T, 2, 64), z(T, 2, 64), cu)
    if isinstance(g, paged4.Paged4):
        yield lambda: g.read(c, cu, z(T, 2, 64), z(T, 2, 64))
        yield lambda: g.prefill(c, z(T, 8, 64), cu, z(T, 8, 64), torch.zeros(8, dtype=torch.uint8))
        yield lambda: g.decode(c, z(T, 8, 64), z(T, 8, 64), torch.zeros(8, dtype=torch.uint8))
    else:
        b = g.new_bounds(device="cpu")
        yield lambda: g.page_bounds(c, b)
        yield lambda: g.sparse(c, b, z(T, 8, 64), cu, 4, torch.zeros(T, 2, 4, dtype=torch.int32), z(T, 8, 64),
                               torch.zeros(8, dtype=torch.uint8))


@pytest.mark.parametrize("kw", [dict(batch=3), dict(n_kv_heads=4), dict(head_dim=128), dict(page_size=32),
                                dict(n_pages=13), dict(max_pages=6)])
def test_caches_of_another_geometry(on_host, kw):
    for g, other in zip(layers(), layers(**kw)):
        for call in binding_calls(g, on_host(other)):
            with pytest.raises(ValueError, match="cache was made for"):
                call()


def test_caches_of_the_other_kind(on_host):
    a, b = layers()
    for g, c in ((a, on_host(b)), (b, on_host(a)), (a, None), (b, object())):
        for call in binding_calls(g, c):
            with pytest.raises(ValueError, match="Paged4?.cache"):
                call()


def test_a_4_bit_cache_takes_layers_of_both_types(on_host):
    """The type of q, k and v is no part of its geometry: the next argument is refused."""
    c = on_host(paged4.Paged4(**SIZES))
    g = paged4.Paged4(**{**SIZES, "dtype": torch.float32})
    with pytest.raises(ValueError, match="q has dtype"):
        g.decode(c, torch.zeros(2, 8, 64, dtype=torch.bfloat16), None, None)


def test_pools_of_a_4_bit_cache(on_host):
    g = paged4.Paged4(**SIZES)
    (kc, ks), v = g.new_pools(device="cpu")
    t, n = torch.zeros(2, 5, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    assert kc.shape == (12, 2, 16, 32) and ks.shape == (12, 2, 16, 2)
    for k, match in (((kc, ks[:-1]), "k_scales has shape"), ((kc.int(), ks), "k_codes has dtype"), (kc, "pair"),
                     ((kc.transpose(1, 2), ks), "contiguous"), ((kc.view(12, 2, 32, 16), ks), "k_codes has shape"),
                     ((kc, None), "must be a torch tensor")):
        with pytest.raises(ValueError, match=match):
            g.cache(k, v, t, n)
    with pytest.raises(ValueError, match="block_table has shape"):
        g.cache((kc, ks), v, torch.zeros(5, 2, dtype=torch.int32), n)
    with pytest.raises(ValueError, match="lens holds"):
        g.cache((kc, ks), v, t, n[:1])


def test_small_tensors(on_host):
    a, b = layers()
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    cu = [0, 2, 5]
    for g in (a, b):
        c = on_host(g)
        k, q = z(5, 2, 64), z(5, 8, 64)
        for args, kw, match in (((z(4, 2, 64), k, cu), {}, "k holds"), ((k, z(5, 1, 64), cu), {}, "v holds"),
                                ((k, k, cu), dict(q=q), "q and q_out"), ((k, k, cu), dict(q=q, q_out=z(4, 8, 64)), "q_out holds"),
                                ((k, k, cu), dict(freqs=z(32)), "freqs has dtype"),
                                ((k, k, cu), dict(freqs=z(32, dt=torch.float32), positions=z(4, dt=torch.int32)), "positions holds"),
                                ((k, k, [0, 5]), {}, "batch \\+ 1"), ((k, k, [0, 2, 1 << 32]), {}, "cu_seqlens.*32-bit"),
                                ((None, k, cu), {}, "k must be a torch tensor")):
            with pytest.raises(ValueError, match=match):
                g.append(c, *args, **kw)
    c, bd = on_host(a), a.new_bounds(device="cpu")
    ws, sel, q = z(8, dt=torch.uint8), z(5, 2, 4, dt=torch.int32), z(5, 8, 64)
    for args, match in (((bd[:-1], q, cu, 4, sel, q, ws), "bounds holds"), ((bd, q, cu, 5, sel, q, ws), "selected holds"),
                        ((bd, q[:4], cu, 4, sel, q, ws), "q holds"), ((bd, q, cu, 1 << 32, sel, q, ws), "n_select.*32-bit")):
        with pytest.raises(ValueError, match=match):
            a.sparse(c, *args)
    with pytest.raises(ValueError, match="bounds holds"):
        a.append(c, z(5, 2, 64), z(5, 2, 64), cu, bounds=bd[:2].contiguous())


def test_library_errors_reach_the_caller(on_host):
    g = paged.Paged(**SIZES)
    with pytest.raises(glide.GlideError):
        g.new_sparse_workspace(5, 0, device="cpu")
    with pytest.raises(glide.GlideError):
        paged4.Paged4(**{**SIZES, "head_dim": 96})
    with pytest.raises(ValueError, match="32-bit"):
        paged4.Paged4(**{**SIZES, "n_pages": 1 << 32})
