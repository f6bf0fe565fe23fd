"""Thin ctypes binding of the paged softmax cache (``glide_paged_*`` in
include/glide.h): attention with a sliding window and sinks over a key-value
cache held in pages, the attention weight that each cached token has received,
and the eviction of the tokens that received least.

Argument marshalling only, as in ``glide.py``: every step runs in the HIP
kernels behind the C ABI, and there is no fallback.
"""
import array
import ctypes
import operator

import torch

from . import glide

FULL = 1 << 30   # a window that never ends: causal softmax attention


def _fits(name, x, bits=32):
    """x, refused where the library's integer would hold another number (ctypes
    drops the bits that do not fit)."""
    if not -(1 << (bits - 1)) <= x < 1 << (bits - 1):
        raise ValueError(f"{name} = {x} is not a {bits}-bit number")
    return x


def _tensor(name, t, device, dtype, numel):
    """Refuse what the library cannot see to be wrong: not a contiguous tensor
    of the cache's device (its index) and the expected type with `numel`
    elements or more.  Returns its address."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if t.dtype is dtype and t.get_device() == device and t.is_contiguous() and t.numel() >= numel:
        return t.data_ptr()
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, the cache on cuda:{device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"{name} holds {t.numel()} elements, at least {numel} needed")


def _cu_arg(g, cu_seqlens):
    """cu_seqlens as an array of the library's integers, and its last entry."""
    cu = list(cu_seqlens)
    if len(cu) != g.batch + 1:
        raise ValueError("cu_seqlens needs batch + 1 entries")
    try:
        return array.array("i", cu), int(cu[-1])
    except (TypeError, OverflowError):
        cu = [_fits("cu_seqlens entry", int(x)) for x in cu]
    return array.array("i", cu), cu[-1]


def _rotation(freqs, interleaved, positions, device, T):
    """The library's struct of a rotation, or None where there is none."""
    at = None if positions is None else _tensor("positions", positions, device, torch.int32, T)
    if freqs is None:
        return None
    return ctypes.byref(glide.Rotation(_tensor("freqs", freqs, device, torch.float32, 0), at,
                                       _fits("2 * freqs", 2 * freqs.numel()), int(bool(interleaved))))


def _append_rows(g, dev, q, k, v, q_out, T):
    """Pointers of an append of T tokens, checked."""
    dt, nq, nkv = g.torch_dtype, T * g.n_q_heads * g.head_dim, T * g.n_kv_heads * g.head_dim
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    return (None if q is None else _tensor("q", q, dev, dt, nq), _tensor("k", k, dev, dt, nkv),
            _tensor("v", v, dev, dt, nkv), None if q is None else _tensor("q_out", q_out, dev, dt, nq))


class PagedCache:
    """The cache of one layer: its tensors, the struct that names them to the
    library, and the geometry that they were checked for.  Made by
    ``Paged.cache``; every ``Paged`` of the same geometry takes it."""

    def __init__(self, k_pool, v_pool, block_table, lens, weights, arg, geometry):
        self.k_pool, self.v_pool, self.weights = k_pool, v_pool, weights
        self.block_table, self.lens = block_table, lens
        self.device = k_pool.device
        self.geometry = geometry
        self._dev = k_pool.get_device()
        self._arg = arg
        self._ref = ctypes.byref(arg)


class Paged:
    """A configured layer over a paged cache (mirrors ``glide_paged_config``).

    ``window``: tokens that a query sees, its own among them (None: all);
    ``n_sinks``: first tokens that stay visible whatever the window.  Pools are
    [n_pages][n_kv_heads][page_size][head_dim]; a transposed view of another
    order works as long as a row's elements are consecutive and rows start on
    16 bytes.
    """

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages, window=None, n_sinks=0,
                 dtype=torch.bfloat16, sm_scale=None, lib=None):
        self.lib = lib if lib is not None else glide.load_library()
        if window is None:
            window = FULL
        batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages, window, n_sinks = (
            _fits(name, operator.index(x)) for name, x in (
                ("batch", batch), ("n_q_heads", n_q_heads), ("n_kv_heads", n_kv_heads), ("head_dim", head_dim),
                ("page_size", page_size), ("n_pages", n_pages), ("max_pages", max_pages), ("window", window),
                ("n_sinks", n_sinks)))
        if sm_scale is None:
            sm_scale = head_dim ** -0.5
        code = {torch.float32: glide.F32, torch.bfloat16: glide.BF16}.get(dtype, 99)
        self.cfg = glide.PagedConfig(batch, n_q_heads, n_kv_heads, head_dim, code, page_size, n_pages, max_pages,
                                     window, n_sinks, float(sm_scale))
        self._ref = ctypes.byref(self.cfg)
        self._cu = ctypes.c_int32 * (batch + 1)
        self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim = batch, n_q_heads, n_kv_heads, head_dim
        self.page_size, self.n_pages, self.max_pages = page_size, n_pages, max_pages
        self.window, self.n_sinks, self.sm_scale, self.torch_dtype = window, n_sinks, float(sm_scale), dtype
        # what a cache's tensors are laid out by (query heads, window and sinks are not)
        self.geometry = (batch, n_kv_heads, head_dim, page_size, n_pages, max_pages, dtype)
        if self.workspace_bytes(0) == 0:
            raise glide.GlideError(-2, "glide_paged_workspace_bytes", self.lib)

    # -- buffers -------------------------------------------------------------
    def workspace_bytes(self, max_total_tokens=0, weights=False):
        return self.lib.glide_paged_workspace_bytes(self._ref, _fits("max_total_tokens", int(max_total_tokens), 64),
                                                    int(bool(weights)))

    def new_workspace(self, max_total_tokens=0, weights=False, device="cuda"):
        """Workspace for every call of up to max_total_tokens packed tokens;
        weights: on a cache that keeps attention weights."""
        n = self.workspace_bytes(max_total_tokens, weights)
        if n == 0:
            raise glide.GlideError(-2, "glide_paged_workspace_bytes", self.lib)
        return torch.empty(n, dtype=torch.uint8, device=device)

    def new_pools(self, weights=False, device="cuda"):
        """K and V pools, and the weights' pool or None.  K and V are not
        cleared: slots that no token was written to are never used.  Weights
        are 0; tokens that a call appends start from 0, but those that a caller
        writes into pages of earlier tokens (and reads with k, v None) have the
        weights that the caller leaves there."""
        shape = (self.n_pages, self.n_kv_heads, self.page_size, self.head_dim)
        k, v = (torch.empty(shape, dtype=self.torch_dtype, device=device) for _ in range(2))
        return k, v, (torch.zeros(shape[:3], dtype=torch.float32, device=device) if weights else None)

    def cache(self, k_pool, v_pool, block_table, lens, weights=None):
        """The cache of one layer.  The tensors are used in place: a caller
        moves lens on and fills block_table between calls."""
        arg = glide.PagedCacheArg()
        shape = (self.n_pages, self.n_kv_heads, self.page_size, self.head_dim)
        for name, t, strides in (("k_pool", k_pool, arg.k_strides), ("v_pool", v_pool, arg.v_strides)):
            if not isinstance(t, torch.Tensor) or not t.is_cuda:
                raise ValueError(f"{name} must be a device tensor")
            if t.dtype != self.torch_dtype:
                raise ValueError(f"{name} has dtype {t.dtype}, expected {self.torch_dtype}")
            if tuple(t.shape) != shape:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
            if t.stride(3) != 1:
                raise ValueError(f"{name}: the elements of a row must be consecutive")
            span = self.head_dim   # elements that the dimensions so far take
            for stride, i in sorted((t.stride(i), i) for i in range(3) if shape[i] > 1):
                if stride < span:
                    raise ValueError(f"{name}: rows overlap (strides {t.stride()})")
                strides[i], span = stride, stride * (shape[i] - 1) + span
        if v_pool.device != k_pool.device:
            raise ValueError("k_pool and v_pool are on different devices")
        dev = k_pool.get_device()
        arg.k, arg.v = k_pool.data_ptr(), v_pool.data_ptr()
        arg.block_table = _tensor("block_table", block_table, dev, torch.int32, self.batch * self.max_pages)
        arg.lens = _tensor("lens", lens, dev, torch.int32, self.batch)
        if tuple(block_table.shape) != (self.batch, self.max_pages):
            raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected "
                             f"{(self.batch, self.max_pages)}")
        if weights is not None:
            arg.weights = _tensor("weights", weights, dev, torch.float32,
                                  self.n_pages * self.n_kv_heads * self.page_size)
        return PagedCache(k_pool, v_pool, block_table, lens, weights, arg, self.geometry)

    # -- calls ---------------------------------------------------------------
    def _check_cache(self, cache):
        """Refuse a cache whose tensors another geometry was checked for: the
        library would follow its addresses with this layer's sizes."""
        if not isinstance(cache, PagedCache):
            raise ValueError("cache must come from Paged.cache")
        if cache.geometry != self.geometry:
            names = ("batch", "n_kv_heads", "head_dim", "page_size", "n_pages", "max_pages", "dtype")
            off = [f"{n} {x}, this layer has {y}" for n, x, y in zip(names, cache.geometry, self.geometry) if x != y]
            raise ValueError("cache was made for " + "; ".join(off))

    def _rows(self, cache, q, k, v, out, lse, T):
        """Pointers of a call over T rows of queries, checked."""
        if type(cache) is not PagedCache or cache.geometry is not self.geometry:
            self._check_cache(cache)
        dev, dt = cache._dev, self.torch_dtype
        nq, nkv = T * self.n_q_heads * self.head_dim, T * self.n_kv_heads * self.head_dim
        if (k is None) != (v is None):
            raise ValueError("k and v go together")
        return (_tensor("q", q, dev, dt, nq), None if k is None else _tensor("k", k, dev, dt, nkv),
                None if v is None else _tensor("v", v, dev, dt, nkv), _tensor("out", out, dev, dt, nq),
                None if lse is None else _tensor("lse", lse, dev, torch.float32, T * self.n_q_heads))

    def _workspace(self, cache, workspace):
        return _tensor("workspace", workspace, cache._dev, torch.uint8, 0), workspace.numel()

    def _call(self, name, cache, stream, *args):
        dev = cache._dev
        if dev != torch.cuda.current_device():
            with torch.cuda.device(dev):
                return self._call(name, cache, stream, *args)
        stream = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
        s = getattr(self.lib, name)(self._ref, cache._ref, *args, stream)
        if s:
            raise glide.GlideError(s, name, self.lib)

    def prefill(self, cache, q, cu_seqlens, out, workspace, k=None, v=None, lse=None, n_observe=0, max_len=0,
                stream=None):
        """Append k, v (if given) and read out one row per token and head.
        q, out [T][Hq][d], k, v [T][Hkv][d], lse [T][Hq] fp32; the weights of
        the last n_observe queries of every sequence are added up, from 0 for
        the tokens of k, v.  Without k, v the tokens are in the cache, and
        their weights are added to as they are."""
        cu = list(map(int, cu_seqlens))
        if len(cu) != self.batch + 1:
            raise ValueError("cu_seqlens needs batch + 1 entries")
        n_observe, max_len, cu_arg = int(n_observe), int(max_len), self._cu(*cu)
        if cu_arg[:] != cu or n_observe >> 31 or max_len >> 63:   # (one test on a short call's path)
            for x in cu:
                _fits("cu_seqlens entry", x)
            _fits("n_observe", n_observe)
            _fits("max_len", max_len, 64)
        qp, kp, vp, op, lp = self._rows(cache, q, k, v, out, lse, max(cu[-1], 0))
        if n_observe and cache.weights is None:
            raise ValueError("n_observe needs a cache with weights")
        ws, n = self._workspace(cache, workspace)
        self._call("glide_paged_prefill", cache, stream, qp, kp, vp, cu_arg, cu[-1],
                   n_observe, max_len, op, lp, ws, n)

    def append(self, cache, k, v, cu_seqlens, q=None, q_out=None, freqs=None, interleaved=False, positions=None,
               bounds=None, stream=None):
        """Write k, v [T][Hkv][d] to their pages, k rotated, and q [T][Hq][d]
        rotated to q_out (which may be q).  freqs: fp32 [rot_dim / 2], radians
        per position (None: no rotation); positions: int32 [T] (None: those in
        the cache).  bounds (``new_bounds``): the pages' least and largest keys,
        brought up to date.  prefill, decode and sparse then take the tokens
        without k, v."""
        if type(cache) is not PagedCache or cache.geometry is not self.geometry:
            self._check_cache(cache)
        dev = cache._dev
        cu, T = _cu_arg(self, cu_seqlens)
        rot = _rotation(freqs, interleaved, positions, dev, T)
        qp, kp, vp, op = _append_rows(self, dev, q, k, v, q_out, max(T, 0))
        bp = None if bounds is None else self._bounds_of(cache, bounds)
        self._call("glide_paged_append", cache, stream, rot, qp, kp, vp, cu.buffer_info()[0], T, op, bp)

    def new_bounds(self, device="cuda"):
        """Room for the least and the largest key elements of every page: not
        cleared (``append`` sets a page's with its first token, ``page_bounds``
        all)."""
        return torch.empty((self.n_pages, self.n_kv_heads, 2, self.head_dim), dtype=self.torch_dtype, device=device)

    def _bounds_of(self, cache, bounds):
        if type(cache) is not PagedCache or cache.geometry is not self.geometry:
            self._check_cache(cache)
        return _tensor("bounds", bounds, cache._dev, self.torch_dtype,
                       2 * self.n_pages * self.n_kv_heads * self.head_dim)

    def page_bounds(self, cache, bounds, max_len=0, stream=None):
        """The bounds of every page of the sequences from the keys in the
        cache: where they were written without ``append``, after an eviction,
        and after tokens were taken back (``append`` only ever widens a page's
        bounds)."""
        bp = self._bounds_of(cache, bounds)
        self._call("glide_paged_bounds", cache, stream, _fits("max_len", int(max_len), 64), bp)

    def decode(self, cache, q, out, workspace, k=None, v=None, lse=None, max_len=0, stream=None):
        """One token per sequence: q, out [B][Hq][d], k, v [B][Hkv][d],
        lse [B][Hq] fp32.  On a cache with weights every query adds its (see
        prefill)."""
        max_len = int(max_len)
        if max_len >> 63:
            _fits("max_len", max_len, 64)
        qp, kp, vp, op, lp = self._rows(cache, q, k, v, out, lse, self.batch)
        ws, n = self._workspace(cache, workspace)
        self._call("glide_paged_decode", cache, stream, qp, kp, vp, max_len, op, lp, ws, n)

    def new_sparse_workspace(self, max_total_tokens, n_select, device="cuda"):
        """Workspace for every ``sparse`` call of up to max_total_tokens rows
        and this n_select."""
        n = self.lib.glide_paged_sparse_workspace_bytes(self._ref, _fits("max_total_tokens", int(max_total_tokens), 64),
                                                        _fits("n_select", int(n_select)))
        if n == 0:
            raise glide.GlideError(-2, "glide_paged_sparse_workspace_bytes", self.lib)
        return torch.empty(n, dtype=torch.uint8, device=device)

    def sparse(self, cache, bounds, q, cu_seqlens, n_select, selected, out, workspace, n_first=1, n_recent=1, lse=None,
               max_len=0, stream=None):
        """Read out one row per query and head over the n_select pages that
        each (query, KV head) selects by the pages' bounds (kept by ``append``,
        made by ``page_bounds``): the first n_first, the last n_recent, and the
        largest scores of the others.  q, out [T][Hq][d], lse [T][Hq] fp32;
        selected [T][Hkv][n_select] int32: the pages' numbers in their
        sequence, -1 behind the last.  The queries' tokens are in the cache.  A
        cache's weights are left as they are: ``evict`` does not know of these
        queries."""
        bp = self._bounds_of(cache, bounds)
        cu, T = _cu_arg(self, cu_seqlens)
        n_select, n_first, n_recent = (_fits(name, int(x)) for name, x in (
            ("n_select", n_select), ("n_first", n_first), ("n_recent", n_recent)))
        max_len = _fits("max_len", int(max_len), 64)
        qp, _, _, op, lp = self._rows(cache, q, None, None, out, lse, max(T, 0))
        sp = _tensor("selected", selected, cache._dev, torch.int32, max(T, 0) * self.n_kv_heads * max(n_select, 0))
        ws, n = self._workspace(cache, workspace)
        self._call("glide_paged_sparse", cache, stream, bp, qp, cu.buffer_info()[0], T, n_select, n_first, n_recent, max_len, sp,
                   op, lp, ws, n)

    def evict(self, cache, budget, n_recent, kept, new_lens, workspace, dst_table=None, stream=None):
        """Keep min(len, budget) tokens per sequence and KV head, in place or
        in dst_table's pages.  kept [B][Hkv][budget] int32: their old
        positions; new_lens [B] int32 (may be the cache's lens).  A kept token
        whose page is not allocated becomes a row of zeros (see glide.h): keep
        the budget within the tokens that are."""
        if type(cache) is not PagedCache or cache.geometry is not self.geometry:
            self._check_cache(cache)
        if cache.weights is None:
            raise ValueError("evict needs a cache with weights")
        budget, n_recent = int(budget), int(n_recent)
        if budget >> 31 or n_recent >> 31:
            _fits("budget", budget)
            _fits("n_recent", n_recent)
        dev = cache._dev
        kp = _tensor("kept", kept, dev, torch.int32, self.batch * self.n_kv_heads * max(budget, 0))
        lp = _tensor("new_lens", new_lens, dev, torch.int32, self.batch)
        dp = None
        if dst_table is not None:
            dp = _tensor("dst_table", dst_table, dev, torch.int32, self.batch * self.max_pages)
            if tuple(dst_table.shape) != (self.batch, self.max_pages):
                raise ValueError(f"dst_table has shape {tuple(dst_table.shape)}, expected "
                                 f"{(self.batch, self.max_pages)}")
        ws, n = self._workspace(cache, workspace)
        self._call("glide_paged_evict", cache, stream, budget, n_recent, dp, kp, lp, ws, n)
