"""Thin ctypes binding of the paged cache held in 4 bits (``glide_nibble_*`` in
include/glide.h): rows rotated and rounded on their way in, attention with a
sliding window and sinks over them, and their values read back.

Argument marshalling only, as in ``paged.py``: every step runs in the HIP
kernels behind the C ABI, and there is no fallback.
"""
import ctypes

import torch

from . import glide
from .paged import Paged, _append_rows, _cu_arg, _fits, _rotation, _tensor

GROUP = 32   # elements of a row that share a scale


class Paged4Cache:
    """The cache of one layer: its tensors, the struct that names them to the
    library, and the geometry that they were checked for.  Made by
    ``Paged4.cache``; every ``Paged4`` of the same geometry takes it."""

    def __init__(self, k_pool, v_pool, block_table, lens, arg, geometry):
        self.k_pool, self.v_pool = k_pool, v_pool
        self.block_table, self.lens = block_table, lens
        self.device = block_table.device
        self.geometry = geometry
        self._dev = block_table.get_device()
        self._arg = arg
        self._ref = ctypes.byref(arg)


class Paged4:
    """A configured layer over a paged cache in 4 bits: the arguments of
    ``paged.Paged``, dtype that of q, k, v and out.  A pool is a pair
    (codes [n_pages][n_kv_heads][page_size][head_dim / 2],
    scales [n_pages][n_kv_heads][page_size][head_dim / 32]) of uint8 tensors.
    """

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages, window=None, n_sinks=0,
                 dtype=torch.bfloat16, sm_scale=None, lib=None):
        g = Paged(batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages, window, n_sinks, dtype,
                  sm_scale, lib)
        self.lib, self.cfg, self._ref = g.lib, g.cfg, g._ref
        self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim = g.batch, g.n_q_heads, g.n_kv_heads, g.head_dim
        self.page_size, self.n_pages, self.max_pages = g.page_size, g.n_pages, g.max_pages
        self.window, self.n_sinks, self.sm_scale, self.torch_dtype = g.window, g.n_sinks, g.sm_scale, g.torch_dtype
        # what a cache's tensors are laid out by (the type of q, k and v is not)
        self.geometry = g.geometry[:-1]

    # -- buffers -------------------------------------------------------------
    def new_pools(self, device="cuda"):
        """K and V pools (codes, scales), not cleared: slots that no token was
        written to are never used."""
        shape = (self.n_pages, self.n_kv_heads, self.page_size)
        return tuple((torch.empty((*shape, self.head_dim // 2), dtype=torch.uint8, device=device),
                      torch.empty((*shape, self.head_dim // GROUP), dtype=torch.uint8, device=device))
                     for _ in range(2))

    def cache(self, k_pool, v_pool, block_table, lens):
        """The cache of one layer.  The tensors are used in place: a caller
        moves lens on and fills block_table between calls."""
        arg = glide.Paged4CacheArg()
        if not isinstance(block_table, torch.Tensor) or not block_table.is_cuda:
            raise ValueError("block_table must be a device tensor")
        dev = block_table.get_device()
        shape = (self.n_pages, self.n_kv_heads, self.page_size)
        for name, pool in (("k", k_pool), ("v", v_pool)):
            if not isinstance(pool, (tuple, list)) or len(pool) != 2:
                raise ValueError(f"{name}_pool must be a pair of codes and scales")
            for part, t, width in zip(("codes", "scales"), pool, (self.head_dim // 2, self.head_dim // GROUP)):
                at = _tensor(f"{name}_{part}", t, dev, torch.uint8, 0)
                if tuple(t.shape) != (*shape, width):
                    raise ValueError(f"{name}_{part} has shape {tuple(t.shape)}, expected {(*shape, width)}")
                setattr(arg, f"{name}_{part}", at)
        arg.block_table = _tensor("block_table", block_table, dev, torch.int32, self.batch * self.max_pages)
        arg.lens = _tensor("lens", lens, dev, torch.int32, self.batch)
        if tuple(block_table.shape) != (self.batch, self.max_pages):
            raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected "
                             f"{(self.batch, self.max_pages)}")
        return Paged4Cache(k_pool, v_pool, block_table, lens, arg, self.geometry)

    def workspace_bytes(self, max_total_tokens=0):
        return self.lib.glide_nibble_workspace_bytes(self._ref, _fits("max_total_tokens", int(max_total_tokens), 64))

    def new_workspace(self, max_total_tokens=0, device="cuda"):
        """Workspace for every call of up to max_total_tokens packed tokens."""
        n = self.workspace_bytes(max_total_tokens)
        if n == 0:
            raise glide.GlideError(-2, "glide_nibble_workspace_bytes", self.lib)
        return torch.empty(n, dtype=torch.uint8, device=device)

    # -- calls ---------------------------------------------------------------
    def _check_cache(self, cache):
        """Refuse a cache whose tensors another geometry was checked for."""
        if not isinstance(cache, Paged4Cache):
            raise ValueError("cache must come from Paged4.cache")
        if cache.geometry != self.geometry:
            names = ("batch", "n_kv_heads", "head_dim", "page_size", "n_pages", "max_pages")
            off = [f"{n} {x}, this layer has {y}" for n, x, y in zip(names, cache.geometry, self.geometry) if x != y]
            raise ValueError("cache was made for " + "; ".join(off))

    _call = Paged._call

    def append(self, cache, k, v, cu_seqlens, q=None, q_out=None, freqs=None, interleaved=False, positions=None,
               stream=None):
        """Round k (rotated) and v [T][Hkv][d] to 4 bits, into their pages, and
        rotate q [T][Hq][d] to q_out (which may be q).  Arguments as for
        ``Paged.append``."""
        if type(cache) is not Paged4Cache or cache.geometry is not self.geometry:
            self._check_cache(cache)
        cu, T = _cu_arg(self, cu_seqlens)
        rot = _rotation(freqs, interleaved, positions, cache._dev, T)
        qp, kp, vp, op = _append_rows(self, cache._dev, q, k, v, q_out, max(T, 0))
        self._call("glide_nibble_append", cache, stream, rot, qp, kp, vp, cu.buffer_info()[0], T, op)

    def read(self, cache, cu_seqlens, k_out, v_out, stream=None):
        """The values that the cache holds of the last cu[b + 1] - cu[b] tokens
        of every sequence b: k_out, v_out [T][Hkv][d], zeros where a token has
        no page."""
        if type(cache) is not Paged4Cache or cache.geometry is not self.geometry:
            self._check_cache(cache)
        cu, T = _cu_arg(self, cu_seqlens)
        n = max(T, 0) * self.n_kv_heads * self.head_dim
        kp = _tensor("k_out", k_out, cache._dev, self.torch_dtype, n)
        vp = _tensor("v_out", v_out, cache._dev, self.torch_dtype, n)
        self._call("glide_nibble_read", cache, stream, cu.buffer_info()[0], T, kp, vp)

    def _rows(self, cache, q, out, lse, T):
        """Pointers of a call over T rows of queries, checked."""
        if type(cache) is not Paged4Cache or cache.geometry is not self.geometry:
            self._check_cache(cache)
        dev, dt, nq = cache._dev, self.torch_dtype, T * self.n_q_heads * self.head_dim
        return (_tensor("q", q, dev, dt, nq), _tensor("out", out, dev, dt, nq),
                None if lse is None else _tensor("lse", lse, dev, torch.float32, T * self.n_q_heads))

    def prefill(self, cache, q, cu_seqlens, out, workspace, lse=None, max_len=0, stream=None):
        """Read out one row per query and head: q, out [T][Hq][d], lse [T][Hq]
        fp32, for the last cu[b + 1] - cu[b] cached tokens of every sequence b.
        max_len: a bound of lens on the host (0: none), which the work is split
        by."""
        cu, T = _cu_arg(self, cu_seqlens)
        max_len = _fits("max_len", int(max_len), 64)
        qp, op, lp = self._rows(cache, q, out, lse, max(T, 0))
        ws = _tensor("workspace", workspace, cache._dev, torch.uint8, 0)
        self._call("glide_nibble_prefill", cache, stream, qp, cu.buffer_info()[0], T, max_len, op, lp, ws, workspace.numel())

    def decode(self, cache, q, out, workspace, lse=None, max_len=0, stream=None):
        """One query per sequence, of its last cached token: q, out [B][Hq][d],
        lse [B][Hq] fp32."""
        max_len = _fits("max_len", int(max_len), 64)
        qp, op, lp = self._rows(cache, q, out, lse, self.batch)
        ws = _tensor("workspace", workspace, cache._dev, torch.uint8, 0)
        self._call("glide_nibble_decode", cache, stream, qp, max_len, op, lp, ws, workspace.numel())
