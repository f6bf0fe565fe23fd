"""Which kernel a call is planned for, and host arithmetic of the kernels
evaluated by the compiler (a sum that overflows is no constant, and an assertion
on it does not compile)."""
import ctypes
import itertools
import subprocess

import pytest
import torch

from paper_2607_24788_amd import build, glide, paged, paged4


def compiles(tmp_path, text):
    src = tmp_path / "check.hip"
    src.write_text(text)
    flags = [f for f in build.FLAGS if not f.startswith("-O")]
    r = subprocess.run([build.HIPCC, *flags, "--cuda-host-only", "-fsyntax-only", str(src)], capture_output=True, text=True)
    return r.returncode == 0, r.stderr


@pytest.mark.parametrize("j0,shift,tmax,want", [
    (0, 5, 1000, None), (0, 6, 1000, 32), (32, 6, 1000, None), (96, 7, 127, None), (64, 7, 96, 96), (64, 7, 95, None),
    (992, 10, 5000, None), (0, 4, 1000, None), (16, 4, 1000, None), ((1 << 30) - 64, 6, (1 << 30) - 1, (1 << 30) - 32),
    (None, 6, 1000, None), (None, 10, (1 << 30) - 1, None)])
def test_tiles_of_a_page(tmp_path, j0, shift, tmax, want):
    """The tile behind one, and behind the last: nothing is added to the mark of no tile."""
    a, b = (("glide::kNoTile" if x is None else str(x)) for x in (j0, want))
    ok, err = compiles(tmp_path, f'#include "select.h"\nstatic_assert(glide::next_in_page({a}, {shift}, {tmax}) == {b}, "");\n')
    assert ok, err


BF16, FP32 = torch.bfloat16, torch.float32
WORKGROUPS, WAVES, TILES = range(3)


def sparse_form(g, new, n_select, max_len=0):
    """How a call of the layer g over `new` rows per sequence attends to them."""
    cu = (ctypes.c_int32 * (len(new) + 1))(0, *itertools.accumulate(new))
    f = g.lib.glide_internal_sparse_form
    f.restype, f.argtypes = ctypes.c_int32, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64]
    return f(ctypes.addressof(g.cfg), ctypes.addressof(cu), n_select, max_len)


@pytest.mark.parametrize("G,page", [(8, 128), (7, 64), (6, 32), (4, 64), (3, 32), (1, 64)])
def test_rows_share_waves_whatever_their_parity(G, page):
    """One row more or less than a multiple of a wave's, of one sequence or of
    many, does not send the call to a kernel that reads every page per row."""
    for new in ([2048], [2047], [2049], [120] * 20, [121] * 20, [119, 120, 121] * 7, [5] * 500):
        g = paged.Paged(len(new), 8 * G, 8, 128, page, 1000, 200, dtype=BF16)
        assert sparse_form(g, new, 12, 9000) == TILES, new


def test_who_attends_to_the_rows():
    def form(new, G=4, page=64, n_select=20, dtype=BF16, Hkv=8, max_len=8000):
        g = paged.Paged(len(new), Hkv * G, Hkv, 128, page, 1000, 500, dtype=dtype)
        return sparse_form(g, new, n_select, max_len)
    assert form([1]) == form([255]) == form([1] * 32) == form([300], Hkv=4) == WORKGROUPS
    assert form([256]) == form([1] * 128, Hkv=16) == WAVES   # few waves; nothing to share
    assert form([2048], dtype=FP32) == form([2048], page=8) == form([2048], G=16) == form([2048], G=9) == WAVES
    assert form([1, 2, 1] * 42, Hkv=16) == WAVES             # 1.33 rows to a wave
    assert form([5] * 60, G=8) == form([1, 3] * 64) == TILES  # 1.67, 2
    assert form([2048], page=16, n_select=20) == WAVES       # pages that fill half a tile: by how many rows select one
    assert form([2048], page=16, n_select=400) == TILES


def nibble_plan(g, new, max_len=0):
    """Of a 4-bit layer's prefill of `new` rows per sequence: rows of a
    workgroup, pieces; of its decode (None): keys of a wave's tile, pieces."""
    cu = None if new is None else (ctypes.c_int32 * (len(new) + 1))(0, *itertools.accumulate(new))
    n, f = ctypes.c_int32(), g.lib.glide_internal_nibble_plan
    f.restype, f.argtypes = ctypes.c_int32, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]
    return f(ctypes.addressof(g.cfg), None if cu is None else ctypes.addressof(cu), max_len, ctypes.addressof(n)), n.value


def test_tiles_of_a_decode():
    """Every kernel of a decode is one that some call is planned for."""
    def plan(units, keys, d, dtype=BF16):
        g = paged4.Paged4(units // 8, 32, 8, d, 64, 1000, 1024, dtype=dtype)
        return nibble_plan(g, None, keys)
    assert plan(8, 40000, 128)[0] == 64 and plan(8, 65536, 128)[0] == plan(64, 7000, 128)[0] == 32
    assert plan(256, 24000, 128) == (32, 6)
    assert plan(776, 300, 64) == plan(1024, 300, 64) == plan(4096, 512, 64) == (32, 1)
    assert plan(768, 300, 64) == plan(4096, 513, 64) == (64, 1) and plan(128, 20000, 64)[0] == 64
    for d in (64, 128):
        for units, keys in ((1024, 300), (2048, 4000), (256, 24000)):
            assert plan(units, keys, d, FP32)[0] == 64


def test_launches_of_kernels_that_are_not_there():
    """An error, not a success with nothing launched."""
    lib = glide.load_library()
    args, pools, seqs = ((ctypes.c_char * 4096)() for _ in range(3))
    ctypes.cast(seqs, ctypes.POINTER(ctypes.c_int32))[0] = 1                           # one sequence,
    ctypes.cast(seqs, ctypes.POINTER(ctypes.c_int32))[2 + 2 * 128 + 1] = 1             # one tile
    invalid = 1                                                                        # hipErrorInvalidValue
    decode = lib._ZN5glide20launch_nibble_decodeERKNS_9PagedArgsERKNS_6Pools4EiiiP12ihipStream_t
    prefill = lib._ZN5glide21launch_nibble_prefillERKNS_9PagedArgsERKNS_6Pools4ERKNS_9PagedSeqsEiiiP12ihipStream_t
    for dtype in (0, 1):
        for d in (64, 128):
            for keys in (0, 16, 48, 128) + ((32,) if dtype == glide.F32 else ()):
                assert decode(args, pools, d, dtype, keys, None) == invalid
            for rows in (0, 32, 64, 512):
                assert prefill(args, pools, seqs, d, dtype, rows, None) == invalid
