"""Host arithmetic of the kernels' planning, evaluated by the compiler: a sum
that overflows is no constant, and an assertion on it does not compile."""
import subprocess

import pytest

from paper_2607_24788_amd import build


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
