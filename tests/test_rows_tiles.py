"""Which rows a workgroup of the attention of chunks works on, from offsets as the device would find them: the kernels' own function, run on the CPU."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("native") / "rows_tiles")
    subprocess.run(["g++", "-O1", "-std=c++17", os.path.join(HERE, "native", "rows_tiles.cpp"), "-o", out], check=True)
    return out


@pytest.mark.parametrize("tables", ["sorted", "any"])
def test_tiles_lie_in_their_rows(program, tables):
    """Sorted offsets: every column is in one tile.  Any offsets: no tile names a row that is not its sequence's."""
    p = subprocess.run([program, tables], stdout=subprocess.PIPE, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout == "ok\n", "%d %s" % (p.returncode, p.stdout[-3000:])
