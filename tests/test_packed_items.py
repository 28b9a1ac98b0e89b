"""The rules by which the packed forward shares its tiles out, compiled for the host from the header that the kernels use."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("items")
    (d / "items.cpp").write_text('#include "packed_items.h"\nusing namespace vardrop;\n'
                                 'extern "C" int few(int tiles, int many, int Hq, int grid) { return few_begin({tiles, many}, Hq, grid); }\n'
                                 'extern "C" int parts(int tiles, int many, int Hq, int causal, int grid) { return in_parts({tiles, many}, Hq, causal, grid); }\n')
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{ROOT}/paper_2501_14183_b200/csrc", "-o", str(d / "items.so"), str(d / "items.cpp")])
    return C.CDLL(str(d / "items.so"))


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("grid", [1, 2, 37, 148, 160])
def test_tiles_in_parts_have_more_than_two_key_tiles(rules, causal, grid):
    """A tile of one head in two parts needs a key tile for each of them at least, so where items are parts the tiles with few key tiles are the other kernel's."""
    seen = set()
    for Hq in range(1, 41):
        for many in range(0, 400):
            tiles, parts = many + 5, rules.parts(many + 5, many, Hq, causal, grid)
            few = rules.few(tiles, many, Hq, grid)
            assert few in (many, tiles)
            assert not parts or few == many, (Hq, many)
            seen.add((parts, few == many))
    assert (0, False) in seen and (1, True) in seen
