"""The rules by which the loss shares its tiles out, compiled for the host from the header that the kernels use."""
import ctypes as C
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <vector>
#include "loss_tiles.h"
using namespace vardrop;
// 0: every chunk of every tile of either gradient is taken once and the parts fit; otherwise what is wrong.  out: longest pair's chunks, all chunks over the pairs
extern "C" int gradients(int n, int columns, int piece, int C, int pairs, int grid, int dh_rows, int dw_parts, int dh, int dw, long long* out) {
    const SplitParams S{pairs, tiles_of(C, 256), piece, dh_rows, dw_parts, dh, dw};
    const Splits s = splits_of(S, n);
    const int tm = tiles_of(n, 256), tv = tiles_of(columns, 256), tc = S.tn, ch = tiles_of(columns, 64), cw = tiles_of(n, 64);
    if (s.dh < 1 || s.dw < 1 || s.dh > kMostSplits || s.dw > dw_parts) return 1;
    if (tm > 0 && static_cast<long long>(s.dh) * tm * 256 > dh_rows) return 2;
    if ((s.dh > 1 && !may_split_dh(S)) || (s.dw > 1 && !may_split_dw(S, n))) return 10;      // (n tokens at least)
    std::vector<int> seen_h(static_cast<size_t>(tm) * tc * s.dh), seen_w(static_cast<size_t>(tv) * tc * s.dw), chunks_h(static_cast<size_t>(tm) * tc), chunks_w(static_cast<size_t>(tv) * tc);
    long long longest = 0, sum = 0;
    for (int pair = 0; pair < grid; ++pair) {
        const GradTiles tiles(S, n, columns, pair, grid);
        PairTile x;
        long long mine = 0;
        int i = 0;
        for (; tiles.at(i, x); ++i) {
            if (x.m < 0 || x.m >= (x.dw ? tv : tm) || x.n < 0 || x.n >= tc || x.part < 0 || x.part >= (x.dw ? s.dw : s.dh) || x.k0 > x.k1) return 3;
            std::vector<int>& seen = x.dw ? seen_w : seen_h;
            if (seen[(static_cast<size_t>(x.part) * (x.dw ? tv : tm) + x.m) * tc + x.n]++) return 4;
            (x.dw ? chunks_w : chunks_h)[static_cast<size_t>(x.m) * tc + x.n] += x.k1 - x.k0;
            mine += x.k1 - x.k0 + kTileCost;
        }
        if (tiles.at(i, x) || tiles.at(i + 1, x)) return 5;      // a pair that has come to its end stays there
        longest = mine > longest ? mine : longest;
        sum += mine;
    }
    for (int v : seen_h) if (v != dh) return 6;
    for (int v : seen_w) if (v != dw) return 7;
    for (int v : chunks_h) if (v != dh * ch) return 8;
    for (int v : chunks_w) if (v != dw * cw) return 9;
    out[0] = longest;
    out[1] = sum / grid;
    return 0;
}
extern "C" int logits(int n, int columns, int grid) {
    const int tm = tiles_of(n, 256), tv = tiles_of(columns, 256);
    std::vector<int> seen(static_cast<size_t>(tm) * tv);
    for (int pair = 0; pair < grid; ++pair) {
        const LogitTiles tiles{tm, tv, 5, pair, grid};
        PairTile x;
        for (int i = 0; tiles.at(i, x); ++i) {
            if (x.m < 0 || x.m >= tm || x.n < 0 || x.n >= tv || x.dw) return 1;
            if (seen[static_cast<size_t>(x.m) * tv + x.n]++) return 2;
        }
    }
    for (int v : seen) if (v != 1) return 3;
    return 0;
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("tiles")
    (d / "tiles.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{ROOT}/paper_2501_14183_b200/csrc", "-o", str(d / "tiles.so"), str(d / "tiles.cpp")])
    return C.CDLL(str(d / "tiles.so"))


def test_every_tile_of_the_logits_is_taken_once(rules):
    rng = random.Random(1)
    for _ in range(300):
        n, columns = rng.choice([0, 1, 255, 256, 257, rng.randint(1, 20000)]), rng.randint(1, 60000)
        assert rules.logits(n, columns, rng.choice([1, 2, 3, 37, 74, 80])) == 0, (n, columns)


def test_every_chunk_of_the_gradients_is_taken_once(rules):
    rng = random.Random(2)
    out = (C.c_longlong * 2)()
    for _ in range(1500):
        n = rng.choice([0, 1, 63, 64, 256, 257, rng.randint(1, 9000), rng.randint(1, 300)])
        piece = 256 * rng.choice([1, 2, 3, rng.randint(1, 128)])
        columns = rng.choice([piece, rng.randint(1, piece)])
        channels, grid = rng.choice([8, 256, 264, 2048, 4096]), rng.choice([1, 2, 37, 73, 74])
        rows = max(256, -(-n // 256) * 256)
        dh_rows, dw_parts = rows * rng.choice([1, 1, 2, 32]) + rng.choice([0, 256]), rng.choice([1, 1, 2, 7, 32])
        dh, dw = rng.choice([(1, 1), (1, 1), (1, 0), (0, 1)])
        case = (n, columns, piece, channels, 74, grid, dh_rows, dw_parts, dh, dw)
        assert rules.gradients(*case, out) == 0, case


@pytest.mark.parametrize("n,piece,channels", [(8192, 16384, 2048), (3800, 4096, 512), (2011, 25088, 1024), (32, 131072, 2048), (65536, 1024, 512), (16384, 8192, 4096)])
def test_pairs_come_to_an_end_together(rules, n, piece, channels):
    """With parts allowed, no pair has more than half as much again as an even share (tiles of 256 x 256 are as fine as it gets)."""
    out = (C.c_longlong * 2)()
    assert rules.gradients(n, piece, piece, channels, 74, 74, 32 * max(256, -(-n // 256) * 256), 32, 1, 1, out) == 0
    assert out[0] <= 1.5 * out[1] + 8, tuple(out)
