// Which tiles of the loss's products each pair of CTAs takes, in which order and in how many parts.  Plain C++, for the device and the host.
#pragma once

#ifdef __CUDACC__
#define VARDROP_TILES_FN __host__ __device__ __forceinline__
#else
#define VARDROP_TILES_FN inline
#endif

namespace vardrop {

constexpr int kPairTile = 256;                       // rows and columns of a tile
constexpr int kChunk = 64;                           // of the contracted axis in a stage
constexpr int kGroupRows = 8;                        // row tiles that neighbouring pairs share out among each other
constexpr int kMostSplits = 32, kSplitChunks = 8;    // parts of a tile's contracted axis; chunks that one has at least (2 us of products)
constexpr int kTileCost = 3;                         // what a tile takes beside its chunks, in chunks

VARDROP_TILES_FN int tiles_of(long long n, int each) { return static_cast<int>((n + each - 1) / each); }

// Too few tiles for the SMs, or a few long ones beside many short: parts of the contracted axis, added up in a fixed order afterwards.  A gradient's tiles are split into as many whole shares of a pair of
// CTAs as they are long.
struct SplitParams {
    int pairs, tn, piece, dh_rows, dw_parts, dh, dw;    // tiles of the channels; columns of G; rows that all parts of d_h may take; parts of d_w; whether wanted
};
struct Splits {
    int dh, dw;
};
VARDROP_TILES_FN Splits splits_of(const SplitParams& S, int n) {
    const int tm = tiles_of(n, kPairTile), tv = tiles_of(S.piece, kPairTile), ch = tiles_of(S.piece, kChunk), cw = tiles_of(n, kChunk);
    const long long work = static_cast<long long>(S.tn) * (static_cast<long long>(tm) * (ch + kTileCost) + static_cast<long long>(tv) * (cw + kTileCost));      // of both: one alone has the same bits
    const long long even = work / S.pairs;
    const int share = even < kSplitChunks ? kSplitChunks : even > (1 << 30) ? 1 << 30 : static_cast<int>(even);
    const auto within = [](int v, int most) { return v > most ? (most < 1 ? 1 : most) : v < 1 ? 1 : v; };
    Splits s;
    s.dh = tm == 0 ? 1 : within(within(ch / share, kMostSplits), S.dh_rows / (tm * kPairTile));
    s.dw = within(cw / share, S.dw_parts);
    return s;
}

// Whether there can be more than one part, whatever has a label: of d_h, of d_w.
VARDROP_TILES_FN bool may_split_dh(const SplitParams& S) { return S.piece / kChunk >= 2 * kSplitChunks; }
VARDROP_TILES_FN bool may_split_dw(const SplitParams& S, int T) { return S.dw_parts > 1 && tiles_of(T, kChunk) >= 2 * kSplitChunks; }

struct PairTile {
    int m, n, k0, k1, part;                             // tile; chunks of the contracted axis; which part of it that is
    bool dw;                                            // of d_w, not of d_h
};
// Tiles of rows x cols in groups of eight rows of tiles: what neighbouring pairs read at a time is some eight tiles of A and nine of B.
// (32 bits throughout: there are fewer than 2^31 tiles and parts of them, and every role of a CTA divides for every tile.)
VARDROP_TILES_FN void place_tile(PairTile& x, unsigned in, unsigned rows, unsigned cols) {
    const unsigned width = kGroupRows * cols, group = in / width, r = in - group * width, left = rows - group * kGroupRows;
    unsigned n, m;
    if (left >= kGroupRows) {
        n = r / kGroupRows;
        m = r - n * kGroupRows;
    } else {
        n = r / left;
        m = r - n * left;
    }
    x.n = static_cast<int>(n);
    x.m = static_cast<int>(group * kGroupRows + m);
}
// Products of n tokens with `columns` rows of w, `deep` chunks each: by turns.
struct LogitTiles {
    int tm, tv, deep, pair, pairs;
    VARDROP_TILES_FN bool at(int i, PairTile& x) const {
        const unsigned t = static_cast<unsigned>(pair) + static_cast<unsigned>(i) * static_cast<unsigned>(pairs);
        if (t >= static_cast<unsigned>(tm) * static_cast<unsigned>(tv)) return false;
        place_tile(x, t, static_cast<unsigned>(tm), static_cast<unsigned>(tv));
        x.k0 = 0;
        x.k1 = deep;
        x.part = 0;
        x.dw = false;
        return true;
    }
};
// Both gradients' products: the one with the longer tiles first, by turns; the pairs that get one less of them begin the others with as many as that one takes.
struct GradTiles {
    int tm, tv, tc, ch, cw, pair, pairs;                // row tiles of d_h and of d_w, tiles of the channels, chunks of d_h's and d_w's contracted axes
    Splits splits;
    unsigned all_1, all_2;
    int mine, ahead, late, odd, extra;
    bool w_first;
    VARDROP_TILES_FN GradTiles(const SplitParams& S, int n, int columns, int pair_, int pairs_) {
        tm = tiles_of(n, kPairTile); tv = tiles_of(columns, kPairTile); tc = S.tn; ch = tiles_of(columns, kChunk); cw = tiles_of(n, kChunk);
        pair = pair_; pairs = pairs_;
        splits = splits_of(S, n);
        const unsigned all_h = S.dh ? static_cast<unsigned>(tm) * tc * splits.dh : 0u, all_w = S.dw ? static_cast<unsigned>(tv) * tc * splits.dw : 0u;
        const int len_h = ch / splits.dh + kTileCost, len_w = cw / splits.dw + kTileCost;
        w_first = len_w > len_h;
        all_1 = w_first ? all_w : all_h;
        all_2 = w_first ? all_h : all_w;
        const int longer = w_first ? len_w : len_h, shorter = w_first ? len_h : len_w, turns = static_cast<int>(all_1 / static_cast<unsigned>(pairs));
        odd = static_cast<int>(all_1 - static_cast<unsigned>(turns) * static_cast<unsigned>(pairs));
        late = odd == 0 ? 0 : pairs - odd;
        extra = odd == 0 ? 0 : (longer + shorter / 2) / shorter;
        mine = turns + (pair < odd ? 1 : 0);
        ahead = pair < odd ? 0 : extra;
    }
    VARDROP_TILES_FN bool at(int i, PairTile& x) const {
        unsigned t;
        if (i < mine) {
            t = static_cast<unsigned>(pair) + static_cast<unsigned>(i) * static_cast<unsigned>(pairs);
            x.dw = w_first;
        } else {
            const unsigned j = static_cast<unsigned>(i - mine), first = static_cast<unsigned>(ahead);
            t = j < first ? j * static_cast<unsigned>(late) + static_cast<unsigned>(pair - odd)
                          : static_cast<unsigned>(extra) * static_cast<unsigned>(late) + (j - first) * static_cast<unsigned>(pairs) + static_cast<unsigned>(pair);
            if (t >= all_2) return false;
            x.dw = !w_first;
        }
        const unsigned rows = static_cast<unsigned>(x.dw ? tv : tm), each = rows * static_cast<unsigned>(tc), parts = static_cast<unsigned>(x.dw ? splits.dw : splits.dh);
        const unsigned chunks = static_cast<unsigned>(x.dw ? cw : ch), part = parts == 1 ? 0 : t / each;
        x.part = static_cast<int>(part);
        place_tile(x, t - part * each, rows, static_cast<unsigned>(tc));
        x.k0 = parts == 1 ? 0 : static_cast<int>(chunks * part / parts);
        x.k1 = static_cast<int>(parts == 1 ? chunks : chunks * (part + 1) / parts);
        return true;
    }
};

}  // namespace vardrop
