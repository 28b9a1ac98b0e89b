// Which tiles each of the packed forward's kernels takes, and in which form.  Plain C++, for the device and the host.
#pragma once

#ifdef __CUDACC__
#define VARDROP_ITEMS_FN __host__ __device__ __forceinline__
#else
#define VARDROP_ITEMS_FN inline
#endif

namespace vardrop {

// Of a plan: its tiles, and those with more key tiles than kFewTiles, which come first.
struct FwdTiles {
    int tiles, many;
};
// Whether items of two neighbouring heads, of the tiles with many key tiles alone, come to one for every SM.
VARDROP_ITEMS_FN bool fills(const FwdTiles& t, int Hq, int grid) { return t.many * ((Hq + 1) >> 1) >= grid; }

// First of the tiles that attn_packed_tile_kernel takes: those with few key tiles, unless the others fill the SMs: then they are the fine ends of its work, and that kernel would stand in
// front of it (16 prompts of 1 to 1999 tokens, 16 heads: 68.2 us with, 64.1 without; 36 sequences of 200 and 1413, not causal: 65.5 and 55.7; eight of nine such batches 1.5 to 18 % faster without,
// 48 sequences of 64 to 605 with 24 heads of 32 3 % slower).
VARDROP_ITEMS_FN int few_begin(const FwdTiles& t, int Hq, int grid) { return fills(t, Hq, grid) ? t.tiles : t.many; }

// Whether items are the key parts of single heads: where items of two heads would leave SMs idle; without a causal mask, whose rows of tiles are alike, where those parts all find an SM.
// (8192 tokens, 2 heads: 122 -> 67 us; 4 causal sequences of 2048, 4 heads, 112 items: 40 -> 30.  16 of 1100, 2 heads, not causal, 144 items that find an SM each: 31 -> 33 as 288 parts.)
// Never where the tiles with few key tiles are among the items: a part needs a key tile of its own.
VARDROP_ITEMS_FN bool in_parts(const FwdTiles& t, int Hq, int causal, int grid) { return !fills(t, Hq, grid) && (causal || t.many * Hq <= grid); }

}  // namespace vardrop
