// Shared pieces of attention over packed sequences: the plan of a batch, tensor maps, workspace layout.
#pragma once

#include "attn_bwd.cuh"

namespace vardrop {

// A plan: a header, then an entry for every 128-token tile of every sequence, those with the most work first.  Entry `level` i of a sequence of n tiles stands for
// query tile i forward (i + 1 key tiles in causal calls) and key tile n - 1 - i backward (i + 1 query tiles), so that one order serves both.  Sequences of a single tile come
// last.
constexpr int kPlanMagic = 0x56445031;
constexpr int kFewTiles = 2;             // forward: tiles with no more key tiles than this are attn_packed_tile_kernel's
enum PlanWord { kPlanStatus = 0, kPlanMagicWord, kPlanTiles, kPlanSeqs, kPlanRows, kPlanCausal, kPlanMany /*entries ahead of those with few key tiles*/, kPlanLong /*entries of sequences of several tiles*/,
                kPlanMostWork /*of one of those, in tiles*/, kPlanWork /*of all of them, fp32*/ };
struct alignas(16) PlanEntry {
    int start;              // row of the sequence's first token
    int len;                // its tokens
    int level;
    int base;               // tiles of the sequences ahead of it: its first tile in layouts where every sequence begins a tile
};

// Tiles that a batch can have at most: a sequence's last one may hold a single token.
inline long long packed_tiles(const vardrop_packed_cfg& c) { return c.T / kTile + (c.n_seqs < c.T ? c.n_seqs : c.T); }

// Backward, an item (a key tile of a key head) whose query tiles take longer than half of what an SM has to do altogether is split into up to four, whose parts of dK and dV
// lie in the workspace until the conversion adds them up: largest items bound a call of few, and grouped heads make them large (12 windows of 1 to 1999 tokens, 8 query heads on 2
// key heads: 148 items, one of 64 steps where an SM's share is 24).  Calls of many tiles do without.
constexpr int kMostParts = 4, kSplitTiles = 1024, kLeastSteps = 8;
inline bool packed_may_split(const vardrop_packed_cfg& c) { return packed_tiles(c) * c.Hkv <= kSplitTiles; }

struct PackedWs {
    size_t delta;           // [Hq, tiles 128] fp32
    size_t dq_acc;          // [tiles 128, Hq, D] fp32
    size_t parts;           // [tiles 128, (dV, dK), part, Hkv, D] fp32
    size_t total;
    int rows;               // tiles 128
};
inline PackedWs packed_layout(const vardrop_packed_cfg& c) {
    PackedWs w;
    w.rows = static_cast<int>(packed_tiles(c) * kTile);
    size_t o = align_up(kWsHeaderBytes, 1024);
    w.delta = o; o += align_up(sizeof(float) * static_cast<size_t>(c.Hq) * w.rows, 1024);
    w.dq_acc = o; o += align_up(sizeof(float) * static_cast<size_t>(c.Hq) * c.D * w.rows, 1024);
    w.parts = o; o += packed_may_split(c) ? align_up(sizeof(float) * 2 * kMostParts * c.Hkv * c.D * static_cast<size_t>(w.rows), 1024) : 0;
    w.total = o;
    return w;
}

struct PackedStrides {
    long long sTq, sHq, sTkv, sHkv;
};
inline PackedStrides packed_strides(const vardrop_packed_cfg& c) {
    PackedStrides s{c.sTq, c.sHq, c.sTkv, c.sHkv};
    if (s.sTq == 0 && s.sHq == 0) { s.sHq = c.D; s.sTq = static_cast<long long>(c.Hq) * c.D; }
    if (s.sTkv == 0 && s.sHkv == 0) { s.sHkv = c.D; s.sTkv = static_cast<long long>(c.Hkv) * c.D; }
    return s;
}

// Tensor map over [T, H, D] bf16 with the given element strides: box = 128 tokens x 64 elements of a head, 128-byte swizzle; the upper half of a row of a tensor with
// D = 32, and rows behind the tensor, read as zero.
int packed_tile_map(CUtensorMap* map, const void* base, int D, int H, int T, long long sT, long long sH);
// Over the fp32 accumulator [rows, H, D]: box = 128 rows x 32 floats of a head.
int packed_acc_map(CUtensorMap* map, const void* base, int rows, int H, int D);

__device__ __forceinline__ void tma_load_3d(void* dst, const void* map, uint64_t* bar, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}
__device__ __forceinline__ void tma_reduce_add_3d(const void* map, const void* src, int c0, int c1, int c2) {
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}

// One warp's share of a tile of consecutive rows: 32 from tok0 on by 16-byte asynchronous copies, zeros from `len` on and in the upper half of a row of 32.
__device__ __forceinline__ void copy_32_tokens(unsigned char* rows, const __nv_bfloat16* from, long long sT, int tok0, int len, int D) {
    const int lane = threadIdx.x & 31, chunk = lane & 7, r = lane >> 3;
    const uint32_t live = chunk * 8 < D ? 16u : 0u;
    const __nv_bfloat16* const begin = from + (live ? chunk * 8 : 0);
    const __nv_bfloat16* src = begin + (tok0 + r) * sT;
    const uint32_t dst = smem_u32(rows) + r * kRowBytes + (static_cast<uint32_t>(chunk ^ r) << 4);
    const int left = len - tok0 - r;
#pragma unroll
    for (int it = 0; it < 8; ++it, src += 4 * sT) cp_async16((dst ^ ((it & 1) * 64u)) + it * 4 * kRowBytes, 4 * it < left ? src : begin, 4 * it < left ? live : 0u);
}

// Short sequences under grouped heads: the query rows of several heads of a group share a tile (they see the same keys), head after head.  Row r of such a tile.
struct PackedRow {
    int head, token;                     // from the tile's first head on
};
__device__ __forceinline__ PackedRow packed_row(int r, int len) {
    const int g = small_div(r, len);
    return PackedRow{g, r - g * len};
}
// Heads of a group that share a tile.
__device__ __forceinline__ int heads_a_tile(int len, int left) { return max(1, min(left, small_div(kTile, len))); }
// One warp's share of such a tile: 32 rows from r0 on, zeros from n_rows on.
__device__ __forceinline__ void copy_32_packed(unsigned char* rows, const __nv_bfloat16* from, long long sT, long long sH, int r0, int n_rows, int len, int D) {
    const int lane = threadIdx.x & 31, chunk = lane & 7, r = lane >> 3;
    const uint32_t live = chunk * 8 < D ? 16u : 0u;
    const __nv_bfloat16* const begin = from + (live ? chunk * 8 : 0);
    const uint32_t dst = smem_u32(rows) + r * kRowBytes + (static_cast<uint32_t>(chunk ^ r) << 4);
#pragma unroll
    for (int it = 0; it < 8; ++it) {
        const int at = r0 + r + 4 * it;
        const bool there = at < n_rows;
        const PackedRow p = packed_row(there ? at : 0, len);
        cp_async16((dst ^ ((it & 1) * 64u)) + it * 4 * kRowBytes, begin + p.token * sT + p.head * sH, there ? live : 0u);
    }
}

__device__ __forceinline__ void tma_store_3d(const void* map, const void* src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}

// What a kernel needs of the plan's header: the number of tiles, 0 where it is not a plan of this call's kind (which the caller reports).
struct PlanView {
    const int32_t* words;
    int n_seqs, T, causal;
    __device__ __forceinline__ const PlanEntry* entries() const { return reinterpret_cast<const PlanEntry*>(words + kWsHeaderBytes / 4); }
};
struct PlanHead {
    bool fits;                           // a plan of this call's kind
    int tiles, many, longer;             // 0 where it is not
};
__device__ __forceinline__ PlanHead plan_head(const PlanView& v) {
    const int4 a = *reinterpret_cast<const int4*>(v.words), b = *reinterpret_cast<const int4*>(v.words + 4);       // both at once
    static_assert(kPlanStatus == 0 && kPlanMagicWord == 1 && kPlanTiles == 2 && kPlanSeqs == 3 && kPlanRows == 4 && kPlanCausal == 5 && kPlanMany == 6 && kPlanLong == 7, "order of the header");
    const bool fits = a.x == VARDROP_OK && a.y == kPlanMagic && a.w == v.n_seqs && b.x == v.T && b.y == v.causal;
    return PlanHead{fits, fits ? a.z : 0, fits ? b.z : 0, fits ? b.w : 0};
}

// How the backward pass splits items: `parts` of an entry at most, one of `steps` query tiles (over all heads of a group) into ceil(steps / chunk).
struct Split {
    int parts, chunk;
};
__device__ __forceinline__ Split split_of(const PlanView& v, const PlanHead& head, int group, int Hkv, int sms, bool may) {
    if (head.longer == 0) return Split{1, 1};
    const int most = v.words[kPlanMostWork] * group;
    const float share = __int_as_float(v.words[kPlanWork]) * static_cast<float>(group * Hkv) / static_cast<float>(sms);
    int chunk = most;
    if (may) chunk = min(most, max(max(kLeastSteps, static_cast<int>(0.5f * share)), (most + kMostParts - 1) / kMostParts));
    return Split{(most + chunk - 1) / chunk, chunk};
}
__device__ __forceinline__ int parts_of(int steps, const Split& s) { return (steps + s.chunk - 1) / s.chunk; }

// Items beyond a CTA's first one are handed out by a counter in the workspace's header, which an earlier launch of the call has set to zero: they come with the most work first, so whoever
// is free takes the largest that is left.  (Turns there and back over the grid left SMs idle for 12 % of the forward and 14 % of the backward of two sequences of 8192 and 5001
// tokens, 16 query heads.)  An item is asked for when the loads of the one before have been issued, not earlier: one held ahead is one that somebody else could have begun.
constexpr int kWsTicketFwd = 8, kWsTicketBwd = 9;        // words of the header
__device__ __forceinline__ long long next_item(int* ticket, int ctas, int lane) {      // ctas: that have had a first one
    int t = 0;
    if (lane == 0) t = atomicAdd(ticket, 1);
    return static_cast<long long>(ctas) + __shfl_sync(0xffffffffu, t, 0);
}

}  // namespace vardrop
