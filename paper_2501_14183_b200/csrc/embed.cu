// Token embeddings: out[t] = scale table[idx[t]], and the table's gradient, d_table[v] (+)= scale sum of d_out[t] over the tokens with idx[t] = v.
//
// embed_fwd_kernel      rows of the table, several tokens to a thread so that their loads overlap.  Bound: memory.
// embed_count_kernel, embed_sort_kernel   tokens sorted by index, equal ones in their own order: a radix sort of (index, token) by digits of up to nine bits, so that up to 511 rows take one pass and up to
//                       2^18 - 1 two: indices that name no row are sorted behind the last one, as one row more.  embed_place_kernel: up to 4096 tokens, by comparing all pairs (8192 take 14 us, two passes 13).
//                       Beside the sorting, whose CTAs are few and whose steps are a chain of latencies, other CTAs of the same launches write zeros to the whole table.
// embed_sum_kernel      even shares of the sorted tokens: whoever meets all tokens of a row writes it, pieces of a row go to the workspace.
// embed_join_kernel     adds up the pieces, in order.
// embed_scan_kernel     few tokens and rows: a CTA a row looks through all indices for itself, one launch instead of four.
//
// The order of every sum is that of the tokens and does not depend on which CTA runs when: results are bit-reproducible.  Bound: memory, and for few tokens the chain of launches.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "vec_io.cuh"

namespace vardrop {

namespace {

constexpr int kEmbedThreads = 256;
// Tokens that a CTA ranks at a time: small tiles, whose ranks are a shorter chain of steps over more CTAs.
constexpr int kSortItems = 4, kSortThreads = 256, kSortTile = kSortThreads * kSortItems;
constexpr int kMaxDigitBits = 9, kMaxBins = 1 << kMaxDigitBits;
constexpr int kMaxSortBlocks = 256;             // beyond, a CTA takes several tiles: the offsets of a digit are summed over all CTAs by each of them
constexpr int kSumBatch = 8;                    // rows that a thread of the sums has on their way
constexpr int kJoinBatch = 8;                   // pieces
constexpr int kSumTokens = 16 * kEmbedThreads;  // that a CTA of the sums holds in shared memory
constexpr int kLeastShare = 8, kMostShare = 128;  // sorted tokens of a share: fewer make more pieces, more leave long chains of loads

struct SortPlan {
    int bits, passes, tiles_per_block, blocks;
};
SortPlan sort_plan(const vardrop_embed_cfg& c) {
    SortPlan p{};
    int bits = 1;
    while ((c.V >> bits) != 0) ++bits;          // of the keys 0 .. V
    p.passes = (bits + kMaxDigitBits - 1) / kMaxDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    const int tiles = (c.T + kSortTile - 1) / kSortTile;
    p.tiles_per_block = (tiles + kMaxSortBlocks - 1) / kMaxSortBlocks;
    p.blocks = (tiles + p.tiles_per_block - 1) / p.tiles_per_block;
    return p;
}

// Columns of a thread: kReps accesses of kVec.  Eight next to each other where rows are vectors of eight; narrower vectors of long rows in as many accesses as make eight, a row of threads apart, so that as many
// bytes are on their way (65536 tokens of 1023 bf16 columns, backward: 121 us with one access, 95 with eight); short rows, and the lookup, which has several tokens on their way, one.
struct Cols {
    int c0, step, C;                            // first column, distance of the accesses, columns there are
};
template <int kVec, int kReps>
__device__ __forceinline__ Cols cols_of(int slab, int lanes, int lane, int C) { return Cols{slab * lanes * kVec * kReps + lane * kVec, lanes * kVec, C}; }
template <class T, int kVec, int kReps>
struct Cells {
    Pack<T, kVec> v[kReps];
    __device__ __forceinline__ float at(int e) const { return to_float(v[e / kVec].e[e % kVec]); }
    __device__ __forceinline__ void set(int e, float x) { v[e / kVec].e[e % kVec] = from_float<T>(x); }
    // without a branch: column 0 where there is none
    __device__ __forceinline__ void load(const T* row, const Cols& k) {
#pragma unroll
        for (int r = 0; r < kReps; ++r) {
            const int c = k.c0 + r * k.step;
            v[r] = load_pack<T, kVec>(row + (c < k.C ? c : 0));
        }
    }
    __device__ __forceinline__ void store(T* row, const Cols& k) const {
#pragma unroll
        for (int r = 0; r < kReps; ++r) {
            const int c = k.c0 + r * k.step;
            if (c < k.C) store_pack(row + c, v[r]);
        }
    }
};
constexpr int kLongRow = 256;
inline int accesses_of(int C) { return C < kLongRow ? 1 : 8 / row_vector(C); }
inline int lanes_of(int C, int per) {
    int lanes = 1;
    while (lanes * per < C && lanes < kEmbedThreads) lanes *= 2;
    return lanes;
}
template <class F>
cudaError_t with_cells(int vec, int reps, F f) {
    if (vec == 8) return f(VecSize<8>{}, VecSize<1>{});
    if (reps == 1) return vec == 4 ? f(VecSize<4>{}, VecSize<1>{}) : vec == 2 ? f(VecSize<2>{}, VecSize<1>{}) : f(VecSize<1>{}, VecSize<1>{});
    return vec == 4 ? f(VecSize<4>{}, VecSize<2>{}) : vec == 2 ? f(VecSize<2>{}, VecSize<4>{}) : f(VecSize<1>{}, VecSize<8>{});
}

// Threads of a row, and sorted tokens of a share: some 1024 threads for every SM, where there are tokens enough.
struct SumPlan {
    int vec, reps, lanes, slabs, share, shares;
};
SumPlan sum_plan(const vardrop_embed_cfg& c) {
    SumPlan p{};
    p.vec = row_vector(c.C);
    p.reps = accesses_of(c.C);
    const int per = p.vec * p.reps;
    p.lanes = lanes_of(c.C, per);
    p.slabs = (c.C + per * p.lanes - 1) / (per * p.lanes);
    const long long wanted = 148ll * 1024 / (static_cast<long long>(p.lanes) * p.slabs);      // (a constant, so that sums do not depend on the device)
    const long long share = (c.T + std::max(wanted, 1ll) - 1) / std::max(wanted, 1ll);
    p.share = static_cast<int>(std::min<long long>(std::max<long long>(share, kLeastShare), std::min(kMostShare, kSumTokens / (kEmbedThreads / p.lanes))));
    p.shares = (c.T + p.share - 1) / p.share;
    return p;
}

struct EmbedWs {
    size_t counts, keys[2], tokens[2], pieces, total;
};
EmbedWs embed_layout(const vardrop_embed_cfg& c) {
    const SortPlan s = sort_plan(c);
    const SumPlan u = sum_plan(c);
    EmbedWs w;
    size_t o = align_up(kWsHeaderBytes, 1024);
    w.counts = o; o += align_up(sizeof(int32_t) * s.passes * s.blocks * kMaxBins, 1024);
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = o; o += align_up(sizeof(int32_t) * static_cast<size_t>(c.T), 1024);
        w.tokens[i] = o; o += align_up(sizeof(int32_t) * static_cast<size_t>(c.T), 1024);
    }
    w.pieces = o; o += align_up(sizeof(float) * 2 * u.shares * static_cast<size_t>(c.C), 1024);
    w.total = o;
    return w;
}

// ---- forward ------------------------------------------------------------------------------------------------------------------
struct EmbedParams {
    const void* table;
    const int32_t* idx;
    void* out;
    int* status;
    int T, V, C, lanes;
    float scale;
};
// A row takes `lanes` threads, a CTA kTokens rows for each group of them.
template <class Tab, class Out, int kVec, int kTokens>
__global__ void __launch_bounds__(kEmbedThreads) embed_fwd_kernel(const EmbedParams P) {
    chain_wait();
    chain_release();
    const int groups = kEmbedThreads / P.lanes, group = threadIdx.x / P.lanes, lane = threadIdx.x & (P.lanes - 1);
    const long long t0 = static_cast<long long>(blockIdx.x) * groups * kTokens + group;
    const Tab* const table = static_cast<const Tab*>(P.table);
    Out* const out = static_cast<Out*>(P.out);
    int row[kTokens];
#pragma unroll
    for (int u = 0; u < kTokens; ++u) {
        const long long t = t0 + u * groups;
        row[u] = t < P.T ? __ldg(P.idx + t) : -1;
        if (row[u] >= P.V) {
            if (lane == 0) set_status(P.status, VARDROP_ERR_INVALID_ARG);
            row[u] = -1;
        }
    }
#pragma unroll 1
    for (int c = lane * kVec; c < P.C; c += P.lanes * kVec) {
        Pack<Tab, kVec> in[kTokens];
        // (without a condition, here and in the sums: a load behind a branch is waited for where the branches join, which made a batch of them a chain)
#pragma unroll
        for (int u = 0; u < kTokens; ++u) in[u] = load_pack<Tab, kVec>(table + static_cast<size_t>(max(row[u], 0)) * P.C + c);
#pragma unroll
        for (int u = 0; u < kTokens; ++u) {
            const long long t = t0 + u * groups;
            if (t >= P.T) break;
            Pack<Out, kVec> v;
#pragma unroll
            for (int e = 0; e < kVec; ++e) v.e[e] = from_float<Out>(row[u] >= 0 ? to_float(in[u].e[e]) * P.scale : 0.f);
            store_pack(out + static_cast<size_t>(t) * P.C + c, v);
        }
    }
}

// ---- tokens by index ------------------------------------------------------------------------------------------------------------
struct SortParams {
    const int32_t *idx, *keys, *tokens;         // idx: the first pass
    int32_t *keys_out, *tokens_out, *counts;    // counts [passes, blocks, bins]
    int* status;
    int T, V, bits, pass, passes, blocks, tiles_per_block;
    uint4* zeros;                               // of the table, in 16-byte words: this launch's share, by the CTAs from `workers` on
    size_t zero_words;
    int workers;
    unsigned char* tail;                        // its last bytes, where they are no whole word
    int tail_bytes;
};
// The CTA's part of the launch's zeros.
__device__ __forceinline__ void write_zeros(const SortParams& P) {
    if (static_cast<int>(blockIdx.x) == P.workers && static_cast<int>(threadIdx.x) < P.tail_bytes) P.tail[threadIdx.x] = 0;
    const size_t step = static_cast<size_t>(gridDim.x - P.workers) * blockDim.x;
#pragma unroll 4
    for (size_t i = static_cast<size_t>(blockIdx.x - P.workers) * blockDim.x + threadIdx.x; i < P.zero_words; i += step) P.zeros[i] = make_uint4(0u, 0u, 0u, 0u);
}
// The key of an index: V where it names no row.
__device__ __forceinline__ int key_of(int v, int V) { return v < 0 || v >= V ? V : v; }
// Keys of kCount vectors of four tokens, the numbers first, first + step, ..; kNoToken behind the last token.  `bad`: an index from V on among them.  (No branch stands between the loads, which
// would make a chain of them: 500 tokens of eight columns took 9.9 us instead of 9.4, 4096 19.1 instead of 18.4.)
constexpr int kNoToken = 0x7fffffff;
template <int kCount>
__device__ __forceinline__ void keys_of(const int32_t* idx, int first, int step, int T, int V, int4 (&k)[kCount], bool& bad) {
    const int full = T >> 2, rest = T & 3, last = T - 1;
    const int4 none = make_int4(kNoToken, kNoToken, kNoToken, kNoToken);
    if (full > 0) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) k[i] = __ldg(reinterpret_cast<const int4*>(idx) + min(first + i * step, full - 1));
    }
    int4 tail = make_int4(__ldg(idx + min(4 * full, last)), __ldg(idx + min(4 * full + 1, last)), __ldg(idx + min(4 * full + 2, last)), 0);
    bad |= (rest > 0 && tail.x >= V) || (rest > 1 && tail.y >= V) || (rest > 2 && tail.z >= V);
    tail = make_int4(rest > 0 ? key_of(tail.x, V) : kNoToken, rest > 1 ? key_of(tail.y, V) : kNoToken, rest > 2 ? key_of(tail.z, V) : kNoToken, kNoToken);
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
        const int q = first + i * step;
        if (q >= full) {
            k[i] = q == full ? tail : none;
        } else {
            bad |= k[i].x >= V || k[i].y >= V || k[i].z >= V || k[i].w >= V;
            k[i] = make_int4(key_of(k[i].x, V), key_of(k[i].y, V), key_of(k[i].z, V), key_of(k[i].w, V));
        }
    }
}

__global__ void __launch_bounds__(kSortThreads) embed_count_kernel(const SortParams P) {
    __shared__ int hist[kMaxBins];
    const int bins = 1 << P.bits;
    for (int d = threadIdx.x; d < bins; d += kSortThreads) hist[d] = 0;
    chain_wait();
    chain_release();
    if (static_cast<int>(blockIdx.x) >= P.workers) {
        write_zeros(P);
        return;
    }
    __syncthreads();
    const long long begin = static_cast<long long>(blockIdx.x) * P.tiles_per_block * kSortTile, end = min(static_cast<long long>(P.T), begin + static_cast<long long>(P.tiles_per_block) * kSortTile);
    bool bad = false;
#pragma unroll 1
    for (long long t = begin + 4 * threadIdx.x; t < end; t += 4 * kSortThreads) {
        int4 k[1];
        keys_of(P.idx, static_cast<int>(t >> 2), 1, P.T, P.V, k, bad);
        if (k[0].x != kNoToken) atomicAdd(hist + (k[0].x & (bins - 1)), 1);
        if (k[0].y != kNoToken) atomicAdd(hist + (k[0].y & (bins - 1)), 1);
        if (k[0].z != kNoToken) atomicAdd(hist + (k[0].z & (bins - 1)), 1);
        if (k[0].w != kNoToken) atomicAdd(hist + (k[0].w & (bins - 1)), 1);
    }
    if (bad) set_status(P.status, VARDROP_ERR_INVALID_ARG);
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += kSortThreads) {
        P.counts[static_cast<size_t>(blockIdx.x) * kMaxBins + d] = hist[d];
        for (int p = 1; p < P.passes; ++p) P.counts[(static_cast<size_t>(p) * P.blocks + blockIdx.x) * kMaxBins + d] = 0;
    }
}

template <int kThreads>
struct SortShared {
    uint16_t count[kThreads / 32][kMaxBins];    // of a digit in a warp's tokens, then in those of the warps ahead
    int base[kMaxBins];                         // place of the digit's next token
    int total[kMaxBins];
    int part[32];
};
// Places of a tile's tokens: warp w has the tokens from 128 w on, 32 at a time.  Leaves the tile's tokens of each digit in `total`.
template <int kThreads>
__device__ __forceinline__ void rank_tile(SortShared<kThreads>& S, int bins, const int (&digit)[kSortItems], const bool (&there)[kSortItems], int (&place)[kSortItems]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int d = lane; d < bins / 2; d += 32) reinterpret_cast<uint32_t*>(S.count[warp])[d] = 0;
    __syncwarp();
    int rank[kSortItems];
    uint32_t peers[kSortItems];
    // Lanes of the same digit, by a vote a bit: __match_any_sync takes 7500 cycles for the 128 of them in a CTA of 32 warps, these 1000.
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) peers[i] = __ballot_sync(0xffffffffu, there[i]);
#pragma unroll
    for (int b = 1; b < kMaxBins; b *= 2) {
        if (b >= bins) break;
#pragma unroll
        for (int i = 0; i < kSortItems; ++i) {
            const uint32_t set = __ballot_sync(0xffffffffu, digit[i] & b);
            peers[i] &= digit[i] & b ? set : ~set;
        }
    }
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
        if (there[i]) rank[i] = S.count[warp][digit[i]] + __popc(peers[i] & ((1u << lane) - 1));
        __syncwarp();
        if (there[i] && (peers[i] >> lane) == 1u) S.count[warp][digit[i]] += static_cast<uint16_t>(__popc(peers[i]));      // the last of them
        __syncwarp();
    }
    __syncthreads();
#pragma unroll
    for (int d = threadIdx.x; d < bins; d += kThreads) {
        int total = 0, n[kThreads / 32];
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) n[w] = S.count[w][d];
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            S.count[w][d] = static_cast<uint16_t>(total);
            total += n[w];
        }
        S.total[d] = total;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) place[i] = there[i] ? S.count[warp][digit[i]] + rank[i] : 0;
}
// base[d] = (tokens of smaller digits) + base[d], from the totals of the digits: a thread has those from kEach of its number on.
template <int kThreads>
__device__ __forceinline__ void digit_bases(SortShared<kThreads>& S, int bins, const int* totals) {
    constexpr int kEach = kMaxBins > kThreads ? kMaxBins / kThreads : 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d0 = threadIdx.x * kEach;
    int own[kEach], sum = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        own[e] = d0 + e < bins ? totals[d0 + e] : 0;
        sum += own[e];
    }
    int up = sum;
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
        const int n = __shfl_up_sync(0xffffffffu, up, s);
        if (lane >= s) up += n;
    }
    if (lane == 31) S.part[warp] = up;
    __syncthreads();
    int before = up - sum;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w)
        if (w < warp) before += S.part[w];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (d0 + e < bins) S.base[d0 + e] += before;
        before += own[e];
    }
    __syncthreads();
}

__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const SortParams P) {
    __shared__ SortShared<kSortThreads> S;
    chain_wait();
    chain_release();
    if (static_cast<int>(blockIdx.x) >= P.workers) {
        write_zeros(P);
        return;
    }
    const int bins = 1 << P.bits, shift = P.pass * P.bits, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int32_t* const counts = P.counts + static_cast<size_t>(P.pass) * P.blocks * kMaxBins;
    // the digit's tokens in all CTAs and in those ahead of this one
    for (int d = tid; d < bins; d += kSortThreads) {
        int all = 0, ahead = 0;
#pragma unroll 16
        for (int b = 0; b < P.blocks; ++b) {
            const int n = __ldcg(counts + static_cast<size_t>(b) * kMaxBins + d);
            all += n;
            if (b < static_cast<int>(blockIdx.x)) ahead += n;
        }
        S.total[d] = all;
        S.base[d] = ahead;
    }
    __syncthreads();
    digit_bases(S, bins, S.total);
    const bool last = P.pass + 1 == P.passes;
    int32_t* const next = P.counts + static_cast<size_t>(P.pass + 1) * P.blocks * kMaxBins;
#pragma unroll 1
    for (int tile = 0; tile < P.tiles_per_block; ++tile) {
        const long long t0 = (static_cast<long long>(blockIdx.x) * P.tiles_per_block + tile) * kSortTile + warp * (32 * kSortItems) + lane;
        int key[kSortItems], token[kSortItems], digit[kSortItems], place[kSortItems];
        bool there[kSortItems];
#pragma unroll
        for (int i = 0; i < kSortItems; ++i) {
            const long long t = t0 + 32 * i, at = min(t, static_cast<long long>(P.T) - 1);
            there[i] = t < P.T;
            key[i] = __ldcg((P.pass == 0 ? P.idx : P.keys) + at);
            token[i] = __ldcg((P.pass == 0 ? P.idx : P.tokens) + at);
        }
#pragma unroll
        for (int i = 0; i < kSortItems; ++i) {
            if (P.pass == 0) {                  // (an index from V on has been reported by the count)
                key[i] = key_of(key[i], P.V);
                token[i] = static_cast<int>(t0 + 32 * i);
            }
            digit[i] = (key[i] >> shift) & (bins - 1);
        }
        rank_tile(S, bins, digit, there, place);
#pragma unroll
        for (int i = 0; i < kSortItems; ++i) {
            const int to = place[i] + S.base[digit[i]];
            if (there[i]) {
                P.keys_out[to] = key[i];
                P.tokens_out[to] = token[i];
            }
            if (!last) {                        // counts of the next pass, once for lanes that count alike
                const int at = static_cast<int>(static_cast<uint32_t>(to) / (P.tiles_per_block * kSortTile)) * kMaxBins + ((key[i] >> (shift + P.bits)) & (bins - 1));
                const uint32_t alike = __match_any_sync(0xffffffffu, there[i] ? at : -1);
                if (there[i] && (alike >> lane) == 1u) atomicAdd(next + at, __popc(alike));
            }
        }
        __syncthreads();
        for (int d = tid; d < bins; d += kSortThreads) S.base[d] += S.total[d];
        __syncthreads();
    }
}

// Few tokens: places by comparing all pairs of them over the whole GPU, with nothing to wait for in between.  A CTA has 32 tokens, one a lane; each of its warps compares them with an eighth of all.
constexpr int kPlaceThreads = 256, kPlaceWarps = kPlaceThreads / 32, kPlaceMost = 4096;
__global__ void __launch_bounds__(kPlaceThreads) embed_place_kernel(const SortParams P) {
    __shared__ __align__(16) int keys[kPlaceMost];
    __shared__ int counts[kPlaceWarps][32];
    chain_wait();
    chain_release();
    if (static_cast<int>(blockIdx.x) >= P.workers) {
        write_zeros(P);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t0 = blockIdx.x * 32, quads = (P.T + 3) / 4;
    bool bad = false;
    int4 own_keys[kPlaceMost / 4 / kPlaceThreads];
    keys_of(P.idx, threadIdx.x, kPlaceThreads, P.T, P.V, own_keys, bad);
#pragma unroll
    for (int i = 0; i < kPlaceMost / 4 / kPlaceThreads; ++i) {
        const int q = threadIdx.x + i * kPlaceThreads;
        if (q < quads) reinterpret_cast<int4*>(keys)[q] = own_keys[i];
    }
    if (bad) set_status(P.status, VARDROP_ERR_INVALID_ARG);
    __syncthreads();
    const int mine = t0 + lane < P.T ? keys[t0 + lane] : 0;
    const int begin = quads * warp / kPlaceWarps, end = quads * (warp + 1) / kPlaceWarps, own = t0 / 4;
    const int4* const all = reinterpret_cast<const int4*>(keys);
    int n = 0;
    const int before = min(end, max(begin, own)), inside = min(end, max(begin, own + 8));
#pragma unroll 4
    for (int q = begin; q < before; ++q) {      // tokens ahead of these: equal keys come first
        const int4 k = all[q];
        n += (k.x <= mine) + (k.y <= mine) + (k.z <= mine) + (k.w <= mine);
    }
    for (int q = before; q < inside; ++q) {
        const int4 k = all[q];
        const int t = 4 * q - t0;
        n += (k.x < mine || (k.x == mine && t < lane)) + (k.y < mine || (k.y == mine && t + 1 < lane)) + (k.z < mine || (k.z == mine && t + 2 < lane)) + (k.w < mine || (k.w == mine && t + 3 < lane));
    }
#pragma unroll 4
    for (int q = inside; q < end; ++q) {
        const int4 k = all[q];
        n += (k.x < mine) + (k.y < mine) + (k.z < mine) + (k.w < mine);
    }
    counts[warp][lane] = n;
    __syncthreads();
    if (warp != 0 || t0 + lane >= P.T) return;
    int place = 0;
#pragma unroll
    for (int w = 0; w < kPlaceWarps; ++w) place += counts[w][lane];
    P.keys_out[place] = mine;
    P.tokens_out[place] = t0 + lane;
}

// ---- sums -----------------------------------------------------------------------------------------------------------------------
struct SumParams {
    const void* d_out;
    const int32_t *keys, *tokens;
    void* d_table;
    float* pieces;                              // [shares, 2, C]: of the row that a share begins in, of the one that it ends in
    int T, V, C, lanes, share, shares, accumulate;
    float scale;
};
template <class Tab, int kVec, int kReps>
__device__ __forceinline__ void row_there(Cells<Tab, kVec, kReps>& old, const SumParams& P, int v, const Cols& k) { old.load(static_cast<const Tab*>(P.d_table) + static_cast<size_t>(v) * P.C, k); }
// `old`: what is there, where that is added to
template <class Tab, int kVec, int kReps>
__device__ __forceinline__ void finish_row(const SumParams& P, int v, const Cols& k, const float (&sum)[kVec * kReps], const Cells<Tab, kVec, kReps>& old) {
    Cells<Tab, kVec, kReps> to;
#pragma unroll
    for (int e = 0; e < kVec * kReps; ++e) to.set(e, P.accumulate ? fmaf(sum[e], P.scale, old.at(e)) : sum[e] * P.scale);
    to.store(static_cast<Tab*>(P.d_table) + static_cast<size_t>(v) * P.C, k);
}
template <class Tab, int kVec, int kReps>
__device__ __forceinline__ void finish_row(const SumParams& P, int v, const Cols& k, const float (&sum)[kVec * kReps]) {
    Cells<Tab, kVec, kReps> old{};
    if (P.accumulate) row_there(old, P, v, k);
    finish_row<Tab, kVec, kReps>(P, v, k, sum, old);
}
// kAdd: rows are added to, and what is there is on its way with the tokens of the batch (a row is read once for each of its tokens in it, out of L1 but for the first).
template <class Tab, class Out, int kVec, int kReps, bool kAdd>
__global__ void __launch_bounds__(kEmbedThreads) embed_sum_kernel(const SumParams P) {
    chain_wait();
    chain_release();
    constexpr int kBatch = kAdd ? kSumBatch / 2 : kSumBatch;
    // the CTA's shares of the sorted tokens at once, so that no row waits for its token's number
    __shared__ int keys[kSumTokens + 2], tokens[kSumTokens];
    const int groups = kEmbedThreads / P.lanes, group = threadIdx.x / P.lanes, lane = threadIdx.x & (P.lanes - 1);
    const long long first_token = static_cast<long long>(blockIdx.x) * groups * P.share;
    const int held = static_cast<int>(min(static_cast<long long>(groups) * P.share, P.T - first_token));
    for (int i = threadIdx.x; i < held; i += kEmbedThreads) {
        keys[i + 1] = __ldcg(P.keys + first_token + i);
        tokens[i] = __ldcg(P.tokens + first_token + i);
    }
    if (threadIdx.x == 0) keys[0] = first_token > 0 ? __ldcg(P.keys + first_token - 1) : -1;
    if (threadIdx.x == 32) keys[held + 1] = first_token + held < P.T ? __ldcg(P.keys + first_token + held) : -1;
    __syncthreads();
    const int share = blockIdx.x * groups + group;
    const Cols k = cols_of<kVec, kReps>(blockIdx.y, P.lanes, lane, P.C);
    if (share >= P.shares || k.c0 >= P.C) return;
    const int begin = group * P.share, end = min(held, begin + P.share);
    const Out* const d_out = static_cast<const Out*>(P.d_out);
    float* const pieces = P.pieces + static_cast<size_t>(share) * 2 * P.C;
    const int ahead = keys[begin], behind = keys[end + 1];
    float sum[kVec * kReps];
    Cells<Tab, kVec, kReps> old{};
    int row = -1;                               // that `sum` is of
    bool first = true;                          // it is the share's first one
    auto leave = [&](bool at_end) {
        if (row < 0 || row == P.V) return;
        const bool from_ahead = first && row == ahead, goes_on = at_end && row == behind;
        if (!from_ahead && !goes_on) {
            finish_row<Tab, kVec, kReps>(P, row, k, sum, old);
            return;
        }
        Cells<float, kVec, kReps> to;
#pragma unroll
        for (int e = 0; e < kVec * kReps; ++e) to.set(e, sum[e]);
        to.store(pieces + (from_ahead ? 0 : P.C), k);
    };
#pragma unroll 1
    for (int i = begin; i < end; i += kBatch) {
        Cells<Out, kVec, kReps> in[kBatch];
        Cells<Tab, kVec, kReps> there[kAdd ? kBatch : 1];
        if (kAdd) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) row_there(there[u], P, min(keys[min(i + u, end - 1) + 1], P.V - 1), k);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) in[u].load(d_out + static_cast<size_t>(tokens[min(i + u, end - 1)]) * P.C, k);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i + u >= end) break;
            const int key = keys[i + u + 1];
            if (key != row) {
                leave(false);
                first = row < 0;
                row = key;
                if (kAdd) old = there[u];
#pragma unroll
                for (int e = 0; e < kVec * kReps; ++e) sum[e] = 0.f;
            }
            if (row == P.V) return;             // nothing but tokens without a row behind it (the row ahead is done)
#pragma unroll
            for (int e = 0; e < kVec * kReps; ++e) sum[e] += in[u].at(e);
        }
    }
    leave(true);
}
// Rows in pieces: the share that a row begins in adds them up, a warp for 256 columns; of rows in many pieces (frequent tokens) all warps of the CTA, every eighth piece each.
constexpr int kJoinWarps = kEmbedThreads / 32, kFewPieces = 8;
template <int kVec, int kReps>
__device__ __forceinline__ void add_pieces(const float* at, size_t step, int count, const Cols& k, float (&sum)[kVec * kReps]) {
#pragma unroll 1
    for (int s = 0; s < count; s += kJoinBatch, at += kJoinBatch * step) {
        Cells<float, kVec, kReps> piece[kJoinBatch];
#pragma unroll
        for (int u = 0; u < kJoinBatch; ++u) piece[u].load(at + step * min(u, count - 1 - s), k);
#pragma unroll
        for (int u = 0; u < kJoinBatch; ++u)
#pragma unroll
            for (int e = 0; e < kVec * kReps; ++e) sum[e] += s + u < count ? piece[u].at(e) : 0.f;
    }
}
template <class Tab, int kVec, int kReps>
__global__ void __launch_bounds__(kEmbedThreads) embed_join_kernel(const SumParams P) {
    __shared__ int many[kJoinWarps][2];                     // row and number of pieces behind its first one, 0: none
    __shared__ float parts[kJoinWarps][32 * kVec * kReps];
    chain_wait();
    chain_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, share = blockIdx.x * kJoinWarps + warp;
    const Cols k = cols_of<kVec, kReps>(blockIdx.y, 32, lane, P.C);
    int row = P.V, count = 0;
    if (share + 1 < P.shares) {
        const long long begin = static_cast<long long>(share) * P.share, end = begin + P.share;
        const int ahead = begin > 0 ? __ldcg(P.keys + begin - 1) : -1, first = __ldcg(P.keys + begin), last = __ldcg(P.keys + end - 1), behind = __ldcg(P.keys + end);
        if (last != P.V && behind == last && !(first == last && ahead == last)) row = last;       // goes on behind this share, and did not begin ahead of it
    }
    if (row != P.V) {                                       // shares behind this one that begin with the row: by 32, then one by one
        const auto begins = [&](int s) { return s < P.shares && __ldcg(P.keys + static_cast<long long>(s) * P.share) == row; };
        count = 1;
        int more;
        do {
            more = __popc(__ballot_sync(0xffffffffu, begins(share + count + 32 * (lane + 1))));
            count += 32 * more;
        } while (more == 32);
        count += __popc(__ballot_sync(0xffffffffu, begins(share + count + lane + 1)));
    }
    const auto piece = [&](int s, int which) { return P.pieces + (static_cast<size_t>(s) * 2 + which) * P.C; };
    const auto own = [&](float (&sum)[kVec * kReps], int s) {
        Cells<float, kVec, kReps> v;
        v.load(piece(s, 1), k);
#pragma unroll
        for (int e = 0; e < kVec * kReps; ++e) sum[e] = v.at(e);
    };
    const size_t step = static_cast<size_t>(2) * P.C;
    if (row != P.V && count <= kFewPieces) {
        float sum[kVec * kReps];
        own(sum, share);
        add_pieces<kVec, kReps>(piece(share + 1, 0), step, count, k, sum);
        finish_row<Tab, kVec, kReps>(P, row, k, sum);
    }
    if (lane == 0) {
        many[warp][0] = row;
        many[warp][1] = count > kFewPieces ? count : 0;
    }
    __syncthreads();
#pragma unroll 1
    for (int w = 0; w < kJoinWarps; ++w) {
        const int pieces = many[w][1], s = blockIdx.x * kJoinWarps + w;
        if (pieces == 0) continue;                          // (of the whole CTA)
        float sum[kVec * kReps] = {};
        add_pieces<kVec, kReps>(piece(s + 1 + warp, 0), kJoinWarps * step, (pieces - warp + kJoinWarps - 1) / kJoinWarps, k, sum);
#pragma unroll
        for (int e = 0; e < kVec * kReps; ++e) parts[warp][e * 32 + lane] = sum[e];
        __syncthreads();
        if (warp == w) {
            own(sum, s);
#pragma unroll
            for (int o = 0; o < kJoinWarps; ++o)
#pragma unroll
                for (int e = 0; e < kVec * kReps; ++e) sum[e] += parts[o][e * 32 + lane];
            finish_row<Tab, kVec, kReps>(P, many[w][0], k, sum);
        }
        __syncthreads();
    }
}

// ---- few tokens and rows ----------------------------------------------------------------------------------------------------------
// A CTA has a row (and up to 256 of its columns) to itself: it looks through the indices, all on their way at once, lists the tokens that have the row, by thread and then in order, and adds theirs up, every group of
// threads each so-many-th token.  (4096 indices a round, each round's sums before the next one's indices, took 13.6 us for the 10272 tokens below instead of 9.4.)
constexpr int kScanLanes = 32, kScanQuads = 11, kScanFew = 4;      // vectors of four indices that a thread looks at, up to 11264 tokens (the list's 44 KB and the counts go without a request for more) and up to 4096
constexpr long long kScanReads = 16ll << 20, kScanCtas = 2368;      // indices that all CTAs read, out of L2; CTAs: sixteen for every SM (29 tokens, 9217 rows of 637: 270 us with 92170 of them), which
//                                                                  holds two to six at a time (40 to 128 registers; three or four where many tokens meet vectors of eight)
// Tokens, and on the average of a row.  A frequent row is one CTA's work, and how the tokens are spread is known on the device alone: the rule takes them as spread, and loses where most of them have one row.
// us for bf16 into rows of 512 fp32, looked through (sorted):
//   tokens, rows       evenly        like one over the rank   a third in one row   all in one row
//    1000,  300      5.4 ( 9.7)           5.9 ( 9.4)              6.8 ( 9.8)        14.5 (11.7)
//    4000,  300      6.5 (15.5)           9.9 (16.7)             19.5 (19.4)          46 (26)
//   10272,  321      9.2 (18.5)          17.7 (21.7)               39 (27)           100 (46)
//   11264,  176      9.2 (17.1)          21.4 (19.0)               42 (25)           108 (44)
//   10272,  321, rows of 64:  8.4 (16.7)  9.2 (19.0)             14.3 (24.5)          31 (44)
constexpr int kScanMost = 4 * kEmbedThreads * kScanQuads, kScanPerRow = 64;
struct ScanParams {
    SumParams sum;
    const int32_t* idx;
    int* status;
};
template <class Tab, class Out, int kVec, int kReps, int kQuads>
__global__ void __launch_bounds__(kEmbedThreads) embed_scan_kernel(const ScanParams S) {
    constexpr int kList = 4 * kEmbedThreads * kQuads, kParts = kEmbedThreads * kVec * kReps;
    __shared__ int list[kList > kParts ? kList : kParts];
    __shared__ int counts[kEmbedThreads / 32];
    float* const parts = reinterpret_cast<float*>(list);           // behind the sums
    chain_wait();
    chain_release();
    const SumParams& P = S.sum;
    const int tid = threadIdx.x, warp = tid >> 5, lane_of_warp = tid & 31, v = blockIdx.x;
    const int groups = kEmbedThreads / P.lanes, group = tid / P.lanes, lane = tid & (P.lanes - 1);
    const Cols k = cols_of<kVec, kReps>(blockIdx.y, P.lanes, lane, P.C);
    const Out* const d_out = static_cast<const Out*>(P.d_out);
    int4 idx[kQuads];
    bool bad = false;
    keys_of(S.idx, tid, kEmbedThreads, P.T, P.V, idx, bad);
    Cells<Tab, kVec, kReps> old{};
    if (P.accumulate && group == 0) row_there(old, P, v, k);
    uint64_t hits = 0;
#pragma unroll
    for (int q = 0; q < kQuads; ++q) {
        const uint32_t four = (idx[q].x == v ? 1u : 0u) | (idx[q].y == v ? 2u : 0u) | (idx[q].z == v ? 4u : 0u) | (idx[q].w == v ? 8u : 0u);
        hits |= static_cast<uint64_t>(four) << (4 * q);
    }
    if (bad && v == 0) set_status(S.status, VARDROP_ERR_INVALID_ARG);
    const int n = __popcll(hits);
    int up = n;
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
        const int ahead = __shfl_up_sync(0xffffffffu, up, s);
        if (lane_of_warp >= s) up += ahead;
    }
    if (lane_of_warp == 31) counts[warp] = up;
    __syncthreads();
    int place = up - n, all = 0;
#pragma unroll
    for (int w = 0; w < kEmbedThreads / 32; ++w) {
        if (w < warp) place += counts[w];
        all += counts[w];
    }
    while (hits) {
        const int b = __ffsll(static_cast<long long>(hits)) - 1;
        list[place++] = 4 * (tid + (b >> 2) * kEmbedThreads) + (b & 3);
        hits &= hits - 1;
    }
    __syncthreads();
    float sum[kVec * kReps] = {};
#pragma unroll 1
    for (int i = group; i < all; i += kSumBatch * groups) {
        Cells<Out, kVec, kReps> in[kSumBatch];
#pragma unroll
        for (int u = 0; u < kSumBatch; ++u) in[u].load(d_out + static_cast<size_t>(list[min(i + u * groups, all - 1)]) * P.C, k);
#pragma unroll
        for (int u = 0; u < kSumBatch; ++u)
#pragma unroll
            for (int e = 0; e < kVec * kReps; ++e) sum[e] += i + u * groups < all ? in[u].at(e) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kVec * kReps; ++e) parts[e * kEmbedThreads + tid] = sum[e];
    __syncthreads();
    if (group != 0 || k.c0 >= P.C || (P.accumulate && all == 0)) return;
    for (int g = 1; g < groups; ++g)
#pragma unroll
        for (int e = 0; e < kVec * kReps; ++e) sum[e] += parts[e * kEmbedThreads + g * P.lanes + lane];
    finish_row<Tab, kVec, kReps>(P, v, k, sum, old);
}

}  // namespace

int embed_validate(const vardrop_embed_cfg& c) {
    if (c.T < 1 || c.V < 1 || c.C < 1) return fail(VARDROP_ERR_INVALID_ARG, "embed: T, V, C >= 1 required (T=%d V=%d C=%d)", c.T, c.V, c.C);
    if (!known_dtype(c.dtype) || !known_dtype(c.out_dtype)) return fail(VARDROP_ERR_INVALID_ARG, "embed: dtype=%d or out_dtype=%d is none of 0, 1, 2", c.dtype, c.out_dtype);
    if (c.accumulate != 0 && c.accumulate != 1) return fail(VARDROP_ERR_INVALID_ARG, "embed: accumulate=%d is neither 0 nor 1", c.accumulate);
    if (!(c.scale - c.scale == 0.f)) return fail(VARDROP_ERR_INVALID_ARG, "embed: scale is not finite");
    if (c.T > (1 << 28) || c.V > (1 << 30) || c.C > (1 << 16)) return fail(VARDROP_ERR_UNSUPPORTED, "embed: T=%d above 2^28, V=%d above 2^30 or C=%d above 65536", c.T, c.V, c.C);
    return VARDROP_OK;
}

size_t embed_workspace_bytes(const vardrop_embed_cfg& c) { return embed_layout(c).total; }

int embed_fwd_launch(const void* table, const int32_t* idx, const vardrop_embed_cfg& c, void* out, void* ws, cudaStream_t stream) {
    const int width = row_vector(c.C), lanes = lanes_of(c.C, width), groups = kEmbedThreads / lanes;
    const EmbedParams P{table, idx, out, static_cast<int*>(ws), c.T, c.V, c.C, lanes, c.scale};
    // several tokens to a thread only where every SM still gets two CTAs
    const bool many = c.T >= 4ll * groups * 2 * sm_count();
    const long long per = static_cast<long long>(groups) * (many ? 4 : 1);
    const dim3 grid(static_cast<unsigned>((c.T + per - 1) / per));
    LaunchScope ls_(K_EMBED_FWD, stream);
    const cudaError_t err = with_dtype(c.dtype, [&](auto tab) {
        return with_dtype(c.out_dtype, [&](auto o) {
            return with_vector(width, [&](auto vec) {
                using Tab = decltype(tab);
                using Out = decltype(o);
                constexpr int kVec = decltype(vec)::value;
                return many ? launch_chained(embed_fwd_kernel<Tab, Out, kVec, 4>, grid, dim3(kEmbedThreads), 0, stream, P)
                            : launch_chained(embed_fwd_kernel<Tab, Out, kVec, 1>, grid, dim3(kEmbedThreads), 0, stream, P);
            });
        });
    });
    return check_cuda(err, "embed: forward launch");
}

int embed_bwd_launch(const void* d_out, const int32_t* idx, const vardrop_embed_cfg& c, void* d_table, void* ws, cudaStream_t stream) {
    const SortPlan s = sort_plan(c);
    const SumPlan u = sum_plan(c);
    const EmbedWs w = embed_layout(c);
    char* const base = static_cast<char*>(ws);
    int32_t* const keys[2] = {reinterpret_cast<int32_t*>(base + w.keys[0]), reinterpret_cast<int32_t*>(base + w.keys[1])};
    int32_t* const tokens[2] = {reinterpret_cast<int32_t*>(base + w.tokens[0]), reinterpret_cast<int32_t*>(base + w.tokens[1])};
    SumParams P{d_out, nullptr, nullptr, d_table, reinterpret_cast<float*>(base + w.pieces), c.T, c.V, c.C, u.lanes, u.share, u.shares, c.accumulate, c.scale};
    const int per = u.vec * u.reps, slabs = (c.C + per * kScanLanes - 1) / (per * kScanLanes);
    if (c.T <= kScanMost && c.T <= static_cast<long long>(kScanPerRow) * c.V && static_cast<long long>(c.T) * c.V * slabs <= kScanReads && static_cast<long long>(c.V) * slabs <= kScanCtas) {
        ScanParams N{P, idx, static_cast<int*>(ws)};
        if (N.sum.lanes > kScanLanes) N.sum.lanes = kScanLanes;
        LaunchScope ls_(K_EMBED_SCAN, stream);
        const cudaError_t err = with_dtype(c.dtype, [&](auto tab) {
            return with_dtype(c.out_dtype, [&](auto o) {
                return with_cells(u.vec, u.reps, [&](auto vec, auto reps) {
                    using Tab = decltype(tab);
                    using Out = decltype(o);
                    constexpr int kVec = decltype(vec)::value, kReps = decltype(reps)::value;
                    const dim3 grid(c.V, slabs);
                    return c.T <= 4 * kEmbedThreads * kScanFew ? launch_chained(embed_scan_kernel<Tab, Out, kVec, kReps, kScanFew>, grid, dim3(kEmbedThreads), 0, stream, N)
                                                               : launch_chained(embed_scan_kernel<Tab, Out, kVec, kReps, kScanQuads>, grid, dim3(kEmbedThreads), 0, stream, N);
                });
            });
        });
        return check_cuda(err, "embed: scan launch");
    }
    SortParams S{idx, nullptr, nullptr, keys[0], tokens[0], reinterpret_cast<int32_t*>(base + w.counts), static_cast<int*>(ws), c.T, c.V, s.bits, 0, s.passes, s.blocks, s.tiles_per_block, nullptr, 0, 0, nullptr, 0};
    // The table's zeros, in as many shares as launches sort.
    const size_t table_bytes = static_cast<size_t>(c.V) * c.C * dtype_bytes(c.dtype), words = c.accumulate ? 0 : table_bytes / 16;
    const int sorts = c.T <= kPlaceMost ? 1 : s.passes + 1;
    if (!c.accumulate && table_bytes % 16 != 0) S.tail = static_cast<unsigned char*>(d_table) + words * 16, S.tail_bytes = static_cast<int>(table_bytes % 16);
    const auto launch_sort = [&](auto kernel, int workers, int threads, int which) {
        const size_t from = words * which / sorts, to = words * (which + 1) / sorts;
        S.zeros = static_cast<uint4*>(d_table) + from;
        S.zero_words = to - from;
        S.workers = workers;
        const size_t most = static_cast<size_t>(sm_count()) * (2048 / threads), wanted = (S.zero_words + threads * 4 - 1) / (threads * 4) + (S.tail_bytes > 0 ? 1 : 0);
        const int fill = static_cast<int>(wanted < most ? wanted : most);
        const cudaError_t e = launch_chained(kernel, dim3(workers + fill), dim3(threads), 0, stream, S);
        S.tail_bytes = 0;
        return e;
    };
    cudaError_t err;
    int at = 0;                                 // of the sorted arrays
    if (c.T <= kPlaceMost) {
        LaunchScope ls_(K_EMBED_PLACE, stream);
        err = launch_sort(embed_place_kernel, (c.T + 31) / 32, kPlaceThreads, 0);
        if (int st = check_cuda(err, "embed: place launch")) return st;
    } else {
        { LaunchScope ls_(K_EMBED_COUNT, stream); err = launch_sort(embed_count_kernel, s.blocks, kSortThreads, 0); }
        if (int st = check_cuda(err, "embed: count launch")) return st;
        for (S.pass = 0; S.pass < s.passes; ++S.pass) {
            at = S.pass & 1;
            S.keys = keys[at ^ 1]; S.tokens = tokens[at ^ 1];
            S.keys_out = keys[at]; S.tokens_out = tokens[at];
            { LaunchScope ls_(K_EMBED_SORT, stream); err = launch_sort(embed_sort_kernel, s.blocks, kSortThreads, S.pass + 1); }
            if (int st = check_cuda(err, "embed: sort launch")) return st;
        }
    }
    P.keys = keys[at];
    P.tokens = tokens[at];
    const int groups = kEmbedThreads / u.lanes;
    const dim3 grid((u.shares + groups - 1) / groups, u.slabs);
    {
        LaunchScope ls_(K_EMBED_SUM, stream);
        err = with_dtype(c.dtype, [&](auto tab) {
            return with_dtype(c.out_dtype, [&](auto o) {
                return with_cells(u.vec, u.reps, [&](auto vec, auto reps) {
                    using Tab = decltype(tab);
                    using Out = decltype(o);
                    constexpr int kVec = decltype(vec)::value, kReps = decltype(reps)::value;
                    return c.accumulate ? launch_chained(embed_sum_kernel<Tab, Out, kVec, kReps, true>, grid, dim3(kEmbedThreads), 0, stream, P)
                                        : launch_chained(embed_sum_kernel<Tab, Out, kVec, kReps, false>, grid, dim3(kEmbedThreads), 0, stream, P);
                });
            });
        });
    }
    if (int st = check_cuda(err, "embed: sum launch")) return st;
    if (u.shares == 1) return VARDROP_OK;
    const dim3 join((u.shares + kJoinWarps - 1) / kJoinWarps, (c.C + 32 * per - 1) / (32 * per));
    {
        LaunchScope ls_(K_EMBED_JOIN, stream);
        err = with_dtype(c.dtype, [&](auto tab) {
            return with_cells(u.vec, u.reps, [&](auto vec, auto reps) { return launch_chained(embed_join_kernel<decltype(tab), decltype(vec)::value, decltype(reps)::value>, join, dim3(kEmbedThreads), 0, stream, P); });
        });
    }
    return check_cuda(err, "embed: join launch");
}

}  // namespace vardrop
