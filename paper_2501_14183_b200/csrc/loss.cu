// Softmax cross entropy over a vocabulary, logits l = scale h w^T, without the logits in memory:
//   lse_t = log sum_v exp(l_tv),  loss_t = lse_t - l_t,label;      G = g_t scale (exp(l_tv - lse_t) - [v = label]),  d_h = G w,  d_w = G^T h
//
// loss_count_kernel   labels of a share of many tokens.
// loss_rows_kernel    tokens that have a label, one behind the other: positions, labels, and backward lse and the factor of their rows; where some have none, also their rows of h.  Only these take
//                     part in any product.  Backward, zeros for the others' d_h.
// loss_stats_kernel   products of 256 tokens x 256 rows of w; of each row of a tile the maximum and the sum of exponentials go to memory, and the label's logit.
// loss_join_kernel    lse and loss from these.
// loss_grad_kernel    backward, for a piece of the vocabulary at a time: the same products again, G of the piece to memory in 16 bits.
// loss_back_kernel    d_h += G w[piece] in fp32 and d_w[piece] = G^T h, the tiles of both in one launch.
// loss_rest_kernel    what that left in several pieces or parts, added up and rounded, to its places.
//
// Bound: the tensor cores, 2 T V C flop forward and 6 T V C backward (2 of them the logits again: to keep them would take 2 T V bytes), and for few tokens reading w.
#include <type_traits>

#include "attn_common.cuh"
#include "loss_tiles.h"
#include "packed_math.cuh"
#include "pair_mma.cuh"
#include "vec_io.cuh"

namespace vardrop {

namespace {

constexpr int kHalfTile = 128;                       // a CTA's rows of a tile
constexpr int kTakeCols = 128;                        // columns that a thread takes out of a finished tile
constexpr int kTakeWarps = 4 * (kPairTile / kTakeCols);
constexpr int kBoxBytes = 64 * 64 * 2;               // what a copy brings
constexpr int kStageBytes = 4 * kBoxBytes;           // two boxes of either operand
constexpr int kStages = 6;
constexpr int kPairThreads = 128 + 32 * kTakeWarps;
constexpr int kPairSmemBytes = 1024 + 1024 + kStages * kStageBytes;
constexpr uint32_t kPairTmemCols = 512;              // two accumulators of 256 columns
constexpr size_t kPieceBytes = 256u << 20;           // of G; larger pieces make fewer passes over d_h
constexpr int kLeastPiece = 1024;
constexpr size_t kPartBytes = 64u << 20;             // of parts of a gradient's products
constexpr float kLog2e = 1.4426950408889634f;

enum LossWord { kLossRows = 16, kLossInverse };      // words of the workspace's header: labelled tokens; the inverse of what G is scaled by

int ceil_div(long long a, long long b) { return static_cast<int>((a + b - 1) / b); }

// ---- layout ---------------------------------------------------------------------------------------------------------------------
struct LossPlan {
    int rows;                   // T up to whole tiles
    int piece, pieces;          // columns of G
    int dh_rows, dw_parts;      // rows that all parts of d_h's products may take; parts of d_w's
    int share, shares;          // tokens of a CTA that finds labels
    size_t place, label, lse, factor, target, most, counts, packed, part, g, dh, dw, total;
};
constexpr int kLeastTokens = 16, kRowsGrid = 296;
LossPlan loss_plan(const vardrop_loss_cfg& c) {
    LossPlan p{};
    p.rows = ceil_div(c.T, kPairTile) * kPairTile;
    p.share = ceil_div(ceil_div(c.T, kRowsGrid), kLeastTokens) * kLeastTokens;
    p.shares = ceil_div(c.T, p.share);
    const long long fit = static_cast<long long>(kPieceBytes / (2ull * p.rows)) / kPairTile * kPairTile, most = fit > kLeastPiece ? fit : kLeastPiece;
    p.pieces = ceil_div(c.V, most);
    p.piece = ceil_div(ceil_div(c.V, p.pieces), kPairTile) * kPairTile;
    p.pieces = ceil_div(c.V, p.piece);
    const long long row_bytes = 4ll * c.C, dh = static_cast<long long>(kPartBytes) / row_bytes, dw = static_cast<long long>(kPartBytes) / (row_bytes * p.piece);
    p.dh_rows = static_cast<int>(dh < p.rows ? p.rows : dh < static_cast<long long>(kMostSplits) * p.rows ? dh : static_cast<long long>(kMostSplits) * p.rows);
    p.dw_parts = p.pieces > 1 || dw < 2 ? 1 : static_cast<int>(dw < kMostSplits ? dw : kMostSplits);
    size_t o = align_up(kWsHeaderBytes, 1024);
    const auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 1024); return at; };
    const size_t T = c.T, C = c.C, rows = p.rows;
    p.place = take(4 * T); p.label = take(4 * T); p.lse = take(4 * T); p.factor = take(4 * T); p.target = take(4 * T);
    p.most = take(4ull * p.shares);
    p.counts = take(4ull * p.shares);
    p.packed = take(2 * rows * C);
    const size_t shared = o;                            // forward and backward each have their own from here on
    p.part = take(8 * rows * (kPairTile / kTakeCols) * ceil_div(c.V, kPairTile));
    const size_t forward = o;
    o = shared;
    p.g = take(2 * rows * p.piece);
    p.dh = take(4ull * p.dh_rows * C);
    p.dw = take(p.dw_parts > 1 ? 4ull * p.piece * C * p.dw_parts : 0);
    p.total = (o > forward ? o : forward) + 1024;       // for a beginning that is not aligned
    return p;
}

// ---- labelled tokens -----------------------------------------------------------------------------------------------------------
struct RowsParams {
    const int32_t* labels;
    const float *lse, *d_loss;                          // backward
    float *loss, *lse_out;                              // forward: zeros where there is no label
    const uint4* h;
    uint4 *packed, *d_h;                                // d_h: zeros where there is no label; NULL: not wanted
    int32_t *place, *label;                             // token and label of a row
    float *row_lse, *factor, *most;                     // most: the largest factor of a share's tokens
    int32_t* counts;                                    // labels of a share, where a launch ahead has counted them
    int* header;
    int T, V, share, vectors;                           // tokens of a CTA; 16-byte vectors of a row
};
constexpr int kRowsThreads = 256, kRowsWarps = kRowsThreads / 32;
__device__ __forceinline__ float block_max(float v, float* shared) {
    v = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kRowsWarps; ++w) v = fmaxf(v, shared[w]);
    return v;
}
__device__ __forceinline__ int has_label(int label, int V) { return label >= 0 && label < V ? 1 : 0; }
// Labels of a share, for many tokens.
__global__ void __launch_bounds__(kRowsThreads) loss_count_kernel(const RowsParams P) {
    __shared__ int sums[kRowsWarps];
    chain_wait();
    chain_release();
    const long long begin = static_cast<long long>(blockIdx.x) * P.share, end = min(static_cast<long long>(P.T), begin + P.share);
    int n = 0;
#pragma unroll 4
    for (long long t = begin + threadIdx.x; t < end; t += kRowsThreads) n += has_label(__ldg(P.labels + t), P.V);
    n = __reduce_add_sync(0xffffffffu, n);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = n;
    __syncthreads();
    if (threadIdx.x != 0) return;
    n = 0;
    for (int w = 0; w < kRowsWarps; ++w) n += sums[w];
    P.counts[blockIdx.x] = n;
}
// Up to kCountHere tokens every CTA counts the labels ahead of its own, and all of them, for itself: 64 KB out of L2 for 16384 tokens, and no launch or wait in between (one CTA for all took 27 us for 8192
// tokens, this takes 4); beyond, a launch counts each share's first (65536 tokens, a sixth of them with labels, 512 channels: 41 -> 24 us, rows four at a time among it).
constexpr int kCountHere = 16384;
__global__ void __launch_bounds__(kRowsThreads) loss_rows_kernel(const RowsParams P) {
    __shared__ int sums[2][kRowsWarps], counts[kRowsWarps];
    __shared__ int rows[kRowsThreads];
    __shared__ float most[kRowsWarps];
    chain_wait();
    chain_release();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long begin = static_cast<long long>(blockIdx.x) * P.share, end = min(static_cast<long long>(P.T), begin + P.share);
    const auto live = [&](int label) { return has_label(label, P.V); };
    int ahead = 0, all = 0;
    if (P.T > kCountHere) {
        for (int i = tid; i < static_cast<int>(gridDim.x); i += kRowsThreads) {
            const int k = __ldcg(P.counts + i);
            all += k;
            if (i < static_cast<int>(blockIdx.x)) ahead += k;
        }
    } else {
        const int quads = P.T >> 2;
#pragma unroll 8
        for (int i = tid; i < quads; i += kRowsThreads) {
            const int4 l = __ldg(reinterpret_cast<const int4*>(P.labels) + i);
            const int k = live(l.x) + live(l.y) + live(l.z) + live(l.w);
            all += k;
            if (4ll * i < begin) ahead += k;            // (shares are multiples of four tokens)
        }
        for (int t = quads * 4 + tid; t < P.T; t += kRowsThreads) {
            const int k = live(__ldg(P.labels + t));
            all += k;
            if (t < begin) ahead += k;
        }
    }
    all = __reduce_add_sync(0xffffffffu, all);
    ahead = __reduce_add_sync(0xffffffffu, ahead);
    if (lane == 0) {
        sums[0][warp] = all;
        sums[1][warp] = ahead;
    }
    __syncthreads();
    all = ahead = 0;
#pragma unroll
    for (int w = 0; w < kRowsWarps; ++w) {
        all += sums[0][w];
        ahead += sums[1][w];
    }
    const int n = all;
    if (blockIdx.x == 0 && tid == 0) P.header[kLossRows] = n;
    float top = 0.f;                                    // of the factors here
    const bool packs = n != P.T;
    if (packs && blockIdx.x == gridDim.x - 1) {         // rows of zeros up to a whole chunk: zero times what lies there need not be zero
        const int fill = (n + kChunk - 1) / kChunk * kChunk;
        for (long long i = static_cast<long long>(n) * P.vectors + tid; i < static_cast<long long>(fill) * P.vectors; i += kRowsThreads) P.packed[i] = make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll 1
    for (long long t0 = begin; t0 < end; t0 += kRowsThreads) {
        const long long t = t0 + tid;
        const int label = t < end ? __ldg(P.labels + t) : -1;
        if (label >= P.V) set_status(P.header, VARDROP_ERR_INVALID_ARG);
        const bool there = live(label) != 0;
        const uint32_t mask = __ballot_sync(0xffffffffu, there);
        __syncthreads();                                // rows and counts of the tokens before are read
        if (lane == 0) counts[warp] = __popc(mask);
        __syncthreads();
        int row = ahead + __popc(mask & ((1u << lane) - 1));
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w) {
            if (w < warp) row += counts[w];
            ahead += counts[w];
        }
        rows[tid] = there ? row : -1;
        if (t < end) {
            if (there) {
                P.place[row] = static_cast<int>(t);
                P.label[row] = label;
                if (P.lse) {
                    const float lse = __ldg(P.lse + t);
                    P.row_lse[row] = lse;
                    const float g = __ldg(P.d_loss + t);
                    P.factor[row] = g;
                    if (isfinite(g)) top = fmaxf(top, fabsf(g));
                    if (fabsf(lse) > 65536.f && isfinite(lse)) set_status(P.header, VARDROP_ERR_UNSUPPORTED);
                }
            } else if (!P.lse) {
                P.loss[t] = 0.f;
                P.lse_out[t] = 0.f;
            }
        }
        if (!packs) continue;
        __syncthreads();
        // four rows of a warp at a time, their loads without a branch
        for (int k = warp; k < kRowsThreads && t0 + k < end; k += 4 * kRowsWarps) {
            int to[4];
            size_t from[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int at = k + u * kRowsWarps;
                to[u] = at < kRowsThreads && t0 + at < end ? rows[at] : -2;
                from[u] = static_cast<size_t>(t0 + at) * P.vectors;
            }
#pragma unroll 1
            for (int i = lane; i < P.vectors; i += 32) {
                uint4 v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = __ldg(P.h + (to[u] >= 0 ? from[u] + i : static_cast<size_t>(i)));
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (to[u] >= 0) P.packed[static_cast<size_t>(to[u]) * P.vectors + i] = v[u];
                    else if (to[u] == -1 && P.d_h) P.d_h[from[u] + i] = make_uint4(0u, 0u, 0u, 0u);
                }
            }
        }
    }
    if (!P.lse) return;
    top = block_max(top, most);
    if (tid == 0) P.most[blockIdx.x] = top;
}
// G is stored times what takes the largest factor to 16320 = 255 2^6: fp16 has room for it, has all its bits down to 2^-28 of it and its last one at 2^-38, and where all factors are alike, as in a mean, the largest entries, factor (p - 1) at the labels,
// lose no bits but those of p (a power of two instead left d_w off by 2.5e-3 of its norm where rounding it alone leaves 1.6e-3).  A warp asks.
__device__ __forceinline__ float scale_up(const float* most, int shares) {
    float top = 0.f;
    for (int i = threadIdx.x & 31; i < shares; i += 32) top = fmaxf(top, __ldcg(most + i));
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
    return top > 0.f ? fminf(16320.f / top, 8.5e37f) : 1.f;
}

// ---- products -------------------------------------------------------------------------------------------------------------------
enum LossMode { kStats, kGrad, kBack };
struct LossMaps {
    CUtensorMap h, packed, w, g;
};
struct PairParams {
    int* header;
    int T, V, C;
    int v0, v1;                                         // the piece
    int pitch;                                          // columns of G
    int add, whole, plain, fp16, shares;                // add: not the first piece; whole: the only one; plain: rows are tokens as they are
    int sectors_h, sectors_w;                           // whether sixteen columns of d_h and of d_w are a sector
    float scale;
    const int32_t *label, *place;
    const float *row_lse, *factor, *most;
    float2* part;                                       // [128 classes each, rows]
    float* target;
    void* g;
    float *dh, *dw;                                     // [parts, rows of tiles, C], [parts, columns of G, C]
    void *d_h, *d_w;
    int rows;                                           // of `part`
    SplitParams split;
};
template <class T>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 v = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A whole 32-byte sector a lane: lanes have different rows, and sixteen bytes of each would be half a sector an instruction.
__device__ __forceinline__ void store_sector(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void load_sector(float (&v)[8], const void* p) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "l"(p) : "memory");
}

// What a thread does with 128 columns of its row of a finished tile: `tm` is where they lie in tensor memory.
template <int kMode, class T, class Tiles>
__device__ __forceinline__ void take_out(const PairParams& P, const PairTile& x, uint32_t tm, int row, int col, int n, float up, const Tiles& tiles) {
    if constexpr (kMode == kStats) {
        const int left = P.V - col;
        if (left <= 0) return;
        const int label = row < n ? __ldg(P.label + row) - col : -1;
        const float k = P.scale * kLog2e;
        float m = -INFINITY, s = 0.f;
#pragma unroll 1
        for (int c = 0; c < kTakeCols && c < left; c += 32) {
            __syncwarp();
            float r[32];
            tmem_ld32(tm + c, r);
            tmem_ld_wait();
            if (label >= c && label < c + 32) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (label == c + e) P.target[row] = r[e] * P.scale;
            }
            if (c + 32 > left) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (c + e >= left) r[e] = -INFINITY;
            }
            float t[4] = {r[0], r[1], r[2], r[3]};
#pragma unroll
            for (int e = 4; e < 32; ++e) t[e & 3] = fmaxf(t[e & 3], r[e]);
            const float top = fmaxf(m, fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])));
            // differences of the sums ahead of the scale: exact however far from zero the logits are; to zero where all of them so far are -inf (classes that are switched off), which then add nothing
            const float base = top == -INFINITY ? 0.f : top;
            float2 sum[2] = {make_float2(s * exp2_fast((m - base) * k), 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const float2 d = mul2(add2(make_float2(r[e], r[e + 1]), both(-base)), both(k));
                sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], make_float2(exp2_fast(d.x), exp2_fast(d.y)));
            }
            s = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
            m = top;
        }
        if (row < n) P.part[static_cast<size_t>(col / kTakeCols) * P.rows + row] = make_float2(m, s);
    } else if constexpr (kMode == kGrad) {
        const bool there = row < n;
        const int left = P.V - P.v0 - col, label = there ? __ldg(P.label + row) - P.v0 - col : -1;
        const float lse = there ? __ldg(P.row_lse + row) : 0.f, factor = there ? __ldg(P.factor + row) * up : 0.f;
        T* const to = static_cast<T*>(P.g) + static_cast<size_t>(row) * P.pitch + col;
#pragma unroll 1
        for (int c = 0; c < kTakeCols; c += 32) {
            __syncwarp();
            float r[32];
            tmem_ld32(tm + c, r);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const float2 d = mul2(fma2(make_float2(r[e], r[e + 1]), both(P.scale), both(-lse)), both(kLog2e));
                r[e] = exp2_fast(d.x);
                r[e + 1] = exp2_fast(d.y);
            }
            if (label >= c && label < c + 32) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (label == c + e) r[e] -= 1.f;
            }
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const float2 v = mul2(make_float2(r[e], r[e + 1]), both(factor));
                r[e] = v.x;
                r[e + 1] = v.y;
            }
            if (!there || c + 32 > left) {              // zeros, whatever the products there are
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (!there || c + e >= left) r[e] = 0.f;
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                uint32_t v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = pack16<T>(r[16 * q + 2 * e], r[16 * q + 2 * e + 1]);
                store_sector(to + c + 16 * q, v);
            }
        }
    } else {
        const bool some = x.k1 > x.k0, there = row < (x.dw ? P.v1 - P.v0 : n), add = !x.dw && P.add;
        const bool direct = x.dw ? tiles.splits.dw == 1 : P.whole && tiles.splits.dh == 1;        // nothing else comes to it
        const float mul = up;
        const size_t rows = x.dw ? P.split.piece : (n + kPairTile - 1) / kPairTile * kPairTile;
        float* const acc = (x.dw ? P.dw : P.dh) + (x.part * rows + row) * P.C + col;
        const size_t to = x.dw ? static_cast<size_t>(P.v0) + row : there && direct ? static_cast<size_t>(__ldg(P.place + row)) : 0;
        T* const out = static_cast<T*>(x.dw ? P.d_w : P.d_h) + to * P.C + col;
#pragma unroll 1
        for (int c = 0; c < kTakeCols && col + c < P.C; c += 32) {
            __syncwarp();
            float r[32];
            tmem_ld32(tm + c, r);
            tmem_ld_wait();
            if (!some) {
#pragma unroll
                for (int e = 0; e < 32; ++e) r[e] = 0.f;
            }
            if (!there) {
            } else if (!direct) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (col + c + 8 * q >= P.C) continue;             // C is a multiple of 8
                    float v[8] = {};
                    if (add) load_sector(v, acc + c + 8 * q);
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(r[8 * q + e] + v[e]);
                    store_sector(acc + c + 8 * q, w);
                }
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = pack16<T>(r[16 * q + 2 * e] * mul, r[16 * q + 2 * e + 1] * mul);
                    T* const at = out + c + 16 * q;
                    if (x.dw ? P.sectors_w : P.sectors_h) {
                        if (col + c + 16 * q < P.C) store_sector(at, w);
                    } else {
                        if (col + c + 16 * q < P.C) *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
                        if (col + c + 16 * q + 8 < P.C) reinterpret_cast<uint4*>(at)[1] = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
            }
        }
    }
}

// warp 0          (of either CTA) loads: a ring of stages, 64 of the contracted axis for 128 rows of A and 128 of B
// warp 1          of the leader: products
// warps 4 to 11   (of either CTA) take a finished tile out, 128 columns of a row a thread, under the products of the next one.  That takes 2.4 us where exponentials are taken (1.1 of them at their
//                 unit's rate; sixteen warps with half as many columns take as long), the products of 512 channels 2.2: below that, this bounds a tile.
template <int kMode, class T>
__global__ void __launch_bounds__(kPairThreads, 1) loss_products_kernel(const __grid_constant__ LossMaps maps, const PairParams P) {
    extern __shared__ unsigned char smem_dyn[];
    uint64_t* const bar_full = reinterpret_cast<uint64_t*>(smem_dyn);       // [kStages] both CTAs' copies (the leader's)
    uint64_t* const bar_empty = bar_full + kStages;                         // [kStages] the products that read the stage are done
    uint64_t* const bar_acc = bar_empty + kStages;                          // [2] the tile is complete
    uint64_t* const bar_taken = bar_acc + 2;                                // [2] and has been taken out by the warps of both CTAs (the leader's)
    uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bar_taken + 2);
    unsigned char* const stages = align_tiles(smem_dyn + 1024);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_rank();
    if (warp == 0) pair_tmem_alloc(tmem_slot, kPairTmemCols);
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(bar_full + i, 1);
            mbar_init(bar_empty + i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_acc + i, 1);
            mbar_init(bar_taken + i, 2 * kTakeWarps);
        }
        mbar_fence_init();
    }
    __syncwarp();
    tc_fence_before();
    pair_sync();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    chain_wait();
    chain_release();

    const int n = P.plain ? P.T : __ldcg(P.header + kLossRows), columns = P.v1 - P.v0;
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const auto tiles = [&] {
        if constexpr (kMode == kBack) return GradTiles(P.split, n, columns, pair, pairs);
        else return LogitTiles{tiles_of(n, kPairTile), tiles_of(columns, kPairTile), tiles_of(P.C, kChunk), pair, pairs};
    }();
    // Whether the contracted axis is the rows of the tensor: of G for d_w, of w and h for either gradient.
    constexpr bool b_mn = kMode == kBack;
    PairTile x;
    bool ok = true;
    if (warp == 0) {
        if (lane == 0) {
            const CUtensorMap* const map_h = n == P.T ? &maps.h : &maps.packed;
            tma_prefetch_desc(map_h);
            tma_prefetch_desc(&maps.w);
            if (kMode == kBack) tma_prefetch_desc(&maps.g);
            uint32_t it = 0;
#pragma unroll 1
            for (int i = 0; ok && tiles.at(i, x); ++i) {
                const int a0 = x.m * kPairTile + static_cast<int>(rank) * kHalfTile, b0 = x.n * kPairTile + static_cast<int>(rank) * kHalfTile;
                const CUtensorMap* const map_a = kMode == kBack ? &maps.g : map_h;
                const CUtensorMap* const map_b = x.dw ? map_h : &maps.w;
                const int row_b = x.dw ? 0 : P.v0;                               // rows of w begin with the piece
#pragma unroll 1
                for (int kc = x.k0; kc < x.k1; ++kc, ++it) {
                    const uint32_t st = it % kStages;
                    ok = mbar_wait(bar_empty + st, ((it / kStages) & 1) ^ 1);
                    if (!ok) break;
                    const uint32_t full = leaders(bar_full + st), to = smem_u32(stages) + st * kStageBytes;
                    if (rank == 0) mbar_expect_tx(bar_full + st, 2 * kStageBytes);
                    const int k = kc * kChunk;
                    pair_load_2d(to, map_a, full, x.dw ? a0 : k, x.dw ? k : a0);
                    pair_load_2d(to + kBoxBytes, map_a, full, x.dw ? a0 + 64 : k, x.dw ? k : a0 + 64);
                    pair_load_2d(to + 2 * kBoxBytes, map_b, full, b_mn ? b0 : k, row_b + (b_mn ? k : b0));
                    pair_load_2d(to + 3 * kBoxBytes, map_b, full, b_mn ? b0 + 64 : k, row_b + (b_mn ? k : b0 + 64));
                }
            }
            // what the leader still sends to this CTA's barriers comes before it leaves
#pragma unroll 1
            for (uint32_t j = it > kStages ? it - kStages : 0; j < it && ok; ++j) ok = mbar_wait(bar_empty + j % kStages, (j / kStages) & 1);
        }
        __syncwarp();
    } else if (warp == 1 && rank == 0) {
        // rows of 128 bytes: eight of them 1024 apart, panels of 64 rows or columns a box
        const uint64_t a_rows = umma_desc_sw128(smem_u32(stages), 16, 1024), a_cols = umma_desc_sw128(smem_u32(stages), kBoxBytes, 1024);
        const uint64_t b_desc = umma_desc_sw128(smem_u32(stages) + 2 * kBoxBytes, b_mn ? kBoxBytes : 16, 1024);
        constexpr uint32_t b_step = b_mn ? 2048 : 32;                            // 16 of the contracted axis
        uint32_t it = 0;
#pragma unroll 1
        for (int i = 0; ok && tiles.at(i, x); ++i) {
            const uint32_t idesc = pair_idesc(P.fp16 != 0, x.dw, b_mn), a_step = x.dw ? 2048 : 32;
            const uint64_t a_desc = x.dw ? a_cols : a_rows;
            const uint32_t d = tmem + (i & 1) * kPairTile;
            ok = __all_sync(0xffffffffu, mbar_wait(bar_taken + (i & 1), ((i >> 1) & 1) ^ 1));
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int kc = x.k0; kc < x.k1; ++kc, ++it) {
                const uint32_t st = it % kStages;
                ok = __all_sync(0xffffffffu, mbar_wait(bar_full + st, (it / kStages) & 1));
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t a = umma_desc_advance(a_desc, st * kStageBytes), b = umma_desc_advance(b_desc, st * kStageBytes);
#pragma unroll
                    for (int ks = 0; ks < kChunk / 16; ++ks) pair_mma(d, umma_desc_advance(a, ks * a_step), umma_desc_advance(b, ks * b_step), idesc, kc > x.k0 || ks > 0 ? 1u : 0u);
                    pair_commit(bar_empty + st);
                }
                __syncwarp();
            }
            if (ok && elect_one()) pair_commit(bar_acc + (i & 1));
            __syncwarp();
        }
    } else if (warp >= 4) {
        const int in_tile = static_cast<int>(rank) * kHalfTile + (warp & 3) * 32 + lane, part = (warp - 4) >> 2;
        const uint32_t tm_at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + part * kTakeCols;
        // kGrad: what G is scaled by; kBack: what takes that away from its products
        float up = 1.f;
        if (kMode == kGrad) {
            up = scale_up(P.most, P.shares);
            if (blockIdx.x == 0 && warp == 4 && lane == 0) P.header[kLossInverse] = __float_as_int(1.f / up);
        } else if (kMode == kBack) {
            up = P.scale * __int_as_float(__ldcg(P.header + kLossInverse));
        }
#pragma unroll 1
        for (int i = 0; tiles.at(i, x); ++i) {
            ok = __all_sync(0xffffffffu, mbar_wait(bar_acc + (i & 1), (i >> 1) & 1));
            if (!ok) break;
            tc_fence_after();
            take_out<kMode, T>(P, x, tm_at + (i & 1) * kPairTile, x.m * kPairTile + in_tile, x.n * kPairTile + part * kTakeCols, n, up, tiles);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) leader_arrive(leaders(bar_taken + (i & 1)));
        }
    }
    if (!ok) set_status(P.header, VARDROP_ERR_TIMEOUT);
    __syncwarp();
    tc_fence_before();
    pair_sync();
    if (warp == 0) pair_tmem_dealloc(tmem, kPairTmemCols);
}

// ---- lse and loss ---------------------------------------------------------------------------------------------------------------
struct JoinParams {
    const float2* part;
    const float* target;
    const int32_t *place, *labels;                      // labels: where rows are tokens as they are
    int* header;
    float *loss, *lse;
    int parts, rows, T, V;                              // parts of the vocabulary; rows of a part's sums
    float scale;
};
constexpr int kJoinRows = 32, kJoinWays = 32, kJoinBatch = 8;
// A maximum and a sum of exponentials relative to it, with further ones added: those of a batch to their largest first.
template <int kCount>
__device__ __forceinline__ float2 joined(float2 sum, const float2 (&v)[kCount], float k) {
    float top = sum.x;
#pragma unroll
    for (int e = 0; e < kCount; ++e) top = fmaxf(top, v[e].x);
    float s = sum.y == 0.f ? 0.f : sum.y * exp2_fast((sum.x - top) * k);
#pragma unroll
    for (int e = 0; e < kCount; ++e) s += v[e].y == 0.f ? 0.f : v[e].y * exp2_fast((v[e].x - top) * k);       // (0: none)
    return make_float2(top, s);
}
__global__ void __launch_bounds__(kJoinRows * kJoinWays) loss_join_kernel(const JoinParams P) {
    __shared__ float2 s[kJoinWays][kJoinRows];
    chain_wait();
    chain_release();
    const int n = P.labels ? P.T : __ldcg(P.header + kLossRows), x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const float k = P.scale * kLog2e;
    const float2 none = make_float2(-INFINITY, 0.f);
#pragma unroll 1
    for (int first = blockIdx.x * kJoinRows; first < n; first += gridDim.x * kJoinRows) {
        const int row = first + x;
        float2 sum = none;
        const float2* const from = P.part + min(row, n - 1);
#pragma unroll 1
        for (int j = y; j < P.parts; j += kJoinWays * kJoinBatch) {
            float2 v[kJoinBatch];
#pragma unroll
            for (int u = 0; u < kJoinBatch; ++u) v[u] = __ldcg(from + static_cast<size_t>(min(j + u * kJoinWays, P.parts - 1)) * P.rows);
#pragma unroll
            for (int u = 0; u < kJoinBatch; ++u)
                if (j + u * kJoinWays >= P.parts) v[u] = none;
            sum = joined(sum, v, k);
        }
        __syncthreads();                                // the rows before are done
        s[y][x] = sum;
        __syncthreads();
        if (y != 0 || row >= n) continue;
        float2 v[kJoinWays - 1];
#pragma unroll
        for (int j = 1; j < kJoinWays; ++j) v[j - 1] = s[j][x];
        sum = joined(sum, v, k);
        const float lse = fmaf(sum.x, P.scale, logf(sum.y));
        const int t = P.labels ? row : P.place[row], label = P.labels ? __ldg(P.labels + row) : 0;
        if (label >= P.V) set_status(P.header, VARDROP_ERR_INVALID_ARG);
        const bool there = label >= 0 && label < P.V;
        P.lse[t] = there ? lse : 0.f;
        P.loss[t] = there ? lse - P.target[row] : 0.f;
    }
}

// ---- gradients' last step -------------------------------------------------------------------------------------------------------
struct RestParams {
    const float *dh, *dw;
    const int32_t* place;                               // token of a row
    const int* header;
    void *d_h, *d_w;
    int T, V, C, whole;
    int h_blocks;                                       // CTAs of d_h
    float scale;
    SplitParams split;
};
constexpr int kRestThreads = 256, kRestRows = 16;       // rows of a CTA
// Rows that are not in their places yet: of d_h where there were several pieces or parts, of d_w where there were parts.  Eight columns a thread.
template <class T>
__global__ void __launch_bounds__(kRestThreads) loss_rest_kernel(const RestParams P) {
    chain_wait();
    chain_release();
    const bool dw = static_cast<int>(blockIdx.x) >= P.h_blocks;
    const int n = __ldcg(P.header + kLossRows), vectors = P.C / 8, count = dw ? P.V : n;
    const Splits splits = splits_of(P.split, n);
    if (dw ? splits.dw == 1 : P.whole && splits.dh == 1) return;
    const int first = (static_cast<int>(blockIdx.x) - (dw ? P.h_blocks : 0)) * kRestRows, rows = min(kRestRows, count - first), parts = dw ? splits.dw : splits.dh;
    const size_t part = static_cast<size_t>(dw ? P.split.piece : (n + kPairTile - 1) / kPairTile * kPairTile) * P.C;
    const float mul = P.scale * __int_as_float(__ldcg(P.header + kLossInverse));
    const float* const base = (dw ? P.dw : P.dh) + static_cast<size_t>(first) * P.C;
#pragma unroll 1
    for (int at = threadIdx.x; at < rows * vectors; at += kRestThreads) {
        const int r = at / vectors, c = (at - r * vectors) * 8;
        const float* from = base + static_cast<size_t>(r) * P.C + c;
        float v[8] = {};
#pragma unroll 4
        for (int s = 0; s < parts; ++s, from += part) {
            const Pack<float, 8> a = load_pack<float, 8>(from);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += a.e[e];
        }
        Pack<T, 8> o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o.e[e] = from_float<T>(v[e] * mul);
        const size_t to = dw ? static_cast<size_t>(first) + r : static_cast<size_t>(__ldcg(P.place + first + r));
        store_pack(static_cast<T*>(dw ? P.d_w : P.d_h) + to * P.C + c, o);
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
// [rows, cols] of 16-bit elements, box = 64 x 64, 128-byte swizzle, zeros outside
int loss_map(CUtensorMap* map, const void* base, bool fp16, long long rows, long long cols) {
    static const EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        const bool found = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) == cudaSuccess && qres == cudaDriverEntryPointSuccess;
        return found ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
    }();
    if (!fn) return fail(VARDROP_ERR_CUDA, "loss: cuTensorMapEncodeTiled entry point not available");
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(cols) * 2};
    const cuuint32_t box[2] = {64, 64}, estr[2] = {1, 1};
    const CUresult r = fn(map, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? VARDROP_OK : fail(VARDROP_ERR_CUDA, "loss: cuTensorMapEncodeTiled failed with code %d", static_cast<int>(r));
}

template <int kMode, class T>
int launch_products(int id, long long tiles, const LossMaps& maps, const PairParams& P, cudaStream_t stream) {
    static thread_local int attr_dev = -1;
    int dev = 0;
    cudaGetDevice(&dev);
    if (attr_dev != dev) {
        if (int st = check_cuda(cudaFuncSetAttribute(loss_products_kernel<kMode, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmemBytes), "loss: smem attribute")) return st;
        attr_dev = dev;
    }
    const long long pairs = sm_count() / 2;
    const int grid = 2 * static_cast<int>(tiles < pairs ? tiles : pairs);
    LaunchScope ls_(id, stream);
    return check_cuda(launch_chained_clusters(2, loss_products_kernel<kMode, T>, dim3(grid), dim3(kPairThreads), kPairSmemBytes, stream, maps, P), "loss: products launch");
}

struct LossCall {
    LossPlan plan;
    LossMaps maps;
    PairParams P;
    char* base;
};
// Where things are, and the launches that both passes begin with.
int loss_begin(LossCall& L, const void* h, const void* w, const int32_t* labels, const vardrop_loss_cfg& c, const float* lse, const float* d_loss, float* loss, float* lse_out, void* d_h,
               void* ws, bool backward, bool plain, cudaStream_t stream) {
    L.plan = loss_plan(c);
    const LossPlan& p = L.plan;
    // (a workspace begins on any 16 bytes; its header does so there, everything else behind the next multiple of 1024, plus 1024)
    char* const base = L.base = reinterpret_cast<char*>(align_up(reinterpret_cast<uintptr_t>(ws), 1024));
    const bool fp16 = c.dtype == 1;
    if (int st = loss_map(&L.maps.h, h, fp16, c.T, c.C)) return st;
    if (int st = loss_map(&L.maps.packed, base + p.packed, fp16, p.rows, c.C)) return st;
    if (int st = loss_map(&L.maps.w, w, fp16, c.V, c.C)) return st;
    if (backward) {
        if (int st = loss_map(&L.maps.g, base + p.g, fp16, p.rows, p.piece)) return st;
    } else {
        L.maps.g = L.maps.packed;
    }
    RowsParams R{labels, lse, d_loss, loss, lse_out, static_cast<const uint4*>(h), reinterpret_cast<uint4*>(base + p.packed), static_cast<uint4*>(d_h), reinterpret_cast<int32_t*>(base + p.place),
                 reinterpret_cast<int32_t*>(base + p.label), reinterpret_cast<float*>(base + p.lse), reinterpret_cast<float*>(base + p.factor),
                 reinterpret_cast<float*>(base + p.most), reinterpret_cast<int32_t*>(base + p.counts), static_cast<int*>(ws), c.T, c.V, p.share, c.C / 8};
    if (!plain && c.T > kCountHere) {
        LaunchScope ls_(K_LOSS_COUNT, stream);
        if (int st = check_cuda(launch_chained(loss_count_kernel, dim3(p.shares), dim3(kRowsThreads), 0, stream, R), "loss: count launch")) return st;
    }
    if (!plain) {
        LaunchScope ls_(K_LOSS_ROWS, stream);
        if (int st = check_cuda(launch_chained(loss_rows_kernel, dim3(p.shares), dim3(kRowsThreads), 0, stream, R), "loss: rows launch")) return st;
    }
    PairParams& P = L.P;
    P = PairParams{};
    P.header = R.header;
    P.T = c.T; P.V = c.V; P.C = c.C; P.v0 = 0; P.v1 = c.V; P.pitch = p.piece; P.shares = p.shares; P.fp16 = fp16; P.scale = c.scale == 0.f ? 1.f : c.scale;
    P.plain = plain;
    P.label = plain ? labels : R.label; P.place = R.place; P.row_lse = R.row_lse; P.factor = R.factor; P.most = R.most;
    P.part = reinterpret_cast<float2*>(base + p.part); P.target = reinterpret_cast<float*>(base + p.target);
    P.g = base + p.g; P.dh = reinterpret_cast<float*>(base + p.dh); P.dw = reinterpret_cast<float*>(base + p.dw); P.rows = p.rows;
    return VARDROP_OK;
}

template <class T>
int loss_backward(LossCall& L, const vardrop_loss_cfg& c, void* d_h, void* d_w, cudaStream_t stream) {
    const LossPlan& p = L.plan;
    const long long tm = p.rows / kPairTile, tc = ceil_div(c.C, kPairTile);
    PairParams& P = L.P;
    P.split = SplitParams{sm_count() / 2, static_cast<int>(tc), p.piece, p.dh_rows, p.dw_parts, d_h != nullptr, d_w != nullptr};
    P.d_h = d_h; P.d_w = d_w; P.whole = p.pieces == 1;
    P.sectors_h = c.C % 16 == 0 && reinterpret_cast<uintptr_t>(d_h) % 32 == 0;
    P.sectors_w = c.C % 16 == 0 && reinterpret_cast<uintptr_t>(d_w) % 32 == 0;
    for (int i = 0; i < p.pieces; ++i) {
        P.v0 = i * p.piece;
        P.v1 = c.V - P.v0 < p.piece ? c.V : P.v0 + p.piece;
        P.add = i > 0;
        const int tv = ceil_div(P.v1 - P.v0, kPairTile);
        if (int st = launch_products<kGrad, T>(K_LOSS_GRAD, tm * tv, L.maps, P, stream)) return st;
        // (how many parts there are is known on the device)
        if (int st = launch_products<kBack, T>(K_LOSS_BACK, (d_h ? tm * tc * kMostSplits : 0) + (d_w ? tv * tc * p.dw_parts : 0), L.maps, P, stream)) return st;
    }
    // what may be left in pieces or parts: small problems have neither, and a launch less
    const bool rows = d_h && (p.pieces > 1 || may_split_dh(P.split)), parts = d_w && may_split_dw(P.split, c.T);
    if (!rows && !parts) return VARDROP_OK;
    const RestParams R{P.dh, P.dw, P.place, P.header, d_h, d_w, c.T, c.V, c.C, P.whole, rows ? ceil_div(c.T, kRestRows) : 0, P.scale, P.split};
    LaunchScope ls_(K_LOSS_REST, stream);
    return check_cuda(launch_chained(loss_rest_kernel<T>, dim3(R.h_blocks + (parts ? ceil_div(c.V, kRestRows) : 0)), dim3(kRestThreads), 0, stream, R), "loss: rest launch");
}

}  // namespace

int loss_validate(const vardrop_loss_cfg& c) {
    if (c.T < 1 || c.V < 1 || c.C < 1) return fail(VARDROP_ERR_INVALID_ARG, "loss: T, V, C >= 1 required (T=%d V=%d C=%d)", c.T, c.V, c.C);
    if (c.dtype != 0 && c.dtype != 1) return fail(c.dtype == 2 ? VARDROP_ERR_UNSUPPORTED : VARDROP_ERR_INVALID_ARG, "loss: dtype=%d is neither bf16 nor fp16", c.dtype);
    if (!(c.scale >= 0.f && c.scale <= 1e30f)) return fail(VARDROP_ERR_INVALID_ARG, "loss: scale outside 0..1e30");
    if (c.C % 8 != 0) return fail(VARDROP_ERR_UNSUPPORTED, "loss: C=%d is no multiple of 8", c.C);
    if (c.T > (1 << 24) || c.V > (1 << 24) || c.C > (1 << 16)) return fail(VARDROP_ERR_UNSUPPORTED, "loss: T=%d or V=%d above 2^24, or C=%d above 65536", c.T, c.V, c.C);
    if (static_cast<long long>(ceil_div(c.T, kPairTile)) * ceil_div(c.V, kPairTile) > (1ll << 30)) return fail(VARDROP_ERR_UNSUPPORTED, "loss: T=%d times V=%d above 2^46", c.T, c.V);
    return VARDROP_OK;
}

size_t loss_workspace_bytes(const vardrop_loss_cfg& c) { return loss_plan(c).total; }

int loss_fwd_launch(const void* h, const void* w, const int32_t* labels, const vardrop_loss_cfg& c, float* loss, float* lse, void* ws, cudaStream_t stream) {
    LossCall L;
    // One row of tiles, whatever has a label: tokens as they are, and a launch less (32 tokens, 1000 classes, 512 channels: 11.7 -> 9.3 us).  Rows without one come to nothing but themselves here.
    const bool plain = c.T <= kPairTile;
    if (int st = loss_begin(L, h, w, labels, c, nullptr, nullptr, loss, lse, nullptr, ws, false, plain, stream)) return st;
    const LossPlan& p = L.plan;
    const int tv = ceil_div(c.V, kPairTile);
    if (int st = launch_products<kStats, __nv_bfloat16>(K_LOSS_STATS, static_cast<long long>(p.rows / kPairTile) * tv, L.maps, L.P, stream)) return st;
    const JoinParams J{L.P.part, L.P.target, L.P.place, plain ? labels : nullptr, L.P.header, loss, lse, ceil_div(c.V, kTakeCols), p.rows, c.T, c.V, L.P.scale};
    LaunchScope ls_(K_LOSS_JOIN, stream);
    return check_cuda(launch_chained(loss_join_kernel, dim3(ceil_div(c.T, kJoinRows) < 2 * sm_count() ? ceil_div(c.T, kJoinRows) : 2 * sm_count()), dim3(kJoinRows * kJoinWays), 0, stream, J), "loss: join launch");
}

int loss_bwd_launch(const void* h, const void* w, const int32_t* labels, const float* lse, const float* d_loss, const vardrop_loss_cfg& c, void* d_h, void* d_w, void* ws, cudaStream_t stream) {
    LossCall L;
    if (int st = loss_begin(L, h, w, labels, c, lse, d_loss, nullptr, nullptr, d_h, ws, true, false, stream)) return st;
    return c.dtype == 1 ? loss_backward<__half>(L, c, d_h, d_w, stream) : loss_backward<__nv_bfloat16>(L, c, d_h, d_w, stream);
}

}  // namespace vardrop
