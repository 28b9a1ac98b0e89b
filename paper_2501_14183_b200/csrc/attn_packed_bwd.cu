// Attention over packed sequences, backward.
//
// packed_prep_kernel       Delta_i = sum_d dO_id O_id, and the cleared dQ accumulator.
// attn_packed_bwd_kernel   one persistent CTA per SM over items of one 128-key tile of a key head, with the query tiles of all its query heads; dQ is added into an fp32
//                          accumulator by bulk reduce-adds.
// packed_short_kernel      sequences of a single tile, all of it; runs as SMs become free.
// packed_convert_kernel    dQ of the others to bf16 rows.
//
// The roles, tensor memory and arithmetic of a step are those of bwd_many_kernel; what differs: tiles of sequences that end inside, heads that share their keys (their dK
// and dV add up in tensor memory over the item), the diagonal of a causal call, and the accumulator in which every sequence begins a tile, so that what a last tile adds behind
// its end (zeros, but zero times a key that is not finite) lies where nothing reads.
//
// P and dS are rounded to bf16, the operand type of the products that take them: half a step, 2^-8 of a value, as the outputs' own.  (dQ is then off by 0.0025 of its norm where rounding it alone
// gives 0.0017; two bf16 terms a value would take those three of five products twice.)
#include "attn_packed.cuh"

namespace vardrop {

namespace {

// P is exp(scaled score - lse), and lse comes with the 24 bits of fp32: from |lse| 2^-20 or so on that is what P is known to, 2^-4 of itself here.  Beyond, the call says so.
constexpr float kMostLse = 65536.f;
__device__ __forceinline__ bool lse_too_far(float lse) { return fabsf(lse) > kMostLse && fabsf(lse) < INFINITY; }

struct PackedBwdParams {
    const __nv_bfloat16 *q, *k, *v, *d_o;   // rows of a sequence's last tile (the other loads go through the tensor maps)
    const float* lse;                 // [Hq, T]
    const float* delta;               // [Hq, rows]
    __nv_bfloat16 *dk, *dv;           // [T, Hkv, D]
    PlanView plan;
    int* status;
    long long sTq, sHq, sTkv, sHkv;
    int T, Hq, Hkv, group, D, rows, causal;
    int may_split;
    float scale, scale_log2, half_inv_scale;      // of dK; in the exponents, and 0.5 / scale there
};

// ---------------------------------------------------------------------------------------------------------
// sequences of a single tile
// ---------------------------------------------------------------------------------------------------------
struct PackedShortParams {
    const __nv_bfloat16 *q, *k, *v, *d_o;
    const float* lse;                 // [Hq, T]
    __nv_bfloat16 *dq, *dk, *dv;
    PlanView plan;
    int* status;
    long long sTq, sHq, sTkv, sHkv;
    int T, Hq, Hkv, group, D, causal;
    int alone;                        // the only launch of the call; otherwise attn_packed_bwd_kernel's is the one before
    float scale, scale_log2;
};

constexpr int kShortThreads = 256;
constexpr int kShortPerSm = 2;
constexpr int kShortSmemBytes = 4 * kTileBytes /*Q, dO, K, V*/ + 2 * kTileBytes /*P, then dS: two 64-key panels*/;

// An item is a key head of such a sequence, with its query heads one after another.  Two threads a query row, 64 keys each.  With whole rows of P and dP at hand
// Delta_i = sum_j P_ij dP_ij comes from them, in fp32: dS then sums to zero over a row as it should, where dO . O with an O of bf16 leaves 2^-9 of a term that for a few keys is as
// large as dS itself (and neither O nor prep, accumulator and conversion are needed).
// A chain of latencies like the forward's: two CTAs to an SM, rolled loops over 32 scores; P and dP stay in tensor memory between the two passes over a row.  P^T dO, dS^T Q and
// dS K take P and dS from shared memory, the first two as transposed views.
// Grouped heads of a short sequence share tiles, as many as have room (39 sequences of 1 to 13 tokens, 24 query heads on 3, forward and backward: 45 us one after another, 29 like this).
// kGrouped: several query heads a key head; dV and dK add up in columns of their own, which takes all of tensor memory and leaves one CTA to an SM.  Otherwise they come over the
// scores' columns.
// Tensor memory: S, P 128 | dP 128, then (dV 64 | dK 64 | dQ 64) over them, or with kGrouped: dQ 64 over S; dV 64 | dK 64 behind.
template <bool kGrouped>
__global__ void __launch_bounds__(kShortThreads, kShortPerSm) packed_short_kernel(const PackedShortParams P) {
    extern __shared__ __align__(1024) unsigned char smem_dyn[];
    __shared__ uint64_t bar;
    __shared__ uint32_t tmem_slot;
    __shared__ float s_delta[2][kTile];
    constexpr uint32_t kCols = kGrouped ? 512 : 256;
    constexpr uint32_t kDv = kGrouped ? 256 : 0, kDk = kGrouped ? 320 : 64, kDq = kGrouped ? 0 : 128;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (smem_u32(smem_dyn) & 1023u) {
        chain_wait();
        if (tid == 0) set_status(P.status, VARDROP_ERR_CUDA);
        return;
    }
    if (warp == 0) {
        tmem_alloc(&tmem_slot, kCols);
        tmem_relinquish();
    }
    if (tid == 0) {
        mbar_init(&bar, 1);
        mbar_fence_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    unsigned char* const sQ = smem_dyn;
    unsigned char* const sdO = sQ + kTileBytes;
    unsigned char* const sK = sdO + kTileBytes;
    unsigned char* const sV = sK + kTileBytes;
    unsigned char* const sP = sV + kTileBytes;
    const uint32_t tmem = tmem_slot;
    const int row = (warp & 3) * 32 + lane, half = warp >> 2;
    const uint32_t tm = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint64_t a_q = umma_desc_sw128(smem_u32(sQ), 16, 1024), b_k = umma_desc_sw128(smem_u32(sK), 16, 1024);           // K-major
    const uint64_t a_do = umma_desc_sw128(smem_u32(sdO), 16, 1024), b_v = umma_desc_sw128(smem_u32(sV), 16, 1024);
    const uint64_t t_p = umma_desc_sw128(smem_u32(sP), kTileBytes, 1024), k_p = umma_desc_sw128(smem_u32(sP), 16, 1024);   // transposed; as it is
    const uint64_t t_q = umma_desc_sw128(smem_u32(sQ), kTileBytes, 1024), t_do = umma_desc_sw128(smem_u32(sdO), kTileBytes, 1024), t_k = umma_desc_sw128(smem_u32(sK), kTileBytes, 1024);
    // (The launch before lets this one in once it has waited for its own predecessor, and that for whatever lies before the call; this one reads nothing that they write and
    // writes other rows.)
    if (P.alone) chain_wait();
    chain_release();
    const PlanHead head = plan_head(P.plan);
    if (!head.fits && blockIdx.x == 0 && tid == 0) set_status(P.status, VARDROP_ERR_INVALID_ARG);
    const int first = head.longer, n_items = (head.tiles - first) * P.Hkv;
    bool ok = true;
    uint32_t phase = 0;
    auto wait = [&]() {                                  // for the products behind the last commit
        ok &= mbar_wait(&bar, phase);
        phase ^= 1;
        tc_fence_after();
    };
#pragma unroll 1
    for (int item = blockIdx.x; item < n_items; item += gridDim.x) {
        const int e = item / P.Hkv, kvh = item - e * P.Hkv;
        const int4 entry = __ldg(reinterpret_cast<const int4*>(P.plan.entries() + first + e));
        const int start = entry.x, len = entry.y, steps = (len + 15) >> 4, groups = (len + 31) >> 5;        // of the keys: k-steps of 16, warps' shares of 32
        const long long kv_off = start * P.sTkv + kvh * P.sHkv;
        int heads = 1;                                   // that share a tile
#pragma unroll 1
        for (int g = 0; g < P.group; g += heads) {
            const int h = kvh * P.group + g;
            if (kGrouped) heads = heads_a_tile(len, P.group - g);
            const int n_rows = heads * len, steps_q = (n_rows + 15) >> 4, groups_q = (n_rows + 31) >> 5;
            // tiles of 32-row shares: Q, dO, and at the item's begin K, V; rows up to the next k-step are zeros, those of shares behind it are not read
            const int n_load = 2 * groups_q + (g == 0 ? 2 * groups : 0);
#pragma unroll 1
            for (int x = warp; x < n_load; x += kShortThreads / 32) {
                if (x < 2 * groups_q) {
                    const int tile = x >= groups_q, r0 = (x - tile * groups_q) * 32;
                    const long long sT = tile ? static_cast<long long>(P.Hq) * P.D : P.sTq, sH = tile ? P.D : P.sHq;
                    const __nv_bfloat16* from = tile ? P.d_o + (static_cast<long long>(start) * P.Hq + h) * P.D : P.q + start * P.sTq + h * P.sHq;
                    unsigned char* to = smem_dyn + tile * kTileBytes + r0 * kRowBytes;
                    if (kGrouped && heads > 1) copy_32_packed(to, from, sT, sH, r0, n_rows, len, P.D);
                    else copy_32_tokens(to, from, sT, r0, len, P.D);
                } else {
                    const int y = x - 2 * groups_q, tile = y >= groups, r0 = (y - tile * groups) * 32;
                    copy_32_tokens((tile ? sV : sK) + r0 * kRowBytes, (tile ? P.v : P.k) + kv_off, P.sTkv, r0, len, P.D);
                }
            }
            const PackedRow at = kGrouped && heads > 1 && row < n_rows ? packed_row(row, len) : PackedRow{0, row};
            const float lse = row < n_rows ? __ldg(P.lse + static_cast<size_t>(h + at.head) * P.T + start + at.token) : 0.f, lse2 = lse * 1.4426950408889634f;
            if (lse_too_far(lse)) set_status(P.status, VARDROP_ERR_UNSUPPORTED);
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_proxy_async_smem();
            tc_fence_before();
            __syncthreads();
            if (warp == 0) {
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t idesc = umma_idesc_bf16(128, steps * 16, 0, 0);
#pragma unroll 1
                    for (int ks = 0; ks < P.D / 16; ++ks) tc_mma_bf16(tmem, umma_desc_advance(a_q, ks * 32), umma_desc_advance(b_k, ks * 32), idesc, ks > 0);
#pragma unroll 1
                    for (int ks = 0; ks < P.D / 16; ++ks) tc_mma_bf16(tmem + 128, umma_desc_advance(a_do, ks * 32), umma_desc_advance(b_v, ks * 32), idesc, ks > 0);
                    tc_commit(&bar);
                }
                __syncwarp();
            }
            wait();
            // ---- P, rounded to bf16 for P^T dO and as it is over S; Delta ----
            const int seen = P.causal ? min(len, at.token + 1) : len, c_end = min(half * 64 + 64, steps * 16);        // keys that this row sees; columns of this thread
            float delta = 0.f;
#pragma unroll 1
            for (int c = half * 64; c < c_end; c += 32) {
                float s[32], d[32];
                uint32_t pk[16];
                tmem_ld32(tm + c, s);
                tmem_ld32(tm + 128 + c, d);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const float p = fast_exp2(fmaf(s[i], P.scale_log2, -lse2));
                    s[i] = c + i < seen ? p : 0.f;
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    d[i] = c + i < seen ? d[i] : 0.f;    // (columns behind the keys hold anything)
                    delta = fmaf(s[i], d[i], delta);
                }
#pragma unroll
                for (int i = 0; i < 32; i += 2) pk[i >> 1] = pack_bf16(s[i], s[i + 1]);
                tmem_st32(tm + c, reinterpret_cast<const uint32_t*>(s));
                store_panel(sP + half * kTileBytes, row, (c >> 5) & 1, pk);
            }
            s_delta[half][row] = delta;
            tmem_st_wait();
            fence_proxy_async_smem();
            tc_fence_before();
            ok = __syncthreads_and(ok);
            if (!ok) { item = n_items; break; }          // a wait gave up somewhere in the CTA: stop
            tc_fence_after();
            delta = s_delta[0][row] + s_delta[1][row];
            // ---- dS ----
            uint32_t ds[32];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int c = half * 64 + x * 32;
                if (c < c_end) {
                    float p[32], d[32];
                    tmem_ld32(tm + c, p);
                    tmem_ld32(tm + 128 + c, d);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; i += 2)
                        ds[x * 16 + (i >> 1)] = pack_bf16(c + i < seen ? p[i] * (d[i] - delta) : 0.f, c + i + 1 < seen ? p[i + 1] * (d[i + 1] - delta) : 0.f);
                }
            }
            tc_fence_before();
            __syncthreads();                             // S and dP have been read
            if (warp == 0) {
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t idesc = umma_idesc_bf16(128, P.D, 1, 1);
#pragma unroll 1
                    for (int ks = 0; ks < steps_q; ++ks) tc_mma_bf16(tmem + kDv, umma_desc_advance(t_p, ks * 2048), umma_desc_advance(t_do, ks * 2048), idesc, (kGrouped && g > 0) || ks > 0);
                    tc_commit(&bar);
                }
                __syncwarp();
            }
            wait();                                      // P has been read
#pragma unroll
            for (int x = 0; x < 2; ++x)
                if (half * 64 + x * 32 < c_end) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<uint4*>(sP + half * kTileBytes + row * kRowBytes + (((x * 4 + q) ^ (row & 7)) << 4)) =
                            make_uint4(ds[x * 16 + 4 * q], ds[x * 16 + 4 * q + 1], ds[x * 16 + 4 * q + 2], ds[x * 16 + 4 * q + 3]);
                }
            fence_proxy_async_smem();
            tc_fence_before();
            ok = __syncthreads_and(ok);
            if (!ok) { item = n_items; break; }
            if (warp == 0) {
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t idesc_k = umma_idesc_bf16(128, P.D, 1, 1), idesc_q = umma_idesc_bf16(128, P.D, 0, 1);
#pragma unroll 1
                    for (int ks = 0; ks < steps; ++ks)   // dQ = dS K
                        tc_mma_bf16(tmem + kDq, umma_desc_advance(k_p, (ks >> 2) * kTileBytes + (ks & 3) * 32), umma_desc_advance(t_k, ks * 2048), idesc_q, ks > 0);
#pragma unroll 1
                    for (int ks = 0; ks < steps_q; ++ks) // dK = dS^T Q
                        tc_mma_bf16(tmem + kDk, umma_desc_advance(t_p, ks * 2048), umma_desc_advance(t_q, ks * 2048), idesc_k, (kGrouped && g > 0) || ks > 0);
                    tc_commit(&bar);
                }
                __syncwarp();
            }
            wait();
            // ---- rows out, half of the columns a thread, through tiles that have been read, so that whole rows are written ----
            const bool last = !kGrouped || g + heads == P.group;
            auto stage = [&](unsigned char* tile, uint32_t col, float mul) {
#pragma unroll 1
                for (int c = half * (P.D / 2); c < (half + 1) * (P.D / 2); c += 16) {
                    float v[16];
                    tmem_ld16(tm + col + c, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        *reinterpret_cast<uint4*>(tile + row * kRowBytes + ((((c >> 3) + q) ^ (row & 7)) << 4)) =
                            make_uint4(pack2(v[8 * q] * mul, v[8 * q + 1] * mul), pack2(v[8 * q + 2] * mul, v[8 * q + 3] * mul),
                                       pack2(v[8 * q + 4] * mul, v[8 * q + 5] * mul), pack2(v[8 * q + 6] * mul, v[8 * q + 7] * mul));
                }
            };
            stage(sQ, kDq, P.scale);
            if (last) {
                stage(sdO, kDv, 1.f);
                stage(sP, kDk, P.scale);
            }
            __syncthreads();
            const int sh = P.D > 32 ? 3 : 2, c = tid & ((1 << sh) - 1);
#pragma unroll 2
            for (int r = tid >> sh; r < n_rows; r += kShortThreads >> sh) {
                const PackedRow to = kGrouped && heads > 1 ? packed_row(r, len) : PackedRow{0, r};
                *reinterpret_cast<uint4*>(P.dq + (static_cast<size_t>(start + to.token) * P.Hq + h + to.head) * P.D + c * 8) = *reinterpret_cast<const uint4*>(sQ + r * kRowBytes + ((c ^ (r & 7)) << 4));
            }
            if (last) {
#pragma unroll 2
                for (int r = tid >> sh; r < len; r += kShortThreads >> sh) {
                    const size_t to = (static_cast<size_t>(start + r) * P.Hkv + kvh) * P.D + c * 8;
                    *reinterpret_cast<uint4*>(P.dv + to) = *reinterpret_cast<const uint4*>(sdO + r * kRowBytes + ((c ^ (r & 7)) << 4));
                    *reinterpret_cast<uint4*>(P.dk + to) = *reinterpret_cast<const uint4*>(sP + r * kRowBytes + ((c ^ (r & 7)) << 4));
                }
            }
            tc_fence_before();
            ok = __syncthreads_and(ok);                  // tiles and columns are free
            if (!ok) { item = n_items; break; }
            tc_fence_after();
        }
        if (item == n_items) break;
    }
    if (!ok) set_status(P.status, VARDROP_ERR_TIMEOUT);
    asm volatile("cp.async.wait_all;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, kCols);
    if (!P.alone && tid == 0) chain_wait();              // this launch is the later one to complete
}

// ---------------------------------------------------------------------------------------------------------
// prep
// ---------------------------------------------------------------------------------------------------------
struct PackedPrepParams {
    const uint4* o;         // [T, Hq, D] bf16
    const uint4* d_o;       // [T, Hq, D] bf16
    float* delta;           // [Hq, rows]
    float4* dq_acc;         // [rows, Hq, D] fp32
    PlanView plan;
    int* ticket;
    int Hq, D, rows;
};
// A CTA takes slices of 1024 16-byte chunks of (token, head) rows by turns; the eight (four) threads of a row reduce Delta by shuffles.
__global__ void __launch_bounds__(256) packed_prep_kernel(const PackedPrepParams P) {
    chain_wait();
    chain_release();
    if (blockIdx.x == 0 && threadIdx.x == 0) *P.ticket = 0;
    const int n_tiles = plan_head(P.plan).longer, sh = P.D > 32 ? 3 : 2, chunks_row = P.Hq << sh;
    const int per_tile = kTile * chunks_row, slices = (per_tile + 1023) / 1024;        // four chunks a thread
#pragma unroll 1
    for (long long k = blockIdx.x; k < static_cast<long long>(n_tiles) * slices; k += gridDim.x) {
        const int e = static_cast<int>(k / slices), slice = static_cast<int>(k - static_cast<long long>(e) * slices);
        const int4 x = __ldg(reinterpret_cast<const int4*>(P.plan.entries() + e));
        const int left = x.y - x.z * kTile;
        uint4 vo[4], vd[4];
        int row[4], c[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int idx = slice * 1024 + u * 256 + static_cast<int>(threadIdx.x);
            row[u] = idx < per_tile ? small_div(idx, chunks_row) : kTile;
            c[u] = idx - row[u] * chunks_row;
            vo[u] = vd[u] = make_uint4(0u, 0u, 0u, 0u);
            if (row[u] < left && row[u] < kTile) {
                const size_t src = static_cast<size_t>(x.x + x.z * kTile + row[u]) * chunks_row + c[u];
                vo[u] = __ldg(P.o + src);
                vd[u] = __ldg(P.d_o + src);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float part = dot8(vo[u], vd[u]);
            part += __shfl_xor_sync(0xffffffffu, part, 1);
            part += __shfl_xor_sync(0xffffffffu, part, 2);
            if (sh == 3) part += __shfl_xor_sync(0xffffffffu, part, 4);
            if (row[u] >= kTile) continue;
            const size_t to = static_cast<size_t>(x.w + x.z) * kTile + row[u];
            if ((c[u] & ((1 << sh) - 1)) == 0) P.delta[static_cast<size_t>(c[u] >> sh) * P.rows + to] = part;
            const size_t dst = to * chunks_row + c[u];
            P.dq_acc[2 * dst] = make_float4(0.f, 0.f, 0.f, 0.f);
            P.dq_acc[2 * dst + 1] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------
// main
// ---------------------------------------------------------------------------------------------------------
constexpr int kManyThreads = 896;
// Register split: launched with 896 x 72 = 64512 registers; 128 x 56 + 256 x 64 + 512 x 80 = 64512.
constexpr int kManySmallRegs = 56;
constexpr int kManyOutRegs = 64;
constexpr int kManyBigRegs = 80;
constexpr uint32_t kManyTmemCols = 512;
constexpr int kManyStages = 3;         // ring of (Q, dO) tiles
constexpr int kManyTeamWarps = 8;
constexpr int kManyHeader = 13312;     // barriers, item list, row statistics
constexpr int kManySmemBytes = kManyHeader + 3 * kTileBytes /*K of two items, V*/ + 2 * kManyStages * kTileBytes /*ring*/ + 2 * kTileBytes /*dS^T, two 64-query panels*/ +
                               2 * kTileBytes /*staging: dQ as fp32, two 32-column panels; dV, dK as bf16*/;

// The first 32 bytes (16 bf16) of 128 rows of a swizzled tile to eight columns of tensor memory, row r to lane r: the A operand of a k-step.
__device__ __forceinline__ void tc_copy_128x256b(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.128x256b [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// Shared-memory matrix descriptor without swizzle, K-major: rows of 16 bytes (8 bf16 of K), eight rows in a row; lbo = bytes to the other half of a k-step,
// sbo = bytes between 8-row groups.
__device__ __forceinline__ uint64_t umma_desc_plain(uint32_t smem_addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    return umma_desc_sw128(smem_addr, lbo_bytes, sbo_bytes) & ~(7ull << 61);
}
// x as three bf16 terms (24 bits), each in the low half of a word; one that is not finite as a single one.  (Below 1.7e38 in magnitude no term rounds to infinity.)
__device__ __forceinline__ void split3(float x, uint32_t& a, uint32_t& b, uint32_t& c) {
    const __nv_bfloat16 h = __float2bfloat16_rn(x);
    const float r = fabsf(x) < INFINITY ? x - __bfloat162float(h) : 0.f;
    const __nv_bfloat16 m = __float2bfloat16_rn(r);
    a = __bfloat16_as_ushort(h);
    b = __bfloat16_as_ushort(m);
    c = __bfloat16_as_ushort(__float2bfloat16_rn(r - __bfloat162float(m)));
}
// P^T = exp2(S^T scale) of a thread's 32 queries, in place, and as bf16, in batches of eight; with kMask 0 for those below `from`.
template <bool kMask>
__device__ __forceinline__ void exp_step_folded(float (&s)[32], uint32_t (&pk)[16], uint64_t scale2, int from) {
#pragma unroll
    for (int g = 0; g < 6; ++g) {
        if (g < 4) {
#pragma unroll
            for (int e = 8 * g; e < 8 * g + 8; e += 2) halves_of(mul_pair(pair_of(s[e], s[e + 1]), scale2), s[e], s[e + 1]);
        }
        if (g >= 1 && g < 5) {
#pragma unroll
            for (int e = 8 * g - 8; e < 8 * g; ++e) {
                s[e] = fast_exp2(s[e]);
                if (kMask && e < from) s[e] = 0.f;
            }
        }
        if (g >= 2) {
#pragma unroll
            for (int e = 8 * g - 16; e < 8 * g - 8; e += 2) pk[e >> 1] = pack_bf16(s[e], s[e + 1]);
        }
    }
}
__device__ __forceinline__ bool group_sync_and(int id, bool ok) {     // barrier among a warpgroup, with an and-reduction of ok
    uint32_t r;
    asm volatile(
        "{\n.reg .pred p, q;\n"
        "setp.ne.b32 q, %1, 0;\n"
        "bar.red.and.pred p, %2, 128, q;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(r)
        : "r"(static_cast<uint32_t>(ok)), "r"(id)
        : "memory");
    return r != 0;
}

// An item: two teams of 256 threads share the key tile; team w takes the queries 64 w to 64 w + 63 of every query tile.
//   warp 0       issues S^T = K Q^T and dV += P^T dO of both teams
//   warp 1       issues dP^T = V dO^T and dK += dS^T Q of both teams
//   warp 2       issues dQ = dS K of a query tile; copies K and V of the next item to tensor memory
//   warp 3       decodes the items; loads K, V of the items and a ring of (Q, dO) tiles with their row statistics
//   warps 4-7    columns 0 to 31 of dQ into the accumulator; dV of a finished item
//   warps 8-11   columns 32 to 63; dK of a finished item
//   warps 12-19  team 0, warps 20-27  team 1: two threads a key row, 32 queries each
// Tensor memory: K 32 | V 32 | dV 64 | dK 64 | dQ 64 | team 0: S^T, P^T 64, dP^T, dS^T 64 | team 1.
constexpr uint32_t kColK = 0, kColV = 32, kColDv = 64, kColDk = 128, kColDq = 192, kColTeam = 256;

__global__ void __launch_bounds__(kManyThreads, 1) attn_packed_bwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                                           const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do,
                                                                           const __grid_constant__ CUtensorMap map_acc, const __grid_constant__ CUtensorMap map_parts,
                                                                           const PackedBwdParams P) {
    extern __shared__ __align__(1024) unsigned char smem_dyn[];      // (every address below is a constant then: no registers)
    // Set-up first: it touches nothing another kernel produces, so it runs while the previous kernel of the stream is still finishing.
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem_dyn);
    uint64_t* bar_k_full = bars;                    // [2] K of an item in shared memory
    uint64_t* bar_k_free = bars + 2;                // [2] its last dQ is done
    uint64_t* bar_v_full = bars + 4;                // V of an item in shared memory
    uint64_t* bar_v_free = bars + 5;                // and in tensor memory
    uint64_t* bar_q_full = bars + 6;                // [kManyStages] slot holds a query tile and its statistics
    uint64_t* bar_q_free = bars + 9;                // [kManyStages] every product reading the slot is done (both issuing warps)
    uint64_t* bar_s = bars + 12;                    // [2] S^T of team w's step complete
    uint64_t* bar_dp = bars + 14;                   // [2] dP^T
    uint64_t* bar_p = bars + 16;                    // [2] P^T in tensor memory
    uint64_t* bar_ds = bars + 18;                   // [2] dS^T in tensor memory
    uint64_t* bar_g = bars + 20;                    // dQ of a query tile complete
    uint64_t* bar_dv_done = bars + 21;              // dV of an item complete
    uint64_t* bar_dv_free = bars + 22;              // and in registers
    uint64_t* bar_dk_done = bars + 23;
    uint64_t* bar_dk_free = bars + 24;
    uint64_t* bar_gfree = bars + 25;                // dQ of a query tile in registers
    uint64_t* bar_panel = bars + 26;                // [2] dS^T in shared memory
    uint64_t* bar_kv = bars + 28;                   // [2] K, V of an item in tensor memory
    uint64_t* bar_item = bars + 30;                 // [8] entry of the item list is written
    uint64_t* bar_left = bars + 39;                 // [3] what an issuing warp whose wait gave up has issued is done
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 38);
    // Key tile jt of a sequence and a key head (kvh: that, and 4096 (1 + part) for one of several parts).  steps: query tiles from the s0-th on of those of all its query heads,
    // `per` of each, which end with the sequence; len < 0 ends the list.
    struct alignas(16) Item { int start, len, jt, kvh, base, steps, per, s0; };
    Item* s_item = reinterpret_cast<Item*>(smem_dyn + 512);         // [8]
    uint4* s_ones = reinterpret_cast<uint4*>(smem_dyn + 768);       // [8] bf16 rows of three ones
    uint4* s_stats = s_ones + 8;                                    // [2][kManyStages][128] three bf16 terms of half of -lse / scale, of half of -Delta, of the slot's rows
    static_assert(42 * 8 <= 512 && 8 * sizeof(Item) <= 256 && 768 + (8 + 2 * kManyStages * kTile) * sizeof(uint4) <= kManyHeader, "header too small");
    unsigned char* sK = smem_dyn + kManyHeader;                     // K of two items
    unsigned char* sV = sK + 2 * kTileBytes;
    unsigned char* sQ = sV + kTileBytes;                            // slots of (Q tile, dO tile)
    unsigned char* sdS = sQ + 2 * kManyStages * kTileBytes;         // dS^T: rows = keys, a 64-query panel of each team
    unsigned char* sOut = sdS + 2 * kTileBytes;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (smem_u32(smem_dyn) & 1023u) {
        chain_wait();
        if (tid == 0) set_status(P.status, VARDROP_ERR_CUDA);
        return;
    }
    if (warp == 0) {
        tmem_alloc(tmem_slot, kManyTmemCols);
        tmem_relinquish();
    }
    if (tid == 0) {
        for (int w = 0; w < 2; ++w) {
            mbar_init(bar_k_full + w, 1);
            mbar_init(bar_k_free + w, 1);
            mbar_init(bar_s + w, 1);
            mbar_init(bar_dp + w, 1);
            mbar_init(bar_p + w, kManyTeamWarps);
            mbar_init(bar_ds + w, kManyTeamWarps);
            mbar_init(bar_panel + w, kManyTeamWarps);
            mbar_init(bar_kv + w, 1);
        }
        mbar_init(bar_v_full, 1);
        mbar_init(bar_v_free, 1);
        for (int s = 0; s < kManyStages; ++s) {
            mbar_init(bar_q_full + s, 2);                     // the boxes' announcing arrival, the statistics
            mbar_init(bar_q_free + s, 2);
        }
        mbar_init(bar_g, 1);
        mbar_init(bar_dv_done, 1);
        mbar_init(bar_dv_free, 4);
        mbar_init(bar_dk_done, 1);
        mbar_init(bar_dk_free, 4);
        mbar_init(bar_gfree, 8);
        for (int i = 0; i < 8; ++i) mbar_init(bar_item + i, 1);
        for (int w = 0; w < 3; ++w) mbar_init(bar_left + w, 1);
        mbar_fence_init();
        tma_prefetch_desc(&map_q);
        tma_prefetch_desc(&map_do);
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
        tma_prefetch_desc(&map_acc);
        if (P.may_split) tma_prefetch_desc(&map_parts);
    }
    if (tid < 8) s_ones[tid] = make_uint4(0x3f803f80u, 0x00003f80u, 0u, 0u);
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    auto begin = [&]() {
        chain_wait();
        chain_release();
    };
    auto item_wait = [&](uint32_t i) { ok &= warp_wait_relaxed(bar_item + (i & 7), (i >> 3) & 1); };
    auto item_read = [&](uint32_t i) {
        const int4* from = reinterpret_cast<const int4*>(s_item + (i & 7));
        const int4 x = from[0], y = from[1];
        return Item{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    };
    auto item_at = [&](uint32_t i) {                           // len -1 for an item that did not come
        item_wait(i);
        Item it = item_read(i);
        if (!ok) it.len = -1;
        return it;
    };
    auto warp_arrive = [&](uint64_t* bar) {                    // all lanes are done
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    };
    auto next_slot = [](uint32_t& st, uint32_t& ph) {
        if (++st == kManyStages) { st = 0; ph ^= 1; }
    };

    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kManySmallRegs));
    begin();
    if (warp < 2) {
        // ------------------------------------------------------------ issue ---------------------------------------------
        // Warp 0: S^T from K and Q, dV from P^T and dO.  Warp 1: dP^T from V and dO, dK from dS^T and Q.  One body: `first` is the product that opens a
        // step, `second` the one that adds up.
        const uint32_t idesc_first = umma_idesc_bf16(128, 64, 0, 0), idesc_second = umma_idesc_bf16(128, P.D, 0, 1);
        const uint64_t d_q = umma_desc_sw128(smem_u32(sQ) + (warp == 0 ? 0 : kTileBytes), 16, 1024);                 // operand of the first product
        const uint64_t m_q = umma_desc_sw128(smem_u32(sQ) + (warp == 0 ? kTileBytes : 0), kTileBytes, 1024);         // of the second
        const uint32_t c_kv = tmem + (warp == 0 ? kColK : kColV), c_acc = tmem + (warp == 0 ? kColDv : kColDk), c_team = tmem + kColTeam + warp * 64;
        // A k-step is two rows of eight: both are the same one, whence the halves.
        const uint64_t d_ones = umma_desc_plain(smem_u32(s_ones), 0, 0), d_stats = umma_desc_plain(smem_u32(s_stats + warp * kManyStages * kTile), 0, 128);
        uint64_t* bar_first = warp == 0 ? bar_s : bar_dp;
        uint64_t* bar_handed = warp == 0 ? bar_p : bar_ds;
        uint64_t* bar_done = warp == 0 ? bar_dv_done : bar_dk_done;
        uint64_t* bar_free = warp == 0 ? bar_dv_free : bar_dk_free;
        uint32_t t = 0, st = 0, ph = 0, sn = 0, pn = 0;        // query tiles so far, their slot; slot of the tile whose first products come next
        auto wait_slot = [&]() {
            ok &= warp_wait_relaxed(bar_q_full + sn, pn);
            tc_fence_after();
        };
        auto first = [&](int w) {
            if (elect_one()) {
                const uint64_t bd = umma_desc_advance(d_q, sn * 2 * kTileBytes + w * 64 * kRowBytes);
                const uint32_t to = c_team + w * 128;
                tc_mma_bf16_ta(to, c_kv, bd, idesc_first, 0u);
                tc_mma_bf16_ta(to, c_kv + 8, umma_desc_advance(bd, 32), idesc_first, 1u);
                if (P.D > 32) {
                    tc_mma_bf16_ta(to, c_kv + 16, umma_desc_advance(bd, 64), idesc_first, 1u);
                    tc_mma_bf16_ta(to, c_kv + 24, umma_desc_advance(bd, 96), idesc_first, 1u);
                }
                tc_mma_bf16(to, d_ones, umma_desc_advance(d_stats, (sn * kTile + w * 64) * 16), idesc_first, 1u);
                tc_commit(bar_first + w);
            }
            __syncwarp();
        };
        Item it = item_at(0);
        if (it.len >= 0) {
            ok &= warp_wait(bar_kv + warp, 0);
            wait_slot();
            first(0);
            first(1);
            next_slot(sn, pn);
        }
#pragma unroll 1
        for (uint32_t i = 0; ok && it.len >= 0; ++i) {
            const int n_q = it.steps;
#pragma unroll 1
            for (int x = 0; x < n_q && ok; ++x, ++t) {
                const bool last = x + 1 == n_q;
                bool more = true;
#pragma unroll 1
                for (int w = 0; w < 2; ++w) {
                    ok &= warp_wait(bar_handed + w, t & 1);
                    if (i > 0 && x + w == 0) ok &= warp_wait(bar_free, (i - 1) & 1);       // the previous item's sum is out
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t bd = umma_desc_advance(m_q, st * 2 * kTileBytes + w * 64 * kRowBytes);
                        const uint32_t a = c_team + w * 128;
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            tc_mma_bf16_ta(c_acc, a + (ks >> 1) * 32 + (ks & 1) * 8, umma_desc_advance(bd, ks * 2048), idesc_second, ks > 0 ? 1u : (x + w > 0 ? 1u : 0u));
                        if (w == 1) {
                            tc_commit(bar_q_free + st);
                            if (last) tc_commit(bar_done);
                        }
                    }
                    __syncwarp();
                    if (last && w == 0) {                // (an item comes when the loads of the one before have been issued)
                        it = item_at(i + 1);
                        more = it.len >= 0;
                    }
                    if (!more) continue;
                    if (w == 0) {
                        if (last) ok &= warp_wait(bar_kv + warp, (i + 1) & 1);
                        wait_slot();
                    }
                    first(w);
                }
                if (more) next_slot(sn, pn);
                next_slot(st, ph);
            }
        }
    } else if (warp == 2) {
        const uint32_t idesc_mnmn = umma_idesc_bf16(128, P.D, 1, 1);       // A MN-major, B MN-major
        const uint64_t a_ds = umma_desc_sw128(smem_u32(sdS), kTileBytes, 1024), b_k = umma_desc_sw128(smem_u32(sK), kTileBytes, 1024);
        const uint64_t k_from = umma_desc_sw128(smem_u32(sK), 16, 1024), v_from = umma_desc_sw128(smem_u32(sV), 16, 1024);
        auto copy_kv = [&](uint32_t i, bool v) {               // an item's K or V to tensor memory
            ok &= v ? warp_wait_relaxed(bar_v_full, i & 1) : warp_wait_relaxed(bar_k_full + (i & 1), (i >> 1) & 1);
            tc_fence_after();
            if (elect_one()) {
                const uint64_t from = v ? v_from : umma_desc_advance(k_from, (i & 1) * kTileBytes);
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    if (ks < 2 || P.D > 32) tc_copy_128x256b(tmem + (v ? kColV : kColK) + ks * 8, umma_desc_advance(from, ks * 32));
                tc_commit(bar_kv + (v ? 1 : 0));
                if (v) tc_commit(bar_v_free);
            }
            __syncwarp();
        };
        uint32_t t = 0;
        Item it = item_at(0);
        if (it.len >= 0) {
            copy_kv(0, false);
            copy_kv(0, true);
        }
#pragma unroll 1
        for (uint32_t i = 0; ok && it.len >= 0; ++i) {
            const int n_q = it.steps;
            const uint64_t bk = umma_desc_advance(b_k, (i & 1) * kTileBytes);
#pragma unroll 1
            for (int x = 0; x < n_q && ok; ++x, ++t) {
                if (x + 1 == n_q) it = item_at(i + 1);
                if (x + 1 == n_q && it.len >= 0) {           // the last products that read this K (V) are both teams' first ones of this tile
                    ok &= warp_wait(bar_s + 1, t & 1);
                    copy_kv(i + 1, false);
                    ok &= warp_wait(bar_dp + 1, t & 1);
                    copy_kv(i + 1, true);
                }
                if (t > 0) ok &= warp_wait_relaxed(bar_gfree, (t - 1) & 1);
                ok &= warp_wait(bar_panel, t & 1);
                ok &= warp_wait(bar_panel + 1, t & 1);
                tc_fence_after();
                if (elect_one()) {                       // dQ = dS K, dS the transposed view of dS^T
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        tc_mma_bf16(tmem + kColDq, umma_desc_advance(a_ds, ks * 2048), umma_desc_advance(bk, ks * 2048), idesc_mnmn, ks > 0 ? 1u : 0u);
                    tc_commit(bar_g);
                    if (x + 1 == n_q) tc_commit(bar_k_free + (i & 1));
                }
                __syncwarp();
            }
        }
    } else {
        // ------------------------------------------------------------ loads, items --------------------------------------
        const PlanHead head = plan_head(P.plan);
        const Split split = split_of(P.plan, head, P.group, P.Hkv, gridDim.x, P.may_split);
        const int units = P.Hkv * split.parts;                 // of a plan entry
        const long long n_items = static_cast<long long>(head.longer) * units;
        // (Every SM takes items, though packed_short_kernel comes next: SMs left to it by the share of its work made 26 of 37 batches 0.5 to 3 % slower, three 0.4 to 3 % faster.)
        const int ctas = gridDim.x;
        auto publish = [&](uint32_t i, long long k) {
            Item it{0, -1, 0, 0, 0, 0, 0, 0};
#pragma unroll 1
            for (; k < n_items; k = next_item(P.status + kWsTicketBwd, ctas, lane)) {
                const int e = static_cast<int>(k / units), unit = static_cast<int>(k - static_cast<long long>(e) * units), kvh = small_div(unit, split.parts), part = unit - kvh * split.parts;
                const int4 x = __ldg(reinterpret_cast<const int4*>(P.plan.entries() + e));
                const int n_t = (x.y + kTile - 1) / kTile, jt = P.causal ? n_t - 1 - x.z : x.z, per = P.causal ? n_t - jt : n_t, steps = per * P.group;
                const int parts = parts_of(steps, split), share = (steps + parts - 1) / parts;
                if (part * share >= steps) continue;           // an entry of fewer parts
                it.start = x.x; it.len = x.y; it.base = x.w;
                it.jt = jt; it.per = per;
                it.kvh = kvh + (parts > 1 ? (1 + part) << 12 : 0);
                it.s0 = part * share;
                it.steps = min(share, steps - it.s0);
                break;
            }
            if (lane == 0) {
                int4* to = reinterpret_cast<int4*>(s_item + (i & 7));
                to[0] = make_int4(it.start, it.len, it.jt, it.kvh);
                to[1] = make_int4(it.base, it.steps, it.per, it.s0);
                mbar_arrive(bar_item + (i & 7));
            }
            __syncwarp();
        };
        // A tile of a head as rows, where the sequence ends inside: zeros behind its end (the next sequence's rows lie there, and what is zero times something not finite is not
        // zero).  The copies are waited for and made visible to the tensor core here, so that whoever waits for the tile need not know how it came.
        auto rows_to = [&](unsigned char* to, const __nv_bfloat16* from, long long sT, int tok0, int len) {
#pragma unroll 1
            for (int g = 0; g < 4; ++g) copy_32_tokens(to + g * 32 * kRowBytes, from, sT, tok0 + g * 32, len, P.D);
        };
        auto rows_done = [&]() {
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_proxy_async_smem();
            __syncwarp();
        };
        auto load_kv = [&](uint32_t i, const Item& it) {
            ok &= warp_wait_relaxed(bar_k_free + (i & 1), ((i >> 1) & 1) ^ 1);
            ok &= warp_wait_relaxed(bar_v_free, (i & 1) ^ 1);
            if (!ok) return;
            unsigned char* to = sK + (i & 1) * kTileBytes;
            const int kvh = it.kvh & 4095;
            if ((it.jt + 1) * kTile <= it.len) {
                if (lane == 0) {
                    mbar_expect_tx(bar_k_full + (i & 1), kTileBytes);
                    tma_load_3d(to, &map_k, bar_k_full + (i & 1), 0, kvh, it.start + it.jt * kTile);
                    mbar_expect_tx(bar_v_full, kTileBytes);
                    tma_load_3d(sV, &map_v, bar_v_full, 0, kvh, it.start + it.jt * kTile);
                }
            } else {
                const long long off = it.start * P.sTkv + kvh * P.sHkv;
                rows_to(to, P.k + off, P.sTkv, it.jt * kTile, it.len);
                rows_to(sV, P.v + off, P.sTkv, it.jt * kTile, it.len);
                rows_done();
                if (lane == 0) {
                    mbar_arrive(bar_k_full + (i & 1));
                    mbar_arrive(bar_v_full);
                }
            }
            __syncwarp();
        };
        uint32_t st = 0, ph = 0;
        bool too_far = false;
        publish(0, blockIdx.x);
        Item next = item_at(0);
        if (next.len >= 0) load_kv(0, next);
#pragma unroll 1
        for (uint32_t i = 0; ok; ++i) {
            const Item it = next;
            if (it.len < 0) break;
            const int n_q = it.steps, x0 = (it.len + kTile - 1) / kTile - it.per;
            int h = (it.kvh & 4095) * P.group + small_div(it.s0, it.per), x = x0 + it.s0 - small_div(it.s0, it.per) * it.per;            // of the step
            // Row statistics of a query tile travel with it, four rows a lane; those of the next tile are asked for ahead of the wait for this one's slot.
            float st_lse[4], st_delta[4];
            auto stats_load = [&](int h, int x) {
                const float* lse_row = P.lse + static_cast<size_t>(h) * P.T + it.start;
                const float* delta_row = P.delta + static_cast<size_t>(h) * P.rows + static_cast<size_t>(it.base) * kTile;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = x * kTile + e * 32 + lane;
                    st_lse[e] = r < it.len ? __ldg(lse_row + r) : 0.f;       // (missing queries have zero rows of Q and dO: any P will do)
                    st_delta[e] = r < it.len ? __ldg(delta_row + r) : 0.f;
                }
            };
            stats_load(h, x);
#pragma unroll 1
            for (int s = 0; s < n_q; ++s) {
                ok &= warp_wait_relaxed(bar_q_free + st, ph ^ 1);
                if (!ok) break;
                unsigned char* to = sQ + st * 2 * kTileBytes;
                const bool whole = (x + 1) * kTile <= it.len;
                if (whole) {                             // the tiles first: the products wait for them a step ahead of anything the statistics are for
                    if (lane == 0) {
                        mbar_expect_tx(bar_q_full + st, 2 * kTileBytes);
                        tma_load_3d(to, &map_q, bar_q_full + st, 0, h, it.start + x * kTile);
                        tma_load_3d(to + kTileBytes, &map_do, bar_q_full + st, 0, h, it.start + x * kTile);
                    }
                } else {
                    rows_to(to, P.q + it.start * P.sTq + h * P.sHq, P.sTq, x * kTile, it.len);
                    rows_to(to + kTileBytes, P.d_o + (static_cast<long long>(it.start) * P.Hq + h) * P.D, static_cast<long long>(P.Hq) * P.D, x * kTile, it.len);
                    rows_done();
                    if (lane == 0) mbar_arrive(bar_q_full + st);
                }
                __syncwarp();
                if (x == it.jt) {                        // one look at every query tile of a head
#pragma unroll
                    for (int e = 0; e < 4; ++e) too_far |= lse_too_far(st_lse[e]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t l[3], d[3];
                    split3(-st_lse[e] * P.half_inv_scale, l[0], l[1], l[2]);
                    split3(-0.5f * st_delta[e], d[0], d[1], d[2]);
                    s_stats[st * kTile + e * 32 + lane] = make_uint4(l[0] | l[1] << 16, l[2], 0u, 0u);
                    s_stats[(kManyStages + st) * kTile + e * 32 + lane] = make_uint4(d[0] | d[1] << 16, d[2], 0u, 0u);
                }
                fence_proxy_async_smem();
                warp_arrive(bar_q_full + st);
                if (++x == x0 + it.per) { x = x0; ++h; }
                if (s + 1 < n_q) stats_load(h, x);
                next_slot(st, ph);
            }
            if (!ok) break;
            publish(i + 1, n_items > ctas ? next_item(P.status + kWsTicketBwd, ctas, lane) : n_items);
            next = item_at(i + 1);
            if (next.len >= 0) load_kv(i + 1, next);
        }
        if (too_far) set_status(P.status, VARDROP_ERR_UNSUPPORTED);
    }
    } else if (warp < 12) {
        // ------------------------------------------------------------ dQ; dV, dK of an item -----------------------------
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kManyOutRegs));
        begin();
        const int g = (warp >> 2) - 1, id = 1 + g, row = tid & (kTile - 1);
        const uint32_t tm = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const bool owner = row == 0, columns = g * 32 < P.D;     // the one thread of the warpgroup that owns its bulk reductions; there are such columns
        unsigned char* panel = sOut + g * kTileBytes;            // this warpgroup's staging panel of 128-byte swizzled rows
        unsigned char* rowp = panel + row * kRowBytes;
        auto panel_free = [&]() {
            if (owner) bulk_wait_group_read0();
            ok = group_sync_and(id, ok);
        };
        // Nothing bounds a named barrier.  A warp whose wait gave up goes on to the last barrier of its query tile, where all four learn of it, and all leave there: no
        // other exit but the end of the list, which all see, since each waits for the entry of the next item ahead of that barrier.
        item_wait(0);
        ok = group_sync_and(id, ok);
        uint32_t t = 0;
#pragma unroll 1
        for (uint32_t i = 0; ok; ++i) {
            const Item it = item_read(i);
            if (it.len < 0) break;
            const int n_q = it.steps;
            // dV or dK of the item's keys: a warp's 32 rows through its part of the panel, eight lanes a row
            auto rows_out = [&](uint32_t col, uint64_t* done, uint64_t* freed, float mul, __nv_bfloat16* dst) {
                if (it.kvh >= 4096) {                    // one of several parts: as fp32, the panel's 32 columns at a time
#pragma unroll 1
                    for (int c = 0; c < P.D; c += 32) {
                        panel_free();
                        if (c == 0) {
                            ok &= warp_wait_relaxed(done, i & 1);
                            tc_fence_after();
                        }
                        float v[32];
                        tmem_ld32(tm + col + c, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            *reinterpret_cast<float4*>(rowp + ((e ^ (row & 7)) << 4)) = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                        fence_proxy_async_smem();
                        if (c + 32 >= P.D) {
                            tc_fence_before();
                            warp_arrive(freed);
                        }
                        ok = group_sync_and(id, ok);
                        if (owner) {
                            tma_store_3d(&map_parts, panel, c, (g * kMostParts + (it.kvh >> 12) - 1) * P.Hkv + (it.kvh & 4095), (it.base + it.jt) * kTile);
                            bulk_commit_group();
                        }
                    }
                    return;
                }
                panel_free();
                ok &= warp_wait_relaxed(done, i & 1);
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < P.D; c += 32) {
                    float v[32];
                    tmem_ld32(tm + col + c, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<uint4*>(rowp + (((c / 8 + q) ^ (row & 7)) << 4)) =
                            make_uint4(pack2(v[8 * q + 0] * mul, v[8 * q + 1] * mul), pack2(v[8 * q + 2] * mul, v[8 * q + 3] * mul),
                                       pack2(v[8 * q + 4] * mul, v[8 * q + 5] * mul), pack2(v[8 * q + 6] * mul, v[8 * q + 7] * mul));
                }
                tc_fence_before();
                warp_arrive(freed);                      // the next item's products wait for these columns
                const int c8 = lane & 7;
                if (c8 * 8 < P.D) {
                    const int row0 = it.jt * kTile + (warp & 3) * 32 + (lane >> 3), left = it.len - row0;         // rows 4 apart, as long as they exist
                    __nv_bfloat16* out = dst + (static_cast<size_t>(it.start + row0) * P.Hkv + (it.kvh & 4095)) * P.D + c8 * 8;
                    const unsigned char* from = panel + ((warp & 3) * 32 + (lane >> 3)) * kRowBytes;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (4 * e < left)
                            *reinterpret_cast<uint4*>(out + static_cast<size_t>(4 * e) * P.Hkv * P.D) =
                                *reinterpret_cast<const uint4*>(from + 4 * e * kRowBytes + ((c8 ^ ((4 * e + (lane >> 3)) & 7)) << 4));
                }
            };
            const int x0 = (it.len + kTile - 1) / kTile - it.per;
            const int g0 = small_div(it.s0, it.per);
            int h = (it.kvh & 4095) * P.group + g0, at = x0 + it.s0 - g0 * it.per;           // of the step
            int x = 0;
#pragma unroll 1
            do {
                if (x + 1 == n_q) {                      // complete ahead of the item's last dQ, and about when it is
                    if (g == 0) rows_out(kColDv, bar_dv_done, bar_dv_free, 1.f, P.dv);
                    else rows_out(kColDk, bar_dk_done, bar_dk_free, P.scale, P.dk);
                }
                panel_free();
                ok &= warp_wait_relaxed(bar_g, t & 1);
                tc_fence_after();
                if (columns) {
                    float v[32];
                    tmem_ld32(tm + kColDq + g * 32, v);
                    tmem_ld_wait();
                    tc_fence_before();
                    warp_arrive(bar_gfree);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        *reinterpret_cast<float4*>(rowp + ((e ^ (row & 7)) << 4)) = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                    fence_proxy_async_smem();
                } else {
                    warp_arrive(bar_gfree);
                }
                if (x + 1 == n_q) item_wait(i + 1);  // (behind the hand-off that the next dQ waits for)
                ok = group_sync_and(id, ok);             // the panel is complete
                if (owner && columns) {
                    tma_reduce_add_3d(&map_acc, panel, g * 32, h, (it.base + at) * kTile);
                    bulk_commit_group();
                }
                if (++at == x0 + it.per) { at = x0; ++h; }
                ++t;
            } while (++x < n_q && ok);
        }
        if (owner) bulk_wait_group0();                   // the last reductions of dQ have landed
    } else {
        // ------------------------------------------------------------ teams ---------------------------------------------
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyBigRegs));
        begin();
        const int w = (warp - 12) >> 3, row = tid & (kTile - 1), half = ((warp - 12) >> 2) & 1;
        const uint32_t tm_s = tmem + kColTeam + w * 128 + half * 32 + (static_cast<uint32_t>((warp & 3) * 32) << 16), tm_d = tm_s + 64;
        unsigned char* panel = sdS + w * kTileBytes;
        uint32_t t = 0;
        bool s_ready = false;                            // a poll takes a hundred cycles to answer: polls go out ahead of where they are needed
#pragma unroll 1
        for (uint32_t i = 0; ok; ++i) {
            const Item it = item_at(i);
            if (it.len < 0) break;
            const int n_q = it.steps;
            // Rows of keys that do not exist are zeros and their dV, dK go nowhere; P^T = 1 keeps what they add to dQ at zero.
            const float scale = it.jt * kTile + row < it.len ? P.scale_log2 : 0.f;
            const uint64_t scale2 = pair_of(scale, scale);
            // step of the next query tile on the diagonal: the first of every head
            int diagonal = -1;
            if (P.causal) {
                const int into = it.s0 - small_div(it.s0, it.per) * it.per;
                diagonal = into == 0 ? 0 : it.per - into;
            }
#pragma unroll 1
            for (int x = 0; x < n_q && ok; ++x, ++t) {
                if (!__all_sync(0xffffffffu, s_ready)) ok &= warp_wait(bar_s + w, t & 1);
                tc_fence_after();
                float s[32], d[32];
                uint32_t pk[16];
                tmem_ld32(tm_s, s);
                tmem_ld_wait();
                if (x == diagonal) {                     // query first + e sees key `row` from e = row - first on
                    diagonal += it.per;
                    exp_step_folded<true>(s, pk, scale2, row - (w * 64 + half * 32));
                } else {
                    exp_step_folded<false>(s, pk, scale2, 0);
                }
                const bool dp_ready = mbar_test(bar_dp + w, t & 1);
                tmem_st16(tm_s, pk);
                tmem_st_wait();
                tc_fence_before();
                warp_arrive(bar_p + w);                  // dV may go, and the next S^T over P^T behind it
                if (!__all_sync(0xffffffffu, dp_ready)) ok &= warp_wait(bar_dp + w, t & 1);
                tc_fence_after();
                tmem_ld32(tm_d, d);
                const bool g_done = t == 0 || mbar_test(bar_g, (t - 1) & 1);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; e += 2) {        // dP^T has -Delta in it
                    halves_of(mul_pair(pair_of(s[e], s[e + 1]), pair_of(d[e], d[e + 1])), d[e], d[e + 1]);
                    pk[e >> 1] = pack_bf16(d[e], d[e + 1]);
                }
                tmem_st16(tm_d, pk);
                tmem_st_wait();
                tc_fence_before();
                warp_arrive(bar_ds + w);                 // dK may go, the next dP^T over dS^T behind it
                if (!__all_sync(0xffffffffu, g_done)) ok &= warp_wait(bar_g, (t - 1) & 1);   // dQ of the previous tile has read the panels
                store_panel(panel, row, half, pk);
                s_ready = mbar_test(bar_s + w, (t + 1) & 1);
                fence_proxy_async_smem();
                warp_arrive(bar_panel + w);              // and dQ
            }
        }
    }
    if (!ok) {
        set_status(P.status, VARDROP_ERR_TIMEOUT);
        if (warp < 3) {                                  // what it has issued is done before tensor memory is given back
            tc_commit_w(bar_left + warp);
            warp_wait(bar_left + warp, 0);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, kManyTmemCols);
}

// ---------------------------------------------------------------------------------------------------------
// dq from the accumulator
// ---------------------------------------------------------------------------------------------------------
struct PackedConvertParams {
    const float4* dq_acc;    // [rows, Hq, D] fp32
    uint4* dq;               // [T, Hq, D] bf16
    const float4* parts;     // [rows, (dV, dK), part, Hkv, D] fp32
    uint4 *dv, *dk;          // [T, Hkv, D] bf16
    PlanView plan;
    int Hq, Hkv, group, D, causal, may_split, main_grid;
    float scale;
};
__global__ void __launch_bounds__(256) packed_convert_kernel(const PackedConvertParams P) {
    chain_wait();
    chain_release();
    const PlanHead head = plan_head(P.plan);
    const int n_tiles = head.longer, sh = P.D > 32 ? 3 : 2, chunks_row = P.Hq << sh;        // 16-byte results per row
    const int per_tile = kTile * chunks_row, slices = (per_tile + 1023) / 1024;
    for (long long k = blockIdx.x; k < static_cast<long long>(n_tiles) * slices; k += gridDim.x) {
        const int e = static_cast<int>(k / slices), slice = static_cast<int>(k - static_cast<long long>(e) * slices);
        const int4 x = __ldg(reinterpret_cast<const int4*>(P.plan.entries() + e));
        const int there = min(kTile, x.y - x.z * kTile) * chunks_row;
        float4 a[4][2];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int idx = slice * 1024 + u * 256 + static_cast<int>(threadIdx.x);
            if (idx >= there) continue;
            const int row = small_div(idx, chunks_row), c = idx - row * chunks_row;
            const float4* src = P.dq_acc + ((static_cast<size_t>(x.w + x.z) * kTile + row) * chunks_row + c) * 2;
            a[u][0] = __ldcg(src);
            a[u][1] = __ldcg(src + 1);
        }
        uint4* to = P.dq + static_cast<size_t>(x.x + x.z * kTile) * chunks_row;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int idx = slice * 1024 + u * 256 + static_cast<int>(threadIdx.x);
            if (idx < there)
                to[idx] = make_uint4(pack2(a[u][0].x * P.scale, a[u][0].y * P.scale), pack2(a[u][0].z * P.scale, a[u][0].w * P.scale),
                                     pack2(a[u][1].x * P.scale, a[u][1].y * P.scale), pack2(a[u][1].z * P.scale, a[u][1].w * P.scale));
        }
    }
    // dV and dK of key tiles that were worked off in parts, which are added up in their order
    const Split split = split_of(P.plan, head, P.group, P.Hkv, P.main_grid, P.may_split);
    if (split.parts == 1) return;
    const int kv_row = P.Hkv << sh, kv_tile = 2 * kTile * kv_row, kv_slices = (kv_tile + 255) / 256;
    for (long long k = blockIdx.x; k < static_cast<long long>(n_tiles) * kv_slices; k += gridDim.x) {
        const int e = static_cast<int>(k / kv_slices), slice = static_cast<int>(k - static_cast<long long>(e) * kv_slices);
        const int4 x = __ldg(reinterpret_cast<const int4*>(P.plan.entries() + e));
        const int n_t = (x.y + kTile - 1) / kTile, jt = P.causal ? n_t - 1 - x.z : x.z, parts = parts_of((P.causal ? n_t - jt : n_t) * P.group, split);
        if (parts == 1) break;               // entries come with the most work first
        const int idx = slice * 256 + static_cast<int>(threadIdx.x), which = idx >= kTile * kv_row ? 1 : 0, in = idx - which * kTile * kv_row;
        const int row = small_div(in, kv_row), c = in - row * kv_row;
        if (idx >= kv_tile || row >= x.y - jt * kTile) continue;
        const float4* src = P.parts + (((static_cast<size_t>(x.w + jt) * kTile + row) * 2 + which) * kMostParts * kv_row + c) * 2;
        float4 a = __ldcg(src), b = __ldcg(src + 1);
        for (int p = 1; p < parts; ++p) {
            src += 2 * kv_row;
            const float4 f = __ldcg(src), g = __ldcg(src + 1);
            a.x += f.x; a.y += f.y; a.z += f.z; a.w += f.w;
            b.x += g.x; b.y += g.y; b.z += g.z; b.w += g.w;
        }
        const float mul = which ? P.scale : 1.f;
        (which ? P.dk : P.dv)[static_cast<size_t>(x.x + jt * kTile + row) * kv_row + c] =
            make_uint4(pack2(a.x * mul, a.y * mul), pack2(a.z * mul, a.w * mul), pack2(b.x * mul, b.y * mul), pack2(b.z * mul, b.w * mul));
    }
}

}  // namespace

int attn_packed_bwd_launch(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* d_o, const void* plan, const vardrop_packed_cfg& c, void* dq,
                           void* dk, void* dv, void* ws, cudaStream_t stream) {
    const PackedWs w = packed_layout(c);
    const PackedStrides L = packed_strides(c);
    char* base = static_cast<char*>(ws);
    const long long HD = static_cast<long long>(c.Hq) * c.D;
    PackedBwdParams P{};
    P.q = static_cast<const __nv_bfloat16*>(q); P.k = static_cast<const __nv_bfloat16*>(k); P.v = static_cast<const __nv_bfloat16*>(v);
    P.d_o = static_cast<const __nv_bfloat16*>(d_o);
    P.lse = lse; P.delta = reinterpret_cast<const float*>(base + w.delta);
    P.dk = static_cast<__nv_bfloat16*>(dk); P.dv = static_cast<__nv_bfloat16*>(dv);
    P.plan = PlanView{static_cast<const int32_t*>(plan), c.n_seqs, c.T, c.causal};
    P.status = reinterpret_cast<int*>(base);
    P.sTq = L.sTq; P.sHq = L.sHq; P.sTkv = L.sTkv; P.sHkv = L.sHkv;
    P.T = c.T; P.Hq = c.Hq; P.Hkv = c.Hkv; P.group = c.Hq / c.Hkv; P.D = c.D; P.rows = w.rows; P.causal = c.causal;
    P.may_split = packed_may_split(c);
    P.scale = c.sm_scale > 0.f ? c.sm_scale : 1.f / sqrtf(static_cast<float>(c.D));
    // -lse / scale has to be finite: in the exponents a scale counts as 2^-120 at least, against which any score below 2^90 is nothing.  dQ and dK get the scale as it is.
    const float least = fmaxf(P.scale, 7.5231638e-37f);
    P.scale_log2 = least * 1.4426950408889634f;
    P.half_inv_scale = 0.5f / least;
    const long long tiles = packed_tiles(c);
    const bool all_short = c.T <= kTile;
    static thread_local int attr_dev = -1;
    int dev = 0;
    cudaGetDevice(&dev);
    if (attr_dev != dev) {
        if (int st = check_cuda(cudaFuncSetAttribute(attn_packed_bwd_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kManySmemBytes), "packed attention: smem attribute")) return st;
        for (auto kernel : {packed_short_kernel<false>, packed_short_kernel<true>})
            if (int st = check_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShortSmemBytes), "packed attention: smem attribute")) return st;
        attr_dev = dev;
    }
    auto launch_short = [&]() {
        PackedShortParams R{};
        R.q = P.q; R.k = P.k; R.v = P.v; R.d_o = P.d_o;
        R.lse = lse;
        R.dq = static_cast<__nv_bfloat16*>(dq); R.dk = P.dk; R.dv = P.dv;
        R.plan = P.plan; R.status = P.status;
        R.sTq = P.sTq; R.sHq = P.sHq; R.sTkv = P.sTkv; R.sHkv = P.sHkv;
        R.T = P.T; R.Hq = P.Hq; R.Hkv = P.Hkv; R.group = P.group; R.D = P.D; R.causal = P.causal;
        R.alone = all_short;
        R.scale = P.scale; R.scale_log2 = P.scale * 1.4426950408889634f;
        const long long items = tiles * c.Hkv, places = static_cast<long long>(P.group > 1 ? 1 : kShortPerSm) * sm_count();
        LaunchScope ls_(K_PACKED_SHORT, stream);
        return check_cuda(launch_chained(P.group > 1 ? packed_short_kernel<true> : packed_short_kernel<false>, dim3(static_cast<unsigned>(items < places ? items : places)),
                                         dim3(kShortThreads), kShortSmemBytes, stream, R), "packed attention: backward launch of short sequences");
    };
    if (all_short) return launch_short();
    {
        PackedPrepParams R{};
        R.o = static_cast<const uint4*>(o); R.d_o = static_cast<const uint4*>(d_o);
        R.delta = reinterpret_cast<float*>(base + w.delta);
        R.dq_acc = reinterpret_cast<float4*>(base + w.dq_acc);
        R.plan = P.plan; R.ticket = P.status + kWsTicketBwd;
        R.Hq = c.Hq; R.D = c.D; R.rows = w.rows;
        const long long slices = tiles * ((kTile * c.Hq * (c.D / 8ll) + 1023) / 1024), places = 8ll * sm_count();
        LaunchScope ls_(K_PACKED_PREP, stream);
        if (int st = check_cuda(launch_chained(packed_prep_kernel, dim3(static_cast<unsigned>(slices < places ? slices : places)), dim3(256), 0, stream, R), "packed attention: backward prep launch")) return st;
    }
    CUtensorMap mq, mk, mv, mdo, macc, mparts{};
    if (P.may_split) {
        if (int st = packed_acc_map(&mparts, base + w.parts, w.rows, 2 * kMostParts * c.Hkv, c.D)) return st;
    }
    if (int st = packed_tile_map(&mq, q, c.D, c.Hq, c.T, L.sTq, L.sHq)) return st;
    if (int st = packed_tile_map(&mk, k, c.D, c.Hkv, c.T, L.sTkv, L.sHkv)) return st;
    if (int st = packed_tile_map(&mv, v, c.D, c.Hkv, c.T, L.sTkv, L.sHkv)) return st;
    if (int st = packed_tile_map(&mdo, d_o, c.D, c.Hq, c.T, HD, c.D)) return st;
    if (int st = packed_acc_map(&macc, base + w.dq_acc, w.rows, c.Hq, c.D)) return st;
    const long long worst = tiles * c.Hkv * (P.may_split ? kMostParts : 1);
    const int grid = static_cast<int>(worst < sm_count() ? worst : sm_count());          // one CTA per SM (all of tensor memory)
    {
        LaunchScope ls_(K_PACKED_BWD, stream);
        if (int st = check_cuda(launch_chained(attn_packed_bwd_kernel, dim3(grid), dim3(kManyThreads), kManySmemBytes, stream, mq, mk, mv, mdo, macc, mparts, P),
                                "packed attention: backward launch")) return st;
    }
    if (int st = launch_short()) return st;
    const long long slices = tiles * ((kTile * c.Hq * (c.D / 8ll) + 1023) / 1024), places = 8ll * sm_count();
    PackedConvertParams F{};
    F.dq_acc = reinterpret_cast<const float4*>(base + w.dq_acc);
    F.dq = static_cast<uint4*>(dq);
    F.plan = P.plan;
    F.parts = reinterpret_cast<const float4*>(base + w.parts);
    F.dv = reinterpret_cast<uint4*>(dv); F.dk = reinterpret_cast<uint4*>(dk);
    F.Hq = c.Hq; F.Hkv = c.Hkv; F.group = P.group; F.D = c.D; F.causal = c.causal; F.may_split = P.may_split; F.main_grid = grid; F.scale = P.scale;
    LaunchScope ls_(K_PACKED_CONVERT, stream);
    return check_cuda(launch_chained(packed_convert_kernel, dim3(static_cast<unsigned>(slices < places ? slices : places)), dim3(256), 0, stream, F), "packed attention: backward convert launch");
}

}  // namespace vardrop
