// Attention over packed sequences, forward.
//
// attn_packed_fwd_kernel   one persistent CTA per SM over items of one 128-query tile of two heads, a warp role for each part of the work: the split of
//                          attn_fwd_kernel (many tiles), whose roles, tensor memory and softmax it shares; what differs stands below.
// attn_packed_tile_kernel  tiles with at most two key tiles: 128-thread CTAs, four to an SM, a tile of a head each, as attn_fwd_tile_kernel.
#include "attn_packed.cuh"
#include "packed_items.h"

namespace vardrop {

namespace {

struct PackedFwdParams {
    const __nv_bfloat16 *q, *k, *v;    // read as rows: V of a sequence's last tile, all of the kernel for few key tiles (the other loads go through the tensor maps)
    __nv_bfloat16* o;                  // [T, Hq, D]
    float* lse;                        // [Hq, T]
    PlanView plan;
    int* status;
    long long sTq, sHq, sTkv, sHkv;
    int T, Hq, group, D;               // group: query heads of a key head
    int causal, grid;                  // CTAs of attn_packed_fwd_kernel
    float scale_log2;                  // sm_scale * log2(e)
};
__device__ __forceinline__ FwdTiles tiles_of(const PlanHead& head) { return FwdTiles{head.tiles, head.many}; }

// An item is the same query tile of two neighbouring heads: under a causal mask both see the same keys, so neither waits for the other, and heads of one group share
// the loads of K and V (others have K and V of their own, stage by stage in turn).  Where those are fewer than the SMs, an item is the query tile of one head, in the places of two: one
// takes its key tiles 0, 2, ..., the other 1, 3, ..., and the two parts of O are joined on their way out.  Roles of a CTA:
//   warps 0, 1       issue the products of head (or part) 0, 1 of an item
//   warp 2           decodes the items; loads Q (double-buffered across items) and a four-stage ring of K/V tiles as boxes
//   warp 3           V of a sequence's last tile as rows, zeros behind its end: P is zero there, but what lies there may be not finite, and zero times that is not zero.
//                    (Rows of Q and K there only reach scores that nothing reads.)
//   warps 4-7        O / l, rounded to bf16 and written as whole rows
//   warps 8-23       four softmax warpgroups, two to a head: one thread per row and 64-key half of a step
constexpr int kFwdTiles = 2;
constexpr int kFwdGroupThreads = 128;
constexpr int kFwdTileThreads = 2 * kFwdGroupThreads;      // softmax threads of a head
constexpr int kFwdThreads = 2 * kFwdGroupThreads + kFwdTiles * kFwdTileThreads;
// Register split: launched with 768 x 80 = 61440 registers; 512 x 96 + 256 x 48 = 61440.
constexpr int kFwdSoftmaxRegs = 96;
constexpr int kFwdOtherRegs = 48;
constexpr int kFwdStages = 4;
constexpr uint32_t kFwdTmemCols = 512;   // of a head: S 128 | P 64 | O 64
constexpr int kFwdSmemBytes = 10240 /*barriers, row maxima and sums, alignment*/ + 2 * kFwdTiles * kTileBytes /*Q tiles of two items*/ + kFwdStages * 2 * kTileBytes /*K, V ring*/ +
                              kTileBytes /*O staging*/;
constexpr float kRescaleStep = 8.f;      // the reference maximum of a row moves only when the running maximum has grown by 2^8
__device__ __forceinline__ float first_reference(float m_first64, float m_rest, float scale_log2) { return (m_rest - m_first64) * scale_log2 > kRescaleStep ? m_rest : m_first64; }
// References and maxima are scores as the products give them, and an exponent is one multiply-add, score scale + shift with shift = -(reference scale).  That product is a rounded one, so the
// exponents of a row are off by up to half a step of it, all alike: 2^-15 up to kFarScore.  Beyond it could be anything (128 and more once scaled scores are 1e9, and a row's largest
// exponential is infinite), so there the reference is taken off the scores ahead of the scale.
constexpr float kFarScore = 1024.f;
constexpr float kFar = 1.401298464324817e-45f;      // for a shift: the least fp32 value, which adds nothing (and is no zero: the library is built without flushing)
__device__ __forceinline__ float shift_of(float reference, float scale_log2) {
    const float shift = -reference * scale_log2;
    return fabsf(shift) > kFarScore ? kFar : shift;
}

__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm volatile("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t d;
    asm volatile("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm volatile("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// barrier among the 256 softmax threads of head w of an item
__device__ __forceinline__ void tile_sync(int w) {
    if (w == 0) asm volatile("bar.sync 2, 256;" ::: "memory");
    else asm volatile("bar.sync 3, 256;" ::: "memory");
}
__device__ __forceinline__ void tile_arrive(int w) {
    if (w == 0) asm volatile("bar.arrive 2, 256;" ::: "memory");
    else asm volatile("bar.arrive 3, 256;" ::: "memory");
}

__global__ void __launch_bounds__(kFwdThreads, 1) attn_packed_fwd_kernel(const __grid_constant__ CUtensorMap map_q,
                                                                          const __grid_constant__ CUtensorMap map_k,
                                                                          const __grid_constant__ CUtensorMap map_v, const PackedFwdParams P) {
    extern __shared__ unsigned char smem_dyn[];
    // Set-up first (shared-memory carve-up, barriers, tensor memory): it touches nothing another kernel produces, so it runs
    // while the previous kernel of the stream is still finishing.
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem_dyn);     // barriers and the TMEM slot sit in front of the tiles
    uint64_t* bar_q_full = bars + 0;                // [2] Q tiles of an item have landed
    uint64_t* bar_q_free = bars + 2;                // [2] every S product of the item has completed (both issue warps)
    uint64_t* bar_kv_full = bars + 4;               // [kFwdStages]
    uint64_t* bar_kv_free = bar_kv_full + kFwdStages;  // [kFwdStages] every product reading the stage has completed (both issue warps)
    uint64_t* bar_s = bar_kv_free + kFwdStages;     // [2] S of tile w's next step is in tensor memory
    uint64_t* bar_sfree = bar_s + kFwdTiles;       // [2] tile w's threads hold S in registers (256 arrivals)
    uint64_t* bar_p = bar_sfree + kFwdTiles;       // [2] P of tile w is in tensor memory (256 arrivals)
    uint64_t* bar_pv = bar_p + kFwdTiles;          // [2] O += P V of tile w's step has completed
    uint64_t* bar_l = bar_pv + kFwdTiles;          // [2] row sums and maxima of tile w's item are in shared memory (256 arrivals)
    uint64_t* bar_ofree = bar_l + kFwdTiles;       // [2] they and O have been read (128 arrivals): the next item may overwrite them
    uint64_t* bar_item = bar_ofree + kFwdTiles;     // [8] entry of the item list is written
    uint64_t* bar_stagger = bar_item + 8;           // P of tile 0's first step is in tensor memory; completes once
    uint64_t* bar_skip = bar_stagger + 1;           // [2] tile 1's softmax warps (8), its issue warp are in an item without a second tile
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_skip + 2);
    float* s_max = reinterpret_cast<float*>(smem_dyn + 768);    // [tile][step parity][half][row] maxima of a step
    float* s_ref = s_max + kFwdTiles * 4 * kTile;               // [tile][row] reference maximum
    float* s_sum = s_ref + kFwdTiles * kTile;                   // [tile][half][row] sums
    float* s_mine = s_sum + kFwdTiles * 2 * kTile;              // [tile][half][row] reference maximum, of its thread alone
    unsigned char* sQ = align_tiles(reinterpret_cast<unsigned char*>(s_mine + kFwdTiles * 2 * kTile));
    unsigned char* sK = sQ + 2 * kFwdTiles * kTileBytes;       // kFwdStages stages of (K tile, V tile)
    unsigned char* sOut = sK + kFwdStages * 2 * kTileBytes;     // staging tile
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (sOut + kTileBytes > smem_dyn + kFwdSmemBytes) {     // dynamic shared memory base not 1024-byte aligned
        chain_wait();
        if (tid == 0) set_status(P.status, VARDROP_ERR_CUDA);
        return;
    }
    if (warp == 0) {
        tmem_alloc(tmem_slot, kFwdTmemCols);
        tmem_relinquish();
    }
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_q_full + i, 1);
            mbar_init(bar_q_free + i, 2);
        }
        for (int st = 0; st < kFwdStages; ++st) {
            mbar_init(bar_kv_full + st, 1 + 32);             // the boxes' announcing arrival, the lanes of the warp that copies rows
            mbar_init(bar_kv_free + st, 2);
        }
        for (int w = 0; w < kFwdTiles; ++w) {
            mbar_init(bar_s + w, 1);
            mbar_init(bar_sfree + w, kFwdTileThreads);
            mbar_init(bar_p + w, kFwdTileThreads);
            mbar_init(bar_pv + w, 1);
            mbar_init(bar_l + w, kFwdTileThreads);
            mbar_init(bar_ofree + w, kFwdGroupThreads);
        }
        for (int i = 0; i < 8; ++i) mbar_init(bar_item + i, 1);
        mbar_init(bar_stagger, 1);
        mbar_init(bar_skip, kFwdTileThreads / 32);
        mbar_init(bar_skip + 1, 1);
        mbar_fence_init();
        tma_prefetch_desc(&map_q);
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    // Work items, decoded by the loader warp one ahead and passed to the other roles through shared memory.  Eight entries: the loads run at most two items ahead of the
    // products, these one of the rows leaving, so an entry has been read long before its place is taken again.
    // Tile w of an item: query tile qt of head h + w.  n_act: heads that exist; -1 ends the list.  mode: both heads have key head kvh; kTwoKv: kvh and kvh + 1; kParts: the parts of one head.
    enum { kOneKv = 0, kTwoKv, kParts };
    struct alignas(16) Item {
        int start, len, qt, h, n_kv, n_act, mode, kvh;
        __device__ __forceinline__ int stages() const { return mode == kTwoKv ? 2 * n_kv : n_kv; }         // of the K/V ring
        __device__ __forceinline__ int per_step() const { return mode == kOneKv ? 1 : 2; }                 // of them, while either tile takes a step
        __device__ __forceinline__ int first_stage(int w) const { return mode == kOneKv ? 0 : w; }
        __device__ __forceinline__ int steps(int w) const { return mode == kParts ? (n_kv + 1 - w) >> 1 : n_kv; }
        __device__ __forceinline__ int key_tile(int w, int j) const { return mode == kParts ? 2 * j + w : j; }
    };
    Item* s_item = reinterpret_cast<Item*>(smem_dyn + 512);
    auto item_at = [&](uint32_t i) {
        Item it;
        ok &= warp_wait_relaxed(bar_item + (i & 7), (i >> 3) & 1);
        const int4* from = reinterpret_cast<const int4*>(s_item + (i & 7));
        const int4 x = from[0], y = from[1];
        it.start = x.x; it.len = x.y; it.qt = x.z; it.h = x.w; it.n_kv = y.x; it.n_act = ok ? y.y : -1; it.mode = y.z; it.kvh = y.w;
        return it;
    };
    // The launch before this one is attn_packed_tile_kernel of the same call, which lets this one in once it has waited for whatever lies before: nothing that is read or
    // written here is its own but the ticket counter, ahead of which the loader waits for it.
    chain_release();

    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFwdOtherRegs));
    if (warp == 2) {
        // ---------------------------------------------------------------- loads ----------------------------------
        uint32_t stage_n = 0, n_done = 0;
        const PlanHead head = plan_head(P.plan);
        const bool parts = in_parts(tiles_of(head), P.Hq, P.causal, P.grid);
        const int per_tile = parts ? P.Hq : (P.Hq + 1) >> 1;
        const long long n_items = static_cast<long long>(few_begin(tiles_of(head), P.Hq, P.grid)) * per_tile;
        auto publish = [&](uint32_t i, long long k) {
            Item it{0, 0, 0, 0, 0, -1, 0, 0};
            if (k < n_items) {
                const int e = static_cast<int>(k / per_tile), hp = static_cast<int>(k - static_cast<long long>(e) * per_tile);
                const int4 x = __ldg(reinterpret_cast<const int4*>(P.plan.entries() + e));
                it.start = x.x; it.len = x.y; it.qt = x.z; it.h = parts ? hp : 2 * hp;
                it.n_kv = P.causal ? it.qt + 1 : (it.len + kTile - 1) / kTile;
                it.n_act = parts ? 2 : min(2, P.Hq - it.h);
                it.kvh = small_div(it.h, P.group);
                it.mode = parts ? kParts : it.n_act == 2 && small_div(it.h + 1, P.group) != it.kvh ? kTwoKv : kOneKv;
            }
            if (lane == 0) {
                int4* to = reinterpret_cast<int4*>(s_item + (i & 7));
                to[0] = make_int4(it.start, it.len, it.qt, it.h);
                to[1] = make_int4(it.n_kv, it.n_act, it.mode, it.kvh);
                mbar_arrive(bar_item + (i & 7));
            }
            __syncwarp();
        };
        bool waited = false;
        publish(0, blockIdx.x);
#pragma unroll 1
        for (uint32_t i = 0; ok; ++i) {
            const Item it = item_at(i);
            if (it.n_act < 0) break;
            const uint32_t qb = n_done & 1;
            ok = warp_wait_relaxed(bar_q_free + qb, ((n_done >> 1) & 1) ^ 1);
            if (!ok) break;
            if (lane == 0) {
                const int tiles = it.mode == kParts ? 1 : it.n_act;
                mbar_expect_tx(bar_q_full + qb, tiles * kTileBytes);
#pragma unroll 1
                for (int w = 0; w < tiles; ++w)
                    tma_load_3d(sQ + (qb * kFwdTiles + w) * kTileBytes, &map_q, bar_q_full + qb, 0, it.h + w, it.start + it.qt * kTile);
            }
            __syncwarp();
            const int heads = it.mode == kTwoKv ? 2 : 1;             // stages of a key tile
            int x = 0, j = 0;
#pragma unroll 1
            for (int l = 0; l < it.stages(); ++l, ++stage_n) {
                const uint32_t st = stage_n % kFwdStages;
                ok = warp_wait_relaxed(bar_kv_free + st, ((stage_n / kFwdStages) & 1) ^ 1);
                if (!ok) break;
                if (lane == 0) {
                    const bool whole = (j + 1) * kTile <= it.len;
                    mbar_expect_tx(bar_kv_full + st, (whole ? 2 : 1) * kTileBytes);
                    tma_load_3d(sK + 2 * st * kTileBytes, &map_k, bar_kv_full + st, 0, it.kvh + x, it.start + j * kTile);
                    if (whole) tma_load_3d(sK + (2 * st + 1) * kTileBytes, &map_v, bar_kv_full + st, 0, it.kvh + x, it.start + j * kTile);
                }
                __syncwarp();
                if (++x == heads) { x = 0; ++j; }
            }
            ++n_done;
            if (!ok) break;
            long long k = n_items;
            if (n_items > gridDim.x) {
                if (!waited) chain_wait();               // the counter is zero now
                waited = true;
                k = next_item(P.status + kWsTicketFwd, gridDim.x, lane);
            }
            publish(i + 1, k);
        }
        if (!waited) chain_wait();                       // this launch is the later one to complete
    } else if (warp == 3) {
        // ---------------------------------------------------------------- V of last tiles -------------------------
        uint32_t stage_n = 0;
#pragma unroll 1
        for (uint32_t i = 0; ok; ++i) {
            const Item it = item_at(i);
            if (it.n_act < 0) break;
            const int heads = it.mode == kTwoKv ? 2 : 1;             // stages of a key tile
            int x = 0, j = 0;
#pragma unroll 1
            for (int l = 0; l < it.stages(); ++l, ++stage_n) {
                const uint32_t st = stage_n % kFwdStages;
                ok = warp_wait_relaxed(bar_kv_free + st, ((stage_n / kFwdStages) & 1) ^ 1);
                if (!ok) break;
                if ((j + 1) * kTile <= it.len) {
                    mbar_arrive(bar_kv_full + st);
                } else {
                    const __nv_bfloat16* from = P.v + it.start * P.sTkv + (it.kvh + x) * P.sHkv;
#pragma unroll 1
                    for (int g = 0; g < 4; ++g) copy_32_tokens(sK + (2 * st + 1) * kTileBytes + g * 32 * kRowBytes, from, P.sTkv, j * kTile + g * 32, it.len, P.D);
                    cp_async_arrive(bar_kv_full + st);
                }
                if (++x == heads) { x = 0; ++j; }
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        // ---------------------------------------------------------------- tensor-core issue ----------------------
        // Issue warp w serves head w of an item.  Both warps follow every stage of the ring and release it with a commit of their own
        // (a commit with nothing outstanding arrives at once), so the release counts are fixed at two.
        const int w = warp;
        uint32_t stage_n = 0, n_done = 0, n_mine = 0, t = 0;      // ring stages passed, items, items and steps of this head
        const int ks_head = P.D / 16;
        // Operand descriptors are built once and stepped by additions.
        const uint64_t d_q = umma_desc_sw128(smem_u32(sQ), 16, 1024);                       // K-major: + 32 bytes per 16 head dimensions
        const uint64_t d_k = umma_desc_sw128(smem_u32(sK), 16, 1024);
        const uint64_t d_v = umma_desc_sw128(smem_u32(sK + kTileBytes), kTileBytes, 1024);  // MN-major: + 2048 bytes per 16 keys
        const uint32_t tm_s = tmem + w * 256, tm_p = tm_s + 128, tm_o = tm_s + 192;
        const uint32_t idesc_o = umma_idesc_bf16(128, P.D, 0, 1);
        auto issue_scores = [&](uint64_t a, uint32_t st, int n_keys) {      // S_w = Q_w K^T, the key count rounded up to 16
            const uint64_t bdesc = umma_desc_advance(d_k, st * 2 * kTileBytes);
            const uint32_t idesc = umma_idesc_bf16(128, (n_keys + 15) & ~15, 0, 0);
            if (elect_one()) {
                tc_mma_bf16(tm_s, a, bdesc, idesc, 0u);
                tc_mma_bf16(tm_s, umma_desc_advance(a, 32), umma_desc_advance(bdesc, 32), idesc, 1u);
                if (ks_head > 2) {
                    tc_mma_bf16(tm_s, umma_desc_advance(a, 64), umma_desc_advance(bdesc, 64), idesc, 1u);
                    tc_mma_bf16(tm_s, umma_desc_advance(a, 96), umma_desc_advance(bdesc, 96), idesc, 1u);
                }
                tc_commit(bar_s + w);
            }
            __syncwarp();
        };
        auto issue_pv = [&](uint32_t st, int n_keys, uint32_t acc) {        // O_w (+)= P_w V
            const uint64_t bdesc = umma_desc_advance(d_v, st * 2 * kTileBytes);
            const int k_steps = (n_keys + 15) >> 4;
            if (elect_one()) {
                if (k_steps == 8) {                 // the usual case, straight-line
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        tc_mma_bf16_ta(tm_o, tm_p + ks * 8, umma_desc_advance(bdesc, ks * 2048), idesc_o, ks > 0 ? 1u : acc);
                } else {
#pragma unroll 1
                    for (int ks = 0; ks < k_steps; ++ks)
                        tc_mma_bf16_ta(tm_o, tm_p + ks * 8, umma_desc_advance(bdesc, ks * 2048), idesc_o, ks > 0 ? 1u : acc);
                }
                tc_commit(bar_pv + w);
            }
            __syncwarp();
        };
        auto wait_full = [&](uint64_t* bar, uint32_t parity, bool rows) {
            ok &= warp_wait_relaxed(bar, parity);
            if (rows) fence_proxy_async_smem();          // rows written by asynchronous copies are read by the tensor core
            tc_fence_after();
        };
        // The scores of the next item's first step go out ahead of the last P V of this one, so that the softmax warps find them when they are done with this one.
        bool primed = false;
        Item it = item_at(0);
#pragma unroll 1
        for (uint32_t i = 0; ok && it.n_act >= 0; ++i) {
            const uint32_t qb = n_done & 1;
            const int per_step = it.per_step(), stages = it.stages();
            Item next;
            if (w < it.n_act) {
                const uint64_t a = umma_desc_advance(d_q, (qb * kFwdTiles + (it.mode == kParts ? 0 : w)) * kTileBytes);
                const int steps = it.steps(w);
                uint32_t sn = stage_n + it.first_stage(w);
                if (!primed) {
                    wait_full(bar_q_full + qb, (n_done >> 1) & 1, false);
                    wait_full(bar_kv_full + sn % kFwdStages, (sn / kFwdStages) & 1, it.len < kTile);
                    // The second head starts a softmax later than the first: in step, both heads' exponentials queue up and then both heads'
                    // hand-offs leave the special-function unit idle.  Not worth its delay for a few steps.  (On a barrier of one phase: bar_p may have gone two phases on
                    // by the time this warp's first stage has landed, and its third waits for a stage of the ring that this warp has yet to release.)
                    if (i == 0 && w == 1 && steps >= 4) ok &= warp_wait_relaxed(bar_stagger, 0);
                    issue_scores(a, sn % kFwdStages, min(kTile, it.len));
                    if (steps == 1) tc_commit_w(bar_q_free + qb);
                }
                primed = false;
                const uint32_t end = stage_n + stages;
                auto release = [&](uint32_t so, uint32_t to) {           // ring stages of this item
#pragma unroll 1
                    for (; so < to && ok; ++so) {
                        ok &= warp_wait_relaxed(bar_kv_full + so % kFwdStages, (so / kFwdStages) & 1);
                        tc_commit_w(bar_kv_free + so % kFwdStages);
                    }
                };
#pragma unroll 1
                for (int j = 0; j < steps && ok; ++j, ++t) {
                    if (j + 1 < steps) {                 // the next S, as soon as the softmax warps hold this one
                        const uint32_t s1 = sn + per_step;
                        const int left = it.len - it.key_tile(w, j + 1) * kTile;
                        wait_full(bar_kv_full + s1 % kFwdStages, (s1 / kFwdStages) & 1, left < kTile);
                        ok &= warp_wait_relaxed(bar_sfree + w, t & 1);
                        tc_fence_after();
                        issue_scores(a, s1 % kFwdStages, min(kTile, left));
                        if (j + 2 == steps) tc_commit_w(bar_q_free + qb);
                    } else {
                        next = item_at(i + 1);
                        const uint32_t s1 = end + next.first_stage(w);
                        // (not with a stage that comes into the place of one that this warp has yet to release: the second part of an odd number of key tiles)
                        if (w < next.n_act && s1 < stage_n + kFwdStages) {
                            wait_full(bar_q_full + (qb ^ 1), ((n_done + 1) >> 1) & 1, false);
                            wait_full(bar_kv_full + s1 % kFwdStages, (s1 / kFwdStages) & 1, next.len < kTile);
                            ok &= warp_wait_relaxed(bar_sfree + w, t & 1);
                            tc_fence_after();
                            issue_scores(umma_desc_advance(d_q, ((qb ^ 1) * kFwdTiles + (next.mode == kParts ? 0 : w)) * kTileBytes), s1 % kFwdStages, min(kTile, next.len));
                            if (next.steps(w) == 1) tc_commit_w(bar_q_free + (qb ^ 1));
                            primed = true;
                        }
                    }
                    ok &= warp_wait_relaxed(bar_p + w, t & 1);
                    if (t == 0 && w == 0 && lane == 0) mbar_arrive(bar_stagger);
                    if (j == 0 && n_mine > 0) ok &= warp_wait_relaxed(bar_ofree + w, (n_mine - 1) & 1);     // O of the previous item has been read
                    tc_fence_after();
                    issue_pv(sn % kFwdStages, min(kTile, it.len - it.key_tile(w, j) * kTile), j > 0);
                    release(stage_n, min(end, stage_n + per_step));      // this step's stages: mine is read by the products above
                    stage_n += per_step;
                    sn += per_step;
                }
                release(stage_n, end);
                stage_n = end;
                ++n_mine;
            } else {                                     // nothing to compute in this item: keep up with its barriers
                ok &= warp_wait_relaxed(bar_q_full + qb, (n_done >> 1) & 1);
                ok &= warp_wait_relaxed(bar_skip, (n_done - n_mine) & 1);      // its softmax warps are here too
                if (lane == 0) mbar_arrive(bar_skip + 1);
                tc_commit_w(bar_q_free + qb);
#pragma unroll 1
                for (int l = 0; l < stages && ok; ++l) {
                    const uint32_t so = stage_n + l;
                    ok &= warp_wait_relaxed(bar_kv_full + so % kFwdStages, (so / kFwdStages) & 1);
                    tc_commit_w(bar_kv_free + so % kFwdStages);
                }
                next = item_at(i + 1);
                stage_n += stages;
            }
            ++n_done;
            it = next;
        }
    }
    } else if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFwdOtherRegs));
        // ---------------------------------------------------------------- O / l, rounded to bf16 ------------------
        // through a staging tile, so that whole 128-byte rows are written; a warp writes the rows it has staged
        const int r = tid & (kFwdGroupThreads - 1);
        const uint32_t lane_sel = static_cast<uint32_t>((warp & 3) * 32) << 16;
        uint32_t t0 = 0, t1 = 0, n0 = 0, n1 = 0;        // steps and items of the two softmax warpgroups so far
        const int c = r & 7, r0 = (r & ~31) + (lane >> 3);
#pragma unroll 1
        for (uint32_t i = 0; ok; ++i) {
            const Item it = item_at(i);
            if (it.n_act < 0) break;
            const bool parts = it.mode == kParts;
#pragma unroll 1
            for (int w = 0; w < (parts ? 1 : it.n_act); ++w) {
                unsigned char* stage = sOut;
#pragma unroll 1
                for (int p = w; p <= (parts ? 1 : w); ++p) {
                    ok &= warp_wait_relaxed(bar_l + p, (p ? n1 : n0) & 1);
                    ok &= warp_wait(bar_pv + p, ((p ? t1 : t0) + it.steps(p) - 1) & 1);
                }
                if (!ok) break;
                tc_fence_after();
                float m_ref = s_ref[w * kTile + r], l_sum = s_sum[2 * w * kTile + r] + s_sum[(2 * w + 1) * kTile + r];
                float mine = 1.f, other = 0.f;           // factors of the parts
                if (parts) {                             // both against the larger reference
                    const float m0 = m_ref, m1 = s_ref[kTile + r];
                    m_ref = fmaxf(m0, m1);
                    mine = fast_exp2((m0 - m_ref) * P.scale_log2);
                    other = fast_exp2((m1 - m_ref) * P.scale_log2);
                    l_sum = l_sum * mine + (s_sum[2 * kTile + r] + s_sum[3 * kTile + r]) * other;
                    other *= 1.f / l_sum;
                }
                mine *= 1.f / l_sum;
                const int row = it.qt * kTile + r;
                unsigned char* rowp = stage + r * kRowBytes;
#pragma unroll 1
                for (int c16 = 0; c16 < P.D / 16; ++c16) {
                    float ov[16];
                    tmem_ld16(tmem + w * 256 + 192 + lane_sel + c16 * 16, ov);
                    tmem_ld_wait();
#pragma unroll
                    for (int d = 0; d < 16; ++d) ov[d] *= mine;
                    if (parts) {
                        float second[16];
                        tmem_ld16(tmem + 256 + 192 + lane_sel + c16 * 16, second);
                        tmem_ld_wait();
#pragma unroll
                        for (int d = 0; d < 16; ++d) ov[d] = fmaf(second[d], other, ov[d]);
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        *reinterpret_cast<uint4*>(rowp + (((c16 * 2 + q) ^ (r & 7)) << 4)) =
                            make_uint4(pack_bf16(ov[8 * q + 0], ov[8 * q + 1]), pack_bf16(ov[8 * q + 2], ov[8 * q + 3]),
                                       pack_bf16(ov[8 * q + 4], ov[8 * q + 5]), pack_bf16(ov[8 * q + 6], ov[8 * q + 7]));
                }
                tc_fence_before();
                if (parts) mbar_arrive(bar_ofree + 1);
                mbar_arrive(bar_ofree + w);                  // O, maximum and sum are in registers or in the staging tile
                if (row < it.len) P.lse[static_cast<size_t>(it.h + w) * P.T + it.start + row] = (m_ref * P.scale_log2 + log2f(l_sum)) * 0.6931471805599453f;
                __syncwarp();
                if (c * 8 < P.D) {
                    __nv_bfloat16* out = P.o + (static_cast<size_t>(it.start + it.qt * kTile + r0) * P.Hq + it.h + w) * P.D + c * 8;
                    const unsigned char* from = stage + r0 * kRowBytes;
                    const int left = it.len - it.qt * kTile - r0;             // rows 4 apart, as long as they exist
#pragma unroll 1
                    for (int x = 0; x < 8; x += 4) {
                        uint4 v[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const uint4*>(from + (x + u) * 4 * kRowBytes + ((c ^ ((r0 + 4 * u) & 7)) << 4));
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if ((x + u) * 4 < left) *reinterpret_cast<uint4*>(out + static_cast<size_t>(x + u) * 4 * P.Hq * P.D) = v[u];
                    }
                }
                __syncwarp();                                // its rows of the staging tile are free
            }
            t0 += it.steps(0); ++n0;
            if (it.n_act > 1) { t1 += it.steps(1); ++n1; }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kFwdSoftmaxRegs));
        // ---------------------------------------------------------------- softmax --------------------------------
        const int w = (warp - 8) >> 3, half = ((warp - 8) >> 2) & 1;     // query tile of the item, 64-key half of a step
        const int r = tid & (kFwdGroupThreads - 1);     // query row inside the tile = tensor-memory lane
        const uint32_t lane_sel = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t tm_s = tmem + w * 256 + half * 64 + lane_sel, tm_p = tmem + w * 256 + 128 + half * 32 + lane_sel, tm_o = tmem + w * 256 + 192 + lane_sel;
        float* my_max = s_max + w * 4 * kTile + r;
        uint32_t n_mine = 0, t = 0;                     // items and steps of this tile so far
#pragma unroll 1
        for (uint32_t i = 0; ok; ++i) {
            const Item it = item_at(i);
            if (it.n_act < 0) break;
            if (w >= it.n_act) {                        // nothing else ties the warps of a tile that an item lacks to the others' pace, and they wait by parity
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_skip);
                ok = warp_wait_relaxed(bar_skip + 1, (i - n_mine) & 1);
                continue;
            }
            // Exponentials are taken against a reference that trails the running maximum.  What every step needs of it is its shift; itself it lies in shared memory.
            float shift = kFar, l_run = 0.f;
            auto refer_to = [&](float reference) {
                s_mine[(2 * w + half) * kTile + r] = reference;
                shift = shift_of(reference, P.scale_log2);
            };
            bool s_ready = false;                       // a poll's answer takes a hundred cycles: polls go out ahead of where they are needed
            // keys that this row sees from this half of a step on (may be none; never none of a row's first 64, so a row's reference is finite: tiles in parts have three key tiles or more)
            int valid = min(it.len, P.causal ? it.qt * kTile + r + 1 : it.len) - it.key_tile(w, 0) * kTile - half * 64;
            const int stride = it.mode == kParts ? 2 * kTile : kTile;
            bool first = true;
#pragma unroll 1
            for (int steps = it.steps(w); steps > 0; --steps, ++t, valid -= stride) {
                if (!__all_sync(0xffffffffu, s_ready)) ok = warp_wait(bar_s + w, t & 1);
                if (!ok) break;
                tc_fence_after();
                float s[64];
                tmem_ld32(tm_s, s);
                tmem_ld32(tm_s + 32, s + 32);
                tmem_ld_wait();
                tc_fence_before();
                mbar_arrive(bar_sfree + w);              // S is in registers: the next one may be produced
                if (valid < 64) {                                     // ragged last step, or the diagonal: keys that are not seen never win the max
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        if (i >= valid) s[i] = -INFINITY;
                }
                float mx[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) mx[i] = s[i];
#pragma unroll
                for (int i = 4; i < 60; i += 8) {                     // three-input maximum: two new values per instruction
#pragma unroll
                    for (int u = 0; u < 4; ++u) mx[u] = max3(mx[u], s[i + u], s[i + 4 + u]);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) mx[u] = fmaxf(mx[u], s[60 + u]);
                // the other half's maximum of the row, through shared memory (arrays of the two step parities, so one barrier a step is enough)
                float* ex = my_max + (t & 1) * 2 * kTile;
                const float m_mine = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                ex[half * kTile] = m_mine;
                const bool pv_done = t == 0 || mbar_test(bar_pv + w, (t - 1) & 1);
                const float above = shift == kFar ? INFINITY : shift;     // a row that is far, or has no reference yet, goes the long way
                tile_sync(w);
                const float m_tile = fmaxf(m_mine, ex[(half ^ 1) * kTile]);
                if (__any_sync(0xffffffffu, fmaf(m_tile, P.scale_log2, above) > kRescaleStep)) {
                    if (first) {
                        first = false;
                        refer_to(first_reference(ex[0], m_tile, P.scale_log2));
                    } else {
                        // O accumulates in tensor memory against the reference.  It is rescaled only when a row's maximum has outgrown that by
                        // 2^8 (probabilities then stay below 256, exact enough in bf16 and far from overflow); each half takes its
                        // share of the columns.
                        const float m_ref = s_mine[(2 * w + half) * kTile + r];
                        const bool grow = (m_tile - m_ref) * P.scale_log2 > kRescaleStep;
                        ok = warp_wait(bar_pv + w, (t - 1) & 1);          // O of the previous step is complete
                        tc_fence_after();
                        const float alpha = grow ? fast_exp2((m_ref - m_tile) * P.scale_log2) : 1.f;
                        if (grow) refer_to(m_tile);
                        l_run *= alpha;
#pragma unroll 1
                        for (int c = half * (P.D / 2); c < (half + 1) * (P.D / 2); c += 16) {     // sixteen columns at a time: the scores stay in registers
                            float ov[16];
                            tmem_ld16(tm_o + c, ov);
                            tmem_ld_wait();
#pragma unroll
                            for (int d = 0; d < 16; ++d) ov[d] *= alpha;
                            tmem_st16(tm_o + c, reinterpret_cast<const uint32_t*>(ov));
                        }
                    }
                    if (shift == kFar) {
                        const float m_ref = s_mine[(2 * w + half) * kTile + r];
#pragma unroll
                        for (int i = 0; i < 64; ++i) s[i] -= m_ref;
                    }
                }
                const uint64_t scale2 = pair_of(P.scale_log2, P.scale_log2), shift2 = pair_of(shift, shift);
                uint64_t l2[2] = {pair_of(0.f, 0.f), pair_of(0.f, 0.f)};          // four running sums: keys i = 0..3 mod 4
                uint32_t pk[32];
                // three batches of eight scores in flight: exponents of batch g, exponentials of batch g - 1, sums and rounding of batch g - 2
#pragma unroll
                for (int g = 0; g < 10; ++g) {
                    if (g < 8) {
#pragma unroll
                        for (int i = 8 * g; i < 8 * g + 8; i += 2) halves_of(fma_pair(pair_of(s[i], s[i + 1]), scale2, shift2), s[i], s[i + 1]);
                    }
                    if (g >= 1 && g < 9) {
#pragma unroll
                        for (int i = 8 * g - 8; i < 8 * g; ++i) s[i] = fast_exp2(s[i]);       // exp2(-inf) = 0 for the masked keys
                    }
                    if (g >= 2) {
#pragma unroll
                        for (int i = 8 * g - 16; i < 8 * g - 8; i += 2) {
                            l2[(i >> 1) & 1] = add_pair(l2[(i >> 1) & 1], pair_of(s[i], s[i + 1]));
                            pk[i >> 1] = pack_bf16(s[i], s[i + 1]);
                        }
                    }
                }
                if (!__all_sync(0xffffffffu, pv_done)) ok &= warp_wait(bar_pv + w, (t - 1) & 1);      // P V of the previous step has read P
                tc_fence_after();
                s_ready = mbar_test(bar_s + w, (t + 1) & 1);
                tmem_st32(tm_p, pk);                                  // keys 2 c and 2 c + 1 in column c
                {
                    float a0, a1, a2, a3;
                    halves_of(l2[0], a0, a1);
                    halves_of(l2[1], a2, a3);
                    l_run += (a0 + a1) + (a2 + a3);
                }
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(bar_p + w);
                if (!ok) break;
            }
            if (!ok) break;
            if (n_mine > 0) ok = warp_wait(bar_ofree + w, (n_mine - 1) & 1);         // the previous item's have been read
            if (half == 0) s_ref[w * kTile + r] = s_mine[2 * w * kTile + r];
            s_sum[(2 * w + half) * kTile + r] = l_run;
            mbar_arrive(bar_l + w);
            ++n_mine;
        }
    }

    if (!ok) {
        set_status(P.status, VARDROP_ERR_TIMEOUT);
        // A softmax warp whose wait gave up has left by itself, and nothing bounds a named barrier: it arrives once more in passing.  The others reach
        // at most one more: the scores of the step behind that one wait for this warp's arrivals too.
        if (warp >= 8) tile_arrive((warp - 8) >> 3);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, kFwdTmemCols);
}


// ---------------------------------------------------------------------------------------------------------
// few key tiles
// ---------------------------------------------------------------------------------------------------------
// A chain of latencies in which every path runs once or twice: no roles and no hand-offs but the CTA barrier, rolled loops over 32 scores that stay in tensor memory and are
// read twice, 48 KB and 128 columns a CTA, so that four CTAs share an SM and fill each other's waits.  All loads are row copies with zeros behind a sequence's end.
// Tensor memory: S 128; P (bf16) over S's columns 0 .. 63 as they are consumed, P V into columns 64 .. 127.
constexpr int kTileFwdThreads = 128;
constexpr uint32_t kTileFwdTmemCols = 128;
constexpr int kTileFwdSmemBytes = 1024 /*alignment*/ + 3 * kTileBytes /*Q, K, V*/;
constexpr int kTileFwdPerSm = 4;

// kAll: every tile of the batch is this kernel's.  Otherwise attn_packed_fwd_kernel follows, and runs as SMs become free.
template <bool kAll>
__global__ void __launch_bounds__(kTileFwdThreads, kTileFwdPerSm) attn_packed_tile_kernel(const PackedFwdParams P) {
    extern __shared__ unsigned char smem_dyn[];
    __shared__ uint64_t bar_s, bar_o;
    __shared__ uint32_t tmem_slot;
    unsigned char* sQ = align_tiles(smem_dyn);
    unsigned char* sK = sQ + kTileBytes;
    unsigned char* sV = sK + kTileBytes;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (warp == 0) {
        tmem_alloc(&tmem_slot, kTileFwdTmemCols);
        tmem_relinquish();
    }
    if (tid == 0) {
        mbar_init(&bar_s, 1);
        mbar_init(&bar_o, 1);
        mbar_fence_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tm = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    const uint32_t idesc_o = umma_idesc_bf16(128, P.D, 0, 1);
    const uint64_t d_q = umma_desc_sw128(smem_u32(sQ), 16, 1024), d_k = umma_desc_sw128(smem_u32(sK), 16, 1024);
    const uint64_t d_v = umma_desc_sw128(smem_u32(sV), kTileBytes, 1024);
    const uint64_t scale2 = pair_of(P.scale_log2, P.scale_log2);
    chain_wait();
    if (!kAll && blockIdx.x == 0 && tid == 0) P.status[kWsTicketFwd] = 0;
    chain_release();
    const PlanHead head = plan_head(P.plan);
    if (!head.fits && blockIdx.x == 0 && tid == 0) set_status(P.status, VARDROP_ERR_INVALID_ARG);
    const int first = kAll ? 0 : few_begin(tiles_of(head), P.Hq, P.grid), n_items = (head.tiles - first) * P.Hq;
    bool ok = true;
    uint32_t t = 0;                                     // key tiles of this CTA so far: parity of bar_s and bar_o

#pragma unroll 1
    for (int item = blockIdx.x; item < n_items; item += gridDim.x) {
        const int e = item / P.Hq, h = item - e * P.Hq, kvh = small_div(h, P.group);
        const int4 entry = __ldg(reinterpret_cast<const int4*>(P.plan.entries() + first + e));
        const int start = entry.x, len = entry.y, qt = entry.z, n_kv = P.causal ? qt + 1 : (len + kTile - 1) / kTile;
        // Grouped heads of a short sequence share a tile: the first of them has the work of all.  (Not where every tile of a head finds a place of its own: what the places of the rows
        // take is then on the path of a chain of latencies, 7.4 -> 9.0 us for a few short prompts.)
        const int in_group = h - kvh * P.group, most = len <= kTile / 2 && n_items > static_cast<int>(gridDim.x) ? heads_a_tile(len, P.group) : 1;
        if (most > 1 && in_group % most != 0) continue;
        const int heads = most > 1 ? min(most, P.group - in_group) : 1;
        const PackedRow at = heads > 1 ? packed_row(min(tid, heads * len - 1), len) : PackedRow{0, tid};
        const __nv_bfloat16* const q = P.q + start * P.sTq + h * P.sHq;
        const __nv_bfloat16* const k = P.k + start * P.sTkv + kvh * P.sHkv;
        const __nv_bfloat16* const v = P.v + start * P.sTkv + kvh * P.sHkv;
        // every warp copies its 32 rows of a tile
        auto load_rows = [&](unsigned char* tile, const __nv_bfloat16* from, long long sT, int t0) {
            copy_32_tokens(tile + warp * 32 * kRowBytes, from, sT, t0 * kTile + warp * 32, len, P.D);
        };
        if (heads > 1) copy_32_packed(sQ + warp * 32 * kRowBytes, q, P.sTq, P.sHq, warp * 32, heads * len, len, P.D);
        else load_rows(sQ, q, P.sTq, qt);
        load_rows(sK, k, P.sTkv, 0);
        asm volatile("cp.async.commit_group;" ::: "memory");
        load_rows(sV, v, P.sTkv, 0);
        asm volatile("cp.async.commit_group;" ::: "memory");
        float o_acc[kDP];                                // more than one key tile: the sum over the tiles before the current one
        float m_run = -INFINITY, l_run = 0.f;
#pragma unroll 1
        for (int j = 0; j < n_kv; ++j, ++t) {
            const int n_keys = min(kTile, len - j * kTile), n_seen = P.causal && j == qt ? min(n_keys, at.token + 1) : n_keys;     // of this row
            if (j > 0) {
#pragma unroll 1
                for (int x = 1; x < 3; ++x) {            // K, V
                    load_rows(sQ + x * kTileBytes, x == 1 ? k : v, P.sTkv, j);
                    asm volatile("cp.async.commit_group;" ::: "memory");
                }
            }
            asm volatile("cp.async.wait_group 1;" ::: "memory");         // Q and K have landed
            fence_proxy_async_smem();
            tc_fence_before();
            __syncthreads();
            if (warp == 0) {
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t idesc = umma_idesc_bf16(128, (n_keys + 15) & ~15, 0, 0);
#pragma unroll 1
                    for (int ks = 0; ks < P.D / 16; ++ks)
                        tc_mma_bf16(tmem, umma_desc_advance(d_q, ks * 32), umma_desc_advance(d_k, ks * 32), idesc, ks > 0);
                    tc_commit(&bar_s);
                }
                __syncwarp();
            }
            ok &= mbar_wait(&bar_s, t & 1);
            tc_fence_after();
            // ---- row maximum, 32 scores at a time ----
            float m_tile = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < n_keys; c += 32) {
                float s[32];
                tmem_ld32(tm + c, s);
                tmem_ld_wait();
                if (__any_sync(0xffffffffu, n_seen - c < 32)) {       // ragged end, or the diagonal: keys that are not seen never win the maximum
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c + i >= n_seen) s[i] = -INFINITY;
                }
                float mx[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) mx[u] = s[u];
#pragma unroll
                for (int i = 4; i < 28; i += 8) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) mx[u] = max3(mx[u], s[i + u], s[i + 4 + u]);
                }
                m_tile = max3(m_tile, max3(mx[0], s[28], mx[1]), max3(max3(s[29], mx[2], s[30]), mx[3], s[31]));
            }
            const float m_new = fmaxf(m_run, m_tile), alpha = fast_exp2((m_run - m_new) * P.scale_log2), shift = shift_of(m_new, P.scale_log2);
            m_run = m_new;
            if (__any_sync(0xffffffffu, shift == kFar)) {
#pragma unroll 1
                for (int c = 0; c < n_keys; c += 32) {
                    float s[32];
                    tmem_ld32(tm + c, s);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) s[i] = shift == kFar ? s[i] - m_new : s[i];
                    tmem_st32(tm + c, reinterpret_cast<const uint32_t*>(s));
                }
                tmem_st_wait();
            }
            // ---- P = exp2(S scale - maximum), rounded to bf16, over the columns of S that have been read ----
            const uint64_t shift2 = pair_of(shift, shift);
            uint64_t l2[2] = {pair_of(0.f, 0.f), pair_of(0.f, 0.f)};
            auto l_sum = [&]() {
                float a0, a1, a2, a3;
                halves_of(l2[0], a0, a1);
                halves_of(l2[1], a2, a3);
                return (a0 + a1) + (a2 + a3);
            };
#pragma unroll 1
            for (int c = 0; c < n_keys; c += 32) {
                float s[32];
                uint32_t pk[16];
                tmem_ld32(tm + c, s);
                tmem_ld_wait();
                if (__any_sync(0xffffffffu, n_seen - c < 32)) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c + i >= n_seen) s[i] = -INFINITY;
                }
#pragma unroll
                for (int g = 0; g < 6; ++g) {            // batches of eight: exponents of g, exponentials of g - 1, sums and rounding of g - 2
                    if (g < 4) {
#pragma unroll
                        for (int i = 8 * g; i < 8 * g + 8; i += 2) halves_of(fma_pair(pair_of(s[i], s[i + 1]), scale2, shift2), s[i], s[i + 1]);
                    }
                    if (g >= 1 && g < 5) {
#pragma unroll
                        for (int i = 8 * g - 8; i < 8 * g; ++i) s[i] = fast_exp2(s[i]);       // exp2(-inf) = 0 for the masked keys
                    }
                    if (g >= 2) {
#pragma unroll
                        for (int i = 8 * g - 16; i < 8 * g - 8; i += 2) {
                            l2[(i >> 1) & 1] = add_pair(l2[(i >> 1) & 1], pair_of(s[i], s[i + 1]));
                            pk[i >> 1] = pack_bf16(s[i], s[i + 1]);
                        }
                    }
                }
                tmem_st16(tm + (c >> 1), pk);            // keys 2 c' and 2 c' + 1 in column c'
            }
            l_run = l_run * alpha + l_sum();
            asm volatile("cp.async.wait_group 0;" ::: "memory");             // V has landed
            fence_proxy_async_smem();
            tmem_st_wait();
            tc_fence_before();
            ok = __syncthreads_and(ok);
            if (!ok) { item = n_items; break; }          // a wait gave up somewhere in the CTA: stop
            if (warp == 0) {
                tc_fence_after();
                if (elect_one()) {
#pragma unroll 1
                    for (int ks = 0; ks < (n_keys + 15) >> 4; ++ks)
                        tc_mma_bf16_ta(tmem + 64, tmem + ks * 8, umma_desc_advance(d_v, ks * 2048), idesc_o, ks > 0);
                    tc_commit(&bar_o);
                }
                __syncwarp();
            }
            ok &= mbar_wait(&bar_o, t & 1);              // (agreed on at the next such barrier: no thread leaves by itself)
            tc_fence_after();
            if (n_kv > 1) {
                if (j == 0) {
                    tmem_ld32(tm + 64, o_acc);
                    if (P.D > 32) tmem_ld32(tm + 96, o_acc + 32);
                    tmem_ld_wait();
                } else {
                    const uint64_t alpha2 = pair_of(alpha, alpha);
#pragma unroll
                    for (int c = 0; c < kDP; c += 32) {
                        if (c < P.D) {
                            float ov[32];
                            tmem_ld32(tm + 64 + c, ov);
                            tmem_ld_wait();
#pragma unroll
                            for (int d = 0; d < 32; d += 2)          // rescale and add in one step
                                halves_of(fma_pair(pair_of(o_acc[c + d], o_acc[c + d + 1]), alpha2, pair_of(ov[d], ov[d + 1])), o_acc[c + d], o_acc[c + d + 1]);
                        }
                    }
                    if (j + 1 == n_kv) {                 // back where a single tile leaves it
                        tmem_st32(tm + 64, reinterpret_cast<const uint32_t*>(o_acc));
                        if (P.D > 32) tmem_st32(tm + 96, reinterpret_cast<const uint32_t*>(o_acc + 32));
                        tmem_st_wait();
                    }
                }
            }
            tc_fence_before();
            if (j + 1 < n_kv) __syncthreads();           // the next step's S goes over these columns
        }
        if (item == n_items) break;
        // ---- O / l, rounded to bf16, through Q's tile so that whole rows are written ----
        {
            const float inv_l = 1.f / l_run;
            unsigned char* rowp = sQ + tid * kRowBytes;
            const int row = qt * kTile + at.token;
            if (heads > 1 ? tid < heads * len : row < len) P.lse[static_cast<size_t>(h + at.head) * P.T + start + row] = (m_run * P.scale_log2 + log2f(l_run)) * 0.6931471805599453f;
#pragma unroll 1
            for (int c16 = 0; c16 < P.D / 16; ++c16) {
                float ov[16];
                tmem_ld16(tm + 64 + c16 * 16, ov);
                tmem_ld_wait();
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    *reinterpret_cast<uint4*>(rowp + (((c16 * 2 + q) ^ (tid & 7)) << 4)) =
                        make_uint4(pack_bf16(ov[8 * q + 0] * inv_l, ov[8 * q + 1] * inv_l), pack_bf16(ov[8 * q + 2] * inv_l, ov[8 * q + 3] * inv_l),
                                   pack_bf16(ov[8 * q + 4] * inv_l, ov[8 * q + 5] * inv_l), pack_bf16(ov[8 * q + 6] * inv_l, ov[8 * q + 7] * inv_l));
            }
            tc_fence_before();
            __syncwarp();                                // a warp writes the rows it has staged
            const int c = lane & 7, r0 = warp * 32 + (lane >> 3);
            if (heads > 1) {
#pragma unroll 1
                for (int r = r0; r < min(warp * 32 + 32, heads * len) && c * 8 < P.D; r += 4) {
                    const PackedRow to = packed_row(r, len);
                    *reinterpret_cast<uint4*>(P.o + (static_cast<size_t>(start + to.token) * P.Hq + h + to.head) * P.D + c * 8) = *reinterpret_cast<const uint4*>(sQ + r * kRowBytes + ((c ^ (r & 7)) << 4));
                }
            } else if (c * 8 < P.D) {
                __nv_bfloat16* out = P.o + (static_cast<size_t>(start + qt * kTile + r0) * P.Hq + h) * P.D + c * 8;
                const unsigned char* from = sQ + r0 * kRowBytes + ((c ^ (r0 & 7)) << 4);
                const unsigned char* from4 = sQ + (r0 + 4) * kRowBytes + ((c ^ ((r0 + 4) & 7)) << 4);
                const int left = min(32 - (lane >> 3), len - qt * kTile - r0);
                const size_t step = static_cast<size_t>(4) * P.Hq * P.D;
#pragma unroll 1
                for (int x = 0; x < left; x += 8, out += 2 * step, from += 8 * kRowBytes, from4 += 8 * kRowBytes) {     // rows 4 apart
                    const uint4 v0 = *reinterpret_cast<const uint4*>(from), v1 = *reinterpret_cast<const uint4*>(from4);
                    *reinterpret_cast<uint4*>(out) = v0;
                    if (x + 4 < left) *reinterpret_cast<uint4*>(out + step) = v1;
                }
            }
            __syncthreads();                             // Q's tile is free for the next item
        }
    }
    if (!ok) set_status(P.status, VARDROP_ERR_TIMEOUT);
    asm volatile("cp.async.wait_all;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, kTileFwdTmemCols);
}
}  // namespace

int attn_packed_fwd_launch(const void* q, const void* k, const void* v, const void* plan, const vardrop_packed_cfg& c, void* o, float* lse, void* ws, cudaStream_t stream) {
    const PackedStrides L = packed_strides(c);
    PackedFwdParams P{};
    P.q = static_cast<const __nv_bfloat16*>(q); P.k = static_cast<const __nv_bfloat16*>(k); P.v = static_cast<const __nv_bfloat16*>(v);
    P.o = static_cast<__nv_bfloat16*>(o); P.lse = lse;
    P.plan = PlanView{static_cast<const int32_t*>(plan), c.n_seqs, c.T, c.causal};
    P.status = static_cast<int*>(ws);
    P.sTq = L.sTq; P.sHq = L.sHq; P.sTkv = L.sTkv; P.sHkv = L.sHkv;
    P.T = c.T; P.Hq = c.Hq; P.group = c.Hq / c.Hkv; P.D = c.D; P.causal = c.causal;
    const float scale = c.sm_scale > 0.f ? c.sm_scale : 1.f / sqrtf(static_cast<float>(c.D));
    P.scale_log2 = scale * 1.4426950408889634f;
    static thread_local int attr_dev = -1;
    int dev = 0;
    cudaGetDevice(&dev);
    if (attr_dev != dev) {
        if (int st = check_cuda(cudaFuncSetAttribute(attn_packed_fwd_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFwdSmemBytes), "packed attention: smem attribute")) return st;
        for (auto kernel : {attn_packed_tile_kernel<false>, attn_packed_tile_kernel<true>})
            if (int st = check_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileFwdSmemBytes), "packed attention: smem attribute")) return st;
        attr_dev = dev;
    }
    const long long tiles = packed_tiles(c), places = static_cast<long long>(kTileFwdPerSm) * sm_count();
    const long long worst = tiles * c.Hq;
    const int grid = static_cast<int>(worst < sm_count() ? worst : sm_count());                 // one CTA per SM
    P.grid = grid;
    const dim3 tile_grid(static_cast<unsigned>(tiles * c.Hq < places ? tiles * c.Hq : places));
    if (c.T <= kFewTiles * kTile) {
        LaunchScope ls_(K_PACKED_TILE, stream);
        return check_cuda(launch_chained(attn_packed_tile_kernel<true>, tile_grid, dim3(kTileFwdThreads), kTileFwdSmemBytes, stream, P), "packed attention: forward launch");
    }
    CUtensorMap mq, mk, mv;
    if (int st = packed_tile_map(&mq, q, c.D, c.Hq, c.T, L.sTq, L.sHq)) return st;
    if (int st = packed_tile_map(&mk, k, c.D, c.Hkv, c.T, L.sTkv, L.sHkv)) return st;
    if (int st = packed_tile_map(&mv, v, c.D, c.Hkv, c.T, L.sTkv, L.sHkv)) return st;
    {
        LaunchScope ls_(K_PACKED_TILE, stream);
        if (int st = check_cuda(launch_chained(attn_packed_tile_kernel<false>, tile_grid, dim3(kTileFwdThreads), kTileFwdSmemBytes, stream, P), "packed attention: forward launch")) return st;
    }
    LaunchScope ls_(K_PACKED_FWD, stream);
    return check_cuda(launch_chained(attn_packed_fwd_kernel, dim3(grid), dim3(kFwdThreads), kFwdSmemBytes, stream, mq, mk, mv, P), "packed attention: forward launch");
}

}  // namespace vardrop
