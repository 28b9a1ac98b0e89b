// The plan of a batch of packed sequences: its tiles in the order of their work, from the offsets, on the device.
#include "attn_packed.cuh"

namespace vardrop {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanBins = 4096;          // tiles are sorted by their work in tiles; what is longer shares the last bin

struct PlanParams {
    const int32_t* cu;
    int32_t* plan;
    int n_seqs, T, causal, bins;
    long long cap;
};

__device__ __forceinline__ int block_scan(int v, int* s_warp) {      // exclusive, over the block; s_warp[32] holds the total
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                     // s_warp of the scan before has been read
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int w = lane < static_cast<int>(blockDim.x >> 5) ? s_warp[lane] : 0;
        const int mine = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += y;
        }
        if (lane == 31) s_warp[32] = w;
        s_warp[lane] = w - mine;
    }
    __syncthreads();
    return x - v + s_warp[warp];
}

// (128 threads for up to 128 sequences, whose barriers are the cheaper ones; 1024 beyond.)
// Counting sort: tiles per amount of work, then each tile's place.  Sequences come a thread each, as many at a time as there are threads; their tiles are shared out over all threads again, so a
// single long sequence takes no longer than many short ones.
__global__ void __launch_bounds__(kPlanThreads) packed_plan_kernel(const PlanParams P) {
    __shared__ int s_warp[33], s_bin[kPlanBins + 1], s_bad, s_most;
    __shared__ unsigned long long s_work;
    __shared__ int s_first[kPlanThreads + 1], s_start[kPlanThreads], s_len[kPlanThreads];
    chain_wait();
    chain_release();
    const int tid = threadIdx.x, nt = blockDim.x;
    const int bins = P.bins + 1;             // the last one: sequences of a single tile
    for (int b = tid; b < bins; b += nt) s_bin[b] = 0;
    if (tid == 0) {
        s_bad = s_most = 0;
        s_work = 0;
    }
    __syncthreads();
    int total = 0, many = 0, longer = 0, most = 0;
    long long sum = 0;                       // (whole numbers: the split of the backward pass hangs on it, and has to be the same from run to run)
    for (int pass = 0; pass < 2; ++pass) {
        int ahead = 0;
        for (int s0 = 0; s0 < P.n_seqs; s0 += nt) {
            if (pass == 0 || P.n_seqs > nt) {
                const int s = s0 + tid;
                int start = 0, end = 0;
                if (s < P.n_seqs) {
                    start = P.cu[s];
                    end = P.cu[s + 1];
                    if (start < 0 || end < start || end > P.T) {
                        s_bad = 1;
                        start = end = 0;
                    }
                }
                const int n = (end - start + kTile - 1) / kTile;
                const int at = block_scan(n, s_warp);
                s_first[tid] = at;
                s_start[tid] = start;
                s_len[tid] = end - start;
                if (tid == 0) s_first[nt] = s_warp[32];
                __syncthreads();
            }
            if (s_bad) break;                                // (as long as no offset decreases the tiles cannot be more than the plan has room for)
            const int count = s_first[nt];
            for (int t = tid; t < count; t += nt) {
                int lo = 0, hi = nt - 1;           // last sequence whose first tile is not behind t: empty ones have their successor's
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (s_first[mid] <= t) lo = mid;
                    else hi = mid - 1;
                }
                const int level = t - s_first[lo], n = (s_len[lo] + kTile - 1) / kTile;
                const int work = P.causal ? level + 1 : n, bin = n == 1 ? P.bins : P.bins - min(work, P.bins);      // bin 0: the most work
                if (pass == 0) {
                    atomicAdd(&s_bin[bin], 1);
                    if (n > 1) {
                        most = max(most, work);
                        sum += work;
                    }
                } else {
                    const int to = atomicAdd(&s_bin[bin], 1);
                    if (to < P.cap) reinterpret_cast<int4*>(P.plan + kWsHeaderBytes / 4)[to] = make_int4(s_start[lo], s_len[lo], level, ahead + s_first[lo]);
                }
            }
            ahead += count;
            __syncthreads();
        }
        if (s_bad) break;
        if (pass == 0) {
            most = __reduce_max_sync(0xffffffffu, most);
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if ((tid & 31) == 0 && most > 0) {
                atomicMax(&s_most, most);
                atomicAdd(&s_work, static_cast<unsigned long long>(sum));
            }
            total = ahead;
            int run = 0;
            for (int b0 = 0; b0 < bins; b0 += nt) {
                const int b = b0 + tid, v = b < bins ? s_bin[b] : 0;
                const int at = block_scan(v, s_warp);
                if (b < bins) s_bin[b] = run + at;
                run += s_warp[32];
            }
            __syncthreads();
            many = P.bins > kFewTiles ? s_bin[P.bins - kFewTiles] : 0;      // where the tiles with that much work begin
            longer = s_bin[P.bins];
            __syncthreads();
        }
    }
    if (tid == 0) {
        const bool bad = s_bad || total > P.cap;
        P.plan[kPlanStatus] = bad ? VARDROP_ERR_INVALID_ARG : VARDROP_OK;
        P.plan[kPlanMagicWord] = kPlanMagic;
        P.plan[kPlanTiles] = bad ? 0 : total;
        P.plan[kPlanSeqs] = P.n_seqs;
        P.plan[kPlanRows] = P.T;
        P.plan[kPlanCausal] = P.causal;
        P.plan[kPlanMany] = bad ? 0 : many;
        P.plan[kPlanLong] = bad ? 0 : longer;
        P.plan[kPlanMostWork] = bad ? 0 : s_most;
        P.plan[kPlanWork] = bad ? 0 : __float_as_int(static_cast<float>(s_work));
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode(CUtensorMap* map, CUtensorMapDataType type, const void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    static const EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        const bool found = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) == cudaSuccess && qres == cudaDriverEntryPointSuccess;
        return found ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
    }();
    if (!fn) return fail(VARDROP_ERR_CUDA, "packed attention: cuTensorMapEncodeTiled entry point not available");
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = fn(map, type, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? VARDROP_OK : fail(VARDROP_ERR_CUDA, "packed attention: cuTensorMapEncodeTiled failed with code %d", static_cast<int>(r));
}

}  // namespace

int packed_tile_map(CUtensorMap* map, const void* base, int D, int H, int T, long long sT, long long sH) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(H), static_cast<cuuint64_t>(T)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(sH) * 2, static_cast<cuuint64_t>(sT) * 2};
    const cuuint32_t box[3] = {kDP, 1, kTile};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, dims, strides, box);
}
int packed_acc_map(CUtensorMap* map, const void* base, int rows, int H, int D) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(H), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[2] = {D * 4ull, static_cast<cuuint64_t>(H) * D * 4};
    const cuuint32_t box[3] = {32, 1, kTile};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, base, dims, strides, box);
}

int packed_validate(const vardrop_packed_cfg& c) {
    if (c.n_seqs < 1 || c.T < 1 || c.Hq < 1 || c.Hkv < 1) return fail(VARDROP_ERR_INVALID_ARG, "packed attention: n_seqs, T, Hq, Hkv >= 1 required (%d, %d, %d, %d)", c.n_seqs, c.T, c.Hq, c.Hkv);
    if (c.Hq % c.Hkv) return fail(VARDROP_ERR_INVALID_ARG, "packed attention: Hq=%d is no multiple of Hkv=%d", c.Hq, c.Hkv);
    if (c.D != 32 && c.D != 64) return fail(VARDROP_ERR_UNSUPPORTED, "packed attention: head dimension %d (32 or 64 supported)", c.D);
    if (c.T > (1 << 24) || c.n_seqs > (1 << 24)) return fail(VARDROP_ERR_UNSUPPORTED, "packed attention: T=%d or n_seqs=%d above 2^24", c.T, c.n_seqs);
    if (c.Hq > 4096) return fail(VARDROP_ERR_UNSUPPORTED, "packed attention: Hq=%d above 4096", c.Hq);
    if (packed_tiles(c) * kTile >= (1ll << 31) || packed_tiles(c) * c.Hq >= (1ll << 31)) return fail(VARDROP_ERR_UNSUPPORTED, "packed attention: too many tiles of T=%d n_seqs=%d Hq=%d", c.T, c.n_seqs, c.Hq);
    if (c.causal != 0 && c.causal != 1) return fail(VARDROP_ERR_INVALID_ARG, "packed attention: causal=%d must be 0 or 1", c.causal);
    if (!(c.sm_scale >= 0.f) || c.sm_scale > 1e30f) return fail(VARDROP_ERR_INVALID_ARG, "packed attention: sm_scale must be >= 0 (0 selects 1/sqrt(D)) and at most 1e30");
    const PackedStrides s = packed_strides(c);
    const int64_t pairs[2][2] = {{s.sTq, s.sHq}, {s.sTkv, s.sHkv}};
    for (const auto& p : pairs) {
        if (p[1] < c.D || p[0] < p[1] || (p[0] | p[1]) % 8 != 0)
            return fail(VARDROP_ERR_INVALID_ARG, "packed attention: strides %lld of a token, %lld of a head must be multiples of 8 with token >= head >= D (or both 0)",
                        static_cast<long long>(p[0]), static_cast<long long>(p[1]));
        if (p[0] > (1ll << 32)) return fail(VARDROP_ERR_UNSUPPORTED, "packed attention: token stride above 2^32 elements");
    }
    return VARDROP_OK;
}

size_t packed_plan_bytes(const vardrop_packed_cfg& c) { return kWsHeaderBytes + static_cast<size_t>(packed_tiles(c)) * sizeof(PlanEntry); }
size_t attn_packed_workspace_bytes(const vardrop_packed_cfg& c) { return packed_layout(c).total; }

int packed_plan_launch(const int32_t* cu_seqlens, const vardrop_packed_cfg& c, void* plan, cudaStream_t stream) {
    PlanParams P{};
    P.cu = cu_seqlens; P.plan = static_cast<int32_t*>(plan);
    P.n_seqs = c.n_seqs; P.T = c.T; P.causal = c.causal;
    const int longest = (c.T + kTile - 1) / kTile;
    P.bins = longest < kPlanBins ? longest : kPlanBins;
    P.cap = packed_tiles(c);
    LaunchScope ls_(K_PACKED_PLAN, stream);
    return check_cuda(launch_chained(packed_plan_kernel, dim3(1), dim3(c.n_seqs <= 128 ? 128 : kPlanThreads), 0, stream, P), "packed attention: plan launch");
}

}  // namespace vardrop
