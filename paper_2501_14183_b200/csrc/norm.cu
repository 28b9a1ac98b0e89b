// Norms before and after a block: checks, launches, and the last step of the parameters' gradients (the other kernels: norm_kernels.cuh).
//
// norm_params_kernel     sums over tokens of all CTAs, in a fixed order.
#include "norm.h"

namespace vardrop {

namespace {

// ---- parameters' gradients ----------------------------------------------------------------------------------------------------
struct ParamsParams {
    const float* partial;
    const float *gate, *w_post, *b_post;
    float *d_gate, *d_w_post, *d_b_post, *d_w_pre, *d_b_pre;
    const int32_t* begin;
    int B, C, gate_rows, slots, ctas, layer, splits;       // splits: CTAs of an instance, 0 where runs go over instances
};
// CTA that has token r of K, where `ctas` share them
__device__ __forceinline__ int cta_of(long long r, long long K, int ctas) { return static_cast<int>(((r + 1) * ctas - 1) / K); }
// Places of an instance's sums: from `first` to `last`, none where the second is smaller.
struct Places {
    int first, last;
};
__device__ __forceinline__ Places places_of(const ParamsParams& P, int b) {
    if (P.splits) return Places{b * P.splits, (b + 1) * P.splits - 1};
    const long long lo = P.begin[b], hi = P.begin[b + 1], K = P.begin[P.B];
    if (lo >= hi) return Places{0, -1};
    const int ctas = static_cast<int>(min(K, static_cast<long long>(P.ctas)));
    return Places{cta_of(lo, K, ctas) + b, cta_of(hi - 1, K, ctas) + b};
}
constexpr int kColsX = 32, kColsY = 32;
// Blocks (x, 0): 32 columns of the first two sums over all tokens; (x, 1): of the last two; (x, 2 + k): of the gates of instances 32 k to 32 k + 31.  32 rows at a time,
// then across them, in a fixed order.
__global__ void __launch_bounds__(kColsX * kColsY) norm_params_kernel(const ParamsParams P) {
    __shared__ float s[2][kColsY][kColsX + 1];
    chain_wait();
    chain_release();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * kColsX + x;
    const bool there = c < P.C, per = P.gate_rows > 1;
    const size_t C = P.C;
    if (blockIdx.y >= 2) {
        const int b = (blockIdx.y - 2) * kColsY + y;
        if (!there || b >= P.gate_rows) return;
        const float w = P.w_post ? __ldg(P.w_post + c) : 1.f, bias = P.b_post ? __ldg(P.b_post + c) : 0.f;
        const float* A = P.partial + c;
        const float* T = A + P.slots * C;
        const Places at = places_of(P, b);
        float a = 0.f, t = 0.f;
#pragma unroll 4
        for (int r = at.first; r <= at.last; ++r) {
            a += A[r * C];
            if (P.layer) t += T[r * C];
        }
        P.d_gate[b * C + c] = fmaf(w, a, bias * t);
        return;
    }
    const bool last = blockIdx.y == 1;
    const int rows = last ? P.ctas : P.slots;
    const float* A = P.partial + (last ? 2 * P.slots * C : 0) + c;
    const float* T = A + rows * C;
    float v0 = 0.f, v1 = 0.f;
    if (there && !last && per) {            // by instances, times their gates; a few of them are shared by lanes
        const int subs = P.B < kColsY ? kColsY / P.B : 1, sub = y % subs;
        for (int b = y / subs; b < P.B; b += kColsY / subs) {
            const Places at = places_of(P, b);
            const float g = __ldg(P.gate + static_cast<size_t>(b) * C + c);
#pragma unroll 4
            for (int r = at.first + sub; r <= at.last; r += subs) {
                v0 += g * A[r * C];
                if (P.layer) v1 += g * T[r * C];
            }
        }
    } else if (there) {
#pragma unroll 8
        for (int r = y; r < rows; r += kColsY) {
            v0 += A[r * C];
            if (P.layer) v1 += T[r * C];
        }
    }
    s[0][y][x] = v0;
    s[1][y][x] = v1;
    __syncthreads();
    if (y < 2) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < kColsY; ++r) sum += s[y][r][x];
        s[y][0][x] = sum;                                // (its column: nobody else reads it ahead of the barrier)
    }
    __syncthreads();
    if (y != 0 || !there) return;
    const float a = s[0][0][x], t = s[1][0][x];
    if (last) {
        if (P.d_w_pre) P.d_w_pre[c] = a;
        if (P.d_b_pre) P.d_b_pre[c] = t;
        return;
    }
    const float g = P.gate && !per ? P.gate[c] : 1.f;
    if (P.d_gate && !per) P.d_gate[c] = fmaf(P.w_post ? P.w_post[c] : 1.f, a, (P.b_post ? P.b_post[c] : 0.f) * t);
    if (P.d_w_post) P.d_w_post[c] = g * a;
    if (P.d_b_post) P.d_b_post[c] = g * t;
}

// ---- launches -------------------------------------------------------------------------------------------------------------------
// CTAs: as many as keep every SM's places taken without a second round, but none without a token.
struct Shares {
    NormShare share;
    int splits, grid;
};
Shares shares(const vardrop_norm_cfg& c, bool selected, int per, int per_sm) {
    const int group = group_of(c.C, per), threads = group < 256 ? 256 : group, groups = threads / group;
    const long long places = static_cast<long long>(sm_count()) * per_sm * 256 / threads, all = static_cast<long long>(c.B) * c.N;
    auto at_most = [&](long long n) { return static_cast<int>(n < places ? (n > 0 ? n : 1) : places > 0 ? places : 1); };
    if (!selected && c.gate_rows <= 1) return Shares{kFlat, 0, at_most((all + groups - 1) / groups)};
    // a run is worked off instance by instance: CTAs for shorter runs where instances have few tokens (37 x 2 x 157 with one or two kept, forward and backward, 13.5 us instead of 25.6)
    if (selected && c.S > 1) return Shares{kRuns, 0, at_most((all + groups - 1) / groups + c.B)};
    const long long most = (static_cast<long long>(c.N) + groups - 1) / groups, even = places / c.B;
    const int splits = static_cast<int>(even < 1 ? 1 : even < most ? even : most);
    return Shares{kSplit, splits, at_most(static_cast<long long>(c.B) * splits)};
}
constexpr int kFwdPerSm = 2, kBwdPerSm = 2;              // CTAs of 256 threads that an SM holds

cudaError_t launch_type(bool bwd, int dtype, int grid, const NormParams& P, cudaStream_t s) {
    return dtype == 0 ? norm_launch_bf16(bwd, grid, P, s) : dtype == 1 ? norm_launch_fp16(bwd, grid, P, s) : norm_launch_fp32(bwd, grid, P, s);
}
NormParams params_of(const vardrop_norm_cfg& c, const int32_t* sel_idx) {
    NormParams P{};
    P.B = c.B; P.N = c.N; P.C = c.C; P.pre = c.pre; P.post = c.post; P.gate_rows = c.gate_rows;
    P.S = sel_idx && c.S > 1 ? c.S : 1;
    P.scale = c.res_scale; P.eps = c.eps; P.inv_c = 1.f / static_cast<float>(c.C);
    return P;
}

}  // namespace

int norm_validate(const vardrop_norm_cfg& c) {
    if (c.B < 1 || c.N < 1 || c.C < 1) return fail(VARDROP_ERR_INVALID_ARG, "norm: B, N, C >= 1 required (B=%d N=%d C=%d)", c.B, c.N, c.C);
    if (c.C > kNormMaxC) return fail(VARDROP_ERR_UNSUPPORTED, "norm: C=%d above %d", c.C, kNormMaxC);
    if (static_cast<long long>(c.B) * c.N >= (1ll << 31)) return fail(VARDROP_ERR_UNSUPPORTED, "norm: B*N above 2^31");
    if (c.dtype < 0 || c.dtype > 2) return fail(VARDROP_ERR_INVALID_ARG, "norm: type %d (0 bf16, 1 fp16, 2 fp32)", c.dtype);
    if (c.pre < 0 || c.pre > 2 || c.post < 0 || c.post > 2) return fail(VARDROP_ERR_INVALID_ARG, "norm: kinds pre=%d post=%d (0 none, 1 rms, 2 layer)", c.pre, c.post);
    if (c.gate_rows != 0 && c.gate_rows != 1 && c.gate_rows != c.B) return fail(VARDROP_ERR_INVALID_ARG, "norm: gate_rows=%d must be 0, 1 or B", c.gate_rows);
    if (c.gate_rows > 65534) return fail(VARDROP_ERR_UNSUPPORTED, "norm: gate_rows=%d above 65534", c.gate_rows);
    if (c.S != 0 && c.S != 1 && c.S != c.B) return fail(VARDROP_ERR_INVALID_ARG, "norm: S=%d must be 1 (shared selection) or B (one per instance)", c.S);
    if (!isfinite(c.res_scale) || !(c.eps >= 0.f) || !isfinite(c.eps)) return fail(VARDROP_ERR_INVALID_ARG, "norm: res_scale and eps >= 0 must be finite");
    return VARDROP_OK;
}

int norm_fwd_launch(const void* x, const void* y, const float* gate, const float* w_post, const float* b_post, const float* w_pre, const float* b_pre, const int32_t* sel_idx,
                    const int32_t* n_sel, const vardrop_norm_cfg& c, void* h, void* u, float* stats, cudaStream_t stream) {
    const Shares w = shares(c, sel_idx != nullptr, kFwdPer, kFwdPerSm);
    const int grid = w.grid;
    NormParams P = params_of(c, sel_idx);
    P.share = w.share; P.splits = w.splits;
    P.x = x; P.y = y; P.gate = gate; P.w_post = w_post; P.b_post = b_post; P.w_pre = w_pre; P.b_pre = b_pre;
    P.sel_idx = sel_idx; P.n_sel = sel_idx ? n_sel : nullptr;
    P.h = h; P.u = u; P.stats = reinterpret_cast<float4*>(stats);
    LaunchScope ls_(K_NORM_FWD, stream);
    return check_cuda(launch_type(false, c.dtype, grid, P, stream), "norm: forward launch");
}

namespace {
// Partial sums and, with a gate an instance, where the instances begin.
struct NormWs {
    Shares s;
    int slots;
    size_t begin, partial, total;
};
NormWs norm_layout(const vardrop_norm_cfg& c, bool selected) {
    NormWs w;
    w.s = shares(c, selected, kBwdPer, kBwdPerSm);
    w.slots = c.gate_rows <= 1 ? w.s.grid : w.s.share == kRuns ? w.s.grid + c.B : c.B * w.s.splits;
    w.begin = kWsHeaderBytes;
    w.partial = w.begin + (c.gate_rows > 1 ? align_up(sizeof(int32_t) * (static_cast<size_t>(c.B) + 1), 256) : 0);
    w.total = w.partial + align_up(sizeof(float) * 2 * (static_cast<size_t>(w.slots) + w.s.grid) * c.C, 256);
    return w;
}
}  // namespace

size_t norm_workspace_bytes(const vardrop_norm_cfg& c) {         // (the query does not say whether tokens are selected)
    const size_t a = norm_layout(c, false).total, b = norm_layout(c, true).total;
    return a > b ? a : b;
}

int norm_bwd_launch(const void* x, const void* y, const float* gate, const float* w_post, const float* b_post, const float* w_pre, const int32_t* sel_idx, const int32_t* n_sel,
                    const int32_t* inv_idx, const float* stats, const void* d_h, const void* d_u, const vardrop_norm_cfg& c, void* dx, void* dy, float* d_gate, float* d_w_post,
                    float* d_b_post, float* d_w_pre, float* d_b_pre, void* ws, cudaStream_t stream) {
    const NormWs w = norm_layout(c, sel_idx != nullptr);
    const int grid = w.s.grid;
    NormParams P = params_of(c, sel_idx);
    P.share = w.s.share; P.splits = w.s.splits;
    P.x = x; P.y = y; P.gate = gate; P.w_post = w_post; P.b_post = b_post; P.w_pre = w_pre;
    P.sel_idx = sel_idx; P.n_sel = sel_idx ? n_sel : nullptr; P.inv_idx = sel_idx ? inv_idx : nullptr;
    P.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
    P.d_h = d_h; P.d_u = d_u; P.dx = dx; P.dy = dy;
    P.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + w.partial);
    P.begin = c.gate_rows > 1 && w.s.share == kRuns ? reinterpret_cast<int32_t*>(static_cast<char*>(ws) + w.begin) : nullptr;
    P.slots = w.slots;
    {
        LaunchScope ls_(K_NORM_BWD, stream);
        if (int st = check_cuda(launch_type(true, c.dtype, grid, P, stream), "norm: backward launch")) return st;
    }
    if (!d_gate && !d_w_post && !d_b_post && !d_w_pre && !d_b_pre) return VARDROP_OK;
    ParamsParams Q{P.partial, gate, w_post, b_post, d_gate, d_w_post, d_b_post, d_w_pre, d_b_pre, P.begin, c.B, c.C, c.gate_rows, P.slots, grid, c.pre == 2 || c.post == 2, w.s.share == kSplit ? w.s.splits : 0};
    LaunchScope ls_(K_NORM_PARAMS, stream);
    return check_cuda(launch_chained(norm_params_kernel, dim3((c.C + kColsX - 1) / kColsX, 2 + (d_gate && c.gate_rows > 1 ? (c.gate_rows + kColsY - 1) / kColsY : 0)), dim3(kColsX * kColsY), 0, stream, Q),
                      "norm: parameters' gradients launch");
}

}  // namespace vardrop
