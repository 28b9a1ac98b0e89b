// Norms before and after a block with its gate and residual scale: h = a x + g o N_post(y), u = N_pre(h), and their gradients.
//
// norm_fwd_kernel        a group of threads per token, its row in registers.
// norm_bwd_kernel        the same; sums over tokens stay in registers until a CTA is done with its rows.
// norm_params_kernel     those sums of all CTAs, in a fixed order.
//
// With z = (t - mean) r, e = w o d for the gradient d of N(t):  dt = r (e - mean(e) - z mean(e o z)), without mean(e) for rms.
// Bound: memory.  Forward x, y in, h, u out; backward x, y, dh, du in, dx, dy out (h again from x and y: read back as h it would come rounded, and the fp32 sums with it).
#include <cuda_fp16.h>

#include "common.cuh"
#include "kernels.h"

namespace vardrop {

namespace {

constexpr int kNormPer = 8;              // elements of a row in a thread
constexpr int kNormMaxC = 8192;

struct NormParams {
    const void *x, *y;
    const float *gate, *w_post, *b_post, *w_pre, *b_pre;
    const int32_t *sel_idx, *n_sel, *inv_idx;
    void *h, *u;
    float4* stats;
    const void *d_h, *d_u;
    void *dx, *dy;
    float* partial;                      // [4][units or CTAs, C]: sums over tokens of t o zy, t, du o zh, du
    int B, N, C, pre, post, gate_rows, S;
    int splits, units;                   // CTAs that share an instance; B splits
    int slots;                           // rows of the first two sums
    float scale, eps, inv_c;
};

// ---- elements -------------------------------------------------------------------------------------------------------------
template <class T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// A thread's columns: kNormPer / kV vectors of kV, a group's threads side by side.
template <class T, int kV, int kGroup>
struct Row {
    static constexpr int kVecs = kNormPer / kV;
    struct alignas(sizeof(T) * kV) Vec { T v[kV]; };
    static __device__ __forceinline__ int col(int t, int j) { return (j * kGroup + t) * kV; }
    static __device__ __forceinline__ void load(const T* row, int t, int C, Vec (&to)[kVecs]) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            if (col(t, j) < C) to[j] = *reinterpret_cast<const Vec*>(row + col(t, j));
            else {
#pragma unroll
                for (int e = 0; e < kV; ++e) to[j].v[e] = from_f<T>(0.f);
            }
        }
    }
    static __device__ __forceinline__ void floats(const Vec (&from)[kVecs], float (&v)[kNormPer]) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j)
#pragma unroll
            for (int e = 0; e < kV; ++e) v[j * kV + e] = to_f<T>(from[j].v[e]);
    }
    static __device__ __forceinline__ void store(T* row, int t, int C, const float (&v)[kNormPer]) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            if (col(t, j) >= C) continue;
            Vec x;
#pragma unroll
            for (int e = 0; e < kV; ++e) x.v[e] = from_f<T>(v[j * kV + e]);
            *reinterpret_cast<Vec*>(row + col(t, j)) = x;
        }
    }
    // of a parameter; `none` where there is none, 0 behind the row's end
    static __device__ __forceinline__ void param(const float* p, int t, int C, float none, float (&v)[kNormPer]) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            if (p && col(t, j) < C) {
                if (kV >= 4) {
#pragma unroll
                    for (int e = 0; e < kV; e += 4) {
                        const float4 f = __ldg(reinterpret_cast<const float4*>(p + col(t, j) + e));
                        v[j * kV + e] = f.x; v[j * kV + e + 1] = f.y; v[j * kV + e + 2] = f.z; v[j * kV + e + 3] = f.w;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < kV; ++e) v[j * kV + e] = __ldg(p + col(t, j) + e);
                }
            } else {
#pragma unroll
                for (int e = 0; e < kV; ++e) v[j * kV + e] = col(t, j) < C ? none : 0.f;
            }
        }
    }
    static __device__ __forceinline__ void param_store(float* p, int t, int C, const float (&v)[kNormPer]) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j)
            if (col(t, j) < C) {
#pragma unroll
                for (int e = 0; e < kV; ++e) p[col(t, j) + e] = v[j * kV + e];
            }
    }
};

// ---- sums over a group ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Two sums at once, to every thread of the group.  Groups of several warps go through shared memory, in two places by turns, so that one barrier a sum is enough.
template <int kGroup>
struct GroupSum {
    float2* place;                       // [2][kGroup / 32] of this group
    int turn = 0, id;
    __device__ __forceinline__ float2 operator()(float a, float b) {
        a = warp_sum(a);
        b = warp_sum(b);
        if (kGroup == 32) return make_float2(a, b);
        constexpr int kWarps = kGroup / 32;
        const int lane = threadIdx.x & 31, warp = (threadIdx.x % kGroup) >> 5;
        float2* at = place + turn * kWarps;
        turn ^= 1;
        if (lane == 0) at[warp] = make_float2(a, b);
        asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kGroup) : "memory");
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            s.x += at[w].x;
            s.y += at[w].y;
        }
        return s;
    }
};

template <int kGroup>
constexpr int kNormThreads = kGroup < 256 ? 256 : kGroup;        // of a CTA

// z = (t - mean) r in place; (mean, r)
template <class R, int kGroup>
__device__ __forceinline__ float2 normalise(float (&t)[kNormPer], int kind, int thread, const NormParams& P, GroupSum<kGroup>& sum) {
    float mean = 0.f;
    if (kind == 2) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < kNormPer; ++e) s += t[e];
        mean = sum(s, 0.f).x * P.inv_c;
    }
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < R::kVecs; ++j) {
        if (R::col(thread, j) >= P.C) continue;          // (zeros there, but not once the mean is off)
#pragma unroll
        for (int e = j * (kNormPer / R::kVecs); e < (j + 1) * (kNormPer / R::kVecs); ++e) {
            t[e] -= mean;
            q += t[e] * t[e];
        }
    }
    const float r = rsqrtf(sum(q, 0.f).x * P.inv_c + P.eps);
#pragma unroll
    for (int e = 0; e < kNormPer; ++e) t[e] *= r;
    return make_float2(mean, r);
}

// ---- forward ----------------------------------------------------------------------------------------------------------------
template <class T, int kV, int kGroup>
__global__ void __launch_bounds__(kNormThreads<kGroup>) norm_fwd_kernel(const NormParams P) {
    using R = Row<T, kV, kGroup>;
    constexpr int kGroups = kNormThreads<kGroup> / kGroup;
    __shared__ float2 s_sum[kGroups][2 * (kGroup / 32)];
    const int group = threadIdx.x / kGroup, t = threadIdx.x % kGroup;
    GroupSum<kGroup> sum{s_sum[group], 0, 1 + group};
    chain_wait();
    chain_release();
#pragma unroll 1
    for (int unit = blockIdx.x; unit < P.units; unit += gridDim.x) {
        const int b = unit / P.splits, srow = P.S > 1 ? b : 0;
        const int n = P.n_sel ? P.n_sel[srow] : P.N;
        const int32_t* sel = P.sel_idx ? P.sel_idx + static_cast<size_t>(srow) * P.N : nullptr;
        const float* gate = P.gate ? P.gate + static_cast<size_t>(P.gate_rows > 1 ? b : 0) * P.C : nullptr;
#pragma unroll 1
        for (int i = (unit - b * P.splits) * kGroups + group; i < n; i += P.splits * kGroups) {
            const size_t row = (static_cast<size_t>(b) * P.N + i) * P.C;
            const size_t from = sel ? (static_cast<size_t>(b) * P.N + sel[i]) * P.C : row;
            typename R::Vec vx[R::kVecs], vy[R::kVecs];
            R::load(static_cast<const T*>(P.x) + from, t, P.C, vx);
            float2 post = make_float2(0.f, 1.f), pre = post;
            float h[kNormPer], w[kNormPer];
            R::floats(vx, h);
#pragma unroll
            for (int e = 0; e < kNormPer; ++e) h[e] *= P.scale;
            if (P.y) {
                R::load(static_cast<const T*>(P.y) + row, t, P.C, vy);
                float y[kNormPer], g[kNormPer];
                R::floats(vy, y);
                if (P.post) {
                    post = normalise<R, kGroup>(y, P.post, t, P, sum);
                    R::param(P.w_post, t, P.C, 1.f, w);
                    R::param(P.b_post, t, P.C, 0.f, g);
#pragma unroll
                    for (int e = 0; e < kNormPer; ++e) y[e] = fmaf(y[e], w[e], g[e]);
                }
                R::param(gate, t, P.C, 1.f, g);
#pragma unroll
                for (int e = 0; e < kNormPer; ++e) h[e] = fmaf(g[e], y[e], h[e]);
            }
            if (P.h) R::store(static_cast<T*>(P.h) + row, t, P.C, h);
            if (P.pre) {
                pre = normalise<R, kGroup>(h, P.pre, t, P, sum);
                float bias[kNormPer];
                R::param(P.w_pre, t, P.C, 1.f, w);
                R::param(P.b_pre, t, P.C, 0.f, bias);
#pragma unroll
                for (int e = 0; e < kNormPer; ++e) h[e] = fmaf(h[e], w[e], bias[e]);
                R::store(static_cast<T*>(P.u) + row, t, P.C, h);
            }
            if (P.stats && t == 0) P.stats[static_cast<size_t>(b) * P.N + i] = make_float4(post.x, post.y, pre.x, pre.y);
        }
    }
}

// ---- backward ---------------------------------------------------------------------------------------------------------------
// Sums over tokens: with t the gradient of h, zy and zh the normed y and h:
//   d_gate = w_post o A + b_post o T,  d_w_post = sum_b g_b o A_b,  d_b_post = sum_b g_b o T_b   with A = sum t o zy, T = sum t over the tokens of an instance,
//   d_w_pre = sum du o zh,  d_b_pre = sum du
// so a thread keeps four sums a column however many parameters there are.  (A gate that all instances share needs them over all tokens only.)
template <class T, int kV, int kGroup>
__global__ void __launch_bounds__(kNormThreads<kGroup>) norm_bwd_kernel(const NormParams P) {
    using R = Row<T, kV, kGroup>;
    constexpr int kGroups = kNormThreads<kGroup> / kGroup;
    __shared__ float2 s_sum[kGroups][2 * (kGroup / 32)];
    __shared__ float s_cols[kGroups > 1 ? kGroups : 1][kGroups > 1 ? kGroup * kNormPer : 1];
    const int group = threadIdx.x / kGroup, t = threadIdx.x % kGroup;
    GroupSum<kGroup> sum{s_sum[group], 0, 1 + group};
    chain_wait();
    chain_release();
    float acc[4][kNormPer];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < kNormPer; ++e) acc[k][e] = 0.f;
    // sums k0 and k0 + 1 of all groups to row `at` of their partial sums
    auto flush = [&](int k0, int at) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float (&a)[kNormPer] = acc[k0 + k];
            if (kGroups > 1) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < kNormPer; ++e) s_cols[group][e * kGroup + t] = a[e];
                __syncthreads();
                if (group == 0) {
#pragma unroll 1
                    for (int g = 1; g < kGroups; ++g)
#pragma unroll
                        for (int e = 0; e < kNormPer; ++e) a[e] += s_cols[g][e * kGroup + t];
                }
            }
            if (group == 0) R::param_store(P.partial + (static_cast<size_t>(k0 == 0 ? k * P.slots : 2 * P.slots + k * gridDim.x) + at) * P.C, t, P.C, a);
#pragma unroll
            for (int e = 0; e < kNormPer; ++e) a[e] = 0.f;
        }
    };
#pragma unroll 1
    for (int unit = blockIdx.x; unit < P.units; unit += gridDim.x) {
        const int b = unit / P.splits, srow = P.S > 1 ? b : 0;
        const int n = P.n_sel ? P.n_sel[srow] : P.N;
        const int32_t* sel = P.sel_idx ? P.sel_idx + static_cast<size_t>(srow) * P.N : nullptr;
        const float* gate = P.gate ? P.gate + static_cast<size_t>(P.gate_rows > 1 ? b : 0) * P.C : nullptr;
        const int first = (unit - b * P.splits) * kGroups + group, step = P.splits * kGroups;
        if (sel) {                                       // rows of dropped tokens
            const float zero[kNormPer] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int i = first; i < P.N; i += step)
                if (P.inv_idx[static_cast<size_t>(srow) * P.N + i] < 0) R::store(static_cast<T*>(P.dx) + (static_cast<size_t>(b) * P.N + i) * P.C, t, P.C, zero);
        }
#pragma unroll 1
        for (int i = first; i < n; i += step) {
            const size_t row = (static_cast<size_t>(b) * P.N + i) * P.C;
            const size_t from = sel ? (static_cast<size_t>(b) * P.N + sel[i]) * P.C : row;
            const float4 st = P.stats[static_cast<size_t>(b) * P.N + i];
            typename R::Vec v[R::kVecs];
            float h[kNormPer], zy[kNormPer], g[kNormPer], d[kNormPer], w[kNormPer];
            R::load(static_cast<const T*>(P.x) + from, t, P.C, v);
            R::floats(v, h);
#pragma unroll
            for (int e = 0; e < kNormPer; ++e) h[e] *= P.scale;
            R::param(gate, t, P.C, 1.f, g);
            if (P.y) {
                R::load(static_cast<const T*>(P.y) + row, t, P.C, v);
                R::floats(v, zy);
                float bias[kNormPer];
                R::param(P.w_post, t, P.C, 1.f, w);
                R::param(P.b_post, t, P.C, 0.f, bias);
                if (P.post) {
#pragma unroll
                    for (int e = 0; e < kNormPer; ++e) zy[e] = (zy[e] - st.x) * st.y;
                }
#pragma unroll
                for (int e = 0; e < kNormPer; ++e) h[e] = fmaf(g[e], fmaf(zy[e], w[e], bias[e]), h[e]);
            }
            if (P.d_h) {
                R::load(static_cast<const T*>(P.d_h) + row, t, P.C, v);
                R::floats(v, d);
            } else {
#pragma unroll
                for (int e = 0; e < kNormPer; ++e) d[e] = 0.f;
            }
            if (P.pre) {
                float du[kNormPer], wp[kNormPer];
                R::load(static_cast<const T*>(P.d_u) + row, t, P.C, v);
                R::floats(v, du);
                R::param(P.w_pre, t, P.C, 1.f, wp);
                float s0 = 0.f, s1 = 0.f;
#pragma unroll
                for (int e = 0; e < kNormPer; ++e) {
                    h[e] = (h[e] - st.z) * st.w;         // (where no column is, du is 0)
                    acc[2][e] += du[e] * h[e];
                    acc[3][e] += du[e];
                    du[e] *= wp[e];
                    s0 += du[e] * h[e];
                    s1 += du[e];
                }
                const float2 s = sum(s0, s1);
                const float m0 = s.x * P.inv_c, m1 = P.pre == 2 ? s.y * P.inv_c : 0.f;
#pragma unroll
                for (int e = 0; e < kNormPer; ++e) d[e] = fmaf(st.w, du[e] - m1 - h[e] * m0, d[e]);
            }
            float out[kNormPer];
#pragma unroll
            for (int e = 0; e < kNormPer; ++e) out[e] = P.scale * d[e];
            R::store(static_cast<T*>(P.dx) + from, t, P.C, out);
            if (P.y) {
                float s0 = 0.f, s1 = 0.f;
#pragma unroll
                for (int e = 0; e < kNormPer; ++e) {
                    acc[0][e] += d[e] * zy[e];
                    acc[1][e] += d[e];
                    d[e] *= g[e];
                }
                if (P.post) {
                    R::param(P.w_post, t, P.C, 1.f, w);
#pragma unroll
                    for (int e = 0; e < kNormPer; ++e) {
                        d[e] *= w[e];                    // (0 where no column is)
                        s0 += d[e] * zy[e];
                        s1 += d[e];
                    }
                    const float2 s = sum(s0, s1);
                    const float m0 = s.x * P.inv_c, m1 = P.post == 2 ? s.y * P.inv_c : 0.f;
#pragma unroll
                    for (int e = 0; e < kNormPer; ++e) d[e] = st.y * (d[e] - m1 - zy[e] * m0);
                }
                R::store(static_cast<T*>(P.dy) + row, t, P.C, d);
            }
        }
        if (P.gate_rows > 1) flush(0, unit);
    }
    if (P.gate_rows <= 1) flush(0, blockIdx.x);
    flush(2, blockIdx.x);
}

// ---- parameters' gradients ----------------------------------------------------------------------------------------------------
struct ParamsParams {
    const float* partial;
    const float *gate, *w_post, *b_post;
    float *d_gate, *d_w_post, *d_b_post, *d_w_pre, *d_b_pre;
    int B, C, gate_rows, splits, slots, ctas;
};
constexpr int kColsX = 32, kColsY = 32;
// Blocks (x, 0): 32 columns of the sums over all tokens; (x, 1 + b): of an instance's gate.  32 rows at a time, then across them, in a fixed order.
__global__ void __launch_bounds__(kColsX * kColsY) norm_params_kernel(const ParamsParams P) {
    __shared__ float s[4][kColsY][kColsX + 1];
    chain_wait();
    chain_release();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * kColsX + x;
    const bool there = c < P.C;
    const bool one = blockIdx.y == 0, per = P.gate_rows > 1;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    const float* A = P.partial + c;
    const float* Tt = A + static_cast<size_t>(P.slots) * P.C;
    const float* U = Tt + static_cast<size_t>(P.slots) * P.C;
    const float* V = U + static_cast<size_t>(P.ctas) * P.C;
    if (there && one) {
        for (int r = y; r < P.slots; r += kColsY) {
            const float g = per ? __ldg(P.gate + static_cast<size_t>(r / P.splits) * P.C + c) : 1.f;
            v[0] += g * A[static_cast<size_t>(r) * P.C];
            v[1] += g * Tt[static_cast<size_t>(r) * P.C];
        }
        for (int r = y; r < P.ctas; r += kColsY) {
            v[2] += U[static_cast<size_t>(r) * P.C];
            v[3] += V[static_cast<size_t>(r) * P.C];
        }
    } else if (there) {
        const int b = blockIdx.y - 1;
        for (int r = b * P.splits + y; r < (b + 1) * P.splits; r += kColsY) {
            v[0] += A[static_cast<size_t>(r) * P.C];
            v[1] += Tt[static_cast<size_t>(r) * P.C];
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k][y][x] = v[k];
    __syncthreads();
    if (y < 4) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < kColsY; ++r) sum += s[y][r][x];
        s[y][0][x] = sum;                                // (its column: nobody else reads it ahead of the barrier)
    }
    __syncthreads();
    if (y != 0 || !there) return;
    const float a = s[0][0][x], t = s[1][0][x];
    const float w = P.w_post ? P.w_post[c] : 1.f, bias = P.b_post ? P.b_post[c] : 0.f;
    if (!one) {
        P.d_gate[static_cast<size_t>(blockIdx.y - 1) * P.C + c] = fmaf(w, a, bias * t);
        return;
    }
    const float g = P.gate && !per ? P.gate[c] : 1.f;
    if (P.d_gate && !per) P.d_gate[c] = fmaf(w, a, bias * t);
    if (P.d_w_post) P.d_w_post[c] = g * a;
    if (P.d_b_post) P.d_b_post[c] = g * t;
    if (P.d_w_pre) P.d_w_pre[c] = s[2][0][x];
    if (P.d_b_pre) P.d_b_pre[c] = s[3][0][x];
}

// ---- launches -------------------------------------------------------------------------------------------------------------------
int group_of(int C) {
    int g = 32;
    while (g * kNormPer < C) g *= 2;
    return g;
}
// CTAs that share an instance's tokens, as many as keep every SM's places taken without a second round, but none without a token.
void shares(const vardrop_norm_cfg& c, int per_sm, int& splits, int& grid) {
    const int group = group_of(c.C), threads = group < 256 ? 256 : group, groups = threads / group;
    const int places = sm_count() * per_sm * 256 / threads;
    const int most = (c.N + groups - 1) / groups;
    splits = places / c.B;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    const long long units = static_cast<long long>(c.B) * splits;
    grid = static_cast<int>(units < places ? units : places);
    if (grid < 1) grid = 1;
}
constexpr int kFwdPerSm = 6, kBwdPerSm = 2;              // CTAs of 256 threads

template <class T, int kV, int kGroup>
cudaError_t launch(bool bwd, int grid, const NormParams& P, cudaStream_t s) {
    constexpr int kThreads = kNormThreads<kGroup>;
    return bwd ? launch_chained(norm_bwd_kernel<T, kV, kGroup>, dim3(grid), dim3(kThreads), 0, s, P) : launch_chained(norm_fwd_kernel<T, kV, kGroup>, dim3(grid), dim3(kThreads), 0, s, P);
}
template <class T, int kV>
cudaError_t launch_group(bool bwd, int grid, const NormParams& P, cudaStream_t s) {
    switch (group_of(P.C)) {
        case 32: return launch<T, kV, 32>(bwd, grid, P, s);
        case 64: return launch<T, kV, 64>(bwd, grid, P, s);
        case 128: return launch<T, kV, 128>(bwd, grid, P, s);
        case 256: return launch<T, kV, 256>(bwd, grid, P, s);
        case 512: return launch<T, kV, 512>(bwd, grid, P, s);
        default: return launch<T, kV, 1024>(bwd, grid, P, s);
    }
}
// Vectors of 16 bytes where every row begins on such a boundary, single elements otherwise.
cudaError_t launch_type(bool bwd, int dtype, int grid, const NormParams& P, cudaStream_t s) {
    const bool wide = P.C % (dtype == 2 ? 4 : 8) == 0;
    if (dtype == 0) return wide ? launch_group<__nv_bfloat16, 8>(bwd, grid, P, s) : launch_group<__nv_bfloat16, 1>(bwd, grid, P, s);
    if (dtype == 1) return wide ? launch_group<__half, 8>(bwd, grid, P, s) : launch_group<__half, 1>(bwd, grid, P, s);
    return wide ? launch_group<float, 4>(bwd, grid, P, s) : launch_group<float, 1>(bwd, grid, P, s);
}
NormParams params_of(const vardrop_norm_cfg& c, const int32_t* sel_idx, int splits) {
    NormParams P{};
    P.B = c.B; P.N = c.N; P.C = c.C; P.pre = c.pre; P.post = c.post; P.gate_rows = c.gate_rows;
    P.S = sel_idx && c.S > 1 ? c.S : 1;
    P.splits = splits; P.units = c.B * splits;
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
    int splits, grid;
    shares(c, kFwdPerSm, splits, grid);
    NormParams P = params_of(c, sel_idx, splits);
    P.x = x; P.y = y; P.gate = gate; P.w_post = w_post; P.b_post = b_post; P.w_pre = w_pre; P.b_pre = b_pre;
    P.sel_idx = sel_idx; P.n_sel = sel_idx ? n_sel : nullptr;
    P.h = h; P.u = u; P.stats = reinterpret_cast<float4*>(stats);
    LaunchScope ls_(K_NORM_FWD, stream);
    return check_cuda(launch_type(false, c.dtype, grid, P, stream), "norm: forward launch");
}

size_t norm_workspace_bytes(const vardrop_norm_cfg& c) {
    int splits, grid;
    shares(c, kBwdPerSm, splits, grid);
    const size_t slots = c.gate_rows > 1 ? static_cast<size_t>(c.B) * splits : grid;
    return kWsHeaderBytes + align_up(sizeof(float) * 2 * (slots + grid) * c.C, 256);
}

int norm_bwd_launch(const void* x, const void* y, const float* gate, const float* w_post, const float* b_post, const float* w_pre, const int32_t* sel_idx, const int32_t* n_sel,
                    const int32_t* inv_idx, const float* stats, const void* d_h, const void* d_u, const vardrop_norm_cfg& c, void* dx, void* dy, float* d_gate, float* d_w_post,
                    float* d_b_post, float* d_w_pre, float* d_b_pre, void* ws, cudaStream_t stream) {
    int splits, grid;
    shares(c, kBwdPerSm, splits, grid);
    NormParams P = params_of(c, sel_idx, splits);
    P.x = x; P.y = y; P.gate = gate; P.w_post = w_post; P.b_post = b_post; P.w_pre = w_pre;
    P.sel_idx = sel_idx; P.n_sel = sel_idx ? n_sel : nullptr; P.inv_idx = sel_idx ? inv_idx : nullptr;
    P.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
    P.d_h = d_h; P.d_u = d_u; P.dx = dx; P.dy = dy;
    P.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + kWsHeaderBytes);
    P.slots = c.gate_rows > 1 ? P.units : grid;
    {
        LaunchScope ls_(K_NORM_BWD, stream);
        if (int st = check_cuda(launch_type(true, c.dtype, grid, P, stream), "norm: backward launch")) return st;
    }
    if (!d_gate && !d_w_post && !d_b_post && !d_w_pre && !d_b_pre) return VARDROP_OK;
    ParamsParams Q{P.partial, gate, w_post, b_post, d_gate, d_w_post, d_b_post, d_w_pre, d_b_pre, c.B, c.C, c.gate_rows, splits, P.slots, grid};
    LaunchScope ls_(K_NORM_PARAMS, stream);
    return check_cuda(launch_chained(norm_params_kernel, dim3((c.C + kColsX - 1) / kColsX, 1 + (d_gate && c.gate_rows > 1 ? c.gate_rows : 0)), dim3(kColsX * kColsY), 0, stream, Q),
                      "norm: parameters' gradients launch");
}

}  // namespace vardrop
