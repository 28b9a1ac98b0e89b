// The feed-forward's activation, y = f(a) or f(a) o b, with a checkpoint of a (and b) in 8 bits from which the backward pass works:
//   d_a = d_y o b o f'(a),  d_b = d_y o f(a),  y = f(a) o b once more (for the weight gradient of the projection behind it)
//
// act_fwd_kernel, act_bwd_kernel    32 values of a row share a power of two, the smallest 2^e with max |a| <= 448 2^e; a value is an e4m3 of that scale, so it is off by at most 2^-4 of itself (or
//                                   2^(e-10) where it is below 2^(e-6)).  A power of two costs no rounding of its own, and what 8 bits stand for is exact in the tensor's type.
//
// Bound: memory (bf16, gated: 4 bytes in, 2 and two codes out a value forward, 2 and two codes in and 6 out backward); gelu's backward pass is near the instruction rate as well.
#include <cuda_fp8.h>

#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "packed_math.cuh"
#include "vec_io.cuh"

namespace vardrop {

namespace {

constexpr int kActThreads = 256, kActWarps = kActThreads / 32;
constexpr int kBlock = 32;                      // values of a row that share a scale
constexpr int kPer = 8;                         // values of a thread: a warp has eight blocks of a row at a time
enum { kRelu = 0, kGelu = 1, kSilu = 2 };

struct ActParams {
    const void *a, *b, *d_y;
    void *y, *d_a, *d_b;
    unsigned char *codes, *scales;              // [1 or 2][B N][C] and [1 or 2][B N][blocks]; forward: NULL where none is wanted
    const int32_t* n_sel;
    long long stride;                           // of a, b, d_a, d_b, in elements
    int B, N, C, S, blocks, chunks;             // chunks: pieces of a row that a warp takes at a time
};

// These kernels are bound by the instructions that they issue long before the memory (gelu of 8192 x 2048 bf16 forward: 71 a value, 49 us); arithmetic on pairs halves it.
__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal(float x) {              // of 1 to some 14 here
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// ---- functions ------------------------------------------------------------------------------------------------------------------------
// P(normal > z) = exp(-z^2 / 2) R(z), 0 <= z.  R is Mills' ratio over sqrt(2 pi), smooth from 1/2 to 0.4 / z: a polynomial in t = 1 / (1 + 0.32 z) times t, fitted to erfcx for the least
// largest relative error, 3.2e-8; in fp32 and with the exponential off by 2^-22 and z^2 / 4 steps.
__device__ __forceinline__ float2 upper_tail(float2 z, float2& e) {
    const float2 s = mul2(mul2(z, z), both(-0.72134752f));
    e = make_float2(exp2_of(s.x), exp2_of(s.y));
    const float2 d = fma2(z, both(0.32f), both(1.f)), t = make_float2(reciprocal(d.x), reciprocal(d.y));
    float2 r = both(-0.021078268f);
    r = fma2(r, t, both(0.0954077f));
    r = fma2(r, t, both(-0.14670828f));
    r = fma2(r, t, both(0.06532883f));
    r = fma2(r, t, both(-0.009378026f));
    r = fma2(r, t, both(0.05865411f));
    r = fma2(r, t, both(0.08782908f));
    r = fma2(r, t, both(0.11462236f));
    r = fma2(r, t, both(0.12766095f));
    r = fma2(r, t, both(0.12766153f));
    return mul2(mul2(r, t), e);
}
__device__ __forceinline__ float2 far_enough(float2 a) { return make_float2(fminf(fabsf(a.x), 40.f), fminf(fabsf(a.y), 40.f)); }       // tails end long before
// exp(-|a|) and 1 / (1 + exp(-|a|)): a denominator of at most 2, where 1 + exp(-a) would leave the range
__device__ __forceinline__ float2 logistic_parts(float2 a, float2& z) {
    z = make_float2(exp2_of(fabsf(a.x) * -1.44269504f), exp2_of(fabsf(a.y) * -1.44269504f));
    return make_float2(reciprocal(1.f + z.x), reciprocal(1.f + z.y));
}
template <int kKind>
__device__ __forceinline__ float2 act_of(float2 a) {
    const float2 up = make_float2(max_or_nan(a.x, 0.f), max_or_nan(a.y, 0.f));
    if (kKind == kRelu) return up;
    if (kKind == kGelu) {                       // a (1 - Q(a)) above 0, a Q(-a) below
        float2 e;
        const float2 z = far_enough(a), q = upper_tail(z, e);
        return fma2(make_float2(-z.x, -z.y), q, up);
    }
    float2 z;
    const float2 r = logistic_parts(a, z);
    return mul2(fma2(make_float2(fminf(a.x, 0.f), fminf(a.y, 0.f)), z, up), r);
}
// f(a) and f'(a)
template <int kKind>
__device__ __forceinline__ void act_slope(float2 a, float2& f, float2& slope) {
    const float2 up = make_float2(max_or_nan(a.x, 0.f), max_or_nan(a.y, 0.f));
    if (kKind == kRelu) {
        f = up;
        slope = make_float2(a.x > 0.f ? 1.f : a.x == a.x ? 0.f : a.x, a.y > 0.f ? 1.f : a.y == a.y ? 0.f : a.y);
    } else if (kKind == kGelu) {
        float2 e;
        const float2 z = far_enough(a), q = upper_tail(z, e);
        f = fma2(make_float2(-z.x, -z.y), q, up);
        slope = fma2(mul2(a, both(0.39894228f)), e, make_float2(a.x < 0.f ? q.x : 1.f - q.x, a.y < 0.f ? q.y : 1.f - q.y));
    } else {
        float2 z;
        const float2 r = logistic_parts(a, z), p = mul2(make_float2(a.x < 0.f ? z.x : 1.f, a.y < 0.f ? z.y : 1.f), r);
        f = mul2(a, p);
        slope = fma2(f, make_float2(1.f - p.x, 1.f - p.y), p);
    }
}

// ---- eight bits ---------------------------------------------------------------------------------------------------------------------
// From the largest magnitude's bits of a block: those of the power of two at or above max / 1.75 (the carry of a mantissa beyond 1.75 = 448 / 2^8), its scale's biased exponent and 2^-e.
__device__ __forceinline__ uint32_t ceiling_of(uint32_t top) { return (top + 0x1fffffu) & 0xff800000u; }
__device__ __forceinline__ int scale_of(uint32_t top) { return max(static_cast<int>(ceiling_of(top) >> 23) - 8, 0); }
__device__ __forceinline__ float to_block(uint32_t top) { return __uint_as_float(min((262u << 23) - ceiling_of(top), 254u << 23)); }
__device__ __forceinline__ float from_block(int scale) { return __uint_as_float(scale ? static_cast<uint32_t>(scale) << 23 : 0x400000u); }
__device__ __forceinline__ uint32_t code2(float2 v) { return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ float2 value2(uint32_t code) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(code), __NV_E4M3);
    return __half22float2(__half2(h));
}
constexpr uint32_t kInfinity = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// The largest value of the type that a code stands for: the next one, 2^16 or 2^128, is none of the type's, so what would round to it is held by this one (off by less than 2^-4 of itself all the same).
template <class T>
__device__ __forceinline__ float most_held() { return std::is_same<T, __half>::value ? 61440.f : 3.1901471898837980e38f; }
// Blocks that hold something beyond that, or not finite: values as their codes are to have them, with a NaN for infinities, which e4m3 does not have.
template <class T>
__device__ __forceinline__ float held_as(float v) { return isfinite(v) ? fminf(fmaxf(v, -most_held<T>()), most_held<T>()) : __int_as_float(0x7fffffff); }

// Where a thread's eight values of a piece lie.  kWide: next to each other, four lanes to a block (C a multiple of 8); otherwise 32 apart, a block for each of them (rows begin on any element).
template <bool kWide>
struct Piece {
    long long row;                              // of [B, N]
    int c;                                      // this lane's first column
    int left;                                   // columns from there on; 0: nothing to do here
    __device__ __forceinline__ bool live(int e) const { return kWide ? left > 0 : 32 * e < left; }
};
template <class T, bool kWide>
struct Values {
    Pack<T, kWide ? kPer : 1> v[kWide ? 1 : kPer];
    __device__ __forceinline__ float at(int e) const { return to_float(kWide ? v[0].e[e] : v[e].e[0]); }
    __device__ __forceinline__ void set(int e, float x) { (kWide ? v[0].e[e] : v[e].e[0]) = from_float<T>(x); }
    // (Without a branch, from the tensor's beginning where there is nothing: a load behind a branch is waited for where the branches join.)
    __device__ __forceinline__ void load(const T* base, size_t off, const Piece<kWide>& at) {
#pragma unroll
        for (int e = 0; e < (kWide ? 1 : kPer); ++e) v[e] = load_pack<T, kWide ? kPer : 1>(base + (at.live(e) ? off + 32 * e : 0));
    }
    __device__ __forceinline__ void store(T* p, const Piece<kWide>& at) const {
#pragma unroll
        for (int e = 0; e < (kWide ? 1 : kPer); ++e)
            if (at.live(e)) store_pack(p + 32 * e, v[e]);
    }
};
// The piece of a warp's task; the next one is the next of the row, or the first one of the next row.
struct Task {
    uint32_t row, chunk;
};
template <bool kWide>
__device__ __forceinline__ Piece<kWide> piece_of(const ActParams& P, int b, int n, const Task& t) {
    Piece<kWide> p;
    const int lane = threadIdx.x & 31;
    p.row = static_cast<long long>(b) * P.N + t.row;
    p.c = static_cast<int>(t.chunk) * (32 * kPer) + (kWide ? lane * kPer : lane);
    p.left = t.row < static_cast<uint32_t>(n) ? P.C - p.c : 0;
    return p;
}

template <class T, bool kWide>
__device__ __forceinline__ void put_codes(const ActParams& P, int which, const Piece<kWide>& p, float2 (&v)[kPer / 2]) {
    const size_t row = which * (static_cast<size_t>(P.B) * P.N) + p.row;
    unsigned char* const at = P.codes + row * P.C + p.c;
    unsigned char* const scales = P.scales + row * P.blocks + p.c / kBlock;
    const uint32_t most = magnitude(most_held<T>());
    if constexpr (kWide) {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < kPer / 2; ++k) top = max(top, max(magnitude(v[k].x), magnitude(v[k].y)));
        if (p.left <= 0) top = 0;
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        if (__any_sync(0xffffffffu, top > most)) {
            uint32_t fine = 0;
#pragma unroll
            for (int k = 0; k < kPer / 2; ++k) {
                v[k] = make_float2(held_as<T>(v[k].x), held_as<T>(v[k].y));
                if (magnitude(v[k].x) < kInfinity) fine = max(fine, magnitude(v[k].x));
                if (magnitude(v[k].y) < kInfinity) fine = max(fine, magnitude(v[k].y));
            }
            if (p.left <= 0) fine = 0;
            fine = max(fine, __shfl_xor_sync(0xffffffffu, fine, 1));
            top = max(fine, __shfl_xor_sync(0xffffffffu, fine, 2));
        }
        if (p.left <= 0) return;
        const float2 mul = both(to_block(top));
        uint2 c;
        c.x = code2(mul2(v[0], mul)) | code2(mul2(v[1], mul)) << 16;
        c.y = code2(mul2(v[2], mul)) | code2(mul2(v[3], mul)) << 16;
        *reinterpret_cast<uint2*>(at) = c;
        if ((p.c & (kBlock - 1)) == 0) *scales = static_cast<unsigned char>(scale_of(top));
    } else {
        const int lane = threadIdx.x & 31;
        uint32_t mine = 0;                      // lane e keeps block e's, for its scale
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            float x = e & 1 ? v[e / 2].y : v[e / 2].x;
            uint32_t top = __reduce_max_sync(0xffffffffu, p.live(e) ? magnitude(x) : 0u);
            if (top > most) {                   // (the whole warp)
                x = held_as<T>(x);
                top = __reduce_max_sync(0xffffffffu, p.live(e) && magnitude(x) < kInfinity ? magnitude(x) : 0u);
            }
            if (p.live(e)) at[32 * e] = static_cast<unsigned char>(code2(make_float2(x * to_block(top), 0.f)));
            if (lane == e) mine = top;
        }
        if (lane < kPer && 32 * lane < p.left + lane) scales[lane] = static_cast<unsigned char>(scale_of(mine));       // blocks that begin within the row
    }
}
// Codes as they lie in memory, so that the loads of several pieces overlap.
template <bool kWide>
struct Held {
    uint2 codes;                                // a byte a value
    uint2 scales;                               // wide: the one of the block; otherwise a byte a value
    __device__ __forceinline__ void load(const ActParams& P, int which, const Piece<kWide>& p) {
        const size_t row = which * (static_cast<size_t>(P.B) * P.N) + p.row;
        const unsigned char* const at = P.codes + (p.live(0) ? row * P.C + p.c : 0);
        const unsigned char* const s = P.scales + (p.live(0) ? row * P.blocks + p.c / kBlock : 0);
        if constexpr (kWide) {
            codes = *reinterpret_cast<const uint2*>(at);
            scales.x = *s;
        } else {
            uint32_t c[kPer], f[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                c[e] = at[p.live(e) ? 32 * e : 0];
                f[e] = s[p.live(e) ? e : 0];
            }
            codes = make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
            scales = make_uint2(f[0] | f[1] << 8 | f[2] << 16 | f[3] << 24, f[4] | f[5] << 8 | f[6] << 16 | f[7] << 24);
        }
    }
    __device__ __forceinline__ float2 pair(int k) const {
        const float2 v = value2((k < 2 ? codes.x : codes.y) >> (16 * (k & 1)) & 0xffffu);
        if constexpr (kWide) return mul2(v, both(from_block(static_cast<int>(scales.x))));
        const uint32_t f = (k < 2 ? scales.x : scales.y) >> (16 * (k & 1));
        return mul2(v, make_float2(from_block(static_cast<int>(f & 0xffu)), from_block(static_cast<int>(f >> 8 & 0xffu))));
    }
};

// kTasks neighbouring pieces to a warp; kTasks = 1: and on to further ones, where there are more than the grid takes at a time.
template <int kTasks, class F>
__device__ __forceinline__ void for_instances(const ActParams& P, F body) {
#pragma unroll 1
    for (int b = blockIdx.y; b < P.B; b += gridDim.y) {
        const int n = P.n_sel ? min(max(__ldg(P.n_sel + (P.S > 1 ? b : 0)), 0), P.N) : P.N;
        const uint32_t all = static_cast<uint32_t>(n) * static_cast<uint32_t>(P.chunks), step = gridDim.x * kActWarps * kTasks;
#pragma unroll 1
        for (uint32_t t0 = (blockIdx.x * kActWarps + (threadIdx.x >> 5)) * kTasks; t0 < all; t0 += step) {
            Task t;
            t.row = t0 / static_cast<uint32_t>(P.chunks);
            t.chunk = t0 - t.row * static_cast<uint32_t>(P.chunks);
            body(b, n, t);
            if (kTasks > 1 || all - t0 <= step) break;      // (the second: no wrap)
        }
    }
}

template <class T, bool kWide, int kKind, bool kGated, int kTasks>
__global__ void __launch_bounds__(kActThreads) act_fwd_kernel(const ActParams P) {
    chain_wait();
    chain_release();
    for_instances<kTasks>(P, [&](int b, int n, Task t) {
        Piece<kWide> p[kTasks];
        Values<T, kWide> a[kTasks], g[kTasks];
#pragma unroll
        for (int u = 0; u < kTasks; ++u) {
            p[u] = piece_of<kWide>(P, b, n, t);
            if (++t.chunk == static_cast<uint32_t>(P.chunks)) {
                t.chunk = 0;
                ++t.row;
            }
            const size_t at = static_cast<size_t>(p[u].row) * P.stride + p[u].c;
            a[u].load(static_cast<const T*>(P.a), at, p[u]);
            if (kGated) g[u].load(static_cast<const T*>(P.b), at, p[u]);
        }
#pragma unroll
        for (int u = 0; u < kTasks; ++u) {
            float2 va[kPer / 2], vb[kPer / 2];
            Values<T, kWide> y;
#pragma unroll
            for (int k = 0; k < kPer / 2; ++k) {
                va[k] = make_float2(a[u].at(2 * k), a[u].at(2 * k + 1));
                float2 f = act_of<kKind>(va[k]);
                if (kGated) {
                    vb[k] = make_float2(g[u].at(2 * k), g[u].at(2 * k + 1));
                    f = mul2(f, vb[k]);
                }
                y.set(2 * k, f.x);
                y.set(2 * k + 1, f.y);
            }
            y.store(static_cast<T*>(P.y) + static_cast<size_t>(p[u].row) * P.C + p[u].c, p[u]);
            if (P.codes) {
                put_codes<T, kWide>(P, 0, p[u], va);
                if (kGated) put_codes<T, kWide>(P, 1, p[u], vb);
            }
        }
    });
}

template <class T, bool kWide, int kKind, bool kGated, int kTasks>
__global__ void __launch_bounds__(kActThreads) act_bwd_kernel(const ActParams P) {
    chain_wait();
    chain_release();
    for_instances<kTasks>(P, [&](int b, int n, Task t) {
        Piece<kWide> p[kTasks];
        Values<T, kWide> d[kTasks];
        Held<kWide> ha[kTasks], hb[kTasks];
#pragma unroll
        for (int u = 0; u < kTasks; ++u) {
            p[u] = piece_of<kWide>(P, b, n, t);
            if (++t.chunk == static_cast<uint32_t>(P.chunks)) {
                t.chunk = 0;
                ++t.row;
            }
            d[u].load(static_cast<const T*>(P.d_y), static_cast<size_t>(p[u].row) * P.C + p[u].c, p[u]);
            ha[u].load(P, 0, p[u]);
            if (kGated) hb[u].load(P, 1, p[u]);
        }
#pragma unroll
        for (int u = 0; u < kTasks; ++u) {
            if (p[u].left <= 0) continue;
            Values<T, kWide> da, db, y;
#pragma unroll
            for (int k = 0; k < kPer / 2; ++k) {
                const float2 va = ha[u].pair(k), dy = make_float2(d[u].at(2 * k), d[u].at(2 * k + 1));
                float2 f, slope, gate = both(1.f);
                act_slope<kKind>(va, f, slope);
                if (kGated) gate = hb[u].pair(k);
                const float2 ra = mul2(kGated ? mul2(dy, gate) : dy, slope);
                da.set(2 * k, ra.x);
                da.set(2 * k + 1, ra.y);
                if (kGated) {
                    const float2 rb = mul2(dy, f);
                    db.set(2 * k, rb.x);
                    db.set(2 * k + 1, rb.y);
                    f = mul2(f, gate);
                }
                y.set(2 * k, f.x);
                y.set(2 * k + 1, f.y);
            }
            const size_t at = static_cast<size_t>(p[u].row) * P.stride + p[u].c;
            da.store(static_cast<T*>(P.d_a) + at, p[u]);
            if (kGated) db.store(static_cast<T*>(P.d_b) + at, p[u]);
            if (P.y) y.store(static_cast<T*>(P.y) + static_cast<size_t>(p[u].row) * P.C + p[u].c, p[u]);
        }
    });
}

template <class F>
cudaError_t with_kind(int kind, bool gated, F f) {
    auto with_gate = [&](auto k) { return gated ? f(k, VecSize<1>{}) : f(k, VecSize<0>{}); };
    return kind == kRelu ? with_gate(VecSize<kRelu>{}) : kind == kGelu ? with_gate(VecSize<kGelu>{}) : with_gate(VecSize<kSilu>{});
}

struct CkptLayout {
    size_t codes, scales, total;
    int blocks;
};
CkptLayout ckpt_layout(const vardrop_act_cfg& c) {
    CkptLayout l;
    const size_t rows = static_cast<size_t>(c.B) * c.N * (c.gated ? 2 : 1);
    l.blocks = (c.C + kBlock - 1) / kBlock;
    l.codes = 0;
    l.scales = align_up(rows * c.C, 256);
    l.total = l.scales + align_up(rows * l.blocks, 256);
    return l;
}

constexpr int kActTasks = 2, kActPerSm = 16, kMaxGridY = 65535;      // kActPerSm: twice or thrice what an SM holds, so that instances of different sizes even out (64 instances of 1 to 1000 rows 145 us with 8, 125 with 16)
template <bool kBwd>
int act_launch(ActParams P, const vardrop_act_cfg& c, const int32_t* n_sel, cudaStream_t stream) {
    P.n_sel = n_sel;
    P.B = c.B; P.N = c.N; P.C = c.C; P.S = c.S;
    P.stride = c.stride ? c.stride : c.C;
    P.blocks = ckpt_layout(c).blocks;
    const bool wide = c.C % 8 == 0;             // (a stride is a multiple of 8 wherever there is one)
    P.chunks = (c.C + 32 * kPer - 1) / (32 * kPer);
    const long long tasks = static_cast<long long>(c.N) * P.chunks;
    // Every row counts, and enough of them for four CTAs on every SM: two pieces to a warp (where they are vectors).  Kept rows are known on the device only: two or three times as many CTAs as the SMs hold, which go through their
    // instance's pieces by strides of the grid (a CTA for each few pieces of all rows, four of five of them without work: 172 of 862 kept rows of 32 instances, gelu of 2048, forward and backward, 52.7 us instead of 37).
    const bool many = !n_sel && wide && tasks * c.B >= 4ll * kActTasks * kActWarps * sm_count();
    const int per = kActWarps * (many ? kActTasks : 1);
    const long long full = (tasks + per - 1) / per, held = (static_cast<long long>(sm_count()) * kActPerSm + c.B - 1) / c.B;
    const dim3 grid(static_cast<unsigned>(n_sel && held < full ? held : full), c.B < kMaxGridY ? c.B : kMaxGridY);
    LaunchScope ls_(kBwd ? K_ACT_BWD : K_ACT_FWD, stream);
    const cudaError_t err = with_dtype(c.dtype, [&](auto t) {
        return with_kind(c.kind, c.gated != 0, [&](auto kind, auto gated) {
            using T = decltype(t);
            constexpr int kKind = decltype(kind)::value;
            constexpr bool kGated = decltype(gated)::value != 0;
            auto go = [&](auto by, auto count) {
                constexpr bool kWide = decltype(by)::value != 0;
                constexpr int kTasks = decltype(count)::value;
                if constexpr (kBwd) return launch_chained(act_bwd_kernel<T, kWide, kKind, kGated, kTasks>, grid, dim3(kActThreads), 0, stream, P);
                else return launch_chained(act_fwd_kernel<T, kWide, kKind, kGated, kTasks>, grid, dim3(kActThreads), 0, stream, P);
            };
            return !wide ? go(VecSize<0>{}, VecSize<1>{}) : many ? go(VecSize<1>{}, VecSize<kActTasks>{}) : go(VecSize<1>{}, VecSize<1>{});
        });
    });
    return check_cuda(err, kBwd ? "act: backward launch" : "act: forward launch");
}

}  // namespace

int act_validate(const vardrop_act_cfg& c) {
    if (c.B < 1 || c.N < 1 || c.C < 1) return fail(VARDROP_ERR_INVALID_ARG, "act: B, N, C >= 1 required (B=%d N=%d C=%d)", c.B, c.N, c.C);
    if (!known_dtype(c.dtype)) return fail(VARDROP_ERR_INVALID_ARG, "act: dtype=%d is none of 0, 1, 2", c.dtype);
    if (c.kind < kRelu || c.kind > kSilu) return fail(VARDROP_ERR_INVALID_ARG, "act: kind=%d is none of 0, 1, 2", c.kind);
    if (c.gated != 0 && c.gated != 1) return fail(VARDROP_ERR_INVALID_ARG, "act: gated=%d is neither 0 nor 1", c.gated);
    if (c.S != 0 && c.S != 1 && c.S != c.B) return fail(VARDROP_ERR_INVALID_ARG, "act: S=%d is none of 0, 1, B", c.S);
    if (c.stride != 0 && (c.stride < c.C || c.stride % 8 != 0)) return fail(VARDROP_ERR_INVALID_ARG, "act: stride=%lld below C or no multiple of 8", static_cast<long long>(c.stride));
    if (static_cast<long long>(c.B) * c.N > 0x7fffffffll || c.C > (1 << 20) || c.stride > (1ll << 32)) return fail(VARDROP_ERR_UNSUPPORTED, "act: B N above 2^31 - 1, C=%d above 2^20 or stride above 2^32", c.C);
    if (static_cast<long long>(c.N) * ((c.C + kBlock - 1) / kBlock) > (1ll << 31)) return fail(VARDROP_ERR_UNSUPPORTED, "act: N=%d times ceil(C / 32), C=%d, above 2^31", c.N, c.C);
    return VARDROP_OK;
}

size_t act_ckpt_bytes(const vardrop_act_cfg& c) { return ckpt_layout(c).total; }

int act_fwd_launch(const void* a, const void* b, const int32_t* n_sel, const vardrop_act_cfg& c, void* y, void* ckpt, cudaStream_t stream) {
    ActParams P{};
    P.a = a; P.b = b; P.y = y;
    if (ckpt) {
        P.codes = static_cast<unsigned char*>(ckpt);
        P.scales = P.codes + ckpt_layout(c).scales;
    }
    return act_launch<false>(P, c, n_sel, stream);
}

int act_bwd_launch(const void* d_y, const void* ckpt, const int32_t* n_sel, const vardrop_act_cfg& c, void* d_a, void* d_b, void* y, cudaStream_t stream) {
    ActParams P{};
    P.d_y = d_y; P.d_a = d_a; P.d_b = d_b; P.y = y;
    P.codes = static_cast<unsigned char*>(const_cast<void*>(ckpt));
    P.scales = P.codes + ckpt_layout(c).scales;
    return act_launch<true>(P, c, n_sel, stream);
}

}  // namespace vardrop
