// The feed-forward's activation, y = f(a) or f(a) o b, with a checkpoint of a (and b) in 8 bits from which the backward pass works:
//   d_a = d_y o b o f'(a),  d_b = d_y o f(a),  y = f(a) o b once more (for the weight gradient of the projection behind it)
//
// act_fwd_kernel, act_bwd_kernel    32 values of a row share a power of two, the smallest 2^e with max |a| <= 448 2^e; a value is an e4m3 of that scale, so it is off by at most 2^-4 of itself (or
//                                   2^(e-10) where it is below 2^(e-6)).  A power of two costs no rounding of its own, and what 8 bits stand for is exact in the tensor's type.
//
// Bound: memory (bf16, gated: 8 bytes and two codes a value forward, 2 and two codes in and 6 out backward); gelu's backward pass is near the instruction rate as well.
#include <cuda_fp8.h>

#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "vec_io.cuh"

namespace vardrop {

namespace {

constexpr int kActThreads = 256;
constexpr int kBlock = 32;                      // values of a row that share a scale
enum { kRelu = 0, kGelu = 1, kSilu = 2 };

struct ActParams {
    const void *a, *b, *d_y;
    void *y, *d_a, *d_b;
    unsigned char *codes, *scales;              // [1 or 2][B N][C] and [1 or 2][B N][blocks]; forward: NULL where none is wanted
    const int32_t* n_sel;
    long long stride;                           // of a, b, d_a, d_b, in elements
    int B, N, C, S, blocks, chunks;             // chunks: pieces of a row that a warp takes at a time
};

__device__ __forceinline__ float upper_tail(float a) { return 0.5f * erfcf(a * -0.70710678f); }      // P(normal <= a)
// kFull: to fp32's last bits; otherwise the fast forms, good to some 2^-21, which 16-bit results do not feel.
template <bool kFull>
__device__ __forceinline__ float exp_of(float a) { return kFull ? expf(a) : __expf(a); }
template <bool kFull>
__device__ __forceinline__ float quotient(float a, float b) { return kFull ? a / b : __fdividef(a, b); }
// 1 / (1 + exp(-a)) with a denominator of at most 2: the fast quotient gives 0 for ones beyond 2^126.
template <bool kFull>
__device__ __forceinline__ float logistic(float a) {
    const float z = exp_of<kFull>(-fabsf(a));
    return quotient<kFull>(a < 0.f ? z : 1.f, 1.f + z);
}
template <int kKind, bool kFull>
__device__ __forceinline__ float act_of(float a) {
    if (kKind == kRelu) return a < 0.f ? 0.f : a;                   // (a NaN stays one)
    if (kKind == kGelu) return a * upper_tail(a);
    return a * logistic<kFull>(a);
}
// f(a) and f'(a)
template <int kKind, bool kFull>
__device__ __forceinline__ void act_slope(float a, float& f, float& slope) {
    if (kKind == kRelu) {
        f = a < 0.f ? 0.f : a;
        slope = a > 0.f ? 1.f : a == a ? 0.f : a;
    } else if (kKind == kGelu) {
        const float p = upper_tail(a);
        f = a * p;
        slope = fmaf(a * 0.39894228f, exp_of<kFull>(-0.5f * a * a), p);
    } else {
        const float p = logistic<kFull>(a);
        f = a * p;
        slope = fmaf(f, 1.f - p, p);
    }
}

// Biased exponent of the block's scale from the largest magnitude's bits.
__device__ __forceinline__ int scale_of(uint32_t top) {
    const int e = static_cast<int>(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u);        // 448 = 1.75 2^8
    return max(e, 0);
}
__device__ __forceinline__ float to_block(int scale) { return __uint_as_float(static_cast<uint32_t>(254 - scale) << 23); }     // 2^-e
__device__ __forceinline__ float from_block(int scale) { return __uint_as_float(scale ? static_cast<uint32_t>(scale) << 23 : 0x400000u); }
__device__ __forceinline__ uint32_t magnitude(float v) {            // for the block's maximum: values that are not finite have no part in it
    const uint32_t m = __float_as_uint(v) & 0x7fffffffu;
    return m < 0x7f800000u ? m : 0u;
}
__device__ __forceinline__ uint32_t code2(float v0, float v1, float mul) {
    uint32_t c = __nv_cvt_float2_to_fp8x2(make_float2(v0 * mul, v1 * mul), __NV_SATFINITE, __NV_E4M3);
    if (isinf(v0)) c |= 0x7fu;                                      // no infinities in e4m3: NaN
    if (isinf(v1)) c |= 0x7f00u;
    return c;
}
__device__ __forceinline__ float2 value2(uint32_t code, float mul) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(code), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    return make_float2(f.x * mul, f.y * mul);
}

// Where a warp's piece lies.  kVec 8: 256 columns, eight to a lane, four lanes to a block; kVec 1: a block, a column a lane.
template <int kVec>
struct Piece {
    long long row;                              // of [B, N]
    int c;                                      // this lane's first column
    bool live;
};
template <int kVec>
__device__ __forceinline__ Piece<kVec> piece_of(const ActParams& P, int b, int n, uint32_t task) {
    Piece<kVec> p;
    const uint32_t i = task / static_cast<uint32_t>(P.chunks), k = task - i * static_cast<uint32_t>(P.chunks);
    p.row = static_cast<long long>(b) * P.N + i;
    p.c = static_cast<int>(k * 32 + (threadIdx.x & 31)) * kVec;
    p.live = i < static_cast<uint32_t>(n) && p.c < P.C;
    return p;
}
// kTasks pieces a warp, those of neighbouring warps next to each other.
constexpr int kActWarps = kActThreads / 32;

// The largest value of the type that a code stands for: the next one, 2^16 or 2^128, is none of the type's, so what would round to it is held by this one (off by less than 2^-4 of itself all the same).
template <class T>
__device__ __forceinline__ float most_held() { return std::is_same<T, __half>::value ? 61440.f : 3.1901471898837980e38f; }
template <class T, int kVec>
__device__ __forceinline__ void put_codes(const ActParams& P, int which, const Piece<kVec>& p, float (&v)[kVec]) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < kVec; ++e) top = max(top, p.live ? magnitude(v[e]) : 0u);
    if (kVec == 1) {
        top = __reduce_max_sync(0xffffffffu, top);
    } else {
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    }
    if (!p.live) return;
    if (top > __float_as_uint(most_held<T>())) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            if (isfinite(v[e])) v[e] = fminf(fmaxf(v[e], -most_held<T>()), most_held<T>());
    }
    const int scale = scale_of(top);
    const float mul = to_block(scale);
    const size_t rows = static_cast<size_t>(P.B) * P.N, row = which * rows + p.row;
    unsigned char* const at = P.codes + row * P.C + p.c;
    if constexpr (kVec == 8) {
        uint2 c;
        c.x = code2(v[0], v[1], mul) | code2(v[2], v[3], mul) << 16;
        c.y = code2(v[4], v[5], mul) | code2(v[6], v[7], mul) << 16;
        *reinterpret_cast<uint2*>(at) = c;
    } else {
        *at = static_cast<unsigned char>(code2(v[0], 0.f, mul));
    }
    if ((p.c & (kBlock - 1)) == 0) P.scales[row * P.blocks + p.c / kBlock] = static_cast<unsigned char>(scale);
}
// Codes as they lie in memory, so that the loads of several pieces overlap.
struct Held {
    uint2 codes;
    int scale;
};
template <int kVec>
__device__ __forceinline__ Held get_codes(const ActParams& P, int which, const Piece<kVec>& p) {
    const size_t row = which * static_cast<size_t>(P.B) * P.N + p.row;
    const unsigned char* const at = P.codes + row * P.C + p.c;
    Held h;
    if constexpr (kVec == 8) h.codes = *reinterpret_cast<const uint2*>(at);
    else h.codes = make_uint2(*at, 0u);
    h.scale = P.scales[row * P.blocks + p.c / kBlock];
    return h;
}
template <int kVec>
__device__ __forceinline__ void values_of(const Held& h, float (&v)[kVec]) {
    const float mul = from_block(h.scale);
    if constexpr (kVec == 8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = value2((k < 2 ? h.codes.x : h.codes.y) >> (16 * (k & 1)) & 0xffffu, mul);
            v[2 * k] = f.x;
            v[2 * k + 1] = f.y;
        }
    } else {
        v[0] = value2(h.codes.x, mul).x;
    }
}

template <class T, int kVec, int kKind, bool kGated, int kTasks>
__global__ void __launch_bounds__(kActThreads) act_fwd_kernel(const ActParams P) {
    constexpr bool kFull = sizeof(T) == 4;
    chain_wait();
    chain_release();
#pragma unroll 1
    for (int b = blockIdx.y; b < P.B; b += gridDim.y) {
        const int n = P.n_sel ? min(max(__ldg(P.n_sel + (P.S > 1 ? b : 0)), 0), P.N) : P.N;
        const uint32_t t0 = blockIdx.x * kActWarps * kTasks + (threadIdx.x >> 5);
        if (t0 >= static_cast<uint32_t>(n) * static_cast<uint32_t>(P.chunks)) continue;
        Piece<kVec> p[kTasks];
        Pack<T, kVec> a[kTasks], g[kTasks];
#pragma unroll
        for (int u = 0; u < kTasks; ++u) {
            p[u] = piece_of<kVec>(P, b, n, t0 + u * kActWarps);
            if (!p[u].live) continue;
            const size_t at = static_cast<size_t>(p[u].row) * P.stride + p[u].c;
            a[u] = load_pack<T, kVec>(static_cast<const T*>(P.a) + at);
            if (kGated) g[u] = load_pack<T, kVec>(static_cast<const T*>(P.b) + at);
        }
#pragma unroll
        for (int u = 0; u < kTasks; ++u) {
            float va[kVec], vb[kVec];
            Pack<T, kVec> y;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                va[e] = p[u].live ? to_float(a[u].e[e]) : 0.f;
                vb[e] = kGated && p[u].live ? to_float(g[u].e[e]) : 1.f;
                y.e[e] = from_float<T>(kGated ? act_of<kKind, kFull>(va[e]) * vb[e] : act_of<kKind, kFull>(va[e]));
            }
            if (p[u].live) store_pack(static_cast<T*>(P.y) + static_cast<size_t>(p[u].row) * P.C + p[u].c, y);
            if (P.codes) {
                put_codes<T, kVec>(P, 0, p[u], va);
                if (kGated) put_codes<T, kVec>(P, 1, p[u], vb);
            }
        }
    }
}

template <class T, int kVec, int kKind, bool kGated, int kTasks>
__global__ void __launch_bounds__(kActThreads) act_bwd_kernel(const ActParams P) {
    constexpr bool kFull = sizeof(T) == 4;
    chain_wait();
    chain_release();
#pragma unroll 1
    for (int b = blockIdx.y; b < P.B; b += gridDim.y) {
        const int n = P.n_sel ? min(max(__ldg(P.n_sel + (P.S > 1 ? b : 0)), 0), P.N) : P.N;
        const uint32_t t0 = blockIdx.x * kActWarps * kTasks + (threadIdx.x >> 5);
        if (t0 >= static_cast<uint32_t>(n) * static_cast<uint32_t>(P.chunks)) continue;
        Piece<kVec> p[kTasks];
        Pack<T, kVec> d[kTasks];
        Held ha[kTasks], hb[kTasks];
#pragma unroll
        for (int u = 0; u < kTasks; ++u) {
            p[u] = piece_of<kVec>(P, b, n, t0 + u * kActWarps);
            if (!p[u].live) continue;
            d[u] = load_pack<T, kVec>(static_cast<const T*>(P.d_y) + static_cast<size_t>(p[u].row) * P.C + p[u].c);
            ha[u] = get_codes<kVec>(P, 0, p[u]);
            if (kGated) hb[u] = get_codes<kVec>(P, 1, p[u]);
        }
#pragma unroll
        for (int u = 0; u < kTasks; ++u) {
            if (!p[u].live) continue;
            float va[kVec], vb[kVec];
            values_of<kVec>(ha[u], va);
            if (kGated) values_of<kVec>(hb[u], vb);
            Pack<T, kVec> da, db, y;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                float f, slope;
                act_slope<kKind, kFull>(va[e], f, slope);
                const float dy = to_float(d[u].e[e]);
                da.e[e] = from_float<T>((kGated ? dy * vb[e] : dy) * slope);
                if (kGated) db.e[e] = from_float<T>(dy * f);
                y.e[e] = from_float<T>(kGated ? f * vb[e] : f);
            }
            const size_t at = static_cast<size_t>(p[u].row) * P.stride + p[u].c;
            store_pack(static_cast<T*>(P.d_a) + at, da);
            if (kGated) store_pack(static_cast<T*>(P.d_b) + at, db);
            if (P.y) store_pack(static_cast<T*>(P.y) + static_cast<size_t>(p[u].row) * P.C + p[u].c, y);
        }
    }
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

constexpr int kActTasks = 4, kMaxGridY = 65535;
template <bool kBwd>
int act_launch(ActParams P, const vardrop_act_cfg& c, const int32_t* n_sel, cudaStream_t stream) {
    P.n_sel = n_sel;
    P.B = c.B; P.N = c.N; P.C = c.C; P.S = c.S;
    P.stride = c.stride ? c.stride : c.C;
    P.blocks = ckpt_layout(c).blocks;
    const bool wide = c.C % 8 == 0;             // (a stride is a multiple of 8 wherever there is one)
    P.chunks = wide ? (c.C + 255) / 256 : P.blocks;
    const long long tasks = static_cast<long long>(c.N) * P.chunks;
    // several pieces to a warp only where every SM still gets four CTAs
    const bool many = tasks * c.B >= 4ll * kActTasks * kActWarps * sm_count();
    const int per = kActWarps * (many ? kActTasks : 1);
    const dim3 grid(static_cast<unsigned>((tasks + per - 1) / per), c.B < kMaxGridY ? c.B : kMaxGridY);
    LaunchScope ls_(kBwd ? K_ACT_BWD : K_ACT_FWD, stream);
    const cudaError_t err = with_dtype(c.dtype, [&](auto t) {
        return with_kind(c.kind, c.gated != 0, [&](auto kind, auto gated) {
            using T = decltype(t);
            constexpr int kKind = decltype(kind)::value;
            constexpr bool kGated = decltype(gated)::value != 0;
            auto go = [&](auto vec, auto count) {
                constexpr int kVec = decltype(vec)::value, kTasks = decltype(count)::value;
                if constexpr (kBwd) return launch_chained(act_bwd_kernel<T, kVec, kKind, kGated, kTasks>, grid, dim3(kActThreads), 0, stream, P);
                else return launch_chained(act_fwd_kernel<T, kVec, kKind, kGated, kTasks>, grid, dim3(kActThreads), 0, stream, P);
            };
            return wide ? (many ? go(VecSize<8>{}, VecSize<kActTasks>{}) : go(VecSize<8>{}, VecSize<1>{})) : (many ? go(VecSize<1>{}, VecSize<kActTasks>{}) : go(VecSize<1>{}, VecSize<1>{}));
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
