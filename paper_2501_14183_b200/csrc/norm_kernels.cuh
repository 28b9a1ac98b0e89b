// Norms before and after a block with its gate and residual scale: h = a x + g o N_post(y), u = N_pre(h), and their gradients.
//
// norm_fwd_kernel        a group of threads per token, its row in registers.
// norm_bwd_kernel        the same; sums over tokens stay in registers until a CTA is done with its rows.
//
// With z = (t - mean) r, e = w o d for the gradient d of N(t):  dt = r (e - mean(e) - z mean(e o z)), without mean(e) for rms.
// Bound: memory.  Forward x, y in, h, u out; backward x, y, dh, du in, dx, dy out (h again from x and y: read back as h it would come rounded, and the fp32 sums with it).
#pragma once

#include <cuda_fp16.h>

#include "norm.h"
#include "norm_walk.h"

namespace vardrop {

namespace {

// ---- pairs: two fp32 values in a 64-bit register, for the packed instructions of sm_100 (one issue slot for two results, each rounded as the scalar instruction's) -------
typedef uint64_t Pair;
__device__ __forceinline__ Pair pair_of(float lo, float hi) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ Pair both(float v) { return pair_of(v, v); }
__device__ __forceinline__ float2 halves(Pair v) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
    return f;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float sum_of(Pair v) { const float2 f = halves(v); return f.x + f.y; }

// ---- elements -------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ Pair widen(uint32_t w, __nv_bfloat16) { return pair_of(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ Pair widen(uint32_t w, __half) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return pair_of(f.x, f.y);
}
__device__ __forceinline__ uint32_t narrow(Pair v, __nv_bfloat16) {
    const float2 f = halves(v);
    const __nv_bfloat162 r = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t narrow(Pair v, __half) {
    const float2 f = halves(v);
    const __half2 r = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// A thread's columns: kPer / kV vectors of kV, a group's threads side by side; element e of the thread is element e % kV of vector e / kV, and pair p elements 2 p and 2 p + 1.
template <class T, int kV, int kGroup, int kPer>
struct Row {
    static constexpr int kVecs = kPer / kV, kPairs = kPer / 2, kVecBytes = kV * static_cast<int>(sizeof(T));
    typedef Pair Values[kPairs];
    static __device__ __forceinline__ int col(int t, int j) { return (j * kGroup + t) * kV; }
    static __device__ __forceinline__ bool whole(int C) { return C == kGroup * kPer; }
    // words of the vectors (a 16-bit element alone takes a word too) to pairs, and back
    static constexpr int kWords = kVecBytes < 4 ? 1 : kVecBytes / 4;
    struct alignas(kVecBytes < 4 ? 4 : kVecBytes) Vec { uint32_t w[kWords]; };
    static __device__ __forceinline__ Vec load(const T* p) {
        Vec v;
        if constexpr (kVecBytes < 4) v.w[0] = *reinterpret_cast<const unsigned short*>(p);
        else v = *reinterpret_cast<const Vec*>(p);
        return v;
    }
    static __device__ __forceinline__ void unpack(const Vec (&v)[kVecs], Values& to) {
#pragma unroll
        for (int p = 0; p < kPairs; ++p) {
            if constexpr (sizeof(T) == 4) {
                const int e = 2 * p;
                to[p] = pair_of(__uint_as_float(v[e / kV].w[e % kV]), __uint_as_float(v[(e + 1) / kV].w[(e + 1) % kV]));
            } else if constexpr (kV == 1) {
                to[p] = widen(v[2 * p].w[0] | v[2 * p + 1].w[0] << 16, T{});
            } else {
                to[p] = widen(v[2 * p / kV].w[p % (kV / 2)], T{});
            }
        }
    }
    static __device__ __forceinline__ void store(T* row, int t, int C, const Values& v) {
        Vec x[kVecs];
#pragma unroll
        for (int p = 0; p < kPairs; ++p) {
            if constexpr (sizeof(T) == 4) {
                const float2 f = halves(v[p]);
                const int e = 2 * p;
                x[e / kV].w[e % kV] = __float_as_uint(f.x);
                x[(e + 1) / kV].w[(e + 1) % kV] = __float_as_uint(f.y);
            } else if constexpr (kV == 1) {
                const uint32_t w = narrow(v[p], T{});
                x[2 * p].w[0] = w & 0xffffu;
                x[2 * p + 1].w[0] = w >> 16;
            } else {
                x[2 * p / kV].w[p % (kV / 2)] = narrow(v[p], T{});
            }
        }
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            if (col(t, j) >= C) continue;
            if constexpr (kVecBytes < 4) *reinterpret_cast<unsigned short*>(row + col(t, j)) = static_cast<unsigned short>(x[j].w[0]);
            else *reinterpret_cast<Vec*>(row + col(t, j)) = x[j];
        }
    }
    // of a parameter; `none` where there is none, 0 behind the row's end
    static __device__ __forceinline__ void param(const float* p, int t, int C, float none, Values& v) {
        float f[kPer];
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            if (p && col(t, j) < C) {
                if constexpr (kV % 4 == 0) {
#pragma unroll
                    for (int e = 0; e < kV; e += 4) {
                        const float4 q = __ldg(reinterpret_cast<const float4*>(p + col(t, j) + e));
                        f[j * kV + e] = q.x; f[j * kV + e + 1] = q.y; f[j * kV + e + 2] = q.z; f[j * kV + e + 3] = q.w;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < kV; ++e) f[j * kV + e] = __ldg(p + col(t, j) + e);
                }
            } else {
#pragma unroll
                for (int e = 0; e < kV; ++e) f[j * kV + e] = col(t, j) < C ? none : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) v[i] = pair_of(f[2 * i], f[2 * i + 1]);
    }
    static __device__ __forceinline__ void param_store(float* to, int t, int C, const Values& v) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const float2 f = halves(v[i]);
            const int c0 = col(t, 2 * i / kV) + 2 * i % kV, c1 = col(t, (2 * i + 1) / kV) + (2 * i + 1) % kV;
            if (c0 < C) to[c0] = f.x;
            if (c1 < C) to[c1] = f.y;
        }
    }
    // zeros again behind the row's end
    static __device__ __forceinline__ void clear_rest(int t, int C, Values& v) {
        if (whole(C)) return;
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const float2 f = halves(v[i]);
            v[i] = pair_of(col(t, 2 * i / kV) < C ? f.x : 0.f, col(t, (2 * i + 1) / kV) < C ? f.y : 0.f);
        }
    }
};

// ---- sums over a group ------------------------------------------------------------------------------------------------------
template <int kLanes>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Barrier of group `id` (of at most four).  A number that is only known at run time reserves all sixteen barriers, and an SM then holds four CTAs.
template <int kGroup>
__device__ __forceinline__ void group_barrier(int id) {
    if (id == 0) asm volatile("bar.sync 1, %0;" ::"n"(kGroup) : "memory");
    else if (id == 1) asm volatile("bar.sync 2, %0;" ::"n"(kGroup) : "memory");
    else if (id == 2) asm volatile("bar.sync 3, %0;" ::"n"(kGroup) : "memory");
    else asm volatile("bar.sync 4, %0;" ::"n"(kGroup) : "memory");
}
// One sum, or two at once, to every thread of the group.  Groups of several warps go through shared memory, in two places by turns, so that one barrier a sum is enough.
template <int kGroup>
struct GroupSum {
    float2* place;                       // [2][warps] of this group
    int turn = 0, id;
    template <bool kTwo>
    __device__ __forceinline__ float2 of(float a, float b) {
        constexpr int kLanes = kGroup < 32 ? kGroup : 32, kWarps = kGroup < 32 ? 1 : kGroup / 32;
        a = lanes_sum<kLanes>(a);
        if (kTwo) b = lanes_sum<kLanes>(b);
        if (kGroup <= 32) return make_float2(a, b);
        const int lane = threadIdx.x & 31, warp = (threadIdx.x % kGroup) >> 5;
        float2* at = place + turn * kWarps;
        turn ^= 1;
        if (lane == 0) at[warp] = make_float2(a, b);
        group_barrier<kGroup>(id);
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 f = at[w];
            s.x += f.x;
            if (kTwo) s.y += f.y;
        }
        return s;
    }
};

template <int kGroup>
constexpr int kNormThreads = kGroup < 256 ? 256 : kGroup;        // of a CTA

// Rows on their way from memory: a ring in shared memory whose places belong to one thread each, filled by asynchronous copies of the thread's own columns, so
// that a group has kStages - 1 rows in flight while it works on one, without registers for them and without barriers.  (Loads into registers behind the row before: 65536 x
// 1024 bf16 forward 188 us, backward 367; like this 118 and 166, bound by the instructions of scalar arithmetic; with pairs 92 and 148.)  Columns of two bytes, which those copies cannot take, are
// loaded when they are needed.
template <class T, int kV, int kGroup, int kPer, int kTensors>
struct Ring {
    using R = Row<T, kV, kGroup, kPer>;
    using Vec = typename R::Vec;
    static constexpr bool kAsync = R::kVecBytes >= 4;
    static constexpr int kThreads = kNormThreads<kGroup>;
    static constexpr int kStageBytes = kThreads * kPer * static_cast<int>(sizeof(T)) * kTensors;
    static constexpr int kFit = 200 * 1024 / kStageBytes;
    static constexpr int kStages = kFit < 1 ? 1 : kFit > 3 ? 3 : kFit;
    static constexpr int kBytes = kAsync ? kStages * kStageBytes : 0;
    Vec* mine;                           // this thread's first place
    __device__ __forceinline__ Vec* at(int stage, int k, int j) const { return mine + ((stage * kTensors + k) * R::kVecs + j) * kThreads; }
    // tensor k of a row (NULL: none) to a stage; commit() behind the last one
    __device__ __forceinline__ void fetch(int stage, int k, const T* row, int t, int C) {
        if constexpr (kAsync) {
            if (!row) return;
#pragma unroll
            for (int j = 0; j < R::kVecs; ++j) {
                if (R::col(t, j) >= C) continue;
                const uint32_t to = smem_u32(at(stage, k, j));
                if (R::kVecBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row + R::col(t, j)) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(row + R::col(t, j)), "n"(R::kVecBytes) : "memory");
            }
        }
    }
    __device__ __forceinline__ void commit() {
        if (kAsync) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ void wait() {             // the oldest stage in flight has landed
        if (kAsync) asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    }
    // a row's columns, zeros behind its end
    __device__ __forceinline__ void read(int stage, int k, const T* row, int t, int C, typename R::Values& to) const {
        Vec v[R::kVecs];
#pragma unroll
        for (int j = 0; j < R::kVecs; ++j) {
            if (R::col(t, j) < C) {
                if constexpr (kAsync) v[j] = *at(stage, k, j);
                else v[j] = R::load(row + R::col(t, j));
            } else {
#pragma unroll
                for (int w = 0; w < R::kWords; ++w) v[j].w[w] = 0u;
            }
        }
        R::unpack(v, to);
    }
};

// t without its mean (kind 2), and the (mean, r) of its norm
template <class R, int kGroup, bool kLayer>
__device__ __forceinline__ float2 centre(typename R::Values& t, int kind, int thread, const NormParams& P, GroupSum<kGroup>& sum) {
    float mean = 0.f;
    if (kLayer && kind == 2) {
        Pair s = t[0];
#pragma unroll
        for (int p = 1; p < R::kPairs; ++p) s = add2(s, t[p]);
        mean = sum.template of<false>(sum_of(s), 0.f).x * P.inv_c;
        const Pair minus = both(-mean);
#pragma unroll
        for (int p = 0; p < R::kPairs; ++p) t[p] = add2(t[p], minus);
        R::clear_rest(thread, P.C, t);
    }
    Pair q[2] = {both(0.f), both(0.f)};
#pragma unroll
    for (int p = 0; p < R::kPairs; ++p) q[p & 1] = fma2(t[p], t[p], q[p & 1]);
    return make_float2(mean, rsqrtf(sum.template of<false>(sum_of(add2(q[0], q[1])), 0.f).x * P.inv_c + P.eps));
}

// A CTA's run of the tokens that all instances keep (kRuns); it is worked off instance by instance.
struct Run {
    long long from, to;                  // of this CTA
    int ctas;                            // with tokens
    int b;                               // instance of the first token
    long long begin;                     // tokens ahead of that instance
};
// Tokens of an instance, and the run of a CTA; every thread of the block calls it.  Kept counts of their own are summed up 256 at a time, by every CTA for itself.
__device__ __forceinline__ int tokens_of(const NormParams& P, int b) { return P.n_sel ? max(0, min(P.N, __ldg(P.n_sel + (P.S > 1 ? b : 0)))) : P.N; }
__device__ __forceinline__ Run run_of(const NormParams& P, long long* s_scan) {       // s_scan[blockDim / 32 + 2]
    Run r{0, 0, 0, 0, 0};
    const int G = gridDim.x, c = blockIdx.x;
    auto share = [&](long long K) {
        r.ctas = static_cast<int>(K < G ? K : G);
        if (c >= r.ctas) return;
        r.from = K * c / r.ctas;
        r.to = K * (c + 1) / r.ctas;
    };
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    long long K = 0, ahead = 0;
    int n = 0;                                           // of the instance looked at last, and the tokens ahead of it
    auto scan = [&](long long b, long long& all) {       // one instance a thread
        n = b < P.B ? tokens_of(P, static_cast<int>(b)) : 0;
        int x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        __syncthreads();
        if (lane == 31) s_scan[warp] = x;
        __syncthreads();
        ahead = all + x - n;
        for (int w = 0; w < warps; ++w) {
            const long long v = s_scan[w];
            if (w < warp) ahead += v;
            all += v;
        }
    };
    auto find = [&](long long b) {                       // the instance in which the run begins
        if (n > 0 && ahead <= r.from && r.from < ahead + n) {
            s_scan[warps] = b;
            s_scan[warps + 1] = ahead;
        }
    };
#pragma unroll 1
    for (long long b0 = 0; b0 < P.B; b0 += blockDim.x) {
        scan(b0 + threadIdx.x, K);
        if (P.begin && c == 0 && b0 + threadIdx.x < P.B) P.begin[b0 + threadIdx.x] = static_cast<int>(ahead);
    }
    if (P.begin && c == 0 && threadIdx.x == 0) P.begin[P.B] = static_cast<int>(K);
    share(K);
    if (r.from >= r.to) return r;                        // (the same for all threads)
    if (P.B <= static_cast<int>(blockDim.x)) {
        find(threadIdx.x);
    } else {
        long long all = 0;
#pragma unroll 1
        for (long long b0 = 0; b0 < P.B; b0 += blockDim.x) {
            scan(b0 + threadIdx.x, all);
            find(b0 + threadIdx.x);
        }
    }
    __syncthreads();
    r.b = static_cast<int>(s_scan[warps]);
    r.begin = s_scan[warps + 1];
    return r;
}
// The parts of a CTA's tokens that lie in one instance, one after another: tokens first, first + step, ... below n, for this group; `slot` is the place of the part's sums.
struct Parts {
    RowIndex first, n, step;
    int b, slot, base_row;
    RowIndex unit;                       // the next one of this CTA, ~0 behind the only one
    long long at, begin;
    Run run;
    __device__ __forceinline__ void start(const NormParams& P, long long* s_scan) {
        unit = blockIdx.x;
        if (P.share == kRuns) {
            run = run_of(P, s_scan);
            at = run.from;
            begin = run.begin;
            unit = run.b;
        }
    }
    __device__ __forceinline__ bool next(const NormParams& P, int group, int groups) {
        if (P.share == kFlat) {
            if (unit == ~0u) return false;
            b = base_row = 0;
            first = unit * groups + group;
            n = P.B * P.N;
            step = gridDim.x * groups;
            slot = static_cast<int>(unit);
            unit = ~0u;
            return true;
        }
        if (P.share == kSplit) {
            if (unit >= static_cast<RowIndex>(P.B * P.splits)) return false;
            b = static_cast<int>(unit) / P.splits;
            base_row = b * P.N;
            first = (static_cast<int>(unit) - b * P.splits) * groups + group;
            n = tokens_of(P, 0);
            step = P.splits * groups;
            slot = static_cast<int>(unit);
            unit += gridDim.x;
            return true;
        }
        if (at >= run.to) return false;
        b = static_cast<int>(unit++);
        base_row = b * P.N;
        const int n_b = tokens_of(P, b);
        first = static_cast<RowIndex>(at - begin) + group;
        n = static_cast<RowIndex>(min(static_cast<long long>(n_b), run.to - begin));
        step = groups;
        slot = blockIdx.x + b;               // (a place of its own: from one such pair to the next the CTA or the instance goes up)
        begin += n_b;
        at = max(at, begin);
        return true;
    }
};
// The source row of a selection is known one row ahead of its copies.
struct RowWalk : RowSteps {
    const int32_t* sel;
    __device__ __forceinline__ RowWalk(const int32_t* s, const Parts& part) : RowSteps{part.n, part.step}, sel(s) {}
    __device__ __forceinline__ RowIndex source(RowIndex i) const { return sel ? (there(i) ? __ldg(sel + i) : 0) : i; }
};

// ---- forward ----------------------------------------------------------------------------------------------------------------
// kLayer: a mean or a bias somewhere.
template <class T, int kV, int kGroup, int kPer, bool kLayer>
__global__ void __launch_bounds__(kNormThreads<kGroup>, 512 / kNormThreads<kGroup>) norm_fwd_kernel(const NormParams P) {
    using Rows = Ring<T, kV, kGroup, kPer, 2>;
    using R = typename Rows::R;
    constexpr int kGroups = kNormThreads<kGroup> / kGroup, kAhead = Rows::kStages - 1;
    extern __shared__ __align__(128) unsigned char smem_dyn[];        // (off such a boundary a warp's copy is split, and its sectors are read twice)
    __shared__ float2 s_sum[kGroups][kGroup < 64 ? 1 : 2 * (kGroup / 32)];
    __shared__ long long s_scan[kNormThreads<kGroup> / 32 + 2];
    const int group = threadIdx.x / kGroup, t = threadIdx.x % kGroup;
    GroupSum<kGroup> sum{s_sum[group], 0, group};
    Rows ring{reinterpret_cast<typename Rows::Vec*>(smem_dyn) + threadIdx.x};
    chain_wait();
    chain_release();
    const T* const X = static_cast<const T*>(P.x);
    const T* const Y = static_cast<const T*>(P.y);
    typename R::Values w_pre, b_pre;                     // of this thread's columns, for all rows
    R::param(P.w_pre, t, P.C, 1.f, w_pre);
    if (kLayer) R::param(P.b_pre, t, P.C, 0.f, b_pre);
    const Pair scale = both(P.scale);
    Parts part;
    part.start(P, s_scan);
#pragma unroll 1
    while (part.next(P, group, kGroups)) {
        const int b = part.b;
        const RowIndex first = part.first;
        const RowWalk walk(P.sel_idx ? P.sel_idx + static_cast<size_t>(P.S > 1 ? b : 0) * P.N : nullptr, part);
        const size_t base = part.base_row;
        // N_post's scale and bias with the gate in them: h = a x + w z + c
        typename R::Values w, c;
        {
            typename R::Values g;
            R::param(P.gate ? P.gate + static_cast<size_t>(P.gate_rows > 1 ? b : 0) * P.C : nullptr, t, P.C, 1.f, g);
            R::param(P.w_post, t, P.C, 1.f, w);
            if (kLayer) R::param(P.b_post, t, P.C, 0.f, c);
#pragma unroll
            for (int p = 0; p < R::kPairs; ++p) {
                w[p] = mul2(w[p], g[p]);
                if (kLayer) c[p] = mul2(c[p], g[p]);
            }
        }
        RowIndex i = first, ahead = first, source = walk.source(ahead);
        int stage = 0;
        auto fetch = [&](int to) {
            if (walk.there(ahead)) {
                ring.fetch(to, 0, X + (base + source) * P.C, t, P.C);
                ring.fetch(to, 1, Y ? Y + (base + ahead) * P.C : nullptr, t, P.C);
            }
            ring.commit();
            ahead += walk.step;
            source = walk.source(ahead);
        };
#pragma unroll
        for (int s = 0; s < kAhead; ++s) fetch(s);
        // Groups of less than a warp leave the loop together; one without a token works on a row without columns.
        const RowIndex behind = kGroup < 32 ? (threadIdx.x & 31) / kGroup : 0;
#pragma unroll 1
        for (; walk.goes_on(i, behind); i += walk.step) {
            const int C = kGroup < 32 && !walk.there(i) ? 0 : P.C;
            const RowIndex from = Rows::kAsync ? 0 : walk.source(i);
            fetch(stage + kAhead < Rows::kStages ? stage + kAhead : stage + kAhead - Rows::kStages);
            ring.wait();
            const size_t row = (base + i) * P.C;
            float2 post = make_float2(0.f, 1.f), pre = post;
            typename R::Values h;
            ring.read(stage, 0, X + (base + from) * P.C, t, C, h);
#pragma unroll
            for (int p = 0; p < R::kPairs; ++p) h[p] = mul2(h[p], scale);
            if (Y) {
                typename R::Values y;
                ring.read(stage, 1, Y + row, t, C, y);
                if (P.post) post = centre<R, kGroup, kLayer>(y, P.post, t, P, sum);
                const Pair r = both(post.y);
#pragma unroll
                for (int p = 0; p < R::kPairs; ++p) {
                    if (kLayer) h[p] = add2(h[p], c[p]);
                    h[p] = fma2(mul2(y[p], r), w[p], h[p]);
                }
            }
            if (P.h) R::store(static_cast<T*>(P.h) + row, t, C, h);
            if (P.pre) {
                pre = centre<R, kGroup, kLayer>(h, P.pre, t, P, sum);
                const Pair r = both(pre.y);
#pragma unroll
                for (int p = 0; p < R::kPairs; ++p) h[p] = kLayer ? fma2(mul2(h[p], r), w_pre[p], b_pre[p]) : mul2(mul2(h[p], r), w_pre[p]);
                R::store(static_cast<T*>(P.u) + row, t, C, h);
            }
            if (P.stats && t == 0 && C) P.stats[base + i] = make_float4(post.x, post.y, pre.x, pre.y);
            if (++stage == Rows::kStages) stage = 0;
        }
    }
}

// ---- backward ---------------------------------------------------------------------------------------------------------------
// Sums over tokens: with t the gradient of h, zy and zh the normed y and h:
//   d_gate = w_post o A + b_post o T,  d_w_post = sum_b g_b o A_b,  d_b_post = sum_b g_b o T_b   with A = sum t o zy, T = sum t over the tokens of an instance,
//   d_w_pre = sum du o zh,  d_b_pre = sum du
// so a thread keeps four sums a column however many parameters there are, without a mean or a bias (kLayer) two.  (A gate that all instances share needs them over all
// tokens only.)
template <class T, int kV, int kGroup, int kPer, bool kLayer>
__global__ void __launch_bounds__(kNormThreads<kGroup>, 512 / kNormThreads<kGroup> > 0 ? 512 / kNormThreads<kGroup> : 1) norm_bwd_kernel(const NormParams P) {
    using Rows = Ring<T, kV, kGroup, kPer, 4>;
    using R = typename Rows::R;
    constexpr int kGroups = kNormThreads<kGroup> / kGroup, kAhead = Rows::kStages - 1, kPairs = R::kPairs;
    extern __shared__ __align__(128) unsigned char smem_dyn[];        // (off such a boundary a warp's copy is split, and its sectors are read twice)
    __shared__ float2 s_sum[kGroups][kGroup < 64 ? 1 : 2 * (kGroup / 32)];
    __shared__ long long s_scan[kNormThreads<kGroup> / 32 + 2];
    __shared__ Pair s_cols[kGroups > 1 ? kGroups : 1][kGroups > 1 ? kGroup * kPairs : 1];
    const int group = threadIdx.x / kGroup, t = threadIdx.x % kGroup;
    GroupSum<kGroup> sum{s_sum[group], 0, group};
    Rows ring{reinterpret_cast<typename Rows::Vec*>(smem_dyn) + threadIdx.x};
    chain_wait();
    chain_release();
    const T* const X = static_cast<const T*>(P.x);
    const T* const Y = static_cast<const T*>(P.y);
    const T* const dH = static_cast<const T*>(P.d_h);
    const T* const dU = static_cast<const T*>(P.d_u);
    typename R::Values w_pre;                            // of this thread's columns, for all rows
    R::param(P.w_pre, t, P.C, 1.f, w_pre);
    typename R::Values acc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int p = 0; p < kPairs; ++p) acc[k][p] = both(0.f);
    const Pair scale = both(P.scale);
    // sums k0 and k0 + 1 of all groups to row `at` of their partial sums
    auto flush = [&](int k0, int at) {
#pragma unroll
        for (int k = 0; k < (kLayer ? 2 : 1); ++k) {
            typename R::Values& a = acc[k0 + k];
            if (kGroups > 1) {
                __syncthreads();
#pragma unroll
                for (int p = 0; p < kPairs; ++p) s_cols[group][p * kGroup + t] = a[p];
                __syncthreads();
                if (group == 0) {
#pragma unroll 4
                    for (int g = 1; g < kGroups; ++g)            // (in this order; loads of several groups at a time)
#pragma unroll
                        for (int p = 0; p < kPairs; ++p) a[p] = add2(a[p], s_cols[g][p * kGroup + t]);
                }
            }
            if (group == 0) R::param_store(P.partial + (static_cast<size_t>(k0 == 0 ? k * P.slots : 2 * P.slots + k * gridDim.x) + at) * P.C, t, P.C, a);
#pragma unroll
            for (int p = 0; p < kPairs; ++p) a[p] = both(0.f);
        }
    };
    if (P.sel_idx) {
        // rows of dropped tokens: equal shares of all; a look at one token at a time is a chain of loads, so a warp looks at 32
        typename R::Values zero;
#pragma unroll
        for (int p = 0; p < kPairs; ++p) zero[p] = both(0.f);
        const long long all = static_cast<long long>(P.B) * P.N;
        const int lane = threadIdx.x & 31, n_warps = kNormThreads<kGroup> / 32, sub = kGroup < 32 ? lane / kGroup : 0;
        // a warp's share, or that of the warps of a group; the groups of a warp take its dropped tokens in turn
        const long long sharers = static_cast<long long>(gridDim.x) * (kGroup > 32 ? kGroups : n_warps), me = static_cast<long long>(blockIdx.x) * (kGroup > 32 ? kGroups : n_warps) + (kGroup > 32 ? group : static_cast<int>(threadIdx.x >> 5));
#pragma unroll 1
        for (long long i0 = me; i0 < all; i0 += sharers * 32) {
            const long long mine = i0 + lane * sharers;
            bool dropped = false;
            if (mine < all) dropped = __ldg(P.inv_idx + (P.S > 1 ? mine : mine % P.N)) < 0;
            unsigned left = __ballot_sync(0xffffffffu, dropped);
#pragma unroll 1
            for (int x = 0; left; ++x, left &= left - 1)
                if (kGroup >= 32 || x % (kGroup < 32 ? 32 / kGroup : 1) == sub) R::store(static_cast<T*>(P.dx) + (i0 + (__ffs(left) - 1) * sharers) * P.C, t, P.C, zero);
        }
    }
    Parts part;
    part.start(P, s_scan);
#pragma unroll 1
    while (part.next(P, group, kGroups)) {
        const int b = part.b;
        const RowIndex first = part.first;
        const RowWalk walk(P.sel_idx ? P.sel_idx + static_cast<size_t>(P.S > 1 ? b : 0) * P.N : nullptr, part);
        const size_t base = part.base_row;
        typename R::Values w, c;                         // N_post's scale and bias with the gate in them
        {
            typename R::Values g;
            R::param(P.gate ? P.gate + static_cast<size_t>(P.gate_rows > 1 ? b : 0) * P.C : nullptr, t, P.C, 1.f, g);
            R::param(P.w_post, t, P.C, 1.f, w);
            if (kLayer) R::param(P.b_post, t, P.C, 0.f, c);
#pragma unroll
            for (int p = 0; p < kPairs; ++p) {
                w[p] = mul2(w[p], g[p]);
                if (kLayer) c[p] = mul2(c[p], g[p]);
            }
        }
        const RowIndex behind = kGroup < 32 ? (threadIdx.x & 31) / kGroup : 0;
        RowIndex ahead = first, source = walk.source(first), from = source;
        int stage = 0;
        float4 st = walk.there(first) ? __ldg(P.stats + base + first) : make_float4(0.f, 0.f, 0.f, 0.f);
        auto fetch = [&](int to) {
            if (walk.there(ahead)) {
                const size_t row = (base + ahead) * P.C;
                ring.fetch(to, 0, X + (base + source) * P.C, t, P.C);
                ring.fetch(to, 1, Y ? Y + row : nullptr, t, P.C);
                ring.fetch(to, 2, dH ? dH + row : nullptr, t, P.C);
                ring.fetch(to, 3, dU ? dU + row : nullptr, t, P.C);
            }
            ring.commit();
            ahead += walk.step;
            source = walk.source(ahead);
        };
#pragma unroll
        for (int s = 0; s < kAhead; ++s) fetch(s);
#pragma unroll 1
        for (RowIndex i = first; walk.goes_on(i, behind); i += walk.step) {
            const int C = kGroup < 32 && !walk.there(i) ? 0 : P.C;
            fetch(stage + kAhead < Rows::kStages ? stage + kAhead : stage + kAhead - Rows::kStages);
            // of the next row, ahead of the wait
            const RowIndex from_next = walk.source(i + walk.step);
            const float4 st_next = walk.there(i + walk.step) ? __ldg(P.stats + base + i + walk.step) : make_float4(0.f, 0.f, 0.f, 0.f);
            ring.wait();
            const size_t row = (base + i) * P.C;
            typename R::Values h, zy, d;
            ring.read(stage, 0, X + (base + from) * P.C, t, C, h);
#pragma unroll
            for (int p = 0; p < kPairs; ++p) h[p] = mul2(h[p], scale);
            if (Y) {
                ring.read(stage, 1, Y + row, t, C, zy);
                const Pair r = both(st.y), minus = both(-st.x);
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    if (kLayer) zy[p] = add2(zy[p], minus);
                    zy[p] = mul2(zy[p], r);
                    if (kLayer) h[p] = add2(h[p], c[p]);
                    h[p] = fma2(zy[p], w[p], h[p]);
                }
            }
            if (dH) {
                ring.read(stage, 2, dH + row, t, C, d);
            } else {
#pragma unroll
                for (int p = 0; p < kPairs; ++p) d[p] = both(0.f);
            }
            if (P.pre) {
                typename R::Values du;
                ring.read(stage, 3, dU + row, t, C, du);
                Pair s0 = both(0.f), s1 = both(0.f);
                const Pair r = both(st.w), minus = both(-st.z);
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    if (kLayer) h[p] = add2(h[p], minus);
                    h[p] = mul2(h[p], r);                // (where no column is, du is 0)
                    acc[2][p] = fma2(du[p], h[p], acc[2][p]);
                    if (kLayer) acc[3][p] = add2(acc[3][p], du[p]);
                    du[p] = mul2(du[p], w_pre[p]);
                    s0 = fma2(du[p], h[p], s0);
                    if (kLayer) s1 = add2(s1, du[p]);
                }
                const float2 s = sum.template of<kLayer>(sum_of(s0), kLayer ? sum_of(s1) : 0.f);
                const Pair m0 = both(-s.x * P.inv_c), m1 = both(kLayer && P.pre == 2 ? -s.y * P.inv_c : 0.f);
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    if (kLayer) du[p] = add2(du[p], m1);
                    d[p] = fma2(r, fma2(h[p], m0, du[p]), d[p]);
                }
            }
            typename R::Values out;
#pragma unroll
            for (int p = 0; p < kPairs; ++p) out[p] = mul2(scale, d[p]);
            R::store(static_cast<T*>(P.dx) + (base + from) * P.C, t, C, out);
            if (Y) {
                Pair s0 = both(0.f), s1 = both(0.f);
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    acc[0][p] = fma2(d[p], zy[p], acc[0][p]);
                    if (kLayer) acc[1][p] = add2(acc[1][p], d[p]);
                    d[p] = mul2(d[p], w[p]);             // (0 where no column is)
                }
                if (P.post) {
#pragma unroll
                    for (int p = 0; p < kPairs; ++p) {
                        s0 = fma2(d[p], zy[p], s0);
                        if (kLayer) s1 = add2(s1, d[p]);
                    }
                    const float2 s = sum.template of<kLayer>(sum_of(s0), kLayer ? sum_of(s1) : 0.f);
                    const Pair m0 = both(-s.x * P.inv_c), m1 = both(kLayer && P.post == 2 ? -s.y * P.inv_c : 0.f), r = both(st.y);
#pragma unroll
                    for (int p = 0; p < kPairs; ++p) {
                        if (kLayer) d[p] = add2(d[p], m1);
                        d[p] = mul2(r, fma2(zy[p], m0, d[p]));
                    }
                }
                R::store(static_cast<T*>(P.dy) + row, t, C, d);
            }
            from = from_next;
            st = st_next;
            if (++stage == Rows::kStages) stage = 0;
        }
        if (P.gate_rows > 1) flush(0, part.slot);
    }
    if (P.gate_rows <= 1) flush(0, blockIdx.x);
    flush(2, blockIdx.x);
}

// ---- launches ----------------------------------------------------------------------------------------------------
// Allows a kernel its dynamic shared memory where that is above what every kernel may take.
template <class K>
cudaError_t allow_smem(K kernel, int bytes, int& attr_dev) {
    if (bytes <= 40 * 1024) return cudaSuccess;
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess || attr_dev == dev) return err;
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (err == cudaSuccess) attr_dev = dev;
    return err;
}
template <class T, int kV, int kGroup, int kPer, bool kLayer>
cudaError_t launch_fwd(int grid, const NormParams& P, cudaStream_t s) {
    constexpr int kBytes = Ring<T, kV, kGroup, kPer, 2>::kBytes;
    static thread_local int attr_dev = -1;
    if (cudaError_t err = allow_smem(norm_fwd_kernel<T, kV, kGroup, kPer, kLayer>, kBytes, attr_dev)) return err;
    return launch_chained(norm_fwd_kernel<T, kV, kGroup, kPer, kLayer>, dim3(grid), dim3(kNormThreads<kGroup>), kBytes, s, P);
}
template <class T, int kV, int kGroup, int kPer, bool kLayer>
cudaError_t launch_bwd(int grid, const NormParams& P, cudaStream_t s) {
    constexpr int kBytes = Ring<T, kV, kGroup, kPer, 4>::kBytes;
    static thread_local int attr_dev = -1;
    if (cudaError_t err = allow_smem(norm_bwd_kernel<T, kV, kGroup, kPer, kLayer>, kBytes, attr_dev)) return err;
    return launch_chained(norm_bwd_kernel<T, kV, kGroup, kPer, kLayer>, dim3(grid), dim3(kNormThreads<kGroup>), kBytes, s, P);
}
// Rows that are not taken in 16-byte vectors are bound by instructions, and a group of a power of two has up to twice the columns that a row has: where fewer elements a
// thread do, it gets fewer (5136 rows of 515 fp32, forward and backward: 43.4 us with 16 and 8, 35.0 with 10 and 6; 17 widths of 131 to 5101 columns, bf16 and fp32, are
// 12 to 105 % slower without it forward and 5 to 45 % both ways, where it applies to them).
template <class T, int kV, int kGroup, bool kLayer>
cudaError_t launch(bool bwd, int grid, const NormParams& P, cudaStream_t s) {
    constexpr bool kWide = kV * sizeof(T) == 16;
    if (bwd) {
        if constexpr (!kWide) {
            if (P.C <= kGroup * kBwdPerFew) return launch_bwd<T, kV, kGroup, kBwdPerFew, kLayer>(grid, P, s);
        }
        return launch_bwd<T, kV, kGroup, kBwdPer, kLayer>(grid, P, s);
    }
    if constexpr (kGroup * kFwdPer <= kNormMaxC) {
        if constexpr (!kWide) {
            if (P.C <= kGroup * kFwdPerFew) return launch_fwd<T, kV, kGroup, kFwdPerFew, kLayer>(grid, P, s);
        }
        return launch_fwd<T, kV, kGroup, kFwdPer, kLayer>(grid, P, s);
    }
    return cudaErrorInvalidValue;
}
template <class T, int kV, bool kLayer>
cudaError_t launch_group(bool bwd, int grid, const NormParams& P, cudaStream_t s) {
    switch (group_of(P.C, bwd ? kBwdPer : kFwdPer)) {
        case 8: return launch<T, kV, 8, kLayer>(bwd, grid, P, s);
        case 16: return launch<T, kV, 16, kLayer>(bwd, grid, P, s);
        case 32: return launch<T, kV, 32, kLayer>(bwd, grid, P, s);
        case 64: return launch<T, kV, 64, kLayer>(bwd, grid, P, s);
        case 128: return launch<T, kV, 128, kLayer>(bwd, grid, P, s);
        case 256: return launch<T, kV, 256, kLayer>(bwd, grid, P, s);
        case 512: return launch<T, kV, 512, kLayer>(bwd, grid, P, s);
        default: return launch<T, kV, 1024, kLayer>(bwd, grid, P, s);
    }
}
template <class T, int kV>
cudaError_t launch_layer(bool bwd, int grid, const NormParams& P, cudaStream_t s) {
    return P.pre == 2 || P.post == 2 ? launch_group<T, kV, true>(bwd, grid, P, s) : launch_group<T, kV, false>(bwd, grid, P, s);
}

}  // namespace

}  // namespace vardrop
