// Global gradient norm over many tensors, and clipping: norm = sqrt(sum g^2), out = g min(1, max_norm / (norm + eps)).
//
// grad_norm_kernel    the squares' sum of each CTA's chunks, in fp64.
// grad_scale_kernel   every CTA adds up those sums for itself (in one order, so all get the same factor) and scales its chunks.
//
// The tensors' table travels in the kernels' parameters: no copy to the device, nothing to keep alive, graphs hold it by value.
// Bound: memory.  The tensors are read twice, as far as they do not fit the L2 cache, and written once.
#include <cuda_fp16.h>

#include <algorithm>
#include <memory>
#include <new>

#include "common.cuh"
#include "kernels.h"

namespace vardrop {

namespace {

constexpr int kClipThreads = 256;
constexpr int kClipPerSm = 4;        // CTAs that an SM holds: 64 registers a thread, for a chunk that is on its way
constexpr int kClipMaxGrid = 2048;          // partial sums of a launch
constexpr int kClipFew = 64, kClipMany = 1024;      // table entries of a launch: the small one's parameters are 1.9 KB, the large one's 29 KB of the 32 KB a launch may take
constexpr int kClipLoads = 4;               // 16-byte vectors a thread has in flight
constexpr int kClipChunkBytes = kClipThreads * kClipLoads * 16;
constexpr int kClipMaxTensors = 16384;

template <int kMax>
struct ClipTable {
    const void* in[kMax];
    void* out[kMax];
    long long n[kMax];
    int first[kMax + 1];                    // chunks ahead of the tensor
    unsigned char dtype[kMax];
    int count;
    double* partial;                        // of all launches; this one's begin at `base`
    int base, partials;
    float max_norm, eps;
    float* norm;
    int* status;
};
static_assert(sizeof(ClipTable<kClipMany>) <= 32764, "a launch takes 32764 bytes of parameters");

struct Chunk {
    int tensor;
    int elem_log2;                          // of the element's size
    long long begin, from, to;              // virtual elements: of the chunk (a multiple of a vector), and that exist
    const unsigned char* base;              // of virtual element 0, a 16-byte boundary
};
// Elements are counted from the 16-byte boundary at or before the tensor's first one, so that every vector of a chunk is aligned; what of it is not the tensor's
// is not touched.
template <int kMax>
__device__ __forceinline__ Chunk chunk_at(const ClipTable<kMax>& P, int c) {
    int lo = 0, hi = P.count - 1;           // last tensor whose first chunk is not behind c (empty tensors have none)
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (P.first[mid] <= c) lo = mid;
        else hi = mid - 1;
    }
    Chunk k;
    k.tensor = lo;
    k.elem_log2 = P.dtype[lo] == 2 ? 2 : 1;
    const uintptr_t p = reinterpret_cast<uintptr_t>(P.in[lo]);
    k.base = reinterpret_cast<const unsigned char*>(p & ~static_cast<uintptr_t>(15));
    k.from = static_cast<long long>(p & 15) >> k.elem_log2;
    k.to = k.from + P.n[lo];
    k.begin = static_cast<long long>(c - P.first[lo]) * (kClipChunkBytes >> k.elem_log2);
    return k;
}

// the words of a vector that exist, zeros elsewhere
__device__ __forceinline__ uint4 load_vector(const Chunk& k, long long e) {
    const int per = 16 >> k.elem_log2;
    const unsigned char* p = k.base + (e << k.elem_log2);
    if (e >= k.from && e + per <= k.to) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (e + per > k.from && e < k.to) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (k.elem_log2 == 2) {
                if (e + i >= k.from && e + i < k.to) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    if (e + 2 * i + u >= k.from && e + 2 * i + u < k.to) w[i] |= static_cast<uint32_t>(reinterpret_cast<const unsigned short*>(p)[2 * i + u]) << (16 * u);
            }
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// This thread's vectors of a chunk.  Nearly every chunk lies inside its tensor: one look for all of it, and no 64-bit comparison a vector.
__device__ __forceinline__ bool inside(const Chunk& k) { return k.begin >= k.from && k.begin + (kClipChunkBytes >> k.elem_log2) <= k.to; }
__device__ __forceinline__ void load_chunk(const Chunk& k, uint4 (&v)[kClipLoads]) {
    if (inside(k)) {
        const uint4* p = reinterpret_cast<const uint4*>(k.base + (k.begin << k.elem_log2)) + threadIdx.x;
#pragma unroll
        for (int j = 0; j < kClipLoads; ++j) v[j] = p[j * kClipThreads];
    } else {
#pragma unroll
        for (int j = 0; j < kClipLoads; ++j) v[j] = load_vector(k, k.begin + (static_cast<long long>(j * kClipThreads + threadIdx.x) << (4 - k.elem_log2)));
    }
}
__device__ __forceinline__ float2 two_of(uint32_t w, int dtype) {        // of a 16-bit type
    if (dtype == 0) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
__device__ __forceinline__ uint32_t word_of(float a, float b, int dtype) {
    if (dtype == 0) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ double block_sum(double v, double* s_warp) {      // to every thread
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kClipThreads / 32; ++w) sum += s_warp[w];
    return sum;
}

// The squares of a 16-byte vector.  Conversions to fp64 run at 16 a cycle and SM, one an element would take 240 us of the 335 that the memory needs for 1.08e9 bf16 values (444
// us together): two squares are added in fp32, at two roundings, wherever both the sums are far inside its range, which squares leave at gradients of 2^64 and 2^-63.
template <int kType>
__device__ __forceinline__ double squares(const uint4 (&v)[kClipLoads]) {
    constexpr int kSums = kType == 2 ? 2 : 4;
    double total = 0.0;
#pragma unroll
    for (int j = 0; j < kClipLoads; ++j) {
        const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
        float2 x[kSums];
        float s[kSums];
#pragma unroll
        for (int i = 0; i < kSums; ++i) {
            x[i] = kType == 2 ? make_float2(__uint_as_float(w[2 * i % 4]), __uint_as_float(w[2 * i % 4 + 1])) : two_of(w[i], kType);
            s[i] = fmaf(x[i].x, x[i].x, x[i].y * x[i].y);
        }
        float least = s[0], most = s[0];
#pragma unroll
        for (int i = 1; i < kSums; ++i) {
            least = fminf(least, s[i]);
            most = fmaxf(most, s[i]);
        }
        if (least > 1e-30f && most < 1e30f) {
#pragma unroll
            for (int i = 0; i < kSums; ++i) total += static_cast<double>(s[i]);
        } else {                                         // (zeros come here too, and what is not finite: minimum and maximum pass over a NaN, but not its sum)
#pragma unroll
            for (int i = 0; i < kSums; ++i) {
                const double a = x[i].x, b = x[i].y;
                total += fma(a, a, b * b);
            }
        }
    }
    return total;
}

template <int kMax>
__global__ void __launch_bounds__(kClipThreads, kClipPerSm) grad_norm_kernel(const __grid_constant__ ClipTable<kMax> P) {
    __shared__ double s_warp[kClipThreads / 32];
    chain_wait();
    chain_release();
    const int chunks = P.first[P.count];
    double sum = 0.0;
    uint4 v[2][kClipLoads];                 // of this chunk and of the next
    int dtype[2];
    auto fetch = [&](int c, int to) {
        if (c >= chunks) return;
        const Chunk k = chunk_at(P, c);
        dtype[to] = P.dtype[k.tensor];
        load_chunk(k, v[to]);
    };
    const int step = gridDim.x;
    int c = blockIdx.x;
    fetch(c, 0);
#pragma unroll 1
    for (; c < chunks; c += 2 * step) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int at = c + half * step;
            fetch(at + step, half ^ 1);
            if (at >= chunks) break;
            sum += dtype[half] == 0 ? squares<0>(v[half]) : dtype[half] == 1 ? squares<1>(v[half]) : squares<2>(v[half]);
        }
    }
    const double total = block_sum(sum, s_warp);
    if (threadIdx.x == 0) P.partial[P.base + blockIdx.x] = total;
}

template <int kMax>
__global__ void __launch_bounds__(kClipThreads, kClipPerSm) grad_scale_kernel(const __grid_constant__ ClipTable<kMax> P) {
    __shared__ double s_warp[kClipThreads / 32];
    // The first chunk is on its way while the norm is still being taken: the launch before this one is always this library's grad_norm_kernel (or a scaling of other tensors), which
    // writes no gradient and lets dependents in behind its own wait only, so whatever made the gradients has completed.
    const int chunks = P.max_norm == 0.f ? 0 : P.first[P.count];
    auto fetch = [&](int c, Chunk& k, uint4 (&v)[kClipLoads]) {
        k = chunk_at(P, c);
        load_chunk(k, v);
    };
    int c = chunks - 1 - static_cast<int>(blockIdx.x);      // from the end: what the norm's pass read last is in L2
    Chunk k{};
    uint4 v[kClipLoads];
    if (c >= 0) fetch(c, k, v);
    chain_wait();
    chain_release();
    double sum = 0.0;
    for (int i = threadIdx.x; i < P.partials; i += kClipThreads) sum += P.partial[i];
    const double norm = sqrt(block_sum(sum, s_warp));
    const bool finite = isfinite(norm);
    if (blockIdx.x == 0 && threadIdx.x == 0 && P.base == 0) {
        *P.norm = static_cast<float>(norm);
        if (!finite) set_status(P.status, VARDROP_ERR_NONFINITE);
    }
    const double ratio = P.max_norm / (norm + P.eps);
    const float factor = finite && ratio < 1.0 ? static_cast<float>(ratio) : 1.f;
#pragma unroll 1
    while (c >= 0) {
        const int dtype = P.dtype[k.tensor];
        unsigned char* out = static_cast<unsigned char*>(P.out[k.tensor]);
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(P.in[k.tensor])) & 15) == 0;
        const bool plain = same && inside(k);
        const bool skip = factor == 1.f && out == P.in[k.tensor];
        out -= k.from << k.elem_log2;                   // of virtual element 0
        const int per = 16 >> k.elem_log2;
#pragma unroll
        for (int j = 0; j < kClipLoads; ++j) {
            if (skip) break;
            const long long e = k.begin + static_cast<long long>(j * kClipThreads + threadIdx.x) * per;
            uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (dtype == 2) {
                    w[i] = __float_as_uint(__uint_as_float(w[i]) * factor);
                } else {
                    const float2 x = two_of(w[i], dtype);
                    w[i] = word_of(x.x * factor, x.y * factor, dtype);
                }
            }
            if (plain || (same && e >= k.from && e + per <= k.to)) {
                *reinterpret_cast<uint4*>(out + (e << k.elem_log2)) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (dtype == 2) {
                        if (e + i >= k.from && e + i < k.to) reinterpret_cast<uint32_t*>(out)[e + i] = w[i];
                    } else {
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            if (e + 2 * i + u >= k.from && e + 2 * i + u < k.to) reinterpret_cast<unsigned short*>(out)[e + 2 * i + u] = static_cast<unsigned short>(w[i] >> (16 * u));
                    }
                }
            }
        }
        c -= gridDim.x;
        if (c >= 0) fetch(c, k, v);
    }
}

// The launches' tables one after another: `tensors` from `at` on, as many as a launch takes.
template <int kMax>
int fill(ClipTable<kMax>& P, const vardrop_tensor* tensors, int at, int count) {
    P.count = count - at < kMax ? count - at : kMax;
    long long chunks = 0;
    for (int i = 0; i < P.count; ++i) {
        const vardrop_tensor& t = tensors[at + i];
        const int log2 = t.dtype == 2 ? 2 : 1;
        const long long shift = static_cast<long long>(reinterpret_cast<uintptr_t>(t.in) & 15) >> log2, per = kClipChunkBytes >> log2;
        P.in[i] = t.in; P.out[i] = t.out; P.n[i] = t.n; P.dtype[i] = static_cast<unsigned char>(t.dtype);
        P.first[i] = static_cast<int>(chunks);
        if (t.n > 0) chunks += (shift + t.n + per - 1) / per;
        if (chunks > (1ll << 30)) return fail(VARDROP_ERR_UNSUPPORTED, "grad_clip: more than 2^30 chunks of 16 KB in a launch");
    }
    P.first[P.count] = static_cast<int>(chunks);
    return VARDROP_OK;
}
// An output may overlap neither another one, which two CTAs would scale at a time, nor another tensor's input, which is read ahead of it or behind.  Tensors that are clipped in place
// mostly come in the order of their addresses, where a look at neighbours is enough.
int outputs_apart(const vardrop_tensor* tensors, int count) {
    struct Span { uintptr_t begin, end; bool written; };
    const auto span = [&](int i, const void* p, bool written) {
        const uintptr_t begin = reinterpret_cast<uintptr_t>(p);
        return Span{begin, begin + (static_cast<uintptr_t>(tensors[i].n) << (tensors[i].dtype == 2 ? 2 : 1)), written};
    };
    uintptr_t last = 0;
    bool ascending = true;
    for (int i = 0; i < count && ascending; ++i) {
        if (tensors[i].n == 0) continue;
        const Span s = span(i, tensors[i].out, true);
        ascending = tensors[i].in == tensors[i].out && s.begin >= last;
        last = s.end;
    }
    if (ascending) return VARDROP_OK;
    const std::unique_ptr<Span[]> spans(new (std::nothrow) Span[2 * static_cast<size_t>(count)]);
    if (!spans) return fail(VARDROP_ERR_INVALID_ARG, "grad_clip: no host memory for %d tensors", count);
    int n = 0;
    for (int i = 0; i < count; ++i) {
        if (tensors[i].n == 0) continue;
        spans[n++] = span(i, tensors[i].out, true);
        if (tensors[i].in != tensors[i].out) spans[n++] = span(i, tensors[i].in, false);
    }
    std::sort(spans.get(), spans.get() + n, [](const Span& a, const Span& b) { return a.begin < b.begin; });
    uintptr_t written = 0, read = 0;                     // ends of the spans so far
    for (int i = 0; i < n; ++i) {
        const Span& s = spans[i];
        if (s.begin < written || (s.written && s.begin < read)) return fail(VARDROP_ERR_INVALID_ARG, "grad_clip: an output overlaps another output or another tensor's input");
        (s.written ? written : read) = std::max(s.written ? written : read, s.end);
    }
    return VARDROP_OK;
}
int grid_of(int chunks) {
    const int most = kClipPerSm * sm_count() < kClipMaxGrid ? kClipPerSm * sm_count() : kClipMaxGrid;
    return chunks < 1 ? 1 : chunks < most ? chunks : most;
}

template <int kMax>
int clip_launch(const vardrop_tensor* tensors, int count, const vardrop_clip_cfg& cfg, float* norm, void* ws, cudaStream_t stream) {
    ClipTable<kMax> P;
    P.partial = reinterpret_cast<double*>(static_cast<char*>(ws) + kWsHeaderBytes);
    P.max_norm = cfg.max_norm; P.eps = cfg.eps; P.norm = norm; P.status = static_cast<int*>(ws);
    P.base = 0; P.partials = 0;
    for (int at = 0; at < count; at += kMax) {          // refuse before anything is launched
        if (int st = fill(P, tensors, at, count)) return st;
    }
    for (int at = 0; at < count; at += kMax) {
        fill(P, tensors, at, count);
        const int grid = grid_of(P.first[P.count]);
        P.base = P.partials;
        LaunchScope ls_(K_GRAD_NORM, stream);
        if (int st = check_cuda(launch_chained(grad_norm_kernel<kMax>, dim3(grid), dim3(kClipThreads), 0, stream, P), "grad_clip: norm launch")) return st;
        P.partials += grid;
    }
    for (int at = 0; at == 0 || at < count; at += kMax) {       // (of no tensors the norm is zero)
        fill(P, tensors, at, count);
        P.base = at;
        LaunchScope ls_(K_GRAD_SCALE, stream);
        if (int st = check_cuda(launch_chained(grad_scale_kernel<kMax>, dim3(cfg.max_norm == 0.f ? 1 : grid_of(P.first[P.count])), dim3(kClipThreads), 0, stream, P), "grad_clip: scale launch")) return st;
        if (cfg.max_norm == 0.f) break;
    }
    return VARDROP_OK;
}

}  // namespace

size_t grad_clip_workspace_bytes() {
    return kWsHeaderBytes + static_cast<size_t>(kClipMaxTensors / kClipMany) * kClipMaxGrid * sizeof(double);
}

int grad_clip_validate(const vardrop_tensor* tensors, int32_t count, const vardrop_clip_cfg& cfg) {
    if (count < 0 || (count > 0 && !tensors)) return fail(VARDROP_ERR_INVALID_ARG, "grad_clip: %d tensors, table at %p", count, static_cast<const void*>(tensors));
    if (count > kClipMaxTensors) return fail(VARDROP_ERR_UNSUPPORTED, "grad_clip: %d tensors (at most %d)", count, kClipMaxTensors);
    if (!(cfg.max_norm >= 0.f) || !(cfg.eps >= 0.f)) return fail(VARDROP_ERR_INVALID_ARG, "grad_clip: max_norm and eps must be >= 0");
    for (int i = 0; i < count; ++i) {
        const vardrop_tensor& t = tensors[i];
        if (t.dtype < 0 || t.dtype > 2) return fail(VARDROP_ERR_INVALID_ARG, "grad_clip: tensor %d has type %d (0 bf16, 1 fp16, 2 fp32)", i, t.dtype);
        if (t.n < 0 || t.n > (1ll << 40)) return fail(VARDROP_ERR_INVALID_ARG, "grad_clip: tensor %d has %lld elements", i, static_cast<long long>(t.n));
        if (t.n == 0) continue;
        const uintptr_t mask = t.dtype == 2 ? 3 : 1, in = reinterpret_cast<uintptr_t>(t.in), out = reinterpret_cast<uintptr_t>(t.out);
        if (!t.in || (in & mask)) return fail(VARDROP_ERR_INVALID_ARG, "grad_clip: tensor %d is NULL or not aligned to its elements", i);
        if (cfg.max_norm == 0.f) continue;
        if (!t.out || (out & mask)) return fail(VARDROP_ERR_INVALID_ARG, "grad_clip: output %d is NULL or not aligned to its elements", i);
        const uintptr_t bytes = static_cast<uintptr_t>(t.n) * (mask + 1);
        if (in != out && in < out + bytes && out < in + bytes) return fail(VARDROP_ERR_INVALID_ARG, "grad_clip: output %d overlaps its input", i);
    }
    return cfg.max_norm == 0.f ? VARDROP_OK : outputs_apart(tensors, count);
}

int grad_clip_launch(const vardrop_tensor* tensors, int32_t count, const vardrop_clip_cfg& cfg, float* norm, void* ws, cudaStream_t stream) {
    return count <= kClipFew ? clip_launch<kClipFew>(tensors, count, cfg, norm, ws, stream) : clip_launch<kClipMany>(tensors, count, cfg, norm, ws, stream);
}

}  // namespace vardrop
