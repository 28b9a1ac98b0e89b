// Consecutive elements of a row as one aligned access, bf16, fp16 or fp32, in fp32 registers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace vardrop {

template <class T, int N>
struct alignas(N * sizeof(T) > 16 ? 16 : N * sizeof(T)) Pack {
    T e[N];
};
// (As whole words: one access whatever the elements' type.)
template <int kBytes>
struct Word;
template <> struct Word<2> { using type = uint16_t; };
template <> struct Word<4> { using type = uint32_t; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<16> { using type = uint4; };
template <class T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
    constexpr int kBytes = N * sizeof(T) > 16 ? 16 : N * sizeof(T);
    using W = typename Word<kBytes>::type;
    Pack<T, N> v;
#pragma unroll
    for (int i = 0; i < static_cast<int>(N * sizeof(T)) / kBytes; ++i) {
        const W w = reinterpret_cast<const W*>(p)[i];
        memcpy(reinterpret_cast<char*>(&v) + i * kBytes, &w, kBytes);
    }
    return v;
}
template <class T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& v) {
    constexpr int kBytes = N * sizeof(T) > 16 ? 16 : N * sizeof(T);
    using W = typename Word<kBytes>::type;
#pragma unroll
    for (int i = 0; i < static_cast<int>(N * sizeof(T)) / kBytes; ++i) {
        W w;
        memcpy(&w, reinterpret_cast<const char*>(&v) + i * kBytes, kBytes);
        reinterpret_cast<W*>(p)[i] = w;
    }
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <class T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// bf16, fp16, fp32 by the numbers that configurations use
inline bool known_dtype(int dtype) { return dtype >= 0 && dtype <= 2; }
inline size_t dtype_bytes(int dtype) { return dtype == 2 ? 4 : 2; }
template <class F>
cudaError_t with_dtype(int dtype, F f) {
    return dtype == 0 ? f(__nv_bfloat16{}) : dtype == 1 ? f(__half{}) : f(float{});
}
// elements of one access in rows of C: the largest power of two up to 8 that divides every row's offset
inline int row_vector(long long C) { return C % 8 == 0 ? 8 : C % 4 == 0 ? 4 : C % 2 == 0 ? 2 : 1; }
template <int N>
struct VecSize {
    static constexpr int value = N;
};
template <class F>
cudaError_t with_vector(int n, F f) {
    return n == 8 ? f(VecSize<8>{}) : n == 4 ? f(VecSize<4>{}) : n == 2 ? f(VecSize<2>{}) : f(VecSize<1>{});
}

}  // namespace vardrop
