// Rows of logits for the kernels that read them: vectors of 16 bytes that start at any element, sums and maxima over a work-group.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sage {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A bfloat16 is held as its bits. VL: elements of a vector of 16 bytes.
template <class T>
struct RowType;
template <>
struct RowType<float> {
    static constexpr int VL = 4;
    __device__ static float at(const u32x4& v, int i) { return __uint_as_float(v[i]); }
    __device__ static float widen(float x) { return x; }
    __device__ static float narrow(float x) { return x; }
};
template <>
struct RowType<uint16_t> {
    static constexpr int VL = 8;
    __device__ static float at(const u32x4& v, int i) { return __uint_as_float(i & 1 ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16); }
    __device__ static float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    __device__ static uint16_t narrow(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }  // to nearest, ties to even
};

// 16 bytes at an address that is aligned to an element only (one load or store: gfx9 takes any alignment in global memory)
template <class T>
__device__ __forceinline__ u32x4 load16(const T* p) {
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
template <class T>
__device__ __forceinline__ void store16(T* p, const u32x4& v) {
    __builtin_memcpy(p, &v, 16);
}

// Elements e0 .. e0 + VL - 1 of a row of n as floats; those behind its end are `fill`.
template <class T>
__device__ __forceinline__ void row_floats(const T* row, int64_t e0, int64_t n, float fill, float* x) {
    constexpr int VL = RowType<T>::VL;
    if (e0 + VL <= n) {
        const u32x4 v = load16(row + e0);
#pragma unroll
        for (int i = 0; i < VL; ++i) x[i] = RowType<T>::at(v, i);
    } else {
#pragma unroll
        for (int i = 0; i < VL; ++i) x[i] = e0 + i < n ? RowType<T>::widen(row[e0 + i]) : fill;
    }
}

// Sums and maxima over the work-group, the same value in every thread. lds: one entry a wave; it is free again when the
// work-group has met once more.
template <int THREADS, class V, class Op>
__device__ __forceinline__ V group_reduce(V v, V* lds, Op op) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = op(v, __shfl_xor(v, d, 64));
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) v = op(v, lds[w]);
    }
    return v;
}

}  // namespace sage
