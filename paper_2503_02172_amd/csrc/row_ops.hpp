// Device helpers of the kernels that read whole rows of a caller's matrix
// (drawing, distillation, embedding rows): rows of float32 or bfloat16 with
// any row stride, so that a row starts at any element.
#pragma once

#include "kgq_internal.hpp"

namespace kgq {

// Elements of a row are float or uint16_t (bfloat16 bits).
__device__ __forceinline__ float row_value(float x) { return x; }
__device__ __forceinline__ float row_value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// float32 to an element: bfloat16 by round to nearest even (the one rounding
// of a bfloat16 output; everything before it is float32 or wider).
template <typename T>
__device__ __forceinline__ T row_element(float x);
template <>
__device__ __forceinline__ float row_element<float>(float x)
{
    return x;
}
template <>
__device__ __forceinline__ uint16_t row_element<uint16_t>(float x)
{
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// 16 bytes of a row at an element's alignment (global memory takes them at
// any address).
template <typename T>
struct RowVec;
template <>
struct RowVec<float> {
    static constexpr int n = 4;
    typedef float type __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct RowVec<uint16_t> {
    static constexpr int n = 8;
    typedef uint16_t type __attribute__((ext_vector_type(8), aligned(2)));
};

// Sum or maximum of a value over the workgroup, every thread gets it, in one
// order whatever the timing. buf: one element per wavefront; a barrier before
// its next use is the caller's.
template <typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V x, Op op)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = op(x, __shfl_xor(x, d, 64));
    return x;
}
template <int WAVES, typename V, typename Op>
__device__ __forceinline__ V block_reduce(V x, V* buf, Op op)
{
    x = wave_reduce(x, op);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
    __syncthreads();
    V r = buf[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) r = op(r, buf[w]);
    return r;
}

struct OpSum {
    template <typename V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};
struct OpMax {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }   // a NaN is passed over
    __device__ __forceinline__ double operator()(double a, double b) const { return fmax(a, b); }
};

}  // namespace kgq
