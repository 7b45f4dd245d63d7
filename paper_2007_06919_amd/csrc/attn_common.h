// What the two attention kernels share: operands of the matrix cores, exchanges between the
// lanes of a column, and the sum of the parts of split keys.
#pragma once

#include "internal.h"
#include "mfma_common.h"

namespace aqd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Operand {
    typedef T type __attribute__((ext_vector_type(8)));   // eight k of a row or column
};

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c, __bf16)
{
    typedef Operand<__bf16>::type V;
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c, _Float16)
{
    typedef Operand<_Float16>::type V;
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}

// two fp32 numbers rounded to T, the first in the low half
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    typedef T V __attribute__((ext_vector_type(2)));
    const V v = {(T)a, (T)b};
    return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float LOG2E = 1.44269504088896340736f;

// The parts of one row: [parts][dim] sums and, behind all rows' sums, [parts][2] references and totals,
// with which row `row` of `rows` is sum_p o_p 2^(ref_p - ref) / sum_p l_p 2^(ref_p - ref). One wave; no weight at all: zeros.
template <typename T>
__device__ __forceinline__ void join_parts(const float *part, long long rows, long long row, int all, int parts, int dim, T *y)
{
    const int lane = threadIdx.x & 63;
    const float *o = part + row * all * dim, *stat = part + rows * all * dim + row * all * 2;
    float ref = -INFINITY;
    for (int p = lane; p < parts; p += 64)
        ref = fmaxf(ref, stat[2 * p]);
    for (int d = 32; d; d >>= 1)
        ref = fmaxf(ref, __shfl_xor(ref, d));
    const float base = ref == -INFINITY ? 0.f : ref;
    float sum[4] = {}, total = 0.f;
    for (int p = 0; p < parts; ++p) {
        const float f = exp2_fast(stat[2 * p] - base);
        total += f * stat[2 * p + 1];
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (lane + 64 * v < dim)
                sum[v] += f * o[(long long)p * dim + lane + 64 * v];
    }
    const float inverse = total != 0.f ? 1.f / total : 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (lane + 64 * v < dim)
            y[lane + 64 * v] = (T)(sum[v] * inverse);
}

}  // namespace
}  // namespace aqd
