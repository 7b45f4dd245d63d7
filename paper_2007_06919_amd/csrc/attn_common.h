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

// sum + both numbers of a pair
__device__ __forceinline__ float add2(uint32_t a, float sum, __bf16)
{
    typedef __bf16 V __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(V, a), V{(__bf16)1.f, (__bf16)1.f}, sum, false);
}
__device__ __forceinline__ float add2(uint32_t a, float sum, _Float16)
{
    typedef _Float16 V __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(V, a), V{(_Float16)1.f, (_Float16)1.f}, sum, false);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float LOG2E = 1.44269504088896340736f;

// The parts of one row, sums [parts][dim] and, behind all rows' sums, [parts][2] references and totals: the row is
// sum_p o_p 2^(ref_p - ref) / sum_p l_p 2^(ref_p - ref), zeros where there is no weight at all. One workgroup of four waves: 64 lanes
// have four channels each, or for shorter rows several parts at a time.
struct JoinScratch {
    float sum[256][4], most[4], total[4];
};
template <typename T>
__device__ __forceinline__ void join_parts(JoinScratch &lds, const float *part, long long rows, long long row, int all, int parts, int dim, T *y)
{
    const float *o = part + row * all * dim, *stat = part + rows * all * dim + row * all * 2;
    const int lanes = (dim + 3) / 4, each = 256 / lanes, c = threadIdx.x % lanes * 4;
    const int first = (int)threadIdx.x < each * lanes ? threadIdx.x / lanes : parts;
    // the first loads of the sums are under way with those of the references
    constexpr int EARLY = 4;
    f32x4 early[EARLY];
    float early_ref[EARLY], early_total[EARLY];
#pragma unroll
    for (int u = 0; u < EARLY; ++u) {
        const int p = first + u * each;
        early[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        early_ref[u] = -INFINITY;
        early_total[u] = 0.f;
        if (p < parts) {
            early[u] = *(const f32x4 *)(o + (long long)p * dim + c);
            early_ref[u] = stat[2 * p];
            early_total[u] = stat[2 * p + 1];
        }
    }
    float ref = -INFINITY;
    for (int p = threadIdx.x; p < parts; p += 256)
        ref = fmaxf(ref, stat[2 * p]);
    for (int d = 32; d; d >>= 1)
        ref = fmaxf(ref, __shfl_xor(ref, d));
    if ((threadIdx.x & 63) == 0)
        lds.most[threadIdx.x >> 6] = ref;
    __syncthreads();
    ref = fmaxf(fmaxf(lds.most[0], lds.most[1]), fmaxf(lds.most[2], lds.most[3]));
    const float base = ref == -INFINITY ? 0.f : ref;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
#pragma unroll
    for (int u = 0; u < EARLY; ++u) {
        const float f = exp2_fast(early_ref[u] - base);
        total += f * early_total[u];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            sum[e] += f * early[u][e];
    }
#pragma unroll 4
    for (int p = first + EARLY * each; p < parts; p += each) {
        const float f = exp2_fast(stat[2 * p] - base);
        const f32x4 v = *(const f32x4 *)(o + (long long)p * dim + c);
        total += f * stat[2 * p + 1];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            sum[e] += f * v[e];
    }
    *(f32x4 *)lds.sum[threadIdx.x] = sum;
    // every lane of a part has its total; those of the first channels are added
    float mine = c == 0 ? total : 0.f;
    for (int d = 32; d; d >>= 1)
        mine += __shfl_xor(mine, d);
    if ((threadIdx.x & 63) == 0)
        lds.total[threadIdx.x >> 6] = mine;
    __syncthreads();
    if ((int)threadIdx.x >= lanes)
        return;
    for (int i = 1; i < each; ++i)
        sum += *(const f32x4 *)lds.sum[threadIdx.x + i * lanes];
    total = lds.total[0] + lds.total[1] + lds.total[2] + lds.total[3];
    const float inverse = total != 0.f ? 1.f / total : 0.f;
    typedef T V __attribute__((ext_vector_type(4), aligned(2)));
    V v;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = (T)(sum[e] * inverse);
    *(V *)(y + c) = v;
}

// 16 or 4 bytes per lane from `offset` bytes past a wave-uniform address straight into LDS at la + 16 * lane
// or 4 * lane (see dma16)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16(const uint8_t *base, uint32_t offset, uint32_t la)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(la), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void copy4(const uint8_t *base, uint32_t offset, uint32_t la)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(la), "v"(offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

}  // namespace
}  // namespace aqd
