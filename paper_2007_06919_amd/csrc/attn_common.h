// What the two attention kernels share: operands of the matrix cores, the row tiles of sequences that
// differ in length, copies into LDS, and the sum of the parts of split keys.
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

// sums over the lanes up to one's own
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);   // the lanes 1, 2, 4 and 8 below, in 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // lane 15 of the 16 below
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // lane 31
    return x;
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

// Where sequences differ in length, most of a grid of the longest one's row tiles for each would have no rows. Row tile `item` of all
// sequences' (tiles_of(b) each, `tiles` at most) instead: those of up to 256 sequences by their number in the sequence, the highest first (they see most keys);
// those of more one sequence after the other. False past the last one.
template <typename F>
__device__ __forceinline__ bool find_tile(int batch, int tiles, int item, F tiles_of, int &sequence_at, int &tile)
{
    const int lane = threadIdx.x & 63;
    if (batch <= 256) {
        int count[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            count[k] = 64 * k + lane < batch ? tiles_of(64 * k + lane) : 0;
        // how many have the number `least` or a higher one
        auto from = [&](int least) {
            int n = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                n += max(count[k] - least, 0);
            return wave_sum(n);
        };
        if (item >= from(0))
            return false;
        int low = 0, high = tiles, above = 0;   // from(low) > item >= from(high) == above
        while (high - low > 1) {
            const int middle = (low + high) / 2, n = from(middle);
            if (n > item) {
                low = middle;
            } else {
                high = middle;
                above = n;
            }
        }
        int rest = item - above;
        tile = low;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint64_t has = __builtin_amdgcn_ballot_w64(count[k] > low);
            const int n = __builtin_popcountll(has);
            if (rest >= 0 && rest < n) {
                const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0));
                sequence_at = 64 * k + __builtin_ctzll(__builtin_amdgcn_ballot_w64(count[k] > low && before == rest));
                return true;
            }
            rest -= n;
        }
        return false;
    }
    // a lane has `each` sequences, then those of the lane that has the item are the lanes'
    int first = 0, last = batch, rest = item;
    for (;;) {
        const int each = (last - first + 63) / 64, begin = min(first + lane * each, last), end = min(begin + each, last);
        int n = 0;
        for (int b = begin; b < end; ++b)
            n += tiles_of(b);
        int upto = n;   // with the lanes below
        for (int d = 1; d < 64; d <<= 1) {
            const int x = __shfl_up(upto, d);
            upto += lane >= d ? x : 0;
        }
        const uint64_t past = __builtin_amdgcn_ballot_w64(upto > rest);
        if (!past)
            return false;
        const int at = __builtin_ctzll(past);
        rest -= __builtin_amdgcn_readlane(upto - n, at);
        first = __builtin_amdgcn_readlane(begin, at);
        last = __builtin_amdgcn_readlane(end, at);
        if (each == 1) {
            sequence_at = first;
            tile = __builtin_amdgcn_readlane(n, at) - 1 - rest;
            return true;
        }
    }
}

// How many parts of `chunk` keys the first `limit` are in, one at least. (limit + chunk may pass 32 bits.)
__device__ __forceinline__ int parts_of(int limit, int chunk) { return limit > 0 ? (limit - 1) / chunk + 1 : 1; }

// The parts of one row, sums o [dim] and references and totals stat [2], `step` rows from part to part: the row is
// sum_p o_p 2^(ref_p - ref) / sum_p l_p 2^(ref_p - ref), zeros where there is no weight at all. WAVES waves (1 for few parts: rows
// are many then, and a wave needs no barrier), of which 16, 32 or 64 lanes have four channels of a part each.
template <int WAVES>
struct JoinScratch {
    f32x4 sum[WAVES][64];
    float most[WAVES], total[WAVES];
};
// Parts that one wave joins: 192 rows of 10 parts 14.8 us with what makes them, 16.6 with four waves a row; 192 of 90 87 and 83.
constexpr int JOIN_FEW = 16;

template <typename T, int WAVES>
__device__ __forceinline__ void join_parts(JoinScratch<WAVES> &lds, const float *o, const float *stat, long long step, int parts, int dim, T *y)
{
    const long long o_step = step * dim, stat_step = step * 2;
    const int lanes = dim <= 64 ? 16 : dim <= 128 ? 32 : 64, each = 64 * WAVES / lanes;
    const int thread = WAVES > 1 ? threadIdx.x : threadIdx.x & 63, wave = thread >> 6;
    const int c = thread % lanes * 4, first = c < dim ? thread / lanes : parts;
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
            early[u] = *(const f32x4 *)(o + p * o_step + c);
            early_ref[u] = stat[p * stat_step];
            early_total[u] = stat[p * stat_step + 1];
        }
    }
    float ref = -INFINITY;
    for (int p = thread; p < parts; p += 64 * WAVES)
        ref = fmaxf(ref, stat[p * stat_step]);
    for (int d = 32; d; d >>= 1)
        ref = fmaxf(ref, __shfl_xor(ref, d));
    if constexpr (WAVES > 1) {
        if ((thread & 63) == 0)
            lds.most[wave] = ref;
        __syncthreads();
        for (int w = 0; w < WAVES; ++w)
            ref = fmaxf(ref, lds.most[w]);
    }
    const float base = ref == -INFINITY ? 0.f : ref;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    auto add = [&](float r, float l, f32x4 v) {
        const float f = exp2_fast(r - base);
        total += f * l;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            sum[e] += f * v[e];
    };
#pragma unroll
    for (int u = 0; u < EARLY; ++u)
        add(early_ref[u], early_total[u], early[u]);
#pragma unroll 4
    for (int p = first + EARLY * each; p < parts; p += each)
        add(stat[p * stat_step], stat[p * stat_step + 1], *(const f32x4 *)(o + p * o_step + c));
    // over the lanes of one channel
    for (int d = lanes; d < 64; d <<= 1) {
        total += __shfl_xor(total, d);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            sum[e] += __shfl_xor(sum[e], d);
    }
    if constexpr (WAVES > 1) {
        lds.sum[wave][thread & 63] = sum;
        if ((thread & 63) == 0)
            lds.total[wave] = total;
        __syncthreads();
        if (wave)
            return;
        total = lds.total[0];
        for (int w = 1; w < WAVES; ++w) {
            total += lds.total[w];
            const f32x4 more = lds.sum[w][thread];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum[e] += more[e];
        }
    }
    if (thread >= lanes || c >= dim)
        return;
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
