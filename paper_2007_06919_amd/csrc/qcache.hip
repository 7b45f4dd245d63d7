// Keys and values into and out of a cache of 4-bit codes with a bf16 scale per group of
// channels. Definition and layout: include/aqd.h.
//
// A lane holds 8 channels of a token's head. A group's largest magnitude with its sign is
// one unsigned integer (the magnitude's bits above a bit that is set for positive numbers), so one
// maximum over a group's lanes finds both and prefers the positive number, with infinities and NaN
// above all others. Adding 1.5 * 2^23 rounds to the nearest even integer and leaves it in the low bits, from
// which the next shift takes it. The values' nibbles of one unit come from four lanes, which
// exchange their words.
//
// A workgroup has tokens of one head; four tokens next to one another share their lines of the cache. The heads of the same tokens
// follow one another in the launch (write and read of 16384 tokens of 8 heads, dim 128, bf16: 41 us, 45 with the tokens of a head
// first; 33.8 since the read's stores pass the L2 by).
//
// Bound by HBM: 85 MB each way there, 67 of them bf16; a write takes 20 us, a read 14 us.

#include <algorithm>

#include "internal.h"

namespace aqd {
namespace {

template <typename T>
struct Eight {
    typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};

template <typename T>
__device__ __forceinline__ void load8(const void *p, long long at, float *f)
{
    const auto v = *(const typename Eight<T>::type *)((const T *)p + at);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        f[e] = (float)v[e];
}

struct Group {
    float inverse, scale;   // of codes, and as stored
    bool number;
};

// the scale of a group from its maximum
__device__ __forceinline__ Group group_of(uint32_t top)
{
    const float a = __uint_as_float(top >> 1 | (top & 1 ? 0u : 0x80000000u));
    Group g;
    g.number = top >> 1 < 0x7F800000u;
    g.scale = (float)(__bf16)(a * -0.125f);
    if (!(fabsf(g.scale) >= 0x1p-119f))
        g.scale = 0.f;
    g.inverse = g.scale != 0.f ? 1.f / g.scale : 0.f;
    if (!g.number)
        g.scale = NAN;
    return g;
}

// the larger of a lane's number and that of a lane of its 16: CONTROL 0xB1 the neighbour, 0x4E two further, 0x141 and 0x140 the
// mirrored one of 8 and of 16, which are those 4 and 8 further once neighbours have one number
template <int CONTROL>
__device__ __forceinline__ uint32_t larger(uint32_t a)
{
    const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, CONTROL, 0xF, 0xF, true);
    return a > b ? a : b;
}

// codes of 8 channels, channel i in nibble i; lanes: those of a group (4, 8 or 16)
__device__ __forceinline__ uint32_t quantise(const float *x, int lanes, Group &g)
{
    float high = x[0], low = x[0], check = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        high = fmaxf(high, x[e]);
        low = fminf(low, x[e]);
        check = __builtin_fmaf(x[e], 0.f, check);   // NaN from an infinity or a NaN
    }
    uint32_t top = __float_as_uint(fmaxf(high, -low)) << 1 | (high >= -low ? 1u : 0u);
    if (check != 0.f)
        top = 0xFFFFFFFFu;
    top = larger<0x4E>(larger<0xB1>(top));
    if (lanes > 4)
        top = larger<0x141>(top);
    if (lanes > 8)
        top = larger<0x140>(top);
    g = group_of(top);
    constexpr float ROUND = 0x1.8p23f;   // and 8, in its low bits
    uint32_t w = 0, rest = 0;
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        w = (w << 4) + __float_as_uint(__builtin_amdgcn_fmed3f(x[e] * g.inverse, -8.f, 7.f) + (ROUND + 8.f));
        rest = (rest << 4) + __builtin_bit_cast(uint32_t, ROUND);
    }
    return g.number ? w - rest : 0x88888888u;
}

// nibbles 0 .. 7 to the places of key channels: 2 j to j, 2 j + 1 to j + 4
__device__ __forceinline__ uint32_t key_word(uint32_t w)
{
    uint32_t even = w & 0x0F0F0F0Fu, odd = (w >> 4) & 0x0F0F0F0Fu;
    even = (even | (even >> 4)) & 0x00FF00FFu;
    odd = (odd | (odd >> 4)) & 0x00FF00FFu;
    return ((even | (even >> 8)) & 0xFFFFu) | (odd | (odd >> 8)) << 16;
}

// the block of a slot's page, and the token in it; null for slots outside of the cache
struct Place {
    uint8_t *block;
    int t;
};

__device__ __forceinline__ Place place_of(const QcacheArgs &A, int token, int head)
{
    const int slot = A.slots[token];
    if (slot < 0 || slot >= A.c.pages * A.c.page)
        return {nullptr, 0};
    return {A.cache + ((long long)(slot >> __builtin_ctz(A.c.page)) * A.c.heads + head) * A.c.block_bytes, slot & (A.c.page - 1)};
}

// lane c = 8 h + 2 n + s of a head's has channels 64 h + 16 n + 8 s .. + 7, and of the values' units m = 8 s + 2 n and the next, whose
// nibbles n' are those of lane 8 h + 2 n' + s
__device__ __forceinline__ uint32_t from_lane(uint32_t w, int n) { return (uint32_t)__shfl((int)w, ((threadIdx.x & 63) & ~6) | n << 1); }

template <typename T, int DIM>
__global__ void __launch_bounds__(256) qcache_write_kernel(QcacheArgs A)
{
    constexpr int LANES = DIM / 8, EACH = 256 / LANES;
    const int c = threadIdx.x % LANES, n = c >> 1 & 3, head = blockIdx.x, group_log = __builtin_ctz(A.c.group), groups = DIM >> group_log;
    const int scales = A.c.page * DIM;
    for (long long at = blockIdx.y * EACH + threadIdx.x / LANES; at < A.tokens; at += gridDim.y * EACH) {
        const int token = (int)at;
        const Place p = place_of(A, token, head);
        if (!p.block)
            continue;   // all lanes of a token together
        float x[8], y[8];
        load8<T>(A.k, token * A.k_token + head * A.k_head + 8 * c, x);
        load8<T>(A.v, token * A.v_token + head * A.v_head + 8 * c, y);
        Group g;
        uint32_t w = quantise(x, A.c.group / 8, g);
        *(uint32_t *)(p.block + p.t * (DIM / 2) + 4 * ((c & 3) * (DIM / 32) + (c >> 2))) = key_word(w);
        const bool first = (8 * c & (A.c.group - 1)) == 0;
        if (first)
            *(uint16_t *)(p.block + scales + 2 * (p.t * groups + (8 * c >> group_log))) = g.number ? __float_as_uint(g.scale) >> 16 : 0x7FC0;
        w = quantise(y, A.c.group / 8, g);
        if (first)
            *(uint16_t *)(p.block + scales + 2 * ((A.c.page + p.t) * groups + (8 * c >> group_log))) = g.number ? __float_as_uint(g.scale) >> 16 : 0x7FC0;
        uint32_t units = 0;
#pragma unroll
        for (int from = 0; from < 4; ++from) {
            const uint32_t two = from_lane(w, from) >> (8 * n);
            units |= ((two & 15u) | (two & 0xF0u) << 12) << (4 * from);
        }
        uint16_t *u = (uint16_t *)(p.block + A.c.page * (DIM / 2) + (p.t >> 2) * (2 * DIM)) + (p.t & 3) + 4 * (c >> 3);
        u[(8 * (c & 1) + 2 * n) * (DIM / 16)] = (uint16_t)units;
        u[(8 * (c & 1) + 2 * n + 1) * (DIM / 16)] = (uint16_t)(units >> 16);
    }
}

template <typename T>
__device__ __forceinline__ void store8(void *p, long long at, const float *f)
{
    typename Eight<T>::type v;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = (T)f[e];
    // past the L2: 16384 tokens of 8 heads, dim 128, bf16, from HBM 14.3 us, 21.2 through it
    __builtin_nontemporal_store(v, (typename Eight<T>::type *)((T *)p + at));
}

// what a code stands for, exactly
__device__ __forceinline__ float value_of(uint32_t code, float scale) { return (__uint_as_float(code | 0x4B000000u) - (0x1p23f + 8.f)) * scale; }

template <typename T, int DIM>
__global__ void __launch_bounds__(256) qcache_read_kernel(QcacheArgs A)
{
    constexpr int LANES = DIM / 8, EACH = 256 / LANES;
    const int c = threadIdx.x % LANES, n = c >> 1 & 3, head = blockIdx.x, group_log = __builtin_ctz(A.c.group), groups = DIM >> group_log;
    const int scales = A.c.page * DIM;
    for (long long at = blockIdx.y * EACH + threadIdx.x / LANES; at < A.tokens; at += gridDim.y * EACH) {
        const int token = (int)at;
        const Place p = place_of(A, token, head);
        if (!p.block)
            continue;
        const uint32_t w = *(const uint32_t *)(p.block + p.t * (DIM / 2) + 4 * ((c & 3) * (DIM / 32) + (c >> 2)));
        const uint16_t *u = (const uint16_t *)(p.block + A.c.page * (DIM / 2) + (p.t >> 2) * (2 * DIM)) + (p.t & 3) + 4 * (c >> 3);
        const uint32_t units = u[(8 * (c & 1) + 2 * n) * (DIM / 16)] | (uint32_t)u[(8 * (c & 1) + 2 * n + 1) * (DIM / 16)] << 16;
        const uint16_t ks = *(const uint16_t *)(p.block + scales + 2 * (p.t * groups + (8 * c >> group_log)));
        const uint16_t vs = *(const uint16_t *)(p.block + scales + 2 * ((A.c.page + p.t) * groups + (8 * c >> group_log)));
        float f[8], s = __uint_as_float((uint32_t)ks << 16);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            f[e] = value_of(w >> (4 * (e / 2 + e % 2 * 4)) & 15u, s);
        store8<T>(A.k, token * A.k_token + head * A.k_head + 8 * c, f);
        s = __uint_as_float((uint32_t)vs << 16);
#pragma unroll
        for (int from = 0; from < 4; ++from) {
            const uint32_t two = from_lane(units, from) >> (4 * n);
            f[2 * from] = value_of(two & 15u, s);
            f[2 * from + 1] = value_of(two >> 16 & 15u, s);
        }
        store8<T>(A.v, token * A.v_token + head * A.v_head + 8 * c, f);
    }
}

constexpr int MOST_GROUPS = 1 << 18;   // tokens past this many workgroups of a head are looped over

template <typename T, int DIM, bool WRITE>
void launch(const QcacheArgs &a, hipStream_t stream)
{
    const int each = 256 / (DIM / 8), most = MOST_GROUPS / a.c.heads + 1, groups = (a.tokens - 1) / each + 1;
    const dim3 grid((unsigned)a.c.heads, (unsigned)std::min({groups, most, 65535}));
    if (WRITE)
        hipLaunchKernelGGL((qcache_write_kernel<T, DIM>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((qcache_read_kernel<T, DIM>), grid, dim3(256), 0, stream, a);
}

template <typename T, bool WRITE>
void launch_dim(const QcacheArgs &a, hipStream_t stream)
{
    if (a.c.dim == 64)
        launch<T, 64, WRITE>(a, stream);
    else if (a.c.dim == 128)
        launch<T, 128, WRITE>(a, stream);
    else
        launch<T, 256, WRITE>(a, stream);
}

template <bool WRITE>
hipError_t launch_typed(const QcacheArgs &a, hipStream_t stream)
{
    if (a.type == AQD_F32)
        launch_dim<float, WRITE>(a, stream);
    else if (a.type == AQD_F16)
        launch_dim<_Float16, WRITE>(a, stream);
    else
        launch_dim<__bf16, WRITE>(a, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_qcache_write(const QcacheArgs &a, hipStream_t stream) { return launch_typed<true>(a, stream); }
hipError_t launch_qcache_read(const QcacheArgs &a, hipStream_t stream) { return launch_typed<false>(a, stream); }

}  // namespace aqd
