// Keys and values into and out of a cache of 4-bit codes with a bf16 scale per group of
// channels. Definition and layout: include/aqd.h.
//
// A lane holds 8 channels of a token's head. The largest magnitude of a group, with
// its sign, is one unsigned integer (the magnitude's bits above a bit that is set
// for positive numbers), so one maximum over a group's lanes finds both and prefers the positive
// number, and infinities and NaN are above all others. The values' nibbles of one unit
// come from four lanes, which exchange their words.

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
};

// the scale of a group from its maximum
__device__ __forceinline__ Group group_of(uint32_t top)
{
    const uint32_t size = top >> 1;
    const float a = __uint_as_float(size | (top & 1 ? 0u : 0x80000000u));
    Group g;
    g.scale = (float)(__bf16)(a * -0.125f);
    if (!(fabsf(g.scale) >= 0x1p-119f))
        g.scale = 0.f;
    g.inverse = g.scale != 0.f ? 1.f / g.scale : 0.f;
    if (size >= 0x7F800000u) {
        g.scale = NAN;
        g.inverse = 0.f;
    }
    return g;
}

// codes of 8 channels, channel i in nibble i; lanes: those of a group
__device__ __forceinline__ uint32_t quantise(const float *x, int lanes, Group &g)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = __float_as_uint(x[e]), key = (b << 1) | (~b >> 31);
        top = key > top ? key : top;
    }
    for (int d = 1; d < lanes; d <<= 1) {
        const uint32_t other = (uint32_t)__shfl_xor((int)top, d);
        top = other > top ? other : top;
    }
    g = group_of(top);
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        // a product with infinity or NaN is not a number: code 8 there
        const float c = g.inverse == 0.f ? 0.f : fminf(fmaxf(rintf(x[e] * g.inverse), -8.f), 7.f);
        w |= (uint32_t)((int)c + 8) << (4 * e);
    }
    return w;
}

// nibbles 0 .. 7 to the places of key channels: 2 j to j, 2 j + 1 to j + 4
__device__ __forceinline__ uint32_t key_word(uint32_t w)
{
    uint32_t even = w & 0x0F0F0F0Fu, odd = (w >> 4) & 0x0F0F0F0Fu;
    even = (even | (even >> 4)) & 0x00FF00FFu;
    odd = (odd | (odd >> 4)) & 0x00FF00FFu;
    return ((even | (even >> 8)) & 0xFFFFu) | (odd | (odd >> 8)) << 16;
}

struct Place {
    uint8_t *block;
    int t;
};

__device__ __forceinline__ Place place_of(const QcacheArgs &A, int slot, int head)
{
    const int number = slot / A.c.page;
    return {A.cache + ((long long)number * A.c.heads + head) * A.c.block_bytes, slot - number * A.c.page};
}

template <typename T>
__global__ void __launch_bounds__(256) qcache_write_kernel(QcacheArgs A, int log)
{
    const int lanes = 1 << log, c = threadIdx.x & (lanes - 1), each = 256 >> log, dim = A.c.dim, groups = dim / A.c.group;
    const int total = A.tokens * A.c.heads, slots = A.c.pages * A.c.page;
    for (long long at = (long long)blockIdx.x * each + (threadIdx.x >> log); at < total; at += (long long)gridDim.x * each) {
        const int token = (int)at / A.c.heads, head = (int)at - token * A.c.heads;
        const int slot = A.slots[token];
        if (slot < 0 || slot >= slots)
            continue;   // all lanes of a head together
        const Place p = place_of(A, slot, head);
        float x[8];
        Group g;
        const int scales = A.c.page * dim;
        load8<T>(A.k, token * A.k_token + head * A.k_head + 8 * c, x);
        uint32_t w = quantise(x, A.c.group / 8, g);
        *(uint32_t *)(p.block + p.t * (dim / 2) + 4 * ((c & 3) * (dim / 32) + (c >> 2))) = key_word(w);
        if (8 * c % A.c.group == 0)
            *(__bf16 *)(p.block + scales + 2 * (p.t * groups + 8 * c / A.c.group)) = (__bf16)g.scale;
        load8<T>(A.v, token * A.v_token + head * A.v_head + 8 * c, x);
        w = quantise(x, A.c.group / 8, g);
        if (8 * c % A.c.group == 0)
            *(__bf16 *)(p.block + scales + 2 * ((A.c.page + p.t) * groups + 8 * c / A.c.group)) = (__bf16)g.scale;
        // c = 8 h + 2 n + s has channels 64 h + 16 n + 8 s .. + 7, and writes units m = 8 s + 2 n and the next
        const int h = c >> 3, n = (c >> 1) & 3, s = c & 1;
        uint32_t units = 0;
#pragma unroll
        for (int from = 0; from < 4; ++from) {
            const uint32_t two = (uint32_t)__shfl((int)w, (threadIdx.x & 63 & ~6) | from << 1) >> (8 * n);
            units |= ((two & 15u) | (two & 0xF0u) << 12) << (4 * from);
        }
        uint16_t *u = (uint16_t *)(p.block + p.t / 4 * (2 * dim) + A.c.page * (dim / 2)) + (p.t & 3) + 4 * h;
        u[(8 * s + 2 * n) * (dim / 16)] = (uint16_t)units;
        u[(8 * s + 2 * n + 1) * (dim / 16)] = (uint16_t)(units >> 16);
    }
}

template <typename T>
__device__ __forceinline__ void store8(void *p, long long at, const float *f)
{
    typename Eight<T>::type v;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = (T)f[e];
    *(typename Eight<T>::type *)((T *)p + at) = v;
}

template <typename T>
__global__ void __launch_bounds__(256) qcache_read_kernel(QcacheArgs A, int log)
{
    const int lanes = 1 << log, c = threadIdx.x & (lanes - 1), each = 256 >> log, dim = A.c.dim, groups = dim / A.c.group;
    const int total = A.tokens * A.c.heads, slots = A.c.pages * A.c.page;
    for (long long at = (long long)blockIdx.x * each + (threadIdx.x >> log); at < total; at += (long long)gridDim.x * each) {
        const int token = (int)at / A.c.heads, head = (int)at - token * A.c.heads;
        const int slot = A.slots[token];
        if (slot < 0 || slot >= slots)
            continue;
        const Place p = place_of(A, slot, head);
        const int scales = A.c.page * dim;
        const uint32_t w = *(const uint32_t *)(p.block + p.t * (dim / 2) + 4 * ((c & 3) * (dim / 32) + (c >> 2)));
        float f[8], s = (float)*(const __bf16 *)(p.block + scales + 2 * (p.t * groups + 8 * c / A.c.group));
#pragma unroll
        for (int e = 0; e < 8; ++e)
            f[e] = (float)((int)(w >> (4 * (e / 2 + e % 2 * 4)) & 15u) - 8) * s;
        store8<T>(A.k, token * A.k_token + head * A.k_head + 8 * c, f);
        s = (float)*(const __bf16 *)(p.block + scales + 2 * ((A.c.page + p.t) * groups + 8 * c / A.c.group));
        const uint16_t *u = (const uint16_t *)(p.block + p.t / 4 * (2 * dim) + A.c.page * (dim / 2)) + (p.t & 3) + 4 * (c >> 3);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            f[e] = (float)((u[(8 * (c & 1) + e) * (dim / 16)] >> (4 * ((c >> 1) & 3)) & 15) - 8) * s;
        store8<T>(A.v, token * A.v_token + head * A.v_head + 8 * c, f);
    }
}

constexpr int MOST_GROUPS = 1 << 20;   // heads past this many workgroups are looped over

template <typename T, bool WRITE>
void launch(const QcacheArgs &a, hipStream_t stream)
{
    const int log = a.c.dim == 64 ? 3 : a.c.dim == 128 ? 4 : 5, each = 256 >> log;
    const long long groups = ((long long)a.tokens * a.c.heads + each - 1) / each;
    const dim3 grid((unsigned)(groups < MOST_GROUPS ? groups : MOST_GROUPS));
    if (WRITE)
        hipLaunchKernelGGL(qcache_write_kernel<T>, grid, dim3(256), 0, stream, a, log);
    else
        hipLaunchKernelGGL(qcache_read_kernel<T>, grid, dim3(256), 0, stream, a, log);
}

template <bool WRITE>
hipError_t launch_typed(const QcacheArgs &a, hipStream_t stream)
{
    if (a.type == AQD_F32)
        launch<float, WRITE>(a, stream);
    else if (a.type == AQD_F16)
        launch<_Float16, WRITE>(a, stream);
    else
        launch<__bf16, WRITE>(a, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_qcache_write(const QcacheArgs &a, hipStream_t stream) { return launch_typed<true>(a, stream); }
hipError_t launch_qcache_read(const QcacheArgs &a, hipStream_t stream) { return launch_typed<false>(a, stream); }

}  // namespace aqd
