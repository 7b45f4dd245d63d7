// Root-mean-square norm of query and key heads and their rotation by position, in one
// pass. Definition: include/aqd.h.
//
// A head lies in the registers of 1 to 64 lanes (a power of two, no more than its pairs
// take), each of which holds both channels of its pairs, so that the sum of squares is
// the only thing that crosses lanes. fp32 throughout, one rounding at the store.
//
// Bound by HBM: a head is read and written once, the table's row and the weights come
// from the caches. 16384 tokens of 40 heads, dim 128, bf16: 336 MB in 69 us, 4.9 TB/s (a copy of that
// size 5.4). One token: 6 us, the launch.

#include "internal.h"

namespace aqd {
namespace {

template <typename T, int N>
struct Some {
    // at an address aligned to its elements only
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

template <typename T, int N>
__device__ __forceinline__ void load(const T *p, float *f)
{
    const auto v = *(const typename Some<T, N>::type *)p;
#pragma unroll
    for (int e = 0; e < N; ++e)
        f[e] = (float)v[e];
}

template <typename T, int N>
__device__ __forceinline__ void store(T *p, const float *f)
{
    typename Some<T, N>::type v;
#pragma unroll
    for (int e = 0; e < N; ++e)
        v[e] = (T)f[e];
    // past the L2: 16384 tokens of 40 heads, dim 128, bf16 69.4 us, 73.6 through it
    __builtin_nontemporal_store(v, (typename Some<T, N>::type *)p);
}

// N pairs are a unit, 1 << LOG lanes hold a head and each has up to V units of it. Rotated
// pairs come first; N divides their number and that of the others.
template <typename T, int N, int V, bool HALVES>
__global__ void __launch_bounds__(256) heads_kernel(HeadsArgs A, int log)
{
    const int lanes = 1 << log, lane = threadIdx.x & (lanes - 1), units = A.dim / (2 * N), half = A.rot / 2, rest = (A.dim - A.rot) / 2;
    const int total = A.tokens * A.heads, each = 256 >> log;
    // (the index may pass total by a grid's heads)
    for (long long at = (long long)blockIdx.x * each + (threadIdx.x >> log); at < total; at += (long long)gridDim.x * each) {
        const int token = (int)at / A.heads, head = (int)at - token * A.heads;
        const HeadsSide &s = head < A.q_heads ? A.q : A.k;
        const int h = head < A.q_heads ? head : head - A.q_heads;
        const T *x = (const T *)s.x + token * s.token + h * s.head;
        T *y = (T *)s.y + token * s.y_token + h * s.y_head;
        const T *w = (const T *)s.weight;
        const float *row = nullptr;
        bool known = true;
        if (A.rot) {
            const int p = A.position[token];
            known = p >= 0 && p < A.positions;
            row = A.table + (long long)(known ? p : 0) * A.rot;
        }
        float a[V][N], b[V][N];
        int ca[V], cb[V];
        float ss = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int first = (lane + lanes * v) * N;
            // channels of the unit's first and second elements; those of neighbours alternate from ca on
            if (!HALVES) {
                ca[v] = 2 * first;
                cb[v] = 2 * first + N;
            } else if (first < half) {
                ca[v] = first;
                cb[v] = first + half;
            } else {
                ca[v] = first + half;
                cb[v] = first + half + rest;
            }
            if (lane + lanes * v >= units)
                continue;
            load<T, N>(x + ca[v], a[v]);
            load<T, N>(x + cb[v], b[v]);
#pragma unroll
            for (int e = 0; e < N; ++e)
                ss += a[v][e] * a[v][e] + b[v][e] * b[v][e];
        }
        if (w) {
            for (int d = lanes >> 1; d; d >>= 1)
                ss += __shfl_xor(ss, d);
            const float r = 1.f / sqrtf(ss / (float)A.dim + A.eps);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (lane + lanes * v >= units)
                    continue;
                float wa[N], wb[N];
                load<T, N>(w + ca[v], wa);
                load<T, N>(w + cb[v], wb);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    a[v][e] *= r * wa[e];
                    b[v][e] *= r * wb[e];
                }
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (lane + lanes * v >= units)
                continue;
            const int first = (lane + lanes * v) * N;
            if (first < half) {
                float c[N], n[N];
                if (known) {
                    load<float, N>(row + first, c);
                    load<float, N>(row + half + first, n);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        c[e] = n[e] = NAN;
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    // neighbours: pair e is elements 2 e and 2 e + 1 of the unit's 2 N
                    float &p = HALVES ? a[v][e] : 2 * e < N ? a[v][2 * e % N] : b[v][2 * e % N];
                    float &q = HALVES ? b[v][e] : 2 * e + 1 < N ? a[v][(2 * e + 1) % N] : b[v][(2 * e + 1) % N];
                    const float turned = __builtin_fmaf(p, c[e], -(q * n[e]));
                    q = __builtin_fmaf(q, c[e], p * n[e]);
                    p = turned;
                }
            }
            store<T, N>(y + ca[v], a[v]);
            store<T, N>(y + cb[v], b[v]);
        }
    }
}

constexpr int MOST_GROUPS = 1 << 20;   // heads past this many workgroups are looped over

template <typename T, int N, int V>
void launch_units(const HeadsArgs &a, hipStream_t stream)
{
    const int units = a.dim / (2 * N);
    int log = 0;
    while (log < 6 && (1 << log) < units)
        ++log;
    const int each = 256 >> log;
    const long long groups = ((long long)a.tokens * a.heads + each - 1) / each;
    const dim3 grid((unsigned)(groups < MOST_GROUPS ? groups : MOST_GROUPS));
    if (a.pairs == AQD_PAIRS_HALVES)
        hipLaunchKernelGGL((heads_kernel<T, N, V, true>), grid, dim3(256), 0, stream, a, log);
    else
        hipLaunchKernelGGL((heads_kernel<T, N, V, false>), grid, dim3(256), 0, stream, a, log);
}

template <typename T, int N>
void launch_width(const HeadsArgs &a, hipStream_t stream)
{
    constexpr int MOST = N < 8 ? 8 / N : 1;   // units of a lane of 64, of heads of 1024
    if (a.dim <= 128 * N)
        launch_units<T, N, 1>(a, stream);
    else
        launch_units<T, N, MOST>(a, stream);
}

// As many pairs at once as 16 bytes hold, or fewer where their number does not divide the rotated pairs and the others: 16384 tokens of
// 40 heads, dim 128, bf16, in eights (128 channels rotated) 70 us, in fours (120) 90, in twos (124) 160, one by one (126) 264.
template <typename T>
void launch_type(const HeadsArgs &a, hipStream_t stream)
{
    const int both = (a.rot / 2) | ((a.dim - a.rot) / 2);   // its lowest bit set is that of the two
    if (sizeof(T) == 2 && both % 8 == 0)
        launch_width<T, 16 / (int)sizeof(T)>(a, stream);
    else if (both % 4 == 0)
        launch_width<T, 4>(a, stream);
    else if (both % 2 == 0)
        launch_width<T, 2>(a, stream);
    else
        launch_width<T, 1>(a, stream);
}

}  // namespace

hipError_t launch_heads(const HeadsArgs &a, hipStream_t stream)
{
    if (a.type == AQD_F32)
        launch_type<float>(a, stream);
    else if (a.type == AQD_F16)
        launch_type<_Float16>(a, stream);
    else
        launch_type<__bf16>(a, stream);
    return hipGetLastError();
}

}  // namespace aqd
