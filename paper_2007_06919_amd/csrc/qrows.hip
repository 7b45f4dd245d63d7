// Rows of real numbers to signed 8-bit codes with one scale per row, by
// themselves (qrows) or behind a residual's addition and a root-mean-square
// norm (qnorm). Definitions: include/aqd.h.
//
// With u = s * w the normalised row is u / rms, and its codes are
// rint(u / rms * 127 / max|u / rms|): the row's factor 1 / rms cancels. So the
// maximum of |u| and the sum of s^2 are reduced together, in one pass over
// registers with one barrier, and only the scale carries 1 / rms. Each code is
// one product with 127 / max and one rounding to the nearest even integer, the
// same bits in any order of evaluation. Squares are summed in fp32.
//
// Bound by HBM: a row is read once and stays in registers between the
// reductions and the codes (norm with residual of 16384 x 4096 bf16 83 us, 5.6
// TB/s; 8192 x 11000 f16 49 us, 5.5; a large copy here 5.45). A few rows take
// 3 to 4 us, launch and latency of the loads and reductions.

#include "internal.h"

namespace aqd {
namespace {

// 16 bytes of a row at an address aligned to its elements only (rows of any
// stride); the hardware takes them in one instruction
template <typename T>
struct Vec {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    typedef signed char codes __attribute__((ext_vector_type(N), aligned(1)));
};

// the vector at column c, zeros past the row's end
template <typename T>
__device__ __forceinline__ typename Vec<T>::type load_vec(const T *p, int c, int cols)
{
    constexpr int N = Vec<T>::N;
    if (c + N <= cols)
        return *(const typename Vec<T>::type *)(p + c);
    typename Vec<T>::type t;
#pragma unroll
    for (int e = 0; e < N; ++e)
        t[e] = c + e < cols ? p[c + e] : (T)0.f;
    return t;
}

// the sum of squares and the bits of the largest |u| (as unsigned integers the
// bits of magnitudes are ordered as the magnitudes are, with infinity and then
// NaN above all of them, so a row that holds either keeps it)
struct Stat {
    float ss;
    uint32_t top;
};

__device__ __forceinline__ void merge(Stat &a, float ss, uint32_t top)
{
    a.ss += ss;
    a.top = top > a.top ? top : a.top;
}

__device__ __forceinline__ void wave_merge(Stat &a)
{
#pragma unroll
    for (int d = 32; d; d >>= 1)
        merge(a, __shfl_xor(a.ss, d), (uint32_t)__shfl_xor((int)a.top, d));
}

// over the WAVES waves of a row; lds: 2 x WAVES entries, used in turn by parity
// so that the next row's writes cannot overtake this row's reads
template <int WAVES>
__device__ __forceinline__ void row_merge(Stat &a, Stat (*lds)[WAVES], int parity)
{
    wave_merge(a);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0)
            lds[parity][threadIdx.x >> 6] = a;
        __syncthreads();
        a = lds[parity][0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i)
            merge(a, lds[parity][i].ss, lds[parity][i].top);
    }
}

struct Quant {
    float inv, scale;
    bool ok;
};

template <bool NORM>
__device__ __forceinline__ Quant quant_of(const Stat &a, int cols, float eps)
{
    Quant q;
    const float top = __uint_as_float(a.top), m = fmaxf(top, 0x1p-119f);   // 127 / m stays finite
    q.ok = top < INFINITY && (!NORM || a.ss < INFINITY);                   // false for NaN
    q.inv = 127.f / m;
    q.scale = NORM ? m / sqrtf(a.ss / (float)cols + eps) / 127.f : m / 127.f;
    if (!q.ok)
        q.scale = NAN;
    return q;
}

template <typename T>
__device__ __forceinline__ void store_codes(int8_t *p, int c, int cols, const float *u, const Quant &q)
{
    constexpr int N = Vec<T>::N;
    typename Vec<T>::codes v;
#pragma unroll
    for (int e = 0; e < N; ++e)
        v[e] = q.ok ? (signed char)(int)rintf(u[e] * q.inv) : 0;
    if (c + N <= cols) {
        *(typename Vec<T>::codes *)(p + c) = v;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (c + e < cols)
                p[c + e] = v[e];
    }
}

template <typename T>
__device__ __forceinline__ void store_row(T *p, int c, int cols, const float *f)
{
    constexpr int N = Vec<T>::N;
    typename Vec<T>::type v;
#pragma unroll
    for (int e = 0; e < N; ++e)
        v[e] = (T)f[e];
    if (c + N <= cols) {
        *(typename Vec<T>::type *)(p + c) = v;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (c + e < cols)
                p[c + e] = v[e];
    }
}

// One row per WAVES waves and ROWS rows per workgroup, V vectors of 16 bytes per
// lane kept in registers. sum may be x or residual: a lane reads what it writes
// before it writes it.
template <typename T, bool NORM, int WAVES, int ROWS, int V>
__global__ void __launch_bounds__(64 * WAVES * ROWS) qrows_kernel(RowsArgs A)
{
    static_assert(WAVES == 1 || ROWS == 1, "several rows per workgroup have one wave each");
    constexpr int N = Vec<T>::N, LANES = 64 * WAVES;
    __shared__ Stat lds[2][WAVES];
    const int lane = threadIdx.x & (LANES - 1);
    int parity = 0;
    for (long long row = (long long)blockIdx.x * ROWS + threadIdx.x / LANES; row < A.rows;
         row += (long long)gridDim.x * ROWS, parity ^= 1) {
        const T *x = (const T *)A.x + row * A.ld_x;
        typename Vec<T>::type raw[V], more[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            raw[v] = load_vec(x, (v * LANES + lane) * N, A.cols);
        if constexpr (NORM) {
            if (A.residual) {
                const T *r = (const T *)A.residual + row * A.ld_residual;
#pragma unroll
                for (int v = 0; v < V; ++v)
                    more[v] = load_vec(r, (v * LANES + lane) * N, A.cols);
            }
        }
        float u[V][N];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < N; ++e)
                u[v][e] = (float)raw[v][e];
        Stat st = {0.f, 0};
        if constexpr (NORM) {
            if (A.residual) {
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        u[v][e] += (float)more[v][e];
            }
            if (A.sum)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    store_row<T>((T *)A.sum + row * A.ld_sum, (v * LANES + lane) * N, A.cols, u[v]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const auto w = load_vec((const T *)A.weight, (v * LANES + lane) * N, A.cols);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    st.ss += u[v][e] * u[v][e];
                    u[v][e] *= (float)w[e];
                }
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t b = __float_as_uint(u[v][e]) & 0x7FFFFFFFu;
                st.top = b > st.top ? b : st.top;
            }
        row_merge<WAVES>(st, lds, parity);
        const Quant q = quant_of<NORM>(st, A.cols, A.eps);
#pragma unroll
        for (int v = 0; v < V; ++v)
            store_codes<T>(A.codes + row * A.ld_codes, (v * LANES + lane) * N, A.cols, u[v], q);
        if (lane == 0)
            A.scales[row] = q.scale;
    }
}

// Rows too long for the registers of a workgroup: read twice (1024 x 200000
// bf16 183 us, 5.6 TB/s with the second read; 16 rows of them 20 us, one
// workgroup's time for its row).
template <typename T, bool NORM>
__global__ void __launch_bounds__(1024) qrows_long_kernel(RowsArgs A)
{
    constexpr int N = Vec<T>::N, WAVES = 16;
    __shared__ Stat lds[2][WAVES];
    int parity = 0;
    for (long long row = blockIdx.x; row < A.rows; row += gridDim.x, parity ^= 1) {
        const T *x = (const T *)A.x + row * A.ld_x;
        const T *r = NORM && A.residual ? (const T *)A.residual + row * A.ld_residual : nullptr;
        auto total = [&](int c, float *u) {
            const auto a = load_vec(x, c, A.cols);
#pragma unroll
            for (int e = 0; e < N; ++e)
                u[e] = (float)a[e];
            if (r) {
                const auto b = load_vec(r, c, A.cols);
#pragma unroll
                for (int e = 0; e < N; ++e)
                    u[e] += (float)b[e];
            }
        };
        auto scaled = [&](int c, float *u) {
            if constexpr (NORM) {
                const auto w = load_vec((const T *)A.weight, c, A.cols);
#pragma unroll
                for (int e = 0; e < N; ++e)
                    u[e] *= (float)w[e];
            }
        };
        Stat st = {0.f, 0};
        for (int c = threadIdx.x * N; c < A.cols; c += 1024 * N) {
            float u[N];
            total(c, u);
#pragma unroll
            for (int e = 0; e < N; ++e)
                st.ss += u[e] * u[e];
            scaled(c, u);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t b = __float_as_uint(u[e]) & 0x7FFFFFFFu;
                st.top = b > st.top ? b : st.top;
            }
        }
        row_merge<WAVES>(st, lds, parity);
        const Quant q = quant_of<NORM>(st, A.cols, A.eps);
        for (int c = threadIdx.x * N; c < A.cols; c += 1024 * N) {
            float u[N];
            total(c, u);
            if (NORM && A.sum)
                store_row<T>((T *)A.sum + row * A.ld_sum, c, A.cols, u);
            scaled(c, u);
            store_codes<T>(A.codes + row * A.ld_codes, c, A.cols, u, q);
        }
        if (threadIdx.x == 0)
            A.scales[row] = q.scale;
    }
}

constexpr long long MOST_GROUPS = 1 << 20;   // rows past this many workgroups are looped over

template <typename T, bool NORM, int WAVES, int ROWS, int V>
void launch_short(const RowsArgs &a, hipStream_t stream)
{
    const long long groups = (a.rows + ROWS - 1) / ROWS;
    const dim3 grid((unsigned)(groups < MOST_GROUPS ? groups : MOST_GROUPS)), block(64 * WAVES * ROWS);
    hipLaunchKernelGGL((qrows_kernel<T, NORM, WAVES, ROWS, V>), grid, block, 0, stream, a);
}

template <typename T, bool NORM>
void launch_type(const RowsArgs &a, hipStream_t stream)
{
    constexpr int N = Vec<T>::N;
    // 32 values a lane and their residuals do not fit in the 128 registers of 16 waves
    constexpr bool KEEP4 = !(NORM && N == 8);
    const int vecs = (a.cols + N - 1) / N;   // 16-byte pieces of a row
    // As few waves as hold a row with few vectors each, and no more than a quarter of their places
    // empty: 8192 rows of 11000 fp16, 16 waves x 2: 60.4 us, 8 x 3: 48.9 (with the norm 170.6 and 131.3);
    // of 8192, 8 x 2: 37.2, 4 x 4: 36.7 (93.9 and 86.6); 32768 of 2048, 4 x 1: 43.6, 2 x 2: 37.6 (86.1, 83.0).
    if (vecs <= 64)
        launch_short<T, NORM, 1, 4, 1>(a, stream);
    else if (vecs <= 128)
        launch_short<T, NORM, 1, 4, 2>(a, stream);
    else if (vecs <= 256)
        launch_short<T, NORM, 2, 1, 2>(a, stream);
    else if (vecs <= 384)
        launch_short<T, NORM, 2, 1, 3>(a, stream);
    else if (vecs <= 512)
        launch_short<T, NORM, 4, 1, 2>(a, stream);
    else if (vecs <= 768)
        launch_short<T, NORM, 4, 1, 3>(a, stream);
    else if (vecs <= 1024)
        launch_short<T, NORM, 4, 1, 4>(a, stream);
    else if (vecs <= 1536)
        launch_short<T, NORM, 8, 1, 3>(a, stream);
    else if (vecs <= 2048)
        launch_short<T, NORM, 16, 1, 2>(a, stream);
    else if (vecs <= 4096 && KEEP4)
        launch_short<T, NORM, 16, 1, KEEP4 ? 4 : 2>(a, stream);
    else {
        const dim3 grid((unsigned)(a.rows < MOST_GROUPS ? a.rows : MOST_GROUPS));
        hipLaunchKernelGGL((qrows_long_kernel<T, NORM>), grid, dim3(1024), 0, stream, a);
    }
}

template <typename T>
void launch_norm(const RowsArgs &a, hipStream_t stream)
{
    if (a.norm)
        launch_type<T, true>(a, stream);
    else
        launch_type<T, false>(a, stream);
}

}  // namespace

hipError_t launch_qrows(const RowsArgs &a, hipStream_t stream)
{
    if (a.type == AQD_F32)
        launch_norm<float>(a, stream);
    else if (a.type == AQD_F16)
        launch_norm<_Float16>(a, stream);
    else
        launch_norm<__bf16>(a, stream);
    return hipGetLastError();
}

}  // namespace aqd
