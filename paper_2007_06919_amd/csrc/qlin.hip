// Linear layers on signed 8-bit codes: y = (x w^T) * x_scales * w_scales + bias,
// plain or as the two halves of a gated unit. Definitions: include/aqd.h.
//
// Both operands hold their sum's index contiguously, which is what the int8 MFMA
// wants of both: a lane's 16 bytes are 16 consecutive k of one row. The weights are
// the MFMA's rows and the tokens its columns, so a lane's accumulators are
// consecutive channels of one token and leave as one wide store. Sums are int32
// and exact; so are the partial sums of a split K range, in any order.

#include "internal.h"
#include "mfma_common.h"

namespace aqd {
namespace {

// ---- epilogue -----------------------------------------------------------------
template <typename T>
struct Four {
    typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};

// z for four consecutive rows of w from row j on (only the first `left` exist)
__device__ __forceinline__ void scaled4(const QlinArgs &A, const v4i acc, int j, int left, float sx, float *z)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        z[e] = (float)acc[e] * sx;
        if (e < left) {
            z[e] *= A.w_scales[j + e];
            if (A.bias)
                z[e] += A.bias[j + e];
        }
    }
}

// z / (1 + exp(-z)): the exponential and the reciprocal are the hardware's (one unit in
// the last place each); exp(-z) = infinity gives -0
__device__ __forceinline__ float silu(float z) { return z * __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

// four consecutive outputs of a token from column j on; value: the gated unit's second half
template <typename T, bool GATE>
__device__ __forceinline__ void emit4(const QlinArgs &A, long long t, int j, const v4i acc, const v4i value, float sx)
{
    const int left = A.n - j;
    if (left <= 0)
        return;
    float z[4];
    scaled4(A, acc, j, left, sx, z);
    if constexpr (GATE) {
        float v[4];
        scaled4(A, value, A.n + j, left, sx, v);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            z[e] = silu(z[e]) * v[e];
    }
    T *y = (T *)A.y + t * A.ld_y + j;
    typename Four<T>::type o;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        o[e] = (T)z[e];
    if (left >= 4) {
        *(typename Four<T>::type *)y = o;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left)
                y[e] = o[e];
    }
}

// ---- partial sums of a split K range ----------------------------------------------
// four consecutive sums of a token from column j (a multiple of 4) on; half: 1 for the
// gated unit's second half
template <bool GATE>
__device__ __forceinline__ void put4(const QlinArgs &A, int part, long long t, int j, int half, const v4i acc)
{
    if (j < A.n_pad)
        *(v4i *)(A.part + (((long long)part * A.rows + t) * (GATE ? 2 : 1) + half) * A.n_pad + j) = acc;
}

template <typename T, bool GATE>
__global__ void __launch_bounds__(256) qlin_combine_kernel(QlinArgs A)
{
    const int quads = (A.n + 3) / 4;
    const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (long long)A.rows * quads)
        return;
    const long long t = idx / quads;
    const int j = 4 * (int)(idx - t * quads);
    const long long line = (long long)A.n_pad * (GATE ? 2 : 1), step = A.rows * line;
    const int32_t *p = A.part + t * line + j;
    v4i acc = {0, 0, 0, 0}, value = {0, 0, 0, 0};
    for (int s = 0; s < A.ksplit; ++s) {
        acc += *(const v4i *)(p + s * step);
        if constexpr (GATE)
            value += *(const v4i *)(p + s * step + A.n_pad);
    }
    emit4<T, GATE>(A, t, j, acc, value, A.x_scales[t]);
}

// ---- any strides: 64 rows of w x 64 tokens, both through registers into LDS ----------
// 16 bytes of a row at c, zeros from k on. Rows start at any byte; the hardware takes an
// unaligned 16-byte load. Nothing at or past the row's k-th byte is read.
__device__ __forceinline__ v4i load16(const int8_t *row, int c, int k)
{
    typedef int v4u __attribute__((ext_vector_type(4), aligned(1)));
    if (c + 16 <= k)
        return *(const v4u *)(row + c);
    v4i v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (c + e < k)
            v[e / 4] |= (int)(uint8_t)row[c + e] << (8 * (e % 4));
    return v;
}

constexpr int ANY_TILE = 64;

// Wave i: the 64 rows of w by tokens 16i .. 16i+15. With the gate the tile's first 32 rows
// are gate rows and the others the value rows of the same outputs.
template <typename T, bool GATE, bool PART>
__global__ void __launch_bounds__(256) qlin_any_kernel(QlinArgs A, long long tile0)
{
    __shared__ v4i lds[2][2][ANY_TILE * 4];   // [buffer][w, x][row][16-byte column, swizzled]
    constexpr int OUT = GATE ? ANY_TILE / 2 : ANY_TILE;
    const int tiles_n = (A.n + OUT - 1) / OUT, tiles_t = (A.rows + ANY_TILE - 1) / ANY_TILE;
    long long tile = tile0 + blockIdx.x;
    const int tn = (int)(tile % tiles_n);
    tile /= tiles_n;
    const int tt = (int)(tile % tiles_t), part = (int)(tile / tiles_t);
    const int k0 = part * A.kchunk, k1 = A.k - k0 < A.kchunk ? A.k : k0 + A.kchunk;

    const int r = threadIdx.x >> 2, c = threadIdx.x & 3;
    const int j = tn * OUT + (GATE ? r % OUT : r);
    const int row_w = (j < A.n ? j : A.n - 1) + (GATE && r >= OUT ? A.n : 0);
    const long long row_x = (long long)tt * ANY_TILE + r;
    const int8_t *pw = A.w + row_w * A.ld_w, *px = A.x + (row_x < A.rows ? row_x : A.rows - 1) * A.ld_x;
    const int slot = r * 4 + (c ^ ((r >> 1) & 3));

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, fc = lane >> 4;
    v4i acc[4] = {};
    v4i w = load16(pw, k0 + 16 * c, k1), x = load16(px, k0 + 16 * c, k1);
    int buf = 0;
    for (int k = k0; k < k1; k += 64, buf ^= 1) {
        lds[buf][0][slot] = w;
        lds[buf][1][slot] = x;
        __syncthreads();
        w = load16(pw, k + 64 + 16 * c, k1);
        x = load16(px, k + 64 + 16 * c, k1);
        const int rb = 16 * wave + fr;
        const v4i b = lds[buf][1][rb * 4 + (fc ^ ((rb >> 1) & 3))];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int ra = 16 * i + fr;
            acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(lds[buf][0][ra * 4 + (fc ^ ((ra >> 1) & 3))], b, acc[i], 0, 0, 0);
        }
    }
    const long long t = (long long)tt * ANY_TILE + 16 * wave + fr;
    if (t >= A.rows)
        return;
    if constexpr (PART) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            put4<GATE>(A, part, t, tn * OUT + (16 * i) % OUT + 4 * fc, 16 * i / OUT, acc[i]);
    } else {
        const float sx = A.x_scales[t];
        if constexpr (GATE) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                emit4<T, true>(A, t, tn * OUT + 16 * i + 4 * fc, acc[i], acc[i + 2], sx);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                emit4<T, false>(A, t, tn * OUT + 16 * i + 4 * fc, acc[i], acc[i], sx);
        }
    }
}

// ---- launches -------------------------------------------------------------------------
constexpr long long MOST_GROUPS = 1 << 23;   // workgroups of one launch

template <typename T, bool GATE>
void launch_combine(const QlinArgs &a, hipStream_t stream)
{
    const long long items = (long long)a.rows * ((a.n + 3) / 4);   // a split's workspace keeps this small
    hipLaunchKernelGGL((qlin_combine_kernel<T, GATE>), dim3((unsigned)((items + 255) / 256)), dim3(256), 0, stream, a);
}

template <typename T, bool GATE>
void launch_any(const QlinArgs &a, hipStream_t stream)
{
    constexpr int OUT = GATE ? ANY_TILE / 2 : ANY_TILE;
    const long long total = (long long)((a.n + OUT - 1) / OUT) * ((a.rows + ANY_TILE - 1) / ANY_TILE) * a.ksplit;
    for (long long at = 0; at < total; at += MOST_GROUPS) {
        const dim3 grid((unsigned)(total - at < MOST_GROUPS ? total - at : MOST_GROUPS));
        if (a.ksplit > 1)
            hipLaunchKernelGGL((qlin_any_kernel<T, GATE, true>), grid, dim3(256), 0, stream, a, at);
        else
            hipLaunchKernelGGL((qlin_any_kernel<T, GATE, false>), grid, dim3(256), 0, stream, a, at);
    }
    if (a.ksplit > 1)
        launch_combine<T, GATE>(a, stream);
}

template <typename T>
void launch_gate(const QlinArgs &a, hipStream_t stream)
{
    if (a.gate)
        launch_any<T, true>(a, stream);
    else
        launch_any<T, false>(a, stream);
}

}  // namespace

int qlin_parts(const QlinArgs &a, size_t *bytes)
{
    const int out = a.gate ? ANY_TILE / 2 : ANY_TILE;
    const long long tiles = (long long)((a.n + out - 1) / out) * ((a.rows + ANY_TILE - 1) / ANY_TILE);
    const int steps = (a.k + 63) / 64;
    const size_t one = (size_t)a.rows * (size_t)((a.n + 3) & ~3) * (a.gate ? 2 : 1) * sizeof(int32_t);
    long long parts = 512 / tiles;
    if (parts > steps / 8)
        parts = steps / 8;
    while (parts > 1 && one * parts > AQD_QLIN_WORKSPACE_BYTES)
        --parts;
    *bytes = parts > 1 ? one * parts : 0;
    return parts > 1 ? (int)parts : 1;
}

hipError_t launch_qlin(const QlinArgs &args, hipStream_t stream)
{
    QlinArgs a = args;
    a.n_pad = (a.n + 3) & ~3;
    const int steps = (a.k + 63) / 64;
    a.kchunk = 64 * ((steps + a.ksplit - 1) / a.ksplit);
    a.ksplit = (a.k + a.kchunk - 1) / a.kchunk;
    if (a.ksplit <= 1)
        a.kchunk = a.k;
    if (a.type == AQD_F32)
        launch_gate<float>(a, stream);
    else if (a.type == AQD_F16)
        launch_gate<_Float16>(a, stream);
    else
        launch_gate<__bf16>(a, stream);
    return hipGetLastError();
}

}  // namespace aqd
