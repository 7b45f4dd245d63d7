// Kernels of the linear layers on signed 8-bit codes: y = (x w^T) * x_scales * w_scales
// + bias, plain or as the two halves of a gated unit (definitions: include/aqd.h). Included by the
// sources that instantiate them, one for each type of y.
//
// Both operands hold their sum's index contiguously, which is what the int8 MFMA
// wants of both: a lane's 16 bytes are 16 consecutive k of one row. The weights are
// the MFMA's rows and the tokens its columns, so a lane's accumulators are
// consecutive channels of one token. Sums are int32 and exact; so are the partial sums of
// a split k range, in any order: every kernel gives the same bits.
#pragma once

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
        if (e < left)
            z[e] = __builtin_fmaf(z[e], A.w_scales[j + e], A.bias ? A.bias[j + e] : 0.f);
    }
}

// z / (1 + exp(-z)) by the hardware's exponential of base 2 and reciprocal (one unit in the last place each). The
// exponential's argument, z log2(e), is rounded once with its constant: 0.62 |z| 2^-23 of the result. In all within (|z| + 4) 2^-23,
// which the codes' own steps of 1/254 of a row's maximum are far above; below z = -87.3 the reciprocal is under the normal
// numbers, and -0
__device__ __forceinline__ float silu(float z) { return z * __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

// z as the fp32 number that it is. Without this, a gated product and its conversion to fp16 become one instruction in some
// kernels, which rounds once where the others round twice: outputs of a split sum were not those of the whole one.
template <typename T>
__device__ __forceinline__ float in_fp32(float z)
{
    if constexpr (std::is_same<T, _Float16>::value)
        asm("" : "+v"(z));
    return z;
}

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
            z[e] = in_fp32<T>(silu(z[e]) * v[e]);
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

// The parts' sums, scaled and stored: bound by its launch and one round of loads from the L2
// (192 x 4096 in four parts, 12.6 MB, 3.9 us).
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
    // four parts' loads in flight at once; past the last part it is read again and not added
    for (int s = 0; s < A.ksplit; s += 4) {
        v4i v[4], w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int32_t *q = p + (s + u < A.ksplit ? s + u : A.ksplit - 1) * step;
            v[u] = *(const v4i *)q;
            if constexpr (GATE)
                w[u] = *(const v4i *)(q + A.n_pad);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (s + u < A.ksplit) {
                acc += v[u];
                if constexpr (GATE)
                    value += w[u];
            }
    }
    emit4<T, GATE>(A, t, j, acc, value, A.x_scales[t]);
}

// ---- loads ------------------------------------------------------------------------------
// Rows may start at any byte. The hardware takes 16-byte loads at multiples of 4 at full speed, at
// other addresses at about a third (16 x 4096 x 4096 with rows of 4097 bytes: 19.7 us, of 4100:
// 7.1); those are loaded as five whole words and shifted. The fifth holds bytes of the
// 16, or is the fourth again: no load leaves the words that hold the row.
typedef int v4u __attribute__((ext_vector_type(4), aligned(1)));

struct Words {
    v4i v;
    int more;
};
// 16 bytes at a wave-uniform base (kept in scalar registers) and a lane's offset. The base is moved
// down to a word first: an offset of 0 has no room for the shift.
template <bool BYTES>
__device__ __forceinline__ Words load_words(const int8_t *base, uint32_t off)
{
    typedef int v4w __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t low = BYTES ? (uint32_t)(uintptr_t)base & 3 : 0;
    auto p = (const __attribute__((address_space(1))) int8_t *)(base - low);
    asm("" : "+s"(p));
    Words r = {};
    const uint32_t o = (off + low) & ~3u;
    if constexpr (BYTES) {
        r.v = *(const __attribute__((address_space(1))) v4w *)(p + o);
        r.more = *(const __attribute__((address_space(1))) int *)(p + (o + ((off + low) & 3 ? 16u : 12u)));
    } else {
        r.v = *(const __attribute__((address_space(1))) v4w *)(p + off);
    }
    return r;
}
// the 16 bytes of what was loaded; shift: the last two bits of their address
template <bool BYTES>
__device__ __forceinline__ v4i shifted(const Words &r, int shift)
{
    if constexpr (!BYTES)
        return r.v;
    return v4i{(int)__builtin_amdgcn_alignbyte((unsigned)r.v[1], (unsigned)r.v[0], (unsigned)shift),
               (int)__builtin_amdgcn_alignbyte((unsigned)r.v[2], (unsigned)r.v[1], (unsigned)shift),
               (int)__builtin_amdgcn_alignbyte((unsigned)r.v[3], (unsigned)r.v[2], (unsigned)shift),
               (int)__builtin_amdgcn_alignbyte((unsigned)r.more, (unsigned)r.v[3], (unsigned)shift)};
}

// The 16 bytes of a row from c on where the row may end (at k >= 16) inside them or before them: nothing
// past it is read. A sum's terms have no order, so the 16 bytes then are the row's last, and
// the terms that another lane or step has too are zeros in the tokens (TOKEN).
template <bool TOKEN>
__device__ __forceinline__ v4i load16(const int8_t *row, int c, int k)
{
    const int at = c < k - 16 ? c : k - 16, gone = c - at;
    v4i v = *(const v4u *)(row + at);
    if constexpr (TOKEN)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int z = gone - 4 * e;
            v[e] = z >= 4 ? 0 : z > 0 ? (int)((uint32_t)v[e] >> (8 * z) << (8 * z)) : v[e];
        }
    return v;
}
// the same where k may be less than 16: byte by byte, zeros from k on
__device__ __forceinline__ v4i load_bytes(const int8_t *row, int c, int k)
{
    v4i v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 15; ++e)
        if (c + e < k)
            v[e / 4] |= (int)(uint8_t)row[c + e] << (8 * (e % 4));
    return v;
}

// ---- tiles of rows at any address ----------------------------------------------------------
// 64 rows of w x 64 tokens, both through registers into LDS, 128 k a stage, loaded a stage and
// a half before they are used. Wave i: the 64 rows of w by tokens 16i .. 16i+15. With the gate the
// tile's first 32 rows are gate rows and the others the value rows of the same outputs. Takes every
// stride (64-bit addresses) and any k. For small launches whose rows start at odd bytes, where it is bound by the
// chain from load to LDS to MFMA (200 x 2000 x 501 packed 7.3 us, 300 x 3000 x 301 6.8), and for what no other takes.
constexpr int KS = 128;   // k of a stage

// XOR of the 16-byte columns of LDS row r (128 bytes): 16-byte reads of consecutive rows at one column
// hit every bank once whether 8 or 16 lanes are served per cycle
__device__ __forceinline__ int swz(int r) { return (r ^ (r >> 3 & 1)) & 7; }

constexpr int ANY_TILE = 64;

template <typename T, bool GATE, bool PART>
__global__ void __launch_bounds__(256) qlin_any_kernel(QlinArgs A, long long tile0)
{
    __shared__ v4i lds[2][2][ANY_TILE * 8];   // [buffer][w, x][row][16-byte column, swizzled]
    constexpr int OUT = GATE ? ANY_TILE / 2 : ANY_TILE;
    const int tiles_n = (A.n + OUT - 1) / OUT, tiles_t = (A.rows + ANY_TILE - 1) / ANY_TILE;
    long long tile = tile0 + blockIdx.x;
    const int tn = (int)(tile % tiles_n);
    tile /= tiles_n;
    const int tt = (int)(tile % tiles_t), part = (int)(tile / tiles_t);
    const int k0 = part * A.kchunk, k1 = A.k - k0 < A.kchunk ? A.k : k0 + A.kchunk;

    const int r = threadIdx.x >> 2, c = threadIdx.x & 3;   // this thread copies columns c and c + 4 of row r
    const int j = tn * OUT + (GATE ? r % OUT : r);
    const long long row_w = (j < A.n ? j : A.n - 1) + (GATE && r >= OUT ? (long long)A.n : 0);
    const long long row_x = (long long)tt * ANY_TILE + r;
    const int8_t *pw = A.w + row_w * A.ld_w + k0, *px = A.x + (row_x < A.rows ? row_x : A.rows - 1) * A.ld_x + k0;
    const int kn = k1 - k0;

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, fc = lane >> 4;
    v4i acc[4] = {};
    Words w[2] = {}, x[2] = {};
    const int shift_w = (int)((uintptr_t)pw & 3), shift_x = (int)((uintptr_t)px & 3);
    int sw = 0, sx = 0;   // the shifts of what is held
    auto words = [](const int8_t *p, int shift) {
        const int *q = (const int *)(p - shift);
        return Words{v4i{q[0], q[1], q[2], q[3]}, q[shift ? 4 : 3]};
    };
    auto load = [&](int k) {
        if (k + KS <= kn) {
            sw = shift_w;
            sx = shift_x;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                w[h] = words(pw + k + 16 * c + 64 * h, shift_w);
                x[h] = words(px + k + 16 * c + 64 * h, shift_x);
            }
        } else if (k < kn) {
            sw = sx = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = k0 + k + 16 * c + 64 * h;   // (a part may be shorter than 16, all of k rarely)
                w[h].v = k1 < 16 ? load_bytes(pw - k0, at, k1) : load16<false>(pw - k0, at, k1);
                x[h].v = k1 < 16 ? load_bytes(px - k0, at, k1) : load16<true>(px - k0, at, k1);
            }
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            lds[buf][0][r * 8 + ((c + 4 * h) ^ swz(r))] = shifted<true>(w[h], sw);
            lds[buf][1][r * 8 + ((c + 4 * h) ^ swz(r))] = shifted<true>(x[h], sx);
        }
    };
    load(0);
    store(0);
    load(KS);
    __syncthreads();
    int buf = 0;
    for (int k = 0; k < kn; k += KS, buf ^= 1) {
        if (k + KS < kn) {
            store(buf ^ 1);
            load(k + 2 * KS);
        }
        const int rb = 16 * wave + fr;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const v4i b = lds[buf][1][rb * 8 + ((fc + 4 * h) ^ swz(rb))];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ra = 16 * i + fr;
                acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(lds[buf][0][ra * 8 + ((fc + 4 * h) ^ swz(ra))], b, acc[i], 0, 0, 0);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
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

// one of n < 2^16 places for workgroup `id`, evenly and neighbours far apart: fractions of the golden ratio
__device__ __forceinline__ int scattered(unsigned id, int n) { return (int)((id * 0x9E3779B1u >> 16) * (unsigned)n >> 16); }

// ---- small launches: both operands straight into registers ----------------------------
// One workgroup per 16 outputs and 16 NB tokens, its waves splitting k, 64 at a time, and adding
// their sums in LDS: no LDS and no barrier in the loop, and the shortest chain from launch to
// store. Rows start at any byte, their 16 (tokens: 16 NB) within 32 bits of offset.
// Bound by the launch and the first loads' latency (77 x 1003 x 514 at odd bytes 5.2 us), then by the
// weights' stream (1 x 4096 x 4096 5.4 to 6.2 us, 16.8 MB; at most 4.1 TB/s, where the tiles below reach 5.1).
constexpr int FEW_WAVES = 4;

template <typename T, bool GATE, bool BYTES, int NB, int U>
__global__ void __launch_bounds__(64 * FEW_WAVES) qlin_few_kernel(QlinArgs A)
{
    constexpr int H = GATE ? 2 : 1;   // row tiles: with the gate, the gate rows and the value rows
    __shared__ v4i sums[FEW_WAVES][H * NB][64];
    // (uniform, so that every condition on it is a scalar branch: MFMAs ignore the execution mask)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, fr = lane & 15, fc = lane >> 4;
    const int j0 = blockIdx.x * 16;
    const long long t0 = (long long)blockIdx.y * 16 * NB;
    const int8_t *pw[2] = {A.w + j0 * A.ld_w, A.w + ((long long)A.n + j0) * A.ld_w}, *px = A.x + t0 * A.ld_x;
    const int left = A.n - 1 - j0;
    const uint32_t vw = (uint32_t)(fr < left ? fr : left) * (uint32_t)A.ld_w + 16 * fc;
    uint32_t vx[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const long long t = 16 * b + fr, most = A.rows - 1 - t0;
        vx[b] = (uint32_t)(t < most ? t : most) * (uint32_t)A.ld_x + 16 * fc;
    }
    const int steps = A.k / 64, from = (int)((long long)steps * wave / FEW_WAVES), to = (int)((long long)steps * (wave + 1) / FEW_WAVES);
    const int start = gridDim.y == 1 && to > from ? scattered(blockIdx.x, to - from) : 0;   // as in qlin_tile_kernel
    v4i acc[H][NB] = {};
    Words a[2][U][H], b[2][U][NB];
    int shift_w[2], shift_x[NB];   // of a lane's rows (their 16-byte pieces are 16 apart: the same for all)
    shift_w[0] = (int)(((uintptr_t)pw[0] + vw) & 3);
    shift_w[1] = (int)(((uintptr_t)pw[1] + vw) & 3);
#pragma unroll
    for (int i = 0; i < NB; ++i)
        shift_x[i] = (int)(((uintptr_t)px + vx[i]) & 3);
    auto mfma = [&](const v4i (&fa)[H], const v4i (&fb)[NB]) {
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
    };
    auto step = [&](const Words (&wa)[H], const Words (&wb)[NB]) {
        v4i fa[H], fb[NB];
#pragma unroll
        for (int i = 0; i < H; ++i)
            fa[i] = shifted<BYTES>(wa[i], shift_w[i]);
#pragma unroll
        for (int i = 0; i < NB; ++i)
            fb[i] = shifted<BYTES>(wb[i], shift_x[i]);
        mfma(fa, fb);
    };
    // two sets of U steps in turn: one in flight, one in the MFMAs; in a set, loads past the range read its last step
    // again and are not used (with a whole set of those at the end 1 x 6144 x 4096 8.5 us, without 7.6)
    if (int s = from; s < to) {
        auto fill = [&](int set, int s) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = s + u < to ? s + u : to - 1, turn = at + start < to ? at + start : at + start - (to - from);
                const int c = 64 * turn;
#pragma unroll
                for (int i = 0; i < H; ++i)
                    a[set][u][i] = load_words<BYTES>(pw[i] + c, vw);
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    b[set][u][i] = load_words<BYTES>(px + c, vx[i]);
            }
        };
        auto use = [&](int set, int s) {
            if (s + U <= to) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    step(a[set][u], b[set][u]);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (s + u < to)
                        step(a[set][u], b[set][u]);
            }
        };
        fill(0, s);
        for (;;) {
            if (s + U < to)
                fill(1, s + U);
            use(0, s);
            s += U;
            if (s >= to)
                break;
            if (s + U < to)
                fill(0, s + U);
            use(1, s);
            s += U;
            if (s >= to)
                break;
        }
    }
    if (64 * steps < A.k && wave == FEW_WAVES - 1) {   // the last k
        const int k = 64 * steps + 16 * fc;
        v4i fa[H], fb[NB];
#pragma unroll
        for (int i = 0; i < H; ++i)
            fa[i] = load16<false>(pw[i] + vw - 16 * fc, k, A.k);
#pragma unroll
        for (int i = 0; i < NB; ++i)
            fb[i] = load16<true>(px + vx[i] - 16 * fc, k, A.k);
        mfma(fa, fb);
    }
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            sums[wave][i * NB + j][lane] = acc[i][j];
    __syncthreads();
    for (int j = wave; j < NB; j += FEW_WAVES) {
        const long long t = t0 + 16 * j + fr;
        v4i c[H] = {};
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w)
#pragma unroll
            for (int h = 0; h < H; ++h)
                c[h] += sums[w][h * NB + j][lane];
        if (t < A.rows)
            emit4<T, GATE>(A, t, j0 + 4 * fc, c[0], c[H - 1], A.x_scales[t]);
    }
}

// ---- tiles through LDS -------------------------------------------------------------------
// A workgroup computes TN rows of w by TM tokens; the next 128 k of both operands (one stage) go
// into LDS ahead of the MFMAs, a ring of RING stages. Wave (i, j) of WN x WM holds TN / WN rows by
// TM / WM tokens in accumulators of 32 x 32; a stage is four steps of 32 k.
//
// COPY: rows start at multiples of 4 bytes and are copied straight into LDS, 16 bytes a lane (lines that
// they straddle cost 10 to 25%: 1000 x 4096 x 4096 21.5 us at multiples of 128, 26.4 at others).
// Otherwise they start anywhere and pass through registers, loaded one stage before they
// are written (RING 2).
// The k that no whole stage has are copied as one more stage, after the others (5264 x 6912 x 560 47.7 us, 51.5
// where they passed through registers after the last MFMA).
//
// While the MFMAs of one step run, the fragments of the next are read; in the last step, after the
// first few MFMAs, the workgroup meets: by then each wave has read all of its stage (so its place
// may be refilled) and its own part of the next one is in LDS. With one or two MFMAs a step that is
// too short a time, and a whole stage's fragments are read ahead (DEEP).
//
// The 16-byte columns of LDS row r (128 bytes) sit XORed with swz(r), which is done by permuting the
// lanes' source columns; fragment reads hit every bank once (no conflict in the counters).
//
// Large products are bound by power: 8192 x 8192 x 8192 takes 449 to 474 us (2320 to 2450 TOPS), its matrix cores busy
// for 63% of the cycles of a clock that falls to 1.7 GHz (on codes of zero 404 us). Small tiles (up to 128 x 64)
// are bound by their copies (24 KiB a stage in 0.25 us: 47 bytes a clock and CU) and their first and last microseconds. The
// 128 x 128 tiles of a sum split in 4 over rows of 16384 bytes (192 x 4096 x 16384) are bound by neither: 20 bytes a clock.
typedef int v16i __attribute__((ext_vector_type(16)));
typedef uint32_t v4u32 __attribute__((ext_vector_type(4)));

// 16 bytes per lane from rsrc's base + voff + soff to LDS address la + 16 * lane. Not
// tracked by the compiler: every wait for it is an explicit wait_vmcnt.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16(v4u32 rsrc, uint32_t voff, uint32_t soff, uint32_t la)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 ::"s"(la), "v"(voff), "s"(rsrc), "s"(soff) : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ v4u32 raw_rsrc(const void *p)
{
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return v4u32{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xFFFFu)), 0xFFFFFFFFu, 0x00020000u};
}

// Position of tile `id` of `total`. Workgroups go round the 8 XCDs, so each XCD takes a contiguous range, in
// strips of up to 4 token tiles along the rows of w: the tiles that run at once on an XCD share their
// operands in its L2. Each eighth of the strips starts an eighth further along (`tn`): where y's rows are a
// power of two of bytes, XCDs that all write the same columns meet on a few memory channels (134 MB of y
// 30.4 us together, 24.6 apart; 8192 x 8192 x 2048 155 -> 148 us when it came in).
struct Place {
    int tn, tt, part, eighth;
};
template <bool PART>
__device__ __forceinline__ Place place(unsigned id, unsigned total, int tiles_n, int tiles_t)
{
    const unsigned x = id & 7, i = id >> 3, q = total >> 3, r = total & 7;
    unsigned t = x * q + (x < r ? x : r) + i;
    Place p = {0, 0, 0, 0};
    if constexpr (PART) {
        const unsigned per = (unsigned)tiles_n * (unsigned)tiles_t;
        p.part = (int)(t / per);
        t -= p.part * per;
    }
    if (tiles_t <= 4) {   // one strip
        p.tn = (int)(t / (unsigned)tiles_t);
        p.tt = (int)(t - p.tn * (unsigned)tiles_t);
        return p;
    }
    const unsigned strip = t / (4u * tiles_n), first = 4 * strip, high = tiles_t - first < 4 ? tiles_t - first : 4;
    t -= strip * 4u * tiles_n;
    p.eighth = (int)(8 * strip / ((tiles_t + 3u) / 4));
    p.tt = (int)(first + t % high);
    t = t / high + (unsigned)((unsigned long long)p.eighth * tiles_n / 8);
    p.tn = (int)(t < (unsigned)tiles_n ? t : t - tiles_n);
    return p;
}

// What a wave's lanes wrote to LDS is there for its other lanes, which the LDS's order within a wave makes so by itself: this
// keeps the compiler to it (no instruction).
__device__ __forceinline__ void lanes_meet()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The sums of a wave to y (or the partial sums): 32 tokens at a time through the wave's own
// 32 x (32 NA) int32 of LDS, so that stores are whole lines of consecutive outputs, and a
// lane keeps the scales of its channels. A lane holds token lane % 32, rows 8 g + 4 (lane / 32)
// .. + 3 of each 32 x 32; the 16-byte columns of a staged token are XORed with the token. With the gate
// the value rows follow the gate rows.
template <typename T, bool GATE, bool PART, bool PAST, int NA, int NB>
__device__ __forceinline__ void store_tile(const QlinArgs &A, const v16i (&acc)[NA][NB], int8_t *stage, int part, long long t0, int j0)
{
    constexpr int WIDE = 32 * NA, SLOTS = WIDE / 4, OUT = GATE && !PART ? WIDE / 2 : WIDE;
    constexpr int V = PART ? 4 : 16 / (int)sizeof(T), LANES = OUT / V;   // outputs per lane, lanes per token
    const int lane = threadIdx.x & 63, o = lane % LANES * V;
    typedef T vecT __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    const int j = j0 + o, left = A.n - j;
    // All scales are loaded before the first store (a load after one could not be moved up, and would be waited for
    // in every round): lane l keeps the scale of token t0 + l, shuffled to the lanes that want it.
    static_assert(NB <= 2, "a lane per token");
    float ws[V] = {}, wb[V] = {}, vs[V] = {}, vb[V] = {}, xs = 0.f;
    if constexpr (!PART) {
        if (lane < 32 * NB && t0 + lane < A.rows)
            xs = A.x_scales[t0 + lane];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = j + e < A.n ? j + e : A.n - 1;
            ws[e] = A.w_scales[c];
            if (A.bias)
                wb[e] = A.bias[c];
            if constexpr (GATE) {
                vs[e] = A.w_scales[A.n + c];
                if (A.bias)
                    vb[e] = A.bias[A.n + c];
            }
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int tw = lane & 31;
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int row = GATE ? 32 * (i / 2) + (i & 1) * (WIDE / 2) : 32 * i;
                const int slot = (row / 4 + 2 * g + (lane >> 5)) ^ (tw & (SLOTS - 1));
                *(v4i *)(stage + (tw * SLOTS + slot) * 16) = v4i{acc[i][b][4 * g], acc[i][b][4 * g + 1], acc[i][b][4 * g + 2], acc[i][b][4 * g + 3]};
            }
        lanes_meet();
        // (past: past the L2, in tiles of large outputs; a choice within a round would be lost where the compiler joins
        // the stores again)
        auto rounds = [&](auto past) {
#pragma unroll
            for (int it = 0; it < 32 * LANES / 64; ++it) {
                const int tr = it * (64 / LANES) + lane / LANES;
                const long long t = t0 + 32 * b + tr;
                auto sums = [&](int row, int e) {
                    return *(const v4i *)(stage + (tr * SLOTS + (((row + e) / 4) ^ (tr & (SLOTS - 1)))) * 16);
                };
                if constexpr (PART) {
                    if (t < A.rows) {
                        // with the gate the staged rows are both halves: j0 counts outputs, o staged rows
                        if constexpr (GATE)
                            put4<true>(A, part, t, j0 + o % (WIDE / 2), o / (WIDE / 2), sums(o, 0));
                        else
                            put4<false>(A, part, t, j, 0, sums(o, 0));
                    }
                } else if (const float sx = __shfl(xs, 32 * b + tr); t < A.rows) {
                    float zs __attribute__((ext_vector_type(V)));
#pragma unroll
                    for (int e = 0; e < V; e += 4) {
                        const v4i c = sums(o, e);
                        v4i d = {};
                        if constexpr (GATE)
                            d = sums(WIDE / 2 + o, e);
#pragma unroll
                        for (int f = 0; f < 4; ++f) {
                            float z = __builtin_fmaf((float)c[f] * sx, ws[e + f], wb[e + f]);
                            if constexpr (GATE)
                                z = in_fp32<T>(silu(z) * __builtin_fmaf((float)d[f] * sx, vs[e + f], vb[e + f]));
                            zs[e + f] = z;
                        }
                    }
                    const vecT y = __builtin_convertvector(zs, vecT);
                    T *out = (T *)A.y + t * A.ld_y + j;
                    if (left >= V) {
                        if constexpr (past.value)
                            __builtin_nontemporal_store(y, (vecT *)out);
                        else
                            *(vecT *)out = y;
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            if (e < left)
                                out[e] = y[e];
                    }
                }
            }
        };
        if (PAST && !PART && A.whole_lines)
            rounds(std::true_type{});
        else
            rounds(std::false_type{});
        lanes_meet();   // the next tokens take their place
    }
}

template <typename T, bool GATE, bool PART, bool COPY, int TN, int TM, int WN, int WM, int RING>
__global__ void __launch_bounds__(64 * WN * WM, RING * (TN + TM) * KS <= 80 << 10 ? (WN * WM + 1) / 2 : 1)
qlin_tile_kernel(QlinArgs A, unsigned tile0, unsigned total)   // (waves per SIMD: registers for two workgroups where LDS has room for them)
{
    constexpr int WAVES = WN * WM, NA = TN / WN / 32, NB = TM / WM / 32, OUT = GATE ? TN / 2 : TN;
    constexpr int STAGE = (TN + TM) * KS, STEPS = KS / 32;
    // a copy is 8 rows of 128 bytes: COPIES per wave and stage, the first WCOPIES of rows of w
    constexpr int WCOPIES = TN / 8 / WAVES, COPIES = (TN + TM) / 8 / WAVES;
    constexpr int M = NA * NB, R = NA + NB;   // MFMAs and fragments of a step
    constexpr bool DEEP = M <= 2;
    static_assert(WCOPIES * 8 * WAVES == TN && COPIES * 8 * WAVES == TN + TM, "whole copies per wave");
    static_assert(!GATE || NA % 2 == 0, "a wave holds gate and value");
    static_assert(RING * STAGE >= WAVES * 32 * 32 * NA * 4 && RING * STAGE <= 160 << 10, "the outputs are staged in the ring");
    static_assert((RING - 1) * COPIES < 64, "waits count to 63");
    static_assert(COPY || (RING == 2 && !DEEP), "through registers: two places, stages of many MFMAs");
    __shared__ __attribute__((aligned(16))) int8_t ring[RING * STAGE];
    const int tiles_n = (A.n + OUT - 1) / OUT, tiles_t = (int)((A.rows + (long long)TM - 1) / TM);
    const Place at = place<PART>(tile0 + blockIdx.x, total, tiles_n, tiles_t);
    const int k0 = at.part * A.kchunk, k1 = A.k - k0 < A.kchunk ? A.k : k0 + A.kchunk;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t base = lds_addr(ring);

    // Copy q of a wave moves LDS rows 8 (wave + WAVES q) .. + 7; the rows of w come first. With the
    // gate, 32 gate rows and the 32 value rows of the same outputs take turns, so that a wave
    // holds both halves of its outputs.
    const int8_t *wbase = A.w + (long long)at.tn * OUT * A.ld_w, *xbase = A.x + (long long)at.tt * TM * A.ld_x;
    const int8_t *vbase = wbase + (GATE ? A.n * A.ld_w : 0);
    uint32_t voff[COPIES];
#pragma unroll
    for (int q = 0; q < COPIES; ++q) {
        const int r = 8 * (wave + WAVES * q) + (lane >> 3), c = (lane & 7) ^ swz(r);
        if (q < WCOPIES) {
            const int j = GATE ? 32 * (r >> 6) + (r & 31) : r, left = A.n - 1 - at.tn * OUT;
            voff[q] = (uint32_t)(j < left ? j : left) * (uint32_t)A.ld_w + 16 * c;
        } else {
            const int t = r - TN;
            const long long left = A.rows - 1 - (long long)at.tt * TM;
            voff[q] = (uint32_t)(t < left ? t : left) * (uint32_t)A.ld_x + 16 * c;
        }
    }
    auto source = [&](int q) { return q >= WCOPIES ? xbase : GATE && (8 * (wave + WAVES * q) & 32) ? vbase : wbase; };
    const v4u32 rw = raw_rsrc(wbase), rv = raw_rsrc(vbase), rx = raw_rsrc(xbase);
    // copy q of the stage at `from` into place `place` of the ring
    struct From {
        uint32_t soff, slide;
    };
    auto copy = [&](int q, From from, int place) {
        copy16(q >= WCOPIES ? rx : GATE && (8 * (wave + WAVES * q) & 32) ? rv : rw, voff[q] + from.slide, from.soff,
               __builtin_amdgcn_readfirstlane(base + (uint32_t)place * STAGE + 1024u * (wave + WAVES * q)));
    };
    // The other way in: the next HOLD copies are on their way through registers. Half a stage of them where
    // the accumulators leave no room for more (and a stage is long).
    constexpr int HOLD = TN * TM >= 256 * 256 ? COPIES / 2 : COPIES;
    Words held[COPY ? 1 : HOLD];
    auto load = [&](int q, int stage) { held[q % HOLD] = load_words<true>(source(q) + k0 + KS * stage, voff[q]); };
    auto store = [&](int q, int place) {
        const int shift = (int)(((uintptr_t)source(q) + voff[q]) & 3);
        *(v4i *)(ring + place * STAGE + 1024 * (wave + WAVES * q) + 16 * lane) = shifted<true>(held[q % HOLD], shift);
    };

    const int wn = wave / WM, wm = wave % WM, fr = lane & 31;
    const int8_t *fa = ring + (wn * (TN / WN) + fr) * KS, *fb = ring + (TN + wm * (TM / WM) + fr) * KS;
    int col[STEPS];   // where a lane finds its 16 bytes of each step in a row
#pragma unroll
    for (int p = 0; p < STEPS; ++p)
        col[p] = ((2 * p + (lane >> 5)) ^ swz(fr)) * 16;
    v16i acc[NA][NB] = {};
    v4i a[DEEP ? 2 * STEPS : 2][NA], b[DEEP ? 2 * STEPS : 2][NB];
    auto read = [&](int set, int i, int off) {
        if (i < NA)
            a[set][i] = *(const v4i *)(fa + off + i * 32 * KS);
        else
            b[set][i - NA] = *(const v4i *)(fb + off + (i - NA) * 32 * KS);
    };
    auto mfma = [&](int set, int m) {
        const int i = m / NB, j = m % NB;
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[set][i], b[set][j], acc[i][j], 0, 0, 0);
    };

    // (copies and loads past the last stage take the last stage again, into a place that nothing reads, so
    // that the counts of copies in flight hold)
    const int stages = (k1 - k0) / KS, last = stages - 1, rest = k0 + KS * stages;   // rest: the k that no whole stage has
    // Where this workgroup starts: a sum's terms have no order. With rows of a power of two of bytes, workgroups that
    // all read the same columns meet on a few memory channels. Where each row of w is read by one of them
    // (one token tile) all start apart (16 x 16384 x 4096 gated all at 0 34.3 us, each a stage after the last 30.1,
    // scattered 26.5; 32 x 8192 x 4096 gated 15.3 by stages, 15.9 scattered, the worst found); of many token tiles each eighth
    // does, whose workgroups share their reads (2048 x 11264 x 4096 gated 186 -> 180 us, 8192 x 8192 x 8192 the same).
    const int start = !stages ? 0 : tiles_t == 1 ? scattered(tile0 + blockIdx.x, stages) : (int)((long long)stages * at.eighth / 8);
    auto turned = [&](int s) { return s + start < stages ? s + start : s + start - stages; };
    // Where the copies of the s-th stage start. The k that no whole stage has are one more; a row ends inside it, and
    // a lane whose 16 bytes would pass the row's last word takes the 16 bytes up to there (load16 does the same).
    const int end = (k1 + 3) & ~3;   // (of whole words; k >= 16)
    auto first = [&](int c) { return rest + 16 * c < end - 16 ? rest + 16 * c : end - 16; };
    const int mine = (lane & 7) ^ swz(8 * wave + (lane >> 3));   // this lane's column in each of its copies
    const uint32_t slide = (uint32_t)(first(mine) - 16 * mine);
    static_assert(WAVES % 2 == 0, "swz is the same in all copies of a wave");
    auto from = [&](int s) {
        return s == stages && rest < k1 ? From{0, slide} : From{(uint32_t)(k0 + KS * turned(s < last ? s : last)), 0};
    };
    int place = 0;
    if (COPY && !stages) {
#pragma unroll
        for (int q = 0; q < COPIES; ++q)
            copy(q, from(0), 0);
    }
    if (DEEP && stages) {
#pragma unroll
        for (int s = 0; s < RING; ++s)
#pragma unroll
            for (int q = 0; q < COPIES; ++q)
                copy(q, from(s), s);
        wait_vmcnt<(RING - 1) * COPIES>();
        asm volatile("s_barrier" ::: "memory");
        static_for<STEPS * R>([&](auto i) { read(i.value / R, i.value % R, col[i.value / R]); });
        auto stage = [&](auto P, int s) {
            // every wave has read stage s, whose place may be refilled, and stage s + 1 has landed
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((RING - 2) * COPIES) : "memory");
            const int next = place + 1 == RING ? 0 : place + 1;
            const From ahead = from(s + RING);
            static_for<STEPS * R>([&](auto i) {
                read((1 - P.value) * STEPS + i.value / R, i.value % R, next * STAGE + col[i.value / R]);
            });
#pragma unroll
            for (int q = 0; q < COPIES; ++q)
                copy(q, ahead, place);
            static_for<STEPS * M>([&](auto m) { mfma(P.value * STEPS + m.value / M, m.value % M); });
            place = next;
        };
        for (int s = 0; s < stages; s += 2) {
            stage(std::integral_constant<int, 0>{}, s);
            if (s + 1 == stages)
                break;
            stage(std::integral_constant<int, 1>{}, s + 1);
        }
    }
    if (!DEEP && stages) {
        if constexpr (COPY) {
#pragma unroll
            for (int s = 0; s < RING - 1; ++s)
#pragma unroll
                for (int q = 0; q < COPIES; ++q)
                    copy(q, from(s), s);
            wait_vmcnt<(RING - 2) * COPIES>();
            asm volatile("s_barrier" ::: "memory");
        } else {
#pragma unroll
            for (int q = 0; q < HOLD; ++q)
                load(q, turned(0));
#pragma unroll
            for (int q = 0; q < COPIES; ++q) {
                store(q, 0);
                if (q + HOLD < COPIES)
                    load(q + HOLD, turned(0));
                else
                    load(q + HOLD - COPIES, turned(1 < last ? 1 : last));
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
            read(0, i, col[0]);
        constexpr int MEET = M >= 16 ? 4 : M >= 8 ? 2 : 1;   // MFMAs of the last step before the workgroup meets
        constexpr int SPREAD = M * (STEPS - 1);              // MFMAs that the copies are spread over
        int off = 0;
        for (int s = 0; s < stages; ++s) {
            const int into = (s + RING - 1) % RING;
            const From ahead = from(s + RING - 1);
            // (through registers)
            const int next_load = turned(s + 1 < last ? s + 1 : last), after = turned(s + 2 < last ? s + 2 : last);
            static_for<STEPS - 1>([&](auto p) {
                static_for<M>([&](auto m) {
                    static_for<R>([&](auto i) {
                        if constexpr (i.value * (M < R ? M : R) / R == m.value)
                            read((p.value + 1) & 1, i.value, off + col[p.value + 1]);
                    });
                    mfma(p.value & 1, m.value);
                    static_for<COPIES>([&](auto q) {
                        if constexpr (q.value * SPREAD / COPIES == p.value * M + m.value) {
                            if constexpr (COPY) {
                                copy(q.value, ahead, into);
                            } else {
                                store(q.value, into);
                                if constexpr (q.value + HOLD < COPIES)
                                    load(q.value + HOLD, next_load);
                                else
                                    load(q.value + HOLD - COPIES, after);
                            }
                        }
                    });
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            const int next = s == last ? off : (s + 1) % RING * STAGE;
            static_for<M>([&](auto m) {
                if constexpr (m.value == MEET) {
                    if constexpr (COPY)
                        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((RING - 2) * COPIES) : "memory");
                    else
                        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                    __builtin_amdgcn_sched_barrier(0);
                }
                static_for<R>([&](auto i) {
                    if constexpr (MEET + i.value * (M - MEET < R ? M - MEET : R) / R == m.value)
                        read(0, i.value, next + col[0]);
                });
                mfma((STEPS - 1) & 1, m.value);
                __builtin_amdgcn_sched_barrier(0);
            });
            off = next;
        }
    }
    // the last k, where 128 does not divide them
    wait_vmcnt<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (rest < k1) {
        const int off = COPY ? stages % RING * STAGE : 0;
        if constexpr (!COPY) {
#pragma unroll
            for (int q = 0; q < COPIES; ++q) {
                const int c = (lane & 7) ^ swz(8 * (wave + WAVES * q) + (lane >> 3));
                *(v4i *)(ring + 1024 * (wave + WAVES * q) + 16 * lane) =
                    q < WCOPIES ? load16<false>(source(q) + (voff[q] - 16 * c), rest + 16 * c, k1)
                                : load16<true>(source(q) + (voff[q] - 16 * c), rest + 16 * c, k1);
            }
            __syncthreads();
        }
#pragma unroll
        for (int p = 0; p < STEPS; ++p) {
            if (rest + 32 * p >= k1)
                break;
#pragma unroll
            for (int i = 0; i < R; ++i)
                read(p & 1, i, off + col[p]);
            if constexpr (COPY) {   // zeros in the tokens for what is past the row, or in another lane or stage too
                const int c = 2 * p + (lane >> 5), gone = rest + 16 * c - first(c), over = end - k1;
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int z = gone - 4 * e;
                        uint32_t mask = z >= 4 ? 0u : z > 0 ? ~0u << (8 * z) : ~0u;
                        if (e == 3 && first(c) == end - 16)
                            mask &= ~0u >> (8 * over);
                        b[p & 1][j][e] &= (int)mask;
                    }
            }
#pragma unroll
            for (int m = 0; m < M; ++m)
                mfma(p & 1, m);
        }
    }

    __syncthreads();   // every wave is done with the ring, which now stages the outputs
    const int j0 = at.tn * OUT + wn * (OUT / WN);
    const long long t0 = (long long)at.tt * TM + wm * (TM / WM);
    store_tile<T, GATE, PART, (TN * TM >= 256 * 128), NA, NB>(A, acc, ring + wave * 32 * NA * 32 * 4, at.part, t0, j0);
}

// ---- launches ---------------------------------------------------------------------------
constexpr unsigned MOST_GROUPS = 1u << 22;   // workgroups of one launch (a multiple of 8: XCDs keep their turns)

template <typename T, bool GATE, bool PART>
void launch_any(const QlinArgs &a, hipStream_t stream)
{
    constexpr int OUT = GATE ? ANY_TILE / 2 : ANY_TILE;
    const long long total = (long long)((a.n + OUT - 1) / OUT) * ((a.rows + ANY_TILE - 1) / ANY_TILE) * a.ksplit;
    for (long long at = 0; at < total; at += MOST_GROUPS) {
        const dim3 grid((unsigned)(total - at < MOST_GROUPS ? total - at : MOST_GROUPS));
        hipLaunchKernelGGL((qlin_any_kernel<T, GATE, PART>), grid, dim3(256), 0, stream, a, at);
    }
}

template <typename T, bool GATE, bool BYTES, int NB, int U>
void launch_few(const QlinArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.n + 15) / 16), (unsigned)((a.rows + 16 * NB - 1) / (16 * NB)));
    hipLaunchKernelGGL((qlin_few_kernel<T, GATE, BYTES, NB, U>), grid, dim3(64 * FEW_WAVES), 0, stream, a);
}

template <typename T, bool GATE, bool PART, bool COPY, int TN, int TM, int WN, int WM, int RING>
void launch_tile(const QlinArgs &a, hipStream_t stream)
{
    constexpr int OUT = GATE ? TN / 2 : TN;
    const unsigned total = (unsigned)((a.n + OUT - 1) / OUT) * (unsigned)((a.rows + TM - 1) / TM) * (unsigned)a.ksplit;
    for (unsigned at = 0; at < total; at += MOST_GROUPS) {
        const dim3 grid(total - at < MOST_GROUPS ? total - at : MOST_GROUPS), block(64 * WN * WM);
        hipLaunchKernelGGL((qlin_tile_kernel<T, GATE, PART, COPY, TN, TM, WN, WM, RING>), grid, block, 0, stream, a, at, total);
    }
}

// rows of w (with the gate: of both halves) x tokens; a gated tile's waves hold pairs of row tiles. False for a shape that
// is not there in this form, for which nothing is launched.
template <typename T, bool GATE, bool PART>
bool launch_shape(const QlinArgs &a, int shape, hipStream_t stream)
{
    switch (shape) {
    case QLIN_ANY: return launch_any<T, GATE, PART>(a, stream), true;
    case QLIN_64x32:
        if constexpr (GATE)
            return launch_tile<T, GATE, PART, true, 128, 32, 2, 1, 4>(a, stream), true;
        else
            return launch_tile<T, GATE, PART, true, 64, 32, 2, 1, 4>(a, stream), true;
    case QLIN_64x64:   // plain only: the gated 128x64 has the same tile
        if constexpr (!GATE)
            return launch_tile<T, GATE, PART, true, 64, 64, 2, 2, 4>(a, stream), true;
        break;
    case QLIN_128x64:
        if constexpr (GATE)
            return launch_tile<T, GATE, PART, true, 128, 64, 2, 2, 3>(a, stream), true;
        else
            return launch_tile<T, GATE, PART, true, 128, 64, 4, 2, 3>(a, stream), true;
    case QLIN_128x128:
        if constexpr (GATE)
            return launch_tile<T, GATE, PART, true, 128, 128, 2, 4, 3>(a, stream), true;
        else
            return launch_tile<T, GATE, PART, true, 128, 128, 4, 2, 3>(a, stream), true;
    case QLIN_128x128_TWO:   // two stages of LDS: two workgroups to a CU
        if constexpr (GATE)
            return launch_tile<T, GATE, PART, true, 128, 128, 2, 4, 2>(a, stream), true;
        else
            return launch_tile<T, GATE, PART, true, 128, 128, 4, 2, 2>(a, stream), true;
    case QLIN_256x128: return launch_tile<T, GATE, PART, true, 256, 128, 4, 2, 3>(a, stream), true;
    case QLIN_256x256: return launch_tile<T, GATE, PART, true, 256, 256, 2, 4, 2>(a, stream), true;
    case QLIN_128x128_ANY: return launch_tile<T, GATE, PART, false, 128, 128, 2, 2, 2>(a, stream), true;
    case QLIN_256x256_ANY: return launch_tile<T, GATE, PART, false, 256, 256, 2, 4, 2>(a, stream), true;
    default: break;
    }
    if constexpr (!PART) {
        const bool bytes = (((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.ld_x | (uintptr_t)a.ld_w) & 3) != 0;
        if (shape == QLIN_FEW16)
            return bytes ? launch_few<T, GATE, true, 1, 4>(a, stream) : launch_few<T, GATE, false, 1, 4>(a, stream), true;
        if (shape == QLIN_FEW64)
            return launch_few<T, GATE, true, 4, 2>(a, stream), true;   // (aligned rows have faster tiles)
    }
    return false;
}

template <typename T>
hipError_t launch_typed(const QlinArgs &a, int shape, hipStream_t stream)
{
    const bool known = a.gate ? launch_shape<T, true, false>(a, shape, stream) : launch_shape<T, false, false>(a, shape, stream);
    return known ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace
}  // namespace aqd
