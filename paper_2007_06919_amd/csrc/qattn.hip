// Attention over the 4-bit cache. Definition and layout: include/aqd.h.
//
// A workgroup has one sequence, one key head, 16 rows (32 of dim 64 where there are so many: the query heads of the key head, times
// the sequence's queries) and a range of tokens; its four waves take 32 tokens in turn, each with a
// softmax of its own, joined at the end. With S^T = K Q^T and O^T = V^T P^T (16 x 16 x 32 products) the
// scores' lanes are the weights' lanes: lane (r, g) has the scores of tokens 4 g .. 4 g + 3 of a tile of 16 for row r,
// which is what the second product takes for k = 8 g .. from two tiles, so no weight changes lanes.
//
// A code becomes an operand by one shift and one and-or for two: c is put below the leading bit of 128 (bf16) or 64
// (fp16), which makes 128 + c or 64 + c. Products with a constant -136 or -72 take the offset, 8 included, out again
// before it is scaled, which leaves the sums of c - 8 with the roundings of sums up to 35 (fp16: 19) times as large: up to five of fp32's 24
// bits. A key's scale multiplies its scores of the group in fp32. A value's scale multiplies its weights, and the products are rounded to T:
// the matrix cores take no more bits at this rate, and the result has no more. Against 64 bits that leaves the error which fp32 weights have
// (64 of 700 to 8192, bf16: 0.0017 of the result's norm with either, nearly all of it the rounding of the result).
//
// Bound by the vector units, and by how even the workgroups are: 64 sequences of 700 to 8192 tokens, 32 query heads on 8, dim 128, groups of 32
// take 82 to 84 us, 334 MB at 4.0 TB/s; 375 vector instructions a step of 32 tokens (112 of them make operands of codes, 150 apply scales) are 54%
// of the cycles, the matrix cores 14%. With groups of 128 and 3 of 120000 (64 heads on 8) 74 us and 8 for the second launch.
// 64 of 8192 with groups of 64 take 113 to 117 us, 5.0 TB/s. One sequence of 1500: 9.2 us, two launches of 5.2 and 4.2.
//
// fp16 weights have few exponents: there the softmax's reference is the largest sum of a score and the exponent of its value's
// scales, so that the largest product of weight and scale is near 1 whatever the values' sizes.

#include <algorithm>

#include "attn_common.h"

namespace aqd {
namespace {

template <typename T>
struct Code;
template <>
struct Code<__bf16> {
    static constexpr uint32_t MASK = 0x000F000Fu, BASE = 0x43004300u, OFF = 0xC308C308u;   // 128 + c; -136
    static constexpr int AT = 0;
    static constexpr bool NARROW = false;
};
template <>
struct Code<_Float16> {
    static constexpr uint32_t MASK = 0x00F000F0u, BASE = 0x54005400u, OFF = 0xD480D480u;   // 64 + c; -72
    static constexpr int AT = 4;
    static constexpr bool NARROW = true;
};

// nibbles J and J + 4 of a word as two operands. mask and base: MASK and BASE in registers, of which the compiler must not
// know the value: with constants it takes two instructions for the and and the or.
template <typename T, int J>
__device__ __forceinline__ uint32_t widen(uint32_t w, uint32_t mask, uint32_t base)
{
    constexpr int shift = 4 * J - Code<T>::AT;
    if constexpr (shift > 0)
        w >>= shift;
    else if constexpr (shift < 0)
        w <<= -shift;
    return (w & mask) | base;
}

// two words at byte offsets of a wave-uniform address, through the scalar cache (a vector load would wait for the copies)
__device__ __forceinline__ void scalar_loads(const int32_t *p, int a, int b, int &x, int &y)
{
    asm volatile("s_load_dword %0, %2, %3\n\ts_load_dword %1, %2, %4\n\ts_waitcnt lgkmcnt(0)" : "=&s"(x), "=&s"(y) : "s"(p), "s"(a), "s"(b));
}

// one sequence as the kernels see it
struct Sequence {
    int begin, n, length;
};
__device__ __forceinline__ int length_of(const QattnArgs &A, int b)
{
    return (int)max(min((long long)min(A.lengths[b], A.max_keys), A.ld_table * A.c.page), 0LL);
}
__device__ __forceinline__ Sequence sequence(const QattnArgs &A, int b)
{
    Sequence s;
    s.begin = A.q_start ? min(max(A.q_start[b], 0), A.queries) : b;
    const int end = A.q_start ? min(max(A.q_start[b + 1], 0), A.queries) : b + 1;
    s.n = min(end - s.begin, A.max_queries);
    s.length = length_of(A, b);
    return s;
}
__device__ __forceinline__ int tiles_of(const QattnArgs &A, int b, int rows)
{
    return (max(sequence(A, b).n, 0) * (A.q_heads / A.c.heads) + rows - 1) / rows;
}
// Sequences of unlike lengths share `slots` workgroups (of a key head and row tile) by their tokens: a workgroup has
// `chunk` of them at most, such that sum(floor(length / chunk) + 1) <= slots. Their results are numbered by sequence.
struct Share {
    int b, chunk, first, parts, full;   // a sequence; its slots, and how many of them are whole chunks
};
constexpr int SHARED = 1024, LEAST = 256;   // most sequences; least tokens of a chunk
struct Shared {
    const QattnArgs &A;
    int lane, near, units;   // near: tokens of the first 64 sequences, in units of 128; units: a chunk

    __device__ __forceinline__ Shared(const QattnArgs &args, int slots) : A(args), lane(threadIdx.x & 63)
    {
        near = lane < A.batch ? (length_of(A, lane) + 127) / 128 : 0;
        int total = near;
#pragma unroll 4
        for (int k = 64; k < A.batch; k += 64)
            total += tokens(k);
        units = max((wave_sum(total) + slots - A.batch - 1) / (slots - A.batch), LEAST / 128);
    }
    __device__ __forceinline__ int tokens(int k) const { return k ? (k + lane < A.batch ? (length_of(A, k + lane) + 127) / 128 : 0) : near; }
    __device__ __forceinline__ Share of(int b) const
    {
        int before = 0, k = 0;
        for (; k + 64 <= b; k += 64)
            before += wave_sum(max((int)((unsigned)(tokens(k) + units - 1) / units), 1));
        const int n = tokens(k), parts = max((int)((unsigned)(n + units - 1) / units), 1), upto = wave_scan(parts);
        const int at = __builtin_amdgcn_readfirstlane(b - k), own = __builtin_amdgcn_readlane(parts, at);
        return {b, 128 * units, before + __builtin_amdgcn_readlane(upto, at) - own, own, (int)((unsigned)__builtin_amdgcn_readlane(n, at) / units)};
    }
    // of workgroup `at`: all full chunks come first, then what is left of each sequence
    __device__ __forceinline__ bool find(int at, Share &s, int &part) const
    {
        int before = 0, b = -1;
        part = -1;
        for (int k = 0; k < A.batch; k += 64) {
            const int full = (unsigned)tokens(k) / units, upto = wave_scan(full) + before;
            const uint64_t has = __builtin_amdgcn_ballot_w64(upto > at);
            if (has) {
                const int from = __builtin_ctzll(has);
                b = k + from;
                part = at - __builtin_amdgcn_readlane(upto - full, from);
                break;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
        }
        if (b < 0)
            b = at - before;
        if (b >= A.batch)
            return false;
        s = of(b);
        if (part >= 0)
            return true;
        part = s.parts - 1;
        return s.parts > s.full;
    }
};
// how many tokens a workgroup's rows see at most
__device__ __forceinline__ int seen_by(const Sequence &s, int rows, int first_row, int per)
{
    const int last = min((first_row + rows - 1) / per, s.n - 1);
    return max(s.length - s.n + 1 + last, 0);
}

// Rows of the workspace: [queries][q_heads][parts], or [slots][max_queries][q_heads] of shared slots.
__device__ __forceinline__ long long part_rows(const QattnArgs &A, int slots, int parts)
{
    return slots ? (long long)slots * A.max_queries * A.q_heads : (long long)A.queries * A.q_heads * parts;
}

template <int DIM, int GROUP, int R>
struct Shape {
    static constexpr int GROUPS = DIM / GROUP;
    static constexpr int CODES = 16 * DIM;                                     // a tile's codes, keys and values, bytes
    static constexpr int SCALES = 64 * GROUPS, SCALE_ROOM = SCALES < 256 ? 256 : SCALES;
    static constexpr int TILE = CODES + SCALE_ROOM, STEP = 2 * TILE;           // a step: two tiles
    static constexpr int COPIES = 2 * (CODES / 1024 + SCALE_ROOM / 256);       // of a step
    static constexpr int RING = DIM == 64 ? 4 : 2;                             // steps under way
    static constexpr int RESULT = 16 * (DIM + 4);                              // a wave's sums of 16 rows, fp32
    static constexpr int WAVE = RING * STEP > 4 * RESULT ? RING * STEP : 4 * RESULT;
};

template <typename T, int DIM, int GROUP, int R>
__global__ void __launch_bounds__(256, DIM == 256 ? (GROUP == 32 ? 1 : 2) : 3) qattn_kernel(QattnArgs A, int tiles, int parts, int chunk, int slots, bool packed)
{
    typedef Shape<DIM, GROUP, R> S;
    constexpr int G = S::GROUPS, U = DIM / 32, TILES = DIM / 16;
    __shared__ __align__(16) uint8_t lds[4 * S::WAVE];
    static_assert(sizeof(lds) <= 81920, "two workgroups to a CU");
    const int per = A.q_heads / A.c.heads;
    const int kv = blockIdx.x % A.c.heads;
    int rest = blockIdx.x / A.c.heads;
    int part, b, row_tile, slot = 0;
    if (packed) {
        part = rest % parts;
        if (!find_tile(A.batch, tiles, rest / parts, [&](int i) { return tiles_of(A, i, 16 * R); }, b, row_tile))
            return;
    } else {
        row_tile = rest % tiles;
        rest /= tiles;
        if (slots) {
            Share s;
            if (!Shared(A, slots).find(rest, s, part))
                return;
            b = s.b, slot = s.first + part, parts = s.parts, chunk = s.chunk;
        } else {
            part = rest % parts;
            b = rest / parts;
        }
    }
    const Sequence seq = sequence(A, b);
    const int first_row = row_tile * 16 * R, rows = seq.n * per;
    if (first_row >= rows)
        return;
    const int limit = seen_by(seq, 16 * R, first_row, per), start = part * chunk, end = start + min(chunk, limit - start);
    if (part && start >= limit)
        return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    uint8_t *ring = lds + wave * S::WAVE;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_addr(ring));
    const int32_t *table = A.tables + b * A.ld_table;

    // copies of the step at token t into the ring's place `at`; bits 0 and 1: the tiles' pages are none of the cache's
    const int last_tile = (limit - 1) >> 4;
    uint32_t code_at[S::CODES / 1024], scale_at[S::SCALE_ROOM / 256];
#pragma unroll
    for (int i = 0; i < S::CODES / 1024; ++i) {
        const int o = i * 1024 + lane * 16;
        code_at[i] = o < 8 * DIM ? o : o - 8 * DIM + A.c.page * (DIM / 2);
    }
#pragma unroll
    for (int i = 0; i < S::SCALE_ROOM / 256; ++i) {
        const int o = i * 256 + lane * 4 < S::SCALES ? i * 256 + lane * 4 : 0;
        scale_at[i] = A.c.page * DIM + (o < 32 * G ? o : o - 32 * G + A.c.page * (2 * G));
    }
    const int page_log = __builtin_ctz(A.c.page);
    auto copy = [&](int t, int at) -> uint32_t {
        uint32_t bad = 0;
        const int firsts[2] = {min(t >> 4, last_tile) * 16, min((t >> 4) + 1, last_tile) * 16};
        int pages[2];
        scalar_loads(table, 4 * (firsts[0] >> page_log), 4 * (firsts[1] >> page_log), pages[0], pages[1]);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const bool known = (unsigned)pages[half] < (unsigned)A.c.pages;
            bad |= known ? 0u : 1u << half;
            const int in = firsts[half] & (A.c.page - 1);
            const uint8_t *block = A.cache + ((long long)(known ? pages[half] : 0) * A.c.heads + kv) * A.c.block_bytes;
            const uint32_t to = ring_at + at * S::STEP + half * S::TILE;
            // (the keys' and values' codes of a tile are DIM / 2 bytes a token each, their scales 2 G)
#pragma unroll
            for (int i = 0; i < S::CODES / 1024; ++i)
                copy16(block + in * (DIM / 2), code_at[i], to + i * 1024);
#pragma unroll
            for (int i = 0; i < S::SCALE_ROOM / 256; ++i)
                copy4(block + in * (2 * G), scale_at[i], to + S::CODES + i * 256);
        }
        return bad;
    };

    uint32_t bads = 0;   // two bits per step in flight, the next one lowest
    const int t_first = start + 32 * wave;
#pragma unroll
    for (int i = 0; i < S::RING; ++i)
        if (t_first + 128 * i < end)
            bads |= copy(t_first + 128 * i, i) << (2 * i);

    // queries as operands, the sign of the scale with them; rows past the last are zeros
    u32x4 q[R][U];
    int seen[R];
    const uint32_t flip = A.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int row = first_row + 16 * k + r, i = row / per;
        seen[k] = row < rows ? seq.length - seq.n + 1 + i : 0;
        const T *p = (const T *)A.q + (seq.begin + i) * A.q_token + (kv * per + row % per) * A.q_head + 8 * g;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            typedef T V __attribute__((ext_vector_type(8), aligned(2)));
            u32x4 w = {0, 0, 0, 0};
            if (row < rows)
                w = __builtin_bit_cast(u32x4, *(const V *)(p + 32 * u));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                q[k][u][e] = w[e] ^ flip;
        }
    }
    const int seen_least = seq.length - seq.n + 1 + first_row / per;
    // (a scale of 0 would make -infinity * 0 of hidden scores; the least number above it leaves every finite score below 2^-20)
    const float scale = fmaxf(fabsf(A.scale) * LOG2E, 0x1p-149f);
    uint32_t mask = Code<T>::MASK, base = Code<T>::BASE;
    asm("" : "+s"(mask));
    asm("" : "+v"(base));
    const u32x4 off = {Code<T>::OFF, Code<T>::OFF, Code<T>::OFF, Code<T>::OFF};

    // what a group's offset adds to the scores of row set k, whatever the tokens; kept where the registers hold it (1% faster)
    constexpr bool KEPT = R * G <= 4;
    auto offset = [&](int k, int j) {
        f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = j * (GROUP / 32); u < (j + 1) * (GROUP / 32); ++u)
            d = mfma16(off, q[k][u], d, T());
        return d;
    };
    f32x4 kept[KEPT ? R : 1][KEPT ? G : 1];
    if constexpr (KEPT)
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int j = 0; j < G; ++j)
                kept[k][j] = offset(k, j);

    f32x4 o[R][TILES];
    float ref[R], total[R];
    auto clear = [&] {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            ref[k] = -INFINITY;
            total[k] = 0.f;
#pragma unroll
            for (int i = 0; i < TILES; ++i)
                o[k][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    clear();
    float low = 0.f;   // by which the reference is above the largest score

    int at = 0;
    for (int t = t_first; t < end; t += 128) {
        // the steps behind this one may be under way
        const int behind = (end - 1 - t) / 128;
        if (behind >= S::RING - 1)
            wait_vmcnt<(S::RING - 1) * S::COPIES>();
        else if (S::RING > 2 && behind == 2)
            wait_vmcnt<2 * S::COPIES>();
        else if (behind == 1)
            wait_vmcnt<S::COPIES>();
        else
            wait_vmcnt<0>();
        const uint8_t *step = ring + at * S::STEP;
        uint32_t kc[2][U], vc[2][U], ks[2][2 * G], vs[2][2 * G];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint8_t *tile = step + half * S::TILE;
            load_words<U>(tile + r * (DIM / 2) + g * (DIM / 8), kc[half]);
            load_words<U>(tile + 8 * DIM + g * (2 * DIM) + r * (DIM / 8), vc[half]);
            load_words<2 * G>(tile + S::CODES + g * (8 * G), ks[half]);
            load_words<2 * G>(tile + S::CODES + 32 * G + g * (8 * G), vs[half]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const uint32_t bad = bads & 3;
        bads >>= 2;
        if (t + 128 * S::RING < end)
            bads |= copy(t + 128 * S::RING, at) << (2 * (S::RING - 1));
        at = at + 1 == S::RING ? 0 : at + 1;

        // scale i of group j in words of two
        const auto number = [](const uint32_t *w, int token, int group) {
            const int i = token * G + group;
            return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        };
        const bool masked = t + 32 > seen_least || bad;
        float s[R][8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            u32x4 key[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t w = kc[half][u];
                key[u] = u32x4{widen<T, 0>(w, mask, base), widen<T, 1>(w, mask, base), widen<T, 2>(w, mask, base), widen<T, 3>(w, mask, base)};
            }
#pragma unroll
            for (int k = 0; k < R; ++k)
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    f32x4 d = KEPT ? kept[KEPT ? k : 0][KEPT ? j : 0] : offset(k, j);
#pragma unroll
                    for (int u = j * (GROUP / 32); u < (j + 1) * (GROUP / 32); ++u)
                        d = mfma16(key[u], q[k][u], d, T());
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float f = number(ks[half], i, j);
                        s[k][4 * half + i] = j ? __builtin_fmaf(d[i], f, s[k][4 * half + i]) : d[i] * f;
                    }
                }
        }
        if (masked) {
            asm volatile("");   // a branch: as selects the step would be a tenth longer
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int token = t + 16 * half + 4 * g + i;
#pragma unroll
                    for (int k = 0; k < R; ++k)
                        s[k][4 * half + i] = token < seen[k] ? (bad >> half & 1 ? NAN : s[k][4 * half + i]) : -INFINITY;
                    // what lies behind the sequence's end may be any scale
                    if (token >= (R == 1 ? seen[0] : limit)) {
                        if constexpr (G > 1) {
#pragma unroll
                            for (int j = 0; j < G / 2; ++j)
                                vs[half][i * (G / 2) + j] = 0;
                        } else {
                            vs[half][i / 2] &= i & 1 ? 0xFFFFu : 0xFFFF0000u;
                        }
                    }
                }
        }
        // of each token the exponent of its largest value scale that is a number (for 32 sequences of 8192 one for each lane's eight would be 2 to
        // 7% faster, but takes the bits of small values next to large ones that weigh little or are hidden)
        float size[8];
        if constexpr (Code<T>::NARROW) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // without its sign, and with a carry that takes infinity and NaN below all numbers: the exponent + 128 in bits 8 to 15
                    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
                    uint32_t top = 0;
#pragma unroll
                    for (int j = i * G / 2; j <= ((i + 1) * G - 1) / 2; ++j) {
                        const u16x2 x = __builtin_bit_cast(u16x2, vs[half][j]) * (unsigned short)2 + (unsigned short)0x100;
                        top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, __builtin_bit_cast(u16x2, top)));
                    }
                    const float low = (float)(top >> 8 & 255u), high = (float)(top >> 24), e = G == 1 ? (i & 1 ? high : low) : fmaxf(low, high);
                    // (weights of values that T rounds to 0 need not be near 1, and their sum has to stay a number; scales that qcache_write makes
                    // are below 2^126, and a weight of 2^-127 would be 0)
                    size[4 * half + i] = __builtin_amdgcn_fmed3f(e - 128.f, -40.f, 125.f);
                }
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            // the largest weight, or product of a weight and a scale
            float top;
            if constexpr (Code<T>::NARROW) {
                top = __builtin_fmaf(s[k][0], scale, size[0]);
#pragma unroll
                for (int i = 1; i < 8; ++i)
                    top = fmaxf(top, __builtin_fmaf(s[k][i], scale, size[i]));
            } else {
                top = s[k][0];
#pragma unroll
                for (int i = 1; i < 8; ++i)
                    top = fmaxf(top, s[k][i]);
                top *= scale;
            }
            // weights up to 2^8 are as good as up to 1: the reference moves seldom
            if (__builtin_amdgcn_ballot_w64(top > ref[k] + (8.f - low))) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float next = fmaxf(ref[k], top + low), fade = next == -INFINITY ? 1.f : exp2_fast(ref[k] - next);
                ref[k] = next;
                total[k] *= fade;
#pragma unroll
                for (int i = 0; i < TILES; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[k][i][e] *= fade;
            }
            const float zero = ref[k] == -INFINITY ? 0.f : -ref[k];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[k][i] = exp2_fast(__builtin_fmaf(s[k][i], scale, zero));
                total[k] += s[k][i];
            }
        }
        static_for<G>([&](auto group) {
            constexpr int J = decltype(group)::value;
            u32x4 p[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                float w[8];
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[4 * half + i] = s[k][4 * half + i] * number(vs[half], i, J);
                        // (a scale that one row sees and another does not may be no number)
                        if (R > 1 && masked && t + 16 * half + 4 * g + i >= seen[k])
                            w[4 * half + i] = 0.f;
                    }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    p[k][i] = pack2<T>(w[2 * i], w[2 * i + 1]);
            }
            static_for<GROUP / 16>([&](auto i) {
                constexpr int tile = J * (GROUP / 16) + decltype(i)::value, h = tile / 4, n = tile % 4;
                const u32x4 value = {widen<T, n>(vc[0][2 * h], mask, base), widen<T, n>(vc[0][2 * h + 1], mask, base), widen<T, n>(vc[1][2 * h], mask, base),
                                     widen<T, n>(vc[1][2 * h + 1], mask, base)};
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    o[k][tile] = mfma16(off, p[k], o[k][tile], T());
                    o[k][tile] = mfma16(value, p[k], o[k][tile], T());
                }
            });
        });
        // bf16: sums of weights up to 2^8 by codes and offsets up to 2^8 can pass the largest number where their values and the result do not
        // (or do so where waves and parts are added). Then once more, with weights up to 2^-40.
        if constexpr (!Code<T>::NARROW)
            if (t + 128 >= end && low == 0.f) {
                uint32_t largest = 0;   // magnitude; infinity and NaN are above all numbers
#pragma unroll
                for (int k = 0; k < R; ++k)
#pragma unroll
                    for (int i = 0; i < TILES; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            largest = max(largest, __float_as_uint(o[k][i][e]) & 0x7FFFFFFFu);
                if (__builtin_amdgcn_ballot_w64(largest >= __float_as_uint(0x1p100f))) {
                    low = 48.f;
                    clear();
                    at = 0;
                    bads = 0;
#pragma nounroll
                    for (int i = 0; i < S::RING; ++i)
                        if (t_first + 128 * i < end)
                            bads |= copy(t_first + 128 * i, i) << (2 * i);
                    t = t_first - 128;
                }
            }
    }

    // join the waves, 16 rows at a time: [row][DIM] sums, then references and totals
    float *sums = (float *)ring;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        __syncthreads();
        total[k] += __shfl_xor(total[k], 16);
        total[k] += __shfl_xor(total[k], 32);
#pragma unroll
        for (int i = 0; i < TILES; ++i)
            *(f32x4 *)(sums + r * (DIM + 4) + 16 * i + 4 * g) = o[k][i];
        if (g == 0) {
            sums[r * (DIM + 4) + DIM] = ref[k];
            sums[r * (DIM + 4) + DIM + 1] = total[k];
        }
        __syncthreads();
        constexpr int LANES = DIM / 4;   // of a row
        for (int i = threadIdx.x; i < 16 * LANES; i += 256) {
            const int row = first_row + 16 * k + i / LANES, c = i % LANES * 4, from = i / LANES * (DIM + 4);
            if (row >= rows)
                break;
            float most = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                most = fmaxf(most, ((const float *)(lds + w * S::WAVE))[from + DIM]);
            const float base = most == -INFINITY ? 0.f : most;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float *p = (const float *)(lds + w * S::WAVE) + from;
                const float f = exp2_fast(p[DIM] - base);
                const f32x4 v = *(const f32x4 *)(p + c);
                l += f * p[DIM + 1];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum[e] += f * v[e];
            }
            const int query = seq.begin + row / per, head = kv * per + row % per;
            if (parts == 1) {
                const float inverse = l != 0.f ? 1.f / l : 0.f;
                typedef T V __attribute__((ext_vector_type(4), aligned(2)));
                V v;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = (T)(sum[e] * inverse);
                *(V *)((T *)A.y + query * A.y_token + head * A.y_head + c) = v;
            } else {
                const long long id = slots ? ((long long)slot * A.max_queries + row / per) * A.q_heads + head : ((long long)query * A.q_heads + head) * parts + part;
                *(f32x4 *)(A.part + id * DIM + c) = sum;
                if (c == 0) {
                    float *stat = A.part + part_rows(A, slots, parts) * DIM + 2 * id;
                    stat[0] = most;
                    stat[1] = l;
                }
            }
        }
    }
}

// query i of sequence b
template <typename T, int WAVES>
__device__ __forceinline__ void join_row(JoinScratch<WAVES> &lds, const QattnArgs &A, const Sequence &seq, const Share &s, int i, int head, int rows, int parts,
                                         int slots)
{
    // the parts that its workgroups' rows have
    const int per = A.q_heads / A.c.heads, first_row = (i * per + head % per) / rows * rows;
    const int limit = seen_by(seq, rows, first_row, per), used = parts_of(limit, s.chunk);
    const long long query = seq.begin + i, step = slots ? (long long)A.max_queries * A.q_heads : 1;
    const long long row = slots ? ((long long)s.first * A.max_queries + i) * A.q_heads + head : (query * A.q_heads + head) * parts;
    join_parts<T, WAVES>(lds, A.part + row * A.c.dim, A.part + part_rows(A, slots, parts) * A.c.dim + 2 * row, step, used, A.c.dim,
                         (T *)A.y + query * A.y_token + head * A.y_head);
}

template <typename T, int WAVES>
__global__ void __launch_bounds__(256) qattn_join_kernel(QattnArgs A, int rows, int parts, int chunk, int slots)
{
    __shared__ JoinScratch<WAVES> lds;
    const int at = WAVES > 1 ? blockIdx.x : blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= A.batch * A.max_queries * A.q_heads)
        return;
    const int head = at % A.q_heads, i = at / A.q_heads % A.max_queries, b = at / A.q_heads / A.max_queries;
    Share s = {b, chunk, 0, parts, 0};
    if (slots) {
        if (length_of(A, b) <= LEAST)
            return;   // one part, in y
        s = Shared(A, slots).of(b);
        if (s.parts == 1)
            return;
    }
    const Sequence seq = sequence(A, b);
    if (i < seq.n)
        join_row<T, WAVES>(lds, A, seq, s, i, head, rows, parts, slots);
}

// the same where row tiles are packed: a workgroup has those of one tile and key head, a wave every fourth row
template <typename T>
__global__ void __launch_bounds__(256) qattn_join_packed_kernel(QattnArgs A, int tiles, int rows, int parts, int chunk)
{
    __shared__ JoinScratch<1> lds;
    int b, row_tile;
    if (!find_tile(A.batch, tiles, blockIdx.x / A.c.heads, [&](int i) { return tiles_of(A, i, rows); }, b, row_tile))
        return;
    const Sequence seq = sequence(A, b);
    const int per = A.q_heads / A.c.heads, kv = blockIdx.x % A.c.heads, end = min((row_tile + 1) * rows, seq.n * per);
    for (int row = row_tile * rows + (threadIdx.x >> 6); row < end; row += 4)
        join_row<T, 1>(lds, A, seq, {b, chunk, 0, parts, 0}, row / per, kv * per + row % per, rows, parts, 0);
}

int row_tiles(const QattnArgs &a, int rows) { return (a.max_queries * (a.q_heads / a.c.heads) + rows - 1) / rows; }
// Row tiles that `queries` rows of sequences together can have, each but one of a sequence full; with those of the longest one for each where
// that is a quarter more, a launch is packed (2000 tokens each: 512 queries of one sequence and one of 63 others 106 us, 203 otherwise,
// with 32 rows a workgroup; 62 with 16).
long long most_tiles(const QattnArgs &a, int rows) { return (long long)a.queries * (a.q_heads / a.c.heads) / rows + a.batch; }
bool packed(const QattnArgs &a, int rows) { return 4LL * a.batch * row_tiles(a, rows) > 5 * most_tiles(a, rows); }
// Rows of a workgroup: 32 of dim 64 where there are as many (8 queries each over 32 sequences of 8192, 32 query heads on 8: 62 us, 66 with 16;
// dim 128 98 and 97, dim 256 253 and 183, where 32 rows leave one workgroup on a CU).
int rows_of(const QattnArgs &a) { return a.c.dim == 64 && a.max_queries * (a.q_heads / a.c.heads) > 16 ? 32 : 16; }

template <typename T, int DIM, int GROUP, int R>
hipError_t launch_rows(const QattnArgs &a, const AttnPlan &p, hipStream_t stream)
{
    const int tiles = row_tiles(a, 16 * R);
    const bool few = packed(a, 16 * R);
    const dim3 grid((unsigned)(a.c.heads * (few ? most_tiles(a, 16 * R) * p.parts : (long long)tiles * (p.slots ? p.slots : p.parts * a.batch))));
    hipLaunchKernelGGL((qattn_kernel<T, DIM, GROUP, R>), grid, dim3(256), 0, stream, a, tiles, p.parts, p.chunk, p.slots, few);
    return hipGetLastError();
}

template <typename T, int DIM, int GROUP>
hipError_t launch_group(const QattnArgs &a, const AttnPlan &p, hipStream_t stream)
{
    if constexpr (DIM == 64)
        if (rows_of(a) == 32)
            return launch_rows<T, DIM, GROUP, 2>(a, p, stream);
    return launch_rows<T, DIM, GROUP, 1>(a, p, stream);
}

template <typename T, int DIM>
hipError_t launch_dim(const QattnArgs &a, const AttnPlan &p, hipStream_t stream)
{
    if constexpr (DIM >= 128)
        if (a.c.group == 128)
            return launch_group<T, DIM, 128>(a, p, stream);
    return a.c.group == 32 ? launch_group<T, DIM, 32>(a, p, stream) : launch_group<T, DIM, 64>(a, p, stream);
}

template <typename T>
hipError_t launch_type(const QattnArgs &a, const AttnPlan &p, hipStream_t stream)
{
    const hipError_t e = a.c.dim == 64    ? launch_dim<T, 64>(a, p, stream)
                         : a.c.dim == 128 ? launch_dim<T, 128>(a, p, stream)
                                          : launch_dim<T, 256>(a, p, stream);
    if (e != hipSuccess || (p.parts == 1 && !p.slots))
        return e;
    const unsigned all = (unsigned)a.batch * a.max_queries * a.q_heads;
    const int rows = rows_of(a);
    if (packed(a, rows))
        hipLaunchKernelGGL((qattn_join_packed_kernel<T>), dim3((unsigned)(a.c.heads * most_tiles(a, rows))), dim3(256), 0, stream, a, row_tiles(a, rows), rows,
                           p.parts, p.chunk);
    else if (p.parts <= JOIN_FEW)
        hipLaunchKernelGGL((qattn_join_kernel<T, 1>), dim3((all + 3) / 4), dim3(256), 0, stream, a, rows, p.parts, p.chunk, p.slots);
    else
        hipLaunchKernelGGL((qattn_join_kernel<T, 4>), dim3(all), dim3(256), 0, stream, a, rows, p.parts, p.chunk, p.slots);
    return hipGetLastError();
}

}  // namespace

AttnPlan qattn_plan(const QattnArgs &a, size_t room)
{
    const int keys = (int)std::min<long long>(a.max_keys, a.ld_table * a.c.page);
    const int rows = rows_of(a);
    const long long groups = a.c.heads * (packed(a, rows) ? most_tiles(a, rows) : (long long)a.batch * row_tiles(a, rows));
    // Three workgroups to a CU, of 128 tokens at a time, and as many rounds of them as there are sequences, up to four, since one may have
    // all the tokens: one of 120000 34 us in one round, 41 in four; 64000 and 7 of 300 49 in one round, 27 in four; 3 of 40000 34 and 38.
    // But none below 256 tokens unless one round holds all of 128 (1 of 1500 9.3 us with 128, 10.0 with 256; 16 of up to 2500, four
    // tokens each: 18.0 and 16.1).
    constexpr int ROUND = 768;
    const int least = groups * ((keys + 127) / 128) <= ROUND ? 128 : LEAST;
    long long parts = std::max(1LL, std::min<long long>(std::min(a.batch, 4) * ROUND / groups, (keys + least - 1) / least));
    const long long one = (long long)a.queries * a.q_heads * (a.c.dim + 2) * 4;
    parts = std::min(parts, (long long)room / std::max(one, 1LL));
    parts = std::max(parts, 1LL);
    const long long chunk = ((keys + parts - 1) / parts + 127) / 128 * 128;
    parts = (keys + chunk - 1) / std::max(chunk, 1LL);
    // More than 8 sequences share two rounds by their lengths: 120000 tokens and 63 of 500 45 us, 149 with the same number of parts for each;
    // 30000 and 31 of 1000 28 and 39; 64 of 8192 113 and 119, of 700 to 8192 70 and 69; 20000 and 199 of 300 35 and 146 (not split
    // otherwise; with less than 4096 tokens they are not: 200 of 1000 51 and 42). Where parts are the least anyway, and of few
    // sequences, the search costs more than it gives: 16 of up to 2500, four queries each, 17.2 and 14.2; 64000 and 7 of 300 29 and 27. (One
    // round: 44, 25, 110, 78; three: 48, 33, 118, 66.)
    if (!packed(a, rows) && a.batch > 8 && a.batch <= SHARED && groups / a.batch <= ROUND && least == LEAST && chunk > LEAST && (parts > 1 || keys >= 4096) &&
        (long long)a.batch * keys / 128 < INT32_MAX / 2) {
        const long long each = (long long)a.max_queries * a.q_heads * (a.c.dim + 2) * 4;
        const long long slots = std::min(std::max(2 * ROUND / (groups / a.batch), a.batch + 64LL), (long long)room / each);
        if (slots >= a.batch + 16)
            return {(int)(slots / a.batch), (int)chunk, (size_t)(each * slots), (int)slots};
    }
    if (parts <= 1)
        return {1, (keys + 127) / 128 * 128, 0, 0};
    return {(int)parts, (int)chunk, (size_t)(one * parts), 0};
}

hipError_t launch_qattn(const QattnArgs &a, const AttnPlan &plan, hipStream_t stream)
{
    return a.type == AQD_F16 ? launch_type<_Float16>(a, plan, stream) : launch_type<__bf16>(a, plan, stream);
}

}  // namespace aqd
