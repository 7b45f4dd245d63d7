// Attention over keys and values of packed sequences. Definition: include/aqd.h.
//
// A workgroup has one sequence, one key head, 128 rows (queries times the query heads of the key head, a query's heads next to
// one another) and a range of keys. Each of its four waves has 32 rows. S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16 products: the
// lane that has the scores of row r and tokens 4 h .. 4 h + 3 and so on is the lane that gives those weights to the
// second product, so weights stay where they are. Q is in registers, tiles of K and V are copied straight into
// a ring in LDS, in an order of their 16-byte pieces that leaves the reads without bank conflicts; V's columns come out of LDS
// by the transposing read. Two workgroups share a CU (three of dim 64, one of 256): one's copies, waits and stores are under the
// other's products.
//
// A step of 32 keys has three parts that do not wait for one another: the scores of the next step and the sums of the
// last one on the matrix cores, the weights of this one on the vector units (a running softmax whose reference moves
// only when the sixteen weights that a lane has of a step sum up to more than 2^12).
//
// Weights are rounded to T for the second product, and summed up as rounded: in fp32 each product would be one of two, a third more of all. Against
// 64 bits the error is 0.0020 of the result's norm, 0.0016 with fp32 weights (bf16, 17 prompts of 40 to 2048; fp16, 100 over 1337:
// 0.00027 and 0.00021); the rounding of the result is 0.0016 of it.
//
// Bound by what the matrix cores and the vector units can issue together: a prompt of 16384, 32 query heads on 8, dim 128, bf16, causal
// takes 2.25 ms, 970 TFLOP/s (a library product of 8192^3 1158), with the matrix cores busy 44% of the cycles, the vector units 51%
// and no bank conflicts. Prompts of 2048 reach 730 TFLOP/s, of 512 430: a workgroup's start (its lengths, queries and first tiles, 4 us) and
// end (3 us) are as long as 10 of its steps. 64 rows a wave do not fit the registers.
//
// The weights of hidden keys are 0, but 0 times an infinity or a NaN is not: rows whose result is no number are done
// again one by one with nothing hidden in their sums. So are those whose sums pass the largest number, or, of split keys, 2^100, as up to
// 128 parts are added. That costs: a prompt of 2048 (32 query heads on 8, dim 128) takes 30 ms where the rows of one wave see a NaN, and 33 where
// all do, for 72 us.

#include <algorithm>

#include "attn_row.h"

namespace aqd {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c, __bf16)
{
    typedef Operand<__bf16>::type V;
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c, _Float16)
{
    typedef Operand<_Float16>::type V;
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}

// 16 bytes of LDS at byte address `at`
__device__ __forceinline__ u32x4 read_piece(uint32_t at)
{
    return *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)at;
}
// Of each 16 lanes, lane 4 i + j has the LDS byte address of 4 numbers of row i; lane c of them gets number c % 4 of lanes
// c / 4, 4 + c / 4, 8 + c / 4 and 12 + c / 4: a column of the four rows.
__device__ __forceinline__ u32x2 read_columns(uint32_t at)
{
    typedef short V __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) V *)(uintptr_t)at));
}

constexpr int ROWS = 128;   // of a workgroup

template <int DIM>
struct Tile {
    static constexpr int KEYS = 32;                                          // of a tile
    static constexpr int ROW = 2 * DIM, PIECES = DIM / 8;                    // bytes and 16-byte pieces of a row
    static constexpr int SIDE = KEYS * ROW, RING = 4;
    static constexpr int COPIES = SIDE / 4096;                               // of a wave, for keys or values of a tile
    static constexpr int LDS = 2 * RING * SIDE;
    // where piece c of row t stands: 16 rows' pieces at one c are in different banks, and so are 64 bytes of 4 rows
    static __device__ __forceinline__ int key_place(int t, int c) { return DIM == 64 ? c ^ (t >> 1 & 7) : c ^ (t & 15); }
    static __device__ __forceinline__ int value_place(int t, int c) { return DIM == 64 ? c ^ (t << 1 & 4) : c ^ (t << 2 & 12); }
};

struct Span2 {
    int begin, n, first, m;   // queries and keys
};
__device__ __forceinline__ Span2 sequence(const AttnArgs &A, int b)
{
    Span2 s;
    s.begin = min(max(A.q_start[b], 0), A.queries);
    s.n = min(min(max(A.q_start[b + 1], 0), A.queries) - s.begin, A.max_queries);
    s.first = min(max(A.k_start[b], 0), A.keys);
    s.m = max(min(max(A.k_start[b + 1], 0), A.keys) - s.first, 0);
    return s;
}
__device__ __forceinline__ int seen_by(const AttnArgs &A, const Span2 &s, int query)
{
    return A.causal ? max(s.m - s.n + 1 + query, 0) : s.m;
}

// DIRECT: rows of keys and values start at multiples of 4 bytes. tiles: of the longest sequence
template <typename T, int DIM, bool DIRECT>
__global__ void __launch_bounds__(256, DIM == 64 ? 3 : DIM == 128 ? 2 : 1) attn_kernel(AttnArgs A, int tiles, int parts, int chunk, bool packed)
{
    typedef Tile<DIM> S;
    constexpr int U = DIM / 16, C = DIM / 32;
    __shared__ __align__(16) uint8_t lds[S::LDS];
    const int per = A.q_heads / A.heads;
    int rest = blockIdx.x;
    const int kv = rest % A.heads;
    rest /= A.heads;
    // the rows with most keys first
    int part = 0, row_tile, b;
    if (packed) {
        if (!find_tile(A.batch, tiles, rest, [&](int i) { return (max(sequence(A, i).n, 0) * per + ROWS - 1) / ROWS; }, b, row_tile))
            return;
    } else {
        b = rest % A.batch;
        rest /= A.batch;
        part = rest % parts;
        row_tile = tiles - 1 - rest / parts;
    }
    const Span2 seq = sequence(A, b);
    const int rows = seq.n * per, first_row = row_tile * ROWS;
    if (first_row >= rows)
        return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    const int limit = seen_by(A, seq, min((first_row + ROWS - 1) / per, seq.n - 1)), start = part * chunk;
    // (a sequence may have more keys than max_keys: the last part takes them all)
    const int end = part + 1 < parts ? start + min(chunk, limit - start) : limit;
    if (part && start >= limit)
        return;
    const int wave_row = first_row + 32 * wave;
    // keys of the wave's last row; none for rows past the last one
    const int wave_end = wave_row < rows ? min(end, seen_by(A, seq, min((wave_row + 32 - 1) / per, seq.n - 1))) : 0;
    const int seen_least = seen_by(A, seq, min(wave_row / per, seq.n - 1));
    const uint8_t *key_base = (const uint8_t *)((const T *)A.k + seq.first * A.k_token + kv * A.k_head);
    const uint8_t *value_base = (const uint8_t *)((const T *)A.v + seq.first * A.v_token + kv * A.v_head);

    // 16-byte piece i of a wave's share of a tile: row, channels, and offset from the tile's first row
    const int dim_pieces = A.dim / 8;
    const long long key_stride = 2 * A.k_token, value_stride = 2 * A.v_token;
    uint32_t key_from[S::COPIES], value_from[S::COPIES];
#pragma unroll
    for (int i = 0; i < S::COPIES; ++i) {
        const int piece = (wave * S::COPIES + i) * 64 + lane, row = piece / S::PIECES, place = piece % S::PIECES;
        key_from[i] = (uint32_t)row * (uint32_t)key_stride + 16 * S::key_place(row, place);
        value_from[i] = (uint32_t)row * (uint32_t)value_stride + 16 * S::value_place(row, place);
    }
    const uint32_t lds_at = __builtin_amdgcn_readfirstlane(lds_addr(lds));
    auto copy_side = [&](bool values, int tile, int slot) {
        const int to = (values ? S::RING : 0) * S::SIDE + slot * S::SIDE;
        const uint8_t *base = (values ? value_base : key_base) + (long long)(start + tile * S::KEYS) * (values ? value_stride : key_stride);
        const int last = end - 1 - (start + tile * S::KEYS);   // row of the tile
        const long long stride = values ? value_stride : key_stride;
        int at = lane;
        if (last < S::KEYS - 1 || A.dim < DIM || !DIRECT)
            asm volatile("" : "+v"(at));   // (or what it takes below would take registers all the time)
#pragma unroll
        for (int i = 0; i < S::COPIES; ++i) {
            const int first = (wave * S::COPIES + i) * 64, row = (first + at) / S::PIECES, place = (first + at) % S::PIECES;
            const int c = values ? S::value_place(row, place) : S::key_place(row, place);
            uint32_t from = values ? value_from[i] : key_from[i];
            // rows past the end are the last one again
            if (last < S::KEYS - 1)
                from = (uint32_t)min(row, last) * (uint32_t)stride + 16 * c;
            if (A.dim < DIM && c >= dim_pieces)
                continue;
            if constexpr (DIRECT) {
                copy16(base, from, lds_at + to + first * 16);
            } else {
                typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2)));
                *(u32x4 *)(lds + to + (first + at) * 16) = *(const V *)(base + from);
            }
        }
    };
    const int count = (end - start + S::KEYS - 1) / S::KEYS;   // tiles
    // The first step has no weights before it: zeros times zeros, the values of a tile before the first. Channels past the last are
    // never copied.
    for (int i = (A.dim < DIM ? 0 : (2 * S::RING - 1) * S::SIDE / 16) + threadIdx.x; i < S::LDS / 16; i += 256)
        ((u32x4 *)lds)[i] = u32x4{0, 0, 0, 0};
    if (A.dim < DIM)
        __syncthreads();

    // in the order in which the tiles are waited for
    if (count > 0) {
        copy_side(false, 0, 0);
        copy_side(true, 0, 0);
    }
    if (count > 1) {
        copy_side(false, 1, 1);
        copy_side(true, 1, 1);
    }
    if (count > 2)
        copy_side(false, 2, 2);

    // queries as operands, the sign of the scale with them
    u32x4 q[U];
    const uint32_t flip = A.scale < 0.f ? 0x80008000u : 0u;
    int seen;   // keys
    {
        const int row = wave_row + r, query = seq.begin + row / per, head = kv * per + row % per;
        seen = row < rows ? seen_by(A, seq, row / per) : 0;
        const T *p = (const T *)A.q + query * A.q_token + head * A.q_head + 8 * h;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            typedef T V __attribute__((ext_vector_type(8), aligned(2)));
            u32x4 w = {0, 0, 0, 0};
            if (row < rows && 16 * u + 8 * h < A.dim)
                w = __builtin_bit_cast(u32x4, *(const V *)(p + 16 * u));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                q[u][e] = w[e] ^ flip;
        }
    }
    // (a scale of 0 would make -infinity * 0 of hidden scores; the least number above it leaves every finite score below 2^-20)
    const float scale = fmaxf(fabsf(A.scale) * LOG2E, 0x1p-149f);

    f32x16 o[C], s[2];   // sums, and the scores of this step and the next
    u32x4 p[2];          // the last step's weights
    float ref = -INFINITY, total = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            o[c][e] = 0.f;
    p[0] = p[1] = u32x4{0, 0, 0, 0};
    // LDS addresses of the lane's pieces in the first tile of keys and of values: other tiles, rows and half rows are constants away.
    // (The compiler would make each from the lane's number again.)
    constexpr int KEY_AT = U < 8 ? U : 8, VALUE_AT = C < 4 ? C : 4;
    uint32_t key_at[KEY_AT], value_at[VALUE_AT];
#pragma unroll
    for (int u = 0; u < KEY_AT; ++u) {
        key_at[u] = lds_at + r * S::ROW + 16 * S::key_place(r, 2 * u + h);
        asm("" : "+v"(key_at[u]));
    }
#pragma unroll
    for (int c = 0; c < VALUE_AT; ++c) {
        // lane 16 a + 4 i + j: row 4 h + i, channels 32 c + 16 (a % 2) + 4 j ..
        const int row = 4 * h + (lane >> 2 & 3), j = lane & 3, piece = 4 * c + 2 * (lane >> 4 & 1) + (j >> 1);
        value_at[c] = lds_at + S::RING * S::SIDE + row * S::ROW + 16 * S::value_place(row, piece) + 8 * (j & 1);
        asm("" : "+v"(value_at[c]));
    }
    // of the tiles at a place in the ring: 16 channels of the keys, and the operand of product i of 2 C of the values
    auto key = [&](int place, int u) { return read_piece(key_at[u % KEY_AT] + place * S::SIDE + u / KEY_AT * 256); };
    auto value = [&](int place, int i) {
        const int v = i / C, c = i % C;
        const uint32_t at = value_at[c % VALUE_AT] + place * S::SIDE + c / VALUE_AT * 256 + 16 * v * S::ROW;
        const u32x2 x = read_columns(at), y = read_columns(at + 8 * S::ROW);
        return u32x4{x[0], x[1], y[0], y[1]};
    };
    // hides the scores that the row does not see, keys t .. + 31
    auto hide = [&](int t, f32x16 &s) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            s[e] = t + (e & 3) + 8 * (e >> 2) + 4 * h < seen ? s[e] : -INFINITY;
    };
    // weights of scores e, e + 1 (as exponents) into p; adds them to sum as rounded
    auto weigh = [&](f32x16 &s, int e, float &sum) {
        p[e / 8][e / 2 % 4] = pack2<T>(exp2_fast(s[e]), exp2_fast(s[e + 1]));
        sum = add2(p[e / 8][e / 2 % 4], sum, T());
    };
    // one step: the next one's scores, the last one's sums, this one's weights, in the order in which they are issued: reads two
    // products ahead, the exponentials of two weights under two matrix instructions
    auto step = [&](int next_place, int last_place, f32x16 &s, f32x16 &next) {
        constexpr int AHEAD = 2;
        u32x4 keys[AHEAD + 1], values[AHEAD + 1];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            keys[u] = key(next_place, u);
            values[u] = value(last_place, u);
        }
        const u32x4 last[2] = {p[0], p[1]};
        const float zero = ref == -INFINITY ? 0.f : -ref;
        float sum = 0.f;
        f32x16 x;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[e] = __builtin_fmaf(s[e], scale, zero);
            next[e] = 0.f;
        }
        __builtin_amdgcn_sched_barrier(0);
        static_assert(U == 2 * C, "products in pairs");
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u + AHEAD < U) {
                keys[(u + AHEAD) % (AHEAD + 1)] = key(next_place, u + AHEAD);
                values[(u + AHEAD) % (AHEAD + 1)] = value(last_place, u + AHEAD);
            }
            next = mfma32(keys[u % (AHEAD + 1)], q[u], next, T());
            o[u % C] = mfma32(values[u % (AHEAD + 1)], last[u / C], o[u % C], T());
#pragma unroll
            for (int e = 16 * u / U; e < 16 * (u + 1) / U; ++e)
                if (e % 2 == 0)
                    weigh(x, e, sum);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the reference need not be the largest score: weights up to 2^12 are as good as up to 1
        if (__builtin_amdgcn_ballot_w64(sum > 4096.f || ref == -INFINITY)) {
            float top = s[0];
#pragma unroll
            for (int e = 1; e < 16; ++e)
                top = fmaxf(top, s[e]);
            top = fmaxf(ref, fmaxf(top, __shfl_xor(top, 32)) * scale);
            const float fade = top == -INFINITY ? 1.f : exp2_fast(ref - top);
            ref = top;
            total *= fade;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    o[c][e] *= fade;
            const float shift = top == -INFINITY ? 0.f : -top;
            sum = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                x[e] = __builtin_fmaf(s[e], scale, shift);
#pragma unroll
            for (int e = 0; e < 16; e += 2)
                weigh(x, e, sum);
        }
        total += sum;
    };

    const int steps = (wave_end - start + 31) / 32;                      // of this wave
    const int open = max(min((seen_least - start) / 32, steps), 0);     // the first of them hide nothing
    // Until keys of the next tile and values of this one have arrived (those of the tile behind may be under way), and no wave
    // reads what is copied now.
    auto arrive = [&](int tile, int far, int last) {
        if (DIRECT && tile + 2 < count)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * S::COPIES) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (tile + 2 < count)
            copy_side(true, tile + 2, far);
        if (tile + 3 < count)
            copy_side(false, tile + 3, last);
    };
    // tile t, at place t % RING of the ring; whether it was the wave's last
    auto run = [&](auto place, int tile, f32x16 &s, f32x16 &next) {
        constexpr int AT = decltype(place)::value, NEXT = (AT + 1) % S::RING, FAR = (AT + 2) % S::RING, LAST = (AT + 3) % S::RING;
        arrive(tile, FAR, LAST);
        if (tile >= open)
            hide(start + 32 * tile, s);
        step(NEXT, LAST, s, next);
        return tile + 1 == steps;
    };
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (steps > 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            s[0][e] = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
            s[0] = mfma32(key(0, u), q[u], s[0], T());
#pragma nounroll
        for (int tile = 0;; tile += 4) {
            if (run(std::integral_constant<int, 0>(), tile, s[0], s[1]) || run(std::integral_constant<int, 1>(), tile + 1, s[1], s[0]) ||
                run(std::integral_constant<int, 2>(), tile + 2, s[0], s[1]) || run(std::integral_constant<int, 3>(), tile + 3, s[1], s[0]))
                break;
        }
    }
    // the other waves' tiles
    int tile = max(steps, 0);
    if (tile < count)
        arrive(tile, (tile + 2) % S::RING, (tile + 3) % S::RING);
    if (steps > 0)
#pragma unroll
        for (int i = 0; i < 2 * C; ++i)
            o[i % C] = mfma32(value((tile + 3) % S::RING, i), p[i / C], o[i % C], T());
    for (++tile; tile < count; ++tile)
        arrive(tile, (tile + 2) % S::RING, (tile + 3) % S::RING);

    total += __shfl_xor(total, 32);
    uint32_t largest = __float_as_uint(total);   // magnitude; infinity and NaN are above all numbers
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            largest = max(largest, __float_as_uint(o[c][e]) & 0x7FFFFFFFu);
    const bool number = largest < __float_as_uint(parts > 1 ? 0x1p100f : INFINITY);
    const float inverse = parts > 1 ? 1.f : total != 0.f ? 1.f / total : 0.f;
    const long long all = (long long)A.queries * A.q_heads;
    int row = wave_row + r;
    asm volatile("" : "+v"(row));   // (made again here, not kept since the start)
    if (__builtin_amdgcn_ballot_w64(!number) == 0 && row < rows) {
        const int query = seq.begin + row / per, head = kv * per + row % per;
        T *y = (T *)A.y + query * A.y_token + head * A.y_head;
        const long long id = ((long long)query * A.q_heads + head) * parts + part;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int channel = 32 * c + 8 * (e / 4) + 4 * h;
                if (channel >= A.dim)
                    continue;
                f32x4 f;
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    f[x] = o[c][e + x] * inverse;
                if (parts > 1) {
                    *(f32x4 *)(A.part + id * A.dim + channel) = f;
                } else {
                    typedef u32x2 V __attribute__((aligned(2)));
                    *(V *)(y + channel) = u32x2{pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3])};
                }
            }
        if (parts > 1 && h == 0) {
            float *stat = A.part + all * parts * A.dim + 2 * id;
            stat[0] = ref;
            stat[1] = total;
        }
    }
    // every wave is done with the ring: those whose rows are no numbers do them again in its memory
    __syncthreads();
    if (__builtin_amdgcn_ballot_w64(!number) == 0)
        return;
    RowScratch &scratch = ((RowScratch *)lds)[wave];
    for (int row = wave_row; row < min(wave_row + 32, rows); ++row) {
        const int i = row / per, query = seq.begin + i, head = kv * per + row % per;
        const T *from = (const T *)A.q + query * A.q_token + head * A.q_head;
        const T *k = (const T *)key_base, *v = (const T *)value_base;
        T *y = (T *)A.y + query * A.y_token + head * A.y_head;
        const long long id = ((long long)query * A.q_heads + head) * parts + part;
        row_attention<DIM>(
            scratch, A.dim, start, min(end, seen_by(A, seq, i)), A.scale, [&](int c) { return (float)from[c]; },
            [&](int j, int c) { return (float)k[j * A.k_token + c]; }, [&](int j, int c) { return (float)v[j * A.v_token + c]; },
            [&](int c, float sum, float reference, float weight) {
                if (parts == 1) {
                    y[c] = (T)(weight != 0.f ? sum / weight : 0.f);
                    return;
                }
                A.part[id * A.dim + c] = sum;
                float *stat = A.part + all * parts * A.dim + 2 * id;
                if (c == 0) {
                    stat[0] = reference;
                    stat[1] = weight;
                }
            });
    }
}

template <typename T, int WAVES>
__global__ void __launch_bounds__(256) attn_join_kernel(AttnArgs A, int parts, int chunk)
{
    __shared__ JoinScratch<WAVES> lds;
    const int at = WAVES > 1 ? blockIdx.x : blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= A.batch * A.max_queries * A.q_heads)
        return;
    const int head = at % A.q_heads, i = at / A.q_heads % A.max_queries, b = at / A.q_heads / A.max_queries;
    const Span2 seq = sequence(A, b);
    if (i >= seq.n)
        return;
    // the parts that its workgroup's rows have
    const int per = A.q_heads / A.heads, last_row = (i * per + head % per) / ROWS * ROWS + ROWS - 1;
    const int limit = seen_by(A, seq, min(last_row / per, seq.n - 1)), used = min(parts_of(limit, chunk), parts);
    const long long query = seq.begin + i;
    const long long row = (query * A.q_heads + head) * parts, all = (long long)A.queries * A.q_heads * parts;
    join_parts<T, WAVES>(lds, A.part + row * A.dim, A.part + all * A.dim + 2 * row, 1, used, A.dim, (T *)A.y + query * A.y_token + head * A.y_head);
}

int row_tiles(const AttnArgs &a) { return (int)(((long long)a.max_queries * (a.q_heads / a.heads) + ROWS - 1) / ROWS); }

// whether the copies can take rows as they lie: at multiples of 4 bytes
bool direct(const AttnArgs &a)
{
    return (((uintptr_t)a.k | (uintptr_t)a.v) & 3) == 0 && ((a.k_token | a.k_head | a.v_token | a.v_head) & 1) == 0;
}

template <typename T, int DIM>
hipError_t launch_rows(const AttnArgs &a, const AttnPlan &p, hipStream_t stream)
{
    const int tiles = row_tiles(a);
    // row tiles that sequences of `queries` rows together can have, each but one of a sequence full
    const long long all = (long long)a.batch * tiles, most = (long long)a.queries * (a.q_heads / a.heads) / ROWS + a.batch;
    // (one of 16384 and 31 of 500 2.4 ms, 7.9 with a grid of the longest; 17 of 40 to 2048 353 us, 355; 17 of 700 to 2048 398, 405)
    const bool packed = p.parts == 1 && 4 * all > 5 * most;
    const dim3 grid((unsigned)(a.heads * (packed ? most : all * p.parts)));
    if (direct(a))
        hipLaunchKernelGGL((attn_kernel<T, DIM, true>), grid, dim3(256), 0, stream, a, tiles, p.parts, p.chunk, packed);
    else
        hipLaunchKernelGGL((attn_kernel<T, DIM, false>), grid, dim3(256), 0, stream, a, tiles, p.parts, p.chunk, packed);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const AttnArgs &a, const AttnPlan &p, hipStream_t stream)
{
    const hipError_t e = a.dim <= 64    ? launch_rows<T, 64>(a, p, stream)
                         : a.dim <= 128 ? launch_rows<T, 128>(a, p, stream)
                                        : launch_rows<T, 256>(a, p, stream);
    if (e != hipSuccess || p.parts == 1)
        return e;
    const unsigned all = (unsigned)a.batch * a.max_queries * a.q_heads;
    if (p.parts <= JOIN_FEW)
        hipLaunchKernelGGL((attn_join_kernel<T, 1>), dim3((all + 3) / 4), dim3(256), 0, stream, a, p.parts, p.chunk);
    else
        hipLaunchKernelGGL((attn_join_kernel<T, 4>), dim3(all), dim3(256), 0, stream, a, p.parts, p.chunk);
    return hipGetLastError();
}

}  // namespace

// The split that a model of the time finds fastest, in us: a workgroup takes START and per 32 keys ALONE, or PAIR where two share a CU;
// a second launch JOIN, a row's share of it, and the parts' bytes. (32 query heads on 8, dim 128: 512 queries over 16384 keys 190 us
// split, 432 whole, 4 over 20000 25 and 494; 500 over 500 are left whole, 20 us, 53 in parts that fill the GPU. 100 over 1337 of 12 heads on 4, dim
// 64: 14 and 31.)
AttnPlan attn_plan(const AttnArgs &a, size_t room)
{
    constexpr double START = 5.0, ALONE = 0.6, PAIR = 1.0, JOIN = 4.0, JOIN_ROW = 0.0004, MEMORY = 4e6;
    constexpr int CUS = 256;
    const int keys = a.max_keys, steps = (keys + 31) / 32;
    const double groups = (double)a.batch * a.heads * row_tiles(a), rows = (double)a.queries * a.q_heads;
    const double one = rows * (a.dim + 2) * 4;
    AttnPlan best = {1, INT32_MAX - 65536, 0, 0};
    double least = 1e30;
    for (int parts : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128}) {
        if (parts > 1 && (one * parts > (double)room || steps < 2 * parts))
            break;
        const int each = (steps + parts - 1) / parts;
        const double all = groups * parts;
        const double t = (all <= CUS ? START + ALONE * each : std::max(1.0, all / (2 * CUS)) * (START + PAIR * each)) +
                         (parts > 1 ? JOIN + JOIN_ROW * rows + 2 * one * parts / MEMORY : 0.0);
        if (t < least) {
            least = t;
            if (parts > 1) {
                const int used = (steps + each - 1) / each;
                best = {used, 32 * each, (size_t)(one * used), 0};
            }
        }
    }
    return best;
}

hipError_t launch_attn(const AttnArgs &a, const AttnPlan &plan, hipStream_t stream)
{
    return a.type == AQD_F16 ? launch_type<_Float16>(a, plan, stream) : launch_type<__bf16>(a, plan, stream);
}

}  // namespace aqd
