// Attention of one query by one wave, key by key, on the vector units: only what the
// query sees is ever multiplied. For rows whose result is no number in the matrix cores' form, where a
// weight of zero does not take an infinity or a NaN out of the sum.
#pragma once

#include "attn_common.h"

namespace aqd {
namespace {

// scratch of a wave in LDS: the query, and the weights of 64 keys
struct RowScratch {
    float q[256], p[64];
};

// query(c), key(j, c), value(j, c): element c of the query, and of key and value j; keys first .. end - 1 are seen.
// out(c, sum, reference, total): sums of weights 2^(score - reference) and of their products. Weights are at most 2^-32, so that 2^31 of them
// times fp32's largest values are a number. Lanes of a wave in step; the scratch is the wave's own.
template <int DIM, typename Query, typename Key, typename Value, typename Out>
__device__ __forceinline__ void row_attention(RowScratch &lds, int dim, int first, int end, float scale, Query query, Key key, Value value, Out out)
{
    const int lane = threadIdx.x & 63;
    constexpr int V = (DIM + 63) / 64;
    __builtin_amdgcn_wave_barrier();
    for (int c = lane; c < dim; c += 64)
        lds.q[c] = query(c) * scale;
    __builtin_amdgcn_wave_barrier();
    constexpr float LOW = 32.f;
    float y[V] = {}, most = -INFINITY, total = 0.f;
    for (int t = first; t < end; t += 64) {
        const int j = t + lane;
        float s = -INFINITY;
        if (j < end) {
            s = 0.f;
            for (int c = 0; c < dim; ++c)
                s = __builtin_fmaf(lds.q[c], key(j, c), s);
            s *= LOG2E;
        }
        float top = s;
        for (int d = 32; d; d >>= 1)
            top = fmaxf(top, __shfl_xor(top, d));
        // -infinity while no score is above it: weights 0 until then (an infinite or NaN score gives NaN below)
        const float next = fmaxf(most, top), base = next == -INFINITY ? 0.f : next;
        const float fade = exp2_fast(most - base), p = j < end ? exp2_fast(s - base - LOW) : 0.f;
        float sum = p;
        for (int d = 32; d; d >>= 1)
            sum += __shfl_xor(sum, d);
        total = total * fade + sum;
        most = next;
        lds.p[lane] = p;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int v = 0; v < V; ++v)
            y[v] *= fade;
        const int count = end - t < 64 ? end - t : 64;
        for (int i = 0; i < count; ++i) {
            const float w = lds.p[i];
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (lane + 64 * v < dim)
                    y[v] = __builtin_fmaf(w, value(t + i, lane + 64 * v), y[v]);
        }
        __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (lane + 64 * v < dim)
            out(lane + 64 * v, y[v], most + LOW, total);
}

}  // namespace
}  // namespace aqd
