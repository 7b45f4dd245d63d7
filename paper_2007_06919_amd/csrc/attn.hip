// Attention over keys and values of packed sequences. Definition: include/aqd.h.

#include "attn_row.h"

namespace aqd {
namespace {

template <typename T>
__global__ void __launch_bounds__(64) attn_row_kernel(AttnArgs A)
{
    __shared__ RowScratch lds;
    const int i = blockIdx.x % A.max_queries, rest = blockIdx.x / A.max_queries, head = rest % A.q_heads, b = rest / A.q_heads;
    const int begin = min(max(A.q_start[b], 0), A.queries), n = min(min(max(A.q_start[b + 1], 0), A.queries) - begin, A.max_queries);
    if (i >= n)
        return;
    const int first = min(max(A.k_start[b], 0), A.keys), m = max(min(max(A.k_start[b + 1], 0), A.keys) - first, 0);
    const int keys = A.causal ? max(m - n + 1 + i, 0) : m, kv = head / (A.q_heads / A.heads);
    const T *q = (const T *)A.q + (begin + i) * A.q_token + head * A.q_head;
    const T *k = (const T *)A.k + first * A.k_token + kv * A.k_head, *v = (const T *)A.v + first * A.v_token + kv * A.v_head;
    T *y = (T *)A.y + (begin + i) * A.y_token + head * A.y_head;
    row_attention<256>(
        lds, A.dim, keys, A.scale, [&](int c) { return (float)q[c]; }, [&](int j, int c) { return (float)k[j * A.k_token + c]; },
        [&](int j, int c) { return (float)v[j * A.v_token + c]; }, [&](int c, float f) { y[c] = (T)f; });
}

}  // namespace

AttnPlan attn_plan(const AttnArgs &a, size_t room)
{
    (void)room;
    return {1, a.max_keys, 0};
}

hipError_t launch_attn(const AttnArgs &a, const AttnPlan &plan, hipStream_t stream)
{
    (void)plan;
    const dim3 grid((unsigned)(a.batch * a.q_heads * a.max_queries));
    if (a.type == AQD_F16)
        hipLaunchKernelGGL(attn_row_kernel<_Float16>, grid, dim3(64), 0, stream, a);
    else
        hipLaunchKernelGGL(attn_row_kernel<__bf16>, grid, dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace aqd
