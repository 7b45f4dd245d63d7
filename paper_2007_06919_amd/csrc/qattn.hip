// Attention over the 4-bit cache. Definition and layout: include/aqd.h.

#include "attn_row.h"

namespace aqd {
namespace {

template <typename T>
__global__ void __launch_bounds__(64) qattn_row_kernel(QattnArgs A)
{
    __shared__ RowScratch lds;
    const int i = blockIdx.x % A.max_queries, rest = blockIdx.x / A.max_queries, head = rest % A.q_heads, b = rest / A.q_heads;
    const int begin = A.q_start ? min(max(A.q_start[b], 0), A.queries) : b;
    const int end = A.q_start ? min(max(A.q_start[b + 1], 0), A.queries) : b + 1;
    const int n = min(end - begin, A.max_queries);
    if (i >= n)
        return;
    const QcacheShape &c = A.c;
    const int length = max((int)min((long long)min(A.lengths[b], A.max_keys), A.ld_table * c.page), 0);
    const int keys = max(length - n + 1 + i, 0), kv = head / (A.q_heads / c.heads), groups = c.dim / c.group;
    const int32_t *table = A.tables + b * A.ld_table;
    const T *q = (const T *)A.q + (begin + i) * A.q_token + head * A.q_head;
    T *y = (T *)A.y + (begin + i) * A.y_token + head * A.y_head;
    const auto block = [&](int j) -> const uint8_t * {
        const int page = table[j / c.page];
        return page >= 0 && page < c.pages ? A.cache + ((long long)page * c.heads + kv) * c.block_bytes : nullptr;
    };
    const int scales = c.page * c.dim;
    row_attention<256>(
        lds, c.dim, keys, A.scale, [&](int e) { return (float)q[e]; },
        [&](int j, int e) {
            const uint8_t *p = block(j);
            if (!p)
                return (float)NAN;
            const int t = j % c.page, w = e / 8, nibble = e % 8 / 2 + e % 2 * 4;
            const uint32_t word = *(const uint32_t *)(p + t * (c.dim / 2) + 4 * (w % 4 * (c.dim / 32) + w / 4));
            return (float)((int)(word >> (4 * nibble) & 15) - 8) * (float)*(const __bf16 *)(p + scales + 2 * (t * groups + e / c.group));
        },
        [&](int j, int e) {
            const uint8_t *p = block(j);
            if (!p)
                return (float)NAN;
            const int t = j % c.page;
            const uint16_t unit = *(const uint16_t *)(p + c.page * c.dim / 2 + 2 * (((t / 4 * 16 + e % 16) * (c.dim / 64) + e / 64) * 4 + t % 4));
            return (float)((unit >> (4 * (e / 16 % 4)) & 15) - 8) * (float)*(const __bf16 *)(p + scales + 2 * ((c.page + t) * groups + e / c.group));
        },
        [&](int e, float f) { y[e] = (T)f; });
}

}  // namespace

AttnPlan qattn_plan(const QattnArgs &a, size_t room)
{
    (void)room;
    return {1, a.max_keys, 0};
}

hipError_t launch_qattn(const QattnArgs &a, const AttnPlan &plan, hipStream_t stream)
{
    (void)plan;
    const dim3 grid((unsigned)(a.batch * a.q_heads * a.max_queries));
    if (a.type == AQD_F16)
        hipLaunchKernelGGL(qattn_row_kernel<_Float16>, grid, dim3(64), 0, stream, a);
    else
        hipLaunchKernelGGL(qattn_row_kernel<__bf16>, grid, dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace aqd
