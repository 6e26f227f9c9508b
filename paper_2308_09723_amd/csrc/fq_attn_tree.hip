// Attention of drafted tokens over the pages of a cache (fq_attention_tree).
#include <hip/hip_runtime.h>

#include "fq_attn.h"

namespace {

using namespace fqa;

template <int ACT>
__global__ __launch_bounds__(256) void fq_attention_tree_kernel(fq_tree_args a, float factor) {
    const int64_t pair = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);      // a node and a query head
    if (pair >= a.sequences * a.nodes * a.q_heads) return;
    const int64_t row = pair / a.q_heads;
    const int h = (int)(pair - row * a.q_heads);
    const int b = (int)(row / a.nodes), i = (int)(row - (int64_t)b * a.nodes);
    const int hk = h / (a.q_heads / a.kv_heads);
    paged_rows rows;
    rows.k = (const uint16_t*)a.cache.k + hk * a.cache.head_stride;
    rows.v = (const uint16_t*)a.cache.v + hk * a.cache.head_stride;
    rows.page_stride = a.cache.page_stride;
    rows.token_stride = a.cache.token_stride;
    rows.table = a.page_table + b * a.table_width;
    rows.page_size = (uint32_t)a.cache.page_size;
    rows.last_page = (uint32_t)(a.cache.pages - 1);
    const int capacity = (int)a.table_width * a.cache.page_size, context = a.context_lens[b];
    const int end = context < 0 ? 0 : (int)min((int64_t)capacity, (int64_t)context + a.nodes);
    const uint16_t* q = (const uint16_t*)a.q.data + row * a.q.row_stride + h * a.q.head_stride;
    float o[2], m, l;
    if (a.mask) {
        const sees_tree sees{context, a.nodes, a.mask + b * a.mask_stride + (int64_t)i * ((a.nodes + 63) / 64)};
        attend_one<ACT>(q, rows, sees, 0, end, a.head_dim, factor, o, &m, &l);
    } else {
        const int64_t last = (int64_t)context + i + 1;
        const sees_first sees{(int)min((int64_t)end, last)};
        attend_one<ACT>(q, rows, sees, 0, context < 0 ? 0 : sees.end, a.head_dim, factor, o, &m, &l);
    }
    store_one<ACT>((uint16_t*)a.out + (row * a.q_heads + h) * a.head_dim, o, l, a.head_dim);
}

}  // namespace

size_t fq_tree_bytes(const fq_tree_args& a) {
    (void)a;
    return 0;
}

int fq_launch_attention_tree(int act_dtype, const fq_tree_args& a, void* workspace, hipStream_t stream) {
    (void)workspace;
    const dim3 grid((unsigned)((a.sequences * a.nodes * a.q_heads + 3) / 4));
    const float factor = a.scale * LOG2E;
    if (act_dtype == FQ_F16) fq_attention_tree_kernel<FQ_F16><<<grid, 256, 0, stream>>>(a, factor);
    else fq_attention_tree_kernel<FQ_BF16><<<grid, 256, 0, stream>>>(a, factor);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}
