// Causal attention over packed sequences (fq_attention_prompt).
#include <hip/hip_runtime.h>
#include <algorithm>

#include "fq_attn.h"

namespace {

using namespace fqa;

constexpr int TILE = 4;              // queries per block
constexpr int SEQUENCES = 128;       // per launch: their table is a kernel argument

// The sequences of a launch, longest first, and the order of their query tiles: the last tiles of the longest sequences, which
// have the most keys, come first, level by level.
struct prompt_items {
    int32_t q_start[SEQUENCES], q_len[SEQUENCES], k_start[SEQUENCES], k_len[SEQUENCES];
    int32_t tiles[SEQUENCES];
    int32_t before[SEQUENCES];       // tiles that come before the levels of which sequence s is the shortest end
    int32_t count;
};

// Tile `rank` in that order: its sequence, and its number within it.
__device__ inline void find_tile(const prompt_items& items, int rank, int* sequence, int* tile) {
    const int lane = threadIdx.x & 63;
    int s = 0;
    for (int i = 0; i < SEQUENCES; i += 64)
        s += __builtin_popcountll(__ballot(i + lane < items.count && items.before[i + lane] <= rank));
    s = __builtin_amdgcn_readfirstlane(s - 1);
    const int in = rank - items.before[s];
    const int level = in / (s + 1);
    *sequence = in - level * (s + 1);
    *tile = items.tiles[s] - 1 - level;
}

template <int ACT>
__global__ __launch_bounds__(256) void fq_attention_prompt_kernel(fq_heads q, fq_heads k, fq_heads v, int q_heads, int group, int D,
                                                                  float factor, uint16_t* out, prompt_items items) {
    int sequence, tile;
    find_tile(items, blockIdx.x, &sequence, &tile);
    const int i = tile * TILE + (threadIdx.x >> 6), h = blockIdx.y;
    const int queries = items.q_len[sequence], keys = items.k_len[sequence];
    if (i >= queries) return;
    packed_rows rows;
    rows.k = (const uint16_t*)k.data + items.k_start[sequence] * k.row_stride + h / group * k.head_stride;
    rows.v = (const uint16_t*)v.data + items.k_start[sequence] * v.row_stride + h / group * v.head_stride;
    rows.k_stride = k.row_stride;
    rows.v_stride = v.row_stride;
    const int64_t row = (int64_t)items.q_start[sequence] + i;
    const int end = max(0, i + 1 + keys - queries);
    float o[2], m, l;
    attend_one<ACT>((const uint16_t*)q.data + row * q.row_stride + h * q.head_stride, rows, sees_first{end}, 0, end, D, factor, o, &m, &l);
    store_one<ACT>(out + (row * q_heads + h) * D, o, l, D);
}

}  // namespace

size_t fq_prompt_bytes(const fq_prompt_args& a) {
    (void)a;
    return 0;
}

int fq_launch_attention_prompt(int act_dtype, const fq_prompt_args& a, void* workspace, hipStream_t stream) {
    (void)workspace;
    for (int first = 0; first < a.sequences; first += SEQUENCES) {
        const int n = std::min(SEQUENCES, a.sequences - first);
        int order[SEQUENCES], tiles[SEQUENCES];
        for (int i = 0; i < n; ++i) {
            order[i] = i;
            tiles[i] = (a.q_offsets[first + i + 1] - a.q_offsets[first + i] + TILE - 1) / TILE;
        }
        std::stable_sort(order, order + n, [&](int x, int y) { return tiles[x] > tiles[y]; });
        prompt_items items = {};
        items.count = n;
        int total = 0;
        for (int s = 0; s < n; ++s) {
            const int b = first + order[s];
            items.q_start[s] = a.q_offsets[b];
            items.q_len[s] = a.q_offsets[b + 1] - a.q_offsets[b];
            items.k_start[s] = a.k_offsets[b];
            items.k_len[s] = a.k_offsets[b + 1] - a.k_offsets[b];
            items.tiles[s] = tiles[order[s]];
        }
        // levels from the longest sequence's last tile down: those that sequences 0 .. s have and s + 1 has not
        for (int s = 0; s < n; ++s) {
            items.before[s] = total;
            total += (s + 1) * (items.tiles[s] - (s + 1 < n ? items.tiles[s + 1] : 0));
        }
        if (total == 0) continue;
        const dim3 grid((unsigned)total, (unsigned)a.q_heads);
        const float factor = a.scale * LOG2E;
        const int group = a.q_heads / a.kv_heads;
        if (act_dtype == FQ_F16)
            fq_attention_prompt_kernel<FQ_F16><<<grid, 64 * TILE, 0, stream>>>(a.q, a.k, a.v, a.q_heads, group, a.head_dim, factor, (uint16_t*)a.out, items);
        else
            fq_attention_prompt_kernel<FQ_BF16><<<grid, 64 * TILE, 0, stream>>>(a.q, a.k, a.v, a.q_heads, group, a.head_dim, factor, (uint16_t*)a.out, items);
        if (hipGetLastError() != hipSuccess) return FQ_ERR_HIP;
    }
    return FQ_OK;
}
