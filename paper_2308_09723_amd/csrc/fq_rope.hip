// Norms of the query and key heads, rotary positions and the cache's writes, one pass over the QKV product's rows.
//
// Per head x of D values: y = x * rsqrt(mean(x^2) + eps) * weight, then the first R values turned by the row's position.  A lane
// holds one unit of a head, 2 W values: in the rotated part W pairs, that is W values from i on and W from i + R / 2 on, or 2 W
// consecutive ones where pairs lie side by side; behind it 2 W consecutive ones.  A pair never leaves its lane; the sum of squares
// goes over a head's lanes (the next power of two of them, those without a unit adding zero).
//
// The kernel is bound by memory: what it reads it writes, and computes ten operations a value.  One pass, and 16 bytes a lane: 16383
// tokens of 96 + 96 + 96 heads of 128 values, 2.42 GB in 469 us = 5.2 TB/s (a copy of 2 GiB: 4.9); 2048 tokens of 32 + 32 heads that lie in the
// Infinity Cache 68 MB in 11.8 us; eight tokens 4.9 us, a launch.
#include <hip/hip_runtime.h>

#include "fq_internal.h"

namespace {

template <int ACT> struct type16;
template <> struct type16<FQ_F16> { typedef _Float16 t; };
template <> struct type16<FQ_BF16> { typedef __bf16 t; };

template <typename T, int W>
__device__ inline void load(const T* p, float* x) {
    typedef T vec __attribute__((ext_vector_type(W)));
    const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = (float)v[i];
}
template <typename T, int W>
__device__ inline void store(T* p, const float* x) {
    typedef T vec __attribute__((ext_vector_type(W)));
    vec v;
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = (T)x[i];
    *reinterpret_cast<vec*>(p) = v;
}

// A token per block, or its heads dealt to gridDim.y blocks; LANES lanes per head (a power of two), 256 / LANES heads at a time.
template <int ACT, int W, int LANES, bool INTERLEAVED>
__global__ __launch_bounds__(256) void fq_qk_norm_rope_kernel(fq_rope_args a) {
    typedef typename type16<ACT>::t T;
    const int64_t token = blockIdx.x;
    const int unit = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int D = a.head_dim, R = a.rot_dim, units = D / (2 * W);
    const bool there = unit < units, turned = unit < R / (2 * W);
    // where the unit's two halves lie in a head
    const int first = INTERLEAVED || !turned ? 2 * W * unit : W * unit;
    const int second = INTERLEAVED || !turned ? first + W : W * unit + R / 2;

    float cos[W], sin[W], wq[2 * W], wk[2 * W];
#pragma unroll
    for (int i = 0; i < W; ++i) cos[i] = 1.0f, sin[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * W; ++i) wq[i] = wk[i] = 1.0f;
    if (turned && there) {
        int64_t p = a.positions[token];
        p = p < 0 ? 0 : p < a.table_rows ? p : a.table_rows - 1;
        const float* row = a.table + p * R + W * unit;
#pragma unroll
        for (int i = 0; i < W; ++i) cos[i] = row[i], sin[i] = row[R / 2 + i];
    }
    if (there && a.q_weight) load<T, W>((const T*)a.q_weight + first, wq), load<T, W>((const T*)a.q_weight + second, wq + W);
    if (there && a.k_weight) load<T, W>((const T*)a.k_weight + first, wk), load<T, W>((const T*)a.k_weight + second, wk + W);
    int64_t place = -1;       // of the token in the cache
    if (a.cache.pages) {
        const int64_t slot = a.slots[token];
        if (slot >= 0 && slot < a.cache.pages * a.cache.page_size) {
            const uint32_t page = (uint32_t)slot / (uint32_t)a.cache.page_size;
            place = page * a.cache.page_stride + (int64_t)((uint32_t)slot - page * (uint32_t)a.cache.page_size) * a.cache.token_stride;
        }
    }
    const T* row = (const T*)a.qkv + token * a.row_stride;
    const int heads = a.q_heads + (place >= 0 ? 2 : 1) * a.kv_heads;
    for (int h = blockIdx.y * (256 / LANES) + group; h < heads; h += gridDim.y * (256 / LANES)) {
        const bool query = h < a.q_heads, key = !query && h < a.q_heads + a.kv_heads;
        float x[2 * W];
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) x[i] = 0.0f;
        if (there) load<T, W>(row + (int64_t)h * D + first, x), load<T, W>(row + (int64_t)h * D + second, x + W);
        if (query || key) {
            if (query ? a.q_weight != nullptr : a.k_weight != nullptr) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * W; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
#pragma unroll
                for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
                const float r = 1.0f / __builtin_sqrtf(sum / (float)D + a.eps);
#pragma unroll
                for (int i = 0; i < 2 * W; ++i) x[i] = x[i] * r * (query ? wq[i] : wk[i]);
            }
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const int p = INTERLEAVED ? 2 * i : i, q = INTERLEAVED ? 2 * i + 1 : i + W;
                if (!turned) continue;
                const float u = x[p], v = x[q];
                x[p] = u * cos[i] - v * sin[i];
                x[q] = v * cos[i] + u * sin[i];
            }
        }
        if (!there) continue;
        auto put = [&](T* to) {
            store<T, W>(to + first, x);
            store<T, W>(to + second, x + W);
        };
        if (query) {
            put((T*)a.q_out + (token * a.q_heads + h) * D);
        } else if (key) {
            const int k = h - a.q_heads;
            if (a.k_out) put((T*)a.k_out + (token * a.kv_heads + k) * D);
            if (place >= 0) put((T*)a.cache.k + place + k * a.cache.head_stride);
        } else {
            put((T*)a.cache.v + place + (h - a.q_heads - a.kv_heads) * a.cache.head_stride);
        }
    }
}

template <int ACT, int W>
int launch(const fq_rope_args& a, hipStream_t stream) {
    const int units = a.head_dim / (2 * W);
    int lanes = 1;
    while (lanes < units) lanes *= 2;
    // few tokens: a block for each round of a token's heads (9 tokens of 288 heads: 10.0 -> 4.8 us)
    const int64_t rounds = ((int64_t)a.q_heads + 2 * a.kv_heads + 256 / lanes - 1) / (256 / lanes), room = 1024 / a.tokens;
    const dim3 grid((unsigned)a.tokens, (unsigned)(room < 1 ? 1 : room < rounds ? room : rounds));
#define FQ_ROPE(L)                                                                                                                    \
    case L:                                                                                                                           \
        if (a.interleaved) fq_qk_norm_rope_kernel<ACT, W, L, true><<<grid, 256, 0, stream>>>(a);                   \
        else fq_qk_norm_rope_kernel<ACT, W, L, false><<<grid, 256, 0, stream>>>(a);                                \
        break;
    switch (lanes) {
        FQ_ROPE(1)
        FQ_ROPE(2)
        FQ_ROPE(4)
        FQ_ROPE(8)
        FQ_ROPE(16)
        default: return FQ_ERR_UNSUPPORTED;
    }
#undef FQ_ROPE
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

}  // namespace

int fq_launch_qk_norm_rope(int act_dtype, const fq_rope_args& a, hipStream_t stream) {
    // 16-byte accesses where pairs of eight fill the head and its rotated part
    const bool wide = a.head_dim % 16 == 0 && a.rot_dim % 16 == 0;
    if (act_dtype == FQ_F16) return wide ? launch<FQ_F16, 8>(a, stream) : launch<FQ_F16, 4>(a, stream);
    return wide ? launch<FQ_BF16, 8>(a, stream) : launch<FQ_BF16, 4>(a, stream);
}
