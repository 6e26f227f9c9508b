// What the attention kernels share: where keys and values lie, which of them a query sees, and one query's attention.
#ifndef FQ_ATTN_H_
#define FQ_ATTN_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fq_internal.h"

namespace fqa {

template <int ACT> struct type16;
template <> struct type16<FQ_F16> { typedef _Float16 t; };
template <> struct type16<FQ_BF16> { typedef __bf16 t; };

constexpr float LOG2E = 1.44269504088896340736f;

// Quotients of numbers below 2^31 by one that the host knows, 1 to 2^31: a multiplication (by m = ceil(2^(31 + k) / d), where 2^k is the
// first power of two that is not below d: the error of n m / 2^(31 + k) is below n / 2^(31 + k) <= 1 / d).
struct divisor {
    uint32_t d, m, shift;
    static divisor of(uint32_t d) {
        uint32_t k = 0;
        while (((uint64_t)1 << k) < d) ++k;
        return {d, k == 0 ? 0 : (uint32_t)((((uint64_t)1 << (31 + k)) + d - 1) / d), k - 1};
    }
    __device__ int quotient(int n) const { return m == 0 ? n : (int)(__umulhi((uint32_t)n, m) >> shift); }
};

// Keys and values of 16 bits, one at a time: ROWS says where they lie.
template <typename ROWS>
struct rows16 {
    // q . k of key j
    template <int ACT>
    __device__ float dot(const uint16_t* q, int j, int D) const {
        typedef typename type16<ACT>::t T;
        typedef T vec8 __attribute__((ext_vector_type(8)));
        const T* k = (const T*)((const ROWS*)this)->key(j);
        float sum = 0.0f;
        for (int c = 0; c < D; c += 8) {
            const vec8 x = *(const vec8*)((const T*)q + c), y = *(const vec8*)(k + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fmaf((float)x[i], (float)y[i], sum);
        }
        return sum;
    }
    // values d and d + 1 of key j (d even)
    template <int ACT>
    __device__ void two(int j, int d, float* v) const {
        typedef typename type16<ACT>::t T;
        typedef T vec2 __attribute__((ext_vector_type(2)));
        const vec2 x = *(const vec2*)((const T*)((const ROWS*)this)->value(j) + d);
        v[0] = (float)x[0];
        v[1] = (float)x[1];
    }
};

// One key head's keys and values of a sequence, packed: rows a stride apart.
struct packed_rows : rows16<packed_rows> {
    const uint16_t *k, *v;
    int64_t k_stride, v_stride;
    __device__ const uint16_t* key(int j) const { return k + j * k_stride; }
    __device__ const uint16_t* value(int j) const { return v + j * v_stride; }
};
// The same in the pages of a cache.
struct paged_rows : rows16<paged_rows> {
    const uint16_t *k, *v;
    int64_t page_stride, token_stride;
    const int32_t* table;       // the sequence's row of the page table
    uint32_t page_size, last_page;
    __device__ int64_t place(int j) const {
        const uint32_t n = (uint32_t)j / page_size, at = (uint32_t)j - n * page_size;
        const int32_t page = table[n];
        return (int64_t)(page < 0 ? 0u : min((uint32_t)page, last_page)) * page_stride + at * token_stride;
    }
    __device__ const uint16_t* key(int j) const { return k + place(j); }
    __device__ const uint16_t* value(int j) const { return v + place(j); }

    // of sequence b and key head `head`
    __device__ static paged_rows of(const fq_tree_args& a, int b, int head) {
        paged_rows x;
        x.k = (const uint16_t*)a.cache.k + head * a.cache.head_stride;
        x.v = (const uint16_t*)a.cache.v + head * a.cache.head_stride;
        x.page_stride = a.cache.page_stride;
        x.token_stride = a.cache.token_stride;
        x.table = a.page_table + b * a.table_width;
        x.page_size = (uint32_t)a.cache.page_size;
        x.last_page = (uint32_t)(a.cache.pages - 1);
        return x;
    }
};

// The query sees keys 0 .. end - 1.
struct sees_first {
    int end;
    __device__ bool operator()(int j) const { return j < end; }
};
// The query sees the context, and the drafted tokens behind it whose bits are set.
struct sees_tree {
    int context, drafted;
    const uint64_t* words;
    __device__ bool operator()(int j) const {
        const int d = j - context;
        return d < 0 || (d < drafted && (words[d >> 6] >> (d & 63) & 1));
    }
};

__device__ inline float wave_max(float x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = __builtin_fmaxf(x, __shfl_xor(x, d));
    return x;
}
__device__ inline float wave_sum(float x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}

// One query's attention over keys begin .. end - 1, by one wave: 64 keys at a time, a key per lane for the scores and two
// values of the head per lane for the sums, with the running maximum and sum of the softmax.  Keys that the query does not see
// are not read as values, so that nothing in them reaches the result.  factor: the scale of the scores times log2(e).
// o: the sums for values 2 lane and 2 lane + 1, not divided by the numerators' sum l; m: the largest score (times factor).
template <int ACT, typename ROWS, typename SEES>
__device__ inline void attend_one(const uint16_t* q, const ROWS& rows, const SEES& sees, int begin, int end, int D, float factor,
                                  float* o, float* m_out, float* l_out) {
    const int lane = threadIdx.x & 63;
    float m = -__builtin_inff(), l = 0.0f;
    o[0] = o[1] = 0.0f;
    for (int base = begin; base < end; base += 64) {
        const int j = base + lane;
        const bool seen = j < end && sees(j);
        float s = -__builtin_inff();
        if (seen) s = rows.template dot<ACT>(q, j, D) * factor;
        uint64_t left = __ballot(seen);
        if (left == 0) continue;
        // (a score that is a NaN makes its numerator one; the maximum passes it by)
        const float top = __builtin_fmaxf(m, wave_max(s));
        const float from = top == -__builtin_inff() ? 0.0f : top;
        const float p = seen ? __builtin_exp2f(s - from) : 0.0f, again = __builtin_exp2f(m - from);
        m = top;
        l = l * again + wave_sum(p);
        o[0] *= again;
        o[1] *= again;
        while (left) {
            const int i = __builtin_ctzll(left);
            left &= left - 1;
            const float w = __shfl(p, i);
            if (2 * lane < D) {
                float v[2];
                rows.template two<ACT>(base + i, 2 * lane, v);
                o[0] = __builtin_fmaf(w, v[0], o[0]);
                o[1] = __builtin_fmaf(w, v[1], o[1]);
            }
        }
    }
    *m_out = m;
    *l_out = l;
}

// 1 / l for a row's sum of numerators.  0: a row that sees no key, zeros; or one whose keys' scores are all -infinity, whose softmax is no number
// (sees(): whether the row sees a key, asked for then).
template <typename SEES>
__device__ inline float inverse(float l, const SEES& sees) {
    if (l != 0.0f) return 1.0f / l;
    return sees() ? __builtin_nanf("") : 0.0f;
}

// attend_one's result, to row `out`.
template <int ACT, typename SEES>
__device__ inline void store_one(uint16_t* out, const float* o, float l, int D, const SEES& sees) {
    typedef typename type16<ACT>::t T;
    typedef T vec2 __attribute__((ext_vector_type(2)));
    const int lane = threadIdx.x & 63;
    if (2 * lane >= D) return;
    const float r = inverse(l, sees);
    vec2 v;
    v[0] = (T)(o[0] * r);
    v[1] = (T)(o[1] * r);
    *(vec2*)((T*)out + 2 * lane) = v;
}

}  // namespace fqa

#endif  // FQ_ATTN_H_
