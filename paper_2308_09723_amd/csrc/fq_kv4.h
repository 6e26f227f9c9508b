// A cache of keys and values held in 4 bits: where a token's codes and scales lie, and what they stand for.
//
// 16 tokens of one head make a record; a page is [kv_heads][page_size / 16] of them.  With S = ceil(head_dim / 32) (values behind
// head_dim are zeros) a record is 576 S bytes:
//   keys' codes     [4 a][16 token][S t][4 b]   values 32 t + 8 a + b (first) and 32 t + 8 a + 4 + b (second) of the token
//   values' codes   [4 a][16 n][S j][4 b]       token 4 a + b's values 32 j + n (first) and 32 j + 16 + n (second)
//   keys' scales    [4 a][S g][4 b]             of token 4 a + b's values 32 g .. 32 g + 31, 16 bits
//   values' scales  [4 a][S g][4 b]
// That is the order in which 16 x 16 x 32 products take them (lane 16 a + x): keys as rows by their values, values as columns by
// their tokens; each token's bytes are its own, so that tokens are written one by one.
//
// A byte holds two codes, sign and magnitude: bits 7, 2 .. 0 the first, bits 6, 5 .. 3 the second.  A magnitude alone in a byte's low
// bits, with the sign on top, is a subnormal 8-bit float (4 bits of exponent, 3 of mantissa), 2^-9 times the code: the hardware's
// conversions of such floats take codes to 16 bits two at a time, four codes of first bytes behind one mask.
//
// The scale of a group is the smallest value s of the 16-bit type with at most 8 (binary16) or 5 (bfloat16) significant bits and
// 7.5 s >= the group's largest magnitude.  A code has 3 bits, so that code times scale has 11 or 8: it IS a value of the type, and
// nothing is rounded when the cache is read.  (What the missing bits cost: scales of bfloat16 are on average 3 % larger than needed,
// the errors of codes likewise.)
#ifndef FQ_KV4_H_
#define FQ_KV4_H_

#include <stdint.h>

#include "../../include/fq.h"

namespace fqkv {

constexpr int RECORD = 16;                    // tokens

#ifdef __HIP__
#define FQ_KV4_EITHER __host__ __device__
#else
#define FQ_KV4_EITHER
#endif

FQ_KV4_EITHER constexpr int groups_of(int head_dim) { return (head_dim + 31) / 32; }
FQ_KV4_EITHER constexpr int record_bytes(int S) { return 576 * S; }
FQ_KV4_EITHER constexpr int64_t page_bytes(int page_size, int kv_heads, int head_dim) {
    return (int64_t)(page_size / RECORD) * kv_heads * record_bytes(groups_of(head_dim));
}
// Within a record: the four bytes of a key's values 32 t + 8 a .. + 7; the byte of a value pair; a group's scale (of keys; of values 32 S behind)
FQ_KV4_EITHER constexpr int key_at(int S, int token, int t, int a) { return (a * 16 + token) * 4 * S + 4 * t; }
FQ_KV4_EITHER constexpr int value_at(int S, int token, int j, int n) { return 256 * S + (token / 4 * 16 + n) * 4 * S + 4 * j + token % 4; }
FQ_KV4_EITHER constexpr int scale_at(int S, int token, int g) { return 512 * S + (token / 4 * S + g) * 8 + token % 4 * 2; }

#ifdef __HIP__
// The first codes of four bytes as 8-bit floats, and the second ones
__device__ __forceinline__ uint32_t firsts(uint32_t x) { return x & 0x87878787u; }
__device__ __forceinline__ uint32_t seconds(uint32_t x) {
    const uint32_t low = x >> 3, high = x << 1;
    return ((low & 0x07070707u) | (high & ~0x07070707u)) & 0x87878787u;
}
// Codes of bytes 0 and 1 (HIGH: 2 and 3) of such a word, as two 16-bit numbers
template <int ACT, bool HIGH>
__device__ __forceinline__ uint32_t codes16(uint32_t x) {
    if constexpr (ACT == FQ_F16)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 512.0f, HIGH));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 512.0f, HIGH));
}
// Four quotients as codes, the nearest numbers (halves to even, 7 for 7.5), sign and magnitude in bits 7, 2 .. 0 of a byte (the sign of a zero is anything)
__device__ __forceinline__ uint32_t coded(const float* q) {
    uint32_t x = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) x = __builtin_amdgcn_cvt_pk_u8_f32(__builtin_fminf(__builtin_fabsf(q[i]), 7.0f), i, x);
    const uint32_t low = __builtin_amdgcn_perm(__float_as_uint(q[1]), __float_as_uint(q[0]), 0x0c0c0703u),
                   high = __builtin_amdgcn_perm(__float_as_uint(q[3]), __float_as_uint(q[2]), 0x07030c0cu);       // their top bytes
    return x | ((low | high) & 0x80808080u);
}
// the code (of bits 7, 2 .. 0) as a number
__device__ __forceinline__ float decoded(uint32_t c) {
    const float m = (float)(c & 7u);
    return c & 0x80u ? -m : m;
}
__device__ __forceinline__ uint32_t from_second(uint32_t b) { return (b >> 3 & 7u) | (b << 1 & 0x80u); }

// A group's scale n 2^k for its largest magnitude m.
struct group_scale {
    float n;
    int k;
    template <int ACT>
    __device__ static group_scale of(float m) {
        constexpr int BITS = ACT == FQ_F16 ? 8 : 5, LEAST = ACT == FQ_F16 ? -24 : -133;
        // m / 7.5, too large by less than 2^-23 of it.  m 2^-k is a multiple of 1 / 8, a quotient that is not whole at least 1 / 60 away from one.
        const float x = m * 0x1.111112p-3f;
        const int e = m > 0.0f ? __builtin_amdgcn_frexp_expf(x) : LEAST;
        group_scale s;
        s.k = e - BITS > LEAST ? e - BITS : LEAST;
        s.n = __builtin_floorf(__builtin_amdgcn_ldexpf(x, -s.k));
        if (7.5f * s.n < __builtin_amdgcn_ldexpf(m, -s.k)) s.n += 1.0f;
        return s;
    }
    __device__ float value() const { return __builtin_amdgcn_ldexpf(n, k); }
    // What quotient() multiplies values with (bfloat16: values times 2^-k, whose product with it may be too large for one)
    template <int ACT>
    __device__ float inverse() const {
        const float x = n == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(n);
        return ACT == FQ_F16 ? __builtin_amdgcn_ldexpf(x, -k) : x;
    }
    // w / s for |w| <= m, halves exactly.  The product with the inverse (whose last bit may be wrong) is off by less than 2^-20.  The quotient is a half
    // exactly or 2^-12 away from one (values have 11 bits, n 8), so that the addition, which leaves multiples of 2^-16, makes halves exact and takes
    // nothing else to the other side of one.
    template <int ACT>
    __device__ float quotient(float w, float inverse) const {
        return __builtin_fmaf(ACT == FQ_F16 ? w : __builtin_amdgcn_ldexpf(w, -k), inverse, 128.0f) - 128.0f;
    }
};
#endif

}  // namespace fqkv

#endif  // FQ_KV4_H_
