// Keys and values into a cache held in 4 bits, and back (fq_kv4_write, fq_kv4_read; layout and scales: fq_kv4.h).
//
// Per group of 32 values w: s from max |w|, q = clamp(rint(w / s), -7, 7).  A lane has 8 values of a head (16 bytes); sixteen lanes four groups of
// a token, neighbours neighbouring groups, whose words lie side by side in the cache; and the four lanes 16 apart the same 8 values of four tokens: where these lie in the
// cache as the four of one word, the bytes of their values' codes are exchanged between the four lanes, and words are stored.  Otherwise each
// byte is.  Rows are dealt out in fours from the first that lies so, since a prompt's tokens lie one behind the other.
//
// Bound by memory (16 bits a value one way, 4.5 the other), close behind by a hundred instructions for eight values: 16383 tokens of 8 heads of 128, 86 MB,
// written in 22.9 us, 3.8 TB/s, read in 18.5, 4.7, bfloat16 23.8 and 18.6; 33 tokens 3.3 us, a token each of 64 sequences 3.5, of 256 3.7.
#include <hip/hip_runtime.h>

#include "fq_attn_tile.h"
#include "fq_internal.h"
#include "fq_kv4.h"

namespace {

using namespace fqkv;

using fqa::pack2;
using fqa::type16;
using fqa::u32x4;

template <int ACT, int HIGH>
__device__ __forceinline__ float half_of(uint32_t x) {
    if constexpr (ACT == FQ_F16) {
        typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
        return (float)__builtin_bit_cast(vec2, x)[HIGH];
    } else {
        return __uint_as_float(HIGH ? x & 0xffff0000u : x << 16);
    }
}
// The largest magnitude of eight values, as its bits: an infinity's, or more for a NaN
__device__ __forceinline__ uint32_t largest(const u32x4& w) {
    typedef uint16_t vec2 __attribute__((ext_vector_type(2)));
    vec2 m = __builtin_bit_cast(vec2, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(vec2, w[i] & 0x7fff7fffu));
    return m[0] > m[1] ? m[0] : m[1];
}

// The four tokens of a block: token first + lane / 16, and where it lies.
struct four_tokens {
    int64_t token;
    bool there;                   // whether it is one, in a slot of the cache
    char* record;                 // of head 0
    int at;                       // token of the record
    bool side_by_side;            // the four are a word's

    __device__ four_tokens(const fq_kv4_args& a) {
        const int64_t s0 = a.slots[0];
        const int ahead = s0 < 0 ? 0 : (int)(s0 & 3);          // rows of the first four that are missing
        token = (int64_t)blockIdx.x * 4 - ahead + ((threadIdx.x & 63) >> 4);
        const bool row = token >= 0 && token < a.tokens;
        const int64_t slot = row ? a.slots[token] : -1;
        there = slot >= 0 && slot < a.cache.pages * a.cache.page_size;
        const uint32_t page = there ? (uint32_t)slot / (uint32_t)a.cache.page_size : 0u;
        const uint32_t in = there ? (uint32_t)slot - page * (uint32_t)a.cache.page_size : 0u;
        at = in & 15;
        record = (char*)a.cache.data + (int64_t)page * a.cache.page_stride + (int64_t)(in >> 4) * record_bytes(a.groups);
        const int64_t first = __shfl(slot, 0);
        side_by_side = __all(there && slot == first + ((threadIdx.x & 63) >> 4) && (first & 3) == 0);
    }
};

// Bytes b of the four lanes' words, for lane 16 b + x: a 4 x 4 transposition
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    const int i = (threadIdx.x & 63) >> 4;
    // neighbouring rows of 16 lanes exchange bytes, then halves of the wave pairs of them (of both, the lower's word is [0])
    auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = __builtin_amdgcn_perm(r[1], r[0], i & 1 ? 0x07030501u : 0x06020400u);
    r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __builtin_amdgcn_perm(r[1], r[0], i & 2 ? 0x07060302u : 0x05040100u);
}
// The word of the lane that is 4 or 8 on, of sixteen
__device__ __forceinline__ uint32_t four_on(uint32_t x) { return __builtin_amdgcn_mov_dpp(x, 0x124, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t eight_on(uint32_t x) { return __builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, true); }

template <int ACT>
__global__ __launch_bounds__(256) void fq_kv4_write_kernel(fq_kv4_args a, fqa::divisor by_groups) {
    typedef typename type16<ACT>::t T;
    constexpr uint32_t INFINITE = ACT == FQ_F16 ? 0x7c00u : 0x7f80u;
    const four_tokens f(a);
    const int S = a.groups, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, all = a.kv_heads * S;
    const int64_t head_bytes = (int64_t)(a.cache.page_size / RECORD) * record_bytes(S);
    for (int base = (blockIdx.y * 4 + wave) * 4; base < 2 * all; base += gridDim.y * 16) {
        const int y = base + (lane & 3), part = lane >> 2 & 3;
        const bool in = y < 2 * all, values = y >= all;
        const int x = in ? (values ? y - all : y) : 0, head = by_groups.quotient(x), g = x - head * S, unit = 4 * g + part;
        u32x4 w = {0, 0, 0, 0};
        if (in && f.there && unit * 8 < a.head_dim) {
            const fq_heads& from = values ? a.v : a.k;
            w = *(const u32x4*)((const T*)from.data + f.token * from.row_stride + head * from.head_stride + unit * 8);
        }
        uint32_t m = largest(w);
        m = max(m, four_on(m));
        m = max(m, eight_on(m));
        const bool sound = m < INFINITE;
        const group_scale s = group_scale::of<ACT>(sound ? half_of<ACT, 0>(m) : 0.0f);
        const float inverse = s.template inverse<ACT>();
        float q[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = sound ? w[i] : 0;
            q[2 * i] = s.template quotient<ACT>(half_of<ACT, 0>(x), inverse);
            q[2 * i + 1] = s.template quotient<ACT>(half_of<ACT, 1>(x), inverse);
        }
        char* to = f.record + head * head_bytes;
        const bool put = in && f.there;
        if (part == 0 && put) *(T*)(to + (values ? 32 * S : 0) + scale_at(S, f.at, g)) = (T)(sound ? s.value() : __builtin_nanf(""));
        // Keys: the lane's codes are a word.  Values: first codes are half the lanes', second codes the other half's, of the same places; each
        // lane of such two makes four bytes of them.
        const uint32_t low = coded(q), high = coded(q + 4);
        const uint32_t other = eight_on(part < 2 ? high : low);
        const uint32_t one = values ? (part < 2 ? low : other) : low, two = values ? (part < 2 ? other : high) : high;
        const uint32_t word = one | (two & 0x07070707u) << 3 | (two & 0x80808080u) >> 1;
        const uint32_t across = transposed(word);
        if (!put) continue;
        if (!values) {
            *(uint32_t*)(to + key_at(S, f.at, g, part)) = word;
        } else {
            const int n = (part & 1) * 8 + (part >> 1) * 4;      // of the lane's first byte
            if (f.side_by_side) {
                *(uint32_t*)(to + value_at(S, f.at & ~3, g, n + (lane >> 4))) = across;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) *(uint8_t*)(to + value_at(S, f.at, g, n + i)) = (uint8_t)(word >> 8 * i);
            }
        }
    }
}

// The same way back.  Rows whose slot is outside the cache are zeros.
template <int ACT>
__global__ __launch_bounds__(256) void fq_kv4_read_kernel(fq_kv4_args a, fqa::divisor by_groups) {
    typedef typename type16<ACT>::t T;
    const four_tokens f(a);
    const int S = a.groups, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, all = a.kv_heads * S;
    const int64_t head_bytes = (int64_t)(a.cache.page_size / RECORD) * record_bytes(S);
    for (int base = (blockIdx.y * 4 + wave) * 4; base < 2 * all; base += gridDim.y * 16) {
        const int y = base + (lane & 3), part = lane >> 2 & 3;
        const bool in = y < 2 * all, values = y >= all;
        const int x = in ? (values ? y - all : y) : 0, head = by_groups.quotient(x), g = x - head * S, unit = 4 * g + part;
        const char* from = f.record + head * head_bytes;
        const bool get = in && f.there;
        uint32_t word = 0;
        float s = 0.0f;
        if (get) {
            s = (float)*(const T*)(from + (values ? 32 * S : 0) + scale_at(S, f.at, g));
            const int n = (part & 1) * 8 + (part >> 1) * 4;
            if (!values) {
                word = *(const uint32_t*)(from + key_at(S, f.at, g, part));
            } else if (f.side_by_side) {
                word = *(const uint32_t*)(from + value_at(S, f.at & ~3, g, n + (lane >> 4)));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) word |= (uint32_t)*(const uint8_t*)(from + value_at(S, f.at, g, n + i)) << 8 * i;
            }
        }
        const uint32_t across = transposed(word);
        if (values && f.side_by_side) word = across;
        const uint32_t one = firsts(word), two = seconds(word);
        const uint32_t other = eight_on(part < 2 ? two : one);
        const uint32_t low = values ? (part < 2 ? one : other) : one, high = values ? (part < 2 ? other : two) : two;
        if (!in || f.token < 0 || f.token >= a.tokens || unit * 8 >= a.head_dim) continue;
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t four = i == 0 ? low : high;
            if constexpr (ACT == FQ_F16) {
                typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
                const vec2 by = {(_Float16)s, (_Float16)s};
                v[2 * i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(vec2, codes16<ACT, false>(four)) * by);
                v[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(vec2, codes16<ACT, true>(four)) * by);
            } else {
                const auto x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(four, 512.0f, false), y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(four, 512.0f, true);
                v[2 * i] = pack2<ACT>(x[0] * s, x[1] * s);
                v[2 * i + 1] = pack2<ACT>(y[0] * s, y[1] * s);
            }
        }
        *(u32x4*)((T*)(values ? a.v_out : a.k_out) + (f.token * a.kv_heads + head) * a.head_dim + unit * 8) = v;
    }
}

dim3 grid_of(const fq_kv4_args& a) {
    const int64_t fours = (a.tokens + 3) / 4 + 1;               // (the first may begin before the first row)
    // few tokens: a block for each round of a token's units
    const int64_t rounds = ((int64_t)a.kv_heads * 8 * a.groups + 63) / 64, room = 2048 / fours;
    return dim3((unsigned)fours, (unsigned)(room < 1 ? 1 : room < rounds ? room : rounds));
}

fqa::divisor groups(const fq_kv4_args& a) { return fqa::divisor::of((uint32_t)a.groups); }

}  // namespace

int fq_launch_kv4_write(int act_dtype, const fq_kv4_args& a, hipStream_t stream) {
    if (act_dtype == FQ_F16) fq_kv4_write_kernel<FQ_F16><<<grid_of(a), 256, 0, stream>>>(a, groups(a));
    else fq_kv4_write_kernel<FQ_BF16><<<grid_of(a), 256, 0, stream>>>(a, groups(a));
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

int fq_launch_kv4_read(int act_dtype, const fq_kv4_args& a, hipStream_t stream) {
    if (act_dtype == FQ_F16) fq_kv4_read_kernel<FQ_F16><<<grid_of(a), 256, 0, stream>>>(a, groups(a));
    else fq_kv4_read_kernel<FQ_BF16><<<grid_of(a), 256, 0, stream>>>(a, groups(a));
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}
