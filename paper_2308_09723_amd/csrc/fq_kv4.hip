// Keys and values into a cache held in 4 bits, and back (fq_kv4_write, fq_kv4_read; layout and scales: fq_kv4.h).
//
// Per group of 32 values w: s from max |w|, q = clamp(rint(w / s), -7, 7).  A lane has 8 values of a head (16 bytes), four lanes a
// group, four neighbouring lanes the same 8 values of four tokens: where these lie in the cache as the four of one word, the
// bytes of their values' codes are exchanged between the four lanes, and words are stored.  Otherwise each byte is.  Rows are dealt
// out in fours from the first that lies so, since a prompt's tokens lie one behind the other.
//
// Bound by memory: 16 bits a value one way, 4.5 the other, forty operations.
#include <hip/hip_runtime.h>

#include "fq_internal.h"
#include "fq_kv4.h"

namespace {

using namespace fqkv;

template <int ACT> struct type16;
template <> struct type16<FQ_F16> { typedef _Float16 t; };
template <> struct type16<FQ_BF16> { typedef __bf16 t; };

// The four tokens of a block: token first + lane % 4, and where it lies.
struct four_tokens {
    int64_t token;
    bool there;                   // whether it is one, in a slot of the cache
    char* record;                 // of head 0
    int at;                       // token of the record
    bool side_by_side;            // the four are a word's

    __device__ four_tokens(const fq_kv4_args& a) {
        const int64_t s0 = a.slots[0];
        const int ahead = s0 < 0 ? 0 : (int)(s0 & 3);          // rows of the first four that are missing
        token = (int64_t)blockIdx.x * 4 - ahead + (threadIdx.x & 3);
        const bool row = token >= 0 && token < a.tokens;
        const int64_t slot = row ? a.slots[token] : -1;
        there = slot >= 0 && slot < a.cache.pages * a.cache.page_size;
        const uint32_t page = there ? (uint32_t)slot / (uint32_t)a.cache.page_size : 0u;
        const uint32_t in = there ? (uint32_t)slot - page * (uint32_t)a.cache.page_size : 0u;
        at = in & 15;
        record = (char*)a.cache.data + (int64_t)page * a.cache.page_stride + (int64_t)(in >> 4) * record_bytes(a.groups);
        const int64_t first = __shfl(slot, (int)(threadIdx.x & 60));
        side_by_side = __all(there && slot == first + (threadIdx.x & 3) && (first & 3) == 0);
    }
};

// Bytes b of the four lanes' words, for lane b: a 4 x 4 transposition within four lanes
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    const int i = threadIdx.x & 3;
    // pairs of lanes exchange bytes, then pairs of pairs
    uint32_t y = __builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true);          // lane i ^ 1
    x = __builtin_amdgcn_perm(y, x, i & 1 ? 0x03070105u : 0x06020400u);
    y = __builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true);                   // lane i ^ 2
    return __builtin_amdgcn_perm(y, x, i & 2 ? 0x03020706u : 0x05040100u);
}

template <int ACT>
__global__ __launch_bounds__(256) void fq_kv4_write_kernel(fq_kv4_args a) {
    typedef typename type16<ACT>::t T;
    typedef T vec8 __attribute__((ext_vector_type(8)));
    const four_tokens f(a);
    const int S = a.groups, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, units = 4 * S;
    const int all = a.kv_heads * units;
    const int64_t head_bytes = (int64_t)(a.cache.page_size / RECORD) * record_bytes(S);
    for (int base = (blockIdx.y * 4 + wave) * 16; base < 2 * all; base += gridDim.y * 64) {
        const int y = base + (lane >> 2);                       // (units come in fours, so that a group is in or out as a whole)
        const bool in = y < 2 * all, values = y >= all;
        const int x = in ? (values ? y - all : y) : 0, head = (int)((uint32_t)x / (uint32_t)units), unit = x - head * units;
        const int g = unit >> 2, part = unit & 3;
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 0.0f;
        if (in && f.there && unit * 8 < a.head_dim) {
            const fq_heads& from = values ? a.v : a.k;
            const vec8 v = *(const vec8*)((const T*)from.data + f.token * from.row_stride + head * from.head_stride + unit * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = (float)v[i];
        }
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float size = __builtin_fabsf(w[i]);
            m = size <= 3.4028234663852886e38f ? __builtin_fmaxf(m, size) : __builtin_inff();       // (a NaN as well)
        }
        m = __builtin_fmaxf(m, __shfl_xor(m, 4));
        m = __builtin_fmaxf(m, __shfl_xor(m, 8));
        const bool sound = m < __builtin_inff();
        const group_scale s = group_scale::of<ACT>(sound ? m : 0.0f);
        const float inverse = s.inverse();
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = sound ? s.code(w[i], inverse) : 0.0f;
        char* to = f.record + head * head_bytes;
        const bool put = in && f.there;
        if (part == 0 && put) *(T*)(to + (values ? 32 * S : 0) + scale_at(S, f.at, g)) = (T)(sound ? s.value() : __builtin_nanf(""));
        // Keys: the lane's codes are a word.  Values: first codes are half the lanes', second codes the other half's, of the same places; each
        // lane of such two makes four bytes of them.
        const uint32_t low = coded(q), high = coded(q + 4);
        const uint32_t other = __shfl_xor(part < 2 ? high : low, 8);
        const uint32_t one = values ? (part < 2 ? low : other) : low, two = values ? (part < 2 ? other : high) : high;
        const uint32_t word = one | (two & 0x07070707u) << 3 | (two & 0x80808080u) >> 1;
        const uint32_t across = transposed(word);
        if (!put) continue;
        if (!values) {
            *(uint32_t*)(to + key_at(S, f.at, g, part)) = word;
        } else {
            const int n = (part & 1) * 8 + (part >> 1) * 4;      // of the lane's first byte
            if (f.side_by_side) {
                *(uint32_t*)(to + value_at(S, f.at & ~3, g, n + (lane & 3))) = across;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) *(uint8_t*)(to + value_at(S, f.at, g, n + i)) = (uint8_t)(word >> 8 * i);
            }
        }
    }
}

// The same way back.  Rows whose slot is outside the cache are zeros.
template <int ACT>
__global__ __launch_bounds__(256) void fq_kv4_read_kernel(fq_kv4_args a) {
    typedef typename type16<ACT>::t T;
    typedef T vec8 __attribute__((ext_vector_type(8)));
    const four_tokens f(a);
    const int S = a.groups, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, units = 4 * S;
    const int all = a.kv_heads * units;
    const int64_t head_bytes = (int64_t)(a.cache.page_size / RECORD) * record_bytes(S);
    for (int base = (blockIdx.y * 4 + wave) * 16; base < 2 * all; base += gridDim.y * 64) {
        const int y = base + (lane >> 2);
        const bool in = y < 2 * all, values = y >= all;
        const int x = in ? (values ? y - all : y) : 0, head = (int)((uint32_t)x / (uint32_t)units), unit = x - head * units;
        const int g = unit >> 2, part = unit & 3;
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
                word = *(const uint32_t*)(from + value_at(S, f.at & ~3, g, n + (lane & 3)));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) word |= (uint32_t)*(const uint8_t*)(from + value_at(S, f.at, g, n + i)) << 8 * i;
            }
        }
        const uint32_t across = transposed(word);
        if (values && f.side_by_side) word = across;
        const uint32_t one = firsts(word), two = seconds(word);
        const uint32_t other = __shfl_xor(part < 2 ? two : one, 8);
        const uint32_t low = values ? (part < 2 ? one : other) : one, high = values ? (part < 2 ? other : two) : two;
        if (!in || f.token < 0 || f.token >= a.tokens || unit * 8 >= a.head_dim) continue;
        vec8 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = (T)(decoded(low >> 8 * i & 0xffu) * s);
            v[4 + i] = (T)(decoded(high >> 8 * i & 0xffu) * s);
        }
        T* out = (T*)(values ? a.v_out : a.k_out) + (f.token * a.kv_heads + head) * a.head_dim + unit * 8;
        *(vec8*)out = v;
    }
}

dim3 grid_of(const fq_kv4_args& a) {
    const int64_t fours = (a.tokens + 3) / 4 + 1;               // (the first may begin before the first row)
    // few tokens: a block for each round of a token's units
    const int64_t rounds = ((int64_t)a.kv_heads * 8 * a.groups + 63) / 64, room = 2048 / fours;
    return dim3((unsigned)fours, (unsigned)(room < 1 ? 1 : room < rounds ? room : rounds));
}

}  // namespace

int fq_launch_kv4_write(int act_dtype, const fq_kv4_args& a, hipStream_t stream) {
    if (act_dtype == FQ_F16) fq_kv4_write_kernel<FQ_F16><<<grid_of(a), 256, 0, stream>>>(a);
    else fq_kv4_write_kernel<FQ_BF16><<<grid_of(a), 256, 0, stream>>>(a);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

int fq_launch_kv4_read(int act_dtype, const fq_kv4_args& a, hipStream_t stream) {
    if (act_dtype == FQ_F16) fq_kv4_read_kernel<FQ_F16><<<grid_of(a), 256, 0, stream>>>(a);
    else fq_kv4_read_kernel<FQ_BF16><<<grid_of(a), 256, 0, stream>>>(a);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}
