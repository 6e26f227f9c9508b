// Low-rank adapters of many requests beside a shared product (fq_adapters): out[m] += scale[id] (x[m] A[id]^T) B[id]^T for the adapter id of each row.
//
// t = x A^T in binary32, K split over blocks (each leaves partial sums), then out += scale t B^T.  Products are made for each of a tile's different
// adapters and all its rows, and a row takes those of its own adapter, whatever others hold.  (Requests' rows lie side by side, so that
// a tile of a prompt has one or two.)
//
// Where rows are few each is likely to have an adapter of its own, whose bytes bind it: the first kernel takes 16 rows as the columns of products of
// 16 x 16 x 32, the second makes dot products, eight ranks a lane.
// More rows: 64 a block, everything through LDS, in pieces that neighbouring lanes read side by side (a load of 64 rows' 16 bytes takes the
// address unit four times as long as one of four rows' 256).  t goes into the second product as the sum of two 16-bit numbers (16 bits and
// more of it), in binary16 after a division by a power of two that brings the row's largest to about one.
//
// Bound by memory: A and B of each adapter, x once, the output twice.  One row, K and N 1024, rank 8: 2.6 + 3.0 us, launches; 64 rows of 64 adapters, K 4096, N 6144,
// rank 16, 20 MB: 6.0 + 6.2; 2900 rows of 5 requests, K 12288, N 36864, rank 64: 28.6 for the inner sums (71 MB of x: 2.5 TB/s), 5.2 to fold them, 106 for the output (428 MB
// read and written: 4.0 TB/s), 138 in all.
#include <hip/hip_runtime.h>
#include <atomic>

#include "fq_attn_tile.h"
#include "fq_internal.h"
#include "fq_lds_limit.h"

namespace {

using fqa::f32x4;
using fqa::load_lds16;
using fqa::pack2;
using fqa::type16;
using fqa::u32x2;
using fqa::u32x4;

// Rows that are taken to have adapters of their own: where that costs little if they have not, and up to 256 where there are many adapters (the host does not see the rows' ids).  us,
// K 4096 and N 6144, 64 adapters of which the rows have one after the other, or three requests one each, so and with 64 rows a block: 64 rows of rank 64 21.4, 150, requests'
// 16.5, 17.3; 256 of rank 16 19.5, 106, and 17.3, 14.3; 256 of rank 64 41, 150, and 39.8, 16.8; 512 of rank 16 31, 106, and 29.8, 15.3.
inline bool few_rows(int64_t rows, int64_t adapters, int rank) { return rows * rank <= 4096 || (adapters > 8 && rows <= 256); }

template <int ACT>
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c) {
    if constexpr (ACT == FQ_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(fqa::f16x8, a), __builtin_bit_cast(fqa::f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(fqa::bf16x8, a), __builtin_bit_cast(fqa::bf16x8, b), c, 0, 0, 0);
}
template <int ACT, int HIGH>
__device__ __forceinline__ float half_of(uint32_t x) {
    if constexpr (ACT == FQ_F16) {
        typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
        return (float)__builtin_bit_cast(vec2, x)[HIGH];
    } else {
        return __uint_as_float(HIGH ? x & 0xffff0000u : x << 16);
    }
}

// The different adapters of a tile's rows, one after the other: id = -1 for a row that has none (lanes beyond the tile's rows as well).
// Lane l has row l's; the tile has up to 64 rows.
struct distinct {
    uint64_t left;
    int id;
    __device__ distinct(int id) : left(__ballot(id >= 0)), id(id) {}
    // the next one (-1: none is left)
    __device__ int next() {
        if (left == 0) return -1;
        const int first = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        left &= ~__ballot(id == first);
        return first;
    }
};

__device__ __forceinline__ int id_of(const fq_adapter_args& a, int64_t row) {
    if (row >= a.rows) return -1;
    const int id = a.ids[row];
    return id >= 0 && id < a.adapters ? id : -1;
}

// ------------------------------------------------------------------------------------------ t = x A^T, few rows
// 16 rows, RT x 16 values of t, one of blockIdx.y's turns of the tile's adapters, one of gridDim.x parts of K, which the block's four waves share out
// step by step of 32.  Results: partial[part][row][rank, rounded up to 16].
// (Two waves a SIMD at least, here and below: with them the compiler keeps the sums in ordinary registers.  Where they went to accumulation registers it
// read the first of them behind the loop without waiting for the last product.)
template <int ACT, int RT>
__global__ __launch_bounds__(256, 2) void fq_adapter_down_few_kernel(fq_adapter_args a) {
    constexpr int WAVES = 4, AHEAD = 4;
    __shared__ f32x4 sums[WAVES - 1][RT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 4, x16 = lane & 15;
    const int64_t row = (int64_t)blockIdx.z * 16 + x16;
    const int ranks = (a.rank + 15) / 16 * 16, steps = (a.K + 31) / 32;
    const int part = blockIdx.x, each = (steps + (int)gridDim.x - 1) / (int)gridDim.x, begin = part * each, end = min(steps, begin + each);
    distinct tile(id_of(a, lane < 16 ? row : a.rows));
    const int mine = __shfl(tile.id, x16);
    const uint16_t* x = (const uint16_t*)a.x + min(row, a.rows - 1) * a.x_stride + 8 * h;
    int turn = 0;
    for (int id = tile.next(); id >= 0; id = tile.next(), ++turn) {
        if (turn % (int)gridDim.y != (int)blockIdx.y) continue;
        for (int r0 = 0; r0 < ranks; r0 += 16 * RT) {
            const uint16_t* w[RT];
            f32x4 t[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                w[r] = (const uint16_t*)a.a + ((int64_t)id * a.rank + min(r0 + 16 * r + x16, a.rank - 1)) * a.K + 8 * h;
                t[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            }
            for (int s = begin + wave; s < end; s += WAVES * AHEAD) {
                u32x4 xs[AHEAD], ws[AHEAD][RT];
                const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int k = 32 * (s + i * WAVES);
                    const bool in = s + i * WAVES < end && k + 8 * h < a.K;
#pragma unroll
                    for (int r = 0; r < RT; ++r) ws[i][r] = in ? *(const u32x4*)(w[r] + k) : zero;
                    xs[i] = in ? *(const u32x4*)(x + k) : zero;
                }
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                    for (int r = 0; r < RT; ++r) t[r] = mfma16<ACT>(ws[i][r], xs[i], t[r]);
            }
            __syncthreads();                      // (the sums of the turn before have been read)
            if (wave > 0)
#pragma unroll
                for (int r = 0; r < RT; ++r) sums[wave - 1][r][lane] = t[r];
            __syncthreads();
            if (wave > 0) continue;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
#pragma unroll
                for (int y = 0; y < WAVES - 1; ++y) t[r] += sums[y][r][lane];
                const int at = r0 + 16 * r + 4 * h;
                if (mine == id && at < a.rank) *(f32x4*)(a.partial + ((int64_t)part * a.rows + row) * ranks + at) = t[r];
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ out += scale t B^T, few rows
// A wave has one row at a time and a column for each LANES lanes (a power of two: eight ranks each), 64 / LANES columns a step, whose weights lie one
// behind the other.
template <int ACT, int LANES>
__global__ __launch_bounds__(256) void fq_adapter_up_few_kernel(fq_adapter_args a, int parts, int steps) {
    typedef typename type16<ACT>::t T;
    constexpr int COLUMNS = 64 / LANES, AHEAD = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, u = lane % LANES, ranks = (a.rank + 15) / 16 * 16;
    const int64_t row = blockIdx.y;
    const int id = id_of(a, row);
    if (id < 0) return;
    const bool in = 8 * u < a.rank;
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = 0.0f;
    if (in) {
        const float scale = a.scales ? a.scales[id] : 1.0f;
        f32x4 x[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll 4
        for (int p = 0; p < parts; ++p) {
            const float* from = a.partial + ((int64_t)p * a.rows + row) * ranks + 8 * u;
            x[0] += *(const f32x4*)from;
            x[1] += *(const f32x4*)(from + 4);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = x[i >> 2][i & 3] * scale;
    }
    const uint16_t* weights = (const uint16_t*)a.b + (int64_t)id * a.N * a.rank + 8 * u;
    T* out = (T*)a.out + row * a.out_stride;
    const int first = ((int)blockIdx.x * 4 + wave) * steps * COLUMNS + lane / LANES;
    for (int s = 0; s < steps; s += AHEAD) {
        u32x4 w[AHEAD];
        float o[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int n = first + (s + i) * COLUMNS;
            const bool there = s + i < steps && n < a.N;
            w[i] = there && in ? *(const u32x4*)(weights + (int64_t)n * a.rank) : u32x4{0, 0, 0, 0};
            o[i] = there && u == 0 ? (float)out[n] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int n = first + (s + i) * COLUMNS;
            float sum = 0.0f;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                sum = __builtin_fmaf(half_of<ACT, 0>(w[i][y]), t[2 * y], sum);
                sum = __builtin_fmaf(half_of<ACT, 1>(w[i][y]), t[2 * y + 1], sum);
            }
#pragma unroll
            for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
            if (u == 0 && s + i < steps && n < a.N) out[n] = (T)(o[i] + sum);
        }
    }
}

// ------------------------------------------------------------------------------------------ t = x A^T, 64 rows a block
// RT x 16 ranks, one of gridDim.x parts of K in chunks of 128, one of gridDim.z's turns of the tile's adapters.  A wave has 16 of the rows.  A chunk's rows of x and A lie in LDS as 16 units of 16
// bytes, moved about within the row so that 16 rows' same unit falls on different banks; the next chunk is on its way beside the present one.
template <int ACT, int RT>
__global__ __launch_bounds__(256, 2) void fq_adapter_down_kernel(fq_adapter_args a) {
    constexpr int ROWS = 64 + 16 * RT, BYTES = ROWS * 256, LOADS = ROWS / 16;       // LOADS: of a wave, four rows each
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 4, x16 = lane & 15;
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const int64_t row0 = (int64_t)blockIdx.y * 64;
    const int ranks = (a.rank + 15) / 16 * 16, chunks = (a.K + 127) / 128;
    const int part = blockIdx.x, each = (chunks + (int)gridDim.x - 1) / (int)gridDim.x, begin = part * each, end = min(chunks, begin + each);
    distinct tile(id_of(a, row0 + lane));
    const int mine = __shfl(tile.id, 16 * wave + x16);
    int turn = 0;
    for (int id = tile.next(); id >= 0; id = tile.next(), ++turn) {
        if (turn % (int)gridDim.z != (int)blockIdx.z) continue;
        const bool busy = __any(mine == id);
        for (int r0 = 0; r0 < ranks; r0 += 16 * RT) {
            f32x4 t[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) t[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            auto load = [&](int c) {
                const uint32_t to = at + (uint32_t)(c & 1) * BYTES;
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const int y = (i * 4 + wave) * 4 + h;          // row of the chunk: 64 of x, then A's
                    const int unit = x16 ^ (y & 15), k = 128 * c + 8 * unit;
                    const uint16_t* from = y < 64 ? (const uint16_t*)a.x + min(row0 + y, a.rows - 1) * a.x_stride
                                                  : (const uint16_t*)a.a + ((int64_t)id * a.rank + min(r0 + y - 64, a.rank - 1)) * a.K;
                    if (k < a.K) load_lds16(to + (uint32_t)(i * 4 + wave) * 1024, from + k);
                    else *(u32x4*)(lds + (c & 1) * BYTES + (i * 4 + wave) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
                }
            };
            __syncthreads();                      // (the chunks of the turn before have been read)
            if (begin < end) load(begin);
            for (int c = begin; c < end; ++c) {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                __syncthreads();
                if (c + 1 < end) load(c + 1);
                if (!busy) continue;
                const char* from = lds + (c & 1) * BYTES;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int unit = (4 * s + h) ^ x16;
                    const u32x4 x = *(const u32x4*)(from + (16 * wave + x16) * 256 + unit * 16);
#pragma unroll
                    for (int r = 0; r < RT; ++r) t[r] = mfma16<ACT>(*(const u32x4*)(from + (64 + 16 * r + x16) * 256 + unit * 16), x, t[r]);
                }
            }
            const int64_t row = row0 + 16 * wave + x16;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int rank = r0 + 16 * r + 4 * h;
                if (mine == id && rank < a.rank) *(f32x4*)(a.partial + ((int64_t)part * a.rows + row) * ranks + rank) = t[r];
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ t as two 16-bit numbers
// Eight values of a row's t, over 2^e: e of the row (binary16) is asked for by exponent().
template <int ACT>
struct split8 {
    float t[8];
    // the parts' sums, times the scale
    __device__ __forceinline__ void sum(const fq_adapter_args& a, int64_t row, int rank0, int ranks, int parts, float scale) {
        f32x4 x[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
        if (rank0 < a.rank) {
            const float* from = a.partial + row * ranks + rank0;
            for (int p = 0; p < parts; ++p) {
                x[0] += *(const f32x4*)(from + (int64_t)p * a.rows * ranks);
                x[1] += *(const f32x4*)(from + (int64_t)p * a.rows * ranks + 4);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = x[i >> 2][i & 3] * scale;
    }
    // the largest magnitude of those that are finite (a division by it leaves infinities and NaNs what they are)
    __device__ __forceinline__ float most() const {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = __builtin_fabsf(t[i]) < __builtin_inff() ? __builtin_fmaxf(m, __builtin_fabsf(t[i])) : m;
        return m;
    }
    // Rounded to zero, and to the number before where next to nothing would be left: what is left then has the same sign and is no zero, so that an infinite
    // weight times both is the infinity that it is times t.  (Of a number of exponent E bfloat16 is off by 2^(E - 16) at most; binary16 by 2^(E - 22), or 2^-24 of a row whose
    // largest is 1/2 .. 1.  There, sums below 2^-23 count as zeros for an infinite weight, as do bfloat16's below 2^-118.)
    __device__ __forceinline__ void split(int e, u32x4* high, u32x4* low) const {
        constexpr float LEAST = ACT == FQ_F16 ? 0x1p-24f : 0x1p-126f, MOST = ACT == FQ_F16 ? 0x1p-23f : 0x1p-118f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float rest[2];
            uint32_t both = 0;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const float u = ACT == FQ_F16 ? __builtin_amdgcn_ldexpf(t[2 * i + x], -e) : t[2 * i + x];
                uint32_t h = ACT == FQ_F16 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(u, 0.0f)) : __float_as_uint(u) >> 16;
                if (__builtin_fabsf(u - half_of<ACT, 0>(h)) < LEAST && __builtin_fabsf(u) >= MOST) --h;
                const float d = u - half_of<ACT, 0>(h);
                rest[x] = d == d ? d : u;                     // (of an infinity: another)
                both |= h << 16 * x;
            }
            (*high)[i] = both;
            (*low)[i] = pack2<ACT>(rest[0], rest[1]);
        }
    }
};

// For many rows, once rather than by each block that needs them: [row][ranks, rounded up to 32] high, the same low, then the rows' exponents.
template <int ACT>
__global__ __launch_bounds__(256) void fq_adapter_fold_kernel(fq_adapter_args a, int parts, uint32_t* folded) {
    const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const int rank0 = threadIdx.x % 16 * 8, ranks = (a.rank + 15) / 16 * 16, wide = (a.rank + 31) / 32 * 32;
    const int id = id_of(a, row);
    split8<ACT> s;
    if (id >= 0) s.sum(a, row, rank0, ranks, parts, a.scales ? a.scales[id] : 1.0f);
    float most = id >= 0 ? s.most() : 0.0f;
#pragma unroll
    for (int d = 1; d < 16; d *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, d));
    const int e = ACT == FQ_F16 ? __builtin_amdgcn_frexp_expf(most) : 0;
    if (id < 0 || rank0 >= wide) return;
    u32x4 high, low;
    s.split(e, &high, &low);
    uint16_t* to = (uint16_t*)folded + row * wide + rank0;
    *(u32x4*)to = high;
    *(u32x4*)(to + a.rows * wide) = low;
    if (rank0 == 0) ((int32_t*)folded)[a.rows * wide + row] = e;
}

// ------------------------------------------------------------------------------------------ out += scale t B^T, 64 rows a block
// 128 columns at a time, `turns` of them one after the other; a wave has 16 of the rows.  Column 8 x + j is column x of product j, so that a lane has
// eight neighbouring columns of four rows, and 16 lanes 256 bytes of each.  Weights come through registers into LDS, the next turn's on their
// way beside the present one: eight columns' together, and 16 bytes to the next eight, so that the columns of a product fall on different banks.
template <int ACT, int RS>
__global__ __launch_bounds__(256, 2) void fq_adapter_up_kernel(fq_adapter_args a, int turns, const uint32_t* folded) {
    constexpr int UNITS = RS * 4 * 128 / 256;         // 16-byte units of a turn's weights that a thread brings in, at most
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 4, x16 = lane & 15;
    const int64_t row0 = (int64_t)blockIdx.y * 64;
    const int wide = (a.rank + 31) / 32 * 32, units = a.rank / 8, group = 8 * 16 * units + 16, bytes = 16 * group;
    const u32x4 zero = {0, 0, 0, 0};
    const distinct tile(id_of(a, row0 + lane));
    if (tile.left == 0) return;
    // the rows' t as products take it: values 32 s + 8 h .. + 7 of row x16; and what becomes of the results: rows 4 h + i
    const int64_t mine = row0 + 16 * wave + x16, first = row0 + 16 * wave + 4 * h;
    const int id_x = __shfl(tile.id, 16 * wave + x16);
    u32x4 high[RS], low[RS];
#pragma unroll
    for (int s = 0; s < RS; ++s) {
        const uint16_t* from = (const uint16_t*)folded + mine * wide + 8 * h + 32 * s;
        const bool in = id_x >= 0 && 32 * s < wide;
        high[s] = in ? *(const u32x4*)from : zero;
        low[s] = in ? *(const u32x4*)(from + a.rows * wide) : zero;
    }
    int id[4], back[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        id[i] = __shfl(tile.id, 16 * wave + 4 * h + i);
        back[i] = ACT == FQ_F16 && id[i] >= 0 ? ((const int32_t*)folded)[a.rows * wide + first + i] : 0;
    }
    u32x4 coming[UNITS];
    auto load = [&](int n0, int which) {
        const uint16_t* from = (const uint16_t*)a.b + ((int64_t)which * a.N + n0) * a.rank;
        const int count = min(128, a.N - n0) * units;
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
            if (i * 256 + (int)threadIdx.x < count) coming[i] = *(const u32x4*)(from + (int64_t)(i * 256 + threadIdx.x) * 8);
    };
    auto arrive = [&](char* to, int n0) {
        const int count = min(128, a.N - n0) * units;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int y = i * 256 + threadIdx.x, eight = y / (8 * units);
            if (y < count) *(u32x4*)(to + eight * 16 + y * 16) = coming[i];
        }
    };
    const int n_first = (int)blockIdx.x * turns * 128, n_end = min(a.N, n_first + turns * 128);
    // (turn, adapter) after (turn, adapter)
    distinct next = tile;
    int next_id = next.next(), next_n = n_first, buffer = 0;
    load(next_n, next_id);
    u32x4 o[4];
    f32x4 sum[8];
    bool begun = false;
    while (next_n < n_end) {
        const int now = next_id, n0 = next_n;
        if (!begun) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = id[i] >= 0 && n0 + 8 * x16 < a.N;
                o[i] = in ? __builtin_nontemporal_load((const u32x4*)((const uint16_t*)a.out + (first + i) * a.out_stride + n0 + 8 * x16)) : zero;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            begun = true;
        }
        char* weights = lds + buffer * bytes;
        arrive(weights, n0);
        next_id = next.next();
        if (next_id < 0) {
            next = tile;
            next_id = next.next();
            next_n += 128;
            begun = false;
        }
        if (next_n < n_end) load(next_n, next_id);
        __syncthreads();
        if (__any(id_x == now)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < RS; ++s) {
                    // (columns behind the last: what lies there goes into results that nobody takes)
                    const u32x4 w = 4 * s + h < units ? *(const u32x4*)(weights + x16 * group + (j * units + 4 * s + h) * 16) : zero;
                    y = mfma16<ACT>(low[s], w, y);
                    y = mfma16<ACT>(high[s], w, y);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[j][i] = id[i] == now ? y[i] : sum[j][i];
            }
        }
        buffer ^= 1;
        if (!begun && n0 + 8 * x16 < a.N) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (id[i] < 0) continue;
                u32x4 z;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float u = sum[2 * j][i], v = sum[2 * j + 1][i];
                    if (ACT == FQ_F16) u = __builtin_amdgcn_ldexpf(u, back[i]), v = __builtin_amdgcn_ldexpf(v, back[i]);
                    z[j] = pack2<ACT>(half_of<ACT, 0>(o[i][j]) + u, half_of<ACT, 1>(o[i][j]) + v);
                }
                *(u32x4*)((uint16_t*)a.out + (first + i) * a.out_stride + n0 + 8 * x16) = z;
            }
        }
    }
}

struct adapter_plan {
    bool few;
    int slots, parts;         // of the first kernel: blocks that take a tile's adapters in turn, parts of K
    int turns;                // of the second: steps of a wave, or turns of a block
    int64_t folded;           // where the folded t begins in the workspace, in floats
};

adapter_plan plan(int64_t rows, int adapters, int rank, int64_t N, int64_t K) {
    adapter_plan p;
    p.few = few_rows(rows, adapters, rank);
    const int64_t tiles = (rows + (p.few ? 15 : 63)) / (p.few ? 16 : 64), most = rows < 16 ? rows : 16;
    // More rows: of a prompt's tiles most have one adapter, some two, whose second turn is another block's (rows of 5 requests, as below: 147.6 us in all by the same, 137.8).
    p.slots = p.few ? (int)(adapters < most ? adapters : most) : adapters < 4 ? adapters : 4;
    const int64_t pieces = p.few ? (K + 31) / 32 : (K + 127) / 128, least = p.few ? 16 : 4;        // pieces of K; of a block, at least
    const int64_t wanted = p.few ? 512 / (tiles * p.slots) : 464 / tiles, fit = (pieces + least - 1) / least;
    p.parts = (int)(wanted < 1 ? 1 : wanted < fit ? wanted : fit);
    // (blocks go to the eight dies in turn: a part's columns of A stay in one die's cache; in all, eight parts 137.8 us, ten 144.7, sixteen 142.0)
    if (p.parts > 8) p.parts = p.parts / 8 * 8;
    const int64_t each = (pieces + p.parts - 1) / p.parts;
    p.parts = (int)((pieces + each - 1) / each);
    int64_t turns;
    if (p.few) {
        int lanes = 1;
        while (8 * lanes < rank) lanes *= 2;
        const int64_t steps = (N * lanes + 63) / 64;           // of a row, all columns
        // (four waves a SIMD, of four steps at least: 64 rows, N 6144, rank 16, 12.2 us in all; of one, sixteen 15.6; 16 rows four steps 8.2, of one 9.6; 64 rows of rank 64, N and K
        // 12288, 51.8, sixteen 51.0)
        turns = (rows * steps + 4095) / 4096;
        turns = turns < 4 ? 4 : turns > 32 ? 32 : turns;
    } else {
        const int64_t all = tiles * ((N + 127) / 128);
        // (eight blocks a compute unit: 2900 rows, N 36864, rank 64, 137.8 us in all; two 145.6, a turn each 148.7)
        turns = all / 2048;
        turns = turns < 1 ? 1 : turns > 8 ? 8 : turns;
    }
    p.turns = (int)turns;
    p.folded = (int64_t)p.parts * rows * ((rank + 15) / 16 * 16);
    return p;
}

int status() { return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP; }

template <int ACT, int LANES>
void up_few(const fq_adapter_args& a, const adapter_plan& p, hipStream_t stream) {
    const int64_t each = (int64_t)4 * p.turns * (64 / LANES);
    fq_adapter_up_few_kernel<ACT, LANES><<<dim3((unsigned)((a.N + each - 1) / each), (unsigned)a.rows), 256, 0, stream>>>(a, p.parts, p.turns);
}

template <int ACT>
int launch_few(const fq_adapter_args& a, const adapter_plan& p, hipStream_t stream) {
    const dim3 grid((unsigned)p.parts, (unsigned)p.slots, (unsigned)((a.rows + 15) / 16));
    if (a.rank <= 16) fq_adapter_down_few_kernel<ACT, 1><<<grid, 256, 0, stream>>>(a);
    else if (a.rank <= 32) fq_adapter_down_few_kernel<ACT, 2><<<grid, 256, 0, stream>>>(a);
    else fq_adapter_down_few_kernel<ACT, 4><<<grid, 256, 0, stream>>>(a);
    const int st = status();
    if (st != FQ_OK) return st;
    if (a.rank <= 8) up_few<ACT, 1>(a, p, stream);
    else if (a.rank <= 16) up_few<ACT, 2>(a, p, stream);
    else if (a.rank <= 32) up_few<ACT, 4>(a, p, stream);
    else if (a.rank <= 64) up_few<ACT, 8>(a, p, stream);
    else up_few<ACT, 16>(a, p, stream);
    return status();
}

template <int ACT, int RT>
int down(const fq_adapter_args& a, const adapter_plan& p, hipStream_t stream) {
    static std::atomic<uint64_t> raised{0};
    const int st = fqd::raise_lds_limit((const void*)fq_adapter_down_kernel<ACT, RT>, raised);
    if (st != FQ_OK) return st;
    const dim3 grid((unsigned)p.parts, (unsigned)((a.rows + 63) / 64), (unsigned)p.slots);
    fq_adapter_down_kernel<ACT, RT><<<grid, 256, 2 * (64 + 16 * RT) * 256, stream>>>(a);
    return status();
}

template <int ACT, int RS>
int up(const fq_adapter_args& a, const adapter_plan& p, const uint32_t* folded, hipStream_t stream) {
    static std::atomic<uint64_t> raised{0};
    const int st = fqd::raise_lds_limit((const void*)fq_adapter_up_kernel<ACT, RS>, raised);
    if (st != FQ_OK) return st;
    const int64_t groups = (a.N + 127) / 128;
    const dim3 grid((unsigned)((groups + p.turns - 1) / p.turns), (unsigned)((a.rows + 63) / 64));
    fq_adapter_up_kernel<ACT, RS><<<grid, 256, 2 * 16 * (16 * a.rank + 16), stream>>>(a, p.turns, folded);
    return status();
}

template <int ACT>
int launch(const fq_adapter_args& a, const adapter_plan& p, hipStream_t stream) {
    if (p.few) return launch_few<ACT>(a, p, stream);
    int st = a.rank <= 16 ? down<ACT, 1>(a, p, stream) : a.rank <= 32 ? down<ACT, 2>(a, p, stream) : down<ACT, 4>(a, p, stream);
    if (st != FQ_OK) return st;
    uint32_t* folded = (uint32_t*)(a.partial + p.folded);
    fq_adapter_fold_kernel<ACT><<<(unsigned)((a.rows + 15) / 16), 256, 0, stream>>>(a, p.parts, folded);
    if ((st = status()) != FQ_OK) return st;
    return a.rank <= 32 ? up<ACT, 1>(a, p, folded, stream) : a.rank <= 64 ? up<ACT, 2>(a, p, folded, stream) : up<ACT, 4>(a, p, folded, stream);
}

}  // namespace

size_t fq_adapter_bytes(int64_t rows, int adapters, int rank, int64_t N, int64_t K) {
    const adapter_plan p = plan(rows, adapters, rank, N, K);
    return ((size_t)p.folded + (p.few ? 0 : (size_t)rows * ((rank + 31) / 32 * 32 + 1))) * sizeof(float);
}

int fq_launch_adapters(int act_dtype, const fq_adapter_args& a, hipStream_t stream) {
    const adapter_plan p = plan(a.rows, a.adapters, a.rank, a.N, a.K);
    return act_dtype == FQ_F16 ? launch<FQ_F16>(a, p, stream) : launch<FQ_BF16>(a, p, stream);
}
