// Low-rank adapters of many requests beside a shared product (fq_adapters): out[m] += scale[id] (x[m] A[id]^T) B[id]^T for the adapter id of each row.
//
// Two kernels: t = x A^T in binary32, K split over blocks (each leaves partial sums), then out += scale t B^T.  Both take 16 rows at a time as the
// columns of 16 x 16 x 32 products, so that a lane's results are all one row's and a row takes those of its own adapter, whatever
// others hold: for each of a tile's different adapters the products are made for all rows.  (Requests' rows lie side by side, so that a tile
// of a prompt has one or two; single tokens have one each, and their adapters' bytes bind them, not the products.)
//
// t goes into the second product as the sum of two 16-bit numbers (16 bits and more of it), in binary16 after a division by a power of
// two that brings the row's largest to about one: nothing is lost that the result's rounding would keep.
//
// Bound by memory: A and B of each adapter, x once, the output twice.
#include <hip/hip_runtime.h>

#include "fq_internal.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int ACT> struct type16;
template <> struct type16<FQ_F16> { typedef _Float16 t; };
template <> struct type16<FQ_BF16> { typedef __bf16 t; };

template <int ACT>
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c) {
    if constexpr (ACT == FQ_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <int ACT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef typename type16<ACT>::t T;
    typedef T vec2 __attribute__((ext_vector_type(2)));
    const f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, vec2));
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

// ------------------------------------------------------------------------------------------ t = x A^T
// MT x 16 rows, RT x 16 values of t, one of blockIdx.y's turns of the tile's adapters, one of gridDim.x parts of K, which the block's four waves share out
// step by step of 32.  Results: partial[part][row][rank, rounded up to 16].
// (Two waves a SIMD at least, here and below: with them the compiler keeps the sums in ordinary registers.  Where they went to accumulation registers it
// read the first of them behind the loop without waiting for the last product.)
template <int ACT, int MT, int RT>
__global__ __launch_bounds__(256, 2) void fq_adapter_down_kernel(fq_adapter_args a) {
    constexpr int WAVES = 4, AHEAD = 4;
    __shared__ f32x4 sums[WAVES - 1][MT * RT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 4, x16 = lane & 15;
    const int64_t row0 = (int64_t)blockIdx.z * (16 * MT);
    const int ranks = (a.rank + 15) / 16 * 16, steps = (a.K + 31) / 32;
    const int part = blockIdx.x, each = (steps + (int)gridDim.x - 1) / (int)gridDim.x, begin = part * each, end = min(steps, begin + each);
    distinct tile(id_of(a, lane < 16 * MT ? row0 + lane : a.rows));
    const int mine[4] = {__shfl(tile.id, x16), __shfl(tile.id, (16 + x16) & 63), __shfl(tile.id, (32 + x16) & 63), __shfl(tile.id, (48 + x16) & 63)};
    int turn = 0;
    for (int id = tile.next(); id >= 0; id = tile.next(), ++turn) {
        if (turn % (int)gridDim.y != (int)blockIdx.y) continue;
        for (int r0 = 0; r0 < ranks; r0 += 16 * RT) {
            const uint16_t *x[MT], *w[RT];
#pragma unroll
            for (int m = 0; m < MT; ++m) x[m] = (const uint16_t*)a.x + min(row0 + 16 * m + x16, a.rows - 1) * a.x_stride + 8 * h;
#pragma unroll
            for (int r = 0; r < RT; ++r) w[r] = (const uint16_t*)a.a + ((int64_t)id * a.rank + min(r0 + 16 * r + x16, a.rank - 1)) * a.K + 8 * h;
            f32x4 t[MT][RT];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < RT; ++r) t[m][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            for (int s = begin + wave; s < end; s += WAVES * AHEAD) {
                u32x4 xs[AHEAD][MT], ws[AHEAD][RT];
                const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int k = 32 * (s + i * WAVES);
                    const bool in = s + i * WAVES < end && k + 8 * h < a.K;
#pragma unroll
                    for (int r = 0; r < RT; ++r) ws[i][r] = in ? *(const u32x4*)(w[r] + k) : zero;
#pragma unroll
                    for (int m = 0; m < MT; ++m) xs[i][m] = in ? *(const u32x4*)(x[m] + k) : zero;
                }
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int r = 0; r < RT; ++r) t[m][r] = mfma16<ACT>(ws[i][r], xs[i][m], t[m][r]);
            }
            __syncthreads();                      // (the sums of the turn before have been read)
            if (wave > 0)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int r = 0; r < RT; ++r) sums[wave - 1][m * RT + r][lane] = t[m][r];
            __syncthreads();
            if (wave > 0) continue;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int64_t row = row0 + 16 * m + x16;
#pragma unroll
                for (int r = 0; r < RT; ++r) {
#pragma unroll
                    for (int y = 0; y < WAVES - 1; ++y) t[m][r] += sums[y][m * RT + r][lane];
                    const int at = r0 + 16 * r + 4 * h;
                    if (mine[m] == id && at < a.rank) *(f32x4*)(a.partial + ((int64_t)part * a.rows + row) * ranks + at) = t[m][r];
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ out += scale t B^T
// MT x 16 rows and NJ x 16 columns a wave at a time, `turns` of them one after the other.  Column 4 i + c of product j is column (4 NJ) i + 4 j + c of
// the wave's, so that a lane has 4 NJ neighbouring ones of its row.  RS: steps of 32 ranks.
template <int ACT, int MT, int NJ, int RS>
__global__ __launch_bounds__(256, 2) void fq_adapter_up_kernel(fq_adapter_args a, int parts, int turns) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 4, x16 = lane & 15;
    const int64_t row0 = (int64_t)blockIdx.y * (16 * MT);
    const int ranks = (a.rank + 15) / 16 * 16;
    const u32x4 zero = {0, 0, 0, 0};
    distinct tile(id_of(a, lane < 16 * MT ? row0 + lane : a.rows));
    if (tile.left == 0) return;
    const int ids[4] = {__shfl(tile.id, x16), __shfl(tile.id, (16 + x16) & 63), __shfl(tile.id, (32 + x16) & 63), __shfl(tile.id, (48 + x16) & 63)};
    // the rows' t: values 32 s + 8 h .. + 7 of row 16 m + x16
    u32x4 high[MT][RS], low[MT][RS];
    float back[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int64_t row = row0 + 16 * m + x16;
        float t[RS][8], most = 0.0f;
        const float scale = ids[m] < 0 ? 0.0f : a.scales ? a.scales[ids[m]] : 1.0f;
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            f32x4 sum[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            if (ids[m] >= 0 && 32 * s + 8 * h < a.rank) {
                const float* from = a.partial + row * ranks + 32 * s + 8 * h;
                for (int p = 0; p < parts; ++p) {
                    sum[0] += *(const f32x4*)(from + (int64_t)p * a.rows * ranks);
                    sum[1] += *(const f32x4*)(from + (int64_t)p * a.rows * ranks + 4);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                t[s][i] = sum[i >> 2][i & 3] * scale;
                most = __builtin_fmaxf(most, __builtin_fabsf(t[s][i]));
            }
        }
        int e = 0;
        if (ACT == FQ_F16) {
            most = __builtin_fmaxf(most, __shfl_xor(most, 16));
            most = __builtin_fmaxf(most, __shfl_xor(most, 32));
            e = __builtin_amdgcn_frexp_expf(most);              // (0 for an infinity)
        }
        back[m] = (float)e;
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float u = t[s][2 * i], v = t[s][2 * i + 1];
                if (ACT == FQ_F16) u = __builtin_amdgcn_ldexpf(u, -e), v = __builtin_amdgcn_ldexpf(v, -e);
                high[m][s][i] = pack2<ACT>(u, v);
                const float du = u - half_of<ACT, 0>(high[m][s][i]), dv = v - half_of<ACT, 1>(high[m][s][i]);
                low[m][s][i] = pack2<ACT>(du == du ? du : 0.0f, dv == dv ? dv : 0.0f);
            }
    }
    for (int turn = 0; turn < turns; ++turn) {
        const int n0 = (((int)blockIdx.x * turns + turn) * 4 + wave) * (16 * NJ);
        if (n0 >= a.N) return;
        f32x4 sum[MT][NJ];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < NJ; ++j) sum[m][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        distinct each = tile;
        for (int id = each.next(); id >= 0; id = each.next()) {
            u32x4 w[NJ][RS];
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int n = min(n0 + 4 * NJ * (x16 >> 2) + 4 * j + (x16 & 3), a.N - 1);
                const uint16_t* from = (const uint16_t*)a.b + ((int64_t)id * a.N + n) * a.rank + 8 * h;
#pragma unroll
                for (int s = 0; s < RS; ++s) w[j][s] = 32 * s + 8 * h < a.rank ? *(const u32x4*)(from + 32 * s) : zero;
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int s = 0; s < RS; ++s) {
                        y = mfma16<ACT>(w[j][s], low[m][s], y);
                        y = mfma16<ACT>(w[j][s], high[m][s], y);
                    }
                    if (ids[m] == id) sum[m][j] = y;
                }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int64_t row = row0 + 16 * m + x16;
            if (ids[m] < 0) continue;
            uint16_t* out = (uint16_t*)a.out + row * a.out_stride;
#pragma unroll
            for (int j = 0; j < NJ; j += 2) {
                const int n = n0 + 4 * NJ * h + 4 * j;             // eight neighbouring columns
                if (n >= a.N) continue;
                u32x4 o = *(const u32x4*)(out + n);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float u = sum[m][j + i / 2][2 * i % 4], v = sum[m][j + i / 2][2 * i % 4 + 1];
                    if (ACT == FQ_F16) u = __builtin_amdgcn_ldexpf(u, (int)back[m]), v = __builtin_amdgcn_ldexpf(v, (int)back[m]);
                    o[i] = pack2<ACT>(half_of<ACT, 0>(o[i]) + u, half_of<ACT, 1>(o[i]) + v);
                }
                *(u32x4*)(out + n) = o;
            }
        }
    }
}

struct adapter_plan {
    int tall;                 // 16-row tiles of a block
    int slots, parts;         // of the first kernel: blocks that take a tile's adapters in turn, parts of K
    int wide, turns;          // of the second: 16-column products of a wave, and how often
};

adapter_plan plan(int64_t rows, int adapters, int rank, int64_t N, int64_t K) {
    adapter_plan p;
    p.tall = rows > 256 ? 4 : 1;
    const int64_t tiles = (rows + 16 * p.tall - 1) / (16 * p.tall), steps = (K + 31) / 32;
    const int64_t most = rows < 16 ? rows : 16;
    p.slots = p.tall > 1 ? (adapters < 2 ? 1 : 2) : (int)(adapters < most ? adapters : most);
    const int64_t wanted = 512 / (tiles * p.slots), fit = (steps + 15) / 16;
    p.parts = (int)(wanted < 1 ? 1 : wanted < fit ? wanted : fit);
    const int64_t each = (steps + p.parts - 1) / p.parts;
    p.parts = (int)((steps + each - 1) / each);
    p.wide = p.tall > 1 && rank <= 64 ? 4 : 2;
    const int64_t groups = (N + 64 * p.wide - 1) / (64 * p.wide);
    int64_t turns = tiles * groups / 768;
    p.turns = (int)(turns < 1 ? 1 : turns < 8 ? turns : 8);
    return p;
}

template <int ACT, int MT>
int down(const fq_adapter_args& a, const adapter_plan& p, hipStream_t stream) {
    const dim3 grid((unsigned)p.parts, (unsigned)p.slots, (unsigned)((a.rows + 16 * MT - 1) / (16 * MT)));
    if (a.rank <= 16) fq_adapter_down_kernel<ACT, MT, 1><<<grid, 256, 0, stream>>>(a);
    else if (a.rank <= 32) fq_adapter_down_kernel<ACT, MT, 2><<<grid, 256, 0, stream>>>(a);
    else fq_adapter_down_kernel<ACT, MT, 4><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

template <int ACT, int MT, int NJ>
int up(const fq_adapter_args& a, const adapter_plan& p, hipStream_t stream) {
    const int64_t groups = (a.N + 64 * NJ - 1) / (64 * NJ);
    const dim3 grid((unsigned)((groups + p.turns - 1) / p.turns), (unsigned)((a.rows + 16 * MT - 1) / (16 * MT)));
    if (a.rank <= 32) fq_adapter_up_kernel<ACT, MT, NJ, 1><<<grid, 256, 0, stream>>>(a, p.parts, p.turns);
    else if (a.rank <= 64) fq_adapter_up_kernel<ACT, MT, NJ, 2><<<grid, 256, 0, stream>>>(a, p.parts, p.turns);
    else fq_adapter_up_kernel<ACT, MT, 2, 4><<<grid, 256, 0, stream>>>(a, p.parts, p.turns);        // (p.wide is 2)
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

template <int ACT>
int launch(const fq_adapter_args& a, const adapter_plan& p, hipStream_t stream) {
    const int st = p.tall > 1 ? down<ACT, 4>(a, p, stream) : down<ACT, 1>(a, p, stream);
    if (st != FQ_OK) return st;
    return p.tall == 1 ? up<ACT, 1, 2>(a, p, stream) : p.wide == 4 ? up<ACT, 4, 4>(a, p, stream) : up<ACT, 4, 2>(a, p, stream);
}

}  // namespace

size_t fq_adapter_bytes(int64_t rows, int adapters, int rank, int64_t N, int64_t K) {
    return (size_t)plan(rows, adapters, rank, N, K).parts * rows * ((rank + 15) / 16 * 16) * sizeof(float);
}

int fq_launch_adapters(int act_dtype, const fq_adapter_args& a, hipStream_t stream) {
    const adapter_plan p = plan(a.rows, a.adapters, a.rank, a.N, a.K);
    return act_dtype == FQ_F16 ? launch<FQ_F16>(a, p, stream) : launch<FQ_BF16>(a, p, stream);
}
