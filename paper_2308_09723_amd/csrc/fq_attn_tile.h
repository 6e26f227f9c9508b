// Attention of 128 queries at a time on the matrix cores.
//
// A block is four waves of 32 queries; keys and values come through LDS in tiles of 64, the next tile's loads in flight while the
// present one is multiplied.  Both products are computed transposed, with 32 x 32 x 16 products whose columns are the wave's
// queries: S^T = K Q^T, then O^T = V^T P^T.  A lane then holds one query's scores (half of a tile's keys; lane + 32 the others), so
// that the softmax's maximum and sum need one exchange between two lanes, and the numerators leave it in the order in which the
// second product takes them: the sum over keys may be taken in any order, and V's transposed reads follow the one that S^T
// comes in.  Neither scores nor numerators pass through LDS.
//
// Running maximum: numerators are taken relative to a maximum that is renewed only when a score exceeds it by 2^8 (times
// factor), so that most tiles leave the sums alone.  binary16 numerators are 2^7 times as large, 2^7 to 2^15 for the largest score: all that
// lie within 2^-21 of it keep the type's relative error, and only below 2^-32 of it they are zeros for the product while their sum has them (relative
// to the maximum itself that is 2^-25, and 131071 keys 2^-25 below one other were missing 0.4 % of a result).
// bfloat16 numerators may be as large as binary32's: there the maximum of a tile is not even looked for until the numerators' sum
// has passed 2^60 (8192 tokens: 518 -> 508 us).  Sums that large are first made small again (level()): a factor that brings sums of
// 2^127 down to a larger maximum may lie below binary32's smallest, and nothing would be left of what is half the result.  A sum that passes 2^128
// within a tile shows in the result, and the queries are computed one by one.
//
// What a query does not see has weight zero in the products, and zero times an infinity or a NaN is a NaN: a wave whose
// results are not finite, or whose sums say that the largest score's numerator was lost, computes its queries again, one by one and seen
// keys alone (attend_one): some hundred times slower (a prompt of 2048 tokens, 32 heads over 8 of 128 values, 69 us, with a NaN among its last
// values 6.5 ms).
#ifndef FQ_ATTN_TILE_H_
#define FQ_ATTN_TILE_H_

#include "fq_attn.h"

namespace fqa {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int ACT>
__device__ inline f32x16 mfma32(const u32x4& a, const u32x4& b, const f32x16& c) {
    if constexpr (ACT == FQ_F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Values of the lane's keys that its query sees, bit 8 (i / 4) + 4 (lane / 32) + i % 4 for score i: the others become -infinity.
__device__ __forceinline__ void keep_seen(f32x16& s, uint32_t seen) {
    const uint32_t mine = seen >> ((threadIdx.x & 32) >> 3);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = mine >> (8 * (i >> 2) + (i & 3)) & 1 ? s[i] : -__builtin_inff();
}
// the lowest n bits (none below 0, all from 32 on)
__device__ inline uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// two values, rounded to nearest
template <int ACT>
__device__ inline uint32_t pack2(float a, float b) {
    typedef typename type16<ACT>::t T;
    typedef T vec2 __attribute__((ext_vector_type(2)));
    f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, vec2));
}

__device__ inline float other_half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float other_half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What all lanes hold alike, in scalar registers
__device__ inline int64_t uniform(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ inline const void* uniform(const void* p) { return (const void*)uniform((int64_t)(uintptr_t)p); }

// Direct load global -> LDS, 16 bytes per lane (lane l to base + 16 l; base wave-uniform).  Assembly, since the builtin's wait
// handling would drain every load in flight; the waits are written out.  M0 needs a wait state behind its write.
__device__ inline void load_lds16(uint32_t base, const void* src) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(base), "v"(src) : "memory", "m0");
}

// The same from an address that all lanes share + a 32-bit lane offset (bytes).  ONCE: nobody reads it again (nontemporal: the
// keys and values of a cache come in 10 % faster).
template <bool ONCE>
__device__ inline void load_lds16(uint32_t base, const void* shared, uint32_t offset) {
    const void* from = uniform(shared);
    if constexpr (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(base), "v"(offset), "s"(from) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(base), "v"(offset), "s"(from) : "memory", "m0");
}

constexpr int HALF = 32;             // keys of half a tile: the first product's rows
constexpr int KEYS = 2 * HALF;       // of a tile that a block shares
constexpr int ROWS = 128;            // queries of a block that shares its tiles

// Where 16-byte unit `unit` of key row `row` lies in a tile: units are moved about within their row so that the lanes of a read
// fall on different banks.  Keys are read 16 bytes a lane, 32 rows of one unit at a time; values eight rows x four units.
template <int UNITS>
__device__ constexpr int key_unit(int row, int unit) { return unit ^ (UNITS == 16 ? row & 15 : row >> 1 & 7); }
template <int UNITS>
__device__ constexpr int value_unit(int row, int unit) {
    return unit ^ (UNITS == 16 ? (row & 3) * 4 + (row >> 2 & 3) : (row >> 1 & 1) * 4 + (row >> 2 & 3));
}

// DP: head_dim as the matrix cores take it, 64, 96 or 128 (the rest of a head is zeros)
template <int DP>
struct tile_shape {
    static constexpr int UNITS = DP == 64 ? 8 : 16;           // 16-byte units of a row in LDS (96: four of them idle)
    static constexpr int PITCH = UNITS * 16;                  // bytes
    static constexpr int BYTES = HALF * PITCH;                // of half a tile of keys, or of values
    static constexpr int STEPS = DP / 16;                     // of the first product
    static constexpr int TILES = DP / 32;                     // of the second
};

// Sums that are not a query's whole result are left in slots: sums, not divided, four of a row together and up to 32 rows side by side, as
// a wave has them (whole lines at a time: a slot is written and read once more), then the maxima that they are relative to (log2;
// -infinity: no key seen) and the sums of numerators.
struct slot_shape {
    int rows, D;                     // rows: fewer than 32, or a multiple of them
    __host__ __device__ int64_t floats() const { return (int64_t)rows * (D + 2); }
    __device__ int at(int r, int d) const {
        const int side = rows < 32 ? rows : 32, of = r / 32;
        return ((of * (D / 4) + d / 4) * side + r - of * 32) * 4 + (d & 3);
    }
    __device__ void put_stats(float* slot, int r, float c, float l) const {
        slot[rows * D + r] = c;
        slot[rows * (D + 1) + r] = l;
    }
};
// attend_one's result, or its sums to row r of a slot
template <int ACT, typename SEES>
__device__ inline void put_one(uint16_t* out, float* slot, const slot_shape& shape, int r, const float* o, float c, float l, const SEES& sees) {
    const int lane = threadIdx.x & 63;
    if (!slot) return store_one<ACT>(out, o, l, shape.D, sees);
    if (2 * lane < shape.D) {
        float* to = slot + shape.at(r, 2 * lane);
        to[0] = o[0];
        to[1] = o[1];
    }
    if (lane == 0) shape.put_stats(slot, r, c, l);
}

// Values d .. d + 3 of a row, joined from slots.
struct partial_sums {
    float c, l;
    f32x4 o;
    __device__ void clear() {
        c = -__builtin_inff();
        l = 0.0f;
        o = {0.0f, 0.0f, 0.0f, 0.0f};
    }
    __device__ void add(float c1, float l1, const f32x4& o1) {
        const float top = __builtin_fmaxf(c, c1), base = top == -__builtin_inff() ? 0.0f : top;
        const float mine = __builtin_amdgcn_exp2f(c - base), its = __builtin_amdgcn_exp2f(c1 - base);
        c = top;
        l = l * mine + l1 * its;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = o[i] * mine + o1[i] * its;
    }
    // values d .. d + 3 of row r of slots slot(begin) .. slot(end - 1), in their order, four of them on their way at once
    template <typename SLOT>
    __device__ void add(int begin, int end, const SLOT& slot, const slot_shape& shape, int r, int d) {
        constexpr int BATCH = 4;
        const int at = shape.at(r, d), stats = shape.rows * shape.D + r;
        for (int n = begin; n < end; n += BATCH) {
            float c1[BATCH], l1[BATCH];
            f32x4 o1[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (n + i >= end) break;
                const float* from = slot(n + i);
                c1[i] = from[stats];
                l1[i] = from[stats + shape.rows];
                o1[i] = *(const f32x4*)(from + at);
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (n + i < end) add(c1[i], l1[i], o1[i]);
        }
    }
    template <int ACT, typename SEES>
    __device__ void store(uint16_t* out, const SEES& sees) const {
        const float scale = inverse(l, sees);
        const u32x2 z = {pack2<ACT>(o[0] * scale, o[1] * scale), pack2<ACT>(o[2] * scale, o[3] * scale)};
        *(u32x2*)out = z;
    }
};

// One wave's state: 32 queries (lane l: query l % 32; the wave's halves hold the same queries)
template <int ACT, int DP>
struct wave_state {
    typedef tile_shape<DP> SH;
    u32x4 q[SH::STEPS];
    f32x16 o[SH::TILES];
    bool stale;          // whether the next tile's maximum is looked for (bfloat16)
    static constexpr float LARGER = ACT == FQ_F16 ? 7.0f : 0.0f;       // the first score's numerator, log2
    float m, c, l;       // what the numerators are relative to (log2; -infinity: none yet), the same (0: none yet), this lane's sum

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int t = 0; t < SH::TILES; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
        stale = true;
        m = -__builtin_inff();
        c = l = 0.0f;
    }

    // the lane's query
    __device__ __forceinline__ void load_query(const uint16_t* row, int D) {
        const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int s = 0; s < SH::STEPS; ++s) {
            const int unit = 2 * s + half;
            const u32x4 zero = {0, 0, 0, 0};
            q[s] = unit * 8 < D ? *(const u32x4*)(row + unit * 8) : zero;
        }
    }
    // Waits for the query here, not at its first use in a loop, where the wait would take in the loads that the loop has under way.
    __device__ __forceinline__ void query_is_here() {
#pragma unroll
        for (int s = 0; s < SH::STEPS; ++s) asm volatile("" : "+v"(q[s]));
    }

    // The same out of 32 rows in LDS that lie as keys do
    __device__ __forceinline__ void read_query(const char* rows) {
        const int lane = threadIdx.x & 63, r = lane & 31;
#pragma unroll
        for (int s = 0; s < SH::STEPS; ++s) q[s] = *(const u32x4*)(rows + r * SH::PITCH + key_unit<SH::UNITS>(r, 2 * s + (lane >> 5)) * 16);
    }

    // S^T of H half-tiles of keys in LDS.  Score i of half-tile t belongs to key 32 t + 8 (i / 4) + 4 (lane / 32) + i % 4.
    template <int H, int MOST = 8>
    __device__ __forceinline__ void scores(const char* keys, f32x16 (&s)[H]) const {
        const int lane = threadIdx.x & 63, half = lane >> 5, row = lane & 31;
#pragma unroll
        for (int t = 0; t < H; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
        // keys are read AHEAD products before they are multiplied (left to itself the compiler reads them one product ahead, which
        // has every product wait for LDS)
        constexpr int N = SH::STEPS * H, AHEAD = N < MOST ? N : MOST;
        u32x4 k[AHEAD];
        auto read = [&](int n) {
            const int t = n % H, step = n / H;
            k[n % AHEAD] = *(const u32x4*)(keys + t * SH::BYTES + row * SH::PITCH + key_unit<SH::UNITS>(row, 2 * step + half) * 16);
        };
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) read(n);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            s[n % H] = mfma32<ACT>(k[n % AHEAD], q[n / H], s[n % H]);
            if (n + AHEAD < N) read(n + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // Sums of more than 2^30 made relative to as much more: to about 1 by factors that are no smaller than 2^-64.
    __device__ __forceinline__ void level() {
        const float most = other_half_max(l);
        if (!__any(most > 0x1p30f)) return;
        const float by = m + (float)__builtin_amdgcn_frexp_expf(most) - m;       // (what binary32 makes of it; 0 of a sum that is not finite)
        const float half = m == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(-0.5f * by);
        if (m != -__builtin_inff()) c = m += by;
        l = l * half * half;
#pragma unroll
        for (int t = 0; t < SH::TILES; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] = o[t][i] * half * half;
    }

    // The sum of both halves; sums that others are added to as slots and LDS hold them: no more than 2^30 times the largest numerator.
    __device__ __forceinline__ void finish(bool joined) {
        if (ACT == FQ_BF16 && joined) level();
        l = other_half_sum(l);
    }

    // Numerators of the scores, in the order that accumulate() takes; maximum, sum and results brought along.
    // WAIT: where a branch leads past the search for the maximum (bfloat16), the compiler may leave one or two wait states for the last product's scores out, and
    // four stand there.  (The build says where they are missing; a prompt of 8192 tokens has all of its own: 479.4 us without, 480.8 with.)
    template <int H, bool WAIT = true>
    __device__ __forceinline__ void soften(f32x16 (&s)[H], float factor, u32x4 (&p)[2 * H]) {
        if (ACT == FQ_F16 || stale) {
            if (ACT == FQ_BF16) level();
            float top = s[0][0];
#pragma unroll
            for (int i = 1; i < 16 * H; ++i) top = __builtin_fmaxf(top, s[i >> 4][i & 15]);
            top = other_half_max(top) * factor - LARGER;
            if (__any(top > m + 8.0f)) {
                const float now = __builtin_fmaxf(m, top), next = now == -__builtin_inff() ? 0.0f : now;
                const float again = __builtin_amdgcn_exp2f(m - next);       // (0 where there was none)
                m = now;
                c = next;
                l *= again;
#pragma unroll
                for (int t = 0; t < SH::TILES; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[t][i] *= again;
            }
        }
        if (ACT == FQ_BF16 && WAIT) {
            asm volatile("s_nop 3");
            __builtin_amdgcn_sched_barrier(0);
        }
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < H; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], factor, -c));
                sum[i & 1] += s[t][i];
            }
#pragma unroll
            for (int i = 0; i < 16; i += 2) p[2 * t + i / 8][i / 2 % 4] = pack2<ACT>(s[t][i], s[t][i + 1]);
        }
        const float both = sum[0] + sum[1];
        l += both;
        if (ACT == FQ_BF16) stale = __any(both > 0x1p60f || m == -__builtin_inff());
    }

    // O^T += V^T P^T over H half-tiles of values in LDS.  V^T: lane l takes column l % 32 of 32; a transposed read hands each lane
    // four keys of its column, out of four rows of which each lane of sixteen points at a quarter.
    template <int H>
    __device__ __forceinline__ void accumulate(const char* values, const u32x4 (&p)[2 * H]) {
        const int lane = threadIdx.x & 63;
        const int row = 4 * (lane >> 5) + (lane & 15) / 4, unit = 2 * (lane >> 4 & 1) + (lane >> 1 & 1), in = (lane & 1) * 8;
#pragma unroll
        for (int k = 0; k < 2 * H; ++k)
#pragma unroll
            for (int t = 0; t < SH::TILES; ++t) {
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = row + 8 * e;
                    const char* at = values + (16 * k + r) * SH::PITCH + value_unit<SH::UNITS>(r, 4 * t + unit) * 16 + in;
                    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4*)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)at);
                    const u32x2 y = __builtin_bit_cast(u32x2, x);
                    v[2 * e] = y[0];
                    v[2 * e + 1] = y[1];
                }
                o[t] = mfma32<ACT>(v, p[k], o[t]);
            }
    }

    // what the sums are relative to (log2), -infinity where there are none
    __device__ __forceinline__ float top() const { return m; }

    // Whether every sum of the wave's queries is finite, and the largest numerator of each what it should be: a score is taken less the reference
    // exactly, but the reference is rounded, and from 2^31 on half a unit of it may make all numerators zeros.
    __device__ __forceinline__ bool sound() const {
        float x = l >= 0.25f || m == -__builtin_inff() ? l * 0.0f : 1.0f;
#pragma unroll
        for (int t = 0; t < SH::TILES; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) x = __builtin_fmaf(o[t][i], 0.0f, x);
        return __all(x == 0.0f);
    }

    // The lane's query's result, or its sums to row r of a slot.  sees(): whether the query sees a key.
    template <typename SEES>
    __device__ __forceinline__ void put(uint16_t* out, float* slot, const slot_shape& shape, int r, const SEES& sees) const {
        if (slot) {
            float* to = slot + shape.at(r, (threadIdx.x & 32) >> 3);
            const int step = shape.at(0, 8);
            quads([&](int d, int i, int t) {
                const f32x4 z = {o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
                if (d < shape.D) *(f32x4*)(to + (4 * t + i / 4) * step) = z;
            });
            if ((threadIdx.x & 32) == 0) shape.put_stats(slot, r, top(), l);
            return;
        }
        const float scale = inverse(l, sees);
        quads([&](int d, int i, int t) {
            const u32x2 z = {pack2<ACT>(o[t][i] * scale, o[t][i + 1] * scale), pack2<ACT>(o[t][i + 2] * scale, o[t][i + 3] * scale)};
            if (d < shape.D) *(u32x2*)(out + d) = z;
        });
    }

    // The wave's results to rows out(r) (32 of them, `count` there), whole lines at a time: through 32 rows of LDS of its own, where the
    // lanes of a store find neighbouring values (stored as the lanes have them a line takes eight writes).
    template <typename OUT, typename SEES>
    __device__ __forceinline__ void put_rows(char* mine, const OUT& out, int count, int D, const SEES& sees) const {
        const int lane = threadIdx.x & 63;
        const float scale = inverse(l, sees);
        quads([&](int d, int i, int t) {
            const u32x2 z = {pack2<ACT>(o[t][i] * scale, o[t][i + 1] * scale), pack2<ACT>(o[t][i + 2] * scale, o[t][i + 3] * scale)};
            const int r = lane & 31;
            *(u32x2*)(mine + r * SH::PITCH + key_unit<SH::UNITS>(r, d / 8) * 16 + (d & 4) * 2) = z;
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the wave's own: no barrier)
        constexpr int STEP = 64 / SH::UNITS;
        const int unit = lane % SH::UNITS;
#pragma unroll 2
        for (int j = 0; j < 32 / STEP; ++j) {
            const int r = lane / SH::UNITS + j * STEP;
            const u32x4 z = *(const u32x4*)(mine + r * SH::PITCH + key_unit<SH::UNITS>(r, unit) * 16);
            if (r < count && unit * 8 < D) *(u32x4*)(out(r) + unit * 8) = z;
        }
    }

    // f(d, i, t): the lane's results i .. i + 3 of block t are values d .. d + 3 of its query
    template <typename F>
    __device__ __forceinline__ static void quads(F f) {
        const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int t = 0; t < SH::TILES; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4) f(32 * t + 2 * i + 4 * half, i, t);
    }
};

}  // namespace fqa

#endif  // FQ_ATTN_TILE_H_
