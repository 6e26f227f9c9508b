// Attention of drafted tokens over a cache held in 4 bits (fq_attention_tree_kv4; what the cache holds: fq_kv4.h).
//
// Work is dealt out as over a cache of 16 bits (fq_attn_units.h).  A key and its value are 1.125 D bytes, and taking their codes to 16 bits
// is 2 D / 8 times 9 instructions, beside 4 D operations for each row on the matrix cores: with few rows the cache's bytes and
// the conversions bind it about equally.  A token each of 64 sequences of 100 - 8191, 8 heads of 128, four rows each: 123 MB in 28.5 us, 4.3 TB/s (bytes 17.5 at the rate of
// a kernel that only reads; 5 us of it are blocks' beginnings), 7.0 to join, binary16 30.8 and 7.2; over 16 bits 76 and 7.4.  8 and 16 rows 39.8 (binary16 37.6), 32 58 (54), and 9 - 11.
//
// Up to 32 rows (fq_attention_kv4_stream_kernel) every wave brings 32 keys at a time into LDS of its own, as they lie in the cache: a
// record of 16 tokens is what one product of 16 x 16 x 32 takes, lane by lane.  S^T = K Q^T goes over the keys' codes, group by group, and
// a group's products are multiplied by its scales in binary32.  The numerators leave S^T in the order in which O^T = V^T P^T takes them.
// binary16 values are code times scale, exactly; bfloat16 has no packed multiplication, and there the numerators are multiplied by the
// values' scales instead, before they are rounded, once, as they are anyway.
//
// Above 32 rows (fq_attention_kv4_tile_kernel) the waves of a block take a tile's codes to 16 bits once, each a record, into tiles that all of them read: keys
// as over a cache of 16 bits, values turned over (a lane has four tokens of a value).  Bound by instructions: for 32 rows and 64 keys a wave has 32 products, 170
// instructions' time for the numerators and, of four waves, 200 for the codes, of eight 100.  Pieces of 700 tokens over 2500 - 3900, two sequences, 32 heads over 8: 131 us with
// the join where the card has been at rest, 0.73 PFLOP/s, 145 one call after the other (in a trace 134 and 17, binary16 144 and 17); over 16 bits 143.
#include <hip/hip_runtime.h>
#include <atomic>

#include "fq_attn_units.h"
#include "fq_kv4.h"
#include "fq_lds_limit.h"

namespace {

using namespace fqa;
using namespace fqkv;

// One key head's keys and values of a sequence, one at a time.
struct kv4_rows {
    const char* head;
    int64_t page_stride;
    const int32_t* table;
    uint32_t page_size, last_page;
    int S;

    // (cache.k: the pages; strides of a page and of a head in bytes)
    __device__ static kv4_rows of(const fq_tree_args& a, int b, int head) {
        kv4_rows x;
        x.head = (const char*)a.cache.k + head * a.cache.head_stride;
        x.page_stride = a.cache.page_stride;
        x.table = a.page_table + b * a.table_width;
        x.page_size = (uint32_t)a.cache.page_size;
        x.last_page = (uint32_t)(a.cache.pages - 1);
        x.S = groups_of(a.head_dim);
        return x;
    }
    __device__ const char* record(int j) const {
        const uint32_t n = (uint32_t)j / page_size, at = (uint32_t)j - n * page_size;
        const int32_t page = table[n];
        return head + (int64_t)(page < 0 ? 0u : min((uint32_t)page, last_page)) * page_stride + (int64_t)(at / RECORD) * record_bytes(S);
    }
    template <int ACT>
    __device__ float dot(const uint16_t* q, int j, int D) const {
        typedef typename type16<ACT>::t T;
        const char* from = record(j);
        const int token = j % RECORD;             // (pages are whole records)
        float sum = 0.0f;
        for (int c = 0; c < D; c += 8) {
            const float s = (float)*(const T*)(from + scale_at(S, token, c / 32));
            const uint32_t x = *(const uint32_t*)(from + key_at(S, token, c / 32, c / 8 % 4)), first = firsts(x), second = seconds(x);
            for (int i = 0; i < 4; ++i) {
                sum = __builtin_fmaf((float)((const T*)q)[c + i], decoded(first >> 8 * i & 0xffu) * s, sum);
                sum = __builtin_fmaf((float)((const T*)q)[c + 4 + i], decoded(second >> 8 * i & 0xffu) * s, sum);
            }
        }
        return sum;
    }
    template <int ACT>
    __device__ void two(int j, int d, float* v) const {
        typedef typename type16<ACT>::t T;
        const char* from = record(j);
        const int token = j % RECORD;
        const float s = (float)*(const T*)(from + 32 * S + scale_at(S, token, d / 32));
        for (int i = 0; i < 2; ++i) {
            const uint32_t x = *(const uint8_t*)(from + value_at(S, token, d / 32, d % 16 + i));
            v[i] = decoded(d % 32 < 16 ? x & 0x87u : from_second(x)) * s;
        }
    }
};

template <int ACT>
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c) {
    if constexpr (ACT == FQ_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The four lanes that hold a row (16 apart)
__device__ __forceinline__ float row_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return other_half_max(__builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float row_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return other_half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Two 16-bit numbers
template <int ACT, int HIGH>
__device__ __forceinline__ float half_of(uint32_t x) {
    if constexpr (ACT == FQ_F16) {
        typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
        return (float)__builtin_bit_cast(vec2, x)[HIGH];
    } else {
        return __uint_as_float(HIGH ? x & 0xffff0000u : x << 16);
    }
}
__device__ __forceinline__ uint32_t times16(uint32_t a, uint32_t b) {
    typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(vec2, a) * __builtin_bit_cast(vec2, b));
}

// Whether a 16-byte unit of a query has a value of 2^120 or more: a group's codes (up to 7, 32 of them) times those may pass 2^128 where keys, codes times scales, do not, and a
// score of -infinity would pass for one that counts nothing.  (bfloat16; such rows are computed one by one.)
__device__ __forceinline__ bool beyond_codes(const u32x4& q) {
    typedef uint16_t vec2 __attribute__((ext_vector_type(2)));
    vec2 m = __builtin_bit_cast(vec2, q[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(vec2, q[i] & 0x7fff7fffu));
    return (m[0] > m[1] ? m[0] : m[1]) >= 0x7b80;
}

// Of four neighbouring tokens' scales (two words) those of the first `count`: what lies behind the last key may be anything.
__device__ __forceinline__ uint32_t first_mask(int count) { return count >= 2 ? ~0u : count == 1 ? 0xffffu : 0u; }

// N words in LDS from a place that is aligned to 4 (N odd), 8 or 16 bytes
template <int N>
__device__ __forceinline__ void read_words(const char* p, uint32_t (&x)[N]) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 v = *(const u32x4*)(p + 4 * i);
            x[i] = v[0], x[i + 1] = v[1], x[i + 2] = v[2], x[i + 3] = v[3];
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const u32x2 v = *(const u32x2*)(p + 4 * i);
            x[i] = v[0], x[i + 1] = v[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = ((const uint32_t*)p)[i];
    }
}

// Where a part's records lie: the entries of the page table that the wave has in LDS.
struct record_places {
    const int32_t* entries;
    uint32_t first;                  // entry 0's place in the table
    divisor by_records;              // of a page
    int records;
    const char* head;
    int64_t page_stride;

    // record r (keys 16 r .. 16 r + 15), the same for all lanes
    template <int BYTES>
    __device__ __forceinline__ const void* place(int r) const {
        const int n = by_records.quotient(r);
        return uniform(head + entries[(uint32_t)n - first] * page_stride + (int64_t)(r - n * records) * BYTES);
    }
};

// Loads of a record: 36 S units of 16 bytes
template <int S>
struct record_loads {
    static constexpr int COUNT = (36 * S + 63) / 64;
    __device__ static __forceinline__ void issue(uint32_t to, const void* from) {
        const uint32_t lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            if (i * 64 + (int)lane < 36 * S) load_lds16<true>(to + i * 1024, (const char*)from + i * 1024, lane * 16);
    }
};

// ------------------------------------------------------------------------------------------ up to 32 rows
// One wave's NT x 16 rows (lane 16 h + x: row x of each 16; of a record's keys 4 h .. 4 h + 3)
template <int ACT, int S, int TILES>
struct few_rows {
    static constexpr int NT = TILES, RECORDS = 2, RING = 4;             // records of a step; steps that a wave's ring has room for
    static constexpr float LARGER = ACT == FQ_F16 ? 7.0f : 0.0f;       // the first score's numerator, log2
    u32x4 q[NT][S];
    f32x4 o[NT][2 * S];              // values 16 i + 4 h .. + 3 of the lane's row
    float m[NT], c[NT], l[NT];       // as wave_state's
    bool stale, beyond;              // beyond: beyond_codes(), of any row

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < 2 * S; ++i) o[n][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            m[n] = -__builtin_inff();
            c[n] = l[n] = 0.0f;
        }
        stale = true;
        beyond = false;
    }
    template <typename ROWS>
    __device__ __forceinline__ void load_query(const ROWS& rows, int D) {
        const int h = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint16_t* row = rows.query(min(16 * n + own_row(), rows.count - 1));
#pragma unroll
            for (int t = 0; t < S; ++t) {
                const int d = 32 * t + 8 * h;
                q[n][t] = d < D ? *(const u32x4*)(row + d) : u32x4{0, 0, 0, 0};
            }
        }
    }
    __device__ __forceinline__ void pass_query(char*) {}
    __device__ __forceinline__ void take_query(const char*) {}
    // (waits for the queries here: see wave_state)
    __device__ __forceinline__ void query_is_here() {
        bool any = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < S; ++t) {
                asm volatile("" : "+v"(q[n][t]));
                if (ACT == FQ_BF16) any = any || beyond_codes(q[n][t]);
            }
        beyond = __any(any);
    }

    // S^T of a record: score r belongs to key 4 h + r
    __device__ __forceinline__ void scores(const char* record, f32x4 (&s)[NT]) const {
        const int lane = threadIdx.x & 63, h = lane >> 4;
        uint32_t k[S], scale[2 * S];
        read_words(record + lane * 4 * S, k);
        read_words(record + 512 * S + h * 8 * S, scale);
#pragma unroll
        for (int n = 0; n < NT; ++n) s[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const uint32_t first = firsts(k[t]), second = seconds(k[t]);
            const u32x4 x = {codes16<ACT, false>(first), codes16<ACT, true>(first), codes16<ACT, false>(second), codes16<ACT, true>(second)};
            const float by[4] = {half_of<ACT, 0>(scale[2 * t]), half_of<ACT, 1>(scale[2 * t]), half_of<ACT, 0>(scale[2 * t + 1]), half_of<ACT, 1>(scale[2 * t + 1])};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f32x4 y = mfma16<ACT>(x, q[n][t], f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                for (int r = 0; r < 4; ++r) s[n][r] = __builtin_fmaf(y[r], by[r], s[n][r]);
            }
        }
    }

    // Sums of more than 2^30 made relative to as much more (see wave_state)
    __device__ __forceinline__ void level(int n) {
        const float most = row_max(l[n]);
        if (!__any(most > 0x1p30f)) return;
        const float by = m[n] + (float)__builtin_amdgcn_frexp_expf(most) - m[n];
        const float half = m[n] == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(-0.5f * by);
        if (m[n] != -__builtin_inff()) c[n] = m[n] += by;
        l[n] = l[n] * half * half;
#pragma unroll
        for (int i = 0; i < 2 * S; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[n][i][r] = o[n][i][r] * half * half;
    }

    // Numerators of the scores of two records in place; maximum, sum and results brought along (see wave_state)
    __device__ __forceinline__ void soften(f32x4 (&s)[2][NT], float factor) {
        bool large = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (ACT == FQ_F16 || stale) {
                if (ACT == FQ_BF16) level(n);
                float top = s[0][n][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = __builtin_fmaxf(top, s[i >> 2][n][i & 3]);
                top = row_max(top) * factor - LARGER;
                if (__any(top > m[n] + 8.0f)) {
                    const float now = __builtin_fmaxf(m[n], top), next = now == -__builtin_inff() ? 0.0f : now;
                    const float again = __builtin_amdgcn_exp2f(m[n] - next);
                    m[n] = now;
                    c[n] = next;
                    l[n] *= again;
#pragma unroll
                    for (int i = 0; i < 2 * S; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[n][i][r] *= again;
                }
            }
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 2][n][i & 3], factor, -c[n]));
                s[i >> 2][n][i & 3] = x;
                sum += x;
            }
            l[n] += sum;
            large = large || sum > 0x1p58f || m[n] == -__builtin_inff();
        }
        if (ACT == FQ_BF16) stale = __any(large);
    }

    // O^T += V^T P^T over two records, of whose values the first `there` are keys
    __device__ __forceinline__ void accumulate(const char* record0, const char* record1, const f32x4 (&p)[2][NT], bool tail, int there) {
        const int lane = threadIdx.x & 63, h = lane >> 4;
        const char* record[2] = {record0, record1};
        uint32_t v[2][S], scale[2][2 * S];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            read_words(record[u] + 256 * S + lane * 4 * S, v[u]);
            read_words(record[u] + 544 * S + h * 8 * S, scale[u]);
        }
        if (tail) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int count = there - 16 * u - 4 * h;
#pragma unroll
                for (int g = 0; g < S; ++g) {
                    scale[u][2 * g] &= first_mask(count);
                    scale[u][2 * g + 1] &= first_mask(count - 2);
                }
            }
        }
        u32x4 x[NT];
        auto pack = [&](int g) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float a = p[u][n][2 * i], b = p[u][n][2 * i + 1];
                        if constexpr (ACT == FQ_BF16) {
                            a *= half_of<ACT, 0>(scale[u][2 * g + i]);
                            b *= half_of<ACT, 1>(scale[u][2 * g + i]);
                        }
                        x[n][2 * u + i] = pack2<ACT>(a, b);
                    }
        };
        if (ACT == FQ_F16) pack(0);
#pragma unroll
        for (int j = 0; j < S; ++j) {
            if (ACT == FQ_BF16) pack(j);
            u32x4 first, second;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t f = firsts(v[u][j]), g = seconds(v[u][j]);
                first[2 * u] = codes16<ACT, false>(f);
                first[2 * u + 1] = codes16<ACT, true>(f);
                second[2 * u] = codes16<ACT, false>(g);
                second[2 * u + 1] = codes16<ACT, true>(g);
                if constexpr (ACT == FQ_F16) {
                    first[2 * u] = times16(first[2 * u], scale[u][2 * j]);
                    first[2 * u + 1] = times16(first[2 * u + 1], scale[u][2 * j + 1]);
                    second[2 * u] = times16(second[2 * u], scale[u][2 * j]);
                    second[2 * u + 1] = times16(second[2 * u + 1], scale[u][2 * j + 1]);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                o[n][2 * j] = mfma16<ACT>(first, x[n], o[n][2 * j]);
                o[n][2 * j + 1] = mfma16<ACT>(second, x[n], o[n][2 * j + 1]);
            }
        }
    }

    // The rows that a lane has scores of: row 16 n + its own
    __device__ __forceinline__ static int own_row() { return threadIdx.x & 15; }

    // A step's records, of which the first `there` keys are keys; those of the row that are seen: seen(row, key)
    template <typename SEEN>
    __device__ __forceinline__ void step(char* at, float factor, bool masked, int there, const SEEN& seen) {
        const int h = (threadIdx.x & 63) >> 4;
        f32x4 s[2][NT];
        scores(at, s[0]);
        scores(at + record_bytes(S), s[1]);
        if (masked) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint32_t bits = seen(n, 0) >> 4 * h;
#pragma unroll
                for (int x = 0; x < 8; ++x) s[x >> 2][n][x & 3] = bits >> (16 * (x >> 2) + (x & 3)) & 1 ? s[x >> 2][n][x & 3] : -__builtin_inff();
            }
        }
        soften(s, factor);
        accumulate(at, at + record_bytes(S), s, there < 32, there);
    }

    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (ACT == FQ_BF16) level(n);
            l[n] = row_sum(l[n]);
        }
    }
    __device__ __forceinline__ bool sound() const {
        float x = 0.0f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            x = __builtin_fmaf(l[n], 0.0f, x);
            if (!(l[n] >= 0.25f || m[n] == -__builtin_inff())) x = 1.0f;
#pragma unroll
            for (int i = 0; i < 2 * S; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) x = __builtin_fmaf(o[n][i][r], 0.0f, x);
        }
        return __all(x == 0.0f) && !beyond;
    }
};

// Four rows: S^T by products of 4 x 4 x 4, sixteen at once, so that no column is a row that is not there (lane 4 b + j: row j; keys 4 b .. 4 b + 3 of
// a step of 64, of whose values the lane converts its own key's).  Scores, scales and numerators are a quarter of the instructions then.  The
// numerators go through LDS (where the keys' codes lay) into the order of the 16 x 16 x 32 products for O^T, whose columns are the four rows, four times.
template <int ACT>
__device__ __forceinline__ f32x4 mfma4(const u32x2& a, const u32x2& b, const f32x4& c) {
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    if constexpr (ACT == FQ_F16)
        return __builtin_amdgcn_mfma_f32_4x4x4f16(__builtin_bit_cast(f16x4, a), __builtin_bit_cast(f16x4, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
}

template <int ACT, int S>
struct four_rows {
    static constexpr int NT = 1, RECORDS = 4, RING = 2;
    static constexpr float LARGER = ACT == FQ_F16 ? 7.0f : 0.0f;
    static constexpr int BYTES = record_bytes(S);
    u32x2 q[S][4][2];                // [t][a][half]: values 32 t + 8 a + 4 half .. + 3 of row j
    f32x4 o[1][2 * S];               // values 16 i + 4 h .. + 3 of row (lane % 16) % 4
    float m[1], c[1], l[1];
    bool stale, beyond;

    __device__ __forceinline__ static int own_row() { return threadIdx.x & 3; }
    __device__ __forceinline__ static float rows_max(float x) {      // over the lanes of a row
        x = __builtin_fmaxf(x, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x124, 0xf, 0xf, true)));       // 4 lanes on in the row of 16
        x = __builtin_fmaxf(x, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x128, 0xf, 0xf, true)));       // 8
        return row_max(x);
    }
    __device__ __forceinline__ static float rows_sum(float x) {
        x += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x124, 0xf, 0xf, true));
        x += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x128, 0xf, 0xf, true));
        return row_sum(x);
    }

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 2 * S; ++i) o[0][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        m[0] = -__builtin_inff();
        c[0] = l[0] = 0.0f;
        stale = true;
        beyond = false;
    }
    // Each lane loads 16 bytes of the four rows and takes its row out of LDS (loaded as they are needed, a row 16 times, they took 3 us)
    u32x4 loaded;
    template <typename ROWS>
    __device__ __forceinline__ void load_query(const ROWS& rows, int D) {
        const int lane = threadIdx.x & 63, d = (lane & 15) * 8;
        loaded = d < D ? *(const u32x4*)(rows.query(min(lane >> 4, rows.count - 1)) + d) : u32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void query_is_here() {
        asm volatile("" : "+v"(loaded));
        beyond = ACT == FQ_BF16 && __any(beyond_codes(loaded));
    }
    __device__ __forceinline__ void pass_query(char* room) {
        const int lane = threadIdx.x & 63;
        if ((lane & 15) < 4 * S) *(u32x4*)(room + ((lane >> 4) * 4 * S + (lane & 15)) * 16) = loaded;
    }
    __device__ __forceinline__ void take_query(const char* room) {
#pragma unroll
        for (int t = 0; t < S; ++t)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const u32x4 x = *(const u32x4*)(room + (own_row() * 4 * S + 4 * t + a) * 16);
                q[t][a][0] = u32x2{x[0], x[1]};
                q[t][a][1] = u32x2{x[2], x[3]};
            }
    }
    __device__ __forceinline__ void again(float by) {
#pragma unroll
        for (int i = 0; i < 2 * S; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[0][i][r] *= by;
    }
    __device__ __forceinline__ void level() {
        const float most = rows_max(l[0]);
        if (!__any(most > 0x1p30f)) return;
        const float by = m[0] + (float)__builtin_amdgcn_frexp_expf(most) - m[0];
        const float half = m[0] == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(-0.5f * by);
        if (m[0] != -__builtin_inff()) c[0] = m[0] += by;
        l[0] = l[0] * half * half;
        again(half);
        again(half);
    }

    template <typename SEEN>
    __device__ __forceinline__ void step(char* at, float factor, bool masked, int there, const SEEN& seen) {
        const int lane = threadIdx.x & 63, b = lane >> 2, x16 = lane & 15, h = lane >> 4;
        // scores of keys 4 b + i; the lane brings in key `lane`
        f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
        char* own = at + (b >> 2) * BYTES;             // the record of the lane's scores
        {
            const char* from = at + h * BYTES + x16 * 4 * S;
            uint32_t k[4][S], scale[2 * S];
#pragma unroll
            for (int a = 0; a < 4; ++a) read_words(from + a * 64 * S, k[a]);
            read_words(own + 512 * S + (b & 3) * 8 * S, scale);
            f32x4 y[S];
#pragma unroll
            for (int t = 0; t < S; ++t) y[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int t = 0; t < S; ++t) {
                    const uint32_t first = firsts(k[a][t]), second = seconds(k[a][t]);
                    y[t] = mfma4<ACT>(u32x2{codes16<ACT, false>(first), codes16<ACT, true>(first)}, q[t][a][0], y[t]);
                    y[t] = mfma4<ACT>(u32x2{codes16<ACT, false>(second), codes16<ACT, true>(second)}, q[t][a][1], y[t]);
                }
#pragma unroll
            for (int t = 0; t < S; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[i] = __builtin_fmaf(y[t][i], i & 1 ? half_of<ACT, 1>(scale[2 * t + i / 2]) : half_of<ACT, 0>(scale[2 * t + i / 2]), s[i]);
        }
        if (masked) {
            const uint32_t first = seen(0, 0), last = seen(0, 32), bits = (b < 8 ? first : last) >> (4 * b & 31);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = bits >> i & 1 ? s[i] : -__builtin_inff();
        }
        // numerators (see wave_state)
        if (ACT == FQ_F16 || stale) {
            if (ACT == FQ_BF16) level();
            const float top = rows_max(__builtin_fmaxf(__builtin_fmaxf(s[0], s[1]), __builtin_fmaxf(s[2], s[3]))) * factor - LARGER;
            if (__any(top > m[0] + 8.0f)) {
                const float now = __builtin_fmaxf(m[0], top), next = now == -__builtin_inff() ? 0.0f : now;
                const float by = __builtin_amdgcn_exp2f(m[0] - next);
                m[0] = now;
                c[0] = next;
                l[0] *= by;
                again(by);
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], factor, -c[0]));
            sum += s[i];
        }
        l[0] += sum;
        if (ACT == FQ_BF16) stale = __any(sum > 0x1p58f || m[0] == -__builtin_inff());
        // to LDS, as products with the values' scales in bfloat16: [record][group][token / 4][row]
        constexpr int GROUPS = ACT == FQ_BF16 ? S : 1;
        {
            uint32_t scale[2 * S];
            if constexpr (ACT == FQ_BF16) {
                read_words(own + 544 * S + (b & 3) * 8 * S, scale);
                if (there < 64) {                      // what lies behind the last key may be anything
#pragma unroll
                    for (int g = 0; g < S; ++g) {
                        scale[2 * g] &= first_mask(there - 4 * b);
                        scale[2 * g + 1] &= first_mask(there - 4 * b - 2);
                    }
                }
            }
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                u32x2 p;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float x = s[2 * i], y = s[2 * i + 1];
                    if constexpr (ACT == FQ_BF16) {
                        x *= half_of<ACT, 0>(scale[2 * g + i]);
                        y *= half_of<ACT, 1>(scale[2 * g + i]);
                    }
                    p[i] = pack2<ACT>(x, y);
                }
                *(u32x2*)(own + g * 128 + (lane & 15) * 8) = p;        // (lane % 16: 4 (b % 4) + j)
            }
        }
        // O^T += V^T P^T, two records at a time
#pragma unroll
        for (int pair = 0; pair < 2; ++pair) {
            const char* record[2] = {at + 2 * pair * BYTES, at + (2 * pair + 1) * BYTES};
            uint32_t v[2][S], scale[2][2 * S];
            u32x2 p[GROUPS][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                read_words(record[u] + 256 * S + lane * 4 * S, v[u]);
                if constexpr (ACT == FQ_F16) {
                    read_words(record[u] + 544 * S + h * 8 * S, scale[u]);
                    if (there < 64) {
                        const int count = there - 32 * pair - 16 * u - 4 * h;
#pragma unroll
                        for (int g = 0; g < S; ++g) {
                            scale[u][2 * g] &= first_mask(count);
                            scale[u][2 * g + 1] &= first_mask(count - 2);
                        }
                    }
                }
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) p[g][u] = *(const u32x2*)(record[u] + g * 128 + (4 * h + (x16 & 3)) * 8);
            }
#pragma unroll
            for (int j = 0; j < S; ++j) {
                u32x4 first, second;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t f = firsts(v[u][j]), g = seconds(v[u][j]);
                    first[2 * u] = codes16<ACT, false>(f);
                    first[2 * u + 1] = codes16<ACT, true>(f);
                    second[2 * u] = codes16<ACT, false>(g);
                    second[2 * u + 1] = codes16<ACT, true>(g);
                    if constexpr (ACT == FQ_F16) {
                        first[2 * u] = times16(first[2 * u], scale[u][2 * j]);
                        first[2 * u + 1] = times16(first[2 * u + 1], scale[u][2 * j + 1]);
                        second[2 * u] = times16(second[2 * u], scale[u][2 * j]);
                        second[2 * u + 1] = times16(second[2 * u + 1], scale[u][2 * j + 1]);
                    }
                }
                const int g = ACT == FQ_BF16 ? j : 0;
                const u32x4 x = {p[g][0][0], p[g][0][1], p[g][1][0], p[g][1][1]};
                o[0][2 * j] = mfma16<ACT>(first, x, o[0][2 * j]);
                o[0][2 * j + 1] = mfma16<ACT>(second, x, o[0][2 * j + 1]);
            }
        }
    }

    __device__ __forceinline__ void finish() {
        if (ACT == FQ_BF16) level();
        l[0] = rows_sum(l[0]);
    }
    __device__ __forceinline__ bool sound() const {
        float x = l[0] >= 0.25f || m[0] == -__builtin_inff() ? l[0] * 0.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < 2 * S; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) x = __builtin_fmaf(o[0][i][r], 0.0f, x);
        return __all(x == 0.0f) && !beyond;
    }
};

// A block's four waves are HEADS key heads x PARTS parts of a tile of 32 PARTS keys; where they share the keys out, they join their sums through
// LDS at the end of a piece.  A wave's ring has RING times two records, all but one of them on their way while that one is used.
template <int ACT, int S, typename STATE, int HEADS>
__global__ __launch_bounds__(256, 2) void fq_attention_kv4_stream_kernel(fq_tree_args a, tree_plan p, divisor by_records) {
    constexpr int NT = STATE::NT, RECORDS = STATE::RECORDS, BYTES = record_bytes(S), RING = STATE::RING, STEP = RECORDS * BYTES, WAVE_BYTES = RING * STEP;
    constexpr int APART = RECORDS * record_loads<S>::COUNT, TOGETHER = record_loads<RECORDS * S>::COUNT;       // loads of a step
    constexpr int WIDE = RECORD * RECORDS, PARTS = 4 / HEADS, TILE = WIDE * PARTS, QUADS = 8 * S;              // QUADS: fours of a row's values
    constexpr int TURN = QUADS == 24 || QUADS == 8 ? 7 : 15;
    static_assert(NT * 16 * QUADS * 16 <= WAVE_BYTES, "the sums of a wave fit its ring");
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 4;
    const int head = wave % HEADS, part_of = wave / HEADS;
    int32_t* entries = (int32_t*)(lds + 4 * WAVE_BYTES) + wave * (TABLE / 4);
    float* stats = (float*)(lds + 4 * WAVE_BYTES + TABLE * 4);       // [4][32][2], and a flag
    const int D = a.head_dim;
    const bool together = a.cache.page_size % WIDE == 0;         // a step's records lie one behind the other
    char* mine = lds + wave * WAVE_BYTES;
    const uint32_t mine_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine;

    const line all(a, p);
    const int64_t begin = blockIdx.x * all.per_block, stop = min(all.total, begin + all.per_block);
    if (begin >= stop) return;
    int b;
    int64_t at_b;
    all.find(begin, &b, &at_b);
    int context = all.context(b), tiles = tiles_of(a, p, context);
    int u = (int)quotient(begin - at_b, tiles + p.extra), t0 = (int)(begin - at_b - (int64_t)u * (tiles + p.extra));
    STATE w;

    for (int64_t pos = begin; pos < stop;) {
        const unit_rows<kv4_rows> rows(a, p, b, u, head, context);
        const int t1 = (int)min((int64_t)tiles, t0 + stop - pos);
        if (t0 < tiles) {                               // (behind them are places that hold nothing)
        const int key0 = t0 * TILE, key1 = p.whole ? rows.keys : min(rows.keys, t1 * TILE);
        w.load_query(rows, D);
        w.clear();
        const int most = part_keys(TABLE / 4, a.cache.page_size, TILE);
        for (int part = key0, part_end; part < key1; part = part_end) {
            part_end = fqa::part_end(part, key1, most);
            const table_part table = load_table<64>(a, b, part, part_end, entries);
            char* room = mine + (RING - 1) * STEP;      // (the step that comes in last)
            if (part == key0) {
                w.query_is_here();                      // (with the table)
                w.pass_query(room);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the wave's own: no barrier)
            const record_places places = {entries, table.first, by_records, a.cache.page_size / RECORD,
                                          (const char*)a.cache.k + rows.head * a.cache.head_stride, a.cache.page_stride};
            const int last = (part_end - 1) / RECORD;
            const int base0 = part + part_of * WIDE, steps = base0 < part_end ? (part_end - base0 + TILE - 1) / TILE : 0;
            auto load = [&](int i) {
                const int r = (base0 + i * TILE) / RECORD;
                const uint32_t to = mine_at + (uint32_t)(i % RING) * STEP;
                if (together) {
                    record_loads<RECORDS * S>::issue(to, places.template place<BYTES>(r));
                } else {
#pragma unroll
                    for (int u = 0; u < RECORDS; ++u)                // (no record behind the last)
                        record_loads<S>::issue(to + u * BYTES, places.template place<BYTES>(min(r + u, last)));
                }
            };
            for (int i = 0; i < min(steps, RING - 1); ++i) load(i);
            if (part == key0) w.take_query(room);
            for (int i = 0; i < steps; ++i) {
                const int base = base0 + i * TILE;
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (what was read from the records that these loads replace is here)
                if (i + RING - 1 < steps) {
                    load(i + RING - 1);
                    if (together) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 1) * TOGETHER) : "memory");
                    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 1) * APART) : "memory");
                } else {
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                }
                w.step(mine + (i % RING) * STEP, p.factor, base + WIDE > min(rows.context, part_end), part_end - base,
                       [&](int n, int on) { return rows.seen(min(16 * n + STATE::own_row(), rows.count - 1), base + on); });
            }
        }
        w.finish();
        float* slot = t0 == 0 && t1 == tiles ? nullptr : p.slot(blockIdx.x, pos == begin, head);
        if constexpr (PARTS == 1) {
            if (!w.sound()) {
                rows.template one_by_one<ACT>(key0, key1, slot, 0, rows.count, 1);
            } else {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int r = 16 * n + (lane & 15);
                    if (r >= rows.count) continue;
                    const float scale = slot ? 1.0f : inverse(w.l[n], [&] { return rows.sees_any(r); });
#pragma unroll
                    for (int i = 0; i < 2 * S; ++i) {
                        const int d = 16 * i + 4 * h;
                        if (d >= D) continue;
                        const f32x4 o = w.o[n][i] * scale;
                        if (slot) *(f32x4*)(slot + p.shape().at(r, d)) = o;
                        else *(u32x2*)(rows.result(r) + d) = u32x2{pack2<ACT>(o[0], o[1]), pack2<ACT>(o[2], o[3])};
                    }
                    if (slot && h == 0) p.shape().put_stats(slot, r, w.m[n], w.l[n]);
                }
            }
        } else {
            // the waves' sums, joined
            __syncthreads();
            if (threadIdx.x == 0) stats[256] = 0.0f;
            __syncthreads();
            if (!w.sound() && lane == 0) stats[256] = 1.0f;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int r = 16 * n + (lane & 15);
                if (h == 0) {
                    stats[(wave * 32 + r) * 2] = w.m[n];
                    stats[(wave * 32 + r) * 2 + 1] = w.l[n];
                }
#pragma unroll
                for (int i = 0; i < 2 * S; ++i) *(f32x4*)((float*)mine + r * 4 * QUADS + ((4 * i + h) ^ (r & TURN)) * 4) = w.o[n][i];
            }
            __syncthreads();
            if (stats[256] != 0.0f) {
                rows.template one_by_one<ACT>(key0, key1, slot, part_of, rows.count, PARTS);
            } else {
                for (int x = part_of * 64 + lane; x < rows.count * QUADS; x += 64 * PARTS) {
                    const int r = x / QUADS, quad = x % QUADS, d = quad * 4;
                    if (d >= D) continue;
                    float c = -__builtin_inff(), l = 0.0f;
#pragma unroll
                    for (int y = 0; y < PARTS; ++y) c = __builtin_fmaxf(c, stats[((head + y * HEADS) * 32 + r) * 2]);
                    const float from = c == -__builtin_inff() ? 0.0f : c;
                    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int y = 0; y < PARTS; ++y) {
                        const int other = head + y * HEADS;
                        const float weight = __builtin_amdgcn_exp2f(stats[(other * 32 + r) * 2] - from);
                        const f32x4 z = *(const f32x4*)((const float*)(lds + other * WAVE_BYTES) + r * 4 * QUADS + (quad ^ (r & TURN)) * 4);
                        l += weight * stats[(other * 32 + r) * 2 + 1];
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[i] += weight * z[i];
                    }
                    if (!slot) {
                        const float scale = inverse(l, [&] { return rows.sees_any(r); });
                        *(u32x2*)(rows.result(r) + d) = u32x2{pack2<ACT>(o[0] * scale, o[1] * scale), pack2<ACT>(o[2] * scale, o[3] * scale)};
                    } else {
                        *(f32x4*)(slot + p.shape().at(r, d)) = o;
                        if (d == 0) p.shape().put_stats(slot, r, c, l);
                    }
                }
            }
            __syncthreads();
        }
        }
        pos += tiles + p.extra - t0;
        t0 = 0;
        if (++u == all.units) {
            u = 0;
            if (++b < a.sequences) context = all.context(b), tiles = tiles_of(a, p, context);
        }
    }
}

// ------------------------------------------------------------------------------------------ above 32 rows
// A word's eight codes times scales, exactly: first codes of bytes 0, 1 and 2, 3, second codes of the same (low, high: the scales of bytes 0, 1
// and 2, 3).  bfloat16 has no packed multiplication: through binary32.
template <int ACT>
__device__ __forceinline__ u32x4 words16(uint32_t x, uint32_t low, uint32_t high) {
    const uint32_t f = firsts(x), g = seconds(x);
    if constexpr (ACT == FQ_F16) {
        return u32x4{times16(codes16<ACT, false>(f), low), times16(codes16<ACT, true>(f), high), times16(codes16<ACT, false>(g), low),
                     times16(codes16<ACT, true>(g), high)};
    } else {
        const float s[4] = {half_of<ACT, 0>(low), half_of<ACT, 1>(low), half_of<ACT, 0>(high), half_of<ACT, 1>(high)};
        const auto f0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(f, 512.0f, false), f1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(f, 512.0f, true);
        const auto g0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(g, 512.0f, false), g1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(g, 512.0f, true);
        return u32x4{pack2<ACT>(f0[0] * s[0], f0[1] * s[1]), pack2<ACT>(f1[0] * s[2], f1[1] * s[3]), pack2<ACT>(g0[0] * s[0], g0[1] * s[1]),
                     pack2<ACT>(g1[0] * s[2], g1[1] * s[3])};
    }
}

// O^T += V^T P^T over H half-tiles of values that lie as [value][key]
template <int H, int PITCH, int ACT, int DP>
__device__ __forceinline__ void accumulate(wave_state<ACT, DP>& w, const char* values, const u32x4 (&p)[2 * H]) {
    const int lane = threadIdx.x & 63;
    const char* mine = values + (lane & 31) * PITCH + (lane >> 5) * 8;
#pragma unroll
    for (int k = 0; k < 2 * H; ++k)
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) {
            const char* at = mine + 32 * t * PITCH + 32 * k;
            const u32x2 x = *(const u32x2*)at, y = *(const u32x2*)(at + 16);
            w.o[t] = mfma32<ACT>(u32x4{x[0], x[1], y[0], y[1]}, p[k], w.o[t]);
        }
}

// A record on its way to 16 bits: keys' words 4 h .. of token x16 (64 lanes: the codes back to back), values' words, scales.
template <int ACT, int S>
struct record_words {
    uint32_t k[S], v[S], key_scale[S], value_scale[2 * S];

    __device__ __forceinline__ void fetch(const void* record) {
        const int lane = threadIdx.x & 63, h = lane >> 4, x16 = lane & 15;
        const char* from = (const char*)record;
#pragma unroll
        for (int t = 0; t < S; ++t) {
            k[t] = *(const uint32_t*)(from + lane * 4 * S + 4 * t);
            v[t] = *(const uint32_t*)(from + 256 * S + lane * 4 * S + 4 * t);
            value_scale[2 * t] = *(const uint32_t*)(from + 544 * S + h * 8 * S + 8 * t);
            value_scale[2 * t + 1] = *(const uint32_t*)(from + 544 * S + h * 8 * S + 8 * t + 4);
            key_scale[t] = *(const uint16_t*)(from + scale_at(S, x16, t));
        }
    }
    // what lies behind the last of `there` keys may be anything
    __device__ __forceinline__ void cut(int there) {
        const int count = there - 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
        for (int g = 0; g < S; ++g) {
            value_scale[2 * g] &= first_mask(count);
            value_scale[2 * g + 1] &= first_mask(count - 2);
        }
    }
    // as record r of a tile: keys as wave_state takes them, values as [value][key]
    template <int PITCH, int DP>
    __device__ __forceinline__ void put(char* keys, char* values, int r) const {
        typedef tile_shape<DP> SH;
        const int lane = threadIdx.x & 63, h = lane >> 4, x16 = lane & 15, key = 16 * (r & 1) + x16;
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const uint32_t both = __builtin_amdgcn_perm(key_scale[t], key_scale[t], 0x01000100u);
            u32x4 x = words16<ACT>(k[t], both, both);
            *(u32x4*)(keys + (r >> 1) * SH::BYTES + key * SH::PITCH + key_unit<SH::UNITS>(key, 4 * t + h) * 16) = x;
            x = words16<ACT>(v[t], value_scale[2 * t], value_scale[2 * t + 1]);
            char* to = values + (32 * t + x16) * PITCH + (16 * r + 4 * h) * 2;
            *(u32x2*)to = u32x2{x[0], x[1]};
            *(u32x2*)(to + 16 * PITCH) = u32x2{x[2], x[3]};
        }
    }
};

// GROUPS x 32 rows a block, as over a cache of 16 bits, its waves a record of a tile each: the next tile's are taken to 16 bits beside the products of the
// present one, the one's after it are on their way.  Values lie as [value][key], rows 8 bytes longer than a tile's keys so that a read's 32 rows
// fall on different banks.
template <int S, int WAVES>
struct tile_room {
    static constexpr int DP = S < 2 ? 64 : 32 * S, TILE = RECORD * WAVES, PITCH = 2 * TILE + 8;
    static constexpr int KEY_BYTES = TILE / 32 * tile_shape<DP>::BYTES, BYTES = KEY_BYTES + DP * PITCH;
    static constexpr int JOIN = 32 * DP * 4;
    template <int GROUPS>
    static constexpr int all() { return GROUPS < WAVES && WAVES * JOIN > 2 * BYTES ? WAVES * JOIN : 2 * BYTES; }
};
template <int ACT, int S, int GROUPS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void fq_attention_kv4_tile_kernel(fq_tree_args a, tree_plan p, divisor by_records) {
    typedef tile_room<S, WAVES> room;
    constexpr int DP = room::DP, TILE = room::TILE, PITCH = room::PITCH;
    typedef tile_shape<DP> SH;
    constexpr int PARTS = WAVES / GROUPS, OWN = TILE / 32 / PARTS, HALVES = OWN < 2 ? OWN : 2;       // OWN: half-tiles of 32 keys that a wave takes
    extern __shared__ __align__(16) char lds[];
    int32_t* entries = (int32_t*)(lds + room::template all<GROUPS>());
    float* stats = (float*)(entries + TABLE);           // [4][32][2], and a flag
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = wave % GROUPS, part_of = wave / GROUPS;
    const int D = a.head_dim;

    const line all(a, p);
    const int64_t block = p.in_line(blockIdx.x), begin = block * all.per_block, stop = min(all.total, begin + all.per_block);
    if (begin >= stop) return;
    int b;
    int64_t at_b;
    all.find(begin, &b, &at_b);
    int context = all.context(b), tiles = tiles_of(a, p, context);
    int u = (int)quotient(begin - at_b, tiles + p.extra), t0 = (int)(begin - at_b - (int64_t)u * (tiles + p.extra));
    wave_state<ACT, DP> w;
    record_words<ACT, S> words;

    for (int64_t pos = begin; pos < stop;) {
        const unit_rows<kv4_rows> rows(a, p, b, u, 0, context);
        const int t1 = (int)min((int64_t)tiles, t0 + stop - pos);
        if (t0 < tiles) {                               // (behind them are places that hold nothing)
        float* slot = t0 == 0 && t1 == tiles ? nullptr : p.slot(block, pos == begin, 0);
        const int key0 = t0 * TILE, key1 = p.whole ? rows.keys : min(rows.keys, t1 * TILE);
        const int r = group * 32 + (lane & 31), row = min(r, rows.count - 1);
        const bool busy = group * 32 < rows.count;
        w.load_query(rows.query(row), D);
        w.clear();
        const int most = part_keys(TABLE, a.cache.page_size, TILE);
        for (int part = key0, part_end; part < key1; part = part_end) {
            part_end = fqa::part_end(part, key1, most);
            __syncthreads();
            const table_part table = load_table<64 * WAVES>(a, b, part, part_end, entries);
            if (32 * S < DP) {                          // values that no record has: zeros
                const u32x4 zero = {0, 0, 0, 0};
                for (int x = threadIdx.x; x < 2 * room::BYTES / 16; x += 64 * WAVES) ((u32x4*)lds)[x] = zero;
            }
            __syncthreads();
            w.query_is_here();                          // (with the table)
            const record_places places = {entries, table.first, by_records, a.cache.page_size / RECORD,
                                          (const char*)a.cache.k + rows.head * a.cache.head_stride, a.cache.page_stride};
            const int last = (part_end - 1) / RECORD, steps = (part_end - part + TILE - 1) / TILE;
            auto fetch = [&](int i) { words.fetch(places.template place<record_bytes(S)>(min((part + i * TILE) / RECORD + wave, last))); };
            auto put = [&](int i) {
                if (part + (i + 1) * TILE > part_end) words.cut(part_end - part - i * TILE - RECORD * wave);
                char* to = lds + (i & 1) * room::BYTES;
                words.template put<PITCH, DP>(to, to + room::KEY_BYTES, wave);
                if (i + 1 < steps) fetch(i + 1);
            };
            fetch(0);
            put(0);
            __syncthreads();
            for (int i = 0; i < steps; ++i) {
                const int base = part + i * TILE;
                const char* tile = lds + (i & 1) * room::BYTES;
                if (i + 1 < steps) put(i + 1);
                if (busy) {
#pragma unroll 1
                    for (int y = 0; y < OWN; y += HALVES) {
                        const int first = base + (part_of * OWN + y) * HALF;
                        if (OWN > HALVES && first >= part_end) break;
                        f32x16 s[HALVES];
                        u32x4 x[2 * HALVES];
                        w.template scores<HALVES, 6>(tile + (part_of * OWN + y) * SH::BYTES, s);
                        if (first + HALVES * HALF > min(rows.context, part_end)) {
#pragma unroll
                            for (int z = 0; z < HALVES; ++z) keep_seen(s[z], rows.seen(row, first + z * HALF));
                        }
                        w.template soften<HALVES>(s, p.factor, x);
                        accumulate<HALVES, PITCH>(w, tile + room::KEY_BYTES + (part_of * OWN + y) * HALF * 2, x);
                    }
                }
                __syncthreads();
            }
        }
        w.finish(PARTS > 1 || slot);
        if constexpr (PARTS > 1) {
            join_parts<ACT, DP, PARTS>(rows, w, lds, room::JOIN, stats, group, GROUPS, part_of, group, key0, key1, slot);
        } else {
            if (!w.sound()) rows.template one_by_one<ACT>(key0, key1, slot, group * 32, min(group * 32 + 32, rows.count), 1);
            else if (r < rows.count) w.put(rows.result(r), slot, p.shape(), r, [&] { return rows.sees_any(r); });
        }
        }
        pos += tiles + p.extra - t0;
        t0 = 0;
        if (++u == all.units) {
            u = 0;
            if (++b < a.sequences) context = all.context(b), tiles = tiles_of(a, p, context);
        }
    }
}

template <int ACT, int S, typename STATE, int HEADS>
int launch_stream(const fq_tree_args& a, const tree_plan& p, const divisor& by_records, hipStream_t stream) {
    static std::atomic<uint64_t> raised{0};
    const int st = fqd::raise_lds_limit((const void*)fq_attention_kv4_stream_kernel<ACT, S, STATE, HEADS>, raised);
    if (st != FQ_OK) return st;
    fq_attention_kv4_stream_kernel<ACT, S, STATE, HEADS><<<(unsigned)p.blocks, 256, 4 * STATE::RING * STATE::RECORDS * record_bytes(S) + TABLE * 4 + 257 * 4, stream>>>(a, p, by_records);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

template <int ACT, int S, int GROUPS, int WAVES>
int launch_tiles(const fq_tree_args& a, const tree_plan& p, const divisor& by_records, hipStream_t stream) {
    typedef tile_room<S, WAVES> room;
    static std::atomic<uint64_t> raised{0};
    const int st = fqd::raise_lds_limit((const void*)fq_attention_kv4_tile_kernel<ACT, S, GROUPS, WAVES>, raised);
    if (st != FQ_OK) return st;
    const int bytes = room::template all<GROUPS>() + TABLE * 4 + (GROUPS < WAVES ? 257 * 4 : 0);
    fq_attention_kv4_tile_kernel<ACT, S, GROUPS, WAVES><<<(unsigned)p.blocks, 64 * WAVES, bytes, stream>>>(a, p, by_records);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

template <int ACT, int S, typename STATE>
int launch_few(const fq_tree_args& a, const tree_plan& p, const divisor& by_records, hipStream_t stream) {
    return p.heads == 4   ? launch_stream<ACT, S, STATE, 4>(a, p, by_records, stream)
           : p.heads == 2 ? launch_stream<ACT, S, STATE, 2>(a, p, by_records, stream)
                          : launch_stream<ACT, S, STATE, 1>(a, p, by_records, stream);
}

template <int ACT, int S>
int launch(const fq_tree_args& a, const tree_plan& p, hipStream_t stream) {
    const divisor by_records = divisor::of((uint32_t)(a.cache.page_size / RECORD));
    const int st = p.unit_rows > 128  ? launch_tiles<ACT, S, 8, 8>(a, p, by_records, stream)
                   : p.unit_rows > 64 ? launch_tiles<ACT, S, 4, 4>(a, p, by_records, stream)
                   : p.rows > 32      ? launch_tiles<ACT, S, 2, 4>(a, p, by_records, stream)
                   : p.rows > 16    ? launch_stream<ACT, S, few_rows<ACT, S, 2>, 1>(a, p, by_records, stream)
                   : p.rows > 4     ? launch_few<ACT, S, few_rows<ACT, S, 1>>(a, p, by_records, stream)
                                    : launch_few<ACT, S, four_rows<ACT, S>>(a, p, by_records, stream);
    if (st != FQ_OK || p.whole) return st;
    return launch_join<ACT, kv4_rows>(a, p, stream);
}

template <int ACT>
int launch(const fq_tree_args& a, const tree_plan& p, hipStream_t stream) {
    switch (groups_of(a.head_dim)) {
        case 1: return launch<ACT, 1>(a, p, stream);
        case 2: return launch<ACT, 2>(a, p, stream);
        case 3: return launch<ACT, 3>(a, p, stream);
        default: return launch<ACT, 4>(a, p, stream);
    }
}

}  // namespace

// Above 128 rows blocks of 256, which take a key to 16 bits half as often as blocks of 128, where there are six tiles for each of them or more (a block begins
// with 5 us in which it multiplies nothing), by the table's width.  us with the join, one call after the other, 256 rows and 128: two sequences of 2500 - 3900 tokens, 2800
// rows of eight heads, 145, 163; eight of 500 - 4095, 192 rows, 39.0, 42.5; eight of 1000 in tables for 4000 34.3, 34.7; one of 20 000, 192 rows, which has five, 48.1, 43.4; of 8000 in
// such a table 36.5, 33.6; one of 8000, eight heads of 64, which has two: a chain of 200 tokens 33.4, 27.5, but a tree of 25, eight query heads each, 20.2, 25.4.
static bool wide(const fq_tree_args& a, int64_t rows) {
    const int64_t tiles = (a.table_width * a.cache.page_size + 127) / 128, units = a.sequences * a.kv_heads * ((rows + 255) / 256);
    return rows > 128 && tiles * units >= 6 * (int64_t)fq_cu_count();
}

// Few rows: waves take heads of their own where there are enough, so that pieces are four times as long, and few are joined in LDS.
// The beginning and end of a unit count as three tiles, one of 128 keys (with the join: a token each of 64 sequences of 100 - 8191 41.2 us where they count as none, 36.5 so; two
// sequences' pieces as above, none 145.6, one 144.7, two 143.2, eight sequences' trees 40.8, 38.9, 42.4).
static tree_plan plan_kv4(const fq_tree_args& a) {
    const int64_t rows = (int64_t)a.nodes * (a.q_heads / a.kv_heads);
    const int heads = rows > 16 ? 1 : a.kv_heads % 4 == 0 ? 4 : a.kv_heads % 2 == 0 ? 2 : 1;
    if (!wide(a, rows)) return plan_units(a, heads, rows <= 64 ? 64 : 128, rows > 32 ? KEYS : (rows > 4 ? 128 : 256) / heads, 3);
    tree_plan p = plan_units(a, 1, 256, 128, 1);
    p.blocks /= 2;                       // (one has a compute unit's LDS for itself)
    return p;
}

size_t fq_tree_kv4_bytes(const fq_tree_args& a) { return slots_bytes(plan_kv4(a)); }

int fq_launch_attention_tree_kv4(int act_dtype, const fq_tree_args& a, void* workspace, hipStream_t stream) {
    tree_plan p = plan_kv4(a);
    p.slots = (float*)workspace;
    return act_dtype == FQ_F16 ? launch<FQ_F16>(a, p, stream) : launch<FQ_BF16>(a, p, stream);
}
