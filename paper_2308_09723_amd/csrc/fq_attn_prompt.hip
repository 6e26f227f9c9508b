// Causal attention over packed sequences (fq_attention_prompt).
#include <hip/hip_runtime.h>
#include <algorithm>
#include <atomic>

#include "fq_attn_tile.h"
#include "fq_lds_limit.h"

namespace {

using namespace fqa;

constexpr int SEQUENCES = 128;       // per launch: their table is a kernel argument

// The sequences of a launch, longest first, and the order of their query tiles: the last tiles of the longest sequences, which
// have the most keys, come first, level by level.
struct prompt_items {
    int32_t q_start[SEQUENCES], q_len[SEQUENCES], k_start[SEQUENCES], k_len[SEQUENCES];
    int32_t tiles[SEQUENCES];
    int32_t before[SEQUENCES];       // tiles that come before the levels of which sequence s is the shortest end
    int32_t count, step;             // step: the largest power of two below count, or 0
};

// Tile `rank` in that order: its sequence, and its number within it.
__device__ inline void find_tile(const prompt_items& items, int rank, int* sequence, int* tile) {
    int s = 0;
    for (int step = items.step; step > 0; step /= 2)
        if (s + step < items.count && items.before[s + step] <= rank) s += step;
    const int in = rank - items.before[s], level = s == 0 ? in : in / (s + 1);
    *sequence = in - level * (s + 1);
    *tile = items.tiles[s] - 1 - level;
}

// What the host has made of a launch.
struct prompt_plan {
    int q_heads, group, D;
    divisor by_group;
    float factor;
    int splits;                      // pieces that a query tile's keys are cut into
    float* slots;                    // one per query tile, head and piece

    int units;                       // query tiles times heads
    int together, of_set;            // heads of a die that it works on at the same time; blocks of it that have them
    divisor by_units, by_heads, by_set, by_together;
    // Blocks go to the eight dies in turn.  Neighbouring heads, which share keys, go to the same die and its cache (8192 tokens, 32
    // heads over 8: 518 -> 510 us, 24 ragged prompts 122 -> 113), some of them at a time where the keys of all would not stay there
    // (96 heads, two sequences of 2048 tokens: 235 -> 223 us); within them all query tiles in the order of the items.
    __device__ void find(int unit, int* rank, int* h) const {
        if (q_heads % 8 != 0) {
            *rank = by_heads.quotient(unit);
            *h = unit - *rank * q_heads;
            return;
        }
        const int of_die = q_heads / 8, i = unit / 8;
        const int set = by_set.quotient(i), in = i - set * of_set, left = of_die - set * together;
        const int heads = left < together ? left : together;
        *rank = heads == together ? by_together.quotient(in) : in / heads;
        *h = unit % 8 * of_die + set * together + in - *rank * heads;
    }
    __host__ __device__ slot_shape shape() const { return {ROWS, D}; }
    __device__ float* slot(int unit, int piece) const { return slots + ((int64_t)unit * splits + piece) * shape().floats(); }
};

// A block: 128 queries of one head, a wave 32 of them (fq_attn_tile.h has the mathematics), and 64 keys and values at a time, twice 32 KiB of LDS
// for heads of 128 values, so that two blocks fill a compute unit, one's products beside the other's numerators.
// Bound by the issue of products and numerators, and by power: 8192 tokens, 32 heads over 8 of 128 values in bfloat16, 550 GF in
// 488 - 541 us = 1.02 - 1.13 PFLOP/s (a library's product of 8192 x 8192 x 8192: 1.21), binary16 542 (540 with maxima looked for as rarely as in
// bfloat16: not theirs).
// Short prompts by the blocks' beginnings and ends: 24 prompts of 17 - 1500 tokens 94 - 113 us = 0.59 - 0.71 PFLOP/s.
template <int ACT, int DP>
__global__ __launch_bounds__(256, 2) void fq_attention_prompt_kernel(fq_heads q, fq_heads k, fq_heads v, prompt_plan p, uint16_t* out,
                                                                     prompt_items items) {
    typedef tile_shape<DP> SH;
    extern __shared__ __align__(16) char lds[];
    const int piece = p.by_units.quotient(blockIdx.x), unit = blockIdx.x - piece * p.units;      // piece of its keys; query tile and head
    const int D = p.D;
    int rank, h, sequence, tile;
    p.find(unit, &rank, &h);
    find_tile(items, rank, &sequence, &tile);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int queries = items.q_len[sequence], keys = items.k_len[sequence];
    const int first = tile * ROWS + wave * 32, i = first + (lane & 31);       // the wave's first query; the lane's
    packed_rows rows;
    rows.k = (const uint16_t*)k.data + items.k_start[sequence] * k.row_stride + p.by_group.quotient(h) * k.head_stride;
    rows.v = (const uint16_t*)v.data + items.k_start[sequence] * v.row_stride + p.by_group.quotient(h) * v.head_stride;
    rows.k_stride = k.row_stride;
    rows.v_stride = v.row_stride;
    const int ahead = keys - queries;        // query i sees keys 0 .. i + ahead
    const int all = max(0, (min(queries, (tile + 1) * ROWS) + ahead + KEYS - 1) / KEYS);      // tiles of keys that the block's last query sees
    const int t0 = p.splits == 1 ? 0 : (int)((uint32_t)all * (uint32_t)piece / (uint32_t)p.splits);
    const int t1 = p.splits == 1 ? all : (int)((uint32_t)all * (uint32_t)(piece + 1) / (uint32_t)p.splits);      // (at most 2^25 tiles, 128 pieces)

    // units of a head that no load fills are zeros from here on
    constexpr int TILE_BYTES = 2 * SH::BYTES;      // of keys, or of values
    if (D < SH::UNITS * 8) {
        const u32x4 zero = {0, 0, 0, 0};
        for (int x = threadIdx.x; x < 4 * TILE_BYTES / 16; x += 256) ((u32x4*)lds)[x] = zero;
        __syncthreads();
    }
    // A thread loads unit (its place in LDS: lane % UNITS) of rows that lie 256 / UNITS apart, which move it alike.
    constexpr int STEP = 256 / SH::UNITS;
    const int row0 = threadIdx.x / SH::UNITS, place = threadIdx.x % SH::UNITS;
    const int key_at = key_unit<SH::UNITS>(row0, place) * 8, value_at = value_unit<SH::UNITS>(row0, place) * 8;
    // (64 rows within 32 bits of each other: scalar address and lane offset)
    const bool near = k.row_stride < (int64_t)1 << 24 && v.row_stride < (int64_t)1 << 24;
    const uint32_t key_off = (uint32_t)((row0 * (uint32_t)k.row_stride + key_at) * 2), value_off = (uint32_t)((row0 * (uint32_t)v.row_stride + value_at) * 2);
    auto load = [&](int t, int buffer) {
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(lds + buffer * 2 * TILE_BYTES) + wave * 1024;
        if (near && (t + 1) * KEYS <= keys) {
            const uint16_t *key = rows.key(t * KEYS), *value = rows.value(t * KEYS);
            if (key_at < D) {
#pragma unroll
                for (int j = 0; j < TILE_BYTES / 4096; ++j) load_lds16<false>(to + j * 4096, key + j * STEP * k.row_stride, key_off);
            }
            if (value_at < D) {
#pragma unroll
                for (int j = 0; j < TILE_BYTES / 4096; ++j) load_lds16<false>(to + TILE_BYTES + j * 4096, value + j * STEP * v.row_stride, value_off);
            }
        } else {                                // (no row behind the last: what lies there may be anything)
#pragma unroll 1
            for (int j = 0; j < TILE_BYTES / 4096; ++j) {
                const int row = min(t * KEYS + row0 + j * STEP, keys - 1);
                if (key_at < D) load_lds16(to + j * 4096, rows.key(row) + key_at);
                if (value_at < D) load_lds16(to + TILE_BYTES + j * 4096, rows.value(row) + value_at);
            }
        }
    };
    wave_state<ACT, DP> w;
    w.clear();
    if (t0 < t1) load(t0, 0);
    {
        // the wave's queries, into the second buffer, whole lines at a time
        const int r0 = lane / SH::UNITS;
        char* mine = lds + 2 * TILE_BYTES + wave * SH::BYTES;
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine;
        const uint16_t* from = (const uint16_t*)q.data + (int64_t)items.q_start[sequence] * q.row_stride + h * q.head_stride;
#pragma unroll
        for (int j = 0; j < SH::BYTES / 1024; ++j) {
            const int r = r0 + j * (64 / SH::UNITS), at = key_unit<SH::UNITS>(r, place) * 8;
            if (at < D) load_lds16(to + j * 1024, from + (int64_t)min(first + r, queries - 1) * q.row_stride + at);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        w.read_query(mine);
        w.query_is_here();
    }
    const int end = i + 1 + ahead;           // keys that the lane's query sees
    for (int t = t0; t < t1; ++t) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const int buffer = (t - t0) & 1;
        if (t + 1 < t1) load(t + 1, buffer ^ 1);
        const int base = t * KEYS;
        if (first < queries && base < first + 32 + ahead) {
            const char* at = lds + buffer * 2 * TILE_BYTES;
            f32x16 s[2];
            u32x4 x[4];
            w.template scores<2>(at, s);
            if (base + KEYS > first + 1 + ahead) {
                keep_seen(s[0], low_bits(end - base));
                keep_seen(s[1], low_bits(end - base - HALF));
            }
            w.template soften<2, false>(s, p.factor, x);
            w.template accumulate<2>(at + TILE_BYTES, x);
        }
    }
    __syncthreads();                         // (nobody reads keys and values any more)
    float* slot = p.splits > 1 ? p.slot(unit, piece) : nullptr;
    w.finish(slot != nullptr);
    if (!w.sound()) {
        for (int x = 0; x < 32 && first + x < queries; ++x) {
            const int64_t r = (int64_t)items.q_start[sequence] + first + x;
            const int sees = first + x + 1 + ahead;
            float o[2], c, sum;
            attend_one<ACT>((const uint16_t*)q.data + r * q.row_stride + h * q.head_stride, rows, sees_first{sees}, t0 * KEYS, min(sees, t1 * KEYS), D,
                            p.factor, o, &c, &sum);
            put_one<ACT>(out + (r * p.q_heads + h) * D, slot, p.shape(), wave * 32 + x, o, c, sum, [&] { return sees > 0; });
        }
    } else if (slot) {
        if (i < queries) w.put(nullptr, slot, p.shape(), wave * 32 + (lane & 31), [&] { return end > 0; });
    } else if (first < queries) {
        uint16_t* to = out + (((int64_t)items.q_start[sequence] + first) * p.q_heads + h) * D;
        w.put_rows(lds + wave * 2 * SH::BYTES, [&](int r) { return to + (int64_t)r * p.q_heads * D; }, queries - first, D,
                   [&] { return end > 0; });
    }
}

// Joins the pieces of a query tile: a lane has four values of a row, a wave 32 rows of eight, so that reads are whole lines.  Bound by
// latency: 224 tiles in two pieces, 7 us.
template <int ACT>
__global__ __launch_bounds__(256) void fq_attention_prompt_join_kernel(prompt_plan p, uint16_t* out, prompt_items items) {
    const int unit = blockIdx.x, D = p.D;
    int rank, h, sequence, tile;
    p.find(unit, &rank, &h);
    find_tile(items, rank, &sequence, &tile);
    const int count = min(ROWS, items.q_len[sequence] - tile * ROWS), groups = (count + 31) / 32;
    for (int x = blockIdx.y * 256 + threadIdx.x; x < groups * (D / 4) * 32; x += 256 * gridDim.y) {
        const int y = x / 32, group = y / (D / 4), d = (y - group * (D / 4)) * 4, r = group * 32 + x % 32;
        if (r >= count) continue;
        partial_sums all;
        all.clear();
        all.add(0, p.splits, [&](int y) { return p.slot(unit, y); }, p.shape(), r, d);
        all.template store<ACT>(out + (((int64_t)items.q_start[sequence] + tile * ROWS + r) * p.q_heads + h) * D + d,
                                [&] { return tile * ROWS + r + 1 + items.k_len[sequence] - items.q_len[sequence] > 0; });
    }
}

template <int ACT, int DP>
int launch(const fq_prompt_args& a, const prompt_plan& p, const prompt_items& items, int total, hipStream_t stream) {
    static std::atomic<uint64_t> raised{0};
    constexpr int LDS = 8 * tile_shape<DP>::BYTES;      // two tiles of keys and of values
    if (LDS > 65536) {
        const int st = fqd::raise_lds_limit((const void*)fq_attention_prompt_kernel<ACT, DP>, raised);
        if (st != FQ_OK) return st;
    }
    fq_attention_prompt_kernel<ACT, DP><<<dim3((unsigned)(total * a.q_heads * p.splits)), 256, LDS, stream>>>(a.q, a.k, a.v, p, (uint16_t*)a.out, items);
    if (hipGetLastError() != hipSuccess) return FQ_ERR_HIP;
    if (p.splits == 1) return FQ_OK;
    fq_attention_prompt_join_kernel<ACT><<<dim3((unsigned)(total * a.q_heads), 4), 256, 0, stream>>>(p, (uint16_t*)a.out, items);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

template <int ACT>
int launch(const fq_prompt_args& a, const prompt_plan& p, const prompt_items& items, int total, hipStream_t stream) {
    if (a.head_dim <= 64) return launch<ACT, 64>(a, p, items, total, stream);
    if (a.head_dim <= 96) return launch<ACT, 96>(a, p, items, total, stream);
    return launch<ACT, 128>(a, p, items, total, stream);
}

// Of sequences first .. first + n - 1: rows, query tiles, the key tiles of all of them, and the most that one has.
struct tile_counts {
    int64_t rows = 0, total = 0, keys = 0;
    int longest = 0;
    tile_counts(const fq_prompt_args& a, int first, int n) {
        for (int b = first; b < first + n; ++b) {
            const int64_t queries = a.q_offsets[b + 1] - a.q_offsets[b], all = a.k_offsets[b + 1] - a.k_offsets[b];
            if (queries == 0) continue;
            const int64_t tiles = (queries + ROWS - 1) / ROWS, last = (all + KEYS - 1) / KEYS;
            const int64_t least = std::max<int64_t>(1, std::min(last, (all - queries + ROWS + KEYS - 1) / KEYS));
            rows += queries;
            total += tiles;
            keys += tiles * (least + std::max<int64_t>(1, last)) / 2;
            longest = std::max(longest, (int)last);
        }
    }
};

constexpr int64_t MOST_BLOCKS = (1 << 24) - 1;       // of a launch (2^32 threads)

// Pieces for the keys of a launch's query tiles: a piece's sums are written and read again, and joining them is a launch.  At most, where tiles are
// few, as many as bring the blocks up to the number that run at once, of eight key tiles and more (1000 tokens of 16 heads in pieces of four tiles
// 24.4 us, of eight 24.7); where they are more, but some of so many keys that the others are done long before, as many as bring those down to a block's
// even share, of sixteen key tiles and more (15 prompts of 24 - 1018 tokens, 16 heads, 21 us whole, 28 in pieces of eight tiles).
//
// Up to there, as many as are through first: a key tile takes 1.1 us, the sums of all rows (all are cut into as many) are written and read at
// 4.3 TB/s, and joining them takes 4 us more.  us, whole and in pieces: three prompts behind 4001 keys, 224 tiles of heads, 70, 56 in 2; 100 queries
// behind 8000 keys 134, 36 - 40 in 8 to 16; one prompt of 3397 tokens, 12 heads of 64, 55, 44 in 3; of 1024 tokens, 32 heads over 8 of 128, 25, 32 in 2; of
// 2324 59, 82 in 2; the same heads, 16 prompts of 512 and 256 queries behind 8000 keys 187, 443 in 4; 127 of 128 and one behind 131000 2261, 1356 in
// 4, 2281 in 14.
int plan_splits(const fq_prompt_args& a, const tile_counts& c) {
    const int64_t units = c.total * a.q_heads, work = c.keys * a.q_heads, room = 2 * fq_cu_count();
    if (units == 0) return 1;
    const bool few = units * 2 <= room;
    const int64_t even = few ? room / units : (2 * c.longest * room + work) / (2 * work);
    const int most = (int)std::min({(int64_t)64, even, (int64_t)c.longest / (few ? 8 : 16), MOST_BLOCKS / units});
    const double share = (double)work / room, sums = 2.0 * c.rows * a.q_heads * (a.head_dim + 2) * sizeof(float) / 4.3e6;      // a piece's of all rows, us
    int best = 1;
    double least = 1.1 * c.longest;
    for (int n = 2; n <= most; ++n) {
        const double t = 1.1 * std::max((double)c.longest / n, share) + n * sums + 4;
        if (t < least) best = n, least = t;
    }
    return best;
}

// Heads of a die whose keys and values, of all sequences of a launch, its 4 MiB of cache holds.
int heads_together(const fq_prompt_args& a, int first, int n) {
    const int64_t keys = (int64_t)a.k_offsets[first + n] - a.k_offsets[first], bytes = std::max<int64_t>(1, keys * a.head_dim * 4);
    const int group = a.q_heads / a.kv_heads, of_die = std::max(1, a.q_heads / 8);
    return (int)std::min<int64_t>(of_die, std::max<int64_t>(1, (4 << 20) / bytes) * group);
}

}  // namespace

bool fq_prompt_fits(const fq_prompt_args& a) {
    for (int first = 0; first < a.sequences; first += SEQUENCES) {
        const int last = std::min(first + SEQUENCES, a.sequences);
        int64_t tiles = 0;
        for (int b = first; b < last; ++b) tiles += (a.q_offsets[b + 1] - a.q_offsets[b] + ROWS - 1) / ROWS;
        if (tiles * a.q_heads > MOST_BLOCKS) return false;
    }
    return true;
}

size_t fq_prompt_bytes(const fq_prompt_args& a) {
    size_t most = 0;
    for (int first = 0; first < a.sequences; first += SEQUENCES) {
        const tile_counts c(a, first, std::min(SEQUENCES, a.sequences - first));
        const int splits = plan_splits(a, c);
        if (splits > 1) most = std::max(most, (size_t)(c.total * a.q_heads * splits) * ROWS * (a.head_dim + 2) * sizeof(float));
    }
    return most;
}

int fq_launch_attention_prompt(int act_dtype, const fq_prompt_args& a, void* workspace, hipStream_t stream) {
    for (int first = 0; first < a.sequences; first += SEQUENCES) {
        const int n = std::min(SEQUENCES, a.sequences - first);
        const tile_counts c(a, first, n);
        const int64_t total = c.total;
        if (total == 0) continue;
        prompt_plan p = {};
        p.q_heads = a.q_heads;
        p.group = a.q_heads / a.kv_heads;
        p.by_group = divisor::of((uint32_t)p.group);
        p.D = a.head_dim;
        p.factor = a.scale * LOG2E;
        p.splits = plan_splits(a, c);
        p.slots = (float*)workspace;
        p.units = (int)total * a.q_heads;
        p.together = p.splits > 1 ? std::max(1, a.q_heads / 8) : heads_together(a, first, n);       // (pieces: all blocks run at once anyway)
        p.of_set = (int)total * p.together;
        p.by_units = divisor::of((uint32_t)p.units);
        p.by_heads = divisor::of((uint32_t)p.q_heads);
        p.by_set = divisor::of((uint32_t)p.of_set);
        p.by_together = divisor::of((uint32_t)p.together);
        int order[SEQUENCES], tiles[SEQUENCES];
        for (int i = 0; i < n; ++i) {
            order[i] = i;
            tiles[i] = (a.q_offsets[first + i + 1] - a.q_offsets[first + i] + ROWS - 1) / ROWS;
        }
        std::sort(order, order + n, [&](int x, int y) { return tiles[x] != tiles[y] ? tiles[x] > tiles[y] : x < y; });
        prompt_items items = {};
        items.count = n;
        while (2 * items.step + !items.step < n) items.step = 2 * items.step + !items.step;
        for (int s = 0; s < n; ++s) {
            const int b = first + order[s];
            items.q_start[s] = a.q_offsets[b];
            items.q_len[s] = a.q_offsets[b + 1] - a.q_offsets[b];
            items.k_start[s] = a.k_offsets[b];
            items.k_len[s] = a.k_offsets[b + 1] - a.k_offsets[b];
            items.tiles[s] = tiles[order[s]];
        }
        // levels from the longest sequence's last tile down: those that sequences 0 .. s have and s + 1 has not
        for (int s = 0, before = 0; s < n; ++s) {
            items.before[s] = before;
            before += (s + 1) * (items.tiles[s] - (s + 1 < n ? items.tiles[s + 1] : 0));
        }
        const int st = act_dtype == FQ_F16 ? launch<FQ_F16>(a, p, items, (int)total, stream) : launch<FQ_BF16>(a, p, items, (int)total, stream);
        if (st != FQ_OK) return st;
    }
    return FQ_OK;
}
