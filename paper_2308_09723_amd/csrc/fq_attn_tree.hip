// Attention of drafted tokens over the pages of a cache (fq_attention_tree).
//
// The rows that share a key head's keys are the sequence's nodes times the query heads of the group: one token of four heads a group
// is four rows, 48 nodes are 192.  A key and its value are 4 D bytes, and 4 D operations for each row; the card does 170 operations in the
// time of a byte.  So few rows are bound by the cache's bytes: up to 32, every wave brings in keys of its own (fq_attention_tree_stream_kernel);
// above, four waves share them (fq_attention_tree_tile_kernel).
//
// Work is dealt out evenly whatever the sequences' lengths are: all sequences' key tiles, key head by key head, make one line, and
// each block takes an equal piece of it, cut where it likes.  Lengths are read on the device, so each block finds its own place (a
// scan over the lengths by each wave).  Where a unit (a sequence's rows of one key head) is cut, the pieces leave their sums,
// not divided, and the maxima they are relative to in the workspace, and a second kernel joins them.
#include <hip/hip_runtime.h>
#include <atomic>
#include <type_traits>

#include "fq_attn_parts.h"
#include "fq_attn_tile.h"
#include "fq_lds_limit.h"

namespace {

using namespace fqa;

constexpr int TABLE = 1024;          // entries of the page table that a block has in LDS

// What the host has made of a call.
struct tree_plan {
    int group, rows;                 // query heads per key head; rows of a key head
    divisor by_group, by_quads, by_side;       // divisors: group; head_dim / 4; rows of a slot that lie side by side
    int heads;                       // key heads that a block takes together
    int row_tiles, unit_rows;        // tiles of unit_rows rows that a head's are cut into
    int tile;                        // keys of a tile
    bool whole;                      // units are not cut: each counts as one tile
    bool by_lanes;                   // up to 64 sequences, of fewer than 2^31 tiles
    bool once;                       // above 32 rows: keys and values are read past the caches
    int blocks;                      // at most
    int slot_rows;                   // rows of a slot of the workspace
    int D;
    float factor;
    float* slots;                    // two per block and head of it

    // blocks that follow each other in the line share a die's cache (blocks go to the eight dies in turn)
    __device__ int in_line(int block) const { return blocks % 8 == 0 ? block % 8 * (blocks / 8) + block / 8 : block; }
    __host__ __device__ slot_shape shape() const { return {slot_rows, D}; }
    // a block's first piece, or its last, of head h of the heads it takes together
    __device__ float* slot(int64_t block, bool first, int h) const { return slots + ((2 * block + !first) * heads + h) * shape().floats(); }
};

__device__ inline int keys_of(const fq_tree_args& a, int context) {
    return context < 0 ? 0 : (int)min(a.table_width * a.cache.page_size, (int64_t)context + a.nodes);
}
__device__ inline int tiles_of(const fq_tree_args& a, const tree_plan& p, int context) {      // (one without keys: its zeros are somebody's)
    return p.whole ? 1 : max(1, (keys_of(a, context) + p.tile - 1) / p.tile);
}

// a / b of numbers that are hardly ever long (a division in 64 bits takes a microsecond)
__device__ inline int64_t quotient(int64_t a, int64_t b) {
    if (((uint64_t)(a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
    return a / b;
}

__device__ inline int64_t wave_sum64(int64_t x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}
// the sum of x over the lanes up to this one
__device__ inline int sum_upto(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);       // from 1, 2, 4, 8 lanes below in the row of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // row 0's sum to row 1, 2's to 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // rows 0 and 1's sum to rows 2 and 3
    return x;
}

// The line of tiles: sequence by sequence, in it unit by unit.  Up to 64 sequences: a lane has one sequence's length, and no length is
// read twice.
struct line {
    const fq_tree_args& a;
    const tree_plan& p;
    int64_t per_block;               // tiles
    int64_t total;
    int units;                       // of a sequence
    int mine, tiles, upto;           // by_lanes: the lane's length, its tiles, all tiles up to it

    __device__ line(const fq_tree_args& a, const tree_plan& p) : a(a), p(p) {
        const int lane = threadIdx.x & 63;
        units = a.kv_heads / p.heads * p.row_tiles;
        mine = tiles = upto = 0;
        if (p.by_lanes) {
            if (lane < a.sequences) {
                mine = a.context_lens[lane];
                tiles = tiles_of(a, p, mine);
            }
            upto = sum_upto(tiles);
            total = (int64_t)__builtin_amdgcn_readlane(upto, 63) * units;
        } else {
            int64_t sum = 0;
            for (int b = lane; b < a.sequences; b += 64) sum += tiles_of(a, p, a.context_lens[b]);
            total = uniform(wave_sum64(sum)) * units;
        }
        per_block = quotient(total + p.blocks - 1, p.blocks);
    }
    __device__ int context(int b) const { return p.by_lanes ? __builtin_amdgcn_readlane(mine, b) : __builtin_amdgcn_readfirstlane(a.context_lens[b]); }
    // where sequence b's tiles begin
    __device__ int64_t begin(int b) const {
        if (p.by_lanes) return (int64_t)(__builtin_amdgcn_readlane(upto, b) - __builtin_amdgcn_readlane(tiles, b)) * units;
        int64_t before = 0;
        for (int x = threadIdx.x & 63; x < b; x += 64) before += tiles_of(a, p, a.context_lens[x]);
        return uniform(wave_sum64(before)) * units;
    }
    // the sequence whose tiles the line has at `at`, and where they begin
    __device__ void find(int64_t at, int* sequence, int64_t* begin) const {
        const int lane = threadIdx.x & 63;
        const int64_t target = quotient(at, units);        // in tiles of one unit
        if (p.by_lanes) {
            const int b = __builtin_popcountll(__ballot(lane < a.sequences && upto <= target));
            *sequence = min(b, (int)a.sequences - 1);
            *begin = this->begin(*sequence);
            return;
        }
        int64_t before = 0;
        for (int first = 0;; first += 64) {
            const int b = first + lane, n = b < a.sequences ? tiles_of(a, p, a.context_lens[b]) : 0;
            int64_t upto = n;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int64_t x = __shfl_up(upto, d);
                if (lane >= d) upto += x;
            }
            const int64_t all = uniform(__shfl(upto, 63));
            if (target < before + all || first + 64 >= a.sequences) {
                const int k = min(63, __builtin_popcountll(__ballot(before + upto <= target)));
                *sequence = __builtin_amdgcn_readfirstlane(min(first + k, (int)a.sequences - 1));
                *begin = uniform(before + __shfl(upto - n, k)) * units;
                return;
            }
            before += all;
        }
    }
};

// Rows of a unit: where a row's query lies, where its result goes, and what it sees.
struct unit_rows {
    const fq_tree_args& a;
    const tree_plan& p;
    int b, head, first, count;       // sequence; key head; first row, rows
    int context, keys;

    // unit u of sequence b, head h of its heads
    __device__ unit_rows(const fq_tree_args& a, const tree_plan& p, int b, int u, int h, int context) : a(a), p(p), b(b), context(context) {
        const int set = u / p.row_tiles;
        head = set * p.heads + h;
        first = (u - set * p.row_tiles) * p.unit_rows;
        count = min(p.unit_rows, p.rows - first);
        keys = keys_of(a, context);
    }
    __device__ const uint16_t* query(int r) const {
        const int node = p.by_group.quotient(first + r), h = head * p.group + (first + r) - node * p.group;
        return (const uint16_t*)a.q.data + ((int64_t)b * a.nodes + node) * a.q.row_stride + h * a.q.head_stride;
    }
    __device__ uint16_t* result(int r) const {
        const int node = p.by_group.quotient(first + r), h = head * p.group + (first + r) - node * p.group;
        return (uint16_t*)a.out + (((int64_t)b * a.nodes + node) * a.q_heads + h) * a.head_dim;
    }
    __device__ paged_rows pages() const {
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
    __device__ const uint64_t* words(int r) const {
        return a.mask + b * a.mask_stride + (int64_t)p.by_group.quotient(first + r) * ((a.nodes + 63) / 64);
    }
    // which of keys base .. base + 31 row r sees
    __device__ uint32_t seen(int r, int base) const {
        uint32_t bits = low_bits(keys - base);
        const int d = base - context;          // the drafted token that bit 0 stands for
        if (d <= -32) return bits;
        if (!a.mask) return bits & low_bits(p.by_group.quotient(first + r) + 1 - d);
        const uint64_t* w = words(r);
        const int n = max(0, d), last = (a.nodes + 63) / 64 - 1;
        uint32_t drafted = 0;
        if (n < a.nodes) {
            const int at = n >> 6, by = n & 63;
            uint64_t x = w[at] >> by;
            if (by > 32 && at < last) x |= w[at + 1] << (64 - by);
            drafted = (uint32_t)x & low_bits(a.nodes - n);
        }
        return bits & (d < 0 ? low_bits(-d) | drafted << -d : drafted);
    }
    // whether row r sees any key
    __device__ bool sees_any(int r) const {
        if (keys <= 0) return false;
        if (!a.mask || context > 0) return true;       // (the context; without one, the first drafted token, which the whole chain sees)
        const uint64_t* w = words(r);
        for (int n = 0; n < keys; n += 64)
            if (w[n >> 6] & (keys - n < 64 ? ((uint64_t)1 << (keys - n)) - 1 : ~(uint64_t)0)) return true;
        return false;
    }
    // row r over keys begin .. end - 1 by one wave, seen keys alone
    template <int ACT>
    __device__ void one(int r, int begin, int end, float* o, float* c, float* l) const {
        if (a.mask) {
            attend_one<ACT>(query(r), pages(), sees_tree{context, a.nodes, words(r)}, begin, end, a.head_dim, p.factor, o, c, l);
        } else {
            const int last = (int)min((int64_t)end, (int64_t)context + p.by_group.quotient(first + r) + 1);
            attend_one<ACT>(query(r), pages(), sees_first{last}, begin, min(end, last), a.head_dim, p.factor, o, c, l);
        }
    }
    // rows from .. to - 1 of a piece in that way, every step-th
    template <int ACT>
    __device__ void one_by_one(int begin, int end, float* slot, int from, int to, int step) const {
        const int lane = threadIdx.x & 63;
        for (int r = from; r < to; r += step) {
            float o[2], c, l;
            one<ACT>(r, begin, end, o, &c, &l);
            put_one<ACT>(result(r), slot, p.shape(), r, o, c, l, [&] { return sees_any(r); });
        }
    }
};

// Where the keys of a part of a piece lie: the page table's entries for it, in LDS.
struct table_part {
    const int32_t* entries;
    uint32_t first, page_size;
    int shift;                       // page_size = 1 << shift, or -1
    int64_t page_stride, token_stride;
    __device__ __forceinline__ int64_t place(int j) const {
        const uint32_t n = shift >= 0 ? (uint32_t)j >> shift : (uint32_t)j / page_size;
        return entries[n - first] * page_stride + (int64_t)((uint32_t)j - n * page_size) * token_stride;
    }
    // The places of keys j, j + step, ... (N of them), the same for all lanes (page_size a power of two): one read of the entries,
    // a lane for each.
    template <int N>
    __device__ __forceinline__ void places(int j, int step, int64_t (&at)[N]) const {
        const int e = entries[((uint32_t)(j + (int)(threadIdx.x % N) * step) >> shift) - first];
#pragma unroll
        for (int i = 0; i < N; ++i)
            at[i] = (int64_t)__builtin_amdgcn_readlane(e, i) * page_stride + (int64_t)((uint32_t)(j + i * step) & (page_size - 1)) * token_stride;
    }
};

// Brings in the entries of keys begin .. end - 1 (few enough: part_keys()); the caller waits.
template <int THREADS>
__device__ inline table_part load_table(const fq_tree_args& a, int b, int begin, int end, int32_t* entries) {
    table_part t;
    t.entries = entries;
    t.page_size = (uint32_t)a.cache.page_size;
    t.shift = (a.cache.page_size & (a.cache.page_size - 1)) == 0 ? __builtin_ctz(a.cache.page_size) : -1;
    t.first = (uint32_t)begin / t.page_size;
    t.page_stride = a.cache.page_stride;
    t.token_stride = a.cache.token_stride;
    const int count = (int)((uint32_t)(end - 1) / t.page_size - t.first) + 1;
    const int32_t* row = a.page_table + b * a.table_width + t.first;
    for (int i = threadIdx.x % THREADS; i < count; i += THREADS) {
        const int32_t page = row[i];
        entries[i] = page < 0 ? 0 : (int32_t)min((uint32_t)page, (uint32_t)(a.cache.pages - 1));
    }
    return t;
}
// Whether the few neighbouring keys of one load lie in one page and within 32 bits of each other
__device__ inline bool near_keys(const fq_tree_args& a, int keys) {
    const int page = a.cache.page_size;
    return (page & (page - 1)) == 0 && page >= keys && a.cache.token_stride < (int64_t)1 << 24;
}

// The end of a piece whose keys PARTS waves of a block have shared out: wave first + i * step has part i of the rows from 32 group on.
// Their sums go through LDS, 32 rows in `bytes` of each wave; stats: [4][32][2] and a flag.
template <int ACT, int DP, int PARTS>
__device__ __forceinline__ void join_parts(const unit_rows& rows, const wave_state<ACT, DP>& w, char* lds, int bytes, float* stats, int first,
                                           int step, int part, int group, int key0, int key1, float* slot) {
    constexpr int TURN = DP / 4 == 24 ? 7 : 15;         // units of four sums are moved about by row
    const int lane = threadIdx.x & 63, wave = first + part * step, D = rows.a.head_dim;
    __syncthreads();                                    // (nobody reads the keys and values that lay here, nor the sums of the piece before)
    if (threadIdx.x == 0) stats[256] = 0.0f;
    __syncthreads();
    if (!w.sound() && lane == 0) stats[256] = 1.0f;
    if (lane < 32) {
        stats[(wave * 32 + lane) * 2] = w.top();
        stats[(wave * 32 + lane) * 2 + 1] = w.l;
    }
    w.quads([&](int d, int i, int t) {
        const f32x16& o = w.o[t];
        const f32x4 x = {o[i], o[i + 1], o[i + 2], o[i + 3]};
        const int r = lane & 31;
        *(f32x4*)((float*)(lds + wave * bytes) + r * DP + ((d / 4) ^ (r & TURN)) * 4) = x;
    });
    __syncthreads();
    if (stats[256] != 0.0f) {
        rows.one_by_one<ACT>(key0, key1, slot, 32 * group + part, min(rows.count, 32 * group + 32), PARTS);
    } else {
        for (int x = part * 64 + lane; x < 32 * (DP / 4); x += 64 * PARTS) {
            const int r = x / (DP / 4), d = x % (DP / 4) * 4, at = 32 * group + r;
            if (at >= rows.count || d >= D) continue;
            float c = -__builtin_inff(), l = 0.0f;
#pragma unroll
            for (int y = 0; y < PARTS; ++y) c = __builtin_fmaxf(c, stats[(first + y * step) * 64 + r * 2]);
            const float from = c == -__builtin_inff() ? 0.0f : c;
            f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int y = 0; y < PARTS; ++y) {
                const int other = first + y * step;
                const float weight = __builtin_amdgcn_exp2f(stats[other * 64 + r * 2] - from);
                const f32x4 z = *(const f32x4*)((const float*)(lds + other * bytes) + r * DP + ((d / 4) ^ (r & TURN)) * 4);
                l += weight * stats[other * 64 + r * 2 + 1];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] += weight * z[i];
            }
            if (!slot) {
                const float scale = inverse(l, [&] { return rows.sees_any(at); });
                const u32x2 z = {pack2<ACT>(o[0] * scale, o[1] * scale), pack2<ACT>(o[2] * scale, o[3] * scale)};
                *(u32x2*)(rows.result(at) + d) = z;
            } else {
                *(f32x4*)(slot + rows.p.shape().at(at, d)) = o;
                if (d == 0) rows.p.shape().put_stats(slot, at, c, l);
            }
        }
    }
    __syncthreads();
}

// ------------------------------------------------------------------------------------------ up to 32 rows
// A wave takes 32 rows of one key head and 32 keys at a time, which it brings into 2 x 32 rows of LDS of its own: the next keys
// are on their way while the present ones are used, values likewise, and no barrier is needed.  Two blocks of 64 KiB fill a
// compute unit.  A block's four waves are HEADS key heads x PARTS parts of a tile of 32 PARTS keys; where they share the keys out, they
// join their sums through LDS at the end of a piece.
//
// Bound by the cache's bytes: 64 sequences of 100 - 8191 tokens, one new token each, 32 heads over 8 of 128 values in bfloat16, 437 MB
// in 75 us = 5.8 TB/s (a kernel that only reads: 7.1).  By latency where keys are few: one sequence of 777 tokens 9 us, reads that
// wait for each other (lengths, page table, keys, sums).
template <int ACT, int DP, int HEADS>
__global__ __launch_bounds__(256, 2) void fq_attention_tree_stream_kernel(fq_tree_args a, tree_plan p) {
    typedef tile_shape<DP> SH;
    constexpr int LOADS = SH::BYTES / 1024;             // 16-byte loads per lane for 32 rows
    constexpr int STEP = 64 / SH::UNITS;                // rows per load
    constexpr int PERIOD = LOADS < 4 ? LOADS : 4;       // loads after which the rows' units lie alike again
    constexpr int JOIN = 32 * DP * 4;                   // bytes of 32 rows of sums
    constexpr int WAVE_BYTES = 2 * SH::BYTES > JOIN ? 2 * SH::BYTES : JOIN;
    constexpr int PARTS = 4 / HEADS;
    constexpr int TILE = 32 * PARTS;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = wave % HEADS, part_of = wave / HEADS;
    int32_t* entries = (int32_t*)(lds + 4 * WAVE_BYTES) + wave * (TABLE / 4);
    float* stats = (float*)(lds + 4 * WAVE_BYTES + TABLE * 4);       // [4][32][2], and a flag
    const int D = a.head_dim;
    char* mine = lds + wave * WAVE_BYTES;
    const uint32_t mine_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine;
    const int row0 = lane / SH::UNITS, spot = lane % SH::UNITS;
    const bool near = near_keys(a, STEP);
    uint32_t key_off[PERIOD], value_off[PERIOD];        // lane offsets of a load, bytes
#pragma unroll
    for (int j = 0; j < PERIOD; ++j) {
        key_off[j] = (uint32_t)row0 * (uint32_t)a.cache.token_stride * 2 + key_unit<SH::UNITS>(row0 + j * STEP, spot) * 16;
        value_off[j] = (uint32_t)row0 * (uint32_t)a.cache.token_stride * 2 + value_unit<SH::UNITS>(row0 + j * STEP, spot) * 16;
    }

    const line all(a, p);
    const int64_t begin = blockIdx.x * all.per_block, stop = min(all.total, begin + all.per_block);
    if (begin >= stop) return;
    int b;
    int64_t at_b;
    all.find(begin, &b, &at_b);
    int context = all.context(b), tiles = tiles_of(a, p, context);
    int u = (int)quotient(begin - at_b, tiles), t0 = (int)(begin - at_b - (int64_t)u * tiles);
    wave_state<ACT, DP> w;

    for (int64_t pos = begin; pos < stop;) {
        const unit_rows rows(a, p, b, u, head, context);
        const int t1 = (int)min((int64_t)tiles, t0 + stop - pos);
        float* slot = t0 == 0 && t1 == tiles ? nullptr : p.slot(blockIdx.x, pos == begin, head);
        const int key0 = t0 * TILE, key1 = p.whole ? rows.keys : min(rows.keys, t1 * TILE);
        const int row = min(lane & 31, rows.count - 1);
        w.load_query(rows.query(row), D);
        w.clear();
        const int most = part_keys(TABLE / 4, a.cache.page_size, TILE);
        for (int part = key0, part_end; part < key1; part = part_end) {
            part_end = fqa::part_end(part, key1, most);
            const table_part table = load_table<64>(a, b, part, part_end, entries);
            if (D < SH::UNITS * 8) {                    // units that no load fills: zeros
                const u32x4 zero = {0, 0, 0, 0};
                for (int x = lane; x < 2 * SH::BYTES / 16; x += 64) ((u32x4*)mine)[x] = zero;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the wave's own: no barrier)
            w.query_is_here();                          // (with the table)
            const uint16_t *k = (const uint16_t*)a.cache.k + rows.head * a.cache.head_stride, *v = (const uint16_t*)a.cache.v + rows.head * a.cache.head_stride;
            int64_t at[LOADS];                          // places of the loads' first rows, where a load lies in a page
            auto load = [&](const uint16_t* from, int base, uint32_t to, const uint32_t (&off)[PERIOD], bool values) {
                if (near && base + 32 <= part_end) {
#pragma unroll
                    for (int j = 0; j < LOADS; ++j) {
                        const int unit = values ? value_unit<SH::UNITS>(row0 + j * STEP, spot) : key_unit<SH::UNITS>(row0 + j * STEP, spot);
                        if (unit * 8 < D) load_lds16<true>(to + j * 1024, from + at[j], off[j % PERIOD]);
                    }
                } else {                                // (no row behind the last: what lies there may be anything)
#pragma unroll 1
                    for (int j = 0; j < LOADS; ++j) {
                        const int r = row0 + j * STEP;
                        const int unit = values ? value_unit<SH::UNITS>(r, spot) : key_unit<SH::UNITS>(r, spot);
                        const uint16_t* src = from + table.place(min(base + r, part_end - 1)) + unit * 8;
                        if (unit * 8 < D) load_lds16(to + j * 1024, src);
                    }
                }
            };
            int base = part + part_of * 32;
            if (base < part_end) {
                if (near && base + 32 <= part_end) table.template places<LOADS>(base, STEP, at);
                load(k, base, mine_at, key_off, false);
                load(v, base, mine_at + SH::BYTES, value_off, true);
            }
            for (; base < part_end; base += TILE) {
                const bool more = base + TILE < part_end;
                f32x16 s[1];
                u32x4 x[2];
                if (near && base + TILE + 32 <= part_end) table.template places<LOADS>(base + TILE, STEP, at);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");       // keys are here
                w.template scores<1>(mine, s);
                if (more) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    load(k, base + TILE, mine_at, key_off, false);
                }
                if (base + 32 > min(rows.context, part_end)) keep_seen(s[0], rows.seen(row, base));
                w.template soften<1>(s, p.factor, x);
                if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");       // values are here
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                w.template accumulate<1>(mine + SH::BYTES, x);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (more) load(v, base + TILE, mine_at + SH::BYTES, value_off, true);
            }
        }
        w.finish(PARTS > 1 || slot);
        if constexpr (PARTS == 1) {
            if (!w.sound()) rows.one_by_one<ACT>(key0, key1, slot, 0, rows.count, 1);
            else if ((lane & 31) < rows.count) w.put(rows.result(row), slot, p.shape(), row, [&] { return rows.sees_any(row); });
        } else {
            join_parts<ACT, DP, PARTS>(rows, w, lds, WAVE_BYTES, stats, head, HEADS, part_of, 0, key0, key1, slot);
        }
        pos += t1 - t0;
        t0 = 0;
        if (++u == all.units) {
            u = 0;
            if (++b < a.sequences) context = all.context(b), tiles = tiles_of(a, p, context);
        }
    }
}

// ------------------------------------------------------------------------------------------ above 32 rows
// GROUPS x 32 rows a block; tiles of 64 keys that all waves read, two of them in LDS, as for prompts.  Four groups: every wave takes
// all keys of a tile.  Two (tiles of 64 rows): two pairs of waves take half a tile each, and join their sums.
//
// 131 000 tokens, 16 drafted, 32 heads over 8 of 128 values (64 rows): 537 MB in 93 us = 5.8 TB/s, bound by what is on its way at once (a tile a
// block; the matrix units are busy 15 % of the time).  Eight sequences of 500 - 4095, 48 drafted (192 rows): 12 GF in 39 us; a block has a
// dozen tiles of keys, and once or twice a beginning and an end that wait for memory.
template <int ACT, int DP, int GROUPS>
__global__ __launch_bounds__(256, 2) void fq_attention_tree_tile_kernel(fq_tree_args a, tree_plan p) {
    typedef tile_shape<DP> SH;
    constexpr int TILE_BYTES = 2 * SH::BYTES;
    constexpr int STEP = 256 / SH::UNITS;
    constexpr int JOIN = 32 * DP * 4;                   // bytes of 32 rows of sums
    static_assert(4 * JOIN <= 4 * TILE_BYTES, "");
    extern __shared__ __align__(16) char lds[];
    constexpr int PARTS = 4 / GROUPS, HALVES = 2 / PARTS;
    int32_t* entries = (int32_t*)(lds + 4 * TILE_BYTES);
    float* stats = (float*)(entries + TABLE);           // [4][32][2], and a flag
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = wave % GROUPS, part_of = wave / GROUPS;
    const int D = a.head_dim;
    const int row0 = threadIdx.x / SH::UNITS, spot = threadIdx.x % SH::UNITS;
    const int key_at = key_unit<SH::UNITS>(row0, spot) * 8, value_at = value_unit<SH::UNITS>(row0, spot) * 8;
    const bool near = near_keys(a, STEP / 4);
    const uint32_t in_page = (uint32_t)(lane / SH::UNITS) * (uint32_t)a.cache.token_stride * 2, key_off = in_page + key_at * 2, value_off = in_page + value_at * 2;

    const line all(a, p);
    const int64_t block = p.in_line(blockIdx.x), begin = block * all.per_block, stop = min(all.total, begin + all.per_block);
    if (begin >= stop) return;
    int b;
    int64_t at_b;
    all.find(begin, &b, &at_b);
    int context = all.context(b), tiles = tiles_of(a, p, context);
    int u = (int)quotient(begin - at_b, tiles), t0 = (int)(begin - at_b - (int64_t)u * tiles);
    wave_state<ACT, DP> w;

    for (int64_t pos = begin; pos < stop;) {
        const unit_rows rows(a, p, b, u, 0, context);
        const int t1 = (int)min((int64_t)tiles, t0 + stop - pos);
        float* slot = t0 == 0 && t1 == tiles ? nullptr : p.slot(block, pos == begin, 0);
        const int key0 = t0 * KEYS, key1 = p.whole ? rows.keys : min(rows.keys, t1 * KEYS);
        const int r = group * 32 + (lane & 31), row = min(r, rows.count - 1);
        const bool busy = group * 32 < rows.count;
        w.load_query(rows.query(row), D);
        w.clear();
        const int most = part_keys(TABLE, a.cache.page_size, KEYS);
        for (int part = key0, part_end; part < key1; part = part_end) {
            part_end = fqa::part_end(part, key1, most);
            __syncthreads();
            const table_part table = load_table<256>(a, b, part, part_end, entries);
            if (D < SH::UNITS * 8) {                    // units that no load fills: zeros
                const u32x4 zero = {0, 0, 0, 0};
                for (int x = threadIdx.x; x < 4 * TILE_BYTES / 16; x += 256) ((u32x4*)lds)[x] = zero;
            }
            __syncthreads();
            w.query_is_here();                          // (with the table)
            const uint16_t *k = (const uint16_t*)a.cache.k + rows.head * a.cache.head_stride, *v = (const uint16_t*)a.cache.v + rows.head * a.cache.head_stride;
            auto load = [&](int base, int buffer) {
                const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(lds + buffer * 2 * TILE_BYTES) + wave * 1024;
                if (near && base + KEYS <= part_end) {
                    int64_t place[TILE_BYTES / 4096];
                    table.template places<TILE_BYTES / 4096>(base + wave * (STEP / 4), STEP, place);
                    auto all_of = [&](auto once) {
#pragma unroll
                        for (int j = 0; j < TILE_BYTES / 4096; ++j) {
                            if (key_at < D) load_lds16<once.value>(to + j * 4096, k + place[j], key_off);
                            if (value_at < D) load_lds16<once.value>(to + TILE_BYTES + j * 4096, v + place[j], value_off);
                        }
                    };
                    if (p.once) all_of(std::true_type());
                    else all_of(std::false_type());
                } else {
#pragma unroll 1
                    for (int j = 0; j < TILE_BYTES / 4096; ++j) {
                        const int64_t place = table.place(min(base + row0 + j * STEP, part_end - 1));
                        if (key_at < D) load_lds16(to + j * 4096, k + place + key_at);
                        if (value_at < D) load_lds16(to + TILE_BYTES + j * 4096, v + place + value_at);
                    }
                }
            };
            load(part, 0);
            for (int base = part, buffer = 0; base < part_end; base += KEYS, buffer ^= 1) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (base + KEYS < part_end) load(base + KEYS, buffer ^ 1);
                if (!busy) continue;
                const char* at = lds + buffer * 2 * TILE_BYTES + part_of * SH::BYTES;
                const int from = base + part_of * HALF;
                f32x16 s[HALVES];
                u32x4 x[2 * HALVES];
                w.template scores<HALVES>(at, s);
                if (from + HALVES * HALF > min(rows.context, part_end)) {
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) keep_seen(s[h], rows.seen(row, from + h * HALF));
                }
                w.template soften<HALVES>(s, p.factor, x);
                w.template accumulate<HALVES>(at + TILE_BYTES, x);
            }
        }
        w.finish(PARTS > 1 || slot);
        if constexpr (PARTS > 1) {
            join_parts<ACT, DP, PARTS>(rows, w, lds, JOIN, stats, group, GROUPS, part_of, group, key0, key1, slot);
        } else {
            if (!w.sound()) rows.one_by_one<ACT>(key0, key1, slot, group * 32, min(group * 32 + 32, rows.count), 1);
            else if (r < rows.count) w.put(rows.result(r), slot, p.shape(), r, [&] { return rows.sees_any(r); });
        }
        pos += t1 - t0;
        t0 = 0;
        if (++u == all.units) {
            u = 0;
            if (++b < a.sequences) context = all.context(b), tiles = tiles_of(a, p, context);
        }
    }
}

// Joins the pieces of a unit that was cut.  A lane has four values of a row, a wave up to 32 rows of them.  A unit of few pieces: each
// wave its own values; of many: the waves share the pieces of the same values out.  Pieces are added in the line's order.
// Bound by latency (lengths, then sums, four on their way at once): 16 rows of 25 pieces 5 us, 64 sequences of 16 rows and 5 pieces 7, eight of 192
// rows and 5 pieces, 23 MB, 9.
template <int ACT>
__global__ __launch_bounds__(1024) void fq_attention_tree_join_kernel(fq_tree_args a, tree_plan p) {
    __shared__ f32x4 sums[16][64];
    __shared__ float stats[16][64][2];
    const int waves = blockDim.x / 64;
    const line all(a, p);
    const int b = (int)(blockIdx.x / (unsigned)all.units), u = (int)blockIdx.x - b * all.units;
    const int context = all.context(b), tiles = tiles_of(a, p, context);
    const int64_t begin = all.begin(b) + (int64_t)u * tiles, end = begin + tiles;
    const int64_t from = quotient(begin, all.per_block), to = quotient(end - 1, all.per_block);        // blocks that have pieces of it
    if (from == to) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.head_dim;
    const bool whole = begin == from * all.per_block;        // (the first block's first piece, or its last)
    // lanes: rows that lie side by side, of as many quads as a wave has room for
    const int side = min(32, p.rows), groups = (p.slot_rows + 31) / 32, quads = 64 / side;
    const int sub = p.by_side.quotient(lane), r0 = lane - sub * side, units = p.heads * groups * (D / 4);
    // Waves share pieces out where a unit's values leave blocks with little else to do, or where there are very many (64 drafted tokens, 8
    // sequences, 9 pieces and 64 values for each wave: shared out 18.5 us, a wave its own values 12.8).
    const bool many = to - from >= (units <= 2 * quads * (int)gridDim.y ? 8 : 32);
    const int share = many ? ((int)(to - from) + waves) / waves : (int)(to - from + 1), mine = many ? wave : 0;
    const int step = quads * (many ? 1 : waves);
    for (int base = blockIdx.y * step; base < units; base += gridDim.y * step) {
        const int y = base + (many ? 0 : wave * quads) + sub, z = p.by_quads.quotient(y), d = (y - z * (D / 4)) * 4;
        const int head = groups == 1 ? z : z / groups, r = (z - head * groups) * 32 + r0;
        const unit_rows rows(a, p, b, u, min(head, p.heads - 1), context);
        const bool there = sub < quads && y < units && r < rows.count;
        partial_sums sum;
        sum.clear();
        if (there) {
            // (a unit's first piece may be its block's last one, the others are their blocks' first)
            const int n0 = mine * share, n1 = min((int)(to - from) + 1, n0 + share);
            sum.add(n0, n1, [&](int y) { return p.slot(from + y, y > 0 || whole, head); }, p.shape(), r, d);
        }
        if (many) {
            __syncthreads();
            sums[wave][lane] = sum.o;
            stats[wave][lane][0] = sum.c;
            stats[wave][lane][1] = sum.l;
            __syncthreads();
            if (wave == 0)
                for (int i = 1; i < waves; ++i) sum.add(stats[i][lane][0], stats[i][lane][1], sums[i][lane]);
        }
        if (there && (wave == 0 || !many)) sum.template store<ACT>(rows.result(r) + d, [&] { return rows.sees_any(r); });
    }
}

// Rows of a tile, where a key head has `rows` of them.
// (129 - 192 rows, heads above 96: three tiles of 64 rather than two of 128, a quarter of whose waves had nothing to do: 48 drafted tokens of
// eight sequences of 500 - 4095, groups of four: 49.8 -> 45.6 us; heads of 96, 160 rows, 32.6, in three 33.4)
int rows_of_tile(int64_t rows, int head_dim) { return rows <= 64 || (rows > 128 && rows <= 192 && head_dim > 96) ? 64 : ROWS; }

tree_plan plan_tree(const fq_tree_args& a) {
    tree_plan p = {};
    p.group = a.q_heads / a.kv_heads;
    p.rows = a.nodes * p.group;      // (fq_tree_fits)
    // Few rows: the waves take neighbouring heads, whose rows of a token lie side by side: 4 x 256 bytes come in 10 % faster than
    // 256.  That makes four times as many pieces as waves that share the keys out, of sums that are no longer few from 16 rows on.
    p.heads = p.rows > 16 ? 1 : a.kv_heads % 4 == 0 ? 4 : a.kv_heads % 2 == 0 ? 2 : 1;
    p.unit_rows = rows_of_tile(p.rows, a.head_dim);
    p.row_tiles = (p.rows + p.unit_rows - 1) / p.unit_rows;
    p.slot_rows = p.rows < 32 ? p.rows : ((p.rows < p.unit_rows ? p.rows : p.unit_rows) + 31) / 32 * 32;
    p.D = a.head_dim;
    p.by_group = divisor::of((uint32_t)p.group);
    p.by_quads = divisor::of((uint32_t)a.head_dim / 4);
    p.by_side = divisor::of((uint32_t)(p.rows < 32 ? p.rows : 32));
    p.tile = p.rows > 32 ? KEYS : 128 / p.heads;
    // Units of few tiles are left whole: a block is through with four tiles as soon as with one and the join, and with eight where there are
    // blocks' worth of units (102 sequences of 223 tokens, 3 units each of 7 tiles: 24.4 -> 18.6 us; one of 250, 2 units of 8: 13.7, whole 18.8).
    const int64_t tiles = (a.table_width * a.cache.page_size + p.tile - 1) / p.tile, units = a.sequences * (a.kv_heads / p.heads) * p.row_tiles;
    p.whole = tiles <= (units >= 128 ? 8 : 4);
    p.by_lanes = a.sequences <= 64 && a.sequences * tiles < INT32_MAX;
    // 131 000 tokens, 537 MB, 64 rows 113.6 -> 103.1 us, 268 MB 49.2 -> 47.1; 100 000, 96 rows 99.6 -> 90.5; what the 256 MiB Infinity Cache may still hold from the last call: 16 sequences
    // of 2000 - 4000, 100 MB, 39.0, past it 41.3.
    p.once = p.row_tiles == 1 && (double)a.sequences * a.table_width * a.cache.page_size * a.kv_heads * a.head_dim * 4 > 0x1p28;
    p.blocks = 2 * fq_cu_count();
    p.factor = a.scale * LOG2E;
    return p;
}

template <int ACT, int DP, int HEADS>
int launch_stream(const fq_tree_args& a, const tree_plan& p, hipStream_t stream) {
    constexpr int WAVE_BYTES = 2 * tile_shape<DP>::BYTES > 128 * DP ? 2 * tile_shape<DP>::BYTES : 128 * DP;
    static std::atomic<uint64_t> raised{0};
    const int st = fqd::raise_lds_limit((const void*)fq_attention_tree_stream_kernel<ACT, DP, HEADS>, raised);
    if (st != FQ_OK) return st;
    fq_attention_tree_stream_kernel<ACT, DP, HEADS><<<(unsigned)p.blocks, 256, 4 * WAVE_BYTES + TABLE * 4 + 257 * 4, stream>>>(a, p);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

template <int ACT, int DP, int GROUPS>
int launch_tiles(const fq_tree_args& a, const tree_plan& p, hipStream_t stream) {
    static std::atomic<uint64_t> raised{0};
    const int st = fqd::raise_lds_limit((const void*)fq_attention_tree_tile_kernel<ACT, DP, GROUPS>, raised);
    if (st != FQ_OK) return st;
    fq_attention_tree_tile_kernel<ACT, DP, GROUPS><<<(unsigned)p.blocks, 256, 8 * tile_shape<DP>::BYTES + TABLE * 4 + 257 * 4, stream>>>(a, p);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

template <int ACT, int DP>
int launch(const fq_tree_args& a, const tree_plan& p, hipStream_t stream) {
    const int st = p.unit_rows > 64 ? launch_tiles<ACT, DP, 4>(a, p, stream)
                   : p.rows > 32    ? launch_tiles<ACT, DP, 2>(a, p, stream)
                   : p.heads == 4   ? launch_stream<ACT, DP, 4>(a, p, stream)
                   : p.heads == 2   ? launch_stream<ACT, DP, 2>(a, p, stream)
                                    : launch_stream<ACT, DP, 1>(a, p, stream);
    if (st != FQ_OK || p.whole) return st;
    // A block for each unit at least, more for its rows while units are few; sixteen waves where few units may be of hundreds of pieces.
    const int64_t units = a.sequences * (a.kv_heads / p.heads) * p.row_tiles;
    const int64_t most = (p.heads * (p.slot_rows < p.rows ? p.slot_rows : p.rows) + 1) / 2, wanted = 1024 / units;
    const dim3 grid((unsigned)units, (unsigned)(wanted < 1 ? 1 : wanted < most ? wanted : most));
    const bool hundreds = units < 16 && a.table_width * a.cache.page_size > 64 * (int64_t)p.tile;
    fq_attention_tree_join_kernel<ACT><<<grid, hundreds ? 1024 : 256, 0, stream>>>(a, p);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

template <int ACT>
int launch(const fq_tree_args& a, const tree_plan& p, hipStream_t stream) {
    if (a.head_dim <= 64) return launch<ACT, 64>(a, p, stream);
    if (a.head_dim <= 96) return launch<ACT, 96>(a, p, stream);
    return launch<ACT, 128>(a, p, stream);
}

}  // namespace

bool fq_tree_fits(const fq_tree_args& a) {
    const int64_t rows = (int64_t)a.nodes * (a.q_heads / a.kv_heads), tile = rows_of_tile(rows, a.head_dim);
    if (rows > 1 << 30) return false;                                            // (they and a tile more are counted in 32 bits)
    return a.sequences * a.kv_heads * ((rows + tile - 1) / tile) < 1 << 24;      // (2^32 threads)
}

size_t fq_tree_bytes(const fq_tree_args& a) {
    const tree_plan p = plan_tree(a);
    return p.whole ? 0 : (size_t)p.blocks * 2 * p.heads * p.shape().floats() * sizeof(float);
}

int fq_launch_attention_tree(int act_dtype, const fq_tree_args& a, void* workspace, hipStream_t stream) {
    tree_plan p = plan_tree(a);
    p.slots = (float*)workspace;
    return act_dtype == FQ_F16 ? launch<FQ_F16>(a, p, stream) : launch<FQ_BF16>(a, p, stream);
}
