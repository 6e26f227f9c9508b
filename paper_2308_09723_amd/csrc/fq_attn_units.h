// Attention of drafted tokens over the pages of a cache: how the work is dealt out and joined, whatever the cache holds.
//
// All sequences' key tiles, key head by key head, make one line, of which each block takes an equal piece (see line); where a unit (a sequence's
// rows of one key head) is cut, the pieces leave their sums in slots of the workspace, and a second kernel joins them.
#ifndef FQ_ATTN_UNITS_H_
#define FQ_ATTN_UNITS_H_

#include <hip/hip_runtime.h>

#include "fq_attn_parts.h"
#include "fq_attn_tile.h"

namespace fqa {

constexpr int TABLE = 1024;          // entries of the page table that a block has in LDS

// What the host has made of a call.
struct tree_plan {
    int group, rows;                 // query heads per key head; rows of a key head
    divisor by_group, by_quads, by_side;       // divisors: group; head_dim / 4; rows of a slot that lie side by side
    int heads;                       // key heads that a block takes together
    int row_tiles, unit_rows;        // tiles of unit_rows rows that a head's are cut into
    int tile;                        // keys of a tile
    int extra;                       // tiles' worth of time that a unit's beginning and end take: so many places in the line that hold nothing
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
                tiles = tiles_of(a, p, mine) + p.extra;
            }
            upto = sum_upto(tiles);
            total = (int64_t)__builtin_amdgcn_readlane(upto, 63) * units;
        } else {
            int64_t sum = 0;
            for (int b = lane; b < a.sequences; b += 64) sum += tiles_of(a, p, a.context_lens[b]) + p.extra;
            total = uniform(wave_sum64(sum)) * units;
        }
        per_block = quotient(total + p.blocks - 1, p.blocks);
    }
    __device__ int context(int b) const { return p.by_lanes ? __builtin_amdgcn_readlane(mine, b) : __builtin_amdgcn_readfirstlane(a.context_lens[b]); }
    // where sequence b's tiles begin
    __device__ int64_t begin(int b) const {
        if (p.by_lanes) return (int64_t)(__builtin_amdgcn_readlane(upto, b) - __builtin_amdgcn_readlane(tiles, b)) * units;
        int64_t before = 0;
        for (int x = threadIdx.x & 63; x < b; x += 64) before += tiles_of(a, p, a.context_lens[x]) + p.extra;
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
            const int b = first + lane, n = b < a.sequences ? tiles_of(a, p, a.context_lens[b]) + p.extra : 0;
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

// Rows of a unit: where a row's query lies, where its result goes, and what it sees.  CACHE: how a head's keys and values are read one by one.
template <typename CACHE>
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
            attend_one<ACT>(query(r), CACHE::of(a, b, head), sees_tree{context, a.nodes, words(r)}, begin, end, a.head_dim, p.factor, o, c, l);
        } else {
            const int last = (int)min((int64_t)end, (int64_t)context + p.by_group.quotient(first + r) + 1);
            attend_one<ACT>(query(r), CACHE::of(a, b, head), sees_first{last}, begin, min(end, last), a.head_dim, p.factor, o, c, l);
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
template <int ACT, int DP, int PARTS, typename UNIT>
__device__ __forceinline__ void join_parts(const UNIT& rows, const wave_state<ACT, DP>& w, char* lds, int bytes, float* stats, int first,
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
        rows.template one_by_one<ACT>(key0, key1, slot, 32 * group + part, min(rows.count, 32 * group + 32), PARTS);
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

// Joins the pieces of a unit that was cut.  A lane has four values of a row, a wave up to 32 rows of them.  A unit of few pieces: each
// wave its own values; of many: the waves share the pieces of the same values out.  Pieces are added in the line's order.
// Bound by latency (lengths, then sums, four on their way at once): 16 rows of 25 pieces 5 us, 64 sequences of 16 rows and 5 pieces 7, eight of 192
// rows and 5 pieces, 23 MB, 9.
template <int ACT, typename CACHE>
__global__ __launch_bounds__(1024) void fq_attention_tree_join_kernel(fq_tree_args a, tree_plan p) {
    __shared__ f32x4 sums[16][64];
    __shared__ float stats[16][64][2];
    const int waves = blockDim.x / 64;
    const line all(a, p);
    const int b = (int)(blockIdx.x / (unsigned)all.units), u = (int)blockIdx.x - b * all.units;
    const int context = all.context(b), tiles = tiles_of(a, p, context);
    const int64_t begin = all.begin(b) + (int64_t)u * (tiles + p.extra), end = begin + tiles;
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
        const unit_rows<CACHE> rows(a, p, b, u, min(head, p.heads - 1), context);
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
inline int rows_of_tile(int64_t rows, int head_dim) { return rows <= 64 || (rows > 128 && rows <= 192 && head_dim > 96) ? 64 : ROWS; }

// The plan of a call whose blocks take `heads` key heads together (up to 32 rows a head; above, one) and unit_rows rows of each, `tile` keys at a time; extra:
// see tree_plan.
inline tree_plan plan_units(const fq_tree_args& a, int heads, int unit_rows, int tile, int extra) {
    tree_plan p = {};
    p.group = a.q_heads / a.kv_heads;
    p.rows = a.nodes * p.group;      // (fq_tree_fits)
    p.heads = heads;
    p.unit_rows = unit_rows;
    p.row_tiles = (p.rows + p.unit_rows - 1) / p.unit_rows;
    p.slot_rows = p.rows < 32 ? p.rows : ((p.rows < p.unit_rows ? p.rows : p.unit_rows) + 31) / 32 * 32;
    p.D = a.head_dim;
    p.by_group = divisor::of((uint32_t)p.group);
    p.by_quads = divisor::of((uint32_t)a.head_dim / 4);
    p.by_side = divisor::of((uint32_t)(p.rows < 32 ? p.rows : 32));
    p.tile = tile;
    // Units of few tiles are left whole: a block is through with four tiles as soon as with one and the join, and with eight where there are
    // blocks' worth of units (102 sequences of 223 tokens, 3 units each of 7 tiles: 24.4 -> 18.6 us; one of 250, 2 units of 8: 13.7, whole 18.8).
    const int64_t tiles = (a.table_width * a.cache.page_size + p.tile - 1) / p.tile, units = a.sequences * (a.kv_heads / p.heads) * p.row_tiles;
    p.whole = tiles <= (units >= 128 ? 8 : 4);
    p.extra = p.whole ? 0 : extra;
    p.by_lanes = a.sequences <= 64 && a.sequences * (tiles + p.extra) < INT32_MAX;
    p.blocks = 2 * fq_cu_count();
    p.factor = a.scale * LOG2E;
    return p;
}

inline size_t slots_bytes(const tree_plan& p) { return p.whole ? 0 : (size_t)p.blocks * 2 * p.heads * p.shape().floats() * sizeof(float); }

// The join of the units that the plan's blocks cut.
template <int ACT, typename CACHE>
int launch_join(const fq_tree_args& a, const tree_plan& p, hipStream_t stream) {
    // A block for each unit at least, more for its rows while units are few; sixteen waves where few units may be of hundreds of pieces.
    const int64_t units = a.sequences * (a.kv_heads / p.heads) * p.row_tiles;
    const int64_t most = (p.heads * (p.slot_rows < p.rows ? p.slot_rows : p.rows) + 1) / 2, wanted = 1024 / units;
    const dim3 grid((unsigned)units, (unsigned)(wanted < 1 ? 1 : wanted < most ? wanted : most));
    const bool hundreds = units < 16 && a.table_width * a.cache.page_size > 64 * (int64_t)p.tile;
    fq_attention_tree_join_kernel<ACT, CACHE><<<grid, hundreds ? 1024 : 256, 0, stream>>>(a, p);
    return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP;
}

}  // namespace fqa

#endif  // FQ_ATTN_UNITS_H_
