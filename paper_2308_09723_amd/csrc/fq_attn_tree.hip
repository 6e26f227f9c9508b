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

#include "fq_attn_units.h"
#include "fq_lds_limit.h"

namespace {

using namespace fqa;

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
        const unit_rows<paged_rows> rows(a, p, b, u, head, context);
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
        const unit_rows<paged_rows> rows(a, p, b, u, 0, context);
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

tree_plan plan_tree(const fq_tree_args& a) {
    // Few rows: the waves take neighbouring heads, whose rows of a token lie side by side: 4 x 256 bytes come in 10 % faster than
    // 256.  That makes four times as many pieces as waves that share the keys out, of sums that are no longer few from 16 rows on.
    const int rows = a.nodes * (a.q_heads / a.kv_heads);
    const int heads = rows > 16 ? 1 : a.kv_heads % 4 == 0 ? 4 : a.kv_heads % 2 == 0 ? 2 : 1;
    tree_plan p = plan_units(a, heads, rows_of_tile(rows, a.head_dim), rows > 32 ? KEYS : 128 / heads, 0);
    // 131 000 tokens, 537 MB, 64 rows 113.6 -> 103.1 us, 268 MB 49.2 -> 47.1; 100 000, 96 rows 99.6 -> 90.5; what the 256 MiB Infinity Cache may still hold from the last call: 16 sequences
    // of 2000 - 4000, 100 MB, 39.0, past it 41.3.
    p.once = p.row_tiles == 1 && (double)a.sequences * a.table_width * a.cache.page_size * a.kv_heads * a.head_dim * 4 > 0x1p28;
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
    return launch_join<ACT, paged_rows>(a, p, stream);
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
    return slots_bytes(plan_tree(a));
}

int fq_launch_attention_tree(int act_dtype, const fq_tree_args& a, void* workspace, hipStream_t stream) {
    tree_plan p = plan_tree(a);
    p.slots = (float*)workspace;
    return act_dtype == FQ_F16 ? launch<FQ_F16>(a, p, stream) : launch<FQ_BF16>(a, p, stream);
}
