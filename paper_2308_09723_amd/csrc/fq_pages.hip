// Pages that sequences share: taking, forking, freeing and gathering them, and copies of what they hold (fq_pages_*).
//
// refs[p] says how many rows of tables hold page p (none: free).  Free pages are handed out in their order, the lowest first, whatever the
// blocks' order: a scan over refs by one block gives each free page its rank, and whoever wants pages his.  References are counted with
// integer atomics, whose order does not matter.
//
// Bookkeeping is bound by latency (a few reads that wait for each other), copies by memory.  Where tables are small one block does
// all of a fork's bookkeeping in one kernel; the copies are a second one, since they want the whole card.  Gathering 1358 pages of 2038 (of 72 KiB in each
// of 16 layers): 6.4 us to find the moves, 4.7 to rename the table's entries, 213 for copies that read and write 1.07 GB, 5.0 TB/s, what a large copy reaches.  A token more
// for each of 64 rows 2.2 us, where each needs a page for it, of 2500 pages, 9.4.
#include <hip/hip_runtime.h>

#include "fq_attn.h"
#include "fq_internal.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 1024;             // of a block that does the bookkeeping
constexpr int MOST_ROWS = FQ_MOST_PAGE_ROWS;

// refs is read past the vector caches: the same kernel's atomics may have changed it
__device__ __forceinline__ int refs_of(const int32_t* refs, int64_t p) { return __hip_atomic_load(refs + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void refer(int32_t* refs, int64_t pages, int32_t page, int by) {
    if (page >= 0 && page < pages) __hip_atomic_fetch_add(refs + page, by, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The sum of x over the threads before this one, and over all (a block of THREADS; sums: LDS of 17 words)
__device__ inline int sum_before(int x, int* sums, int* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
    }
    __syncthreads();                      // (sums of the call before have been read)
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const int s = sums[w];
        before += w < wave ? s : 0;
        total += s;
    }
    *all = total;
    return before + upto - x;
}

// Hands page(k, p) the free pages below `end`, k their ranks, until `wanted` are found; how many were found (up to wanted).  One block.
template <typename PAGE>
__device__ inline int each_free(const int32_t* refs, int64_t end, int wanted, int* sums, const PAGE& page) {
    constexpr int EACH = 8;
    int found = 0;
    for (int64_t base = 0; base < end && found < wanted; base += THREADS * EACH) {
        const int64_t p = base + threadIdx.x * EACH;
        uint32_t free = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (p + i < end && refs_of(refs, p + i) <= 0) free |= 1u << i;
        int all;
        int k = found + sum_before(__builtin_popcount(free), sums, &all);
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (free >> i & 1) {
                if (k < wanted) page(k, p + i);
                ++k;
            }
        found += all;
    }
    return found < wanted ? found : wanted;
}

__device__ __forceinline__ int pages_of(int len, int page_size) { return len <= 0 ? 0 : (len - 1) / page_size + 1; }

// ------------------------------------------------------------------------------------------ forks
// What becomes of child i: whole pages that it shares with its parent, and whether it has a last page that is not whole
struct child_of {
    int parent, len, whole;
    bool part;
    __device__ child_of(const fq_fork_args& a, int i) : child_of(a, a.parents[i], a.lens) {}
    __device__ child_of(const fq_fork_args& a, int parent, const int32_t* lens) : parent(parent) {
        const bool there = parent >= 0 && parent < a.rows;
        len = there ? lens[parent] : 0;
        const int64_t used = pages_of(len, a.page_size);
        const bool fits = used <= a.width;          // (a table has no more than it has room for)
        whole = (int)(fits ? (len > 0 ? len / a.page_size : 0) : a.width);
        part = fits && len > 0 && len % a.page_size != 0;
    }
};

// The first child of each row
__device__ inline void fork_first(const fq_fork_args& a) {
    for (int r = threadIdx.x; r < a.rows; r += THREADS) a.first[r] = INT32_MAX;
    __syncthreads();
    for (int i = threadIdx.x; i < a.children; i += THREADS) {
        const int p = a.parents[i];
        if (p >= 0 && p < a.rows) __hip_atomic_fetch_min(a.first + p, i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

// Tables and references of whole pages, entry by entry: threads `at`, at + step, ...
__device__ inline void fork_entries(const fq_fork_args& a, int64_t at, int64_t step) {
    const int64_t entries = (int64_t)a.children * a.width;
    for (int64_t e = at; e < entries; e += step) {
        const int i = (int)(e / a.width), j = (int)(e - (int64_t)i * a.width);
        const child_of c(a, i);
        const int32_t* row = a.table + (int64_t)c.parent * a.width;
        int32_t page = -1;
        if (j < c.whole) {
            page = row[j];
            refer(a.refs, a.pages, page, 1);
        } else if (j == c.whole && c.part && a.release && __hip_atomic_load(a.first + c.parent, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i) {
            page = row[j];                          // the row's own passes to its first child
        }
        a.table_out[e] = page;
        if (j == 0) a.lens_out[i] = c.len;
    }
    if (a.width == 0)
        for (int64_t i = at; i < a.children; i += step) a.lens_out[i] = child_of(a, (int)i).len;
    if (!a.release) return;
    const int64_t old = (int64_t)a.rows * a.width;
    for (int64_t e = at; e < old; e += step) {
        const int r = (int)(e / a.width), j = (int)(e - (int64_t)r * a.width), len = a.lens[r];
        if (j >= pages_of(len, a.page_size)) continue;
        const bool passed = j == len / a.page_size && __hip_atomic_load(a.first + r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != INT32_MAX;
        if (!passed) refer(a.refs, a.pages, a.table[e], -1);
    }
}

// Children whose last page is not whole and not their parent's own: listed in from[], in their order
__device__ inline int fork_wanted(const fq_fork_args& a, int* sums) {
    int wanted = 0;
    for (int base = 0; base < a.children; base += THREADS) {
        const int i = base + threadIdx.x;
        bool wants = false;
        if (i < a.children) {
            const child_of c(a, i);
            wants = c.part && !(a.release && __hip_atomic_load(a.first + c.parent, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i);
        }
        int all;
        const int k = wanted + sum_before(wants, sums, &all);
        if (wants) a.from[k] = i;                   // (for now: who wants a page)
        wanted += all;
    }
    __syncthreads();
    return wanted;
}
// Pages for them: who(k) is the k-th
struct who_wants {
    int child, parent, whole;
};
template <typename WHO>
__device__ inline void fork_last(const fq_fork_args& a, int* sums, int wanted, const WHO& who) {
    const int found = each_free(a.refs, a.pages, wanted, sums, [&](int k, int64_t p) {
        const who_wants w = who(k);
        a.table_out[(int64_t)w.child * a.width + w.whole] = (int32_t)p;
        a.refs[p] = 1;
        a.from[k] = a.table[(int64_t)w.parent * a.width + w.whole];
        a.to[k] = (int32_t)p;
    });
    // children that there was no page for: nothing is left of them
    for (int k = found; k < wanted; ++k) {
        const who_wants w = who(k);
        for (int j = threadIdx.x; j < w.whole; j += THREADS) {
            int32_t* entry = a.table_out + (int64_t)w.child * a.width + j;
            refer(a.refs, a.pages, *entry, -1);
            *entry = -1;
        }
        if (threadIdx.x == 0) a.lens_out[w.child] = -1;
    }
    if (threadIdx.x == 0) *a.moves = found;
}

// All of it by one block, up to SMALL children and rows: what becomes of each is worked out once, and the entries' reads do not wait for each other.
// References change once for each page of an old row, by its children's number (less one where it is given up), since one compute unit counts but one at a
// time; where old rows stay that are more than twice the children, once for each child's, so that a large table is not gone through for a few of its rows.  Bound by latency: 4
// children of 4 rows 6.4 us, 256 of 256 of up to 33 pages 16 (17.5 where each child and each old row counted its own).  With the copies' launch, old rows staying, 4 children
// of 1024 rows of 2048 entries 13.5, by rows 417; 256 of 257 rows of 64 17.8 by rows, by children 23.6.
constexpr int SMALL = 1024;
__global__ __launch_bounds__(THREADS) void fq_pages_fork_kernel(fq_fork_args a, fqa::divisor by_width) {
    __shared__ int sums[THREADS / 64 + 1];
    __shared__ int32_t lens[SMALL];
    __shared__ int first[SMALL], count[SMALL];      // child of each row; children
    __shared__ int whole[SMALL], source[SMALL];     // of a child: full pages; its parent, -1 - its parent where the last page passes to it, INT32_MIN: none
    __shared__ int changed[SMALL];                  // of a row: entries whose references change; then who wants pages
    constexpr int EACH = 8;
    const int t = threadIdx.x, width = (int)a.width, parent = t < a.children ? a.parents[t] : -1;
    const bool there = parent >= 0 && parent < a.rows;
    first[t] = INT32_MAX;
    count[t] = 0;
    lens[t] = t < a.rows ? a.lens[t] : 0;
    __syncthreads();
    bool wants = false;
    if (t < a.children) {
        const child_of c(a, parent, lens);
        if (there) {
            atomicMin(&first[parent], t);
            atomicAdd(&count[parent], 1);
        }
        whole[t] = c.whole;
        a.lens_out[t] = c.len;
        source[t] = there ? parent : INT32_MIN;
        wants = c.part;
    }
    __syncthreads();
    if (wants && a.release && first[parent] == t) {
        source[t] = -1 - parent;
        wants = false;
    }
    if (t < a.rows) {
        const child_of row(a, t, lens);
        // (the last page of a row that is given up and has no child goes with the others; if it has one, to that)
        changed[t] = count[t] == (a.release ? 1 : 0) ? 0 : row.whole + (a.release && count[t] == 0 && row.part ? 1 : 0);
    }
    __syncthreads();
    const bool by_row = a.release || a.rows <= 2 * a.children;
    const int entries = a.children * width, old = by_row ? a.rows * width : 0;       // (no more than twice what the launch has counted)
    for (int e0 = t; e0 < max(entries, old); e0 += THREADS * EACH) {
        int32_t page[EACH], of[EACH];
#pragma unroll
        for (int y = 0; y < EACH; ++y) {
            const int e = e0 + y * THREADS, i = by_width.quotient(e), j = e - i * width;
            page[y] = of[y] = -1;
            if (e < entries) {
                const int from = source[i];
                if (from != INT32_MIN && (j < whole[i] || (from < 0 && j == whole[i]))) page[y] = a.table[(from < 0 ? -1 - from : from) * width + j];
            }
            if (e < old && j < changed[i]) of[y] = a.table[e];
        }
#pragma unroll
        for (int y = 0; y < EACH; ++y) {
            const int e = e0 + y * THREADS;
            if (e < entries) a.table_out[e] = page[y];
            if (!by_row) refer(a.refs, a.pages, page[y], 1);       // (full pages: the copy of one that is not comes later)
            if (e < old) refer(a.refs, a.pages, of[y], count[by_width.quotient(e)] - (a.release ? 1 : 0));
        }
    }
    __syncthreads();
    int wanted;
    const int k = sum_before(wants, sums, &wanted);
    if (wants) changed[k] = t;
    __syncthreads();
    fork_last(a, sums, wanted, [&](int k) { return who_wants{changed[k], source[changed[k]], whole[changed[k]]}; });
}
__global__ __launch_bounds__(THREADS) void fq_pages_fork_first_kernel(fq_fork_args a) { fork_first(a); }
__global__ __launch_bounds__(256) void fq_pages_fork_entries_kernel(fq_fork_args a) {
    fork_entries(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}
__global__ __launch_bounds__(THREADS) void fq_pages_fork_last_kernel(fq_fork_args a) {
    __shared__ int sums[THREADS / 64 + 1];
    const int wanted = fork_wanted(a, sums);
    fork_last(a, sums, wanted, [&](int k) {
        const int i = a.from[k];
        const child_of c(a, i);
        return who_wants{i, c.parent, c.whole};
    });
}

// ------------------------------------------------------------------------------------------ taking and freeing
// Pages for the tokens that rows are to have: the pages of all rows make one line, of which free page k is the k-th.
__global__ __launch_bounds__(THREADS) void fq_pages_take_kernel(fq_take_args a) {
    __shared__ int sums[THREADS / 64 + 1];
    __shared__ int upto[MOST_ROWS + 1];             // pages that rows before want
    int total = 0;
    for (int base = 0; base < a.rows; base += THREADS) {
        const int i = base + threadIdx.x;
        int wants = 0;
        if (i < a.rows) {
            const int len = a.lens[i], wanted = a.wanted[i];
            const int64_t have = pages_of(len, a.page_size), then = pages_of(wanted, a.page_size);
            if (len >= 0 && wanted > len && then <= a.width) wants = (int)(then - have);
        }
        int all;                                    // (at most 2^17 each of 2^13 rows)
        const int before = sum_before(wants, sums, &all);
        if (i < a.rows) upto[i] = total + before;
        total += all;
    }
    if (threadIdx.x == 0) upto[a.rows] = total;
    __syncthreads();
    const int wanted = total;
    const int found = each_free(a.refs, a.pages, wanted, sums, [&](int k, int64_t p) {
        int low = 0, high = a.rows;                 // the last row whose pages begin at k or before
        while (high - low > 1) {
            const int middle = (low + high) / 2;
            if (upto[middle] <= k) low = middle;
            else high = middle;
        }
        a.table[(int64_t)low * a.width + pages_of(a.lens[low], a.page_size) + (k - upto[low])] = (int32_t)p;
        a.refs[p] = 1;
    });
    __syncthreads();
    for (int i = threadIdx.x; i < a.rows; i += THREADS) {
        const int len = a.lens[i], then = a.wanted[i], first = upto[i], last = upto[i + 1];
        if (len < 0 || then <= len || pages_of(then, a.page_size) > a.width) continue;
        if (last <= found || first == last) {
            a.lens[i] = then;
        } else {                                    // what it has of them goes back
            const int64_t at = (int64_t)i * a.width + pages_of(len, a.page_size);
            for (int k = first; k < min(last, found); ++k) {
                refer(a.refs, a.pages, a.table[at + k - first], -1);
                a.table[at + k - first] = -1;
            }
        }
    }
}

// The rows' references.  A row that is named twice is freed once: whoever takes an entry out of the table gives its reference up.
__global__ __launch_bounds__(256) void fq_pages_free_kernel(fq_free_args a) {
    const int64_t r = a.which ? a.which[blockIdx.x] : blockIdx.x;
    if (r < 0 || r >= a.rows) return;
    int32_t* row = a.table + r * a.width;
    const int64_t used = min((int64_t)pages_of(__hip_atomic_load(a.lens + r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), a.page_size), a.width);
    for (int64_t j = threadIdx.x; j < used; j += 256)
        refer(a.refs, a.pages, __hip_atomic_exchange(row + j, -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), -1);
    __syncthreads();
    if (threadIdx.x == 0) __hip_atomic_store(a.lens + r, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ------------------------------------------------------------------------------------------ gathering
// The used pages, U of them, to pages 0 .. U - 1: those from U on go into the free ones below, both in their order.
__global__ __launch_bounds__(THREADS) void fq_pages_compact_kernel(fq_compact_args a) {
    __shared__ int sums[THREADS / 64 + 1];
    constexpr int EACH = 4;
    int count = 0;
    for (int64_t p = threadIdx.x; p < a.pages; p += THREADS) count += a.refs[p] > 0;
    int used;
    sum_before(count, sums, &used);
    const int holes = each_free(a.refs, used, INT32_MAX, sums, [&](int k, int64_t p) { a.to[k] = (int32_t)p; });
    __syncthreads();
    int found = 0;
    for (int64_t base = used; base < a.pages; base += THREADS * EACH) {
        const int64_t p = base + threadIdx.x * EACH;
        int refs[EACH], mine = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            refs[i] = p + i < a.pages ? a.refs[p + i] : 0;
            mine += refs[i] > 0;
        }
        int all;
        int k = found + sum_before(mine, sums, &all);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (p + i >= a.pages) continue;
            int32_t to = (int32_t)(p + i);
            if (refs[i] > 0) {
                to = a.to[k];
                a.from[k] = (int32_t)(p + i);
                a.refs[to] = refs[i];
                a.refs[p + i] = 0;
                ++k;
            }
            a.place[p + i] = to;
        }
        found += all;
    }
    if (threadIdx.x == 0) {
        a.moves[0] = holes;
        a.moves[1] = used;
    }
}
__global__ __launch_bounds__(256) void fq_pages_rename_kernel(fq_compact_args a) {
    const int64_t entries = (int64_t)a.rows * a.width;
    const int used = a.moves[1];
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < entries; e += (int64_t)gridDim.x * 256) {
        const int r = (int)(e / a.width), j = (int)(e - (int64_t)r * a.width);
        const int32_t page = a.table[e];
        if (page >= used && page < a.pages && j < pages_of(a.lens[r], a.page_size)) a.table[e] = a.place[page];
    }
}

// ------------------------------------------------------------------------------------------ copies
// Pages from[m] to pages to[m], for every m below `moves` (or *count), of every buffer: pieces of 16 KiB, one block's turn each.  (148 pages of 72 KiB in 8
// layers 26 us: 6.7 TB/s, some of it from the Infinity Cache.)
__global__ __launch_bounds__(256) void fq_pages_copy_kernel(fq_copy_args a) {
    constexpr int EACH = 4;                                       // 16-byte units of a thread
    const int64_t moves = a.count ? *a.count : a.moves, pieces = moves * a.pieces;
    for (int64_t x = blockIdx.x; x < pieces; x += gridDim.x) {
        const int64_t m = x / a.pieces;
        int64_t piece = x - m * a.pieces;
        int b = 0;
        while (b + 1 < a.buffers && piece >= a.first[b + 1]) ++b;  // (few buffers)
        piece -= a.first[b];
        const fq_page_buffer& buffer = a.buffer[b];
        const int64_t each = (buffer.page_bytes + 256 * EACH * 16 - 1) / (256 * EACH * 16), tensor = piece / each, at = (piece - tensor * each) * (256 * EACH);
        const int64_t from = a.from[m], to = a.to[m];
        if (from < 0 || from >= a.pages || to < 0 || to >= a.pages || from == to) continue;
        char* data = (char*)buffer.data + tensor * buffer.stride;
        const u32x4* source = (const u32x4*)(data + from * buffer.page_stride);
        u32x4* target = (u32x4*)(data + to * buffer.page_stride);
        const int64_t units = buffer.page_bytes / 16;
        u32x4 v[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int64_t u = at + i * 256 + threadIdx.x;
            if (u < units) v[i] = __builtin_nontemporal_load(source + u);
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int64_t u = at + i * 256 + threadIdx.x;
            if (u < units) target[u] = v[i];
        }
    }
}

int status() { return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_HIP; }

unsigned blocks_for(int64_t entries) {
    const int64_t blocks = (entries + 255) / 256;
    return (unsigned)(blocks < 1 ? 1 : blocks > 2048 ? 2048 : blocks);
}

}  // namespace

int fq_launch_pages_copy(const fq_page_buffer* buffers, int count, fq_copy_args a, hipStream_t stream) {
    // (as many buffers as the kernel's arguments hold at a time)
    for (int first = 0; first < count; first += FQ_COPY_BUFFERS) {
        a.buffers = count - first < FQ_COPY_BUFFERS ? count - first : FQ_COPY_BUFFERS;
        a.pieces = 0;
        for (int b = 0; b < a.buffers; ++b) {
            a.buffer[b] = buffers[first + b];
            a.first[b] = a.pieces;
            a.pieces += buffers[first + b].count * ((buffers[first + b].page_bytes + 16383) / 16384);
        }
        const int64_t pieces = a.pieces * a.moves;
        if (pieces == 0) continue;
        fq_pages_copy_kernel<<<(unsigned)(pieces < 2048 ? pieces : 2048), 256, 0, stream>>>(a);
        const int st = status();
        if (st != FQ_OK) return st;
    }
    return FQ_OK;
}

int fq_launch_pages_fork(const fq_fork_args& a, hipStream_t stream) {
    const int64_t entries = ((int64_t)a.children + (a.release ? a.rows : 0)) * a.width;
    if (entries <= 64 * THREADS && a.children <= SMALL && a.rows <= SMALL && a.width > 0) {
        fq_pages_fork_kernel<<<1, THREADS, 0, stream>>>(a, fqa::divisor::of((uint32_t)a.width));
        return status();
    }
    fq_pages_fork_first_kernel<<<1, THREADS, 0, stream>>>(a);
    fq_pages_fork_entries_kernel<<<blocks_for(entries), 256, 0, stream>>>(a);
    fq_pages_fork_last_kernel<<<1, THREADS, 0, stream>>>(a);
    return status();
}

int fq_launch_pages_take(const fq_take_args& a, hipStream_t stream) {
    fq_pages_take_kernel<<<1, THREADS, 0, stream>>>(a);
    return status();
}

int fq_launch_pages_free(const fq_free_args& a, int count, hipStream_t stream) {
    fq_pages_free_kernel<<<(unsigned)count, 256, 0, stream>>>(a);
    return status();
}

int fq_launch_pages_compact(const fq_compact_args& a, hipStream_t stream) {
    fq_pages_compact_kernel<<<1, THREADS, 0, stream>>>(a);
    if (a.rows > 0 && a.width > 0) fq_pages_rename_kernel<<<blocks_for((int64_t)a.rows * a.width), 256, 0, stream>>>(a);
    return status();
}
