// The parts in which a block goes through a piece's keys: as many at a time as it has room for entries of the page table.
// Key numbers reach 2^31 - 1025 and a part 2^30 keys, so that the sum of a part's beginning and its length may lie beyond 32 bits.
// (Plain C++, so that the host's compiler can check it at its limits.)
#ifndef FQ_ATTN_PARTS_H_
#define FQ_ATTN_PARTS_H_

#include <stdint.h>

#ifdef __HIP__
#define FQ_EITHER __host__ __device__
#else
#define FQ_EITHER
#endif

namespace fqa {

// Keys of a part, whole tiles, where `entries` of the page table fit (a part may begin within a page: one entry is for that)
FQ_EITHER inline int part_keys(int entries, int page_size, int tile) {
    const int64_t keys = (int64_t)(entries - 1) * page_size, most = (int64_t)1 << 30;
    return (int)(keys < most ? keys : most) / tile * tile;
}

// Where the part from key `begin` on ends, of keys up to `end` (begin < end)
FQ_EITHER inline int part_end(int begin, int end, int keys) { return end - begin <= keys ? end : begin + keys; }

}  // namespace fqa

#endif  // FQ_ATTN_PARTS_H_
