// Walks the parts of a piece's keys as the kernels over a paged cache do, at the lengths that the library admits.
#include <stdio.h>

#include "../paper_2308_09723_amd/csrc/fq_attn_parts.h"

int main() {
    const int most = INT32_MAX - 1024;
    const int pages[] = {1, 2, 7, 16, 64, 1000, 4096, 1 << 20, 1 << 22, (1 << 22) + 1, 1 << 28, 1 << 30, most};
    const int shapes[][2] = {{256, 32}, {256, 64}, {256, 128}, {1024, 64}};      // entries, tile
    long walks = 0, wrong = 0;
    for (int page : pages)
        for (const auto& shape : shapes) {
            const int keys = fqa::part_keys(shape[0], page, shape[1]);
            if (keys <= 0 || keys % shape[1] != 0) ++wrong;
            const int ends[] = {1, 31, 1 << 20, 1 << 30, (1 << 30) + 5, most - 65472, most - 1, most};
            const int begins[] = {0, 1 << 29, 1 << 30, 3 << 29, most - 200000};
            for (int end : ends)
                for (int from : begins) {
                    const int begin = from / shape[1] * shape[1];
                    if (begin >= end) continue;
                    ++walks;
                    int64_t covered = begin;
                    bool good = true;
                    for (int part = begin; good && part < end;) {
                        const int stop = fqa::part_end(part, end, keys);
                        good = part == covered && stop > part && stop <= end && (stop == end || stop - part == keys) &&
                               (stop - 1) / page - part / page + 1 <= shape[0];
                        covered = stop;
                        part = stop;
                    }
                    if (!good || covered != end) {
                        ++wrong;
                        printf("pages of %d, %d entries, tiles of %d: keys %d .. %d\n", page, shape[0], shape[1], begin, end);
                    }
                }
        }
    printf("%ld walks, %ld wrong\n", walks, wrong);
    return wrong != 0;
}
