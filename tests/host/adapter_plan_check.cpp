// How a call of the adapters is shared out (csrc/adapter_plan.h): for each line "seqs tokens adapters rank offsets drop mats depth wide wide_y"
// the rows of a tile, the slices of its columns, how often a wavefront goes round in one, and the rows of a piece of the sums over tokens.
#include "adapter_plan.h"

#include <cstdio>

using namespace rwkvq;

struct Rows {
    int n_seqs, n_tokens, n_adapters, rank;
    bool offsets;
    struct { bool seed; } drop;
};

int main() {
    Rows r;
    int offsets, drop, mats, depth, wide, wide_y;
    while (std::scanf("%d %d %d %d %d %d %d %d %d %d", &r.n_seqs, &r.n_tokens, &r.n_adapters, &r.rank, &offsets, &drop, &mats, &depth, &wide, &wide_y) == 10) {
        r.offsets = offsets; r.drop.seed = drop;
        const int rows = tile_rows(r, mats, (double)mats * wide), slice = slice_of(r, rows, mats, wide, depth, wide_y);
        const int at_a_time = kAdapterWaves * wave_cols(padded_rank(r.rank) / 16, rows / 16);
        std::printf("%d %d %d %d\n", rows, (wide + slice - 1) / slice, (std::min(slice, wide) + at_a_time - 1) / at_a_time,
                    cut_of(r, (long long)mats * outer_chunks(r.rank, depth, wide)));
    }
    return 0;
}
