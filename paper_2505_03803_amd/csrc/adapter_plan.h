// How adapters.hip shares its calls out: rules on their sizes, plain functions of the description of the rows (AdapterRowsDev, or what has its fields),
// some of which the kernels evaluate as well.
#pragma once
#include <algorithm>

namespace rwkvq {

// The rank as the kernels pad it: 16, 32, 64 or 128.
constexpr int padded_rank(int rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : rank <= 64 ? 64 : 128; }
// How many pieces or tiles of up to `cut` rows of one sequence a call has: with offsets, which the host does not know, room for as many as there can be.
template <class Rows>
constexpr long long pieces(const Rows& r, int cut) {
    if (r.offsets) return (long long)r.n_tokens / cut + r.n_seqs;
    return ((long long)(r.n_tokens / r.n_seqs) + cut - 1) / cut * r.n_seqs;
}

// Single tokens, whose rows are gathered by adapter, and the workgroups that a tile of them takes at most (gather_rows).
constexpr int kGathered = 2048;                    // rows of such a call at most
template <class Rows>
constexpr int groups_of(const Rows& r) {
    const long long most = (long long)r.n_adapters + 1 + r.n_seqs / 16;
    return most < r.n_seqs && r.n_seqs > 16 ? (int)most : r.n_seqs;
}
template <class Rows>
constexpr bool single_tokens(const Rows& r) {
    return !r.offsets && r.n_tokens == r.n_seqs && r.n_seqs > 1 && r.n_seqs <= kGathered && !r.drop.seed;
}

// Rows of a tile: 16, of which two workgroups fit a compute unit, one's copies beside the other's products, unless there are enough tiles of 32 as
// well, or tiles of 16 would take too much of Q through the caches.  Measured, 16 against 32 (us): K = N = 4096, rank 16: 8192 rows 45 / 54; rank 32: 4096
// rows 30 / 31, 8192 49 / 54, 16384 92 / 95; rank 64: 2048 rows 22 / 25, 3000 30 / 29, 4096 41 / 37, 8192 76 / 59; K = N = 1024, 16384 rows: rank 32
// 27 / 24, 64 37 / 31; N = 14336: 4320 rows at rank 16 79 / 75, 32 107 / 80, 64 130 / 104, 2000 at rank 64 59 / 48, 1000 28 / 29.  So 32 from 170
// tiles of 16 above rank 32 and 620 up to it, or 5 2^23 values of Q that tiles of 32 take, never for rank 16.  Above rank 64 the registers of 16 rows are full.
// `wide`: columns of y of all matrices.
template <class Rows>
int tile_rows(const Rows& r, int n_mats, double wide) {
    if (r.rank <= 16 || r.rank > 64 || r.n_tokens / r.n_seqs <= 16) return 16;
    return pieces(r, 16) * n_mats > (r.rank > 32 ? 170 : 620) || r.rank * wide * pieces(r, 32) > 5 << 23 ? 32 : 16;
}
// Columns of y that a wavefront takes at a time, of ranks up to 16 RT in tiles of 16 MT rows, and the wavefronts of a workgroup.
constexpr int kAdapterWaves = 8;
constexpr int wave_cols(int RT, int MT) { return RT <= 2 || MT == 2 ? 64 : 32; }
// Slices of a tile, which read the same x, are on one die, a multiple of eight workgroups apart (4321 rows beside 14336 columns in three 82 -> 80 us, 333 rows
// of four matrices 17 -> 14); those of fewer tiles than sixteen, which would be on few dies, are not (one token 7 us, on one die 9.5).
constexpr bool spread(long long tiles) { return tiles >= 16; }
// Columns of a workgroup: all of them from 256 workgroups on; of fewer, as many slices as make the fullest compute unit's time least, by what goes through
// its cache: every slice takes h again, (rows + rank) values for each of the depth, then rank values of Q, base and y for each of its columns.
// Workgroups that share a unit take 0.7 of their times together, 0.85 above rank 32; one that fills a unit waits for the one in front.  Measured, 1, 2, 3
// and 4 slices (us): 3500 rows, K = N = 4096, rank 16 23.3, 21.7, 26.8, 29.3; 2500 rows at rank 64 28.4, 31.2, 32.5, 41.9; 4321 rows beside N = 14336
// at rank 32 97, 94, 80, 95; 3000 rows with K = 14336 at rank 32 48, 62, 72, 81; 2048 rows at rank 128 in 2 and 3 34 and 53.  Groups of single tokens,
// whose number the host does not know, as many as one a unit where they are few, otherwise one and a half (four matrices, 16 rows of 16 adapters 9 us,
// one and a half 11; 128 of 8 14, 17; 64 rows of 32 at rank 64 one and a half 45, one 50).
// rows: of a tile; widest, deepest: of the matrices; wide_y: y is binary32.
template <class Rows>
int slice_of(const Rows& r, int rows, int n_mats, int widest, int deepest, bool wide_y) {
    const int R = padded_rank(r.rank);
    const int most = (widest + 255) / 256;
    auto width = [&](long long slices) { return (int)(((widest + slices - 1) / slices + 63) / 64 * 64); };
    if (single_tokens(r)) {
        const long long wgs = (long long)n_mats * std::min(groups_of(r), std::max(r.n_adapters, (r.n_seqs + 15) / 16));
        return width(wgs >= 256 ? 1 : std::min<long long>(most, ((wgs <= 64 ? 256 : 384) + wgs - 1) / wgs));
    }
    const long long tiles = pieces(r, rows), wgs = tiles * n_mats;
    const bool fills = R > 64 || (rows == 32 && (R > 32 || r.drop.seed || wide_y));       // a unit (waves_of)
    const double together = fills ? 1.0 : R > 32 ? 0.85 : 0.7, h = 2.0 * (rows + R) * deepest, column = 2.0 * R + rows * (wide_y ? 8.0 : 4.0);
    int best = width(1);
    double least = 0;
    for (int slices = 1; wgs < 256 && slices <= most && (slices == 1 || slices * wgs <= 768); ++slices) {
        const int wide = width(slices);
        const long long die = (tiles + 7) / 8 * slices * n_mats, fullest = slices > 1 && spread(tiles) ? (die + 31) / 32 : (slices * wgs + 255) / 256;
        const double time = (fullest == 1 ? 1.0 : together * fullest) * (h + column * wide);
        if (slices == 1 || time < least) {
            least = time;
            best = wide;
        }
    }
    return best;
}

// Columns of a workgroup of the sums over tokens, and how many workgroups a matrix's N + K columns are.
constexpr int outer_tiles(int rank) { return rank <= 64 ? 4 : 2; }
constexpr int outer_cols(int rank) { return 64 * outer_tiles(rank); }
constexpr int outer_chunks(int rank, int N, int K) { return (N + outer_cols(rank) - 1) / outer_cols(rank) + (K + outer_cols(rank) - 1) / outer_cols(rank); }
// Rows of a piece: 64, and twice as many while two workgroups a compute unit are left, since every piece leaves sums of rank (K + N) floats (gradients of 8192
// rows at rank 64: pieces of 256 rows 146 us, of 512 123, of 1024 132).
template <class Rows>
constexpr int cut_of(const Rows& r, long long chunks) {
    int cut = 64;
    while (cut < 4096 && pieces(r, 2 * cut) * chunks >= 512) cut *= 2;
    return cut;
}

}  // namespace rwkvq
