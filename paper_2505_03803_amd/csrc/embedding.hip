// Rows of a table by token, and the table's gradient (include/rwkvq.h).
#include "pieces.h"

namespace rwkvq {

// A thread takes eight columns of a token's row.
template <int TDT, int ODT>
__global__ void __launch_bounds__(256) embedding_kernel(EmbeddingDev p) {
    const uint32_t pieces = (uint32_t)(p.d + 7) / 8;
    const long long all = (long long)p.n_tokens * pieces, step = (long long)gridDim.x * 256;
    long long item = (long long)blockIdx.x * 256 + threadIdx.x;
    for (RowWalk w((uint32_t)item, pieces, (uint32_t)step); item < all; item += step, w.next()) {
        const int col = 8 * (int)w.at, left = p.d - col, token = p.tokens[w.row];
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (token >= 0 && token < p.vocab) {
            load8<TDT>(x, p.table, (long long)token * p.d + col, left, p.table_whole);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= p.scale;
        }
        store8<ODT>(p.out, w.row * p.out_stride + col, x, left, p.rows_whole);
    }
}

template <int TDT>
static void embed(const EmbeddingDev& p, int odt, dim3 grid, hipStream_t s) {
    switch (odt) {
        case DT_F16: hipLaunchKernelGGL((embedding_kernel<TDT, DT_F16>), grid, dim3(256), 0, s, p); break;
        case DT_BF16: hipLaunchKernelGGL((embedding_kernel<TDT, DT_BF16>), grid, dim3(256), 0, s, p); break;
        default: hipLaunchKernelGGL((embedding_kernel<TDT, DT_F32>), grid, dim3(256), 0, s, p);
    }
}
hipError_t launch_embedding(EmbeddingDev p, int tdt, int odt, hipStream_t s) {
    p.table_whole = p.d % (tdt == DT_F32 ? 4 : 8) == 0;
    p.rows_whole = p.out_stride % (odt == DT_F32 ? 4 : 8) == 0;
    const long long all = (long long)p.n_tokens * ((p.d + 7) / 8);
    const dim3 grid((unsigned)std::min<long long>((all + 255) / 256, 4096));
    switch (tdt) {
        case DT_F16: embed<DT_F16>(p, odt, grid, s); break;
        case DT_BF16: embed<DT_BF16>(p, odt, grid, s); break;
        default: embed<DT_F32>(p, odt, grid, s);
    }
    return hipGetLastError();
}

// ---- the gradient: tokens sorted, runs of equal ones summed in the order of their places --------------------------------

constexpr int kSortTile = 8192;               // tokens whose order is found by counting
constexpr int kRankRows = 32;                 // of which a workgroup takes so many

__device__ __forceinline__ uint32_t key_of(const EmbeddingDev& p, int i) {
    const int token = p.tokens[i];
    return token >= 0 && token < p.vocab ? (uint32_t)token : (uint32_t)p.vocab;     // tokens without a row come last
}

// The place of a token among those of its tile: how many are smaller, or equal and in front of it.  A workgroup takes 32 tokens, each in two lanes of
// every wavefront; its sixteen wavefronts compare them with a sixteenth of the tile each, four keys a read from LDS, a half of the lanes every
// other four.  Two vector instructions a pair and a read from LDS for every four: 8192 tokens 10.7 us.
__global__ void __launch_bounds__(1024) rank_kernel(EmbeddingDev p) {
    __shared__ __align__(16) uint32_t others[16][kSortTile / 16];
    __shared__ int counts[16][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int chunk = blockIdx.x * kRankRows, tile = chunk / kSortTile * kSortTile, size = min(kSortTile, p.n_tokens - tile), mine = chunk + (lane & 31);
    // keys of a wavefront: a multiple of 32 of them, so that those of the workgroup's tokens are one wavefront's
    const int span = ((size + 15) / 16 + 31) / 32 * 32, from = tile + wave * span;
    const uint32_t key = mine < p.n_tokens ? key_of(p, mine) : 0;
    for (int i = lane; i < span; i += 64) others[wave][i] = from + i < tile + size ? key_of(p, from + i) : 0xFFFFFFFFu;
    __syncthreads();
    int count = 0;
    const int half = lane >> 5 << 2;
    auto four = [&](int i) { return *(const uint4_t*)&others[wave][i + half]; };
    const int before = min(max(chunk - from, 0), span), inside = min(max(chunk + kRankRows - from, 0), span);
#pragma unroll 4
    for (int i = 0; i < before; i += 8) {
        const uint4_t k = four(i);
#pragma unroll
        for (int j = 0; j < 4; ++j) count += k[j] <= key;
    }
    for (int i = before; i < inside; i += 8) {
        const uint4_t k = four(i);
#pragma unroll
        for (int j = 0; j < 4; ++j) count += k[j] < key || (k[j] == key && from + i + half + j < mine);
    }
#pragma unroll 4
    for (int i = inside; i < span; i += 8) {
        const uint4_t k = four(i);
#pragma unroll
        for (int j = 0; j < 4; ++j) count += k[j] < key;
    }
    counts[wave][lane] = count;
    __syncthreads();
    if (threadIdx.x < kRankRows && mine < p.n_tokens) {
        count = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) count += counts[w][lane] + counts[w][lane + 32];
        p.tile_keys[tile + count] = key;
        p.tile_order[tile + count] = mine;
    }
}

// How many of the sorted keys [from, to) are below `key`, or below or equal.
__device__ __forceinline__ int below(const uint32_t* keys, int from, int to, uint32_t key, bool equal) {
    const int first = from;
    while (from < to) {
        const int mid = (from + to) >> 1;
        const uint32_t k = keys[mid];
        if (k < key || (equal && k == key)) from = mid + 1;
        else to = mid;
    }
    return from - first;
}
// The places of tokens in sorted tiles among all of them.
__global__ void __launch_bounds__(256) merge_kernel(EmbeddingDev p) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= p.n_tokens) return;
    const uint32_t key = p.tile_keys[i];
    const int own = i / kSortTile;
    int place = i - own * kSortTile;
    for (int t = 0; t * kSortTile < p.n_tokens; ++t)
        if (t != own) place += below(p.tile_keys, t * kSortTile, min((t + 1) * kSortTile, p.n_tokens), key, t < own);
    p.keys[place] = key;
    p.order[place] = p.tile_order[i];
}

// E pieces of V columns of a lane, 8 in all: piece e is at column 64 V e + V lane of a wavefront's 512, so that loads of either width
// are of neighbouring columns.  V: 16 bytes of 16-bit (8) or binary32 (4) values where rows begin at multiples of that, otherwise 1.
template <int DT_, int V>
struct Columns {
    static constexpr int E = 8 / V;
    int first, d;
    __device__ __forceinline__ int at(int e) const { return first + 64 * V * e; }
    __device__ __forceinline__ bool live(int e) const { return at(e) < d; }          // d is a multiple of V
    __device__ __forceinline__ void load(float (&f)[8], const void* p, long long row) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            Piece<DT_, V> v;
            v.clear();
            if (live(e)) v.load(p, row + at(e));
            float w[V];
            v.widen(w);
#pragma unroll
            for (int j = 0; j < V; ++j) f[e * V + j] = w[j];
        }
    }
    __device__ __forceinline__ void load_sums(float (&f)[8], const float* p, long long row) const {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int j = 0; j < V; j += V < 4 ? 1 : 4) {
                if constexpr (V < 4) {
                    f[e] = live(e) ? p[row + at(e)] : 0.0f;
                } else {
                    float4_t v = {0, 0, 0, 0};
                    if (live(e)) v = *(const float4_t*)(p + row + at(e) + j);
#pragma unroll
                    for (int c = 0; c < 4; ++c) f[e * V + j + c] = v[c];
                }
            }
    }
    __device__ __forceinline__ void store_sums(float* p, long long row, const float (&f)[8]) const {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (live(e)) {
                if constexpr (V < 4) {
                    p[row + at(e)] = f[e];
                } else {
#pragma unroll
                    for (int j = 0; j < V; j += 4) {
                        const float* const v = f + e * V + j;
                        *(float4_t*)(p + row + at(e) + j) = float4_t{v[0], v[1], v[2], v[3]};
                    }
                }
            }
    }
    // a row of the table: its sum times the scale, added to what was there if asked for
    __device__ __forceinline__ void store_row(const EmbeddingDev& p, uint32_t key, float (&sum)[8], const float (&old)[8]) const {
        const long long row = (long long)key * d;
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] = p.accumulate ? fmaf(p.scale, sum[c], old[c]) : p.scale * sum[c];
        store_sums(p.dtable, row, sum);
    }
};
// Sorted places of a wavefront, how many such, of how many times 512 columns, in all; rows of the table that a wavefront looks for among the tokens.
struct RunPlan { int tile, tiles, chunks, units, rows; };

// The sums of the runs that begin and end in a tile of sorted places go to their rows; of a run that goes on behind the tile, or began in front of
// it, the tile leaves its part: [tile][0] where it began in front, [tile][1] where it begins here.  A wavefront takes 512 columns and has eight
// rows on their way.  Other wavefronts of the launch write zeros to rows of no token.  What bounds it: the table's writing (8192 tokens, 65536 rows
// of 4096: 1.14 GB in 220 us, 5.2 TB/s).  Clearing the whole table in front, 16 KiB a workgroup, takes 156 us, but leaves its last 256 MB to be
// written while the sums run: 251 us in all against 241.
template <int DT_, int V>
__global__ void __launch_bounds__(64) run_kernel(EmbeddingDev p, RunPlan plan) {
    const int lane = threadIdx.x, unit = blockIdx.x;
    if (unit >= plan.units) {
        const int first = (unit - plan.units) * plan.rows, row = first + lane;
        bool absent = false;
        if (lane < plan.rows && row < p.vocab) {
            const int at = below(p.keys, 0, p.n_tokens, (uint32_t)row, false);
            absent = at == p.n_tokens || p.keys[at] != (uint32_t)row;
        }
        const uint64_t which = p.accumulate ? 0 : __builtin_amdgcn_ballot_w64(absent);
        for (int r = 0; r < plan.rows; ++r) {
            if (!(which >> r & 1)) continue;
            float* const to = p.dtable + (size_t)(first + r) * p.d;
            if (p.d % 4 == 0)
                for (int c = 4 * lane; c < p.d; c += 256) *(float4_t*)(to + c) = float4_t{0, 0, 0, 0};
            else
                for (int c = lane; c < p.d; c += 64) to[c] = 0.0f;
        }
        return;
    }
    const int tile = unit / plan.chunks;
    const Columns<DT_, V> cols{(unit % plan.chunks) * 512 + V * lane, p.d};
    const int i0 = tile * plan.tile, i1 = min(i0 + plan.tile, p.n_tokens);
    const uint32_t none = (uint32_t)p.vocab;
    const uint32_t front = i0 > 0 ? p.keys[i0 - 1] : 0xFFFFFFFFu, behind = i1 < p.n_tokens ? p.keys[i1] : 0xFFFFFFFFu;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int i = i0; i < i1; i += 8) {
        float x[8][8], old[8][8];
        uint32_t key[9];
#pragma unroll
        for (int j = 0; j < 9; ++j) key[j] = i + j < i1 ? p.keys[i + j] : i + j == i1 ? behind : 0xFFFFFFFFu;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < i1 && key[j] < none) cols.load(x[j], p.out, p.order[i + j] * p.out_stride);
        if (p.accumulate)                                             // rows that end here: asked for before the first is needed
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i + j < i1 && key[j] < none && key[j] != key[j + 1] && key[j] != front) cols.load_sums(old[j], p.dtable, (long long)key[j] * p.d);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (i + j >= i1 || key[j] >= none) break;
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] += x[j][c];
            const bool last = i + j + 1 == i1;
            if (!last && key[j + 1] == key[j]) continue;
            const bool before = key[j] == front, after = last && behind == key[j];
            if (before || after) cols.store_sums(p.partial, ((long long)tile * 2 + !before) * p.d, sum);
            else cols.store_row(p, key[j], sum, old[j]);
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] = 0.0f;
        }
    }
}

// Runs over more than one tile, joined by the tile in which they begin: by one wavefront, or, of more than eight tiles, in four shares (4096
// tokens of which a third are alike, 64 columns: 40 -> 24 us for the whole gradient; 65536 of two kinds, 4096 columns 493 -> 412).
constexpr int JW = 4;                         // wavefronts that share a long run
template <int V>
__global__ void __launch_bounds__(64 * JW) join_kernel(EmbeddingDev p, RunPlan plan) {
    __shared__ float sums[JW - 1][512];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tile = blockIdx.x / plan.chunks;
    const Columns<DT_F32, V> cols{((int)blockIdx.x % plan.chunks) * 512 + V * lane, p.d};
    const int i0 = tile * plan.tile, i1 = i0 + plan.tile;
    if (i1 >= p.n_tokens) return;
    const uint32_t key = p.keys[i1 - 1], behind = p.keys[i1], front = p.keys[max(i0 - 1, 0)];      // asked for together
    if (key >= (uint32_t)p.vocab || behind != key || (i0 > 0 && front == key)) return;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, old[8];
    if (!wave) {
        cols.load_sums(sum, p.partial, ((long long)tile * 2 + 1) * p.d);
        if (p.accumulate) cols.load_sums(old, p.dtable, (long long)key * p.d);
    }
    int last = tile;                                             // the last tile that begins with the run
    for (bool on = true; on;) {
        const int next = last + 1 + lane;
        const uint64_t same = __builtin_amdgcn_ballot_w64(next < plan.tiles && p.keys[(long long)next * plan.tile] == key);
        on = same == ~0ull;
        last += on ? 64 : __builtin_ctzll(~same);
    }
    const bool shared = last - tile > 8;
    if (wave && !shared) return;
    const int share = shared ? (last - tile + JW - 1) / JW : last - tile, from = min(tile + share * wave, last), to = min(from + share, last);
#pragma unroll 8
    for (int t = from + 1; t <= to; ++t) {
        float x[8];
        cols.load_sums(x, p.partial, (long long)t * 2 * p.d);
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] += x[c];
    }
    if (shared) {
        if (wave)
#pragma unroll
            for (int c = 0; c < 8; ++c) sums[wave - 1][64 * c + lane] = sum[c];
        __syncthreads();
        if (wave) return;
        for (int w = 0; w < JW - 1; ++w)
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] += sums[w][64 * c + lane];
    }
    cols.store_row(p, key, sum, old);
}

// Few tokens, in one launch without sorting: a workgroup takes a token and 512 columns, looks for the token's others, leaves if one is in front of
// it, and sums the rows of all in the order of their places, shared out to its wavefronts where they are more than 8.  Other workgroups write zeros to
// rows of no token.  Every workgroup reads all tokens, but nothing waits for a launch in front: 777 tokens of 1023 columns 8.5 us instead of 18.5, 256
// of 1024 6.6 instead of 15; 1000 of two tokens, the longest runs, 22 instead of 21.  From 2048 workgroups on sorting is faster: 1000 of 4096 columns
// 20 us instead of 29.
constexpr int kFewRows = 16, FW = 8;
template <int DT_, int V>
__global__ void __launch_bounds__(64 * FW) few_kernel(EmbeddingDev p, RunPlan plan) {
    __shared__ uint64_t same[64];
    __shared__ int present[kFewRows];
    __shared__ float sums[FW - 1][512];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), unit = blockIdx.x;
    if (unit >= plan.units) {
        const long long apart = (long long)(gridDim.x - plan.units) * kFewRows;
        for (long long first = (long long)(unit - plan.units) * kFewRows; first < p.vocab; first += apart) {
            if (tid < kFewRows) present[tid] = 0;
            __syncthreads();
            for (int i = tid; i < p.n_tokens; i += 64 * FW) {
                const long long at = p.tokens[i] - first;
                if (at >= 0 && at < kFewRows) present[at] = 1;
            }
            __syncthreads();
            for (int r = 0; r < kFewRows && first + r < p.vocab; ++r) {
                if (present[r]) continue;
                float* const to = p.dtable + (size_t)(first + r) * p.d;
                if (p.d % 4 == 0)
                    for (int c = 4 * tid; c < p.d; c += 256 * FW) *(float4_t*)(to + c) = float4_t{0, 0, 0, 0};
                else
                    for (int c = tid; c < p.d; c += 64 * FW) to[c] = 0.0f;
            }
            __syncthreads();
        }
        return;
    }
    const int i = unit / plan.chunks, words = (p.n_tokens + 63) / 64;
    const uint32_t key = key_of(p, i);
    if (key >= (uint32_t)p.vocab) return;
    for (int w = wave; w < words; w += FW) {
        const int t = 64 * w + lane;
        const uint64_t m = __builtin_amdgcn_ballot_w64(t < p.n_tokens && p.tokens[t] == (int)key);
        if (lane == 0) same[w] = m;
    }
    __syncthreads();
    const uint64_t mine = lane < words ? same[lane] : 0;                        // those of the lane's 64 places
    const uint64_t earlier = lane < i / 64 ? mine : lane == i / 64 ? mine & ((1ull << (i & 63)) - 1) : 0;
    if (__builtin_amdgcn_ballot_w64(earlier != 0)) return;
    const uint64_t some = __builtin_amdgcn_ballot_w64(mine != 0);
    int count = __popcll(mine);
#pragma unroll
    for (int o = 1; o < 64; o *= 2) count += __shfl_xor(count, o);
    // the rows of the places in the words of `which`, eight on their way
    auto run = [&](const Columns<DT_, V>& cols, float (&sum)[8], uint64_t which) {
        uint64_t m = 0;
        int w = 0;
        for (;;) {
            int at[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (!m && which) {
                    w = __builtin_ctzll(which);
                    which &= which - 1;
                    m = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), w) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)mine, w);
                }
                at[j] = m ? 64 * w + __builtin_ctzll(m) : -1;
                m &= m - 1;
            }
            if (at[0] < 0) break;
            float x[8][8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at[j] >= 0) cols.load(x[j], p.out, at[j] * p.out_stride);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at[j] >= 0)
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum[c] += x[j][c];
        }
    };
    const Columns<DT_, V> cols{(unit % plan.chunks) * 512 + V * lane, p.d};
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, old[8];
    if (p.accumulate && !wave) cols.load_sums(old, p.dtable, (long long)key * p.d);
    if (count <= 8) {
        if (wave) return;
        run(cols, sum, some);
    } else {
        const int share = (words + FW - 1) / FW, from = min(share * wave, 63), to = min(share * (wave + 1), 63);
        run(cols, sum, some & ((1ull << to) - (1ull << from)));
        if (wave)
#pragma unroll
            for (int c = 0; c < 8; ++c) sums[wave - 1][64 * c + lane] = sum[c];
        __syncthreads();
        if (wave) return;
        for (int w = 0; w < FW - 1; ++w)
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] += sums[w][64 * c + lane];
    }
    cols.store_row(p, key, sum, old);
}

static size_t round16(size_t n) { return (n + 15) / 16 * 16; }
// Sorted places of a wavefront: 32, or fewer where that leaves less than 2048 wavefronts.
static RunPlan run_plan(int n_tokens, int d) {
    RunPlan r{};
    r.chunks = (d + 511) / 512;
    r.tile = 32;
    while (r.tile > 8 && (long long)((n_tokens + r.tile - 1) / r.tile) * r.chunks < 2048) r.tile /= 2;
    r.tiles = (n_tokens + r.tile - 1) / r.tile;
    r.units = r.tiles * r.chunks;
    return r;
}
static bool few(int n_tokens, int d) { return n_tokens <= 1024 && n_tokens * ((d + 511) / 512) <= 2048; }
size_t embedding_backward_workspace_bytes(int n_tokens, int d) {
    if (few(n_tokens, d)) return 16;                             // of which nothing is used
    const size_t list = round16(4 * (size_t)n_tokens);
    return (n_tokens > kSortTile ? 4 : 2) * list + (size_t)run_plan(n_tokens, d).tiles * 2 * d * 4;
}
// Rows of the table of a wavefront: 64 where that makes a thousand wavefronts (65536 rows of 4096: 244 us, with 16 rows 251), otherwise 16.
static int absent_rows(int vocab) { return vocab >= 65536 ? 64 : 16; }
// Both launches over runs, of which the first also clears rows of no token.
bool embedding_backward_fits(int n_tokens, int vocab, int d) {
    const double units = (double)((n_tokens + 31) / 32) * ((d + 511) / 512);       // where there are many
    const double most = std::max((units + vocab / absent_rows(vocab) + 8) * 64.0, units * (64 * JW));
    return most < 4294967296.0;
}
template <int DT_, int V>
static void sum_runs(const EmbeddingDev& p, const RunPlan& plan, hipStream_t s) {
    if (few(p.n_tokens, p.d)) {
        const unsigned absent = p.accumulate ? 0 : std::min((p.vocab - 1) / kFewRows + 1, 65536);
        hipLaunchKernelGGL((few_kernel<DT_, V>), dim3(plan.units + absent), dim3(64 * FW), 0, s, p, plan);
        return;
    }
    const unsigned absent = p.accumulate ? 0 : (unsigned)(p.vocab + plan.rows - 1) / plan.rows;
    hipLaunchKernelGGL((run_kernel<DT_, V>), dim3(plan.units + absent), dim3(64), 0, s, p, plan);
    if (plan.tiles > 1) hipLaunchKernelGGL(join_kernel<V == 8 ? 4 : V>, dim3((unsigned)plan.units), dim3(64 * JW), 0, s, p, plan);
}
// Keys and places in their order, and where sums of pieces go.
static void sort_tokens(EmbeddingDev& p, void* workspace, hipStream_t s) {
    char* at = (char*)workspace;
    const size_t list = round16(4 * (size_t)p.n_tokens);
    p.keys = (uint32_t*)at; at += list;
    p.order = (int*)at; at += list;
    p.tile_keys = p.keys; p.tile_order = p.order;
    if (p.n_tokens > kSortTile) {
        p.tile_keys = (uint32_t*)at; at += list;
        p.tile_order = (int*)at; at += list;
    }
    p.partial = (float*)at;
    hipLaunchKernelGGL(rank_kernel, dim3((unsigned)(p.n_tokens + kRankRows - 1) / kRankRows), dim3(1024), 0, s, p);
    if (p.n_tokens > kSortTile) hipLaunchKernelGGL(merge_kernel, dim3((p.n_tokens + 255) / 256), dim3(256), 0, s, p);
}
hipError_t launch_embedding_backward(EmbeddingDev p, int dt, void* workspace, hipStream_t s) {
    RunPlan plan{};
    if (few(p.n_tokens, p.d)) {
        plan.chunks = (p.d + 511) / 512; plan.units = p.n_tokens * plan.chunks;
    } else {
        sort_tokens(p, workspace, s);
        plan = run_plan(p.n_tokens, p.d);
        plan.rows = absent_rows(p.vocab);
    }
    const int unit = dt == DT_F32 ? 4 : 8;
    const bool whole = p.d % unit == 0 && p.out_stride % unit == 0;
    switch (dt) {
        case DT_F16: whole ? sum_runs<DT_F16, 8>(p, plan, s) : sum_runs<DT_F16, 1>(p, plan, s); break;
        case DT_BF16: whole ? sum_runs<DT_BF16, 8>(p, plan, s) : sum_runs<DT_BF16, 1>(p, plan, s); break;
        default: whole ? sum_runs<DT_F32, 4>(p, plan, s) : sum_runs<DT_F32, 1>(p, plan, s);
    }
    return hipGetLastError();
}

}  // namespace rwkvq
