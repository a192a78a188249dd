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
constexpr int kRunTile = 32;                  // sorted places of a wavefront of the sums
constexpr int kAbsentRows = 16;               // rows of the table that a wavefront looks for among the tokens

__device__ __forceinline__ uint32_t key_of(const EmbeddingDev& p, int i) {
    const int token = p.tokens[i];
    return token >= 0 && token < p.vocab ? (uint32_t)token : (uint32_t)p.vocab;     // tokens without a row come last
}

// The place of a token among those of its tile: how many are smaller, or equal and in front of it.  A workgroup takes 64 tokens, a lane each; its
// sixteen wavefronts compare them with a sixteenth of the tile each, whose keys are the same for all lanes.  Two vector
// instructions a pair: 8192 tokens are 2.1 million of them, 8000 cycles of the device.
__global__ void __launch_bounds__(1024) rank_kernel(EmbeddingDev p) {
    __shared__ int counts[16][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = blockIdx.x * 64 / kSortTile * kSortTile, end = min(tile + kSortTile, p.n_tokens), chunk = blockIdx.x * 64, mine = chunk + lane;
    const uint32_t key = mine < p.n_tokens ? key_of(p, mine) : 0xFFFFFFFFu;
    const int from = tile + wave * (kSortTile / 16), to = min(from + kSortTile / 16, end);
    int count = 0, i = from;
#pragma unroll 8
    for (; i < min(to, chunk); ++i) count += key_of(p, i) <= key;
    for (; i < min(to, chunk + 64); ++i) {
        const uint32_t other = key_of(p, i);
        count += other < key || (other == key && i < mine);
    }
#pragma unroll 8
    for (; i < to; ++i) count += key_of(p, i) < key;
    counts[wave][lane] = count;
    __syncthreads();
    if (wave == 0 && mine < p.n_tokens) {
#pragma unroll
        for (int w = 1; w < 16; ++w) count += counts[w][lane];
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

// The sums of the runs that begin and end in a tile of sorted places go to their rows; of a run that goes on behind the tile, or began in front of
// it, the tile leaves its part: [tile][0] where it began in front, [tile][1] where it begins here.  A wavefront takes 512 columns, eight of them a
// lane, and has eight rows on their way.  Other wavefronts of the launch write zeros to rows of no token.
template <int DT_>
__global__ void __launch_bounds__(64) run_kernel(EmbeddingDev p, int chunks, int tiles) {
    const int lane = threadIdx.x;
    if ((int)blockIdx.x >= chunks * tiles) {
        const int first = ((int)blockIdx.x - chunks * tiles) * kAbsentRows, row = first + lane;
        bool absent = false;
        if (lane < kAbsentRows && row < p.vocab) {
            const int at = below(p.keys, 0, p.n_tokens, (uint32_t)row, false);
            absent = at == p.n_tokens || p.keys[at] != (uint32_t)row;
        }
        const uint64_t which = __builtin_amdgcn_ballot_w64(absent);
        for (int r = 0; r < kAbsentRows; ++r) {
            if (!(which >> r & 1)) continue;
            float* const to = p.dtable + (size_t)(first + r) * p.d;
            if (p.d % 4 == 0)
                for (int c = 4 * lane; c < p.d; c += 256) *(float4_t*)(to + c) = float4_t{0, 0, 0, 0};
            else
                for (int c = lane; c < p.d; c += 64) to[c] = 0.0f;
        }
        return;
    }
    const int tile = blockIdx.x / chunks, col = (blockIdx.x % chunks) * 512 + 8 * lane, left = p.d - col;
    const int i0 = tile * kRunTile, i1 = min(i0 + kRunTile, p.n_tokens);
    const uint32_t none = (uint32_t)p.vocab;
    const uint32_t front = i0 > 0 ? p.keys[i0 - 1] : 0xFFFFFFFFu, behind = i1 < p.n_tokens ? p.keys[i1] : 0xFFFFFFFFu;
    const bool whole_table = p.d % 4 == 0;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int i = i0; i < i1; i += 8) {
        float x[8][8];
        uint32_t key[9];
#pragma unroll
        for (int j = 0; j < 9; ++j) key[j] = i + j < i1 ? p.keys[i + j] : i + j == i1 ? behind : 0xFFFFFFFFu;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (i + j < i1 && key[j] < none && left > 0) load8<DT_>(x[j], p.out, p.order[i + j] * p.out_stride + col, left, p.rows_whole);
            else
#pragma unroll
                for (int c = 0; c < 8; ++c) x[j][c] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (i + j >= i1 || key[j] >= none) break;
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] += x[j][c];
            const bool last = i + j + 1 == i1;
            if (!last && key[j + 1] == key[j]) continue;
            const bool before = key[j] == front, after = last && behind == key[j];
            if (before || after) {
                store8<DT_F32>(p.partial, ((long long)tile * 2 + !before) * p.d + col, sum, left, whole_table);
            } else if (left > 0) {
                const long long at = (long long)key[j] * p.d + col;
                float old[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (p.accumulate) load8<DT_F32>(old, p.dtable, at, left, whole_table);
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] = p.accumulate ? fmaf(p.scale, sum[c], old[c]) : p.scale * sum[c];
                store8<DT_F32>(p.dtable, at, sum, left, whole_table);
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] = 0.0f;
        }
    }
}

// Runs over more than one tile, joined by the tile in which they begin.
__global__ void __launch_bounds__(64) join_kernel(EmbeddingDev p, int chunks, int tiles) {
    const int tile = blockIdx.x / chunks, col = (blockIdx.x % chunks) * 512 + 8 * (int)threadIdx.x, left = p.d - col;
    const int i0 = tile * kRunTile, i1 = i0 + kRunTile;
    if (i1 >= p.n_tokens || left <= 0) return;
    const uint32_t key = p.keys[i1 - 1];
    if (key >= (uint32_t)p.vocab || p.keys[i1] != key || (i0 > 0 && p.keys[i0 - 1] == key)) return;
    const int end = i1 + below(p.keys, i1, p.n_tokens, key, true), last = (end - 1) / kRunTile;
    const bool whole = p.d % 4 == 0;
    float sum[8];
    load8<DT_F32>(sum, p.partial, ((long long)tile * 2 + 1) * p.d + col, left, whole);
#pragma unroll 8
    for (int t = tile + 1; t <= last; ++t) {
        float x[8];
        load8<DT_F32>(x, p.partial, (long long)t * 2 * p.d + col, left, whole);
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] += x[c];
    }
    const long long at = (long long)key * p.d + col;
    float old[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (p.accumulate) load8<DT_F32>(old, p.dtable, at, left, whole);
#pragma unroll
    for (int c = 0; c < 8; ++c) sum[c] = p.accumulate ? fmaf(p.scale, sum[c], old[c]) : p.scale * sum[c];
    store8<DT_F32>(p.dtable, at, sum, left, whole);
}

static size_t round16(size_t n) { return (n + 15) / 16 * 16; }
static int run_tiles(int n_tokens) { return (n_tokens + kRunTile - 1) / kRunTile; }
size_t embedding_backward_workspace_bytes(int n_tokens, int d) {
    const size_t list = round16(4 * (size_t)n_tokens);
    return (n_tokens > kSortTile ? 4 : 2) * list + (size_t)run_tiles(n_tokens) * 2 * d * 4;
}
bool embedding_backward_fits(int n_tokens, int vocab, int d) {
    const double chunks = (d + 511) / 512;
    return (chunks * run_tiles(n_tokens) + vocab / kAbsentRows + 1) * 64.0 < 4294967296.0;
}
hipError_t launch_embedding_backward(EmbeddingDev p, int dt, void* workspace, hipStream_t s) {
    p.rows_whole = p.out_stride % (dt == DT_F32 ? 4 : 8) == 0;
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
    hipLaunchKernelGGL(rank_kernel, dim3((p.n_tokens + 63) / 64), dim3(1024), 0, s, p);
    if (p.n_tokens > kSortTile) hipLaunchKernelGGL(merge_kernel, dim3((p.n_tokens + 255) / 256), dim3(256), 0, s, p);
    const int chunks = (p.d + 511) / 512, tiles = run_tiles(p.n_tokens);
    const dim3 grid((unsigned)(chunks * tiles + (p.accumulate ? 0 : (p.vocab + kAbsentRows - 1) / kAbsentRows))), block(64);
    switch (dt) {
        case DT_F16: hipLaunchKernelGGL(run_kernel<DT_F16>, grid, block, 0, s, p, chunks, tiles); break;
        case DT_BF16: hipLaunchKernelGGL(run_kernel<DT_BF16>, grid, block, 0, s, p, chunks, tiles); break;
        default: hipLaunchKernelGGL(run_kernel<DT_F32>, grid, block, 0, s, p, chunks, tiles);
    }
    if (tiles > 1) hipLaunchKernelGGL(join_kernel, dim3((unsigned)(chunks * tiles)), block, 0, s, p, chunks, tiles);
    return hipGetLastError();
}

}  // namespace rwkvq
