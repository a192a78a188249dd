// Low-rank adapters beside frozen matrices (include/rwkvq.h), y_t = base_t + s_a B_a h_t with h_t = A_a drop(x_t), and their gradients:
//   g_t = s_a B_a^T dy_t,   dx_t = base_t + drop(A_a^T g_t),   dA_a = sum_t g_t drop(x_t)^T,   dB_a = s_a sum_t dy_t h_t^T.
#include "adapter_plan.h"
#include "dropout.h"
#include "matrix_core.h"
#include "pieces.h"

#include <type_traits>

namespace rwkvq {

// Arguments of a launch lie in host memory or behind a cold cache: what a workgroup needs is in four lines of 64 bytes, read together.
struct alignas(128) AdapterLine { AdapterMatDev m; };
struct alignas(128) AdapterCall {
    AdapterRowsDev rows;
    int y_dt, slice, pieces;                       // columns of a workgroup; tiles, of which the grid may have more
    uint32_t first;                                // number of the first matrix
    bool backward;                                 // x = dy, y = dx, h = g, p = b turned, q = a turned
    AdapterLine mats[kAdapterMats];
};
struct OuterMatDev {
    const uint16_t *x, *dy;
    const uint16_t *g, *h;                         // in three parts, [token][part][padded rank]
    float *da, *db;
    long long x_stride, dy_stride;
    size_t at;                                     // of its sums among those of a piece
    int N, K, chunks;
};
struct OuterCall {
    AdapterRowsDev rows;
    OuterMatDev mats[kAdapterMats];
    int* owner;                                    // adapter of each piece, -1: none
    float* partial;                                // [piece][matrix][rank K | N rank]
    size_t size;                                   // floats of a piece
    int n_mats, chunks, cut, slots;
    uint32_t first;
};
struct TurnCall {
    AdapterRowsDev rows;
    const uint16_t* from[2 * kAdapterMats];
    uint16_t* to[2 * kAdapterMats];
    int height[2 * kAdapterMats], width[2 * kAdapterMats];
    const float* h[kAdapterMats];
    uint16_t* h_parts[kAdapterMats];
    int n_mats;
};

// Rows of sequence b, within 0 .. n_tokens whatever the offsets hold.
__device__ __forceinline__ void rows_of(const AdapterRowsDev& r, int b, int& t0, int& t1) {
    if (r.offsets) {
        t0 = min(max(r.offsets[b], 0), r.n_tokens);
        t1 = min(max(r.offsets[b + 1], t0), r.n_tokens);
    } else {
        const int len = r.n_tokens / r.n_seqs;
        t0 = b * len; t1 = t0 + len;
    }
}
// Adapter of sequence b, -1 if it has none.
__device__ __forceinline__ int adapter_of(const AdapterRowsDev& r, int b) {
    const int a = r.adapters ? r.adapters[b] : 0;
    return a >= 0 && a < r.n_adapters ? a : -1;
}
// Piece number `slot` of a call: up to `cut` rows of one sequence, its adapter and the adapter's scale.  With offsets sequence b has the numbers from
// offsets[b] / cut + b on, one more than it needs at times: then t0 >= t1.  Every thread of the workgroup calls it; the one that finds the sequence
// reads what else there is to know, for all.
struct RowSpan { int t0, t1, id; float scale; };
__device__ __forceinline__ RowSpan span_of_sequence(const AdapterRowsDev& r, int cut, int b, int idx, int t0, int t1) {
    RowSpan s;
    s.t0 = min(t0 + idx * cut, t1);                // idx cut <= n_tokens
    s.t1 = min(s.t0 + cut, t1);
    s.id = s.t0 < s.t1 ? adapter_of(r, b) : -1;
    s.scale = s.id >= 0 && r.scales ? r.scales[s.id] : 1.0f;
    return s;
}
__device__ __forceinline__ RowSpan piece_of(const AdapterRowsDev& r, int cut, int slot, RowSpan* found) {
    if (!r.offsets) {
        const int per = (r.n_tokens / r.n_seqs + cut - 1) / cut, b = slot / per;
        int t0, t1;
        rows_of(r, b, t0, t1);
        return span_of_sequence(r, cut, b, slot - b * per, t0, t1);
    }
    if (threadIdx.x == 0) *found = RowSpan{0, 0, -1, 1.0f};
    __syncthreads();
    for (int b = threadIdx.x; b < r.n_seqs; b += blockDim.x) {
        int t0, t1;
        rows_of(r, b, t0, t1);
        const int first = t0 / cut + b;
        if (slot >= first && slot <= t1 / cut + b) *found = span_of_sequence(r, cut, b, slot - first, t0, t1);
    }
    __syncthreads();
    RowSpan s;
    s.t0 = __builtin_amdgcn_readfirstlane(found->t0);
    s.t1 = __builtin_amdgcn_readfirstlane(found->t1);
    s.id = __builtin_amdgcn_readfirstlane(found->id);
    s.scale = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(found->scale)));
    return s;
}
// Single tokens: the rows of a tile are up to sixteen of one adapter, wherever they are, so that its weights are read once for all of them.  With fewer
// adapters than rows workgroup i takes the i-th sixteen of all adapters', counted in LDS, and the grid is as large as these can be; otherwise, and for up
// to sixteen rows, that of row b has work if an even sixteen of the rows in front of it have the same adapter.  That costs 1 us less, but workgroups without
// work come and go, and the others meet on few dies: four matrices at rank 16, 128 rows of 8 adapters 14 us instead of 40, 2048 of 100 87 instead of 164.
struct Gathered {
    uint64_t same[kGathered / 64];
    int rows[16], totals[8], id, skip;
};
constexpr int kGatherScratch = 8 * kGathered + 16;
__device__ __forceinline__ int gather_rows(const AdapterRowsDev& r, int group, char* scratch, Gathered& at, int& id) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = r.n_seqs, masks = (n + 63) / 64;
    const bool counted = groups_of(r) < n;
    int* const ids = (int*)scratch;
    int* const counts = ids + kGathered;                                      // of none, then of the adapters
    for (int t = tid; t < n; t += 512) ids[t] = adapter_of(r, t);
    if (counted)
        for (int i = tid; i <= r.n_adapters; i += 512) counts[i] = 0;
    __syncthreads();
    if (counted) {
        for (int t = tid; t < n; t += 512) atomicAdd(&counts[ids[t] + 1], 1);
        __syncthreads();
        const int per = r.n_adapters / 512 + 1, first = tid * per;
        int own = 0;
        for (int i = first; i < min(first + per, r.n_adapters + 1); ++i) own += (counts[i] + 15) / 16;
        int sum = own;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int v = __shfl_up(sum, o, 64);
            if (lane >= o) sum += v;
        }
        if (lane == 63) at.totals[wave] = sum;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const int v = at.totals[w];
            before += w < wave ? v : 0;
            all += v;
        }
        if (group >= all) return 0;
        int left = group - (before + sum - own);
        if (left >= 0 && left < own)
            for (int i = first;; ++i) {
                const int here = (counts[i] + 15) / 16;
                if (left < here) {
                    at.id = i - 1; at.skip = 16 * left;
                    break;
                }
                left -= here;
            }
        __syncthreads();
        id = at.id;
    } else {
        id = ids[group];
    }
    for (int i = wave; i < masks; i += 8) {
        const int other = 64 * i + lane;
        const uint64_t m = __builtin_amdgcn_ballot_w64(other < n && ids[min(other, n - 1)] == id);
        if (lane == 0) at.same[i] = m;
    }
    __syncthreads();
    int all = 0, skip = 0;
    for (int i = 0; i < masks; ++i) {
        const uint64_t m = at.same[i];
        const int low = group - 64 * i;
        if (!counted) skip += low >= 64 ? __builtin_popcountll(m) : low <= 0 ? 0 : __builtin_popcountll(m & ((1ull << low) - 1));
        all += __builtin_popcountll(m);
    }
    if (counted) skip = at.skip;
    else if (skip % 16) return 0;
    for (int i = wave; i < masks; i += 8) {
        const uint64_t m = at.same[i];
        int rank = __builtin_popcountll(m & ((1ull << lane) - 1)) - skip;
        for (int j = 0; j < i; ++j) rank += __builtin_popcountll(at.same[j]);
        if ((m >> lane & 1) && rank >= 0 && rank < 16) at.rows[rank] = 64 * i + lane;
    }
    __syncthreads();
    return min(all - skip, 16);
}

// Copies of 16 bytes a lane from memory to LDS by the load unit, to `to` + 16 lane.
__device__ __forceinline__ void copy_to_lds(const void* from, char* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// A barrier for what went through LDS: copies and loads may stay on their way.
__device__ __forceinline__ void meet() {
    wait_lds();
    RWKVQ_BARRIER();
}
// Tiles in LDS have rows of C pieces of 16 bytes; piece c of a row lies at place c ^ swizzle(row), so that the sixteen rows of an operand, whose
// lanes read the same piece, are in different banks.
template <int C>
__device__ __forceinline__ int swizzle(int row) { return (row / (16 / C)) & (C - 1); }

// Both products of a tile of up to 16 MT rows of one adapter: first h = P x^T (P: rank rows of `depth` values), then y = base + Q h (Q: `wide` rows of
// rank values).  The wavefronts share out the depth of the first, sums meet in LDS, and the columns of the second.  A workgroup takes
// `slice` columns of y and computes h for itself: where few tiles leave most of the device without work, h is cheaper taken several times than
// passed on through memory and another launch.
// What bounds it is what goes through a compute unit's cache: sixteen lanes that load 16 bytes of a row each, as the operands want them, get a third of what
// whole lines give (9.5 against 30 TB/s out of L2).  So tiles of x, P and Q are copied to LDS by whole lines, and y leaves through LDS.
// h goes into the second product as PARTS parts of 16 bits (two: 16 bits of bf16, 22 of fp16, beside the rounding of a 16-bit y; three for binary32 y), fp16
// ones under a power of two for each row that brings its largest value to 2^14, so that none is lost below fp16's range.
// Measured: 8192 rows, K = N = 4096, rank 64 with dropout 58 us (floor 40: 3.5 TB/s of x, base and y, beside 1 MB of P and Q for every 32 rows through a unit's
// cache), 4321 rows of 4096 beside 14336 columns at rank 32 78 (floor 57), 256 single tokens of 64 adapters, four matrices at rank 16, 25 (floor 18).
// GATHER: single tokens (gather_rows).  DROP: there is dropout, of x or, backwards, of what is added to y.
template <int RT, int MT, int PARTS> struct AdapterLds {
    static constexpr int W = kAdapterWaves, R = 16 * RT, ROWS = 16 * MT, PITCH = R + 4;
    static constexpr int STEPS = (PARTS * R + 31) / 32, HROW = 64 * STEPS + 16;                      // bytes of a row of h's parts
    static constexpr int CG = wave_cols(RT, MT), YPITCH = CG + 4;                                     // columns of a wavefront at a time
    static constexpr int CS = RT <= 2 || MT == 2 ? 64 : 32, D = RT == 1 ? 2 : 1;                      // columns of a step, steps on their way
    static constexpr int step = 2 * CS * (ROWS + R), ring = W * D * step;
    static constexpr int sums = W / 2 * ROWS * PITCH * 4, out = 16 * YPITCH * 4;                      // out: of a wavefront
    static constexpr int q = sums > W * out ? sums : W * out, q_tile = CG * R * 2;                    // sums and out share a place
    static constexpr int parts = q + W * q_tile, inverse = parts + ROWS * HROW, after = inverse + 4 * ROWS;
    static constexpr int found = ring > after ? ring : after, gathered = found + 16, bytes = gathered + (int)sizeof(Gathered);
};
// Wavefronts a SIMD: those of two workgroups where LDS and, for tiles of 32 rows with binary32 y or masks, registers allow.
template <int RT, int MT, int PARTS, bool DROP>
constexpr int waves_of() { return AdapterLds<RT, MT, PARTS>::bytes <= 80 * 1024 && !(MT == 2 && (PARTS == 3 || DROP)) ? 4 : 2; }
template <bool BF16, int RT, int MT, int PARTS, bool DROP, bool GATHER>
__global__ void __launch_bounds__(512, (waves_of<RT, MT, PARTS, DROP>())) adapter_kernel(AdapterCall p) {
    typedef AdapterLds<RT, MT, PARTS> L;
    constexpr int W = L::W, R = L::R, ROWS = L::ROWS, D = L::D, CS = L::CS, CG = L::CG, CT = CG / 16, QS = RT == 1 ? 1 : RT / 2, QC = R / 8;
    constexpr bool WIDE = PARTS == 3;                                         // y is binary32
    constexpr int PER = CG / 8, PASS = PER / 4;                               // lanes of a row of y, rounds for sixteen rows
    extern __shared__ __align__(16) char lds[];
    const AdapterRowsDev r = p.rows;
    const AdapterMatDev m = p.mats[blockIdx.z].m;
    asm volatile("" ::"s"(r.adapters), "s"(m.x), "s"(m.y_stride), "s"(m.wide), "s"(p.slice));
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    if ((int)blockIdx.x >= p.pieces) return;
    Gathered& gathered = *(Gathered*)(lds + L::gathered);
    int count, t0, id;
    float scale = 1.0f;
    if constexpr (GATHER) {
        static_assert(L::ring >= kGatherScratch, "the steps' place");
        t0 = 0;
        count = gather_rows(r, blockIdx.x, lds, gathered, id);
        if (id >= 0 && r.scales) scale = r.scales[id];
    } else {
        const RowSpan s = piece_of(r, ROWS, blockIdx.x, (RowSpan*)(lds + L::found));
        t0 = s.t0; count = s.t1 - s.t0; id = s.id; scale = s.scale;
    }
    if (count <= 0) return;
    auto row_at = [&](int i) -> long long { return GATHER ? gathered.rows[min(i, count - 1)] : t0 + min(i, count - 1); };
    const float before = p.backward ? scale : r.drop.factor, behind = p.backward ? r.drop.factor : scale;
    Dropout drop = r.drop;
    drop.call += blockIdx.z + p.first;
    const Keeper keeper = DROP ? Keeper(drop) : Keeper();

    // y: a wavefront takes CG columns at a time; lane l has 8 of them, PER lanes a row
    const int from = blockIdx.y * p.slice, to = min(from + p.slice, m.wide), out_col = 8 * (lane % PER), out_at = lane / PER;
    long long out_row[MT][PASS];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < PASS; ++j) out_row[i][j] = row_at(16 * i + 64 / PER * j + out_at);
    typedef uint4_t Base[MT][PASS][WIDE ? 2 : 1];
    Base base;
    auto fetch_base = [&](int c0) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < PASS; ++j)
#pragma unroll
                for (int e = 0; e < (WIDE ? 2 : 1); ++e) {
                    base[i][j][e] = uint4_t{0, 0, 0, 0};
                    if (m.base && c0 + out_col < to)
                        base[i][j][e] = *(const uint4_t*)((const char*)m.base + (out_row[i][j] * m.base_stride + c0 + out_col) * (WIDE ? 4 : 2) + 16 * e);
                }
    };
    // rows of Q for CG columns; those behind the rank or the last column repeat others
    char* const q_tile = lds + L::q + wave * L::q_tile;
    auto fetch_q = [&](int c0) {
        if (id < 0 || c0 >= to) return;
        const uint16_t* const Q = m.q + (size_t)id * r.rank * m.wide;
#pragma unroll
        for (int i = 0; i < CG * QC / 64; ++i) {
            const int at = 64 * i + lane, col = at / QC, c = (at % QC) ^ swizzle<QC>(col);
            copy_to_lds(Q + (size_t)min(c0 + col, m.wide - 1) * r.rank + (8 * c < r.rank ? 8 * c : 0), q_tile + 1024 * i);
        }
    };

    if (id >= 0) {
        float4_t acc[MT][RT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < RT; ++j) acc[i][j] = float4_t{0, 0, 0, 0};
        // CS columns of x and P, 1 KiB of whole or half lines a copy.  Columns behind the depth repeat the last ones, rows of P behind the rank others
        constexpr int C = CS / 8, PER_COPY = 64 / C, XC = ROWS / PER_COPY, PC = R / PER_COPY;
        const uint16_t* const P = m.p + (size_t)id * r.rank * m.depth;
        const uint16_t* x[XC];
#pragma unroll
        for (int i = 0; i < XC; ++i) x[i] = m.x + row_at(PER_COPY * i + lane / C) * m.x_stride;
        char* const ring = lds + wave * D * L::step;
        // 32 columns number h of a step.  Of ranks up to 32 a wavefront has 64 that lie together; above, halves of lines, whose other halves its
        // neighbour reads at the same time, in one order whatever a step has of them: tiles of either size have the same sums
        auto first = [&](int st, int h) { return RT <= 2 ? 64 * (wave + W * st) + 32 * h : 32 * (wave + W * (CS / 32 * st + h)); };
        auto fetch = [&](int st) {
            char* const at = ring + st % D * L::step;
            auto column = [&](int i) {
                const int c = lane % C ^ swizzle<C>(PER_COPY * i + lane / C);
                return min(first(st, c >> 2) + 8 * (c & 3), m.depth - 8);
            };
#pragma unroll
            for (int i = 0; i < XC; ++i) copy_to_lds(x[i] + column(i), at + 1024 * i);
#pragma unroll
            for (int i = 0; i < PC; ++i)
                copy_to_lds(P + (size_t)min(PER_COPY * i + lane / C, r.rank - 1) * m.depth + column(i), at + 1024 * (XC + i));
        };
        constexpr int BLOCK = RT <= 2 ? 64 : 32;
        const int blocks = (m.depth - BLOCK * wave + BLOCK * W - 1) / (BLOCK * W), steps = (blocks * BLOCK + CS - 1) / CS;     // of this wavefront
#pragma unroll
        for (int st = 0; st < D; ++st)
            if (st < steps) fetch(st);
        for (int st = 0; st < steps; ++st) {
            const char* const at = ring + st % D * L::step;
            uint4_t xf[CS / 32][MT], pf[CS / 32][RT];
            int k0[CS / 32];
#pragma unroll
            for (int h = 0; h < CS / 32; ++h) k0[h] = first(st, h) + 8 * g;
            uint4_t keep[CS / 32][MT];                                       // while the copies are on their way
            if (DROP && !p.backward)
#pragma unroll
                for (int h = 0; h < CS / 32; ++h)
#pragma unroll
                    for (int i = 0; i < MT; ++i) keep[h][i] = keeper.masks((uint32_t)k0[h] >> 3, (uint32_t)row_at(16 * i + n));
            if (st + D <= steps) wait_copies<(XC + PC) * (D - 1)>();         // all but those of the D - 1 steps behind this one
            else wait_copies<0>();
#pragma unroll
            for (int h = 0; h < CS / 32; ++h) {
                const int place = ((4 * h + g) ^ swizzle<C>(n)) << 4;
#pragma unroll
                for (int i = 0; i < MT; ++i) xf[h][i] = *(const uint4_t*)(at + (16 * i + n) * 2 * CS + place);
#pragma unroll
                for (int j = 0; j < RT; ++j) pf[h][j] = *(const uint4_t*)(at + (16 * (MT + j) + n) * 2 * CS + place);
            }
            wait_lds();
            if (st + D < steps) fetch(st + D);
#pragma unroll
            for (int h = 0; h < CS / 32; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (k0[h] >= m.depth) xf[h][i] = uint4_t{0, 0, 0, 0};
                    if (DROP && !p.backward) xf[h][i] &= keep[h][i];
                }
#pragma unroll
            for (int h = 0; h < CS / 32; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < RT; ++j) acc[i][j] = mfma_bits<BF16>(pf[h][j], xf[h][i], acc[i][j]);
        }
        wait_copies<0>();
        meet();                                                              // nobody reads or copies into the steps any more
        fetch_q(from + CG * wave);
        fetch_base(from + CG * wave);
        // lane (n, g): row n, values 4 g .. + 3 of a tile
        auto place = [&](int w, int i, int j) { return (float4_t*)(lds + 4 * ((w * ROWS + 16 * i + n) * L::PITCH + 16 * j + 4 * g)); };
        if (wave >= W / 2)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < RT; ++j) *place(wave - W / 2, i, j) = acc[i][j];
        meet();
        if (wave < W / 2)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < RT; ++j) *place(wave, i, j) += acc[i][j];
        meet();
    } else {
        fetch_base(from + CG * wave);
    }
    // sixteen threads a row
    char* const parts = lds + L::parts;
    float* const inverse = (float*)(lds + L::inverse);
    if (tid < 16 * ROWS) {
        const int q = tid & 15, at = tid >> 4;
        float4_t h[(RT + 3) / 4];
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < (RT + 3) / 4; ++i) {
            const int c = 4 * q + 64 * i;
            h[i] = float4_t{0, 0, 0, 0};
            if (id >= 0 && c < r.rank) {
#pragma unroll
                for (int w = 0; w < W / 2; ++w) h[i] += *(const float4_t*)(lds + 4 * ((w * ROWS + at) * L::PITCH + c));
#pragma unroll
                for (int j = 0; j < 4; ++j) h[i][j] *= before;
            }
            if (m.h && blockIdx.y == 0 && at < count) {
                if (!p.backward) {
                    if (c < r.rank) *(float4_t*)(m.h + row_at(at) * r.rank + c) = h[i];
                } else if (c < R) {                                          // g, only read by the sums over tokens
                    uint2_t w[3];
                    split4<3>(h[i], w);
#pragma unroll
                    for (int o = 0; o < 3; ++o) *(uint2_t*)((uint16_t*)m.h + (row_at(at) * 3 + o) * R + c) = w[o];
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                h[i][j] *= behind;
                most = fmaxf(most, fabsf(h[i][j]));
            }
        }
        if (!BF16) {
#pragma unroll
            for (int off = 8; off; off >>= 1) most = fmaxf(most, __shfl_xor(most, off, 64));
            const int e = (int)(__float_as_uint(most) >> 23) - 127, up = min(14 - e, 126);
            if (q == 0) inverse[at] = ldexpf(1.0f, -up);
#pragma unroll
            for (int i = 0; i < (RT + 3) / 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) h[i][j] = ldexpf(h[i][j], up);
        }
#pragma unroll
        for (int i = 0; i < (RT + 3) / 4; ++i) {
            const int c = 4 * q + 64 * i;
            if (c < R) {
                float4_t rest = h[i];
#pragma unroll
                for (int o = 0; o < PARTS; ++o) {
                    const uint2_t w = {Elem<BF16>::pack(rest[0], rest[1]), Elem<BF16>::pack(rest[2], rest[3])};
                    *(uint2_t*)(parts + at * L::HROW + 2 * (o * R + c)) = w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) rest[j] -= widen16<BF16>((uint16_t)(w[j / 2] >> (16 * (j & 1))));
                }
                if (RT == 1 && PARTS == 3) *(uint2_t*)(parts + at * L::HROW + 2 * (3 * R + c)) = uint2_t{0, 0};
            }
        }
    }
    uint4_t keep[MT][PASS];                                                   // of the next columns
    auto draw = [&](int c0) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < PASS; ++j) {
                keep[i][j] = uint4_t{~0u, ~0u, ~0u, ~0u};
                if (p.backward) keep[i][j] = keeper.masks((uint32_t)(c0 + out_col) >> 3, (uint32_t)out_row[i][j]);
            }
    };
    if (DROP) draw(from + CG * wave);
    meet();
    wait_copies<0>();

    char* const out_tile = lds + wave * L::out;
    for (int c0 = from + CG * wave; c0 < to; c0 += CG * W) {
        const bool more = c0 + CG * W < to;
        float4_t acc[MT][CT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < CT; ++j) acc[i][j] = float4_t{0, 0, 0, 0};
        if (id >= 0) {
            uint4_t qf[CT][QS];
#pragma unroll
            for (int j = 0; j < CT; ++j)
#pragma unroll
                for (int k = 0; k < QS; ++k)
                    qf[j][k] = *(const uint4_t*)(q_tile + (16 * j + n) * 2 * R + (((RT == 1 ? g & 1 : 4 * k + g) ^ swizzle<QC>(16 * j + n)) << 4));
            wait_lds();
            if (more) fetch_q(c0 + CG * W);
#pragma unroll
            for (int st = 0; st < L::STEPS; ++st)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const uint4_t hf = *(const uint4_t*)(parts + (16 * i + n) * L::HROW + 64 * st + 16 * g);
#pragma unroll
                    for (int j = 0; j < CT; ++j) acc[i][j] = mfma_bits<BF16>(qf[j][st % QS], hf, acc[i][j]);
                }
        }
        uint4_t out[MT][PASS][WIDE ? 2 : 1];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            // lane (n, g) holds columns 4 g .. + 3 of each tile of row n; row by row it goes out
            if (id >= 0) {
#pragma unroll
                for (int j = 0; j < CT; ++j) *(float4_t*)(out_tile + 4 * (n * L::YPITCH + 16 * j + 4 * g)) = acc[i][j];
            }
#pragma unroll
            for (int j = 0; j < PASS; ++j) {
                const int at = 64 / PER * j + out_at;
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (WIDE) {
                        y[e] = __uint_as_float(base[i][j][WIDE ? e / 4 : 0][e & 3]);
                    } else {
                        const uint16_t v = (uint16_t)(base[i][j][0][e / 2] >> (16 * (e & 1)));
                        y[e] = p.y_dt == DT_BF16 ? bf16_bits_to_f32(v) : f16_bits_to_f32(v);
                    }
                }
                if (id >= 0) {
                    const float down = BF16 ? 1.0f : inverse[16 * i + at];
                    const char* const from = out_tile + 4 * (at * L::YPITCH + out_col);
                    const float4_t a = *(const float4_t*)from, b = *(const float4_t*)(from + 16);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float z = e < 4 ? a[e & 3] : b[e & 3];
                        if (DROP) z = masked(z, keep[i][j], e);
                        y[e] = BF16 ? y[e] + z : fmaf(z, down, y[e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (WIDE) {
                        out[i][j][0][e] = __float_as_uint(y[e]);
                        out[i][j][WIDE ? 1 : 0][e] = __float_as_uint(y[4 + e]);
                    } else {
                        out[i][j][0][e] = p.y_dt == DT_BF16 ? Elem<true>::pack(y[2 * e], y[2 * e + 1]) : Elem<false>::pack(y[2 * e], y[2 * e + 1]);
                    }
                }
            }
        }
        // memory answers in order: the next rows of Q have to be there, then the next base is asked for, and the stores come last
        if (DROP && more) draw(c0 + CG * W);
        wait_copies<0>();
        if (more) fetch_base(c0 + CG * W);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < PASS; ++j)
#pragma unroll
                for (int e = 0; e < (WIDE ? 2 : 1); ++e)
                    if (16 * i + 64 / PER * j + out_at < count && c0 + out_col < to)
                        *(uint4_t*)((char*)m.y + (out_row[i][j] * m.y_stride + c0 + out_col) * (WIDE ? 4 : 2) + 16 * e) = out[i][j][e];
    }
}

template <bool BF16, int RT, int MT, int PARTS, bool DROP, bool GATHER>
static hipError_t start(const AdapterCall& p, dim3 grid, hipStream_t s) {
    static std::atomic<unsigned long long> raised{0};
    constexpr int bytes = AdapterLds<RT, MT, PARTS>::bytes;
    static_assert(bytes <= 160 * 1024, "a unit's LDS");
    const hipError_t e = raise_lds((const void*)adapter_kernel<BF16, RT, MT, PARTS, DROP, GATHER>, bytes, raised);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((adapter_kernel<BF16, RT, MT, PARTS, DROP, GATHER>), grid, dim3(512), bytes, s, p);
    return hipGetLastError();
}
template <bool BF16, int RT, int MT, int PARTS>
static hipError_t products(const AdapterCall& p, bool gather, dim3 grid, hipStream_t s) {
    if (p.rows.drop.seed) return start<BF16, RT, MT, PARTS, true, false>(p, grid, s);
    if (MT == 1 && gather) return start<BF16, RT, 1, PARTS, false, true>(p, grid, s);
    return start<BF16, RT, MT, PARTS, false, false>(p, grid, s);
}
template <bool BF16, int RT>
static hipError_t products(const AdapterCall& p, int rows, bool gather, dim3 grid, hipStream_t s) {
    const bool wide = p.y_dt == DT_F32;
    if constexpr (RT == 2 || RT == 4)
        if (rows == 32) return wide ? products<BF16, RT, 2, 3>(p, gather, grid, s) : products<BF16, RT, 2, 2>(p, gather, grid, s);
    return wide ? products<BF16, RT, 1, 3>(p, gather, grid, s) : products<BF16, RT, 1, 2>(p, gather, grid, s);
}
template <bool BF16>
static hipError_t products(const AdapterCall& p, int rows, bool gather, dim3 grid, hipStream_t s) {
    const int rank = p.rows.rank;
    return rank <= 16   ? products<BF16, 1>(p, rows, gather, grid, s)
           : rank <= 32 ? products<BF16, 2>(p, rows, gather, grid, s)
           : rank <= 64 ? products<BF16, 4>(p, rows, gather, grid, s)
                        : products<BF16, 8>(p, rows, gather, grid, s);
}
// (more than one slice only of fewer than 256 workgroups)
bool adapters_fit(const AdapterRowsDev& r) { return (double)pieces(r, 16) * kAdapterMats * 512.0 < 4294967296.0; }
static hipError_t launch_products(AdapterCall& p, int n_mats, int dt, hipStream_t s) {
    int widest = 64, deepest = 0;                     // also where no y is asked for
    double wide = 0;
    for (int i = 0; i < n_mats; ++i) {
        const AdapterMatDev& m = p.mats[i].m;
        widest = std::max(widest, m.wide); deepest = std::max(deepest, m.depth);
        wide += m.wide;
    }
    const int rows = tile_rows(p.rows, n_mats, wide);
    p.slice = slice_of(p.rows, rows, n_mats, widest, deepest, p.y_dt == DT_F32);
    const unsigned slices = (unsigned)((widest + p.slice - 1) / p.slice);
    p.pieces = single_tokens(p.rows) ? groups_of(p.rows) : (int)pieces(p.rows, rows);
    const dim3 grid((unsigned)(slices > 1 && spread(p.pieces) ? (p.pieces + 7) / 8 * 8 : p.pieces), slices, (unsigned)n_mats);
    return dt == DT_BF16 ? products<true>(p, rows, single_tokens(p.rows), grid, s) : products<false>(p, rows, single_tokens(p.rows), grid, s);
}

hipError_t launch_adapters(const AdapterRowsDev& rows, const AdapterMatDev* mats, int n_mats, int dt, int y_dt, hipStream_t s) {
    for (int i = 0; i < n_mats; i += kAdapterMats) {
        AdapterCall p{};
        p.rows = rows; p.y_dt = y_dt; p.first = (uint32_t)i;
        const int n = std::min(kAdapterMats, n_mats - i);
        for (int j = 0; j < n; ++j) p.mats[j].m = mats[i + j];
        const hipError_t e = launch_products(p, n, dt, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- gradients ----------------------------------------------------------------------------------------------------------

// Weights [rows][cols] of each adapter that a sequence has, as [cols][rows], 64 x 64 of them a workgroup through LDS, so that the backward pass is the kernel
// of the forward one; and h in three bf16 parts, once for all workgroups that read it.  A launch in a chain: 4 us for three adapters of rank 8, 5 for 8192
// rows at rank 64.
__global__ void __launch_bounds__(256) turn_kernel(TurnCall p) {
    __shared__ uint16_t tile[64][66];
    __shared__ int used;
    const AdapterRowsDev& r = p.rows;
    if ((int)blockIdx.z >= 2 * p.n_mats) {                                   // h in three parts
        const int mat = blockIdx.z - 2 * p.n_mats, R = padded_rank(r.rank), step = gridDim.x * gridDim.y * 256;
        for (long long i = (blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x; i < (long long)r.n_tokens * (R / 4); i += step) {
            const long long t = i / (R / 4);
            const int c = 4 * (int)(i % (R / 4));
            float4_t v = {0, 0, 0, 0};
            if (c < r.rank) v = *(const float4_t*)(p.h[mat] + t * r.rank + c);
            uint2_t w[3];
            split4<3>(v, w);
#pragma unroll
            for (int o = 0; o < 3; ++o) *(uint2_t*)(p.h_parts[mat] + (t * 3 + o) * R + c) = w[o];
        }
        return;
    }
    const int rows = p.height[blockIdx.z], cols = p.width[blockIdx.z], id = blockIdx.y, across = (cols + 63) / 64;
    const int r0 = ((int)blockIdx.x / across) * 64, c0 = ((int)blockIdx.x % across) * 64;
    if (r0 >= rows) return;
    if (r.adapters) {
        if (threadIdx.x == 0) used = 0;
        __syncthreads();
        for (int b = threadIdx.x; b < r.n_seqs; b += 256)
            if (r.adapters[b] == id) used = 1;
        __syncthreads();
        if (!used) return;
    } else if (id != 0) {
        return;
    }
    const uint16_t* const from = p.from[blockIdx.z] + (size_t)id * rows * cols;
    uint16_t* const to = p.to[blockIdx.z] + (size_t)id * rows * cols;
    // rows and cols are multiples of 8
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int y = (threadIdx.x >> 3) + 32 * i, x = 8 * (threadIdx.x & 7);
        uint4_t v = {0, 0, 0, 0};
        if (r0 + y < rows && c0 + x < cols) v = *(const uint4_t*)(from + (size_t)(r0 + y) * cols + c0 + x);
#pragma unroll
        for (int j = 0; j < 4; ++j) *(uint32_t*)&tile[y][x + 2 * j] = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int y = (threadIdx.x >> 3) + 32 * i, x = 8 * (threadIdx.x & 7);
        uint4_t v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (uint32_t)tile[x + 2 * j][y] | (uint32_t)tile[x + 2 * j + 1][y] << 16;
        if (c0 + y < cols && r0 + x < rows) *(uint4_t*)(to + (size_t)(c0 + y) * rows + r0 + x) = v;
    }
}

// Sums over tokens.  A workgroup takes a piece of `cut` rows of one sequence and some columns of v: for the gradient of A v = drop(x) and q = g, for
// that of B v = dy and q = h; the product of their transposes, 32 tokens at a time, with four wavefronts of VC tiles of 16 columns each.  Tiles of both
// lie in LDS by token and are read by columns, in the order of tokens that column_frag has, the same for both; v is on its way two steps ahead, q one, in
// registers.  q is binary32: three bf16 parts, 24 bits, since the result is a binary32 sum, made once before; fp16 values of v as two bf16 parts, exact,
// of which the products of both lowest parts are left out (2^-24 of the term).  What bounds it: v comes once, q for every 256 columns from the caches; 8192
// tokens of 4096 + 4096 columns at rank 64 41 us, 25.8 GFLOP of parts at 630 TFLOP/s, matrix cores 31 % busy, 141 MB read (3.4 TB/s).
// Reads by columns take 32 bytes of eight rows at once: pairs of pieces of a row, C of them, change places with its number.
template <int C>
__device__ __forceinline__ int pair_swizzle(int row) { return C >= 8 ? (row & 7) << 1 : (row / (8 / C) & (C - 1)) << 1; }
template <int RT> struct OuterLds {
    static constexpr int R = 16 * RT, QC = R / 8, VC = outer_tiles(R), COLS = 64 * VC, VROW = 2 * COLS, QROW = 6 * R;
    static constexpr int v = 32 * VROW, q = 32 * QROW, found = 2 * (v + q), bytes = found + 16;
};
template <bool BF16, int RT>
__global__ void __launch_bounds__(256, 2) outer_kernel(OuterCall p) {
    typedef OuterLds<RT> L;
    constexpr int QC = L::QC, VC = L::VC, COLS = L::COLS, VROW = L::VROW, QROW = L::QROW;
    constexpr int VN = L::v / 4096, QN = (L::q + 4095) / 4096;                // pieces of 16 bytes of a thread and step
    extern __shared__ __align__(16) char lds[];
    const AdapterRowsDev r = p.rows;
    // those of a piece, which read the same q, are `slots` numbers apart: on one die where that is a multiple of eight
    const int slot = blockIdx.x % p.slots;
    int chunk = blockIdx.x / p.slots, mat = 0;
    while (chunk >= p.mats[mat].chunks) chunk -= p.mats[mat++].chunks;
    const OuterMatDev m = p.mats[mat];
    const RowSpan s = piece_of(r, p.cut, slot, (RowSpan*)(lds + L::found));
    const int id = s.id;
    if (blockIdx.x < p.slots && threadIdx.x == 0) p.owner[slot] = id;
    if (id < 0) return;
    const int x_chunks = (m.K + COLS - 1) / COLS;
    const bool of_a = chunk < x_chunks;
    const int c0 = (of_a ? chunk : chunk - x_chunks) * COLS, wide = of_a ? m.K : m.N;
    const uint16_t* const v = of_a ? m.x : m.dy;
    const long long stride = of_a ? m.x_stride : m.dy_stride;
    const uint16_t* const q = of_a ? m.g : m.h;
    Dropout drop = r.drop;
    drop.call += (uint32_t)mat + p.first;
    const bool masked = of_a && drop.seed;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int steps = (s.t1 - s.t0 + 31) / 32;

    // a thread's piece i of a step of v: token v_row + APART i and eight columns; of q: token, part and eight values.  Places behind the piece and the
    // last column are 0
    constexpr int PER = COLS / 8, APART = 256 / PER;
    const int v_row = tid / PER, col = c0 + 8 * (tid % PER);
    auto fetch_v = [&](uint4_t (&to)[VN], int st) {
#pragma unroll
        for (int i = 0; i < VN; ++i) {
            const int t = s.t0 + 32 * st + v_row + APART * i;
            to[i] = uint4_t{0, 0, 0, 0};
            if (t < s.t1 && col < wide) to[i] = *(const uint4_t*)(v + (long long)t * stride + col);
        }
    };
    uint4_t qn[QN];
    auto fetch_q = [&](int st) {
#pragma unroll
        for (int i = 0; i < QN; ++i) {
            const int at = tid + 256 * i, t = s.t0 + 32 * st + at / (3 * QC);
            qn[i] = uint4_t{0, 0, 0, 0};
            if (at < 96 * QC && t < s.t1) qn[i] = *(const uint4_t*)(q + ((size_t)t * 3 * QC + at % (3 * QC)) * 8);
        }
    };
    uint4_t va[VN], vb[VN];
    fetch_v(va, 0);
    fetch_q(0);
    fetch_v(vb, 1);
    auto sweep = [&](auto first, auto drops) {
        constexpr bool OF_A = decltype(first)::value, MASKED = decltype(drops)::value;
        float4_t acc[VC][RT];
#pragma unroll
        for (int i = 0; i < VC; ++i)
#pragma unroll
            for (int j = 0; j < RT; ++j) acc[i][j] = float4_t{0, 0, 0, 0};
        const Keeper keeper = MASKED ? Keeper(drop) : Keeper();
        auto step = [&](int st, uint4_t (&vn)[VN]) {
            char *const vt = lds + (st & 1) * L::v, *const qt = lds + 2 * L::v + (st & 1) * L::q;
#pragma unroll
            for (int i = 0; i < VN; ++i) {
                const int row = v_row + APART * i;
                if (MASKED) vn[i] &= keeper.masks((uint32_t)col >> 3, (uint32_t)(s.t0 + 32 * st + row));
                *(uint4_t*)(vt + row * VROW + 16 * ((tid % PER) ^ pair_swizzle<8>(row))) = vn[i];
            }
#pragma unroll
            for (int i = 0; i < QN; ++i) {
                const int at = tid + 256 * i, row = at / (3 * QC), c = at % (3 * QC);
                if (at < 96 * QC) *(uint4_t*)(qt + row * QROW + 16 * (c ^ pair_swizzle<RT>(row))) = qn[i];
            }
            meet();
            fetch_q(st + 1);
            fetch_v(vn, st + 2);
            // operands by columns: lane (n, g) reads tokens 4 g + n / 4 and 16 on, and ends up with column n of tokens 4 g .. + 3 and 16 + 4 g .. + 3
            const int row = 4 * g + (n >> 2);
            auto columns = [&](const char* tile, int pitch, int piece) {
                const char* const at = tile + row * pitch + 16 * piece + 8 * (n & 1);
                const uint2_t a = lds_transposed(at), b = lds_transposed(at + 16 * pitch);
                return uint4_t{a.x, a.y, b.x, b.y};
            };
            uint4_t vf[VC], low[BF16 ? 1 : VC];
#pragma unroll
            for (int i = 0; i < VC; ++i) {
                vf[i] = columns(vt, VROW, (2 * (VC * wave + i) + (n >> 1 & 1)) ^ pair_swizzle<8>(row));
                if constexpr (!BF16) {
                    const uint4_t f = vf[i];
                    split_f16(f, vf[i], low[i]);
                }
            }
#pragma unroll
            for (int j = 0; j < RT; ++j)
#pragma unroll
                for (int o = 0; o < 3; ++o) {
                    const uint4_t qf = columns(qt, QROW, o * QC + ((2 * j + (n >> 1 & 1)) ^ pair_swizzle<RT>(row)));
#pragma unroll
                    for (int i = 0; i < VC; ++i) {
                        acc[i][j] = OF_A ? mfma_bits<true>(vf[i], qf, acc[i][j]) : mfma_bits<true>(qf, vf[i], acc[i][j]);
                        if constexpr (!BF16)
                            if (o < 2) acc[i][j] = OF_A ? mfma_bits<true>(low[i], qf, acc[i][j]) : mfma_bits<true>(qf, low[i], acc[i][j]);
                    }
                }
        };
        for (int st = 0; st < steps; st += 2) {
            step(st, va);
            if (st + 1 < steps) step(st + 1, vb);
        }
        // dA: lane (n, g) holds value n of the rank and four columns; dB: column n and four values of the rank
        float* const out = p.partial + (size_t)slot * p.size + m.at;
        const float factor = OF_A ? r.drop.factor : s.scale;
#pragma unroll
        for (int i = 0; i < VC; ++i)
#pragma unroll
            for (int j = 0; j < RT; ++j) {
                const int c = c0 + 16 * (VC * wave + i) + (OF_A ? 4 * g : n), k = 16 * j + (OF_A ? n : 4 * g);
                if (c >= wide || k >= r.rank) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] *= factor;
                *(float4_t*)(out + (OF_A ? (size_t)k * m.K + c : (size_t)r.rank * m.K + (size_t)c * r.rank + k)) = acc[i][j];
            }
    };
    if (!of_a) sweep(std::false_type{}, std::false_type{});
    else if (masked) sweep(std::true_type{}, std::true_type{});
    else sweep(std::true_type{}, std::false_type{});
}

// The gradients of an adapter: the sums of its pieces, in their order, eight on their way (sixteen of 2 MB 7 us).
__global__ void __launch_bounds__(256) gather_kernel(OuterCall p) {
    const AdapterRowsDev& r = p.rows;
    const int id = blockIdx.y;
    const size_t i = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x);
    if (i >= p.size) return;
    float4_t sum = {0, 0, 0, 0};
    for (int s = 0; s < p.slots; s += 8) {
        float4_t v[8];                                                       // eight pieces on their way
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = float4_t{0, 0, 0, 0};
            if (s + j < p.slots && p.owner[s + j] == id) v[j] = *(const float4_t*)(p.partial + (size_t)(s + j) * p.size + i);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += v[j];
    }
    int mat = 0;
    while (mat + 1 < p.n_mats && i >= p.mats[mat + 1].at) ++mat;
    const OuterMatDev& m = p.mats[mat];
    const size_t at = i - m.at, a = (size_t)r.rank * m.K;
    if (at < a) *(float4_t*)(m.da + (size_t)id * a + at) = sum;
    else *(float4_t*)(m.db + (size_t)id * r.rank * m.N + (at - a)) = sum;
}

static size_t round16(size_t n) { return (n + 15) / 16 * 16; }
static long long outer_chunks(const AdapterRowsDev& r, const AdapterMatDev* mats, int n) {
    long long c = 0;
    for (int i = 0; i < n; ++i) c += outer_chunks(r.rank, mats[i].depth, mats[i].wide);
    return c;
}
static size_t parts_bytes(const AdapterRowsDev& r) { return (size_t)r.n_tokens * 6 * padded_rank(r.rank); }
// What a group of matrices needs: turned weights, g and h in parts, owners of the pieces, their sums.
static size_t group_bytes(const AdapterRowsDev& r, const AdapterMatDev* mats, int n, size_t* turned, size_t* owner) {
    size_t weights = 0, sums = 0;
    for (int i = 0; i < n; ++i) {
        weights += (size_t)r.n_adapters * r.rank * ((size_t)mats[i].wide + mats[i].depth) * 2;
        sums += (size_t)r.rank * ((size_t)mats[i].wide + mats[i].depth) * 4;
    }
    const size_t slots = (size_t)pieces(r, cut_of(r, outer_chunks(r, mats, n)));
    *turned = round16(weights);
    *owner = round16(4 * slots);
    return *turned + 2 * n * parts_bytes(r) + *owner + slots * sums;
}
size_t adapters_backward_workspace_bytes(const AdapterRowsDev& r, const AdapterMatDev* mats, int n_mats) {
    size_t most = 0, a, b;
    for (int i = 0; i < n_mats; i += kAdapterMats) most = std::max(most, group_bytes(r, mats + i, std::min(kAdapterMats, n_mats - i), &a, &b));
    return most;
}
bool adapters_backward_fit(const AdapterRowsDev& r, const AdapterMatDev* mats, int n_mats) {
    if (r.n_adapters > 65535) return false;
    for (int i = 0; i < n_mats; i += kAdapterMats) {
        const int n = std::min(kAdapterMats, n_mats - i);
        const long long chunks = outer_chunks(r, mats + i, n);
        if ((double)pieces(r, cut_of(r, chunks)) * chunks * 256.0 >= 4294967296.0) return false;
        double size = 0;
        for (int j = 0; j < n; ++j) {
            size += (double)r.rank * ((double)mats[i + j].wide + mats[i + j].depth);
            const double tiles = ((r.rank + 63) / 64) * (double)((std::max(mats[i + j].wide, mats[i + j].depth) + 63) / 64);
            if (std::max(tiles, 512.0) * r.n_adapters * (3.0 * n) * 256.0 >= 4294967296.0) return false;
        }
        if ((size / 4 + 256) * r.n_adapters >= 4294967296.0) return false;
    }
    return true;
}

template <bool BF16, int RT>
static hipError_t sum_tokens(const OuterCall& o, dim3 grid, hipStream_t s) {
    static std::atomic<unsigned long long> raised{0};
    static_assert(OuterLds<RT>::bytes <= 160 * 1024, "a unit's LDS");
    const hipError_t e = raise_lds((const void*)outer_kernel<BF16, RT>, OuterLds<RT>::bytes, raised);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((outer_kernel<BF16, RT>), grid, dim3(256), OuterLds<RT>::bytes, s, o);
    return hipGetLastError();
}
template <bool BF16>
static hipError_t sum_tokens(const OuterCall& o, dim3 grid, hipStream_t s) {
    const int rank = o.rows.rank;
    return rank <= 16   ? sum_tokens<BF16, 1>(o, grid, s)
           : rank <= 32 ? sum_tokens<BF16, 2>(o, grid, s)
           : rank <= 64 ? sum_tokens<BF16, 4>(o, grid, s)
                        : sum_tokens<BF16, 8>(o, grid, s);
}

// mats: x = dy, y = dx, h = g (set here), depth = N, wide = K, p = b, q = a; grads: what else a matrix has.
static hipError_t backward_group(const AdapterRowsDev& rows, const AdapterMatDev* mats, const AdapterGradDev* grads, int n, int first, int dt,
                                 char* workspace, hipStream_t s) {
    size_t turned, owner;
    group_bytes(rows, mats, n, &turned, &owner);
    AdapterCall c{};
    c.rows = rows; c.y_dt = dt; c.first = (uint32_t)first; c.backward = true;
    OuterCall o{};
    o.rows = rows; o.n_mats = n; o.first = (uint32_t)first;
    uint16_t* weights = (uint16_t*)workspace;
    char* parts = workspace + turned;
    o.owner = (int*)(parts + 2 * n * parts_bytes(rows));
    o.partial = (float*)((char*)o.owner + owner);
    TurnCall turn{};
    turn.rows = rows; turn.n_mats = n;
    unsigned tiles = 0;
    for (int i = 0; i < n; ++i) {
        AdapterMatDev& m = c.mats[i].m;
        m = mats[i];
        const uint16_t** const both[2] = {&m.p, &m.q};
        for (int j = 0; j < 2; ++j) {
            const int length = j ? m.wide : m.depth, at = 2 * i + j;
            turn.from[at] = *both[j]; turn.to[at] = weights;
            turn.height[at] = j ? rows.rank : m.depth; turn.width[at] = j ? m.wide : rows.rank;
            *both[j] = weights;
            weights += (size_t)rows.n_adapters * rows.rank * length;
            tiles = std::max(tiles, (unsigned)((rows.rank + 63) / 64) * (unsigned)((length + 63) / 64));
        }
        m.h = (float*)parts; parts += parts_bytes(rows);
        turn.h[i] = grads[i].h; turn.h_parts[i] = (uint16_t*)parts; parts += parts_bytes(rows);
        OuterMatDev& d = o.mats[i];
        d.x = grads[i].x; d.x_stride = grads[i].x_stride; d.dy = m.x; d.dy_stride = m.x_stride; d.g = (uint16_t*)m.h; d.h = turn.h_parts[i];
        d.da = grads[i].da; d.db = grads[i].db; d.K = m.wide; d.N = m.depth;
        d.at = o.size; d.chunks = outer_chunks(rows.rank, d.N, d.K);
        o.size += (size_t)rows.rank * ((size_t)d.K + d.N);
        o.chunks += d.chunks;
        if (!m.y) m.wide = 0;
    }
    tiles = std::max(tiles, (unsigned)std::min<long long>(512, ((long long)rows.n_tokens * (padded_rank(rows.rank) / 4) + 255) / 256));
    hipLaunchKernelGGL(turn_kernel, dim3(tiles, rows.n_adapters, 3 * n), dim3(256), 0, s, turn);
    const hipError_t e = launch_products(c, n, dt, s);
    if (e != hipSuccess) return e;
    o.cut = cut_of(rows, o.chunks);
    o.slots = (int)pieces(rows, o.cut);
    const dim3 grid((unsigned)o.slots * o.chunks);
    const hipError_t summed = dt == DT_BF16 ? sum_tokens<true>(o, grid, s) : sum_tokens<false>(o, grid, s);
    if (summed != hipSuccess) return summed;
    hipLaunchKernelGGL(gather_kernel, dim3((unsigned)((o.size / 4 + 255) / 256), rows.n_adapters), dim3(256), 0, s, o);
    return hipGetLastError();
}
hipError_t launch_adapters_backward(const AdapterRowsDev& rows, const AdapterMatDev* mats, const AdapterGradDev* grads, int n_mats, int dt,
                                    void* workspace, hipStream_t s) {
    for (int i = 0; i < n_mats; i += kAdapterMats) {
        const hipError_t e = backward_group(rows, mats + i, grads + i, std::min(kAdapterMats, n_mats - i), i, dt, (char*)workspace, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace rwkvq
