// Low-rank adapters beside frozen matrices (include/rwkvq.h), y_t = base_t + s_a B_a h_t with h_t = A_a drop(x_t), and their gradients:
//   g_t = s_a B_a^T dy_t,   dx_t = base_t + drop(A_a^T g_t),   dA_a = sum_t g_t drop(x_t)^T,   dB_a = s_a sum_t dy_t h_t^T.
#include "dropout.h"
#include "matrix_core.h"
#include "pieces.h"

#include <type_traits>

namespace rwkvq {

struct AdapterCall {
    AdapterRowsDev rows;
    AdapterMatDev mats[kAdapterMats];
    int y_dt, slice, slices;                       // columns of a workgroup, workgroups of a tile
    uint32_t first;                                // number of the first matrix
    bool backward;                                 // x = dy, y = dx, h = g, p = b turned, q = a turned
};
struct OuterMatDev {
    const uint16_t *x, *dy;
    const float *g, *h;
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
    int n_mats, chunks, cut;
    uint32_t first;
};
struct TurnCall {
    AdapterRowsDev rows;
    const uint16_t* from[2 * kAdapterMats];
    uint16_t* to[2 * kAdapterMats];
    int height[2 * kAdapterMats], width[2 * kAdapterMats];
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
// Piece number `slot` of a call: up to `cut` rows of one sequence.  With offsets sequence b has the numbers from offsets[b] / cut + b on, one more than
// it needs at times: then t0 >= t1.  Every thread of the workgroup calls it.
struct RowSpan { int b, t0, t1; };
__device__ __forceinline__ RowSpan piece_of(const AdapterRowsDev& r, int cut, int slot, int* found) {
    RowSpan s;
    int idx;
    if (r.offsets) {
        if (threadIdx.x == 0) *found = -1;
        __syncthreads();
        for (int b = threadIdx.x; b < r.n_seqs; b += blockDim.x) {
            int t0, t1;
            rows_of(r, b, t0, t1);
            if (slot >= t0 / cut + b && slot <= t1 / cut + b) *found = b;
        }
        __syncthreads();
        s.b = __builtin_amdgcn_readfirstlane(*found);
        if (s.b < 0) { s.t0 = s.t1 = 0; return s; }
        rows_of(r, s.b, s.t0, s.t1);
        idx = slot - (s.t0 / cut + s.b);
    } else {
        const int per = (r.n_tokens / r.n_seqs + cut - 1) / cut;
        s.b = slot / per;
        rows_of(r, s.b, s.t0, s.t1);
        idx = slot - s.b * per;
    }
    s.t0 = min(s.t0 + idx * cut, s.t1);            // idx cut <= n_tokens
    s.t1 = min(s.t0 + cut, s.t1);
    return s;
}
static long long pieces(const AdapterRowsDev& r, int cut) {
    if (r.offsets) return (long long)r.n_tokens / cut + r.n_seqs;
    return (long long)((r.n_tokens / r.n_seqs + cut - 1) / cut) * r.n_seqs;
}

__device__ __forceinline__ void load8_of(float (&f)[8], const void* p, long long i, int dt) {
    if (dt == DT_F16) load8<DT_F16>(f, p, i, 8, true);
    else if (dt == DT_BF16) load8<DT_BF16>(f, p, i, 8, true);
    else load8<DT_F32>(f, p, i, 8, true);
}
__device__ __forceinline__ void store8_of(void* p, long long i, const float (&f)[8], int dt) {
    if (dt == DT_F16) store8<DT_F16>(p, i, f, 8, true);
    else if (dt == DT_BF16) store8<DT_BF16>(p, i, f, 8, true);
    else store8<DT_F32>(p, i, f, 8, true);
}
// Eight 16-bit values of which only those with their bit in `keep` stay.
__device__ __forceinline__ uint4_t kept(uint4_t v, uint32_t keep) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t k = keep >> (2 * j);
        v[j] &= ((k & 1) ? 0xFFFFu : 0u) | ((k & 2) ? 0xFFFF0000u : 0u);
    }
    return v;
}

// Both products of a tile of up to 16 MT rows of one sequence: first h = P x^T (P: rank rows of `depth` values), then y = base + Q h (Q: `wide` rows of
// rank values).  The eight wavefronts share out the depth of the first, sums meet in LDS, and the columns of the second.  A workgroup takes
// `slice` columns of y and computes h for itself: where few tiles leave most of the device without work, h is cheaper taken several times than
// passed on through memory and another launch.
// h goes into the second product as PARTS parts of 16 bits (two: 16 bits of bf16, 22 of fp16, beside the rounding of a 16-bit y; three for binary32), fp16
// ones under a power of two for each row that brings its largest value to 2^14, so that none is lost below fp16's range.
template <bool BF16, int RT, int MT, int PARTS>
__global__ void __launch_bounds__(512) adapter_kernel(AdapterCall p) {
    constexpr int R = 16 * RT, ROWS = 16 * MT, PITCH = R + 4;
    constexpr int STEPS = (PARTS * R + 31) / 32, HROW = 64 * STEPS + 16;      // bytes of a row of h's parts
    __shared__ float sums[4][ROWS][PITCH];
    __shared__ __align__(16) char parts[ROWS * HROW];
    __shared__ float inverse[ROWS];
    __shared__ int found;
    const AdapterRowsDev& r = p.rows;
    const AdapterMatDev& m = p.mats[blockIdx.y];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int slot = blockIdx.x / p.slices, part = blockIdx.x % p.slices;
    const RowSpan s = piece_of(r, ROWS, slot, &found);
    if (s.t0 >= s.t1) return;
    const int count = s.t1 - s.t0, id = adapter_of(r, s.b);
    const float scale = id >= 0 && r.scales ? r.scales[id] : 1.0f;
    const float before = p.backward ? scale : r.drop.factor, behind = p.backward ? r.drop.factor : scale;
    Dropout drop = r.drop;
    drop.call += blockIdx.y + p.first;

    if (id >= 0) {
        float4_t acc[MT][RT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < RT; ++j) acc[i][j] = float4_t{0, 0, 0, 0};
        const uint16_t* const P = m.p + (size_t)id * r.rank * m.depth;
        const uint16_t* x[MT];
        uint32_t row[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            row[i] = (uint32_t)(s.t0 + min(16 * i + n, count - 1));
            x[i] = m.x + (long long)row[i] * m.x_stride;
        }
        auto sweep = [&](auto masked) {
            // wavefront w takes 64 columns at 64 w, 64 w + 512, ..
            for (int k0 = 64 * wave; k0 < m.depth; k0 += 512) {
                uint4_t xf[2][MT], pf[2][RT];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = k0 + 32 * h + 8 * g;
                    const bool live = k < m.depth;
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        xf[h][i] = uint4_t{0, 0, 0, 0};
                        if (live) xf[h][i] = *(const uint4_t*)(x[i] + k);
                    }
#pragma unroll
                    for (int j = 0; j < RT; ++j) {
                        pf[h][j] = uint4_t{0, 0, 0, 0};
                        if (live && 16 * j + n < r.rank) pf[h][j] = *(const uint4_t*)(P + (size_t)(16 * j + n) * m.depth + k);
                    }
                }
                if constexpr (decltype(masked)::value) {
                    const Keeper keeper(drop);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < MT; ++i) xf[h][i] = kept(xf[h][i], keeper.bits((uint32_t)(k0 + 32 * h + 8 * g) >> 3, row[i]));
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int j = 0; j < RT; ++j) acc[i][j] = mfma_bits<BF16>(pf[h][j], xf[h][i], acc[i][j]);
            }
        };
        if (drop.seed && !p.backward) sweep(std::true_type{});
        else sweep(std::false_type{});
        // lane (n, g): row n, values 4 g .. + 3 of a tile
        auto place = [&](int w, int i, int j) { return (float4_t*)&sums[w][16 * i + n][16 * j + 4 * g]; };
        if (wave >= 4)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < RT; ++j) *place(wave - 4, i, j) = acc[i][j];
        __syncthreads();
        if (wave < 4)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < RT; ++j) *place(wave, i, j) += acc[i][j];
        __syncthreads();
    }
    // sixteen threads a row
    if (tid < 16 * ROWS) {
        const int q = tid & 15, at = tid >> 4;
        float4_t h[(RT + 3) / 4];
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < (RT + 3) / 4; ++i) {
            const int c = 4 * q + 64 * i;
            h[i] = float4_t{0, 0, 0, 0};
            if (id >= 0 && c < R) {
#pragma unroll
                for (int w = 0; w < 4; ++w) h[i] += *(const float4_t*)&sums[w][at][c];
#pragma unroll
                for (int j = 0; j < 4; ++j) h[i][j] *= before;
            }
            if (m.h && part == 0 && at < count && c < r.rank) *(float4_t*)(m.h + (long long)(s.t0 + at) * r.rank + c) = h[i];
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
                    *(uint2_t*)(parts + at * HROW + 2 * (o * R + c)) = w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) rest[j] -= widen16<BF16>((uint16_t)(w[j / 2] >> (16 * (j & 1))));
                }
                if (RT == 1 && PARTS == 3) *(uint2_t*)(parts + at * HROW + 2 * (3 * R + c)) = uint2_t{0, 0};
            }
        }
    }
    __syncthreads();

    // columns: a wavefront takes 64 at a time, of which the tile of lane (n, g) ends up with 16 g .. 16 g + 15 of row n
    const uint16_t* const Q = m.q + (id >= 0 ? (size_t)id * r.rank * m.wide : 0);
    const int from = part * p.slice, to = min(from + p.slice, m.wide);
    const bool masked = drop.seed && p.backward;
    for (int c0 = from + 64 * wave; c0 < to; c0 += 512) {
        constexpr int QS = RT == 1 ? 1 : RT / 2;
        float4_t acc[MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = float4_t{0, 0, 0, 0};
        if (id >= 0) {
            uint4_t qf[4][QS];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = c0 + 16 * (n >> 2) + 4 * j + (n & 3);
#pragma unroll
                for (int k = 0; k < QS; ++k) {
                    const int c = RT == 1 ? 8 * (g & 1) : 32 * k + 8 * g;
                    qf[j][k] = uint4_t{0, 0, 0, 0};
                    if (col < to && c < r.rank) qf[j][k] = *(const uint4_t*)(Q + (size_t)col * r.rank + c);
                }
            }
#pragma unroll
            for (int st = 0; st < STEPS; ++st)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const uint4_t hf = *(const uint4_t*)(parts + (16 * i + n) * HROW + 64 * st + 16 * g);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = mfma_bits<BF16>(qf[j][st % QS], hf, acc[i][j]);
                }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int at = 16 * i + n;
            if (at >= count) continue;
            const long long t = s.t0 + at;
            const float down = BF16 ? 1.0f : inverse[at];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int col = c0 + 16 * g + 8 * half;
                if (col >= to) continue;
                float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (m.base) load8_of(y, m.base, t * m.base_stride + col, p.y_dt);
                uint32_t keep = id >= 0 ? 0xFFu : 0u;
                if (masked && id >= 0) keep = Keeper(drop).bits((uint32_t)col >> 3, (uint32_t)t);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float z = acc[i][2 * half + j / 4][j & 3];
                    if (keep >> j & 1) y[j] = m.base ? fmaf(z, down, y[j]) : z * down;
                }
                store8_of(m.y, t * m.y_stride + col, y, p.y_dt);
            }
        }
    }
}

template <bool BF16, int RT, int MT>
static hipError_t products(const AdapterCall& p, dim3 grid, hipStream_t s) {
    if (p.y_dt == DT_F32) hipLaunchKernelGGL((adapter_kernel<BF16, RT, MT, 3>), grid, dim3(512), 0, s, p);
    else hipLaunchKernelGGL((adapter_kernel<BF16, RT, MT, 2>), grid, dim3(512), 0, s, p);
    return hipGetLastError();
}
template <bool BF16, int RT>
static hipError_t products(const AdapterCall& p, int mt, dim3 grid, hipStream_t s) {
    return mt == 1 ? products<BF16, RT, 1>(p, grid, s) : products<BF16, RT, 2>(p, grid, s);
}
template <bool BF16>
static hipError_t products(const AdapterCall& p, int mt, dim3 grid, hipStream_t s) {
    return p.rows.rank <= 16   ? products<BF16, 1>(p, mt, grid, s)
           : p.rows.rank <= 32 ? products<BF16, 2>(p, mt, grid, s)
           : p.rows.rank <= 64 ? products<BF16, 4>(p, mt, grid, s)
                               : products<BF16, 8>(p, mt, grid, s);
}
// Rows of a tile, and columns of a workgroup: as many workgroups as two a compute unit, of no fewer than 256 columns each.
static int tile_rows(const AdapterRowsDev& r) { return r.n_tokens / r.n_seqs <= 16 ? 16 : 32; }
static int slice_of(const AdapterRowsDev& r, int n_mats, int widest) {
    const long long wgs = pieces(r, tile_rows(r)) * n_mats;
    const long long most = (widest + 255) / 256, wanted = std::max(1ll, std::min(most, 512 / std::max(1ll, wgs)));
    return (int)(((widest + wanted - 1) / wanted + 63) / 64 * 64);
}
bool adapters_fit(const AdapterRowsDev& r, int widest) {
    const int slice = slice_of(r, 1, widest);
    return (double)pieces(r, tile_rows(r)) * ((widest + slice - 1) / slice) * kAdapterMats * 512.0 < 4294967296.0;
}
static hipError_t launch_products(AdapterCall p, int n_mats, int dt, hipStream_t s) {
    int widest = 64;                                  // also where no y is asked for
    for (int i = 0; i < n_mats; ++i) widest = std::max(widest, p.mats[i].wide);
    const int rows = tile_rows(p.rows);
    p.slice = slice_of(p.rows, n_mats, widest);
    p.slices = (widest + p.slice - 1) / p.slice;
    const dim3 grid((unsigned)(pieces(p.rows, rows) * p.slices), (unsigned)n_mats);
    return dt == DT_BF16 ? products<true>(p, rows / 16, grid, s) : products<false>(p, rows / 16, grid, s);
}

hipError_t launch_adapters(const AdapterRowsDev& rows, const AdapterMatDev* mats, int n_mats, int dt, int y_dt, hipStream_t s) {
    for (int i = 0; i < n_mats; i += kAdapterMats) {
        AdapterCall p{};
        p.rows = rows; p.y_dt = y_dt; p.first = (uint32_t)i;
        const int n = std::min(kAdapterMats, n_mats - i);
        for (int j = 0; j < n; ++j) p.mats[j] = mats[i + j];
        const hipError_t e = launch_products(p, n, dt, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- gradients ----------------------------------------------------------------------------------------------------------

// Weights [rows][cols] of each adapter that a sequence has, as [cols][rows]; a workgroup turns 64 x 64 of them.
__global__ void __launch_bounds__(256) turn_kernel(TurnCall p) {
    __shared__ uint16_t tile[64][66];
    __shared__ int used;
    const AdapterRowsDev& r = p.rows;
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
    const int x = threadIdx.x & 63;
    for (int y = threadIdx.x >> 6; y < 64; y += 4)
        if (r0 + y < rows && c0 + x < cols) tile[y][x] = from[(size_t)(r0 + y) * cols + c0 + x];
    __syncthreads();
    for (int y = threadIdx.x >> 6; y < 64; y += 4)
        if (c0 + y < cols && r0 + x < rows) to[(size_t)(c0 + y) * rows + r0 + x] = tile[x][y];
}

// Sums over tokens.  A workgroup takes a piece of `cut` rows of one sequence and 128 columns of v: for the gradient of A v = drop(x) and q = g, for that of B
// v = dy and q = h; the product of their transposes, 32 tokens at a time, with four wavefronts of 32 columns each.  Tiles of both lie
// in LDS by token and are read by columns, in the order of tokens that column_frag has, the same for both.
// q is binary32: three bf16 parts, 24 bits, since the result is a binary32 sum; fp16 values of v as two bf16 parts, exact, of which the products of both
// lowest parts are left out (2^-24 of the term).
constexpr int kOuterCols = 128;
template <bool BF16, int RT>
__global__ void __launch_bounds__(256) outer_kernel(OuterCall p) {
    constexpr int R = 16 * RT, VROW = 2 * kOuterCols + 16, QROW = 2 * R + 16, PLANES = BF16 ? 1 : 2;
    __shared__ __align__(16) char vt[PLANES][32 * VROW];
    __shared__ __align__(16) char qt[3][32 * QROW];
    __shared__ int found;
    const AdapterRowsDev& r = p.rows;
    const int slot = blockIdx.x / p.chunks;
    int chunk = blockIdx.x % p.chunks, mat = 0;
    while (chunk >= p.mats[mat].chunks) chunk -= p.mats[mat++].chunks;
    const OuterMatDev& m = p.mats[mat];
    const RowSpan s = piece_of(r, p.cut, slot, &found);
    const int id = s.t0 < s.t1 ? adapter_of(r, s.b) : -1;
    if (blockIdx.x % p.chunks == 0 && threadIdx.x == 0) p.owner[slot] = id;
    if (id < 0) return;
    const int x_chunks = (m.K + kOuterCols - 1) / kOuterCols;
    const bool of_a = chunk < x_chunks;
    const int c0 = (of_a ? chunk : chunk - x_chunks) * kOuterCols, wide = of_a ? m.K : m.N;
    const uint16_t* const v = of_a ? m.x : m.dy;
    const long long stride = of_a ? m.x_stride : m.dy_stride;
    const float* const q = of_a ? m.g : m.h;
    Dropout drop = r.drop;
    drop.call += (uint32_t)mat + p.first;
    const bool masked = of_a && drop.seed;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;

    // thread: 16 bytes at column 8 (tid % 16) of tokens tid / 16 and 16 on; and four values of q at a time
    constexpr int QN = (32 * R / 4 + 255) / 256;
    uint4_t vn[2];
    float4_t qn[QN];
    auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = t + tid / 16 + 16 * i, col = c0 + 8 * (tid & 15);
            vn[i] = uint4_t{0, 0, 0, 0};
            if (at < s.t1 && col < wide) {
                vn[i] = *(const uint4_t*)(v + (long long)at * stride + col);
                if (masked) vn[i] = kept(vn[i], Keeper(drop).bits((uint32_t)col >> 3, (uint32_t)at));
            }
        }
#pragma unroll
        for (int i = 0; i < QN; ++i) {
            const int e = tid + 256 * i, at = t + e / (R / 4), c = 4 * (e % (R / 4));
            qn[i] = float4_t{0, 0, 0, 0};
            if (e < 32 * R / 4 && at < s.t1 && c < r.rank) qn[i] = *(const float4_t*)(q + (long long)at * r.rank + c);
        }
    };
    float4_t acc[2][RT];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[i][j] = float4_t{0, 0, 0, 0};
    fetch(s.t0);
    for (int t = s.t0; t < s.t1; t += 32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int to = (tid / 16 + 16 * i) * VROW + 16 * (tid & 15);
            if constexpr (BF16) {
                *(uint4_t*)(vt[0] + to) = vn[i];
            } else {
                uint4_t hi, lo;
                split_f16(vn[i], hi, lo);
                *(uint4_t*)(vt[0] + to) = hi;
                *(uint4_t*)(vt[PLANES - 1] + to) = lo;
            }
        }
#pragma unroll
        for (int i = 0; i < QN; ++i) {
            const int e = tid + 256 * i, to = (e / (R / 4)) * QROW + 8 * (e % (R / 4));
            if (e < 32 * R / 4) {
                uint2_t w[3];
                split4<3>(qn[i], w);
#pragma unroll
                for (int o = 0; o < 3; ++o) *(uint2_t*)(qt[o] + to) = w[o];
            }
        }
        __syncthreads();
        if (t + 32 < s.t1) fetch(t + 32);
        uint4_t vf[PLANES][2];
#pragma unroll
        for (int o = 0; o < PLANES; ++o)
#pragma unroll
            for (int i = 0; i < 2; ++i) vf[o][i] = column_frag<VROW>(vt[o], 0, 2 * wave + i, n, g);
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
            for (int o = 0; o < 3; ++o) {
                const uint4_t qf = column_frag<QROW>(qt[o], 0, j, n, g);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int u = 0; u < PLANES; ++u)
                        if (u + o < 3) acc[i][j] = of_a ? mfma_bits<true>(vf[u][i], qf, acc[i][j]) : mfma_bits<true>(qf, vf[u][i], acc[i][j]);
            }
        __syncthreads();
    }
    // dA: lane (n, g) holds value n of the rank and four columns; dB: column n and four values of the rank
    float* const out = p.partial + (size_t)slot * p.size + m.at;
    const float factor = of_a ? r.drop.factor : r.scales ? r.scales[id] : 1.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) {
            const int col = c0 + 32 * wave + 16 * i + (of_a ? 4 * g : n), k = 16 * j + (of_a ? n : 4 * g);
            if (col >= wide || k >= r.rank) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] *= factor;
            *(float4_t*)(out + (of_a ? (size_t)k * m.K + col : (size_t)r.rank * m.K + (size_t)col * r.rank + k)) = acc[i][j];
        }
}

// The gradients of an adapter: the sums of its pieces, in their order.
__global__ void __launch_bounds__(256) gather_kernel(OuterCall p, int slots) {
    const AdapterRowsDev& r = p.rows;
    const int id = blockIdx.y;
    const size_t i = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x);
    if (i >= p.size) return;
    float4_t sum = {0, 0, 0, 0};
    for (int s = 0; s < slots; ++s)
        if (p.owner[s] == id) sum += *(const float4_t*)(p.partial + (size_t)s * p.size + i);
    int mat = 0;
    while (mat + 1 < p.n_mats && i >= p.mats[mat + 1].at) ++mat;
    const OuterMatDev& m = p.mats[mat];
    const size_t at = i - m.at, a = (size_t)r.rank * m.K;
    if (at < a) *(float4_t*)(m.da + (size_t)id * a + at) = sum;
    else *(float4_t*)(m.db + (size_t)id * r.rank * m.N + (at - a)) = sum;
}

static size_t round16(size_t n) { return (n + 15) / 16 * 16; }
// Rows of a piece: twice as many while a thousand workgroups are left, since every piece leaves sums of rank (K + N) floats.
static int cut_of(const AdapterRowsDev& r, long long chunks) {
    int cut = 256;
    while (cut < 4096 && pieces(r, 2 * cut) * chunks >= 1024) cut *= 2;
    return cut;
}
static long long outer_chunks(const AdapterMatDev* mats, int n) {
    long long c = 0;
    for (int i = 0; i < n; ++i) c += (mats[i].wide + kOuterCols - 1) / kOuterCols + (mats[i].depth + kOuterCols - 1) / kOuterCols;
    return c;
}
// What a group of matrices needs: turned weights, g, owners of the pieces, their sums.
static size_t group_bytes(const AdapterRowsDev& r, const AdapterMatDev* mats, int n, size_t* turned, size_t* owner) {
    size_t weights = 0, sums = 0;
    for (int i = 0; i < n; ++i) {
        weights += (size_t)r.n_adapters * r.rank * ((size_t)mats[i].wide + mats[i].depth) * 2;
        sums += (size_t)r.rank * ((size_t)mats[i].wide + mats[i].depth) * 4;
    }
    const size_t slots = (size_t)pieces(r, cut_of(r, outer_chunks(mats, n)));
    *turned = round16(weights);
    *owner = round16(4 * slots);
    return *turned + (size_t)n * r.n_tokens * r.rank * 4 + *owner + slots * sums;
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
        const long long chunks = outer_chunks(mats + i, n);
        if ((double)pieces(r, cut_of(r, chunks)) * chunks * 256.0 >= 4294967296.0) return false;
        double size = 0;
        for (int j = 0; j < n; ++j) {
            size += (double)r.rank * ((double)mats[i + j].wide + mats[i + j].depth);
            const double tiles = ((r.rank + 63) / 64) * (double)((std::max(mats[i + j].wide, mats[i + j].depth) + 63) / 64);
            if (tiles * r.n_adapters * (2.0 * n) * 256.0 >= 4294967296.0) return false;
        }
        if ((size / 4 + 256) * r.n_adapters >= 4294967296.0) return false;
    }
    return true;
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
    float* g = (float*)(workspace + turned);
    o.owner = (int*)((char*)g + (size_t)n * rows.n_tokens * rows.rank * 4);
    o.partial = (float*)((char*)o.owner + owner);
    TurnCall turn{};
    turn.rows = rows;
    unsigned tiles = 0;
    for (int i = 0; i < n; ++i) {
        AdapterMatDev& m = c.mats[i];
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
        m.h = g + (size_t)i * rows.n_tokens * rows.rank;
        OuterMatDev& d = o.mats[i];
        d.x = grads[i].x; d.x_stride = grads[i].x_stride; d.dy = m.x; d.dy_stride = m.x_stride; d.g = m.h; d.h = grads[i].h;
        d.da = grads[i].da; d.db = grads[i].db; d.K = m.wide; d.N = m.depth;
        d.at = o.size; d.chunks = (d.K + kOuterCols - 1) / kOuterCols + (d.N + kOuterCols - 1) / kOuterCols;
        o.size += (size_t)rows.rank * ((size_t)d.K + d.N);
        o.chunks += d.chunks;
        if (!m.y) m.wide = 0;
    }
    hipLaunchKernelGGL(turn_kernel, dim3(tiles, rows.n_adapters, 2 * n), dim3(256), 0, s, turn);
    const hipError_t e = launch_products(c, n, dt, s);
    if (e != hipSuccess) return e;
    o.cut = cut_of(rows, o.chunks);
    const long long slots = pieces(rows, o.cut);
    const dim3 grid((unsigned)(slots * o.chunks));
    auto outer = [&](auto bf16) {
        constexpr bool BF16 = decltype(bf16)::value;
        if (rows.rank <= 16) hipLaunchKernelGGL((outer_kernel<BF16, 1>), grid, dim3(256), 0, s, o);
        else if (rows.rank <= 32) hipLaunchKernelGGL((outer_kernel<BF16, 2>), grid, dim3(256), 0, s, o);
        else if (rows.rank <= 64) hipLaunchKernelGGL((outer_kernel<BF16, 4>), grid, dim3(256), 0, s, o);
        else hipLaunchKernelGGL((outer_kernel<BF16, 8>), grid, dim3(256), 0, s, o);
    };
    if (dt == DT_BF16) outer(std::true_type{});
    else outer(std::false_type{});
    hipLaunchKernelGGL(gather_kernel, dim3((unsigned)((o.size / 4 + 255) / 256), rows.n_adapters), dim3(256), 0, s, o, (int)slots);
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
