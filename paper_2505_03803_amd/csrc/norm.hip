// Layer norm over the last n of every row's groups x n values, and its gradients (include/rwkvq.h).
#include "pieces.h"

namespace rwkvq {

// V floats of a weight, or what stands for it; `whole`: 16 bytes at a time.
template <int V>
__device__ __forceinline__ void load_floats(float (&f)[V], const float* p, long long i, bool live, float otherwise, bool whole) {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = otherwise;
    if (!p || !live) return;
    if constexpr (V >= 4)
        if (whole) {
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                const float4_t v = *(const float4_t*)(p + i + j);
                f[j] = v[0]; f[j + 1] = v[1]; f[j + 2] = v[2]; f[j + 3] = v[3];
            }
            return;
        }
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = p[i + j];
}

// Which part of a call a thread has.  A team of `size` lanes (a power of two up to 64, or the workgroup) takes a group of a row, lane l the
// pieces l, l + size, ..; the teams of a workgroup share out `groups` neighbouring groups and, where there are more teams, `rows` rows.
struct Teams { int size, groups, rows; bool whole; };      // whole: weight and bias at multiples of 16 bytes
struct Seat {
    int lane, g, row;                             // row: -1 for a lane without work
    __device__ __forceinline__ Seat(const Teams& t, const NormDev& p, bool block) {
        if (block) { lane = threadIdx.x; g = blockIdx.y; row = 0; return; }
        const int team = threadIdx.x / t.size, gi = team % t.groups;
        lane = threadIdx.x % t.size; g = blockIdx.y * t.groups + gi;
        row = team / t.groups < t.rows && g < p.groups ? team / t.groups : -1;
    }
};
// The sums of a team, in each of its lanes.  For a workgroup: `lds` has 2 * NT / 64 floats, another set at every other call.
template <int NT, bool BLOCK>
__device__ __forceinline__ void team_sum2(float& a, float& b, int size, float* lds) {
    if (BLOCK) size = 64;
    for (int off = size >> 1; off; off >>= 1) { a += __shfl_xor(a, off, 64); b += __shfl_xor(b, off, 64); }
    if constexpr (BLOCK) {
        if ((threadIdx.x & 63) == 0) { lds[2 * (threadIdx.x >> 6)] = a; lds[2 * (threadIdx.x >> 6) + 1] = b; }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) { a += lds[2 * i]; b += lds[2 * i + 1]; }
    }
}

// Rows held in registers: x is read once, the next row while this one is reduced; weight and bias once per workgroup where they fit
// beside it.  What bounds it: HBM bandwidth (2048 rows of 5120 bf16 values 9.9 us, 4.2 TB/s; 6898 of 4864 binary32 ones 52 us, 5.2 TB/s), and a
// launch's latency for few rows (one of 4096 fp16 values: 2.8 us).
template <int DT_, int V, int E, bool BLOCK>
__global__ void __launch_bounds__(256) norm_kernel(NormDev p, Teams teams) {
    constexpr bool keep = E * V <= 32;
    __shared__ float lds[2][8];
    const Seat seat(teams, p, BLOCK);
    const int g0 = seat.g * p.n, rows = BLOCK ? 1 : teams.rows, size = BLOCK ? 256 : teams.size;
    auto at = [&](int e) { return (seat.lane + e * size) * V; };
    auto live = [&](int e) { return seat.row >= 0 && at(e) < p.n; };
    float w[keep ? E : 1][V], b[keep ? E : 1][V];
    if constexpr (keep)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            load_floats<V>(w[e], p.weight, g0 + at(e), live(e), 1.0f, teams.whole);
            load_floats<V>(b[e], p.bias, g0 + at(e), live(e), 0.0f, teams.whole);
        }
    Piece<DT_, V> next[E];
    auto fetch = [&](long long m) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            next[e].clear();
            if (live(e) && m < p.M) next[e].load(p.x, m * p.x_stride + g0 + at(e));
        }
    };
    const float over_n = 1.0f / (float)p.n;
    fetch((long long)blockIdx.x * rows + seat.row);
    for (long long m0 = (long long)blockIdx.x * rows; m0 < p.M; m0 += (long long)gridDim.x * rows) {
        const long long m = m0 + seat.row;
        float x[E][V], sum = 0.0f, none = 0.0f, q = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            next[e].widen(x[e]);
#pragma unroll
            for (int j = 0; j < V; ++j) sum += x[e][j];
        }
        fetch(m + (long long)gridDim.x * rows);
        team_sum2<256, BLOCK>(sum, none, size, lds[0]);
        const float mean = sum * over_n;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[e][j] -= mean;
                if (live(e)) q = fmaf(x[e][j], x[e][j], q);
            }
        team_sum2<256, BLOCK>(q, none, size, lds[1]);
        const float rstd = 1.0f / sqrtf(q * over_n + p.eps);
        if (m < p.M)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (live(e)) {
                    float we[V], be[V], y[V];
                    if constexpr (!keep) {
                        load_floats<V>(we, p.weight, g0 + at(e), true, 1.0f, teams.whole);
                        load_floats<V>(be, p.bias, g0 + at(e), true, 0.0f, teams.whole);
                    }
#pragma unroll
                    for (int j = 0; j < V; ++j) y[j] = fmaf(x[e][j] * rstd, keep ? w[keep ? e : 0][j] : we[j], keep ? b[keep ? e : 0][j] : be[j]);
                    Piece<DT_, V>::store(p.y, m * p.y_stride + g0 + at(e), y);
                }
        if (seat.lane == 0 && seat.row >= 0 && m < p.M) {
            if (p.mean) p.mean[m * p.groups + seat.g] = mean;
            if (p.rstd) p.rstd[m * p.groups + seat.g] = rstd;
        }
    }
}

// The gradients of rows held in registers, dx and a workgroup's share of dweight and dbias in one pass over dy and x.  Each team sums its
// columns over its rows in registers and leaves them in row blockIdx.x * rows + .. of the partial sums.  What bounds it: HBM bandwidth (8192 rows of
// 4096 bf16 values: 49.5 us, 4.1 TB/s, and 4.8 us for the sums of partials), for odd rows the number of loads (777 rows of 1023 binary32 ones: 6.3 us).
template <int DT_, int V, int E, bool BLOCK>
__global__ void __launch_bounds__(256) norm_backward_kernel(NormDev p, Teams teams) {
    __shared__ float lds[2][8];
    const Seat seat(teams, p, BLOCK);
    const int g0 = seat.g * p.n, rows = BLOCK ? 1 : teams.rows, size = BLOCK ? 256 : teams.size, wide = p.groups * p.n;
    auto at = [&](int e) { return (seat.lane + e * size) * V; };
    auto live = [&](int e) { return seat.row >= 0 && at(e) < p.n; };
    float w[E][V], dw[E][V], db[E][V];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        load_floats<V>(w[e], p.weight, g0 + at(e), live(e), 1.0f, teams.whole);
#pragma unroll
        for (int j = 0; j < V; ++j) dw[e][j] = db[e][j] = 0.0f;
    }
    Piece<DT_, V> xn[E], dn[E];
    float mean_n = 0.0f, rstd_n = 0.0f;
    auto fetch = [&](long long m) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            xn[e].clear(); dn[e].clear();
            if (live(e) && m < p.M) {
                xn[e].load(p.x, m * p.x_stride + g0 + at(e));
                dn[e].load(p.dy, m * p.dy_stride + g0 + at(e));
            }
        }
        const bool there = seat.row >= 0 && m < p.M;
        mean_n = there ? p.mean[m * p.groups + seat.g] : 0.0f;
        rstd_n = there ? p.rstd[m * p.groups + seat.g] : 0.0f;
    };
    const float over_n = 1.0f / (float)p.n;
    int turn = 0;
    fetch((long long)blockIdx.x * rows + seat.row);
    for (long long m0 = (long long)blockIdx.x * rows; m0 < p.M; m0 += (long long)gridDim.x * rows, turn ^= 1) {
        const long long m = m0 + seat.row;
        const float mean = mean_n, rstd = rstd_n;
        float x[E][V], d[E][V], c1 = 0.0f, c2 = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            xn[e].widen(x[e]); dn[e].widen(d[e]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[e][j] = live(e) ? (x[e][j] - mean) * rstd : 0.0f;   // a mean times a rstd that binary32 does not hold is nobody's
                const float g = d[e][j] * w[e][j];                  // 0 where dy was not read
                c1 += g;
                c2 = fmaf(g, x[e][j], c2);
                dw[e][j] = fmaf(d[e][j], x[e][j], dw[e][j]);
                db[e][j] += d[e][j];
            }
        }
        fetch(m + (long long)gridDim.x * rows);
        if (p.dx) {
            team_sum2<256, BLOCK>(c1, c2, size, lds[turn]);
            c1 *= over_n; c2 *= over_n;
            if (m < p.M)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (live(e)) {
                        float o[V];
#pragma unroll
                        for (int j = 0; j < V; ++j) o[j] = rstd * (d[e][j] * w[e][j] - c1 - x[e][j] * c2);
                        Piece<DT_, V>::store(p.dx, m * p.dx_stride + g0 + at(e), o);
                    }
        }
    }
    if (p.dweight && seat.row >= 0) {
        float* const to = p.partial + ((size_t)blockIdx.x * rows + seat.row) * 2 * wide + g0;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (live(e))
#pragma unroll
                for (int j = 0; j < V; ++j) { to[at(e) + j] = dw[e][j]; to[wide + at(e) + j] = db[e][j]; }
    }
}

// The sums of two values over a workgroup of NT threads, in every thread.
template <int NT>
__device__ __forceinline__ void block_sum2(float& a, float& b, float* lds) {
    __syncthreads();
    team_sum2<NT, true>(a, b, 64, lds);
}

// Rows and groups by a workgroup each, one element at a time, x read three times.  A launch holds fewer than 2^32 threads, so that beyond
// kLoops of them a workgroup takes several.
constexpr long long kLoops = 1 << 22;
template <int DT_>
__global__ void __launch_bounds__(256) norm_loop_kernel(NormDev p) {
    typedef typename Type<DT_>::raw raw;
    __shared__ float lds[8];
    for (long long seg = blockIdx.x; seg < (long long)p.M * p.groups; seg += gridDim.x) {
        const long long m = seg / p.groups;
        const int g0 = (int)(seg % p.groups) * p.n;
        const raw* const x = (const raw*)p.x + m * p.x_stride + g0;
        raw* const y = (raw*)p.y + m * p.y_stride + g0;
        float s = 0.0f, none = 0.0f;
        for (int c = threadIdx.x; c < p.n; c += 256) s += Type<DT_>::widen(x[c]);
        block_sum2<256>(s, none, lds);
        const float mean = s / (float)p.n;
        float q = 0.0f;
        for (int c = threadIdx.x; c < p.n; c += 256) { const float d = Type<DT_>::widen(x[c]) - mean; q = fmaf(d, d, q); }
        block_sum2<256>(q, none, lds);
        const float rstd = 1.0f / sqrtf(q / (float)p.n + p.eps);
        for (int c = threadIdx.x; c < p.n; c += 256) {
            float v = (Type<DT_>::widen(x[c]) - mean) * rstd;
            if (p.weight) v *= p.weight[g0 + c];
            if (p.bias) v += p.bias[g0 + c];
            y[c] = Type<DT_>::narrow(v);
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[seg] = mean;
            if (p.rstd) p.rstd[seg] = rstd;
        }
    }
}

template <int DT_>
__global__ void __launch_bounds__(256) norm_dx_loop_kernel(NormDev p) {
    typedef typename Type<DT_>::raw raw;
    __shared__ float lds[8];
    for (long long seg = blockIdx.x; seg < (long long)p.M * p.groups; seg += gridDim.x) {
        const long long m = seg / p.groups;
        const int g0 = (int)(seg % p.groups) * p.n;
        const raw* const x = (const raw*)p.x + m * p.x_stride + g0;
        const raw* const dy = (const raw*)p.dy + m * p.dy_stride + g0;
        raw* const dx = (raw*)p.dx + m * p.dx_stride + g0;
        const float mean = p.mean[seg], rstd = p.rstd[seg];
        float s = 0.0f, q = 0.0f;
        for (int c = threadIdx.x; c < p.n; c += 256) {
            const float g = Type<DT_>::widen(dy[c]) * (p.weight ? p.weight[g0 + c] : 1.0f);
            s += g;
            q = fmaf(g, (Type<DT_>::widen(x[c]) - mean) * rstd, q);
        }
        block_sum2<256>(s, q, lds);
        s /= (float)p.n; q /= (float)p.n;
        for (int c = threadIdx.x; c < p.n; c += 256) {
            const float g = Type<DT_>::widen(dy[c]) * (p.weight ? p.weight[g0 + c] : 1.0f);
            dx[c] = Type<DT_>::narrow(rstd * (g - s - (Type<DT_>::widen(x[c]) - mean) * rstd * q));
        }
    }
}

// dweight and dbias of rows blockIdx.y, blockIdx.y + gridDim.y, ..: a thread per column.
template <int DT_>
__global__ void __launch_bounds__(256) norm_columns_kernel(NormDev p) {
    typedef typename Type<DT_>::raw raw;
    const int wide = p.groups * p.n, c = blockIdx.x * 256 + threadIdx.x;
    if (c >= wide) return;
    const int g = c / p.n;
    float a = 0.0f, b = 0.0f;
    for (int m = blockIdx.y; m < p.M; m += gridDim.y) {
        const float d = Type<DT_>::widen(((const raw*)p.dy)[m * p.dy_stride + c]);
        const long long seg = (long long)m * p.groups + g;
        a = fmaf(d, (Type<DT_>::widen(((const raw*)p.x)[m * p.x_stride + c]) - p.mean[seg]) * p.rstd[seg], a);
        b += d;
    }
    float* const to = p.partial + (size_t)blockIdx.y * 2 * wide;
    to[c] = a;
    to[wide + c] = b;
}

// out[c] = the sum of partial[i][c] over i < count, in a fixed order: 16 threads a column, then their sums.
__global__ void __launch_bounds__(1024) sum_partials_kernel(const float* partial, int count, int width, int half, float* out0, float* out1) {
    __shared__ float lds[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), part = threadIdx.x >> 6;
    float s = 0.0f;
    if (c < width)
#pragma unroll 8
        for (int i = part; i < count; i += 16) s += partial[(size_t)i * width + c];
    lds[part][threadIdx.x & 63] = s;
    __syncthreads();
    if (part == 0 && c < width) {
#pragma unroll
        for (int i = 1; i < 16; ++i) s += lds[i][threadIdx.x];
        if (c < half) out0[c] = s;
        else out1[c - half] = s;
    }
}

hipError_t launch_sum_partials(const float* partial, int count, int width, int half, float* out0, float* out1, hipStream_t s) {
    hipLaunchKernelGGL(sum_partials_kernel, dim3((width + 63) / 64), dim3(1024), 0, s, partial, count, width, half, out0, out1);
    return hipGetLastError();
}

static int column_parts(int M, int wide) {
    const int across = (wide + 255) / 256;
    return std::max(1, std::min({M, 1024 / across, 256}));
}

// Which kernel: rows in registers (a wavefront's lanes or the workgroup, E pieces of V values a lane), or the loops over memory for rows
// that no workgroup's registers hold.  Pieces are 16 bytes where every row and group begins at a multiple of that.
constexpr int kWaveValues = 16;                   // values of a row that a lane holds: where a wavefront has the row
constexpr int block_values(int V, bool backward) { return (V > 1 ? 64 : 32) >> (backward ? 1 : 0); }     // and where the workgroup has it
struct Pick { int V, E; bool block, loop; Teams teams; int grid_x, grid_y, partials; };
static Pick pick(const NormDev& p, int dt, bool backward) {
    Pick k{};
    const int whole = dt == DT_F32 ? 4 : 8;
    const bool aligned = p.n % whole == 0 && p.x_stride % whole == 0 && p.y_stride % whole == 0 && p.dy_stride % whole == 0 && p.dx_stride % whole == 0;
    k.V = aligned ? whole : 1;
    const int pieces = (p.n + k.V - 1) / k.V;
    const long long segments = (long long)p.M * p.groups;
    // a wavefront takes a row that it holds, unless few rows would leave most of the device without one
    k.block = pieces > 64 * (kWaveValues / k.V) || (pieces > 64 && segments < 2048);
    if (!k.block) {
        k.teams.size = 1;
        while (k.teams.size < 64 && k.teams.size < pieces) k.teams.size *= 2;
        const int per = 256 / k.teams.size;
        k.teams.groups = std::min(p.groups, per);
        k.teams.rows = per / k.teams.groups;
    } else {
        k.teams.size = 256; k.teams.groups = k.teams.rows = 1;
    }
    k.teams.whole = (((uintptr_t)p.weight | (uintptr_t)p.bias) & 15) == 0;
    const int each = (pieces + k.teams.size - 1) / k.teams.size;
    for (int E : {1, 2, 3, 4, 6, 8, 16, 32, 64})
        if (k.E < each) k.E = E;
    k.loop = k.E * k.V > (k.block ? block_values(k.V, backward) : kWaveValues);
    k.grid_y = (p.groups + k.teams.groups - 1) / k.teams.groups;
    const long long row_sets = (p.M + k.teams.rows - 1) / k.teams.rows;
    // workgroups that stay for several rows: eight to a compute unit forwards; backwards, where each leaves 8 bytes a column, as many only if
    // they stay for 16 rows, and two otherwise (8192 rows of 4096 bf16: 256 in all take 68 us, 512 50, 768 53, 1024 62)
    const long long all = std::min(std::max(row_sets * k.grid_y / 16, 512ll), 2048ll);
    const int wanted = (int)std::max(1ll, (backward ? all : 2048) / k.grid_y);
    k.grid_x = (int)std::min<long long>(row_sets, wanted);
    k.partials = k.grid_x * k.teams.rows;
    if (k.grid_y > 65535) k.loop = true;
    return k;
}

size_t norm_backward_workspace_bytes(int M, int groups, int n) {
    // the most that any type and alignment of such a call needs
    size_t most = column_parts(M, groups * n);
    for (int dt : {(int)DT_F16, (int)DT_F32})
        for (int odd = 0; odd < 2; ++odd) {
            NormDev p{};
            p.M = M; p.groups = groups; p.n = n; p.x_stride = odd;
            const Pick k = pick(p, dt, true);
            if (!k.loop) most = std::max(most, (size_t)k.partials);
        }
    return most * 2 * groups * n * sizeof(float);
}

template <int DT_, int V, int E, bool BLOCK>
static void launch_rows(const NormDev& p, const Pick& k, bool backward, hipStream_t s) {
    const dim3 grid(k.grid_x, k.grid_y), block(256);
    if constexpr (E * V <= (BLOCK ? block_values(V, true) : kWaveValues))
        if (backward) hipLaunchKernelGGL((norm_backward_kernel<DT_, V, E, BLOCK>), grid, block, 0, s, p, k.teams);
    if constexpr (E * V <= (BLOCK ? block_values(V, false) : kWaveValues))
        if (!backward) hipLaunchKernelGGL((norm_kernel<DT_, V, E, BLOCK>), grid, block, 0, s, p, k.teams);
}
template <int DT_, int V, bool BLOCK>
static void launch_rows(const NormDev& p, const Pick& k, bool backward, hipStream_t s) {
    switch (k.E) {
        case 1: launch_rows<DT_, V, 1, BLOCK>(p, k, backward, s); break;
        case 2: launch_rows<DT_, V, 2, BLOCK>(p, k, backward, s); break;
        case 3: launch_rows<DT_, V, 3, BLOCK>(p, k, backward, s); break;
        case 4: launch_rows<DT_, V, 4, BLOCK>(p, k, backward, s); break;
        case 6: launch_rows<DT_, V, 6, BLOCK>(p, k, backward, s); break;
        case 8: launch_rows<DT_, V, 8, BLOCK>(p, k, backward, s); break;
        case 16: launch_rows<DT_, V, 16, BLOCK>(p, k, backward, s); break;
        case 32: launch_rows<DT_, V, 32, BLOCK>(p, k, backward, s); break;
    }
}
template <int DT_>
static void launch_rows(const NormDev& p, const Pick& k, bool backward, hipStream_t s) {
    constexpr int whole = DT_ == DT_F32 ? 4 : 8;
    if (k.V == 1) k.block ? launch_rows<DT_, 1, true>(p, k, backward, s) : launch_rows<DT_, 1, false>(p, k, backward, s);
    else k.block ? launch_rows<DT_, whole, true>(p, k, backward, s) : launch_rows<DT_, whole, false>(p, k, backward, s);
}

template <int DT_>
static hipError_t norm_forward(const NormDev& p, hipStream_t s) {
    const Pick k = pick(p, DT_, false);
    if (k.loop) hipLaunchKernelGGL(norm_loop_kernel<DT_>, dim3((unsigned)std::min((long long)p.M * p.groups, kLoops)), dim3(256), 0, s, p);
    else launch_rows<DT_>(p, k, false, s);
    return hipGetLastError();
}
hipError_t launch_norm(const NormDev& p, int dt, hipStream_t s) {
    return dt == DT_F16 ? norm_forward<DT_F16>(p, s) : dt == DT_BF16 ? norm_forward<DT_BF16>(p, s) : norm_forward<DT_F32>(p, s);
}

template <int DT_>
static hipError_t norm_backward(const NormDev& p, hipStream_t s) {
    const Pick k = pick(p, DT_, true);
    const int wide = p.groups * p.n;
    int parts = k.partials;
    if (!k.loop) {
        launch_rows<DT_>(p, k, true, s);
    } else {
        parts = column_parts(p.M, wide);
        if (p.dweight) hipLaunchKernelGGL(norm_columns_kernel<DT_>, dim3((wide + 255) / 256, parts), dim3(256), 0, s, p);
        if (p.dx) hipLaunchKernelGGL(norm_dx_loop_kernel<DT_>, dim3((unsigned)std::min((long long)p.M * p.groups, kLoops)), dim3(256), 0, s, p);
    }
    if (p.dweight) return launch_sum_partials(p.partial, parts, 2 * wide, wide, p.dweight, p.dbias, s);
    return hipGetLastError();
}
hipError_t launch_norm_backward(const NormDev& p, int dt, hipStream_t s) {
    return dt == DT_F16 ? norm_backward<DT_F16>(p, s) : dt == DT_BF16 ? norm_backward<DT_BF16>(p, s) : norm_backward<DT_F32>(p, s);
}

}  // namespace rwkvq
