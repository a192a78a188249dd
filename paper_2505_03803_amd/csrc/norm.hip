// Layer norm over the last n of every row's groups x n values, and its gradients (include/rwkvq.h).
#include "common.h"

namespace rwkvq {

template <int DT_> struct Type;
template <> struct Type<DT_F16> {
    typedef uint16_t raw;
    static __device__ __forceinline__ float widen(raw v) { return f16_bits_to_f32(v); }
    static __device__ __forceinline__ raw narrow(float v) { return f32_to_f16_bits(v); }
};
template <> struct Type<DT_BF16> {
    typedef uint16_t raw;
    static __device__ __forceinline__ float widen(raw v) { return bf16_bits_to_f32(v); }
    static __device__ __forceinline__ raw narrow(float v) { return __builtin_bit_cast(raw, (__bf16)v); }   // NaN stays NaN
};
template <> struct Type<DT_F32> {
    typedef float raw;
    static __device__ __forceinline__ float widen(raw v) { return v; }
    static __device__ __forceinline__ raw narrow(float v) { return v; }
};

// The sums of two values over a workgroup of NT threads, in every thread.
template <int NT>
__device__ __forceinline__ void block_sum2(float& a, float& b, float* lds) {
#pragma unroll
    for (int off = 32; off; off >>= 1) { a += __shfl_xor(a, off, 64); b += __shfl_xor(b, off, 64); }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { lds[2 * (threadIdx.x >> 6)] = a; lds[2 * (threadIdx.x >> 6) + 1] = b; }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) { a += lds[2 * i]; b += lds[2 * i + 1]; }
}

// A workgroup per row and group, one element at a time, x read three times.
template <int DT_>
__global__ void __launch_bounds__(256) norm_loop_kernel(NormDev p) {
    typedef typename Type<DT_>::raw raw;
    __shared__ float lds[8];
    const long long seg = blockIdx.x;
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

template <int DT_>
__global__ void __launch_bounds__(256) norm_dx_loop_kernel(NormDev p) {
    typedef typename Type<DT_>::raw raw;
    __shared__ float lds[8];
    const long long seg = blockIdx.x;
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

size_t norm_backward_workspace_bytes(int M, int groups, int n) {
    return (size_t)column_parts(M, groups * n) * 2 * groups * n * sizeof(float);
}

template <int DT_>
static hipError_t norm_forward(const NormDev& p, hipStream_t s) {
    hipLaunchKernelGGL(norm_loop_kernel<DT_>, dim3((unsigned)((long long)p.M * p.groups)), dim3(256), 0, s, p);
    return hipGetLastError();
}
hipError_t launch_norm(const NormDev& p, int dt, hipStream_t s) {
    return dt == DT_F16 ? norm_forward<DT_F16>(p, s) : dt == DT_BF16 ? norm_forward<DT_BF16>(p, s) : norm_forward<DT_F32>(p, s);
}

template <int DT_>
static hipError_t norm_backward(const NormDev& p, hipStream_t s) {
    const int wide = p.groups * p.n;
    if (p.dweight) {
        const int parts = column_parts(p.M, wide);
        hipLaunchKernelGGL(norm_columns_kernel<DT_>, dim3((wide + 255) / 256, parts), dim3(256), 0, s, p);
        const hipError_t e = launch_sum_partials(p.partial, parts, 2 * wide, wide, p.dweight, p.dbias, s);
        if (e != hipSuccess) return e;
    }
    if (p.dx) hipLaunchKernelGGL(norm_dx_loop_kernel<DT_>, dim3((unsigned)((long long)p.M * p.groups)), dim3(256), 0, s, p);
    return hipGetLastError();
}
hipError_t launch_norm_backward(const NormDev& p, int dt, hipStream_t s) {
    return dt == DT_F16 ? norm_backward<DT_F16>(p, s) : dt == DT_BF16 ? norm_backward<DT_BF16>(p, s) : norm_backward<DT_F32>(p, s);
}

}  // namespace rwkvq
