// Dropout by a counter-based generator (include/rwkvq.h), with what it is added to.
#include "dropout.h"
#include "pieces.h"

namespace rwkvq {

// A thread takes eight columns of a row, all of one counter.
template <int DT_>
__global__ void __launch_bounds__(256) dropout_kernel(DropoutDev p) {
    const uint32_t blocks = (uint32_t)(p.n + 7) / 8;
    const long long all = (long long)p.M * blocks, step = (long long)gridDim.x * 256;
    const Keeper keeper(p.drop);
    long long item = (long long)blockIdx.x * 256 + threadIdx.x;
    for (RowWalk w((uint32_t)item, blocks, (uint32_t)step); item < all; item += step, w.next()) {
        const int col = 8 * (int)w.at, left = p.n - col;
        float x[8], y[8];
        load8<DT_>(x, p.x, w.row * p.x_stride + col, left, p.whole);
        if (p.base) load8<DT_>(y, p.base, w.row * p.base_stride + col, left, p.whole);
        const uint32_t all = ~0u;
        const uint4_t keep = p.drop.limit ? keeper.masks(w.at, w.row) : uint4_t{all, all, all, all};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float z = masked(x[j], keep, j);
            if (p.base) y[j] = masked(1.0f, keep, j) != 0.0f ? fmaf(z, p.drop.factor, y[j]) : y[j];      // -0 stays -0
            else y[j] = z * p.drop.factor;
        }
        store8<DT_>(p.y, w.row * p.y_stride + col, y, left, p.whole);
    }
}

hipError_t launch_dropout(DropoutDev p, int dt, hipStream_t s) {
    const int unit = dt == DT_F32 ? 4 : 8;
    p.whole = p.x_stride % unit == 0 && p.y_stride % unit == 0 && (!p.base || p.base_stride % unit == 0);
    const long long all = (long long)p.M * ((p.n + 7) / 8);
    const dim3 grid((unsigned)std::min<long long>((all + 255) / 256, 4096)), block(256);
    switch (dt) {
        case DT_F16: hipLaunchKernelGGL(dropout_kernel<DT_F16>, grid, block, 0, s, p); break;
        case DT_BF16: hipLaunchKernelGGL(dropout_kernel<DT_BF16>, grid, block, 0, s, p); break;
        default: hipLaunchKernelGGL(dropout_kernel<DT_F32>, grid, block, 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace rwkvq
