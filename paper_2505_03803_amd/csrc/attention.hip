// Linear attention with a decay for each head (include/rwkvq.h): out_t = r_t (S_{t-1} + diag(u) k_t^T v_t),
// S_t = exp(-w) S_{t-1} + k_t^T v_t, and its gradients.  With G_t the gradient of S_t,
//   G_{t-1} = exp(-w) G_t + r_t^T dout_t,  dr_t = dout_t S_{t-1}^T + u k_t (dout_t . v_t),  dk_t = v_t G_t^T + u r_t (dout_t . v_t),
//   dv_t = k_t G_t + (r_t . u k_t) dout_t,  du = sum_t r_t k_t (dout_t . v_t),  dw = -sum_t exp(-w) <G_t, S_{t-1}>,
// the last one as -sum_t r_t Z_{t-1} dout_t - <G_T, Z_T> with Z the derivative of S by -w, Z_t = exp(-w) (Z_{t-1} + S_{t-1}).
#include "common.h"

namespace rwkvq {

template <bool BF16>
__device__ __forceinline__ float widen16(uint16_t v) { return BF16 ? bf16_bits_to_f32(v) : f16_bits_to_f32(v); }
template <bool BF16>
__device__ __forceinline__ uint16_t narrow16(float v) {
    return BF16 ? __builtin_bit_cast(uint16_t, (__bf16)v) : f32_to_f16_bits(v);
}

// Rows of sequence b, within 0 .. n_tokens whatever the offsets hold.
__device__ __forceinline__ void rows_of(const HeadsDev& h, int b, int& t0, int& t1) {
    if (h.offsets) {
        t0 = min(max(h.offsets[b], 0), h.n_tokens);
        t1 = min(max(h.offsets[b + 1], t0), h.n_tokens);
    } else {
        const int len = h.n_tokens / h.n_seqs;
        t0 = b * len; t1 = t0 + len;
    }
}
// Slot of sequence b's states, -1 if it is to be left out.
__device__ __forceinline__ int slot_of(const HeadsDev& h, int b) {
    if (!h.slots) return b;
    const int s = h.slots[b];
    return s >= 0 && s < h.n_slots ? s : -1;
}

// A workgroup per sequence and head, token by token; thread j holds column j of the state.
template <int DP, bool BF16>
__global__ void __launch_bounds__(DP) attend_tokens_kernel(HeadsDev h) {
    __shared__ float rs[DP], ks[DP], ru[DP];
    const int b = blockIdx.x / h.H, head = blockIdx.x % h.H, j = threadIdx.x, D = h.D, slot = slot_of(h, b);
    if (slot < 0) return;
    int t0, t1;
    rows_of(h, b, t0, t1);
    const size_t at = ((size_t)slot * h.H + head) * D * D;
    const bool live = j < D;
    const float lam = expf(-h.w[head]), u = live ? h.u[head * D + j] : 0.0f;
    float S[DP];
#pragma unroll
    for (int c = 0; c < DP; ++c) S[c] = live && c < D && h.state ? h.state[at + (size_t)c * D + j] : 0.0f;
    for (int t = t0; t < t1; ++t) {
        float r = 0.0f, k = 0.0f, v = 0.0f;
        if (live) {
            r = widen16<BF16>(h.r[t * h.r_stride + head * D + j]);
            k = widen16<BF16>(h.k[t * h.k_stride + head * D + j]);
            v = widen16<BF16>(h.v[t * h.v_stride + head * D + j]);
        }
        __syncthreads();
        rs[j] = r; ks[j] = k; ru[j] = r * u * k;
        __syncthreads();
        float o = 0.0f, now = 0.0f;
#pragma unroll
        for (int c = 0; c < DP; ++c) {
            o = fmaf(rs[c], S[c], o);
            now += ru[c];
            S[c] = fmaf(lam, S[c], ks[c] * v);
        }
        if (live) h.out[t * h.out_stride + head * D + j] = narrow16<BF16>(fmaf(now, v, o));
    }
    if (live && h.state_out)
#pragma unroll
        for (int c = 0; c < DP; ++c)
            if (c < D) h.state_out[at + (size_t)c * D + j] = S[c];
}

// dr, dw and du: forwards, thread c with row c of the state and of its derivative by -w.
template <int DP, bool BF16>
__global__ void __launch_bounds__(DP) attend_dr_kernel(HeadsDev h) {
    __shared__ float vs[DP], ds[DP], sum[DP];
    const int b = blockIdx.x / h.H, head = blockIdx.x % h.H, c = threadIdx.x, D = h.D, slot = slot_of(h, b);
    float* const part = h.partial + (size_t)blockIdx.x * (D + 1);
    if (slot < 0) {
        if (c < D) part[c] = 0.0f;
        if (c == 0) part[D] = 0.0f;
        return;
    }
    int t0, t1;
    rows_of(h, b, t0, t1);
    const size_t at = (((size_t)slot * h.H + head) * D + c) * D;
    const bool live = c < D;
    const float lam = expf(-h.w[head]), u = live ? h.u[head * D + c] : 0.0f;
    float S[DP], Z[DP], dw = 0.0f, du = 0.0f;
#pragma unroll
    for (int j = 0; j < DP; ++j) { S[j] = live && j < D && h.state ? h.state[at + j] : 0.0f; Z[j] = 0.0f; }
    for (int t = t0; t < t1; ++t) {
        float r = 0.0f, k = 0.0f, v = 0.0f, d = 0.0f;
        if (live) {
            r = widen16<BF16>(h.r[t * h.r_stride + head * D + c]);
            k = widen16<BF16>(h.k[t * h.k_stride + head * D + c]);
            v = widen16<BF16>(h.v[t * h.v_stride + head * D + c]);
            d = widen16<BF16>(h.dout[t * h.out_stride + head * D + c]);
        }
        __syncthreads();
        vs[c] = v; ds[c] = d;
        __syncthreads();
        float g = 0.0f, z = 0.0f, now = 0.0f;
#pragma unroll
        for (int j = 0; j < DP; ++j) {
            g = fmaf(ds[j], S[j], g);
            z = fmaf(ds[j], Z[j], z);
            now = fmaf(ds[j], vs[j], now);
            Z[j] = lam * (Z[j] + S[j]);
            S[j] = fmaf(lam, S[j], k * vs[j]);
        }
        dw = fmaf(r, z, dw);
        du = fmaf(r * k, now, du);
        if (live) h.dr[t * h.r_stride + head * D + c] = narrow16<BF16>(fmaf(u * k, now, g));
    }
    if (live && h.dstate)
#pragma unroll
        for (int j = 0; j < DP; ++j)
            if (j < D) dw = fmaf(h.dstate[at + j], Z[j], dw);
    sum[c] = dw;
    __syncthreads();
    if (c == 0) {
        for (int i = 1; i < DP; ++i) dw += sum[i];
        part[D] = -dw;
    }
    if (live) part[c] = du;
}

// dk, dv and the gradient of the state in front: backwards, thread j with row j and with column j of G.
template <int DP, bool BF16>
__global__ void __launch_bounds__(DP) attend_dkv_kernel(HeadsDev h) {
    __shared__ float vs[DP], ds[DP], rs[DP], ks[DP], ru[DP];
    const int b = blockIdx.x / h.H, head = blockIdx.x % h.H, j = threadIdx.x, D = h.D, slot = slot_of(h, b);
    if (slot < 0) return;
    int t0, t1;
    rows_of(h, b, t0, t1);
    const size_t at = ((size_t)slot * h.H + head) * D * D;
    const bool live = j < D;
    const float lam = expf(-h.w[head]), u = live ? h.u[head * D + j] : 0.0f;
    for (int pass = 0; pass < 2; ++pass) {                   // 0: column j, for dv; 1: row j, for dk and the state
        float G[DP];
#pragma unroll
        for (int c = 0; c < DP; ++c)
            G[c] = live && c < D && h.dstate ? h.dstate[at + (pass ? (size_t)j * D + c : (size_t)c * D + j)] : 0.0f;
        for (int t = t1 - 1; t >= t0; --t) {
            float r = 0.0f, k = 0.0f, v = 0.0f, d = 0.0f;
            if (live) {
                r = widen16<BF16>(h.r[t * h.r_stride + head * D + j]);
                k = widen16<BF16>(h.k[t * h.k_stride + head * D + j]);
                v = widen16<BF16>(h.v[t * h.v_stride + head * D + j]);
                d = widen16<BF16>(h.dout[t * h.out_stride + head * D + j]);
            }
            __syncthreads();
            vs[j] = v; ds[j] = d; rs[j] = r; ks[j] = k; ru[j] = r * u * k;
            __syncthreads();
            float g = 0.0f, now = 0.0f;
#pragma unroll
            for (int c = 0; c < DP; ++c) {
                g = fmaf(pass ? vs[c] : ks[c], G[c], g);
                now = pass ? fmaf(ds[c], vs[c], now) : now + ru[c];
                G[c] = fmaf(lam, G[c], pass ? r * ds[c] : rs[c] * d);
            }
            if (live) {
                if (pass) h.dk[t * h.k_stride + head * D + j] = narrow16<BF16>(fmaf(u * r, now, g));
                else h.dv[t * h.v_stride + head * D + j] = narrow16<BF16>(fmaf(now, d, g));
            }
        }
        __syncthreads();
        if (pass && live && h.dstate_in)
#pragma unroll
            for (int c = 0; c < DP; ++c)
                if (c < D) h.dstate_in[at + (size_t)j * D + c] = G[c];
    }
}

// dw [H] and du [H][D] from their parts, [n_seqs][H][D + 1].
__global__ void __launch_bounds__(256) attend_sum_kernel(HeadsDev h, int parts) {
    const int i = blockIdx.x * 256 + threadIdx.x, wide = h.D + 1;
    if (i >= h.H * wide) return;
    float s = 0.0f;
    for (int p = 0; p < parts; ++p) s += h.partial[(size_t)p * h.H * wide + i];
    if (i % wide == h.D) h.dw[i / wide] = s;
    else h.du[i / wide * h.D + i % wide] = s;
}

size_t attention_workspace_bytes(const HeadsDev&) { return 0; }
size_t attention_backward_workspace_bytes(const HeadsDev& h) { return (size_t)h.n_seqs * h.H * (h.D + 1) * sizeof(float); }

template <int DP, bool BF16>
static hipError_t backward(const HeadsDev& h, hipStream_t s) {
    const dim3 grid((unsigned)(h.n_seqs * h.H));
    hipLaunchKernelGGL((attend_dr_kernel<DP, BF16>), grid, dim3(DP), 0, s, h);
    hipLaunchKernelGGL((attend_dkv_kernel<DP, BF16>), grid, dim3(DP), 0, s, h);
    hipLaunchKernelGGL(attend_sum_kernel, dim3((h.H * (h.D + 1) + 255) / 256), dim3(256), 0, s, h, h.n_seqs);
    return hipGetLastError();
}
template <bool BF16>
static hipError_t attention(const HeadsDev& h, bool grad, hipStream_t s) {
    const dim3 grid((unsigned)(h.n_seqs * h.H));
    if (grad) return h.D <= 64 ? backward<64, BF16>(h, s) : backward<128, BF16>(h, s);
    if (h.D <= 64) hipLaunchKernelGGL((attend_tokens_kernel<64, BF16>), grid, dim3(64), 0, s, h);
    else hipLaunchKernelGGL((attend_tokens_kernel<128, BF16>), grid, dim3(128), 0, s, h);
    return hipGetLastError();
}
hipError_t launch_attention(const HeadsDev& h, int dt, hipStream_t s) {
    return dt == DT_BF16 ? attention<true>(h, false, s) : attention<false>(h, false, s);
}
hipError_t launch_attention_backward(const HeadsDev& h, int dt, hipStream_t s) {
    return dt == DT_BF16 ? attention<true>(h, true, s) : attention<false>(h, true, s);
}

}  // namespace rwkvq
