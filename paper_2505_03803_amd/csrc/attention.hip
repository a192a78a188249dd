// Linear attention with a decay for each head (include/rwkvq.h): out_t = r_t (S_{t-1} + diag(u) k_t^T v_t),
// S_t = exp(-w) S_{t-1} + k_t^T v_t, and its gradients.  With G_t the gradient of S_t,
//   G_{t-1} = exp(-w) G_t + r_t^T dout_t,  dr_t = dout_t S_{t-1}^T + u k_t (dout_t . v_t),  dk_t = v_t G_t^T + u r_t (dout_t . v_t),
//   dv_t = k_t G_t + (r_t . u k_t) dout_t,  du = sum_t r_t k_t (dout_t . v_t),  dw = -sum_t exp(-w) <G_t, S_{t-1}>.
#include "matrix_core.h"

namespace rwkvq {

template <bool BF16>
__device__ __forceinline__ float widen16(uint16_t v) { return BF16 ? bf16_bits_to_f32(v) : f16_bits_to_f32(v); }
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
// A head's decay; an infinite one forgets all but the token in front, which 0 times it would make NaN.
__device__ __forceinline__ float decay_of(const HeadsDev& h, int head) {
    const uint32_t w = __builtin_amdgcn_readfirstlane(__float_as_uint(h.w[head]));
    return __uint_as_float(w == 0x7F800000u ? 0x7F7FFFFFu : w);      // the largest finite one, without leaving scalar registers
}
// Slot of sequence b's states, -1 if it is to be left out.
__device__ __forceinline__ int slot_of(const HeadsDev& h, int b) {
    if (!h.slots) return b;
    const int s = h.slots[b];
    return s >= 0 && s < h.n_slots ? s : -1;
}

// One token for each sequence: a workgroup per sequence and head.  LANES lanes hold a row of the state, four columns each, a thread
// ROWS rows; all of a state is on its way before any of it is used, and is written back where it is.  What bounds it: HBM
// bandwidth (the state read and written once), for few sequences a launch and two ways to memory.  Heads of up to 32, 64 and 128 channels
// have 8, 16 and 32 lanes a row, so that a row is one or two cache lines.  256 sequences of 64 heads of 64: 111 us, 4.9 TB/s, the rate of a copy; one
// sequence 3.6 us (rows loaded one after the other 8.1 us).
template <int LANES, int ROWS, bool BF16>
__global__ void __launch_bounds__(256) attend_step_kernel(HeadsDev h) {
    constexpr int per = 256 / LANES;              // rows at a time
    __shared__ float4_t sums[4][LANES];
    const int b = blockIdx.x / h.H, head = blockIdx.x % h.H, lane = threadIdx.x % LANES, first = threadIdx.x / LANES, D = h.D, slot = slot_of(h, b);
    if (slot < 0) return;
    const size_t at = ((size_t)slot * h.H + head) * D * D;
    const int col = 4 * lane;
    const bool live = col < D;
    const uint16_t* const r = h.r + b * h.r_stride + head * D;
    const uint16_t* const k = h.k + b * h.k_stride + head * D;
    const float* const u = h.u + head * D;
    float4_t S[ROWS];
    uint16_t rr[ROWS], kk[ROWS];
    float uu[ROWS];
    uint2_t vv = {0, 0};
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = first + per * i;
        S[i] = float4_t{0, 0, 0, 0};
        if (live && row < D && h.state) S[i] = *(const float4_t*)(h.state + at + (size_t)row * D + col);
    }
    if (live) vv = *(const uint2_t*)(h.v + b * h.v_stride + head * D + col);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = first + per * i;
        rr[i] = kk[i] = 0; uu[i] = 0.0f;
        if (row < D) { rr[i] = r[row]; kk[i] = k[row]; uu[i] = u[row]; }
    }
    const float lam = expf(-h.w[head]);
    const float v[4] = {widen16<BF16>((uint16_t)vv.x), widen16<BF16>((uint16_t)(vv.x >> 16)), widen16<BF16>((uint16_t)vv.y), widen16<BF16>((uint16_t)(vv.y >> 16))};
    float4_t o = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = first + per * i;
        const float rf = widen16<BF16>(rr[i]), kf = widen16<BF16>(kk[i]), uk = uu[i] * kf;
        float4_t next;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            o[j] = fmaf(rf, fmaf(uk, v[j], S[i][j]), o[j]);
            next[j] = fmaf(lam, S[i][j], kf * v[j]);
        }
        if (live && row < D && h.state_out) *(float4_t*)(h.state_out + at + (size_t)row * D + col) = next;
    }
#pragma unroll
    for (int off = LANES; off < 64; off <<= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], off, 64);
    if ((threadIdx.x & 63) < LANES) sums[threadIdx.x >> 6][lane] = o;
    __syncthreads();
    if (threadIdx.x < LANES && live) {
        o = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
        *(uint2_t*)(h.out + b * h.out_stride + head * D + col) = uint2_t{Elem<BF16>::pack(o[0], o[1]), Elem<BF16>::pack(o[2], o[3])};
    }
}

// ---- chunks of 64 tokens on the matrix cores ---------------------------------------------------------------------------
//
// Inside a chunk, with S the state in front of it and l = exp(-w), token a (0-based) of a sweep has
//   out_a = l^a q_a S + sum_{i<a} l^(a-1-i) (q_a . key_i) val_i + bonus,      S' = l^n S + sum_i l^(n-1-i) key_i^T val_i,
// five products on matrix cores.  The same sweep, with other operands and for two of them from the last token to the first, is
//   out:  q = r,    key = k,    val = v,    bonus (sum_c r u k) v
//   dr:   q = dout, key = v,    val = k,    bonus (dout . v) u k,    the state transposed
//   dk:   q = v,    key = dout, val = r,    bonus (v . dout) u r,    backwards, state G transposed
//   dv:   q = k,    key = r,    val = dout, bonus (sum_c k u r) dout, backwards, state G.
// The gradient of w.  Its definition weighs every pair of tokens i < t, with X_ti = l^(t-1-i) (r_t . k_i) (dout_t . v_i), by the lag t - 1 - i
// (-w's exponent).  Pairs of one chunk are summed so.  The lag of any other pair is the place a of t in its chunk, plus what follows i in its
// own chunk, plus the chunks between.  With R_t the dot of r_t with the state's part of dr_t, K_i that of k_i with the state's part of dk_i, and
// a second state N that counts the tokens of whole chunks that what is in S has passed since the segment's front, N' = l^n (N + n S),
//   -dw = (pairs of one chunk) + sum_t (a_t R_t + l^a r_t N dout_t) + sum_i (n - 1 - a_i) K_i + sum over segments <G, N>, both behind the segment.
// Each term has its own lag as its weight and nothing cancels, so that the error is one of dw's terms and of nothing else in the sequences.  (Without
// N, from differences of R, K and <G, S> at the ends of blocks of tokens, a large score without a lag leaves its rounding times the block's length.)
// The sweep for dr carries N; S and N meet x in 24 bits there, as G does in the one for dk, and sums over a chunk are carried on in binary64.
//
// A workgroup takes a segment of a sequence, one head and 64 channels of val, chunk by chunk: four wavefronts compute outputs, each those of 16
// tokens of a chunk (transposed: a lane holds one token and four consecutive channels or earlier tokens, so that the scores of a token are the
// next product's operand without leaving their registers), and four carry the state, a quarter of its rows each, and publish it in LDS as
// the next chunk's operand.  One set of four for both needs more registers than two sets on a unit have (forward, 8192 tokens of 64 heads:
// 70 us against 61).  Segments of a sequence run side by side; what those in front of one leave in its state is summed up before, by a pass over
// keys and values alone.
// What bounds it.  Forward: HBM bandwidth nearly (r, k, v and parts read and out written, 280 MB by the counters in 66 us = 4.2 TB/s of the 4.88 of a large
// copy, behind a pass of 33 us for what segments leave), with LDS busy half of the cycles.  Backward: a wavefront's own chain of LDS reads, products and
// conversions, chunk after chunk (dr; dk and dv: matrix cores busy 20 and 22 % of the cycles, LDS 45 and 46 %, 0.14 vector instructions a cycle and SIMD; one
// workgroup of twelve wavefronts a unit, whose registers and LDS leave no room for another).
// Precision: 16-bit inputs go in as they are, fp16 ones that meet a computed operand as two bf16 parts (exact); weighted scores and
// states as two bf16 parts (17 bits: half an ulp of a bf16 or fp16 output is 2^-9 or 2^-12 of it), of which fp16's products of both low parts are left
// out (2^-18); the weighted keys of a state's update as three (24 bits), since states are binary32 results, and so states behind the gradient of w.
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef float float2_t __attribute__((ext_vector_type(2)));
constexpr int kChunk = 64;                    // tokens
constexpr int kVals = 64;                     // channels of val of a workgroup

struct Segment { int b, idx, count, first_slot, t0, t1, a0, a1; };     // sequence, its place in it of how many; rows of both

// Segment number `slot` of a call: `cut` tokens each, sequence b from slot offsets[b] / cut + b on (one too many at times: count <= idx).
__device__ __forceinline__ Segment segment_of(const HeadsDev& h, int cut, int slot, int* found) {
    Segment s;
    if (h.offsets) {
        for (int b = threadIdx.x; b < h.n_seqs; b += blockDim.x) {
            const int t0 = min(max(h.offsets[b], 0), h.n_tokens), t1 = min(max(h.offsets[b + 1], t0), h.n_tokens);
            const int from = t0 / cut + b;
            if (slot >= from && slot <= t1 / cut + b) *found = b;
        }
        __syncthreads();
        s.b = __builtin_amdgcn_readfirstlane(*found);
        if (s.b < 0) { s.idx = 0; s.count = 0; return s; }
        rows_of(h, s.b, s.t0, s.t1);
        s.first_slot = s.t0 / cut + s.b;
    } else {
        const int len = h.n_tokens / h.n_seqs, per = (len + cut - 1) / cut;
        s.b = slot / per;
        s.t0 = s.b * len; s.t1 = s.t0 + len;
        s.first_slot = s.b * per;
    }
    s.idx = slot - s.first_slot;
    s.count = max(1, (s.t1 - s.t0 + cut - 1) / cut);
    s.a0 = min(s.t0 + s.idx * cut, s.t1);
    s.a1 = min(s.a0 + cut, s.t1);
    return s;
}

// Infinities and NaN.  On the matrix cores a weight of 0 times a later token's infinity would reach the earlier tokens of its chunk, so val
// is staged with 0 in the place of either, and the token and channel are marked: outputs of that channel from that token on, and
// its column of the state, are made NaN instead (so is what an infinity would have made infinite).  Keys only meet scores, which are masked
// after their product, unless they are the val of another sweep over the same tiles.  A mark is 64 times the chunk's number and 63 less the
// token, so that the largest is the latest chunk's first; nothing needs clearing.
struct Marks {
    static constexpr int bytes = 2 * 4 * (2 * kVals + 1) + 8;      // for each buffer: channels of val, channels of keys, whether there is any
    int* at;
    __device__ __forceinline__ Marks(char* lds) : at((int*)lds) {}
    __device__ __forceinline__ int* channel(int turn, bool key) const { return at + (2 * turn + key) * kVals; }
    __device__ __forceinline__ int& any(int turn) const { return at[4 * kVals + turn]; }
    __device__ __forceinline__ void clear(int tid) const {
        if (tid < 4 * kVals + 2) at[tid] = -1;
    }
    // the first marked token of a channel, or kChunk
    static __device__ __forceinline__ int first(int mark, int number) { return mark >> 6 == number ? 63 - (mark & 63) : kChunk; }
    static __device__ __forceinline__ float nan() { return __uint_as_float(0x7FC00000u); }
};

// LDS of a sweep.  Where it has room for two chunks' tiles and states (`two`), one barrier a chunk is enough: the state behind a chunk is
// published beside the one that the outputs still read (forward 70 -> 61 us).  Forward sweeps of fp16 heads of up to 64 channels keep one, so that two
// workgroups fit a unit; dr's of fp16 heads and of heads above 64 channels have room for one beside N.
// Rows of 32 or 48 bytes more than the values, for fewer bank conflicts, are no faster (dr 113 and 112 us against 112), and
// cost bf16 the second workgroup (85 us against 66).  swaps: there is a sweep whose val are the keys.
template <int DP, bool BF16, int GRAD, bool PAIR = false, bool SWAPS = false> struct Lds {
    static constexpr bool swaps = SWAPS;
    static constexpr int threads = PAIR ? 768 : 512;
    static constexpr bool split_keys = SWAPS && !BF16;                           // fp16 keys as two bf16 parts too: they are somebody's val
    static constexpr bool passed_too = GRAD == 1 || (PAIR && !SWAPS);            // N beside the state, for the gradient of w
    static constexpr int key_row = 2 * DP + 16, val_row = 2 * kVals + 16;       // bytes; 16 more than the values: rows begin at different banks
    static constexpr int key = 0, key_lo = key + kChunk * key_row, val = key_lo + (split_keys ? kChunk * key_row : 0), val_lo = val + kChunk * val_row;
    static constexpr int parts = GRAD || PAIR ? 3 : 2, part = kVals * key_row;   // of a published state
    static constexpr int state = val_lo + (BF16 ? 0 : kChunk * val_row), passed = state + parts * part, buffer = passed + (passed_too ? parts * part : 0);
    static constexpr bool two = 2 * buffer + 4 * DP + 1152 + Marks::bytes <= 160 * 1024 && (BF16 || DP > 64 || PAIR);
    static constexpr int u = two ? 2 * buffer : buffer, sums = u + 4 * DP;
    static constexpr int marks = sums + (GRAD || PAIR ? 12 * 8 + 4 * 4 * kVals : 0), bytes = marks + Marks::bytes;
    static_assert(bytes <= 160 * 1024, "a unit's LDS");
};

// Two values as packed bf16 and what is left of them.
__device__ __forceinline__ uint32_t split2(float& a, float& b) {
    uint32_t h = Elem<true>::pack(a, b);
    asm("" : "+v"(h));                            // the compiler would convert a once more for its own half
    a -= __uint_as_float(h << 16);
    b -= __uint_as_float(h & 0xFFFF0000u);
    return h;
}
// Four values as two or three bf16 parts, 17 or 24 bits.
template <int PARTS>
__device__ __forceinline__ void split4(const float4_t& x, uint2_t (&out)[PARTS]) {
    float v[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int i = 0; i < PARTS - 1; ++i) out[i] = uint2_t{split2(v[0], v[1]), split2(v[2], v[3])};
    out[PARTS - 1] = uint2_t{Elem<true>::pack(v[0], v[1]), Elem<true>::pack(v[2], v[3])};
}
// Eight fp16 values as two bf16 parts, exact.
__device__ __forceinline__ void split_f16(const uint4_t& x, uint4_t& hi, uint4_t& lo) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint2_t p = vq_split(x[i]);
        hi[i] = p.x; lo[i] = p.y;
    }
}
__device__ __forceinline__ uint2_t lds_transposed(const char* at) {
    typedef __attribute__((address_space(3))) short4_t* Ptr;
    return __builtin_bit_cast(uint2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)at));
}
// The operand whose lane (n, g) holds column 16 c + n of rows 4 g .. + 3 and 16 + 4 g .. + 3 of a tile's rows 32 ks ..: the order of
// tokens in which scores lie in their registers.
template <int ROW>
__device__ __forceinline__ uint4_t column_frag(const char* tile, int ks, int c, int n, int g) {
    const char* const at = tile + (32 * ks + 4 * g + (n >> 2)) * ROW + 32 * c + 8 * (n & 3);
    const uint2_t a = lds_transposed(at), b = lds_transposed(at + 16 * ROW);
    return uint4_t{a.x, a.y, b.x, b.y};
}

// acc += weight * a state in memory; element (x, vt)[j] is key 16 (KT wave + x) + 4 g + j, val v0 + 16 vt + n.  All loads before the first use.
template <int KT>
__device__ __forceinline__ void add_state(float4_t (&acc)[KT][4], const float* from, float weight, bool transposed, int D, int v0, int wave, int n, int g) {
    float4_t in[KT][4];
    if (transposed) {
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int vt = 0; vt < 4; ++vt) {
                const int key = 16 * (KT * wave + x) + 4 * g, val = v0 + 16 * vt + n;
                in[x][vt] = *(const float4_t*)(from + (val < D && key < D ? val * D + key : 0));
            }
    } else {
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int vt = 0; vt < 4; ++vt) {
                const int key = 16 * (KT * wave + x) + 4 * g, val = v0 + 16 * vt + n, at = val < D && key < D ? key * D + val : 0, row = val < D && key < D ? D : 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) in[x][vt][j] = from[at + j * row];
            }
    }
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int vt = 0; vt < 4; ++vt) {
            const bool live = 16 * (KT * wave + x) + 4 * g < D && v0 + 16 * vt + n < D;
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[x][vt][j] += live ? weight * in[x][vt][j] : 0.0f;
        }
}
template <int KT>
__device__ __forceinline__ void store_state(const float4_t (&acc)[KT][4], float* to, int D, int v0, int wave, int n, int g) {
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int vt = 0; vt < 4; ++vt) {
            const int key = 16 * (KT * wave + x) + 4 * g, val = v0 + 16 * vt + n;
            if (val < D && key < D)
#pragma unroll
                for (int j = 0; j < 4; ++j) to[(size_t)(key + j) * D + val] = acc[x][vt][j];
        }
}
template <int KT>
__device__ __forceinline__ void clear(float4_t (&acc)[KT][4]) {
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int vt = 0; vt < 4; ++vt) acc[x][vt] = float4_t{0, 0, 0, 0};
}

// Parts: what the segments of a direction add to a state, in the order in which lanes hold one, [slot][head][64 channels of val][x][vt][wave][lane]
// of float4.  The segment whose own part nobody needs (the last one of the sweep) has there the state that the sequence begins with.
template <int KT>
__device__ __forceinline__ size_t part_size(int D) { return (size_t)(64 * KT) * kVals * ((D + kVals - 1) / kVals); }
template <int KT>
__device__ __forceinline__ size_t part_place(int block, int x, int vt, int wave, int lane) { return 4 * (size_t)((((block * KT + x) * 4 + vt) * 4 + wave) * 64 + lane); }
template <int KT>
__device__ __forceinline__ void store_part(const float4_t (&acc)[KT][4], float* to, int v0, int wave, int lane) {
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int vt = 0; vt < 4; ++vt) *(float4_t*)(to + part_place<KT>(v0 / kVals, x, vt, wave, lane)) = acc[x][vt];
}
template <int KT>
__device__ __forceinline__ void load_part(float4_t (&in)[KT][4], const float* from, bool transposed, int v0, int wave, int lane) {
    const int n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int vt = 0; vt < 4; ++vt) {
            if (!transposed) {
                in[x][vt] = *(const float4_t*)(from + part_place<KT>(v0 / kVals, x, vt, wave, lane));
            } else {                              // key and val exchange their roles: four lanes of another tile have the lane's four values
                const int key = 16 * (KT * wave + x), tile = v0 / 16 + vt;
                const float* const at = from + part_place<KT>(key / kVals, tile % KT, key % kVals / 16, tile / KT, 16 * (n >> 2) + 4 * g) + (n & 3);
#pragma unroll
                for (int j = 0; j < 4; ++j) in[x][vt][j] = at[4 * j];
            }
        }
}
template <int KT>
__device__ __forceinline__ void add(float4_t (&acc)[KT][4], const float4_t (&in)[KT][4], float weight) {
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int vt = 0; vt < 4; ++vt) acc[x][vt] += weight * in[x][vt];
}

// The state at a segment's front, in the order of the sweep.
template <int KT>
__device__ __forceinline__ void start_state(float4_t (&acc)[KT][4], const HeadsDev& h, const Segment& s, int cut, bool scanned, const float* initial, const float* parts,
                                            bool reverse, bool transposed, bool parts_transposed, int head, int slot, float w, int v0, int wave, int lane) {
    clear(acc);
    const size_t size = part_size<KT>(h.D);
    if (s.count <= 1) {
        if (initial) add_state(acc, initial + ((size_t)slot * h.H + head) * h.D * h.D, 1.0f, transposed, h.D, v0, wave, lane & 15, lane >> 4);
        return;
    }
    auto part = [&](int idx) { return parts + ((size_t)(s.first_slot + idx) * h.H + head) * size; };
    if (scanned) {
        load_part(acc, part(s.idx), parts_transposed, v0, wave, lane);
        return;
    }
    // those in front of the segment, nearest first, then what the sequence begins with: loads of two at a time before their use
    const int before = reverse ? s.count - 1 - s.idx : s.idx, away = reverse ? s.t1 - s.a1 : s.a0 - s.t0, count = before + (initial ? 1 : 0);
    auto which = [&](int i) { return part(i == before ? (reverse ? 0 : s.count - 1) : reverse ? s.idx + 1 + i : s.idx - 1 - i); };
    auto weight = [&](int i) { return expf(-(float)(i == before ? away : i * cut) * w); };
    float4_t a[KT][4], b[KT][4];
    for (int i = 0; i < count; i += 2) {
        load_part(a, which(i), parts_transposed, v0, wave, lane);
        if (i + 1 < count) load_part(b, which(i + 1), parts_transposed, v0, wave, lane);
        add(acc, a, weight(i));
        if (i + 1 < count) add(acc, b, weight(i + 1));
    }
}

// A chunk's rows on their way into LDS: COUNT chunks of 16 bytes for each of NT threads, rows of PER such chunks.  Addresses are 32-bit
// offsets from the lowest of the chunk's 64 rows.  What hangs over an end is loaded from inside instead (a chunk's last row, a head's first
// channels): later tokens reach no output that is stored and have the weight 0 in the state (x is 0 there, which ends in sums over
// tokens), channels of keys behind a head's last meet zeros of q.
__device__ __forceinline__ uint32_t row_offset(int row, bool reverse, long long stride, int col) {
    return 2 * ((uint32_t)(reverse ? kChunk - 1 - row : row) * (uint32_t)stride + (uint32_t)col);
}
template <int NT, int COUNT, int PER>
struct Rows {
    uint4_t data[COUNT];
    uint32_t offset[COUNT];                       // of a whole chunk
    // infinities and NaN, whose exponents of all ones carry into the sign's place, to zeros and marks
    template <bool BF16>
    __device__ __forceinline__ void mark(const Marks& marks, int turn, bool is_key, int number) {
        constexpr uint32_t exponent = BF16 ? 0x7F807F80u : 0x7C007C00u, one = BF16 ? 0x00800080u : 0x04000400u;
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) any |= (data[i][c] & exponent) + one;
        if ((any & 0x80008000u) == 0) return;
        marks.any(turn) = number;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = id + NT * i, row = c / PER, col = 8 * (c % PER);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t half = 0xFFFFu << (16 * (e & 1));
                uint32_t word = data[i][e >> 1];
                if (((word & exponent & half) ^ (exponent & half)) == 0) {
                    word &= ~half;
                    atomicMax(marks.channel(turn, is_key) + col + e, 64 * number + 63 - row);
                }
                data[i][e >> 1] = word;
            }
        }
    }
    int id;                                       // the thread's number among the NT
    __device__ __forceinline__ void begin(int thread, long long stride, int width, bool reverse) {
        id = thread;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = id + NT * i, col = 8 * (c % PER);
            offset[i] = row_offset(c / PER, reverse, stride, col < width ? col : 0);
        }
    }
    // the next nt rows: a whole chunk, or what a segment has beyond whole ones
    __device__ __forceinline__ void fetch(const char* lowest, int nt, long long stride, int width, bool reverse) {
        if (nt >= kChunk) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) data[i] = *(const uint4_t*)(lowest + offset[i]);
        } else if (nt > 0) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int c = id + NT * i, col = 8 * (c % PER);
                data[i] = *(const uint4_t*)(lowest + row_offset(min(c / PER, nt - 1), reverse, stride, col < width ? col : 0));
            }
        }
    }
    __device__ __forceinline__ void store(char* tile, int row_bytes) const {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = id + NT * i;
            *(uint4_t*)(tile + (c / PER) * row_bytes + 16 * (c % PER)) = data[i];
        }
    }
    // fp16 values as two bf16 parts
    __device__ __forceinline__ void store_split(char* hi, char* lo, int row_bytes) const {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = id + NT * i;
            uint4_t x, y;
            split_f16(data[i], x, y);
            *(uint4_t*)(hi + (c / PER) * row_bytes + 16 * (c % PER)) = x;
            *(uint4_t*)(lo + (c / PER) * row_bytes + 16 * (c % PER)) = y;
        }
    }
};
// Where the rows of a tensor's next chunk begin: its lowest row of 64, not all of which need be the segment's.
struct Walk {
    const char* at;
    long long row;
    __device__ __forceinline__ Walk(const uint16_t* base, long long stride, int a0, int a1, bool reverse)
        : at((const char*)base + 2 * stride * (reverse ? a1 - kChunk : a0)), row(reverse ? -2 * stride : 2 * stride) {}
    __device__ __forceinline__ void pass(int rows) { at += row * rows; }
};
// Chunks of both directions meet at multiples of 64 tokens from a segment's front: backwards, a shorter one comes first.
__device__ __forceinline__ int first_chunk(int len, bool reverse) { return reverse ? len - (len - 1) / kChunk * kChunk : min(kChunk, len); }
// Powers of exp(-w) from which a chunk's weights are made.  A lane meets tokens 16 it + 4 g + j: their weights are near[j] times a
// power that the whole wavefront shares, so that four registers and a few scalars stand for them all.
struct Powers {
    float near[4];                                // 15 - 4 g - j
    float far[4], whole;                          // 16 i; kChunk (uniform)
    __device__ __forceinline__ void set(float w, int g) {
#pragma unroll
        for (int j = 0; j < 4; ++j) near[j] = expf(-(float)(15 - 4 * g - j) * w);
#pragma unroll
        for (int i = 0; i < 4; ++i) far[i] = uniform(expf(-(float)(16 * i) * w));
        whole = uniform(expf(-(float)kChunk * w));
    }
    static __device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
};
// Weights exp(-(nt - 1 - i) w) of tokens i = 32 ks .. + 31 of a chunk in the state behind it, in the order of column_frag.
template <bool TAIL>
__device__ __forceinline__ void key_weights(float (&kw)[8], const Powers& pow, int ks, int nt, float w, int g) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = 32 * ks + 16 * (e >> 2) + 4 * g + (e & 3);
        kw[e] = !TAIL ? pow.near[e & 3] * pow.far[3 - 2 * ks - (e >> 2)] : i < nt ? expf(-(float)(nt - 1 - i) * w) : 0.0f;
    }
}
struct Whole { static constexpr bool tail = false; };
struct Tail { static constexpr bool tail = true; };
// A fragment of keys (16-bit ones, or two bf16 parts of fp16 ones) times its weights as three bf16 parts.
template <bool BF16, bool SPLIT>
__device__ __forceinline__ void weighted_keys(const uint4_t& k, const uint4_t& low, const float (&kw)[8], uint4_t (&out)[3]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t pair = k[i];
        float a = widen16<BF16 || SPLIT>((uint16_t)pair), b = widen16<BF16 || SPLIT>((uint16_t)(pair >> 16));
        if (SPLIT) {
            const uint32_t rest = low[i];
            a += widen16<true>((uint16_t)rest); b += widen16<true>((uint16_t)(rest >> 16));
        }
        a *= kw[2 * i]; b *= kw[2 * i + 1];
        out[0][i] = split2(a, b);
        out[1][i] = split2(a, b);
        out[2][i] = Elem<true>::pack(a, b);
    }
}

// S += (weighted keys)^T val over 32 tokens of a staged chunk, the weighted keys as PARTS bf16 parts.
template <bool BF16, class L, int PARTS, int KT>
__device__ __forceinline__ void update_state(float4_t (&S)[KT][4], const uint4_t (&keys)[KT], const uint4_t (&low)[KT], const float (&kw)[8], const uint4_t (&vf)[4], const uint4_t (&vl)[4]) {
#pragma unroll
    for (int x = 0; x < KT; ++x) {
        uint4_t kp[3];
        weighted_keys<BF16, L::split_keys>(keys[x], low[x], kw, kp);
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll
            for (int vt = 0; vt < 4; ++vt) {
                S[x][vt] = mfma_bits<true>(kp[part], vf[vt], S[x][vt]);
                if (!BF16 && part < PARTS - 1) S[x][vt] = mfma_bits<true>(kp[part], vl[vt], S[x][vt]);
            }
    }
}
// The operands of 32 staged tokens: columns of val (fp16: two parts), and of a wavefront's share of the keys.
template <bool BF16>
__device__ __forceinline__ void val_columns(const char* hi, const char* lo, int ks, int n, int g, uint4_t (&vf)[4], uint4_t (&vl)[4]) {
#pragma unroll
    for (int vt = 0; vt < 4; ++vt) {
        vf[vt] = column_frag<2 * kVals + 16>(hi, ks, vt, n, g);
        if (!BF16) vl[vt] = column_frag<2 * kVals + 16>(lo, ks, vt, n, g);
    }
}
template <class L, int KT>
__device__ __forceinline__ void key_columns(const char* lds, int ks, int wave, int n, int g, uint4_t (&keys)[KT], uint4_t (&low)[KT]) {
#pragma unroll
    for (int x = 0; x < KT; ++x) {
        keys[x] = column_frag<L::key_row>(lds + L::key, ks, KT * wave + x, n, g);
        if (L::split_keys) low[x] = column_frag<L::key_row>(lds + L::key_lo, ks, KT * wave + x, n, g);
    }
}
template <int KT>
__device__ __forceinline__ void scale(float4_t (&S)[KT][4], float by) {
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int vt = 0; vt < 4; ++vt) S[x][vt] *= by;
}

// The parts of one direction, before the sweeps; transposed: key is what the state in memory calls val.  Four wavefronts with a quarter of the state's
// rows each, two tiles in LDS and so one barrier a chunk.  What bounds it: HBM bandwidth (8192 tokens of 64 heads: 33 us, 4.1 TB/s).  Both
// directions of the backward pass are one launch, four workgroups a unit; forward has half as many, and registers for that (36 us with those for
// four; backward 47 instead of 40 with those for three).  A second chunk on its way gains nothing (35 us).
struct LocalDev { const uint16_t *key, *val; long long key_stride, val_stride; const float* initial; float* parts; bool reverse, transposed; };
struct LocalsDev { LocalDev dir[2]; };

template <int DP, bool BF16, int DIRS>
__global__ void __launch_bounds__(256, DP > 64 ? 2 : 2 * DIRS) attend_local_kernel(HeadsDev h, LocalsDev locals, int cut, int blocks) {
    typedef Lds<DP, BF16, 0> L;
    constexpr int KT = DP / 64;
    __shared__ __attribute__((aligned(16))) char both[2][L::state];
    __shared__ int found;
    const LocalDev& p = locals.dir[blockIdx.y];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int slot_at = blockIdx.x / (h.H * blocks), head = blockIdx.x / blocks % h.H, v0 = blockIdx.x % blocks * kVals;
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    const Segment s = segment_of(h, cut, slot_at, &found);
    if (s.idx >= s.count || s.count <= 1) return;
    const int slot = slot_of(h, s.b), D = h.D;
    if (slot < 0) return;
    const float w = decay_of(h, head);
    float* const to = p.parts + ((size_t)slot_at * h.H + head) * part_size<KT>(D);
    float4_t S[KT][4];
    clear(S);
    if (s.idx == (p.reverse ? 0 : s.count - 1)) {
        if (!p.initial) return;
        add_state(S, p.initial + ((size_t)slot * h.H + head) * D * D, 1.0f, p.transposed, D, v0, wave, n, g);
        store_part(S, to, v0, wave, lane);
        return;
    }
    const int len = s.a1 - s.a0;
    Rows<256, DP / 32, DP / 8> kr;
    Rows<256, 2, 8> vr;
    kr.begin(threadIdx.x, p.key_stride, D, p.reverse);
    vr.begin(threadIdx.x, p.val_stride, D - v0, p.reverse);
    Walk key_at(p.key + head * D, p.key_stride, s.a0, s.a1, p.reverse), val_at(p.val + head * D + v0, p.val_stride, s.a0, s.a1, p.reverse);
    const long long key_stride = p.key_stride, val_stride = p.val_stride;
    const bool reverse = p.reverse;
    auto fetch = [&](int nt) {
        kr.fetch(key_at.at, nt, key_stride, D, reverse);
        vr.fetch(val_at.at, nt, val_stride, D - v0, reverse);
        key_at.pass(nt); val_at.pass(nt);
    };
    int nt = first_chunk(len, reverse);
    fetch(nt);
    Powers pow;
    pow.set(w, g);
    int turn = 0;                                 // two tiles: a barrier a chunk
    auto chunk = [&](auto kind, int nt, int next) {
        constexpr bool tail = decltype(kind)::tail;
        char* const lds = both[turn];
        kr.store(lds + L::key, L::key_row);
        if constexpr (BF16) vr.store(lds + L::val, L::val_row);
        else vr.store_split(lds + L::val, lds + L::val_lo, L::val_row);
        __syncthreads();
        turn ^= 1;
        fetch(next);
        scale(S, tail ? expf(-(float)nt * w) : pow.whole);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uint4_t vf[4], vl[4], keys[KT], low[KT];
            float kw[8];
            key_weights<tail>(kw, pow, ks, nt, w, g);
            val_columns<BF16>(lds + L::val, lds + L::val_lo, ks, n, g, vf, vl);
            key_columns<L>(lds, ks, wave, n, g, keys, low);
            update_state<BF16, L, 3>(S, keys, low, kw, vf, vl);
        }
    };
    for (int left = len; left > 0;) {
        const int next = min(kChunk, left - nt);
        if (nt < kChunk) chunk(Tail{}, nt, next);
        else chunk(Whole{}, nt, next);
        left -= nt;
        nt = next;
    }
    store_part(S, to, v0, wave, lane);
}

// Many segments per sequence: the state at each one's front in place of its part, a thread per element, eight loads in flight.  What bounds it: a
// launch and the way to memory (26 segments of 20 heads: 7 us).
__global__ void __launch_bounds__(256) attend_scan_kernel(HeadsDev h, LocalsDev locals, int cut, int size) {
    const LocalDev& p = locals.dir[blockIdx.z];
    const int at = blockIdx.y * 256 + threadIdx.x;
    if (at >= size) return;
    for (long long item = blockIdx.x; item < (long long)h.n_seqs * h.H; item += gridDim.x) {
        const int b = (int)(item / h.H), head = (int)(item % h.H);
        int t0, t1;
        rows_of(h, b, t0, t1);
        const int count = max(1, (t1 - t0 + cut - 1) / cut), first = h.offsets ? t0 / cut + b : b * count;
        if (count <= 1 || slot_of(h, b) < 0) continue;
        float* const x = p.parts + ((size_t)first * h.H + head) * size + at;
        const size_t stride = (size_t)h.H * size;
        const float w = decay_of(h, head), decay = expf(-(float)cut * w);
        const float ragged = expf(-(float)(t1 - t0 - (count - 1) * cut) * w);      // of the last segment, which may be shorter
        float run = p.initial ? x[(p.reverse ? 0 : count - 1) * stride] : 0.0f;
        for (int from = 0; from < count; from += 8) {        // eight loads in flight
            float own[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int m = p.reverse ? count - 1 - from - i : from + i;
                own[i] = from + i < count - 1 ? x[m * stride] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int m = p.reverse ? count - 1 - from - i : from + i;
                if (from + i < count) x[m * stride] = run;
                run = fmaf(m == count - 1 ? ragged : decay, run, own[i]);
            }
        }
    }
}

// Value j of four packed 16-bit ones.
template <bool BF16>
__device__ __forceinline__ float half_of(const uint2_t& v, int j) {
    const uint32_t pair = v[j >> 1];
    return widen16<BF16>((uint16_t)(pair >> (16 * (j & 1))));
}

struct SweepDev {
    const uint16_t *q, *key, *val, *x;
    long long q_stride, key_stride, val_stride, out_stride, x_stride;
    uint16_t* out;
    const float *initial, *parts;       // of the sweep's own state
    float* last;                        // where the state behind the sequence goes, or nullptr
    bool reverse, transposed, parts_transposed;        // transposed: key is what the state in memory calls val; and what the parts do
    __device__ __forceinline__ SweepDev swapped() const {
        SweepDev s = *this;
        s.key = val; s.val = key; s.key_stride = val_stride; s.val_stride = key_stride;
        return s;
    }
};
struct SweepsDev {
    SweepDev sweep[3];
    const float *grad_initial, *grad_parts;
    float* du_parts;
    double* dw_parts;                   // [slots][H][4]
};

// What both kinds of wavefront know of their segment.
struct Place {
    Segment s;
    int slot_at, slot, head, v0, D, len, lane, wave, n, g;
    float w;
};
// A thread's share of the staging of a sweep's chunks.  Of twelve wavefronts the first eight bring the keys, the last eight val.
template <int DP, bool BF16, class L>
struct Staging {
    Rows<512, DP / 64, DP / 8> key;
    Rows<512, 1, 8> val;
    Walk key_at, val_at;
    long long key_stride, val_stride;
    int D, width;
    bool reverse, keys, vals;
    __device__ __forceinline__ Staging(const SweepDev& p, const Place& at)
        : key_at(p.key + at.head * at.D, p.key_stride, at.s.a0, at.s.a1, p.reverse),
          val_at(p.val + at.head * at.D + at.v0, p.val_stride, at.s.a0, at.s.a1, p.reverse),
          key_stride(p.key_stride), val_stride(p.val_stride), D(at.D), width(at.D - at.v0), reverse(p.reverse),
          keys(L::threads == 512 || at.wave < 8), vals(L::threads == 512 || at.wave >= 4) {
        if (keys) key.begin(threadIdx.x, key_stride, D, reverse);
        if (vals) val.begin(threadIdx.x - (L::threads - 512), val_stride, width, reverse);
    }
    // the next chunk, of nt rows
    __device__ __forceinline__ void fetch(int nt) {
        if (keys) key.fetch(key_at.at, nt, key_stride, D, reverse);
        if (vals) val.fetch(val_at.at, nt, val_stride, width, reverse);
        key_at.pass(nt); val_at.pass(nt);
    }
    // into buffer `turn` at `lds`, as the segment's chunk `number`
    __device__ __forceinline__ void store(char* lds, const Marks& marks, int turn, int number) {
        if (vals) val.template mark<BF16>(marks, turn, false, number);
        if (L::swaps && keys) key.template mark<BF16>(marks, turn, true, number);
        if (keys) {
            if constexpr (L::split_keys) key.store_split(lds + L::key, lds + L::key_lo, L::key_row);
            else key.store(lds + L::key, L::key_row);
        }
        if (vals) {
            if constexpr (BF16) val.store(lds + L::val, L::val_row);
            else val.store_split(lds + L::val, lds + L::val_lo, L::val_row);
        }
    }
};

template <class L, int KT>
__device__ __forceinline__ void mark_state(float4_t (&S)[KT][4], const Marks& marks, int turn, int number, int wave, int n, int g) {
    bool row[KT][4] = {};
    if constexpr (L::swaps)
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j) row[x][j] = Marks::first(marks.channel(turn, true)[16 * (KT * wave + x) + 4 * g + j], number) < kChunk;
#pragma unroll
    for (int vt = 0; vt < 4; ++vt) {
        const bool col = Marks::first(marks.channel(turn, false)[16 * vt + n], number) < kChunk;
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[x][vt][j] = col || row[x][j] ? Marks::nan() : S[x][vt][j];
    }
}

// The state of a sweep: four wavefronts, each with a quarter of the rows; where the sweep has shares of the gradient of w for it (L::passed_too) N
// as well, which meets G at the segment's end.  Returns the lane's share of that.
template <int DP, bool BF16, class L>
__device__ __forceinline__ double carry_state(const HeadsDev& h, const SweepDev& p, const SweepsDev& all, const Place& at, int cut, bool scanned, char* lds) {
    constexpr int KT = DP / 64;
    const int wave = at.wave - 4, n = at.n, g = at.g, D = at.D;
    const float w = at.w;
    const Segment& s = at.s;
    Staging<DP, BF16, L> rows(p, at);
    int nt = first_chunk(at.len, p.reverse);
    rows.fetch(nt);
    float4_t S[KT][4], N[L::passed_too ? KT : 1][4];
    clear(N);
    start_state(S, h, s, cut, scanned, p.initial, p.parts, p.reverse, p.transposed, p.parts_transposed, at.head, at.slot, w, at.v0, wave, at.lane);
    Powers pow;
    pow.set(w, g);
    auto publish = [&](const float4_t (&st)[KT][4], char* to) {
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int vt = 0; vt < 4; ++vt) {
                uint2_t v[L::parts];
                split4(st[x][vt], v);
#pragma unroll
                for (int i = 0; i < L::parts; ++i) *(uint2_t*)(to + i * L::part + (16 * vt + n) * L::key_row + 2 * (16 * (KT * wave + x) + 4 * g)) = v[i];
            }
    };
    const Marks marks(lds + L::marks);
    char* buffer = lds;
    int turn = 0, number = 0;
    if constexpr (L::passed_too && L::two) publish(N, lds + L::passed);
    auto chunk = [&](auto kind, int nt, int next) {
        constexpr bool tail = decltype(kind)::tail;
        publish(S, buffer + L::state);
        if constexpr (L::passed_too && !L::two) publish(N, buffer + L::passed);
        rows.store(buffer, marks, turn, number);
        __syncthreads();
        rows.fetch(next);
        const float whole = tail ? expf(-(float)nt * w) : pow.whole;
        if constexpr (L::passed_too) {
            add(N, S, (float)nt);
            scale(N, whole);
            if (L::two) publish(N, lds + (turn ^ 1) * L::buffer + L::passed);       // nobody reads there since the barrier; beside the products (134 -> 128 us)
        }
        scale(S, whole);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uint4_t vf[4], vl[4], keys[KT], low[KT];
            float kw[8];
            key_weights<tail>(kw, pow, ks, nt, w, g);
            val_columns<BF16>(buffer + L::val, buffer + L::val_lo, ks, n, g, vf, vl);
            key_columns<L>(buffer, ks, wave, n, g, keys, low);
            update_state<BF16, L, 3>(S, keys, low, kw, vf, vl);
        }
        if (__builtin_amdgcn_readfirstlane(marks.any(turn)) == number) mark_state<L>(S, marks, turn, number, wave, n, g);
        if (L::two) turn ^= 1, buffer = lds + turn * L::buffer;
        else __syncthreads();
        ++number;
    };
    for (int left = at.len; left > 0;) {
        const int next = min(kChunk, left - nt);
        if (nt < kChunk) chunk(Tail{}, nt, next);
        else chunk(Whole{}, nt, next);
        left -= nt;
        nt = next;
    }
    if (p.last && s.idx == (p.reverse ? 0 : s.count - 1)) store_state(S, p.last + ((size_t)at.slot * h.H + at.head) * D * D, D, at.v0, wave, n, g);
    double dw = 0.0;
    if constexpr (L::passed_too) {
        start_state(S, h, s, cut, scanned, all.grad_initial, all.grad_parts, true, true, true, at.head, at.slot, w, at.v0, wave, at.lane);
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int vt = 0; vt < 4; ++vt)
#pragma unroll
                for (int j = 0; j < 4; ++j)           // places behind a head's last channels hold whatever was loaded for them
                    if (16 * (KT * wave + x) + 4 * g < D && at.v0 + 16 * vt + n < D) dw += (double)S[x][vt][j] * (double)N[x][vt][j];
    }
    return dw;
}

// x, in a scalar register, as something that changes with `by`: conditions on it are made where they are used, not kept for each lane in
// more scalar registers than there are.
template <bool YES>
__device__ __forceinline__ int per_chunk(int x, int by) {
    if (YES && !__builtin_constant_p(x)) asm("" : "+s"(x) : "s"(by));
    return x;
}

// The outputs of a sweep: four wavefronts with sixteen tokens of each chunk.  Returns the lane's share of dw, and those of du.
//   GRAD 1: the shares of dw that dr's sweep has, with x = r;  2: those of dk's and du, with x = k;  0: neither.  STORE: the outputs; where two sets of
//   wavefronts share dr's sweep the one that stores has the state's shares of dw, the other N's and those of pairs of one chunk.
//   SWAP: the tiles and the state are those of the sweep for dv, whose key and val exchange their roles in the one for dk.
template <int DP, bool BF16, class L, int GRAD, bool STORE, bool SWAP, bool U_IN_DOT>
__device__ __forceinline__ double outputs(const HeadsDev& h, const SweepDev& p, const Place& at, int wave, float (&du)[GRAD == 2 ? 16 : 1], char* lds) {
    constexpr int KS = DP / 32, parts = GRAD ? L::parts : 2;
    constexpr bool passed = GRAD == 1 && (L::threads == 512 || !STORE);
    constexpr int key_tile = SWAP ? L::val : L::key, key_low = SWAP ? L::val_lo : L::key_lo, val_tile = SWAP ? L::key : L::val, val_low = SWAP ? L::key_lo : L::val_lo;
    const int n = at.n, g = at.g, v0 = at.v0, a = 16 * wave + n;
    const float w = at.w;
    Staging<DP, BF16, L> rows(SWAP ? p.swapped() : p, at);
    const bool reverse = p.reverse;
    const long long q_stride = p.q_stride, x_stride = p.x_stride, out_stride = p.out_stride;
    Walk q_at(p.q + at.head * at.D, q_stride, at.s.a0, at.s.a1, reverse), x_at(GRAD ? p.x + at.head * at.D + v0 : p.q, x_stride, at.s.a0, at.s.a1, reverse),
        out_at(p.out + at.head * at.D + v0, out_stride, at.s.a0, at.s.a1, reverse);
    uint4_t qr[KS], xr[2];                        // x as an operand, and where the lane's outputs are
    uint2_t xdr[4];
    const int q_col = SWAP ? 4 * g : 8 * g;
    const uint32_t q_off = row_offset(a, reverse, q_stride, q_col), x_off = GRAD ? row_offset(a, reverse, x_stride, 0) : 0,
                   out_off = row_offset(a, reverse, out_stride, 4 * g);
    auto fetch = [&](int nt) {
        const int D = per_chunk<L::threads == 768 && !L::swaps>(at.D, nt);
        rows.fetch(nt);
        if (nt > 0) {
            const int row = min(a, nt - 1);
            const char* const from = q_at.at + (nt < kChunk ? row_offset(row, reverse, q_stride, q_col) : q_off);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                qr[i] = uint4_t{0, 0, 0, 0};
                if constexpr (SWAP) {             // in the order of column_frag
                    uint2_t a = {0, 0}, b = {0, 0};
                    if (D == DP || 32 * i + 4 * g < D) a = *(const uint2_t*)(from + 64 * i);
                    if (D == DP || 32 * i + 16 + 4 * g < D) b = *(const uint2_t*)(from + 64 * i + 32);
                    qr[i] = uint4_t{a.x, a.y, b.x, b.y};
                } else if (D == DP || 32 * i + 8 * g < D) {
                    qr[i] = *(const uint4_t*)(from + 64 * i);
                }
            }
        }
        q_at.pass(nt);
    };
    auto fetch_x = [&](int nt) {
        const int D = per_chunk<L::threads == 768 && !L::swaps>(at.D, nt);
        if (nt > 0) {
            const int row = min(a, nt - 1);
            if constexpr (GRAD) {
                const char* const xf = x_at.at + (nt < kChunk ? row_offset(row, reverse, x_stride, 0) : x_off);
                if constexpr (passed)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        xr[i] = uint4_t{0, 0, 0, 0};
                        if (a < nt && (D == DP || v0 + 32 * i + 8 * g < D)) xr[i] = *(const uint4_t*)(xf + 16 * g + 64 * i);
                    }
#pragma unroll
                for (int vt = 0; vt < 4; ++vt) {
                    xdr[vt] = uint2_t{0, 0};
                    if (a < nt && (D == DP || v0 + 16 * vt + 4 * g < D)) xdr[vt] = *(const uint2_t*)(xf + 8 * g + 32 * vt);
                }
            }
        }
        x_at.pass(nt);
    };
    int nt = first_chunk(at.len, reverse);
    fetch(nt);
    fetch_x(nt);
    const int u0 = U_IN_DOT ? 0 : v0, tid = 64 * wave + at.lane;
    if (tid < DP) *(float*)(lds + L::u + 4 * tid) = u0 + tid < at.D ? h.u[at.head * at.D + u0 + tid] : 0.0f;

    // weights of pairs (token a, token 16 it + 4 g + j), and of the state in front.
    // Every wavefront takes all four tiles: without branches their loads and products overlap, and the last wavefront has four anyway.
    float pw[4][4];
    bool lower[4], own[4];                        // of the lane's own tile: earlier tokens, and the lane's
    const float front = expf(-(float)a * w);
#pragma unroll
    for (int it = 0; it < 4; ++it) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int lag = a - 1 - (16 * it + 4 * g + j);
            pw[it][j] = lag >= 0 ? expf(-(float)lag * w) : 0.0f;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) { lower[j] = 4 * g + j < n; own[j] = 4 * g + j == n; }
    double dw = 0.0;

    const Marks marks(lds + L::marks);
    char* buffer = lds;
    int turn = 0, number = 0;
    auto chunk = [&](int nt, int next, int left) {
        const int tile = per_chunk<L::threads == 768 && !L::swaps>(wave, left), D = per_chunk<L::threads == 768 && !L::swaps>(at.D, left);
        rows.store(buffer, marks, turn, number);
        __syncthreads();
        uint4_t qf[KS], qh[KS], ql[KS], xf[2], xl[2];
        uint2_t xd[4];
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            qf[i] = qr[i];
            if constexpr (BF16) qh[i] = qf[i];
            else split_f16(qf[i], qh[i], ql[i]);
        }
        if constexpr (GRAD) {
            if constexpr (passed)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (BF16) xf[i] = xr[i];
                    else split_f16(xr[i], xf[i], xl[i]);
                }
#pragma unroll
            for (int vt = 0; vt < 4; ++vt) xd[vt] = xdr[vt];
        }
        fetch(next);
        if (GRAD != 1) fetch_x(next);

        auto key_frag = [&](int tile, int row, int i) {
            const char* const from = buffer + tile + row * L::key_row + 64 * i;
            if (!SWAP) return *(const uint4_t*)(from + 16 * g);
            const uint2_t x = *(const uint2_t*)(from + 8 * g), y = *(const uint2_t*)(from + 32 + 8 * g);
            return uint4_t{x.x, x.y, y.x, y.y};
        };
        // the state in front; for the gradient of w its part of the outputs with x, weighted by the token's place in the chunk, and N's
        float4_t out[4];
        double state_dot = 0.0;
#pragma unroll
        for (int vt = 0; vt < 4; ++vt) {
            auto product = [&](int state) {
                float4_t o = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int part = parts - 1; part >= 0; --part) {
                        const char* const from = buffer + state + part * L::part;
                        const uint4_t st = SWAP ? column_frag<L::key_row>(from, i, vt, n, g)
                                                : *(const uint4_t*)(from + (16 * vt + n) * L::key_row + 2 * (32 * i + 8 * g));
                        o = mfma_bits<true>(st, qh[i], o);
                        if (!BF16 && part < parts - 1) o = mfma_bits<true>(st, ql[i], o);
                    }
                return o;
            };
            out[vt] = float4_t{0, 0, 0, 0};
            if constexpr (STORE) out[vt] = front * product(L::state);
            if constexpr (GRAD) {
                float4_t weighted = (float)a * out[vt];
                if constexpr (passed) weighted += front * product(L::passed);
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) sum = fmaf(half_of<BF16>(xd[vt], j), weighted[j], sum);
                state_dot += (double)sum;
            }
        }
        if (GRAD == 1) fetch_x(next);             // here, where the registers of x are free again (fp16 187 -> 171 us, 128 channels 199 -> 193)
        if (GRAD && a < nt) dw += state_dot;      // weights of places behind the last token may be infinite

        // scores of the wavefront's tokens with those before them
        uint4_t ph[2], pl[2];
        float dot = 0.0f;                         // of the bonus: a token's score with itself, or that with u
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int ks = it >> 1, e = 2 * (it & 1);
            float4_t sc = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const uint4_t kf = key_frag(key_tile, 16 * it + n, i);
                if constexpr (L::split_keys) {
                    const uint4_t kl = key_frag(key_low, 16 * it + n, i);
                    sc = mfma_bits<true>(kl, ql[i], sc);
                    sc = mfma_bits<true>(kl, qh[i], sc);
                    sc = mfma_bits<true>(kf, ql[i], sc);
                    sc = mfma_bits<true>(kf, qh[i], sc);
                } else {
                    sc = mfma_bits<BF16>(kf, qf[i], sc);
                }
            }
            if constexpr (STORE && !U_IN_DOT) {
                float self = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) self += own[j] ? sc[j] : 0.0f;
                dot += it == tile ? self : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[j] = (it < tile) | ((it == tile) & lower[j]) ? pw[it][j] * sc[j] : 0.0f;
            if constexpr (passed) {                                    // x . val of the same pairs, weighted with their lags
                float4_t xv = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int from = (16 * it + n) * L::val_row + 2 * (32 * i + 8 * g);
                    const uint4_t v = *(const uint4_t*)(buffer + val_tile + from);
                    if (!BF16) {
                        const uint4_t vl = *(const uint4_t*)(buffer + val_low + from);
                        xv = mfma_bits<true>(vl, xl[i], xv);
                        xv = mfma_bits<true>(vl, xf[i], xv);
                        xv = mfma_bits<true>(v, xl[i], xv);
                    }
                    xv = mfma_bits<true>(v, xf[i], xv);
                }
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += (it < tile) | ((it == tile) & lower[j]) ? sc[j] * ((float)(a - 1 - (16 * it + 4 * g + j)) * xv[j]) : 0.0f;
                if (a < nt) dw += (double)sum;
            }
            if constexpr (STORE) {
                uint2_t sp[2];
                split4(sc, sp);
                ph[ks][e] = sp[0].x; ph[ks][e + 1] = sp[0].y; pl[ks][e] = sp[1].x; pl[ks][e + 1] = sp[1].y;
            }
        }
        if constexpr (STORE) {
        if constexpr (U_IN_DOT) {
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const uint4_t kf = key_frag(key_tile, a, i), kl = L::split_keys ? key_frag(key_low, a, i) : kf;
#pragma unroll
                for (int c2 = 0; c2 < 2; ++c2) {
                    const float4_t u = *(const float4_t*)(lds + L::u + 4 * (32 * i + 8 * g + 4 * c2));
#pragma unroll
                    for (int c4 = 0; c4 < 4; ++c4) {
                        const uint32_t qq = qf[i][2 * c2 + (c4 >> 1)], kk = kf[2 * c2 + (c4 >> 1)];
                        float k = widen16<BF16 || L::split_keys>((uint16_t)(kk >> (16 * (c4 & 1))));
                        if constexpr (L::split_keys) {
                            const uint32_t rest = kl[2 * c2 + (c4 >> 1)];
                            k += widen16<true>((uint16_t)(rest >> (16 * (c4 & 1))));
                        }
                        dot = fmaf(widen16<BF16>((uint16_t)(qq >> (16 * (c4 & 1)))) * u[c4], k, dot);
                    }
                }
            }
        }
        dot += __shfl_xor(dot, 16, 64);
        dot += __shfl_xor(dot, 32, 64);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uint4_t vf[4], vl[4];
            val_columns<BF16>(buffer + val_tile, buffer + val_low, ks, n, g, vf, vl);
#pragma unroll
            for (int vt = 0; vt < 4; ++vt) {
                out[vt] = mfma_bits<true>(vf[vt], pl[ks], out[vt]);
                if (!BF16) out[vt] = mfma_bits<true>(vl[vt], ph[ks], out[vt]);
                out[vt] = mfma_bits<true>(vf[vt], ph[ks], out[vt]);
            }
        }
        // the bonus, with u at the channels of val unless the dot has it; the gradient of u
        {
#pragma unroll
            for (int vt = 0; vt < 4; ++vt) {
                const uint2_t vh = *(const uint2_t*)(buffer + val_tile + a * L::val_row + 2 * (16 * vt + 4 * g));
                const float4_t u = U_IN_DOT ? float4_t{1, 1, 1, 1} : *(const float4_t*)(lds + L::u + 4 * (16 * vt + 4 * g));
                float v[4] = {__uint_as_float(vh.x << 16), __uint_as_float(vh.x & 0xFFFF0000u), __uint_as_float(vh.y << 16), __uint_as_float(vh.y & 0xFFFF0000u)};
                if (!BF16) {
                    const uint2_t l = *(const uint2_t*)(buffer + val_low + a * L::val_row + 2 * (16 * vt + 4 * g));
                    v[0] += __uint_as_float(l.x << 16); v[1] += __uint_as_float(l.x & 0xFFFF0000u);
                    v[2] += __uint_as_float(l.y << 16); v[3] += __uint_as_float(l.y & 0xFFFF0000u);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float now = dot * v[j];
                    out[vt][j] = fmaf(now, u[j], out[vt][j]);
                    if (GRAD == 2) du[4 * vt + j] = fmaf(half_of<BF16>(xd[vt], j), now, du[4 * vt + j]);
                }
            }
        }
        if (a < nt) {
            char* const to = (char*)out_at.at + out_off;
#pragma unroll
            for (int vt = 0; vt < 4; ++vt)
                if (D == DP || v0 + 16 * vt + 4 * g < D)
                    *(uint2_t*)(to + 32 * vt) = uint2_t{Elem<BF16>::pack(out[vt][0], out[vt][1]), Elem<BF16>::pack(out[vt][2], out[vt][3])};
        }
        }
        if (__builtin_amdgcn_readfirstlane(marks.any(turn)) == number) {
            if constexpr (STORE) {
                int first = kChunk;               // of the keys, in any channel
                if constexpr (L::swaps) {
                    first = Marks::first(marks.channel(turn, !SWAP)[at.lane], number);
#pragma unroll
                    for (int off = 32; off; off >>= 1) first = min(first, __shfl_xor(first, off, 64));
                }
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const int channel = 16 * (c >> 2) + 4 * g + (c & 3), from = min(first, Marks::first(marks.channel(turn, SWAP)[channel], number));
                    if (a < nt && a >= from && v0 + channel < D) *(uint16_t*)((char*)out_at.at + out_off + 32 * (c >> 2) + 2 * (c & 3)) = 0x7FC0;      // NaN in both types
                    if (GRAD == 2 && from < kChunk) du[c] = Marks::nan();
                }
            }
            if (GRAD) dw = (double)Marks::nan();
        }
        out_at.pass(nt);
        if (L::two) turn ^= 1, buffer = lds + turn * L::buffer;
        else __syncthreads();
        ++number;
    };
    for (int left = at.len; left > 0;) {
        const int next = min(kChunk, left - nt);
        chunk(nt, next, left);
        left -= nt;
        nt = next;
    }
    return dw;
}

// Where a workgroup is; false if it has nothing to do.
__device__ __forceinline__ bool find_place(Place& at, const HeadsDev& h, int cut, int blocks, int* found, const Marks& marks) {
    const int tid = threadIdx.x;
    at.slot_at = blockIdx.x / (h.H * blocks); at.head = blockIdx.x / blocks % h.H; at.v0 = blockIdx.x % blocks * kVals; at.D = h.D;
    at.lane = tid & 63; at.wave = __builtin_amdgcn_readfirstlane(tid >> 6); at.n = at.lane & 15; at.g = at.lane >> 4;
    if (tid == 0) *found = -1;
    marks.clear(tid);
    __syncthreads();
    at.s = segment_of(h, cut, at.slot_at, found);
    at.slot = at.s.idx < at.s.count ? slot_of(h, at.s.b) : -1;
    if (at.slot < 0) return false;
    at.len = at.s.a1 - at.s.a0;
    at.w = decay_of(h, at.head);
    return true;
}
// A workgroup's parts of dw, and of du from four of its wavefronts (`which`: 0 .. 3, or -1).
template <int WAVES, bool DU>
__device__ __forceinline__ void leave_sums(const HeadsDev& h, const SweepsDev& all, const Place& at, int half, double dw, const float* du, int which, char* lds) {
    double* const each = (double*)lds;
    float* const across = (float*)(each + 12);
#pragma unroll
    for (int off = 32; off; off >>= 1) dw += __shfl_xor(dw, off, 64);
    if (at.lane == 0) each[at.wave] = dw;
    if constexpr (DU) {
        if (which >= 0)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float sum = du[i];
#pragma unroll
                for (int off = 8; off; off >>= 1) sum += __shfl_xor(sum, off, 64);
                if (at.n == 0) across[kVals * which + 16 * (i >> 2) + 4 * at.g + (i & 3)] = sum;
            }
    }
    __syncthreads();
    const int tid = threadIdx.x;
    if (DU && tid < kVals && at.v0 + tid < at.D)
        all.du_parts[((size_t)at.slot_at * h.H + at.head) * at.D + at.v0 + tid] = across[tid] + across[kVals + tid] + across[2 * kVals + tid] + across[3 * kVals + tid];
    if (tid == 0) {
        double sum = 0.0;
        for (int i = 0; i < WAVES; ++i) sum += each[i];
        all.dw_parts[((size_t)at.slot_at * h.H + at.head) * 4 + 2 * half + at.v0 / kVals] = -sum;
    }
}
// The same of one that has nothing to do.
template <bool DU>
__device__ __forceinline__ void leave_zeros(const HeadsDev& h, const SweepsDev& all, const Place& at, int half) {
    const int tid = threadIdx.x;
    if (DU && tid < kVals && at.v0 + tid < at.D) all.du_parts[((size_t)at.slot_at * h.H + at.head) * at.D + at.v0 + tid] = 0.0f;
    if (tid == 0) all.dw_parts[((size_t)at.slot_at * h.H + at.head) * 4 + 2 * half + at.v0 / kVals] = 0.0;
}

// One sweep: four wavefronts for the outputs, four for the state, which meet at the same barriers.  Forward, 8192 tokens of 64 heads of 64: 66 us in
// bf16, 97 in fp16, whose values are two parts.
template <int DP, bool BF16, int GRAD>
__device__ __forceinline__ void sweep(const HeadsDev& h, const SweepsDev& all, const SweepDev& p, int cut, int scanned, int blocks, int* found, char* lds) {
    typedef Lds<DP, BF16, GRAD> L;
    Place at;
    if (!find_place(at, h, cut, blocks, found, Marks(lds + L::marks))) {
        if constexpr (GRAD != 0) leave_zeros<GRAD == 2>(h, all, at, GRAD - 1);
        return;
    }
    float du[GRAD == 2 ? 16 : 1] = {};
    const double dw = at.wave < 4 ? outputs<DP, BF16, L, GRAD, true, false, GRAD == 0>(h, p, at, at.wave, du, lds)
                                  : carry_state<DP, BF16, L>(h, p, all, at, cut, scanned != 0, lds);
    if constexpr (GRAD != 0) leave_sums<8, GRAD == 2>(h, all, at, GRAD - 1, dw, du, at.wave < 4 ? at.wave : -1, lds + L::sums);
}
template <int DP, bool BF16>
__global__ void __launch_bounds__(512, DP > 64 ? 2 : 4) attend_forward_kernel(HeadsDev h, SweepsDev all, int cut, int scanned, int blocks) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int found;
    sweep<DP, BF16, 0>(h, all, all.sweep[0], cut, scanned, blocks, &found, lds);
}

// Heads of up to 64 channels, backward: twelve wavefronts around one state, of which eight read the tiles.  DK: the sweeps for dv and dk
// in one (their states are each other's transpose, their scores come from the same two tiles); otherwise the sweep for dr, whose second set of
// wavefronts has N's shares of dw and those of pairs of one chunk (all shares in one set: 154 us instead of 140).  4 sequences of 2048 tokens, 64 heads
// of 64, bf16: 128 us for dr, 134 for dk and dv (fp16: 171 and 169).
template <bool BF16, bool DK>
__device__ __forceinline__ void pair(const HeadsDev& h, const SweepsDev& all, int cut, int scanned, int* found, char* lds) {
    typedef Lds<64, BF16, 0, true, DK> L;
    Place at;
    if (!find_place(at, h, cut, 1, found, Marks(lds + L::marks))) {
        leave_zeros<DK>(h, all, at, DK);
        return;
    }
    float du[DK ? 16 : 1] = {}, none[1];
    const SweepDev& p = all.sweep[DK ? 2 : 0];
    const double dw = at.wave < 4   ? outputs<64, BF16, L, DK ? 0 : 1, true, false, DK>(h, p, at, at.wave, none, lds)
                      : at.wave < 8 ? carry_state<64, BF16, L>(h, p, all, at, cut, scanned != 0, lds)
                      : DK          ? outputs<64, BF16, L, DK ? 2 : 1, DK, DK, false>(h, all.sweep[1], at, at.wave - 8, du, lds)
                                    : outputs<64, BF16, L, DK ? 2 : 1, DK, DK, false>(h, p, at, at.wave - 8, du, lds);
    leave_sums<12, DK>(h, all, at, DK, dw, du, at.wave >= 8 ? at.wave - 8 : -1, lds + L::sums);
}

// The sweeps of the backward pass need nothing of each other.  KIND 0: dr;
// 1: dk and dv; kEach: all, the longest first (five ragged sequences of 1001 tokens, 16 heads of 128, fp16: 66 us; as two launches 41 + 40).  WHOLE: heads of
// exactly 128 channels, whose places are all in use, which takes conditions out of a kernel that has too few registers (65 -> 61 us; that of 64 channels
// gains nothing by it, 138 to 158 us with and without, the forward sweep neither).
constexpr int kEach = 3;
template <bool BF16, int KIND>
__global__ void __launch_bounds__(768, 3) attend_pair_kernel(HeadsDev h, SweepsDev all, int cut, int scanned) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int found;
    if (KIND == 1 || (KIND == kEach && blockIdx.y == 0)) pair<BF16, true>(h, all, cut, scanned, &found, lds);
    else pair<BF16, false>(h, all, cut, scanned, &found, lds);
}
template <bool BF16, int KIND, bool WHOLE>
__global__ void __launch_bounds__(512, 2) attend_backward_kernel(HeadsDev h, SweepsDev all, int cut, int scanned) {
    if (WHOLE) h.D = 128;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int found;
    if (KIND == 0 || (KIND == kEach && blockIdx.y == 0)) sweep<128, BF16, 1>(h, all, all.sweep[0], cut, scanned, 2, &found, lds);
    else if (blockIdx.y == (KIND == kEach)) sweep<128, BF16, 2>(h, all, all.sweep[1], cut, scanned, 2, &found, lds);
    else sweep<128, BF16, 0>(h, all, all.sweep[2], cut, scanned, 2, &found, lds);
}

// du [H][D] from its parts [slots][H][D], dw [H] from [slots][H][4], of which `blocks` are used in each half: sixteen threads an entry, in a
// fixed order.
__global__ void __launch_bounds__(256) attend_sum_kernel(HeadsDev h, const float* du_parts, const double* dw_parts, int slots, int blocks) {
    __shared__ double lds[16][17];
    const int i = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4, n_du = h.H * h.D;
    double s = 0.0;
    if (i < n_du) {
        float f = 0.0f;
        for (int p = part; p < slots; p += 16) f += du_parts[(size_t)p * n_du + i];
        s = (double)f;
    } else if (i < n_du + h.H) {
        for (int p = part; p < slots; p += 16) {
            const double* const at = dw_parts + ((size_t)p * h.H + i - n_du) * 4;
            for (int b = 0; b < blocks; ++b) s += at[b] + at[2 + b];
        }
    }
    lds[part][threadIdx.x & 15] = s;
    __syncthreads();
    if (part != 0) return;
    for (int p = 1; p < 16; ++p) s += lds[p][threadIdx.x];
    if (i < n_du) h.du[i] = (float)s;
    else if (i < n_du + h.H) h.dw[i - n_du] = (float)s;
}

// How a call is cut: `cut` tokens a segment, `slots` segments at most; split: a sequence can have more than one; scan: one launch turns
// the segments' parts into the states in front of them, otherwise each segment adds up those before it.
// Segments are as long as the device stays full.  Forward two workgroups fit a unit: 512 in all (8192 tokens of 64 heads: shorter segments for 1024 are slower,
// the pass in front has more to do); ragged sequences that are more than that by themselves end at different times, and shorter segments even
// that out (sixteen of 1 to 1184 tokens, 80 heads: 98 us for 512, 92 for 1024, 101 and a scan for 2048; four sequences of 32 heads 24 against 32).
// Backward one workgroup fits: 256, and no pass in front where sequences are as many by themselves (4 x 2048 tokens x 64 heads: 245 us
// against 294 for 512); above 64 channels the three sweeps are one launch, and 128 (75 us against 92).  No segment is shorter than 128 tokens, two
// chunks (256: 800 tokens of 16 heads 19 us instead of 16), but what fits 256 is not cut (224 tokens: 13 us in one segment, 15 in two).
// Backward none is longer than 2048 (16384 tokens of 40 heads of 128: 1395 us against 1829 for a segment a workgroup; 32768 of 64 heads of 64: 1354
// against 1221).
// A scan pays from 17 segments on: 14 segments 28 us without, 25 + 6 and a launch with it; 26 42 against 30 + 7; 32, backward, 63 against 41 + 7.
struct Plan { int cut, slots, blocks, part_size, longest; bool split, scan; size_t part_floats, du_floats, dw_doubles; };
static Plan plan_of(const HeadsDev& h, bool grad) {
    Plan p;
    p.blocks = (h.D + kVals - 1) / kVals;
    const long long work = (long long)h.n_tokens * h.H * p.blocks;
    const int len = h.offsets ? h.n_tokens : h.n_tokens / h.n_seqs;
    p.cut = (int)std::max(128ll, (work / (!grad ? (h.offsets && (long long)h.n_seqs * h.H * p.blocks > 512 ? 1024 : 512) : h.D > 64 ? 128 : 256) + kChunk - 1) / kChunk * kChunk);
    if (grad) p.cut = std::min(p.cut, 2048);
    if (len <= 256) p.cut = std::max(p.cut, 256);
    p.split = len > p.cut;
    p.slots = h.offsets ? h.n_tokens / p.cut + h.n_seqs : h.n_seqs * ((len + p.cut - 1) / p.cut);
    p.scan = len / p.cut > 16;
    p.part_size = (h.D <= 64 ? 64 : 128) * kVals * p.blocks;
    p.longest = std::min(len, p.cut);
    p.part_floats = p.split ? (size_t)p.slots * h.H * p.part_size : 0;
    p.dw_doubles = (size_t)p.slots * h.H * 4;
    p.du_floats = (size_t)p.slots * h.H * h.D;
    return p;
}
static bool single_tokens(const HeadsDev& h) { return !h.offsets && h.n_tokens == h.n_seqs; }

// A launch holds fewer than 2^32 threads along x: 256 for a token's step of a head, 512 or 768 for a segment.
bool attention_fits(const HeadsDev& h, bool grad) {
    const Plan p = plan_of(h, grad);
    const unsigned long long groups = !grad && single_tokens(h) ? (unsigned long long)h.n_seqs * h.H : (unsigned long long)p.slots * h.H * p.blocks;
    return groups * (!grad ? (single_tokens(h) ? 256 : 512) : h.D > 64 ? 512 : 768) < 1ull << 32;
}

size_t attention_workspace_bytes(const HeadsDev& h) { return single_tokens(h) ? 0 : plan_of(h, false).part_floats * sizeof(float); }
size_t attention_backward_workspace_bytes(const HeadsDev& h) {
    const Plan p = plan_of(h, true);
    return (2 * p.part_floats + p.du_floats) * sizeof(float) + p.dw_doubles * sizeof(double);
}

template <int DP, bool BF16, int DIRS>
static hipError_t launch_locals(const HeadsDev& h, const LocalsDev& l, const Plan& p, hipStream_t s) {
    if (!p.split) return hipSuccess;
    hipLaunchKernelGGL((attend_local_kernel<DP, BF16, DIRS>), dim3((unsigned)(p.slots * h.H * p.blocks), DIRS), dim3(256), 0, s, h, l, p.cut, p.blocks);
    if (p.scan)
        hipLaunchKernelGGL(attend_scan_kernel, dim3((unsigned)std::min(65536ll, (long long)h.n_seqs * h.H), (p.part_size + 255) / 256, DIRS), dim3(256), 0, s, h, l, p.cut, p.part_size);
    return hipGetLastError();
}
template <bool BF16, int KIND>
static hipError_t launch_pair(const HeadsDev& h, const SweepsDev& all, const Plan& p, hipStream_t s) {
    static std::atomic<unsigned long long> raised{0};
    constexpr int bytes = std::max(Lds<64, BF16, 0, true, false>::bytes, Lds<64, BF16, 0, true, true>::bytes);
    const hipError_t e = raise_lds((const void*)attend_pair_kernel<BF16, KIND>, bytes, raised);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attend_pair_kernel<BF16, KIND>), dim3((unsigned)(p.slots * h.H), KIND == kEach ? 2 : 1), dim3(768), bytes, s, h, all, p.cut, (int)p.scan);
    return hipGetLastError();
}
template <bool BF16, int KIND, bool WHOLE>
static hipError_t launch_wide(const HeadsDev& h, const SweepsDev& all, const Plan& p, hipStream_t s) {
    static std::atomic<unsigned long long> raised{0};
    constexpr int bytes = std::max(std::max(Lds<128, BF16, 0>::bytes, Lds<128, BF16, 1>::bytes), Lds<128, BF16, 2>::bytes);
    const hipError_t e = raise_lds((const void*)attend_backward_kernel<BF16, KIND, WHOLE>, bytes, raised);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attend_backward_kernel<BF16, KIND, WHOLE>), dim3((unsigned)(p.slots * h.H * 2), KIND == kEach ? 3 : KIND + 1), dim3(512), bytes, s, h, all, p.cut, (int)p.scan);
    return hipGetLastError();
}
template <int DP, bool BF16>
static hipError_t forward(const HeadsDev& h, hipStream_t s) {
    const Plan p = plan_of(h, false);
    LocalsDev l{};
    l.dir[0] = LocalDev{h.k, h.v, h.k_stride, h.v_stride, h.state, h.partial, false, false};
    const hipError_t e = launch_locals<DP, BF16, 1>(h, l, p, s);
    if (e != hipSuccess) return e;
    SweepsDev all{};
    all.sweep[0] = SweepDev{h.r, h.k, h.v, nullptr, h.r_stride, h.k_stride, h.v_stride, h.out_stride, 0, h.out, h.state, h.partial, h.state_out, false, false, false};
    static std::atomic<unsigned long long> raised{0};
    constexpr int bytes = Lds<DP, BF16, 0>::bytes;
    const hipError_t r = raise_lds((const void*)attend_forward_kernel<DP, BF16>, bytes, raised);
    if (r != hipSuccess) return r;
    hipLaunchKernelGGL((attend_forward_kernel<DP, BF16>), dim3((unsigned)(p.slots * h.H * p.blocks)), dim3(512), bytes, s, h, all, p.cut, (int)p.scan, p.blocks);
    return hipGetLastError();
}
template <int DP, bool BF16, bool WHOLE>
static hipError_t backward(const HeadsDev& h, hipStream_t s) {
    const Plan p = plan_of(h, true);
    double* const dw_parts = (double*)h.partial;
    float *const S = (float*)(dw_parts + p.dw_doubles), *const G = S + p.part_floats, *const du_parts = G + p.part_floats;
    LocalsDev l{};
    l.dir[0] = LocalDev{h.v, h.k, h.v_stride, h.k_stride, h.state, S, false, true};
    l.dir[1] = LocalDev{h.r, h.dout, h.r_stride, h.out_stride, h.dstate, G, true, false};
    hipError_t e = launch_locals<DP, BF16, 2>(h, l, p, s);
    if (e != hipSuccess) return e;
    SweepsDev all{};
    all.sweep[0] = SweepDev{h.dout, h.v, h.k, h.r, h.out_stride, h.v_stride, h.k_stride, h.r_stride, h.r_stride, h.dr, h.state, S, nullptr, false, true, false};
    all.sweep[1] = SweepDev{h.v, h.dout, h.r, h.k, h.v_stride, h.out_stride, h.r_stride, h.k_stride, h.k_stride, h.dk, h.dstate, G, nullptr, true, true, true};
    all.sweep[2] = SweepDev{h.k, h.r, h.dout, nullptr, h.k_stride, h.r_stride, h.out_stride, h.v_stride, 0, h.dv, h.dstate, G, h.dstate_in, true, false, false};
    all.grad_initial = h.dstate; all.grad_parts = G; all.du_parts = du_parts; all.dw_parts = dw_parts;
    if constexpr (DP == 64) {
        // both kinds at once, and a launch less, for at most 512 workgroups and 512 tokens each: 400 tokens of 16 heads 17 us instead of 29.  More and
        // longer ones are better apart, the kernel that has both has too few registers (512 in all, 2048 tokens each: 291 us instead of 258).
        if (p.longest <= 512 && p.slots * h.H <= 256) {
            e = launch_pair<BF16, kEach>(h, all, p, s);
        } else {
            e = launch_pair<BF16, 0>(h, all, p, s);
            if (e == hipSuccess) e = launch_pair<BF16, 1>(h, all, p, s);
        }
        if (e != hipSuccess) return e;
    } else {
        // likewise: segments of 128 tokens 66 us instead of 81 (above), of 2048 tokens (4 sequences, 32 heads of 128) 423 instead of 413
        if (p.longest <= 256) {
            e = launch_wide<BF16, kEach, WHOLE>(h, all, p, s);
        } else {
            e = launch_wide<BF16, 0, WHOLE>(h, all, p, s);
            if (e == hipSuccess) e = launch_wide<BF16, 1, WHOLE>(h, all, p, s);
        }
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(attend_sum_kernel, dim3((h.H * (h.D + 1) + 15) / 16), dim3(256), 0, s, h, du_parts, dw_parts, p.slots, p.blocks);
    return hipGetLastError();
}
template <bool BF16>
static hipError_t attention(const HeadsDev& h, bool grad, hipStream_t s) {
    if (grad)
        return h.D <= 64 ? backward<64, BF16, false>(h, s) : h.D == 128 ? backward<128, BF16, true>(h, s) : backward<128, BF16, false>(h, s);
    if (!single_tokens(h)) return h.D <= 64 ? forward<64, BF16>(h, s) : forward<128, BF16>(h, s);
    const dim3 grid((unsigned)(h.n_seqs * h.H)), block(256);
    if (h.D <= 32) hipLaunchKernelGGL((attend_step_kernel<8, 1, BF16>), grid, block, 0, s, h);
    else if (h.D <= 64) hipLaunchKernelGGL((attend_step_kernel<16, 4, BF16>), grid, block, 0, s, h);
    else hipLaunchKernelGGL((attend_step_kernel<32, 16, BF16>), grid, block, 0, s, h);
    return hipGetLastError();
}
hipError_t launch_attention(const HeadsDev& h, int dt, hipStream_t s) {
    return dt == DT_BF16 ? attention<true>(h, false, s) : attention<false>(h, false, s);
}
hipError_t launch_attention_backward(const HeadsDev& h, int dt, hipStream_t s) {
    return dt == DT_BF16 ? attention<true>(h, true, s) : attention<false>(h, true, s);
}

}  // namespace rwkvq
