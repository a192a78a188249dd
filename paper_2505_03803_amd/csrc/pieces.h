// Values of any of the three types, one at a time or 16 bytes of them.
#pragma once
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

// V values of a row, 16 bytes of them (V > 1) or one.
template <int DT_, int V> struct Piece;
template <int DT_> struct Piece<DT_, 1> {
    typename Type<DT_>::raw v;
    __device__ __forceinline__ void clear() { v = 0; }
    __device__ __forceinline__ void load(const void* p, long long i) { v = ((const typename Type<DT_>::raw*)p)[i]; }
    __device__ __forceinline__ void widen(float (&f)[1]) const { f[0] = Type<DT_>::widen(v); }
    static __device__ __forceinline__ void store(void* p, long long i, const float (&f)[1]) { ((typename Type<DT_>::raw*)p)[i] = Type<DT_>::narrow(f[0]); }
};
template <> struct Piece<DT_F32, 4> {
    float4_t v;
    __device__ __forceinline__ void clear() { v = float4_t{0, 0, 0, 0}; }
    __device__ __forceinline__ void load(const void* p, long long i) { v = *(const float4_t*)((const float*)p + i); }
    __device__ __forceinline__ void widen(float (&f)[4]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = v[j];
    }
    static __device__ __forceinline__ void store(void* p, long long i, const float (&f)[4]) { *(float4_t*)((float*)p + i) = float4_t{f[0], f[1], f[2], f[3]}; }
};
template <int DT_> struct Piece<DT_, 8> {
    uint4_t v;
    __device__ __forceinline__ void clear() { v = uint4_t{0, 0, 0, 0}; }
    __device__ __forceinline__ void load(const void* p, long long i) { v = *(const uint4_t*)((const uint16_t*)p + i); }
    __device__ __forceinline__ void widen(float (&f)[8]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t w = v[j];
            f[2 * j] = Type<DT_>::widen((uint16_t)w); f[2 * j + 1] = Type<DT_>::widen((uint16_t)(w >> 16));
        }
    }
    static __device__ __forceinline__ void store(void* p, long long i, const float (&f)[8]) {
        uint4_t o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = (uint32_t)Type<DT_>::narrow(f[2 * j]) | ((uint32_t)Type<DT_>::narrow(f[2 * j + 1]) << 16);
        *(uint4_t*)((uint16_t*)p + i) = o;
    }
};
// Eight neighbouring values from place i on as binary32, `left` of them if fewer are in the row (the others are 0); `whole`: 16 bytes at a time.
template <int DT_>
__device__ __forceinline__ void load8(float (&f)[8], const void* p, long long i, int left, bool whole) {
    if (whole && left >= 8) {
        if constexpr (DT_ == DT_F32) {
            const float4_t a = *(const float4_t*)((const float*)p + i), b = *(const float4_t*)((const float*)p + i + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { f[j] = a[j]; f[4 + j] = b[j]; }
        } else {
            Piece<DT_, 8> v;
            v.load(p, i);
            v.widen(f);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = j < left ? Type<DT_>::widen(((const typename Type<DT_>::raw*)p)[i + j]) : 0.0f;
}
template <int DT_>
__device__ __forceinline__ void store8(void* p, long long i, const float (&f)[8], int left, bool whole) {
    if (whole && left >= 8) {
        if constexpr (DT_ == DT_F32) {
            *(float4_t*)((float*)p + i) = float4_t{f[0], f[1], f[2], f[3]};
            *(float4_t*)((float*)p + i + 4) = float4_t{f[4], f[5], f[6], f[7]};
        } else {
            Piece<DT_, 8>::store(p, i, f);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) ((typename Type<DT_>::raw*)p)[i + j] = Type<DT_>::narrow(f[j]);
}

// Work items that lie in rows of `across` of them: the item a thread begins with, and its next ones `step` items on without another division.
struct RowWalk {
    uint32_t row, at, across, rows_on, on;
    __device__ __forceinline__ RowWalk(uint32_t first, uint32_t across_, uint32_t step)
        : row(first / across_), at(first % across_), across(across_), rows_on(step / across_), on(step % across_) {}
    __device__ __forceinline__ void next() {
        row += rows_on; at += on;
        if (at >= across) { at -= across; ++row; }
    }
};

}  // namespace rwkvq
