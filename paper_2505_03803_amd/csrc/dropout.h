// Dropout whose mask is never stored: which elements stay follows from a seed and from their place.
#pragma once
#include "common.h"

namespace rwkvq {

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
// Philox 4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds, each two products of 32-bit
// words whose halves are exchanged and mixed with the other words and with a key that advances by the golden ratio and by sqrt(3) - 1.
__device__ __forceinline__ uint4_t philox(uint4_t c, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
        c = uint4_t{xor3((uint32_t)(b >> 32), c.y, k0), (uint32_t)b, xor3((uint32_t)(a >> 32), c.w, k1), (uint32_t)a};
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    return c;
}

// seed[0] is the key, seed[1] + call the number of the call, both read when the work runs.  The counter of the eight columns from 8 i on of a row
// is (i, row, number); its four words are eight numbers of 16 bits, the low half of a word first, and a column is dropped where its number is
// below `limit`: one counter for 16 bytes of 16-bit values, so that the generator (20 products of 32 bits, each at a quarter of the
// rate of an addition) stays behind what memory takes.
// What stays, as masks of 16 bits in the order of eight 16-bit values: a number above limit - 1 is all ones.  `limit` is not 0 here.
struct Keeper {
    uint32_t k0, k1, n0, n1, most;                 // most: limit - 1, twice
    Keeper() = default;
    __device__ __forceinline__ explicit Keeper(const Dropout& d) {
        const uint64_t key = d.seed[0], number = d.seed[1] + d.call;
        k0 = (uint32_t)key; k1 = (uint32_t)(key >> 32);
        n0 = (uint32_t)number; n1 = (uint32_t)(number >> 32);
        most = (d.limit - 1) * 0x10001u;
    }
    // columns 8 i .. + 7 of the row
    __device__ __forceinline__ uint4_t masks(uint32_t i, uint32_t row) const {
        uint4_t w = philox(uint4_t{i, row, n0, n1}, k0, k1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t m = w[j];
            // number - most, not below 0; at most 1; 0 - that.  (Written in C this becomes compares and selects, five instructions a word.)
            asm("v_pk_sub_u16 %0, %0, %1 clamp\n\tv_pk_min_u16 %0, %0, %2\n\tv_pk_sub_u16 %0, 0, %0" : "+v"(m) : "s"(most), "v"(0x00010001u));
            w[j] = m;
        }
        return w;
    }
};
// Element j of eight binary32 values under such masks: all of it or 0.
__device__ __forceinline__ float masked(float v, const uint4_t& m, int j) {
    const int32_t whole = j & 1 ? (int32_t)m[j / 2] >> 16 : (int32_t)(m[j / 2] << 16) >> 16;
    return __uint_as_float(__float_as_uint(v) & (uint32_t)whole);
}

}  // namespace rwkvq
