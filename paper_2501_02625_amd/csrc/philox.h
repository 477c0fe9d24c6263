// Dropout masks from a counter-based generator: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", 2011).  A mask is a function of (seed, offset, row, column) alone, so it need not be kept from the forward pass: the backward
// pass draws it again (that of the adapters once, for two kernels: a bit an element in its workspace).
//
// One call gives the 8 x 16 random bits of eight consecutive elements of a row: the counter is (column / 8, row, offset low, offset
// high), the key (seed low, seed high), and element j takes half j % 2 (the low one first) of word (j % 8) / 2.  The element is kept
// where its bits are at least `least` = rint(65536 p); the kept ones are multiplied by 65536 / (65536 - least), which makes the mean
// exact for the probability that is really drawn.  Sixteen bits an element rather than 32 halve the rounds: they, not memory, would
// bound the kernels otherwise (ten rounds are twenty 32 x 32 -> 64 bit products, each at a quarter of the rate of an add).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace halo {

struct DropoutMask {
    uint32_t least;              // 0: everything is kept (no mask), 65536: nothing is
    float factor;                // 65536 / (65536 - least), or 0
    uint32_t key0, key1;
    uint32_t offset0, offset1;
};

inline DropoutMask make_dropout_mask(double p, uint64_t seed, uint64_t offset) {
    DropoutMask d{};
    d.least = (uint32_t)__builtin_rint(p * 65536.0);
    d.factor = d.least < 65536 ? (float)(65536.0 / (65536.0 - d.least)) : 0.0f;
    d.key0 = (uint32_t)seed; d.key1 = (uint32_t)(seed >> 32);
    d.offset0 = (uint32_t)offset; d.offset1 = (uint32_t)(offset >> 32);
    return d;
}

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// The random bits of elements 8 group .. 8 group + 7 of `row`.
__device__ __forceinline__ uint4 dropout_bits(const DropoutMask& d, uint32_t row, uint32_t group) {
    uint32_t c0 = group, c1 = row, c2 = d.offset0, c3 = d.offset1, k0 = d.key0, k1 = d.key1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = xor3((uint32_t)(p1 >> 32), c1, k0);
        c1 = (uint32_t)p1;
        c2 = xor3((uint32_t)(p0 >> 32), c3, k1);
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

__device__ __forceinline__ bool dropout_kept(const DropoutMask& d, const uint4& bits, int j) {
    const uint32_t w = j < 2 ? bits.x : j < 4 ? bits.y : j < 6 ? bits.z : bits.w;
    return ((j & 1) ? w >> 16 : w & 0xFFFFu) >= d.least;
}

}  // namespace halo
