// Eight consecutive elements of a row, bf16 or fp32, as they are in memory and as fp32 values: what a lane loads and stores at a time.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace halo {

// Eight consecutive elements as they are in memory.
template <typename E> struct Eight;
template <> struct Eight<uint16_t> {
    uint4 q;
    __device__ __forceinline__ void load(const uint16_t* p, bool) { q = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ float get(int j) const {
        const uint32_t w = j < 2 ? q.x : j < 4 ? q.y : j < 6 ? q.z : q.w;
        return __uint_as_float((j & 1) ? w & 0xFFFF0000u : w << 16);
    }
    __device__ __forceinline__ static uint16_t bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
    __device__ __forceinline__ static void store(uint16_t* p, const float* y) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (uint32_t)bits(y[2 * i]) | (uint32_t)bits(y[2 * i + 1]) << 16;
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ static void store_one(uint16_t* p, float y) { *p = bits(y); }
};
template <> struct Eight<float> {
    float4 lo, hi;
    // second: the row has elements in the upper half (its pitch is a multiple of four only)
    __device__ __forceinline__ void load(const float* p, bool second) {
        lo = *reinterpret_cast<const float4*>(p);
        hi = second ? *reinterpret_cast<const float4*>(p + 4) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    __device__ __forceinline__ float get(int j) const {
        const float4& q = j < 4 ? lo : hi;
        return (j & 3) == 0 ? q.x : (j & 3) == 1 ? q.y : (j & 3) == 2 ? q.z : q.w;
    }
    __device__ __forceinline__ static void store(float* p, const float* y) {
        *reinterpret_cast<float4*>(p) = make_float4(y[0], y[1], y[2], y[3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(y[4], y[5], y[6], y[7]);
    }
    __device__ __forceinline__ static void store_one(float* p, float y) { *p = y; }
};

}  // namespace halo
