// Dropout with a mask that is drawn again wherever it is needed (philox.h), added to a residual: out = residual + drop(in).  The
// gradient of the branch is the same call on the gradient, without the residual.
#pragma clang fp contract(off)

#include "adapters.h"

namespace halo {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 2;       // groups of eight elements per thread, all loads issued before the first is used

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

// A workgroup takes kThreads * kGroups groups of eight elements, row after row; groups: per row.  Row and group of a thread come from one
// division of the workgroup's first index (the same for all its threads) and a 32-bit one.  Workgroups are numbered along x and then y, because
// a dimension of a launch has at most 2^32 - 1 threads: of more, only what is left modulo 2^32 begins, without an error.
template <typename E, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(const E* in, int64_t ld_in, const E* residual, int64_t ld_res, E* out, int64_t ld_out, int64_t rows, uint32_t cols,
               uint32_t groups, DropoutMask d) {
    const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kThreads * kGroups);
    const int64_t row0 = first / groups;
    const uint32_t group0 = (uint32_t)(first - row0 * groups);
    Eight<E> x[kGroups], r[kGroups];
    int64_t row[kGroups];
    uint32_t group[kGroups];
    bool on[kGroups];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        const uint32_t at = group0 + i * kThreads + threadIdx.x, over = at / groups;
        row[i] = row0 + over;
        group[i] = at - over * groups;
        on[i] = row[i] < rows;
        if (on[i]) {
            const uint32_t c = group[i] * 8;
            x[i].load(in + row[i] * ld_in + c, c + 4 < cols);
            if (RESIDUAL) r[i].load(residual + row[i] * ld_res + c, c + 4 < cols);
        }
    }
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        if (!on[i]) continue;
        const uint4 bits = dropout_bits(d, (uint32_t)row[i], group[i]);
        const uint32_t c = group[i] * 8;
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = dropout_kept(d, bits, j) ? x[i].get(j) * d.factor : 0.0f;
            if (RESIDUAL) y[j] += r[i].get(j);
        }
        E* o = out + row[i] * ld_out + c;
        if (c + 8 <= cols) {
            Eight<E>::store(o, y);
        } else {                           // the end of a row: what lies behind it is not the caller's
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (c + j < cols) Eight<E>::store_one(o + j, y[j]);
        }
    }
}

template <typename E>
hipError_t launch_typed(const DropoutArgs& a, hipStream_t s) {
    const int64_t groups = (a.cols + 7) / 8, per = kThreads * kGroups, blocks = (a.rows * groups + per - 1) / per;
    constexpr int64_t kAlongX = 1 << 20;                 // 2^28 threads; with the most rows and columns, 2^12 of them along y
    const dim3 grid((unsigned)(blocks < kAlongX ? blocks : kAlongX), (unsigned)((blocks + kAlongX - 1) / kAlongX));
    const E *in = reinterpret_cast<const E*>(a.in), *res = reinterpret_cast<const E*>(a.residual);
    E* out = reinterpret_cast<E*>(a.out);
    if (res)
        hipLaunchKernelGGL((dropout_kernel<E, true>), grid, dim3(kThreads), 0, s, in, a.ld_in, res, a.ld_res, out,
                           a.ld_out, a.rows, (uint32_t)a.cols, (uint32_t)groups, a.drop);
    else
        hipLaunchKernelGGL((dropout_kernel<E, false>), grid, dim3(kThreads), 0, s, in, a.ld_in, res, a.ld_res, out,
                           a.ld_out, a.rows, (uint32_t)a.cols, (uint32_t)groups, a.drop);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s) {
    if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
    return a.f32 ? launch_typed<float>(a, s) : launch_typed<uint16_t>(a, s);
}

}  // namespace halo
