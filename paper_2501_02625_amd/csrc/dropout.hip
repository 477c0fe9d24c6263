// Dropout with a mask that is drawn again wherever it is needed (philox.h), added to a residual: out = residual + drop(in).  The
// gradient of the branch is the same call on the gradient, without the residual.
#pragma clang fp contract(off)

#include "adapters.h"

namespace halo {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load_as_f32(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float load_as_f32(const float* p) { return *p; }

__device__ __forceinline__ void store_from_f32(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_from_f32(uint16_t* p, float x) { *p = __builtin_bit_cast(uint16_t, (__bf16)x); }

// A thread per group of eight elements of a row.
template <typename E>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(const E* in, int64_t ld_in, const E* residual, int64_t ld_res, E* out, int64_t ld_out, int64_t rows, int64_t cols,
               int64_t groups, DropoutMask d) {
    const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (idx >= rows * groups) return;
    const int64_t row = idx / groups, group = idx % groups;
    const uint4 bits = dropout_bits(d, (uint32_t)row, (uint32_t)group);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t c = group * 8 + j;
        if (c >= cols) break;
        float y = dropout_kept(d, bits, j) ? load_as_f32(in + row * ld_in + c) * d.factor : 0.0f;
        if (residual) y += load_as_f32(residual + row * ld_res + c);
        store_from_f32(out + row * ld_out + c, y);
    }
}

template <typename E>
void launch_typed(const DropoutArgs& a, hipStream_t s) {
    const int64_t groups = (a.cols + 7) / 8, blocks = (a.rows * groups + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(dropout_kernel<E>, dim3((unsigned)blocks), dim3(kThreads), 0, s, reinterpret_cast<const E*>(a.in), a.ld_in,
                       reinterpret_cast<const E*>(a.residual), a.ld_res, reinterpret_cast<E*>(a.out), a.ld_out, a.rows, a.cols,
                       groups, a.drop);
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s) {
    if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
    if ((a.rows * ((a.cols + 7) / 8) + kThreads - 1) / kThreads > 0x7FFFFFFF) return hipErrorInvalidValue;
    if (a.f32) launch_typed<float>(a, s);
    else launch_typed<uint16_t>(a, s);
    return hipGetLastError();
}

}  // namespace halo
