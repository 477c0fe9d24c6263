// The gradient of the epilogue of a product (halo_activation_bwd): E_Z = E act'(Z), and the bias' gradient, its column sums.
#pragma clang fp contract(off)

#include "activation.h"
#include "around.h"
#include "eight.h"

namespace halo {
namespace {

constexpr int kThreads = 256;

template <typename E>
__device__ __forceinline__ float widen(E x) {
    if constexpr (sizeof(E) == 2) return __uint_as_float((uint32_t)x << 16);
    else return x;
}

// One thread a column of one part of the rows.
template <typename E, int ACT>
__global__ void __launch_bounds__(kThreads) act_grad_kernel(ActGrad a, int64_t rows_per_part) {
    const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.cols) return;
    const int64_t r0 = blockIdx.y * rows_per_part, r1 = r0 + rows_per_part < a.rows ? r0 + rows_per_part : a.rows;
    float sum = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        const float e = widen(reinterpret_cast<const E*>(a.E)[r * a.ld_e + c]);
        const float z = ACT == HALO_ACT_NONE ? 0.0f : widen(reinterpret_cast<const E*>(a.Z)[r * a.ld_z + c]);
        const float d = activation_slope<ACT>(e, z);
        if (a.EZ) Eight<E>::store_one(reinterpret_cast<E*>(a.EZ) + r * a.ld_ez + c, d);
        sum += d;
    }
    if (a.GB) a.part[blockIdx.y * a.cols + c] = sum;
}

int64_t parts_of(int64_t rows) { return rows < 64 ? rows : 64; }

template <typename E, int ACT>
hipError_t launch_typed(const ActGrad& a, hipStream_t s) {
    const int64_t most = parts_of(a.rows), per = most ? (a.rows + most - 1) / most : 1, parts = (a.rows + per - 1) / per;
    if (parts)
        hipLaunchKernelGGL((act_grad_kernel<E, ACT>), dim3((unsigned)((a.cols + kThreads - 1) / kThreads), (unsigned)parts), dim3(kThreads), 0,
                           s, a, per);
    if (a.GB) return launch_sum_parts(a.part, a.GB, nullptr, nullptr, parts, a.cols, s);
    return hipGetLastError();
}
template <typename E>
hipError_t launch_act(const ActGrad& a, hipStream_t s) {
    switch (a.act) {
        case HALO_ACT_RELU: return launch_typed<E, HALO_ACT_RELU>(a, s);
        case HALO_ACT_GELU: return launch_typed<E, HALO_ACT_GELU>(a, s);
        case HALO_ACT_GELU_TANH: return launch_typed<E, HALO_ACT_GELU_TANH>(a, s);
        case HALO_ACT_SILU: return launch_typed<E, HALO_ACT_SILU>(a, s);
        default: return launch_typed<E, HALO_ACT_NONE>(a, s);
    }
}

// 64 columns a workgroup, 16 threads a column, each every 16th part; the sixteen sums meet in LDS.
__global__ void __launch_bounds__(1024) sum_parts_kernel(const float* part, float* out, const float* part2, float* out2, int64_t parts,
                                                         int64_t cols) {
    __shared__ float s[16][64];
    if (blockIdx.y) {
        part = part2;
        out = out2;
    }
    const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int at = threadIdx.x >> 6;
    float t = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int64_t p = at; p < parts; p += 16) t += part[p * cols + c];
    }
    s[at][threadIdx.x & 63] = t;
    __syncthreads();
    if (at || c >= cols) return;
    t = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += s[i][threadIdx.x];
    out[c] = t;
}

}  // namespace

size_t act_grad_workspace_floats(int64_t rows, int64_t cols) { return (size_t)parts_of(rows) * (size_t)cols; }

hipError_t launch_act_grad(const ActGrad& a, hipStream_t s) { return a.f32 ? launch_act<float>(a, s) : launch_act<uint16_t>(a, s); }

hipError_t launch_sum_parts(const float* part, float* out, const float* part2, float* out2, int64_t parts, int64_t cols, hipStream_t s) {
    if (!out) {
        out = out2;
        part = part2;
        out2 = nullptr;
    }
    hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)((cols + 63) / 64), out2 ? 2 : 1), dim3(1024), 0, s, part, out, part2, out2, parts, cols);
    return hipGetLastError();
}

}  // namespace halo
