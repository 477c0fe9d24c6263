// The gradient of the epilogue of a product (halo_activation_bwd): E_Z = E act'(Z), and the bias' gradient, its column sums, in one pass.
// What bounds it is memory, and of small matrices the two launches.  8192 x 14336 in bf16 with gelu: 145 us, 4.9 TB/s (a large copy reaches
// 5.1), and 4.5 for the sum over 73 parts of the rows; with two rows of a thread's on their way instead of four 165.
#pragma clang fp contract(off)

#include <type_traits>

#include "activation.h"
#include "around.h"
#include "eight.h"

namespace halo {
namespace {

// A wavefront has 512 columns, eight a lane, or fewer of narrow matrices and then several rows at once; the four of a workgroup have the
// same columns and take turns at the rows of its part.  Their sums meet in LDS and go to `part`, a row for each part.
template <typename E, int ACT, int LANES>
__global__ void __launch_bounds__(256) act_grad_kernel(ActGrad a, int64_t rows_per_part) {
    constexpr int ROWS = 256 / LANES;        // at once
    __shared__ float meet[ROWS][LANES * 8];
    const int lane = threadIdx.x % LANES, at = threadIdx.x / LANES;
    const int64_t c = ((int64_t)blockIdx.x * LANES + lane) * 8, left = a.cols - c;
    const int64_t r0 = blockIdx.y * rows_per_part, r1 = r0 + rows_per_part < a.rows ? r0 + rows_per_part : a.rows;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    auto rows = [&](auto whole) {
#pragma unroll 4
        for (int64_t r = r0 + at; r < r1; r += ROWS) {
            Eight<E> e, z;
            e.load(reinterpret_cast<const E*>(a.E) + r * a.ld_e + c, left > 4);
            z = e;
            if constexpr (ACT != HALO_ACT_NONE) z.load(reinterpret_cast<const E*>(a.Z) + r * a.ld_z + c, left > 4);
            float d[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                d[j] = activation_slope<ACT>(e.get(j), z.get(j));
                sum[j] += d[j];
            }
            if (!a.EZ) continue;
            E* p = reinterpret_cast<E*>(a.EZ) + r * a.ld_ez + c;
            if constexpr (decltype(whole)::value) {
                Eight<E>::store(p, d);
            } else {
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < left) Eight<E>::store_one(p + j, d[j]);
            }
        }
    };
    if (left >= 8) rows(std::true_type());
    else if (left > 0) rows(std::false_type());
    if (!a.GB) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) meet[at][lane * 8 + j] = sum[j];
    __syncthreads();
    for (int i = threadIdx.x; i < LANES * 8; i += 256) {
        const int64_t col = (int64_t)blockIdx.x * LANES * 8 + i;
        if (col >= a.cols) break;
        float t = 0.0f;
#pragma unroll
        for (int k = 0; k < ROWS; ++k) t += meet[k][i];
        a.part[blockIdx.y * a.cols + col] = t;
    }
}

// Parts of the rows: as many as make some two thousand workgroups, with a row for each of their threads at least.  1031 x 1003 in fp32, at
// least one / two / four rows: 5.3 us / 7.2 / 10.6 (and 4.2 for the sum over the parts, whichever).
int lanes_of(int64_t cols) { return cols <= 64 ? 8 : cols <= 128 ? 16 : cols <= 256 ? 32 : 64; }
int64_t parts_of(int64_t rows, int64_t cols) {
    const int lanes = lanes_of(cols);
    const int64_t tiles = (cols + lanes * 8 - 1) / (lanes * 8), at_once = 256 / lanes;
    const int64_t most = tiles < 2048 ? 2048 / tiles : 1, parts = (rows + at_once - 1) / at_once;
    return parts < most ? parts : most;
}

template <typename E, int ACT>
hipError_t launch_typed(const ActGrad& a, hipStream_t s) {
    const int lanes = lanes_of(a.cols);
    const int64_t most = parts_of(a.rows, a.cols), per = most ? (a.rows + most - 1) / most : 1, parts = (a.rows + per - 1) / per;
    if (parts) {
        const dim3 grid((unsigned)((a.cols + lanes * 8 - 1) / (lanes * 8)), (unsigned)parts);
        if (lanes == 8) hipLaunchKernelGGL((act_grad_kernel<E, ACT, 8>), grid, dim3(256), 0, s, a, per);
        else if (lanes == 16) hipLaunchKernelGGL((act_grad_kernel<E, ACT, 16>), grid, dim3(256), 0, s, a, per);
        else if (lanes == 32) hipLaunchKernelGGL((act_grad_kernel<E, ACT, 32>), grid, dim3(256), 0, s, a, per);
        else hipLaunchKernelGGL((act_grad_kernel<E, ACT, 64>), grid, dim3(256), 0, s, a, per);
    }
    if (a.GB) return launch_sum_parts(a.part, a.GB, nullptr, nullptr, parts, a.cols, a.cols, s);
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

// 32 columns a workgroup, 32 threads a column, each every 32nd part; the sums meet in LDS.
__global__ void __launch_bounds__(1024) sum_parts_kernel(const float* part, float* out, const float* part2, float* out2, int64_t parts,
                                                         int64_t cols, int64_t pitch) {
    __shared__ float s[32][33];
    if (blockIdx.y) {
        part = part2;
        out = out2;
    }
    const int64_t c = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
    const int at = threadIdx.x >> 5;
    float t = 0.0f;
    if (c < cols) {
#pragma unroll 4
        for (int64_t p = at; p < parts; p += 32) t += part[p * pitch + c];
    }
    s[at][threadIdx.x & 31] = t;
    __syncthreads();
    if (at || c >= cols) return;
    t = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += s[i][threadIdx.x];
    out[c] = t;
}

}  // namespace

size_t act_grad_workspace_floats(int64_t rows, int64_t cols) { return (size_t)parts_of(rows, cols) * (size_t)cols; }

hipError_t launch_act_grad(const ActGrad& a, hipStream_t s) { return a.f32 ? launch_act<float>(a, s) : launch_act<uint16_t>(a, s); }

hipError_t launch_sum_parts(const float* part, float* out, const float* part2, float* out2, int64_t parts, int64_t cols, int64_t pitch,
                            hipStream_t s) {
    if (!out) {
        out = out2;
        part = part2;
        out2 = nullptr;
    }
    hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)((cols + 31) / 32), out2 ? 2 : 1), dim3(1024), 0, s, part, out, part2, out2, parts,
                       cols, pitch);
    return hipGetLastError();
}

}  // namespace halo
