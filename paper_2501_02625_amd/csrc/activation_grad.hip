// The gradient of the epilogue of a product (halo_activation_bwd): E_Z = E act'(Z), and the bias' gradient, its column sums, in one pass.
// What bounds it is memory, and of small matrices the launches: one up to 128 rows, otherwise two.  8192 x 14336 in bf16 with gelu: 145 us,
// 4.9 TB/s (a large copy reaches 5.1), and 4.5 for the sum over 73 parts of the rows.
#pragma clang fp contract(off)

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
    // Rows of a thread that are requested at once.  gelu in a graph, one / two / four: fp32, 1024 x 14336 31.7 us / 32.4 / 33.0, 1024 x 4096
    // 13.8 / 15.2 / 15.7 (registers); bf16, 128 x 512 two 5.0, four 4.5, 128 x 14336 5.6 and 5.1, 8192 x 14336 150 either way.
    constexpr int AHEAD = sizeof(E) == 2 ? 4 : 1;
    __shared__ float meet[ROWS][LANES * 8];
    const int lane = threadIdx.x % LANES, at = threadIdx.x / LANES;
    const int64_t c = ((int64_t)blockIdx.x * LANES + lane) * 8, left = a.cols - c;
    const int64_t r0 = blockIdx.y * rows_per_part, r1 = r0 + rows_per_part < a.rows ? r0 + rows_per_part : a.rows;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    // Rows are requested before the first of them is stored: EZ may be E or Z, and no load would pass a store.  Behind the last row
    // it is read again, and left out.
    if (left > 0) {
        for (int64_t r = r0 + at; r < r1; r += AHEAD * ROWS) {
            Eight<E> e[AHEAD], z[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int64_t row = r + k * ROWS < r1 ? r + k * ROWS : r1 - 1;
                e[k].load(reinterpret_cast<const E*>(a.E) + row * a.ld_e + c, left > 4);
                if constexpr (ACT != HALO_ACT_NONE) z[k].load(reinterpret_cast<const E*>(a.Z) + row * a.ld_z + c, left > 4);
                else z[k] = e[k];
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (r + k * ROWS >= r1) break;
                float d[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    d[j] = activation_slope<ACT>(e[k].get(j), z[k].get(j));
                    sum[j] += d[j];
                }
                if (!a.EZ) continue;
                E* p = reinterpret_cast<E*>(a.EZ) + (r + k * ROWS) * a.ld_ez + c;
                if (left >= 8) {
                    Eight<E>::store(p, d);
                } else {
#pragma unroll
                    for (int j = 0; j < 7; ++j)
                        if (j < left) Eight<E>::store_one(p + j, d[j]);
                }
            }
        }
    }
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
        if (gridDim.y == 1) a.GB[col] = t;
        else a.part[blockIdx.y * a.cols + col] = t;
    }
}

// Parts of the rows: as many as make some two thousand workgroups, with a row for each of their threads at least, and 512 at most, for each
// is read again.  In a graph, at most 2048 / 512 / 256: bf16, 8192 x 512 15.3 us / 10.6 / 10.7, 2048 x 512 7.3 / 7.4 / 6.6, 8192 x 1003 17.4 /
// 17.1 / 16.7, 16384 x 1003 26.7 / 24.5 / 25.9.  At least one / two / four rows a thread: 300 x 1003 6.0 / 6.1 / 7.0, 1031 x 4096 11.6 /
// 10.3 / 9.9, fp32 1031 x 1003 7.1 / 7.1 / 8.5.
//
// Few rows are one part, 64 columns to a workgroup so that there are many, and need no second launch.  bf16, in a graph, one part / several:
// 64 x 512 3.4 us / 4.9, 64 x 14336 3.7 / 6.6, 128 x 512 4.5 / 5.2, 128 x 14336 5.1 / 7.8, 192 x 512 5.8 / 5.3, 256 x 4096 7.1 / 6.6; the
// host's part of a launch, 3 us, comes on top where calls are not captured.
constexpr int64_t kFewRows = 128;
int lanes_of(int64_t rows, int64_t cols) { return rows <= kFewRows ? 8 : cols <= 64 ? 8 : cols <= 128 ? 16 : cols <= 256 ? 32 : 64; }
int64_t parts_of(int64_t rows, int64_t cols) {
    if (rows <= kFewRows) return rows > 0;
    const int lanes = lanes_of(rows, cols);
    const int64_t tiles = (cols + lanes * 8 - 1) / (lanes * 8), at_once = 256 / lanes;
    const int64_t most = tiles < 4 ? 512 : tiles < 2048 ? 2048 / tiles : 1, parts = (rows + at_once - 1) / at_once;
    return parts < most ? parts : most;
}

template <typename E, int ACT>
hipError_t launch_typed(const ActGrad& a, hipStream_t s) {
    const int lanes = lanes_of(a.rows, a.cols);
    const int64_t most = parts_of(a.rows, a.cols), per = most ? (a.rows + most - 1) / most : 1, parts = (a.rows + per - 1) / per;
    if (parts) {
        const dim3 grid((unsigned)((a.cols + lanes * 8 - 1) / (lanes * 8)), (unsigned)parts);
        if (lanes == 8) hipLaunchKernelGGL((act_grad_kernel<E, ACT, 8>), grid, dim3(256), 0, s, a, per);
        else if (lanes == 16) hipLaunchKernelGGL((act_grad_kernel<E, ACT, 16>), grid, dim3(256), 0, s, a, per);
        else if (lanes == 32) hipLaunchKernelGGL((act_grad_kernel<E, ACT, 32>), grid, dim3(256), 0, s, a, per);
        else hipLaunchKernelGGL((act_grad_kernel<E, ACT, 64>), grid, dim3(256), 0, s, a, per);
    }
    if (a.GB && parts != 1) return launch_sum_parts(a.part, a.GB, nullptr, nullptr, parts, a.cols, a.cols, s);
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
