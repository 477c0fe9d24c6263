// Norm of the rows of a matrix (halo_layer_norm_fwd) and its gradient (halo_layer_norm_bwd).
#pragma clang fp contract(off)

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
__device__ __forceinline__ float vector_at(const void* p, int f32, int c, float none) {
    if (!p) return none;
    return f32 ? reinterpret_cast<const float*>(p)[c] : widen(reinterpret_cast<const uint16_t*>(p)[c]);
}

// The sum of x over the workgroup, for every thread.
__device__ __forceinline__ float workgroup_sum(float x, float* s) {
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    return (s[0] + s[1]) + (s[2] + s[3]);
}

template <typename E>
__global__ void __launch_bounds__(kThreads) norm_fwd_kernel(NormFwd a) {
    __shared__ float s[4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const E* x = reinterpret_cast<const E*>(a.X) + row * a.ld_x;
    E* y = reinterpret_cast<E*>(a.Y) + row * a.ld_y;
    float mean = 0.0f, t = 0.0f;
    if (!a.rms) {
        for (int c = threadIdx.x; c < a.cols; c += kThreads) t += widen(x[c]);
        mean = workgroup_sum(t, s) / (float)a.cols;
    }
    t = 0.0f;
    for (int c = threadIdx.x; c < a.cols; c += kThreads) {
        const float d = widen(x[c]) - mean;
        t += d * d;
    }
    const float rstd = 1.0f / __builtin_sqrtf(workgroup_sum(t, s) / (float)a.cols + a.eps);
    for (int c = threadIdx.x; c < a.cols; c += kThreads)
        Eight<E>::store_one(y + c, (widen(x[c]) - mean) * rstd * vector_at(a.weight, a.weight_f32, c, 1.0f) +
                                       vector_at(a.bias, a.weight_f32, c, 0.0f));
    if (threadIdx.x == 0) {
        if (a.mean && !a.rms) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    }
}

template <typename E>
__global__ void __launch_bounds__(kThreads) norm_bwd_rows_kernel(NormBwd a) {
    __shared__ float s[4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const E *e = reinterpret_cast<const E*>(a.E) + row * a.ld_e, *x = reinterpret_cast<const E*>(a.X) + row * a.ld_x;
    const E* base = a.base ? reinterpret_cast<const E*>(a.base) + row * a.ld_base : nullptr;
    E* ex = reinterpret_cast<E*>(a.EX) + row * a.ld_ex;
    const float mean = a.mean ? a.mean[row] : 0.0f, rstd = a.rstd[row];
    float t1 = 0.0f, t2 = 0.0f;
    for (int c = threadIdx.x; c < a.cols; c += kThreads) {
        const float d = widen(e[c]) * vector_at(a.weight, a.weight_f32, c, 1.0f);
        t1 += d;
        t2 += d * ((widen(x[c]) - mean) * rstd);
    }
    const float m1 = a.rms ? 0.0f : workgroup_sum(t1, s) / (float)a.cols, m2 = workgroup_sum(t2, s) / (float)a.cols;
    for (int c = threadIdx.x; c < a.cols; c += kThreads) {
        const float d = widen(e[c]) * vector_at(a.weight, a.weight_f32, c, 1.0f), xh = (widen(x[c]) - mean) * rstd;
        float r = (d - m1 - xh * m2) * rstd;
        if (base) r += widen(base[c]);
        Eight<E>::store_one(ex + c, r);
    }
    }
}

unsigned row_groups(int64_t rows) { return (unsigned)(rows < 65536 ? rows : 65536); }

// One thread a column of one part of the rows.
template <typename E>
__global__ void __launch_bounds__(kThreads) norm_bwd_columns_kernel(NormBwd a, int64_t rows_per_part, int64_t parts) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.cols) return;
    const int64_t r0 = blockIdx.y * rows_per_part, r1 = r0 + rows_per_part < a.rows ? r0 + rows_per_part : a.rows;
    float gw = 0.0f, gb = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        const float e = widen(reinterpret_cast<const E*>(a.E)[r * a.ld_e + c]);
        gb += e;
        if (a.GW) gw += e * ((widen(reinterpret_cast<const E*>(a.X)[r * a.ld_x + c]) - (a.mean ? a.mean[r] : 0.0f)) * a.rstd[r]);
    }
    a.part[(int64_t)blockIdx.y * a.cols + c] = gw;
    a.part[(parts + blockIdx.y) * (int64_t)a.cols + c] = gb;
}

int64_t parts_of(int64_t rows) { return rows < 64 ? rows : 64; }

template <typename E>
hipError_t launch_bwd(const NormBwd& a, hipStream_t s) {
    if (a.GW || a.GB) {                  // before EX, which may be E itself
        const int64_t most = parts_of(a.rows), per = most ? (a.rows + most - 1) / most : 1, parts = (a.rows + per - 1) / per;
        if (parts)
            hipLaunchKernelGGL((norm_bwd_columns_kernel<E>), dim3((a.cols + kThreads - 1) / kThreads, (unsigned)parts), dim3(kThreads), 0, s,
                               a, per, parts);
        const hipError_t e = launch_sum_parts(a.part, a.GW, a.part + parts * a.cols, a.GB, parts, a.cols, s);
        if (e != hipSuccess) return e;
    }
    if (a.EX && a.rows) hipLaunchKernelGGL((norm_bwd_rows_kernel<E>), dim3(row_groups(a.rows)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

size_t norm_bwd_workspace_floats(int64_t rows, int64_t cols) { return 2 * (size_t)parts_of(rows) * (size_t)cols; }

hipError_t launch_norm_fwd(const NormFwd& a, hipStream_t s) {
    if (a.f32) hipLaunchKernelGGL((norm_fwd_kernel<float>), dim3(row_groups(a.rows)), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((norm_fwd_kernel<uint16_t>), dim3(row_groups(a.rows)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormBwd& a, hipStream_t s) { return a.f32 ? launch_bwd<float>(a, s) : launch_bwd<uint16_t>(a, s); }

}  // namespace halo
