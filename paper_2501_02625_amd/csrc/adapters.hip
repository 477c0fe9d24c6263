// Low-rank adapters of many requests beside a projection that they share, and their gradients.  Token t has the adapter
// a = adapter_of[t] with U_a [rank x m], V_a [n x rank] and the scale s_a:
//   T = drop(X) U_a^T        Y = base + s_a T V_a^T
//   S = s_a E V_a            E_X = base + drop'(S U_a)       G_U = sum over a's tokens of S_t drop(X)_t       G_V = s_a sum of E_t T_t
// Products of bf16 values accumulate in fp32; T and S stay fp32.
#pragma clang fp contract(off)

#include "adapters.h"

namespace halo {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float f32(uint16_t bits) { return __uint_as_float((uint32_t)bits << 16); }

__device__ __forceinline__ int rank_of(const AdapterPool& p, int a) {
    if (!p.ranks) return p.max_rank;
    const int r = p.ranks[a];
    return r < 0 ? 0 : r > p.max_rank ? p.max_rank : r;
}
__device__ __forceinline__ float scale_of(const AdapterPool& p, int a) { return p.scale ? p.scale[a] : 1.0f; }
__device__ __forceinline__ bool has_adapter(const AdapterPool& p, int a) { return a >= 0 && a < p.slots; }

__device__ __forceinline__ float dropped(const uint16_t* x, const DropoutMask& d, int64_t row, int64_t k) {
    if (d.least == 0) return f32(x[k]);
    const uint4 bits = dropout_bits(d, (uint32_t)row, (uint32_t)(k >> 3));
    return dropout_kept(d, bits, (int)(k & 7)) ? f32(x[k]) * d.factor : 0.0f;
}

// A wavefront per (token, rank column).  T = drop(X) U^T, or, with E, S = scale E V.
__global__ void __launch_bounds__(64)
thin_kernel(AdapterPool p, const uint16_t* in, int64_t ld, int backward, float* out, DropoutMask d) {
    const int64_t t = blockIdx.x;
    const int c = blockIdx.y, lane = threadIdx.x;
    const int a = p.adapter_of[t];
    float sum = 0.0f;
    if (has_adapter(p, a) && c < rank_of(p, a)) {
        const uint16_t* x = in + t * ld;
        if (backward) {
            const uint16_t* v = p.V + (int64_t)a * p.n * p.max_rank + c;
            for (int64_t k = lane; k < p.n; k += 64) sum += f32(x[k]) * f32(v[k * p.max_rank]);
            sum *= scale_of(p, a);
        } else {
            const uint16_t* u = p.U + ((int64_t)a * p.max_rank + c) * p.m;
            for (int64_t k = lane; k < p.m; k += 64) sum += dropped(x, d, t, k) * f32(u[k]);
        }
    }
    for (int h = 32; h > 0; h >>= 1) sum += __shfl_xor(sum, h);
    if (lane == 0) out[t * p.max_rank + c] = sum;
}

// A thread per output element.  Y = base + scale T V^T, or, backward, E_X = base + drop'(S U).
__global__ void __launch_bounds__(kThreads)
wide_kernel(AdapterPool p, const float* thin, int backward, const void* base, int64_t ld_base, void* out, int64_t ld_out, int out_f32,
            DropoutMask d) {
    const int64_t t = blockIdx.x, wide = backward ? p.m : p.n;
    const int64_t j = (int64_t)blockIdx.y * kThreads + threadIdx.x;
    if (j >= wide) return;
    const int a = p.adapter_of[t];
    float y = 0.0f;
    if (has_adapter(p, a)) {
        const int rank = rank_of(p, a);
        const float* x = thin + t * p.max_rank;
        if (backward) {
            const uint16_t* u = p.U + (int64_t)a * p.max_rank * p.m + j;
            for (int c = 0; c < rank; ++c) y += x[c] * f32(u[(int64_t)c * p.m]);
            if (d.least) {
                const uint4 bits = dropout_bits(d, (uint32_t)t, (uint32_t)(j >> 3));
                y = dropout_kept(d, bits, (int)(j & 7)) ? y * d.factor : 0.0f;
            }
        } else {
            const uint16_t* v = p.V + ((int64_t)a * p.n + j) * p.max_rank;
            for (int c = 0; c < rank; ++c) y += x[c] * f32(v[c]);
            y *= scale_of(p, a);
        }
    }
    if (out_f32) {
        if (base) y += reinterpret_cast<const float*>(base)[t * ld_base + j];
        reinterpret_cast<float*>(out)[t * ld_out + j] = y;
    } else {
        if (base) y += f32(reinterpret_cast<const uint16_t*>(base)[t * ld_base + j]);
        reinterpret_cast<uint16_t*>(out)[t * ld_out + j] = __builtin_bit_cast(uint16_t, (__bf16)y);
    }
}

// A thread per (adapter, rank column, wide column), over all tokens in order.
__global__ void __launch_bounds__(kThreads)
grad_kernel(AdapterPool p, const uint16_t* big, int64_t ld, const float* thin, int of_v, float* out, DropoutMask d) {
    const int64_t wide = of_v ? p.n : p.m;
    const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int c = blockIdx.y;
    const int a = blockIdx.z;
    if (j >= wide) return;
    float sum = 0.0f;
    if (c < rank_of(p, a)) {
        for (int64_t t = 0; t < p.b; ++t) {
            if (p.adapter_of[t] != a) continue;
            const float x = of_v ? f32(big[t * ld + j]) : dropped(big + t * ld, d, t, j);
            sum += x * thin[t * p.max_rank + c];
        }
        if (of_v) sum *= scale_of(p, a);
    }
    if (of_v) out[((int64_t)a * wide + j) * p.max_rank + c] = sum;
    else out[((int64_t)a * p.max_rank + c) * wide + j] = sum;
}

unsigned blocks_of(int64_t n) { return (unsigned)((n + kThreads - 1) / kThreads); }

}  // namespace

size_t adapters_fwd_workspace(int64_t, int64_t, int64_t, int, int) { return 0; }
size_t adapters_bwd_workspace(int64_t b, int64_t, int64_t, int, int max_rank) { return (size_t)b * max_rank * 4; }

hipError_t launch_adapters_fwd(const AdaptersFwd& a, hipStream_t s) {
    const AdapterPool& p = a.pool;
    hipLaunchKernelGGL(thin_kernel, dim3((unsigned)p.b, p.max_rank), dim3(64), 0, s, p, a.X, a.ld_x, 0, a.T, a.drop);
    hipLaunchKernelGGL(wide_kernel, dim3((unsigned)p.b, blocks_of(p.n)), dim3(kThreads), 0, s, p, a.T, 0, a.base, a.ld_base, a.Y, a.ld_y,
                       a.out_f32, a.drop);
    return hipGetLastError();
}

hipError_t launch_adapters_bwd(const AdaptersBwd& a, hipStream_t s) {
    const AdapterPool& p = a.pool;
    float* S = reinterpret_cast<float*>(a.workspace);
    if (p.b > 0 && (a.EX || a.GU))
        hipLaunchKernelGGL(thin_kernel, dim3((unsigned)p.b, p.max_rank), dim3(64), 0, s, p, a.E, a.ld_e, 1, S, a.drop);
    if (p.b > 0 && a.EX)
        hipLaunchKernelGGL(wide_kernel, dim3((unsigned)p.b, blocks_of(p.m)), dim3(kThreads), 0, s, p, S, 1, a.base, a.ld_base, a.EX,
                           a.ld_ex, a.out_f32, a.drop);
    if (a.GU)
        hipLaunchKernelGGL(grad_kernel, dim3(blocks_of(p.m), p.max_rank, p.slots), dim3(kThreads), 0, s, p, a.X, a.ld_x, S, 0, a.GU, a.drop);
    if (a.GV)
        hipLaunchKernelGGL(grad_kernel, dim3(blocks_of(p.n), p.max_rank, p.slots), dim3(kThreads), 0, s, p, a.E, a.ld_e, a.T, 1, a.GV, a.drop);
    return hipGetLastError();
}

}  // namespace halo
