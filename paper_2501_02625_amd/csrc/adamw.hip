// One AdamW step over many tensors at once (halo_adamw), states in 32 or in 8 bits.
//
// 8 bits: what is kept is an e4m3 code times a scale that 256 elements share, for v of its root.  Rounded to nearest, v, which moves
// by (1 - beta2) of its distance in a step, would stay where it is: the codes are 6 to 12 % apart.  Rounded at random between the two
// neighbours, with the probability that makes the mean right (of m, and of v, not of its root: the mean of the root's square would be
// above v by the variance of the rounding, every step again), they follow.
#pragma clang fp contract(off)

#include <cmath>

#include "around.h"
#include "eight.h"
#include "philox.h"

namespace halo {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 256;                  // elements that share a scale: 32 lanes of eight
constexpr int kPerGroup = kThreads * 8;      // elements of a workgroup
constexpr int kTensors = 48;                 // of a launch; they come as arguments, of which a kernel has 4 KB

struct Batch {
    AdamwStep step;
    int count;
    uint32_t end[kTensors];                  // of each tensor, the number of the first workgroup behind it
    AdamwTensor tensor[kTensors];
};
static_assert(sizeof(Batch) <= 4096, "kernel arguments");

enum { PARAM_F32, PARAM_BF16, PARAM_MASTER };

// The code of the e4m3 number next to q, 0 <= q <= 448, up or down by the random u.  SQUARE: by q's square.
template <bool SQUARE>
__device__ __forceinline__ uint32_t code_of(float q, uint32_t u) {
    const uint32_t bits = __float_as_uint(q);
    float lo, step;
    uint32_t code;
    if (bits >= 0x3C800000u) {               // 2^-6: three bits of fraction
        code = (bits >> 20) - (120u << 3);
        lo = __uint_as_float(bits & 0xFFF00000u);
        step = __uint_as_float((bits & 0x7F800000u) - (3u << 23));
    } else {                                 // steps of 2^-9
        code = (uint32_t)(q * 512.0f);
        lo = (float)code * 0.001953125f;
        step = 0.001953125f;
    }
    const float r = (float)u;
    bool up;
    if constexpr (SQUARE) up = ((q - lo) * (q + lo)) * 65536.0f > r * (step * (lo + step + lo));
    else up = (q - lo) * 65536.0f > r * step;
    return code + (up ? 1u : 0u);
}

__device__ __forceinline__ float value_of(uint32_t code) {
    return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

template <int PARAM, bool GRAD32, bool STATE8>
__global__ void __launch_bounds__(kThreads) adamw_kernel(Batch b) {
    int t = 0;
    while (t + 1 < b.count && blockIdx.x >= b.end[t]) ++t;
    const AdamwTensor& x = b.tensor[t];
    const uint32_t first = t ? b.end[t - 1] : 0;
    AdamwStep c = b.step;
    if (c.step_ptr || c.lr_ptr || c.grad_scale_ptr) {
        if (c.step_ptr) c.step = *c.step_ptr;
        if (c.step < 1) c.step = 1;
        if (c.step_ptr) c.offset += (uint64_t)c.step;
        if (c.grad_scale_ptr) c.grad_scale = *c.grad_scale_ptr;
        const double lr = c.lr_ptr ? (double)*c.lr_ptr : c.lr;
        c.decay = (float)(1.0 - lr * c.weight_decay);
        c.rate = (float)(lr / (1.0 - pow(c.beta1_64, (double)c.step)));
        c.root = (float)(1.0 / sqrt(1.0 - pow(c.beta2_64, (double)c.step)));
    }
    const int64_t i0 = (int64_t)(blockIdx.x - first) * kPerGroup + threadIdx.x * 8;
    const int n = x.size - i0 >= 8 ? 8 : x.size > i0 ? (int)(x.size - i0) : 0;         // elements of this thread
    DropoutMask d{};
    d.key0 = c.key0; d.key1 = c.key1; d.offset0 = (uint32_t)c.offset; d.offset1 = (uint32_t)(c.offset >> 32);
    const uint32_t group = (uint32_t)(i0 >> 3), kind0 = 4u * (uint32_t)x.number;
    float m[8], v[8], p[8], g[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        m[j] = v[j] = p[j] = g[j] = 0.0f;
        if (j >= n) continue;
        const int64_t i = i0 + j;
        if constexpr (GRAD32) g[j] = reinterpret_cast<const float*>(x.grad)[i];
        else g[j] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(x.grad)[i] << 16);
        if constexpr (PARAM == PARAM_F32) p[j] = reinterpret_cast<const float*>(x.param)[i];
        else if constexpr (PARAM == PARAM_MASTER) p[j] = x.master[i];
        else p[j] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(x.param)[i] << 16);
        if constexpr (STATE8) {
            m[j] = value_of(reinterpret_cast<const uint8_t*>(x.m)[i]) * x.m_scale[i / kBlock];
            v[j] = value_of(reinterpret_cast<const uint8_t*>(x.v)[i]) * x.v_scale[i / kBlock];
            v[j] = v[j] * v[j];
        } else {
            m[j] = reinterpret_cast<const float*>(x.m)[i];
            v[j] = reinterpret_cast<const float*>(x.v)[i];
        }
    }
    float root[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        g[j] = g[j] * c.grad_scale;
        m[j] = c.beta1 * m[j] + c.rest1 * g[j];
        v[j] = c.beta2 * v[j] + c.rest2 * (g[j] * g[j]);
        root[j] = __builtin_sqrtf(v[j]);
        p[j] = p[j] * c.decay - c.rate * (m[j] / (root[j] * c.root + c.eps));
    }
    if constexpr (PARAM == PARAM_BF16) {
        const uint4 u = dropout_bits(d, kind0, group);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t bits = __float_as_uint(p[j]), r = bits + ((w[j >> 1] >> (16 * (j & 1))) & 0xFFFFu);
            if (j < n) reinterpret_cast<uint16_t*>(x.param)[i0 + j] = p[j] != p[j] ? 0x7FC0 : (uint16_t)(r >> 16);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= n) continue;
            if constexpr (PARAM == PARAM_F32) reinterpret_cast<float*>(x.param)[i0 + j] = p[j];
            else {
                x.master[i0 + j] = p[j];
                Eight<uint16_t>::store_one(reinterpret_cast<uint16_t*>(x.param) + i0 + j, p[j]);
            }
        }
    }
    if constexpr (!STATE8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= n) continue;
            reinterpret_cast<float*>(x.m)[i0 + j] = m[j];
            reinterpret_cast<float*>(x.v)[i0 + j] = v[j];
        }
    } else {
        // the largest of 32 lanes, as bit patterns: a NaN is above an infinity, and that above all numbers
        uint32_t am = 0, av = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t bm = __float_as_uint(m[j]) & 0x7FFFFFFFu, bv = __float_as_uint(root[j]) & 0x7FFFFFFFu;
            am = bm > am && j < n ? bm : am;
            av = bv > av && j < n ? bv : av;
        }
#pragma unroll
        for (int l = 1; l < 32; l <<= 1) {
            const uint32_t om = (uint32_t)__shfl_xor((int)am, l), ov = (uint32_t)__shfl_xor((int)av, l);
            am = om > am ? om : am;
            av = ov > av ? ov : av;
        }
        constexpr uint32_t kLeast = (127u - 110u) << 23;
        am = am > kLeast ? am : kLeast;
        av = av > kLeast ? av : kLeast;
        const float fm = __uint_as_float(am), fv = __uint_as_float(av);
        if (n && (threadIdx.x & 31) == 0) {
            x.m_scale[i0 / kBlock] = fm / 448.0f;
            x.v_scale[i0 / kBlock] = fv / 448.0f;
        }
        const float im = 448.0f / fm, iv = 448.0f / fv;
        const uint4 um = dropout_bits(d, kind0 + 1, group), uv = dropout_bits(d, kind0 + 2, group);
        const uint32_t wm[4] = {um.x, um.y, um.z, um.w}, wv[4] = {uv.x, uv.y, uv.z, uv.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= n) continue;
            const float qm = __builtin_fminf(__builtin_fabsf(m[j]) * im, 448.0f), qv = __builtin_fminf(root[j] * iv, 448.0f);
            uint32_t cm = code_of<false>(qm, (wm[j >> 1] >> (16 * (j & 1))) & 0xFFFFu);
            uint32_t cv = code_of<true>(qv, (wv[j >> 1] >> (16 * (j & 1))) & 0xFFFFu);
            cm |= m[j] < 0.0f ? 0x80u : 0u;
            if (cv == 0 && root[j] > 0.0f) cv = 1;
            if (am >= 0x7F800000u) cm = 0x7F;
            if (av >= 0x7F800000u) cv = 0x7F;
            reinterpret_cast<uint8_t*>(x.m)[i0 + j] = (uint8_t)cm;
            reinterpret_cast<uint8_t*>(x.v)[i0 + j] = (uint8_t)cv;
        }
    }
}

template <int PARAM, bool GRAD32, bool STATE8>
hipError_t launch_typed(const AdamwStep& step, const AdamwTensor* tensors, int count, hipStream_t s) {
    for (int at = 0; at < count;) {
        Batch b;
        b.step = step;
        b.count = 0;
        int64_t groups = 0;
        for (; at < count && b.count < kTensors; ++at) {
            if (tensors[at].size == 0) continue;
            const int64_t more = (tensors[at].size + kPerGroup - 1) / kPerGroup;
            if (b.count && groups + more > (int64_t(1) << 23)) break;                  // 2^31 threads
            groups += more;
            b.tensor[b.count] = tensors[at];
            b.end[b.count++] = (uint32_t)groups;
        }
        if (!b.count) break;
        for (int i = b.count; i < kTensors; ++i) {
            b.end[i] = (uint32_t)groups;
            b.tensor[i] = AdamwTensor{};
        }
        hipLaunchKernelGGL((adamw_kernel<PARAM, GRAD32, STATE8>), dim3((unsigned)groups), dim3(kThreads), 0, s, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <int PARAM>
hipError_t launch_param(const AdamwStep& step, const AdamwTensor* tensors, int count, int grad_f32, int state8, hipStream_t s) {
    if (grad_f32) return state8 ? launch_typed<PARAM, true, true>(step, tensors, count, s) : launch_typed<PARAM, true, false>(step, tensors, count, s);
    return state8 ? launch_typed<PARAM, false, true>(step, tensors, count, s) : launch_typed<PARAM, false, false>(step, tensors, count, s);
}

}  // namespace

void adamw_numbers(double step, double lr, double beta1, double beta2, double weight_decay, float* decay, float* rate, float* root) {
    *decay = (float)(1.0 - lr * weight_decay);
    *rate = (float)(lr / (1.0 - std::pow(beta1, step)));
    *root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, step)));
}

hipError_t launch_adamw(const AdamwStep& step, const AdamwTensor* tensors, int count, int param, int grad_f32, int state8, hipStream_t s) {
    if (param == PARAM_F32) return launch_param<PARAM_F32>(step, tensors, count, grad_f32, state8, s);
    if (param == PARAM_BF16) return launch_param<PARAM_BF16>(step, tensors, count, grad_f32, state8, s);
    return launch_param<PARAM_MASTER>(step, tensors, count, grad_f32, state8, s);
}

}  // namespace halo
