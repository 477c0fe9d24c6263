// One AdamW step over many tensors at once (halo_adamw), states in 32 or in 8 bits.
//
// 8 bits: what is kept is an e4m3 code times a scale that 256 elements share, for v of its root.  Rounded to nearest, v, which moves
// by (1 - beta2) of its distance in a step, would stay where it is: the codes are 6 to 12 % apart.  Rounded at random between the two
// neighbours, with the probability that makes the mean right (of m, and of v, not of its root: the mean of the root's square would be
// above v by the variance of the rounding, every step again), they follow.
//
// What bounds it: memory with states in 32 bits (12.6M elements in fp32 71 us, 5.0 TB/s; a large copy reaches 5.1), with 8 bits
// instructions as much, some hundred an element: 219M elements in bf16 492 to 530 us on different cards, 4.1 to 4.5 TB/s; 467 without the
// random numbers where it takes 530.  There one round instead of two 545, and loads that stay in the caches 537; before the roots were what
// they are, four rounds as two.
#pragma clang fp contract(off)

#include <cmath>

#include "around.h"
#include "halo_internal.h"
#include "philox.h"
#include "wave_ops.h"

namespace halo {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 256;                  // elements that share a scale: 32 lanes of eight
constexpr int kRounds = 2;                   // groups of eight elements per thread, all loads issued before the first is used
constexpr int kPerRound = kThreads * 8, kPerGroup = kPerRound * kRounds;      // elements of a workgroup
constexpr int kTensors = 48;                 // of a launch; they come as arguments, of which a kernel has 4 KB

struct Batch {
    AdamwStep step;
    int count;
    uint32_t end[kTensors];                  // of each tensor, the number of the first workgroup behind it
    AdamwTensor tensor[kTensors];
};
static_assert(sizeof(Batch) <= 4096, "kernel arguments");

enum { PARAM_F32, PARAM_BF16, PARAM_MASTER };

// The upper half of a word of random bits as the upper half of a number, and the lower one: u * 65536.
__device__ __forceinline__ uint32_t upper_half_of(const uint4& u, int j) {
    const uint32_t w = j < 2 ? u.x : j < 4 ? u.y : j < 6 ? u.z : u.w;
    return (j & 1) ? w & 0xFFFF0000u : w << 16;
}
__device__ __forceinline__ uint32_t half_of(const uint4& u, int j) {
    const uint32_t w = j < 2 ? u.x : j < 4 ? u.y : j < 6 ? u.z : u.w;
    return (j & 1) ? w >> 16 : w & 0xFFFFu;
}

// The code of the e4m3 number next to q, 0 <= q <= 448, up or down by the random bits.  SQUARE: by q's square.  From 2^-6 on a number has
// three bits of fraction, and whether it goes up is a question about its fraction alone: about the bits behind those three, or, of the square,
// about f = q over the step, 8 <= f < 16, and k, f rounded down: (f - k)(f + k) against u (2 k + 1).  (All of it but for powers of two, which
// change no rounding, what the definition says in terms of q, lo and hi.)
template <bool SQUARE>
__device__ __forceinline__ uint32_t code_of_normal(float q, const uint4& u, int j) {
    const uint32_t bits = __float_as_uint(q);
    bool up;
    if constexpr (SQUARE) {
        const uint32_t fb = (bits & 0x007FFFFFu) | 0x41000000u;
        const float f = __uint_as_float(fb), k = __uint_as_float(fb & 0xFFF00000u);
        up = (f - k) * (f + k) > (float)half_of(u, j) * __builtin_fmaf(k, 2.0f / 65536.0f, 1.0f / 65536.0f);
    } else {
        up = bits << 12 > upper_half_of(u, j);
    }
    return (bits >> 20) - (120u << 3) + (up ? 1u : 0u);
}
// Below 2^-6 the steps are 2^-9.  A square that is not 0 does not become 0.
template <bool SQUARE>
__device__ __forceinline__ uint32_t code_of_small(float q, float x, const uint4& u, int j) {
    const float t = q * 512.0f, k = __builtin_truncf(t), r = (float)half_of(u, j);
    bool up;
    if constexpr (SQUARE) up = (t - k) * (t + k) > r * __builtin_fmaf(k, 2.0f / 65536.0f, 1.0f / 65536.0f);
    else up = (t - k) * 65536.0f > r;
    const uint32_t code = (uint32_t)k + (up ? 1u : 0u);
    return SQUARE && x > 0.0f && code == 0 ? 1u : code;
}
// Codes of eight values, signs included (of m).  Small ones are rare, and a wavefront that has none does not look at each.
template <bool SQUARE>
__device__ __forceinline__ void codes_of(const float* x, float inverse, const uint4& u, uint32_t* out) {
    float q[8], least = 448.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        q[j] = __builtin_fminf(__builtin_fabsf(x[j]) * inverse, 448.0f);
        least = __builtin_fminf(least, q[j]);
    }
    uint32_t c[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = code_of_normal<SQUARE>(q[j], u, j);
    if (__builtin_amdgcn_ballot_w64(least < 0.015625f)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t small = code_of_small<SQUARE>(q[j], x[j], u, j);
            c[j] = q[j] < 0.015625f ? small : c[j];
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = 4 * h + e;
            w |= c[j] << (8 * e);
            if constexpr (!SQUARE) w |= (__float_as_uint(x[j]) & 0x80000000u) >> (24 - 8 * e);
        }
        out[h] = w;
    }
}

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

// Eight consecutive elements as they are in memory: fp32, bf16 or e4m3 codes.  n: how many there are (8, but at a tensor's end).
template <int BYTES>
struct Run {
    static constexpr int WORDS = 2 * BYTES;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const void* base, int64_t i, int n) {
        const char* p = reinterpret_cast<const char*>(base) + i * BYTES;
        if (n == 8) {
            if constexpr (BYTES == 1) {
                const v2u q = __builtin_nontemporal_load(reinterpret_cast<const v2u*>(p));
                w[0] = q[0]; w[1] = q[1];
            } else {
#pragma unroll
                for (int k = 0; k < WORDS / 4; ++k) {
                    const v4u q = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p) + k);
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[4 * k + e] = q[e];
                }
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < WORDS; ++k) w[k] = 0;
#pragma unroll
        for (int j = 0; j < 7; ++j) {
            if (j >= n) break;
            if constexpr (BYTES == 4) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
            else if constexpr (BYTES == 2) w[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
            else w[j >> 2] |= (uint32_t)reinterpret_cast<const uint8_t*>(p)[j] << (8 * (j & 3));
        }
    }
    __device__ __forceinline__ void store(void* base, int64_t i, int n) const {
        char* p = reinterpret_cast<char*>(base) + i * BYTES;
        if (n == 8) {
            if constexpr (BYTES == 1) {
                __builtin_nontemporal_store((v2u){w[0], w[1]}, reinterpret_cast<v2u*>(p));
            } else {
#pragma unroll
                for (int k = 0; k < WORDS / 4; ++k)
                    __builtin_nontemporal_store((v4u){w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]}, reinterpret_cast<v4u*>(p) + k);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < 7; ++j) {
            if (j >= n) break;
            if constexpr (BYTES == 4) reinterpret_cast<uint32_t*>(p)[j] = w[j];
            else if constexpr (BYTES == 2) reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            else reinterpret_cast<uint8_t*>(p)[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
        }
    }
    __device__ __forceinline__ void get(float* x) const {
        if constexpr (BYTES == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(w[j]);
        } else if constexpr (BYTES == 2) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __uint_as_float((j & 1) ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
                x[4 * k] = lo[0]; x[4 * k + 1] = lo[1]; x[4 * k + 2] = hi[0]; x[4 * k + 3] = hi[1];
            }
        }
    }
};

// The largest of a number's bits over the 32 lanes that share a scale, for each of them.
template <int J>
__device__ __forceinline__ uint32_t more_of(uint32_t x) {
    const uint32_t y = __float_as_uint(lane_xor<J>(__uint_as_float(x), 0));
    return y > x ? y : x;
}
__device__ __forceinline__ uint32_t most_of_32(uint32_t x) { return more_of<4>(more_of<3>(more_of<2>(more_of<1>(more_of<0>(x))))); }

// root = sqrt(v) and quotient = m / (root * by + eps), each rounded to nearest as the language's root and division are, of which this
// is the inner part: what they spend on arguments near the ends of the range is left out where a wavefront has none of those.  Then the
// remainders v - s s and m - d q are exact, and one Newton step from the hardware's reciprocal root (two from its reciprocal) rounds
// correctly: of the root a test tries every significand, with even and odd exponents; the quotient's steps are those of the division, and the same
// test takes quotients next to the middle between two numbers.
// (The language's own for all: 566 us for 219M elements in bf16 with states in 8 bits instead of 523.)
__device__ __forceinline__ void roots_and_quotients(const float (&v)[8], const float (&m)[8], float by, float eps,
                                                    float (&root)[8], float (&quotient)[8], uint32_t& most_m) {
    auto bits = [](float x) { return __float_as_uint(x); };
    auto at = [](int power) { return (uint32_t)(127 + power) << 23; };
    uint32_t most_v = 0, least_v = ~0u, least_m = ~0u;
    most_m = 0;
    float most_d = 0.0f, least_d = __uint_as_float(0x7F800000u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float s0 = __builtin_amdgcn_rsqf(__builtin_fmaxf(v[j], 0x1p-100f)), s = v[j] * s0;
        root[j] = __builtin_fmaf(__builtin_fmaf(-s, s, v[j]), 0.5f * s0, s);
        const float d = root[j] * by + eps;
        float y = __builtin_amdgcn_rcpf(d);
        y = __builtin_fmaf(__builtin_fmaf(-d, y, 1.0f), y, y);
        float q = m[j] * y;
        q = __builtin_fmaf(__builtin_fmaf(-d, q, m[j]), y, q);
        quotient[j] = __builtin_fmaf(__builtin_fmaf(-d, q, m[j]), y, q);
        const uint32_t bv = bits(v[j]), bm = bits(m[j]) & 0x7FFFFFFFu;             // 0 is 2^32 - 1 among the least
        most_v = bv > most_v ? bv : most_v;
        least_v = bv - 1 < least_v ? bv - 1 : least_v;
        most_m = bm > most_m ? bm : most_m;
        least_m = bm - 1 < least_m ? bm - 1 : least_m;
        most_d = __builtin_fmaxf(most_d, d);
        least_d = __builtin_fminf(least_d, d);
    }
    const bool inside = most_v <= at(100) && least_v >= at(-100) && most_m <= at(60) && least_m >= at(-60) && most_d <= 0x1p60f &&
                        least_d >= 0x1p-60f;
    if (__builtin_amdgcn_ballot_w64(!inside)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            root[j] = __builtin_sqrtf(v[j]);
            quotient[j] = m[j] / (root[j] * by + eps);
        }
    }
}

template <int PARAM, bool GRAD32, bool STATE8>
__global__ void __launch_bounds__(kThreads) adamw_kernel(Batch b) {
    // the tensor: of a wavefront's lanes, those whose tensor ends before this workgroup
    const int lane = threadIdx.x & 63;
    const bool behind = lane < kTensors && blockIdx.x >= b.end[lane < kTensors ? lane : 0];
    const int t = __builtin_amdgcn_readfirstlane(__builtin_popcountll(__builtin_amdgcn_ballot_w64(behind)));
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
        // even lanes have beta1's number and odd ones beta2's: functions in 64 bits take as long as an element's whole step.  (With pow()
        // instead of the logarithm from the host 564 us for 219M elements in bf16 with states in 8 bits; numbers from the host: 497.)
        const double rest = 1.0 - exp2((double)c.step * ((lane & 1) ? c.log_beta2 : c.log_beta1));
        const float number = (float)((lane & 1) ? 1.0 / sqrt(rest) : lr / rest);
        c.rate = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(number), 0));
        c.root = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(number), 1));
    }
    DropoutMask d{};
    d.key0 = c.key0; d.key1 = c.key1; d.offset0 = (uint32_t)c.offset; d.offset1 = (uint32_t)(c.offset >> 32);
    const uint32_t kind0 = 4u * (uint32_t)x.number;
    constexpr int PB = PARAM == PARAM_BF16 ? 2 : 4, SB = STATE8 ? 1 : 4;
    const int64_t start = (int64_t)(blockIdx.x - first) * kPerGroup + threadIdx.x * 8;
    Run<PB> rp[kRounds];
    Run<GRAD32 ? 4 : 2> rg[kRounds];
    Run<SB> rm[kRounds], rv[kRounds];
    float sm[kRounds], sv[kRounds];
    int left[kRounds];
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int64_t i = start + k * kPerRound;
        const int n = left[k] = x.size - i >= 8 ? 8 : x.size > i ? (int)(x.size - i) : 0;
        rp[k].load(PARAM == PARAM_MASTER ? x.master : x.param, i, n);
        rg[k].load(x.grad, i, n);
        rm[k].load(x.m, i, n);
        rv[k].load(x.v, i, n);
        sm[k] = sv[k] = 0.0f;
        if constexpr (STATE8) {
            if (n) {
                sm[k] = x.m_scale[i / kBlock];
                sv[k] = x.v_scale[i / kBlock];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int64_t i = start + k * kPerRound;
        const int n = left[k];
        const uint32_t group = (uint32_t)(i >> 3);
        float p[8], g[8], m[8], v[8], root[8];
        rp[k].get(p);
        rg[k].get(g);
        rm[k].get(m);
        rv[k].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (STATE8) {
                m[j] = m[j] * sm[k];
                v[j] = v[j] * sv[k];
                v[j] = v[j] * v[j];
            }
            g[j] = g[j] * c.grad_scale;
            m[j] = c.beta1 * m[j] + c.rest1 * g[j];
            v[j] = c.beta2 * v[j] + c.rest2 * (g[j] * g[j]);
        }
        float quotient[8];
        uint32_t am;                         // the largest |m|, as its bits
        roots_and_quotients(v, m, c.root, c.eps, root, quotient, am);
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = p[j] * c.decay - c.rate * quotient[j];
        if constexpr (PARAM == PARAM_BF16) {
            const uint4 u = dropout_bits(d, kind0, group);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                uint32_t r[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int j = 2 * h + e;
                    r[e] = p[j] != p[j] ? 0x7FC00000u : __float_as_uint(p[j]) + half_of(u, j);
                }
                rp[k].w[h] = __builtin_amdgcn_perm(r[1], r[0], 0x07060302u);
            }
            rp[k].store(x.param, i, n);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) rp[k].w[j] = __float_as_uint(p[j]);
            rp[k].store(PARAM == PARAM_MASTER ? x.master : x.param, i, n);
            if constexpr (PARAM == PARAM_MASTER) {
                Run<2> r;
#pragma unroll
                for (int h = 0; h < 4; ++h) r.w[h] = pack_bf16x2(p[2 * h], p[2 * h + 1]);
                r.store(x.param, i, n);
            }
        }
        if constexpr (!STATE8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                rm[k].w[j] = __float_as_uint(m[j]);
                rv[k].w[j] = __float_as_uint(v[j]);
            }
        } else {
            // the largest of 32 lanes, as bit patterns: a NaN is above an infinity, and that above all numbers.  (What lies behind the
            // tensor's end is 0.)
            constexpr uint32_t kLeast = (127u - 110u) << 23;
            uint32_t av = kLeast;
            am = am > kLeast ? am : kLeast;
#pragma unroll
            for (int j = 0; j < 8; ++j) av = __float_as_uint(root[j]) > av ? __float_as_uint(root[j]) : av;
            am = most_of_32(am);
            av = most_of_32(av);
            const float fm = __uint_as_float(am), fv = __uint_as_float(av);
            if (n && (threadIdx.x & 31) == 0) {
                x.m_scale[i / kBlock] = fm / 448.0f;
                x.v_scale[i / kBlock] = fv / 448.0f;
            }
            const float im = 448.0f / fm, iv = 448.0f / fv;
            const uint4 um = dropout_bits(d, kind0 + 1, group), uv = dropout_bits(d, kind0 + 2, group);
            codes_of<false>(m, im, um, rm[k].w);
            codes_of<true>(root, iv, uv, rv[k].w);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (am >= 0x7F800000u) rm[k].w[h] = 0x7F7F7F7Fu;
                if (av >= 0x7F800000u) rv[k].w[h] = 0x7F7F7F7Fu;
            }
        }
        rm[k].store(x.m, i, n);
        rv[k].store(x.v, i, n);
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
