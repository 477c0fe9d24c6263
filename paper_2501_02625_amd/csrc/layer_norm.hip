// Norm of the rows of a matrix (halo_layer_norm_fwd) and its gradient (halo_layer_norm_bwd).
//
// What bounds both is memory.  A row is held in registers by a team of LANES lanes, eight elements at a time and GROUPS times, so that it is
// read once: the mean, then the squares about it, then the result.  Teams go from row to row, with the next row's loads on their way
// while this one is worked on; weight and bias stay in registers.  bf16, 8192 x 4096 with a bias: 25 us, 5.4 TB/s (a large copy reaches 5.1),
// one row of 4096 2.1 us; the gradient with a base and G_W, 2048 x 4096: 14.5 us, 4.6 TB/s, and 4.0 for the sum over 512 parts of
// the rows; 128 x 4096, in one launch, 4.4.
#pragma clang fp contract(off)

#include <type_traits>

#include "around.h"
#include "eight.h"
#include "norm_plan.h"
#include "wave_ops.h"

namespace halo {
namespace {

// Sum over the lanes of a team of at most a wavefront, for each of its lanes.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x, int bperm_addr) {
    x += lane_xor<0>(x, 0);
    x += lane_xor<1>(x, 0);
    x += lane_xor<2>(x, 0);
    if constexpr (LANES > 8) x += lane_xor<3>(x, 0);
    if constexpr (LANES > 16) x += lane_xor<4>(x, 0);
    if constexpr (LANES > 32) x += lane_xor<5>(x, bperm_addr);
    return x;
}

// Sums over a team.  A team of several wavefronts is the whole workgroup, or one of TEAMS that run in step; their parts meet in LDS, in one of
// two places in turn: a place is written again only behind the barrier of the other one, in front of which it was read.
template <int LANES, int TEAMS, int N>
struct TeamSum {
    static constexpr int WAVES = LANES > 64 ? LANES / 64 : 1;
    float (*s)[N][TEAMS][WAVES];
    int turn = 0, bperm_addr = (int)((threadIdx.x & 63) ^ 32) << 2;
    __device__ __forceinline__ void operator()(float (&x)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = lanes_sum<LANES>(x[i], bperm_addr);
        if constexpr (LANES > 64) {
            const int team = threadIdx.x / LANES, wave = threadIdx.x % LANES / 64;
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) s[turn][i][team][wave] = x[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) x[i] += s[turn][i][team][w];
            }
            turn ^= 1;
        }
    }
};

// Eight elements of weight or bias, fp32 or bf16 (then in lo alone); what lies beyond the vector's end is not read.
template <bool F32>
struct Weights {
    uint4 lo, hi;
    __device__ __forceinline__ void load(const void* p, int c, int left) {
        lo = hi = make_uint4(0, 0, 0, 0);
        if (left <= 0) return;
        // the vector's address and a 32-bit offset, which costs one register where a full address costs two
        const char* q = reinterpret_cast<const char*>(p);
        const uint32_t at = (uint32_t)c * (F32 ? 4 : 2);
        if (left >= 8) {
            lo = *reinterpret_cast<const uint4*>(q + at);
            if constexpr (F32) hi = *reinterpret_cast<const uint4*>(q + (at + 16));
            return;
        }
        uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 7; ++j) {
            if (j >= left) break;
            if constexpr (F32) w[j] = *reinterpret_cast<const uint32_t*>(q + (at + 4 * j));
            else w[j >> 1] |= (uint32_t)*reinterpret_cast<const uint16_t*>(q + (at + 2 * j)) << (16 * (j & 1));
        }
        lo = make_uint4(w[0], w[1], w[2], w[3]);
        hi = make_uint4(w[4], w[5], w[6], w[7]);
    }
    __device__ __forceinline__ void fill(float x) {
        uint32_t w = __float_as_uint(x);
        if constexpr (!F32) w |= w >> 16;    // 0 and 1 have their bits in the upper half
        lo = hi = make_uint4(w, w, w, w);
    }
    __device__ __forceinline__ float get(int j) const {
        const uint4& q = F32 ? (j < 4 ? lo : hi) : lo;
        const int k = F32 ? j & 3 : j >> 1;
        const uint32_t w = k == 0 ? q.x : k == 1 ? q.y : k == 2 ? q.z : q.w;
        return __uint_as_float(F32 ? w : (j & 1) ? w & 0xFFFF0000u : w << 16);
    }
};

// Zeros in the place of what lies behind the end of the row, from element n on.
__device__ __forceinline__ void cut(Eight<uint16_t>& x, int n) {
    uint32_t w[4] = {x.q.x, x.q.y, x.q.z, x.q.w};
#pragma unroll
    for (int h = 0; h < 4; ++h) w[h] &= (2 * h < n ? 0xFFFFu : 0u) | (2 * h + 1 < n ? 0xFFFF0000u : 0u);
    x.q = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void cut(Eight<float>& x, int n) {
    x.lo = make_float4(n > 0 ? x.lo.x : 0.0f, n > 1 ? x.lo.y : 0.0f, n > 2 ? x.lo.z : 0.0f, n > 3 ? x.lo.w : 0.0f);
    x.hi = make_float4(n > 4 ? x.hi.x : 0.0f, n > 5 ? x.hi.y : 0.0f, n > 6 ? x.hi.z : 0.0f, 0.0f);
}

// What was computed from x before is not known to be what is computed from it afterwards.
__device__ __forceinline__ void forget(Eight<uint16_t>& x) { asm volatile("" : "+v"(x.q.x), "+v"(x.q.y), "+v"(x.q.z), "+v"(x.q.w)); }
__device__ __forceinline__ void forget(Eight<float>& x) {
    asm volatile("" : "+v"(x.lo.x), "+v"(x.lo.y), "+v"(x.lo.z), "+v"(x.lo.w));
    asm volatile("" : "+v"(x.hi.x), "+v"(x.hi.y), "+v"(x.hi.z), "+v"(x.hi.w));
}

template <typename E>
__device__ __forceinline__ void store_part(E* p, const float* y, int n) {
    if (n >= 8) {
        Eight<E>::store(p, y);
        return;
    }
#pragma unroll
    for (int j = 0; j < 7; ++j)
        if (j < n) Eight<E>::store_one(p + j, y[j]);
}

// What the kernels have in common.  FULL: that many groups of a row lie inside it for sure (the rules of the launchers).  LEAN: rows so
// long that neither the next row nor weight and bias find room in registers beside the row; group comes after
// group, for what is loaded late is not to be loaded all at once.
template <int LANES, int GROUPS, bool SUMS>
struct Shape {
    static constexpr int FULL = GROUPS / 2;
    static constexpr bool LEAN = GROUPS >= (SUMS ? 4 : 8);
    static __device__ __forceinline__ void in_order() {
        if constexpr (LEAN) __builtin_amdgcn_sched_barrier(0);
    }
    static __device__ __forceinline__ int column(int g) { return (g * LANES + (int)threadIdx.x % LANES) * 8; }
    // Called for every row: the comparisons with what is left of a row are made anew.  Kept over the loop, as the compiler would, they
    // fill the scalar registers and then scratch memory.
    static __device__ __forceinline__ void anew(int (&left)[GROUPS]) {
#pragma unroll
        for (int g = FULL; g < GROUPS; ++g) asm volatile("" : "+v"(left[g]));
    }
    // The address of a group: the row's and a 32-bit offset.
    template <typename E>
    static __device__ __forceinline__ E* group(E* row, int g) {
        using Byte = std::conditional_t<std::is_const_v<E>, const char, char>;
        return reinterpret_cast<E*>(reinterpret_cast<Byte*>(row) + (uint32_t)column(g) * (uint32_t)sizeof(E));
    }
};
template <class S, typename E, int GROUPS>
__device__ __forceinline__ void load_row(Eight<E> (&x)[GROUPS], const E* row, const int (&left)[GROUPS]) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
        if (g < S::FULL || left[g] > 0) x[g].load(S::group(row, g), g < S::FULL || left[g] > 4);
}
template <typename E, int FULL, int GROUPS>
__device__ __forceinline__ void cut_row(Eight<E> (&x)[GROUPS], const int (&left)[GROUPS]) {
#pragma unroll
    for (int g = FULL; g < GROUPS; ++g)
        if (left[g] < 8) cut(x[g], left[g]);
}

// W32: weight and bias are held as fp32 (they are, or they are absent).
template <typename E, bool W32, int LANES, int GROUPS, int TEAMS>
__global__ void __launch_bounds__(LANES* TEAMS) norm_fwd_kernel(NormFwd a) {
    using S = Shape<LANES, GROUPS, false>;
    using Sum = TeamSum<LANES, TEAMS, 1>;
    __shared__ float s[2][1][TEAMS][Sum::WAVES];
    Sum sum{s};
    const int team = TEAMS > 1 ? threadIdx.x / LANES : 0, lane = threadIdx.x % LANES;
    const int64_t stride = (int64_t)gridDim.x * TEAMS;
    const E* X = reinterpret_cast<const E*>(a.X);
    Weights<W32> w[GROUPS], b[GROUPS];
    Eight<E> x[GROUPS], next[GROUPS];
    int left[GROUPS];                        // columns from a group's first one on
    int64_t row = (int64_t)blockIdx.x * TEAMS + team;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) left[g] = a.cols - S::column(g);
    auto load_weights = [&](int g) {
        w[g].fill(1.0f);
        b[g].fill(0.0f);
        if (a.weight) w[g].load(a.weight, S::column(g), left[g]);
        if (a.bias) b[g].load(a.bias, S::column(g), left[g]);
    };
    if constexpr (!S::LEAN) {
        if (row < a.rows) load_row<S>(next, X + row * a.ld_x, left);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) load_weights(g);
    }
    const float cols = (float)a.cols;
    // teams in step: as many rounds as the workgroup's first team has rows
    for (int64_t first = (int64_t)blockIdx.x * TEAMS; first < a.rows; first += stride, row += stride) {
        S::anew(left);
        if constexpr (S::LEAN) {
            if (row < a.rows) load_row<S>(x, X + row * a.ld_x, left);
        } else {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) x[g] = next[g];
            if (row + stride < a.rows) load_row<S>(next, X + (row + stride) * a.ld_x, left);
        }
        cut_row<E, S::FULL, GROUPS>(x, left);
        float mean = 0.0f, t[1] = {0.0f};
        if (!a.rms) {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int j = 0; j < 8; ++j) t[0] += x[g].get(j);
            sum(t);
            mean = t[0] / cols;
        }
        t[0] = 0.0f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            if (g < S::FULL || left[g] >= 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = x[g].get(j) - mean;
                    t[0] = __builtin_fmaf(d, d, t[0]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 7; ++j) {
                    const float d = j < left[g] ? x[g].get(j) - mean : 0.0f;
                    t[0] = __builtin_fmaf(d, d, t[0]);
                }
            }
        }
        sum(t);
        const float rstd = 1.0f / __builtin_sqrtf(t[0] / cols + a.eps);
        if (row >= a.rows) continue;
        E* y = reinterpret_cast<E*>(a.Y) + row * a.ld_y;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            S::in_order();
            if constexpr (S::LEAN) load_weights(g);
            float out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                out[j] = __builtin_fmaf((x[g].get(j) - mean) * rstd, w[g].get(j), b[g].get(j));
            if (g < S::FULL) Eight<E>::store(S::group(y, g), out);
            else if (left[g] > 0) store_part(S::group(y, g), out, left[g]);
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// G_W and G_B of 64 columns over all rows, by a workgroup of THREADS: eight lanes have a row's part.
template <typename E, int THREADS>
__device__ __forceinline__ void few_rows_columns(const NormBwd& a, int block, float (&meet)[THREADS / 64][2][64]) {
    const int lane = threadIdx.x & 7, c = block * 64 + lane * 8, left = a.cols - c;
    float sum[2][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[0][j] = sum[1][j] = 0.0f;
    if (left > 0) {
#pragma unroll 4
        for (int64_t r = threadIdx.x >> 3; r < a.rows; r += THREADS / 8) {
            Eight<E> e, x;
            e.load(reinterpret_cast<const E*>(a.E) + r * a.ld_e + c, left > 4);
            float mean = 0.0f, rstd = 0.0f;
            cut(x, 0);
            if (a.GW) {
                x.load(reinterpret_cast<const E*>(a.X) + r * a.ld_x + c, left > 4);
                mean = a.mean ? a.mean[r] : 0.0f;
                rstd = a.rstd[r];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum[0][j] = __builtin_fmaf(e.get(j), (x.get(j) - mean) * rstd, sum[0][j]);
                sum[1][j] += e.get(j);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int d = 8; d < 64; d *= 2) sum[i][j] += __shfl_xor(sum[i][j], d);
            if ((threadIdx.x & 63) < 8) meet[threadIdx.x >> 6][i][lane * 8 + j] = sum[i][j];
        }
    __syncthreads();
    if (threadIdx.x >= 128) return;
    const int which = threadIdx.x >> 6, col = block * 64 + (threadIdx.x & 63);
    float* out = which ? a.GB : a.GW;
    if (!out || col >= a.cols) return;
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) t += meet[w][which][threadIdx.x & 63];
    out[col] = t;
}

// EX, and with SUMS the sums of the columns over the workgroup's rows, which go to part: the teams add theirs to one another in LDS.
// Without SUMS the first row_groups workgroups have the rows, and those behind them, of few rows, the sums.
template <typename E, bool W32, int LANES, int GROUPS, int TEAMS, bool SUMS>
__global__ void __launch_bounds__(LANES* TEAMS) norm_bwd_kernel(NormBwd a, unsigned row_groups) {
    if constexpr (!SUMS) {
        __shared__ float columns[LANES * TEAMS / 64][2][64];
        if (blockIdx.x >= row_groups) {
            few_rows_columns<E, LANES * TEAMS>(a, blockIdx.x - row_groups, columns);
            return;
        }
    } else {
        row_groups = gridDim.x;
    }
    using S = Shape<LANES, GROUPS, SUMS>;
    using Sum = TeamSum<LANES, TEAMS, 2>;
    __shared__ float s[2][2][TEAMS][Sum::WAVES];
    constexpr int WIDE = LANES * GROUPS * 8;
    __shared__ __align__(16) float meet[SUMS && TEAMS > 1 ? 2 * TEAMS * WIDE : 1];
    Sum sum{s};
    const int team = TEAMS > 1 ? threadIdx.x / LANES : 0, lane = threadIdx.x % LANES;
    const int64_t stride = (int64_t)row_groups * TEAMS;
    const E *X = reinterpret_cast<const E*>(a.X), *Er = reinterpret_cast<const E*>(a.E), *base = reinterpret_cast<const E*>(a.base);
    const bool need_x = a.EX || a.GW;
    Weights<W32> w[GROUPS];
    Eight<E> x[GROUPS], e[GROUPS], next_x[GROUPS], next_e[GROUPS];
    float mean = 0.0f, rstd = 0.0f, next_mean = 0.0f, next_rstd = 0.0f;
    float gw[GROUPS][8], gb[GROUPS][8];
    int left[GROUPS];
    int64_t row = (int64_t)blockIdx.x * TEAMS + team;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) left[g] = a.cols - S::column(g);
    auto load = [&](int64_t r, Eight<E>(&to_x)[GROUPS], Eight<E>(&to_e)[GROUPS], float& to_mean, float& to_rstd) {
        if (r < a.rows) {
            load_row<S>(to_e, Er + r * a.ld_e, left);
            if (need_x) {
                load_row<S>(to_x, X + r * a.ld_x, left);
                to_mean = a.mean ? a.mean[r] : 0.0f;
                to_rstd = a.rstd[r];
            }
        } else {                             // a row of zeros adds nothing
            to_mean = to_rstd = 0.0f;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                cut(to_x[g], 0);
                cut(to_e[g], 0);
            }
        }
    };
    auto load_weights = [&](int g) {
        w[g].fill(1.0f);
        if (a.weight) w[g].load(a.weight, S::column(g), left[g]);
    };
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        cut(x[g], 0);                        // without X
        if constexpr (!S::LEAN) cut(next_x[g], 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) gw[g][j] = gb[g][j] = 0.0f;
    }
    if constexpr (!S::LEAN) {
        load(row, next_x, next_e, next_mean, next_rstd);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) load_weights(g);
    }
    const float cols = (float)a.cols;
    for (int64_t first = (int64_t)blockIdx.x * TEAMS; first < a.rows; first += stride, row += stride) {
        S::anew(left);
        if constexpr (S::LEAN) {
            load(row, x, e, mean, rstd);
        } else {
            mean = next_mean;
            rstd = next_rstd;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                x[g] = next_x[g];
                e[g] = next_e[g];
            }
            load(row + stride, next_x, next_e, next_mean, next_rstd);
        }
        cut_row<E, S::FULL, GROUPS>(x, left);
        cut_row<E, S::FULL, GROUPS>(e, left);
        float t[2] = {0.0f, 0.0f};
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            S::in_order();
            if constexpr (S::LEAN) load_weights(g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float ej = e[g].get(j), xh = (x[g].get(j) - mean) * rstd, d = ej * w[g].get(j);
                if constexpr (SUMS) {
                    gb[g][j] += ej;
                    gw[g][j] = __builtin_fmaf(ej, xh, gw[g][j]);
                }
                t[0] += d;
                t[1] = __builtin_fmaf(d, xh, t[1]);
            }
        }
        if (!a.EX) continue;                 // uniform
        Eight<E> add[GROUPS];
        if (!S::LEAN && base && row < a.rows) load_row<S>(add, base + row * a.ld_base, left);
        sum(t);
        if (row >= a.rows) continue;
        if constexpr (GROUPS >= 4) {         // xh and d are computed again rather than kept, which would take twice the row's registers
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                forget(x[g]);
                forget(e[g]);
            }
        }
        const float m1 = a.rms ? 0.0f : t[0] / cols, m2 = t[1] / cols;
        E* ex = reinterpret_cast<E*>(a.EX) + row * a.ld_ex;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            if (g >= S::FULL && left[g] <= 0) continue;
            S::in_order();
            if constexpr (S::LEAN) {
                load_weights(g);
                if (base) add[g].load(S::group(base + row * a.ld_base, g), left[g] > 4);
            }
            float out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xh = (x[g].get(j) - mean) * rstd, d = e[g].get(j) * w[g].get(j);
                out[j] = __builtin_fmaf(-xh, m2, d - m1) * rstd;
                if (base) out[j] += add[g].get(j);
            }
            if (g < S::FULL) Eight<E>::store(S::group(ex, g), out);
            else store_part(S::group(ex, g), out, left[g]);
        }
    }
    if constexpr (SUMS) {
        // rows of parts begin at multiples of four floats
        const int64_t pitch = (a.cols + 3) / 4 * 4;
        float *part_w = a.part + (int64_t)blockIdx.x * pitch, *part_b = a.part + ((int64_t)gridDim.x + blockIdx.x) * pitch;
        if constexpr (TEAMS > 1) {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                Eight<float>::store(meet + team * WIDE + S::column(g), gw[g]);
                Eight<float>::store(meet + (TEAMS + team) * WIDE + S::column(g), gb[g]);
            }
            __syncthreads();
            for (int i = threadIdx.x; i < 2 * WIDE; i += LANES * TEAMS) {
                const int which = i / WIDE, c = i % WIDE;
                if (c >= a.cols || !(which ? a.GB : a.GW)) continue;
                float v = 0.0f;
#pragma unroll
                for (int k = 0; k < TEAMS; ++k) v += meet[(which * TEAMS + k) * WIDE + c];
                (which ? part_b : part_w)[c] = v;
            }
        } else {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                if (g >= S::FULL && left[g] <= 0) continue;
                if (a.GW) store_part(part_w + S::column(g), gw[g], left[g]);
                if (a.GB) store_part(part_b + S::column(g), gb[g], left[g]);
            }
        }
    }
}

// The sums of the columns alone, for rows that leave no registers for them beside the row: a wavefront has 512 columns, and every fourth of
// the rows of its workgroup.
template <typename E>
__global__ void __launch_bounds__(256) norm_columns_kernel(NormBwd a, int64_t rows_per_part) {
    __shared__ float meet[4][2][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 512 + lane * 8, left = a.cols - c;
    const int64_t r0 = blockIdx.y * rows_per_part, r1 = r0 + rows_per_part < a.rows ? r0 + rows_per_part : a.rows;
    float gw[8], gb[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) gw[j] = gb[j] = 0.0f;
    if (left > 0) {
#pragma unroll 4
        for (int64_t r = r0 + wave; r < r1; r += 4) {
            Eight<E> e, x;
            e.load(reinterpret_cast<const E*>(a.E) + r * a.ld_e + c, left > 4);
            float mean = 0.0f, rstd = 0.0f;
            cut(x, 0);
            if (a.GW) {
                x.load(reinterpret_cast<const E*>(a.X) + r * a.ld_x + c, left > 4);
                mean = a.mean ? a.mean[r] : 0.0f;
                rstd = a.rstd[r];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                gb[j] += e.get(j);
                gw[j] = __builtin_fmaf(e.get(j), (x.get(j) - mean) * rstd, gw[j]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        meet[wave][0][lane * 8 + j] = gw[j];
        meet[wave][1][lane * 8 + j] = gb[j];
    }
    __syncthreads();
    const int64_t pitch = (a.cols + 3) / 4 * 4;
    for (int i = threadIdx.x; i < 1024; i += 256) {
        const int which = i >> 9, k = i & 511, col = blockIdx.x * 512 + k;
        if (col >= a.cols) continue;
        a.part[((int64_t)which * gridDim.y + blockIdx.y) * pitch + col] =
            (meet[0][which][k] + meet[1][which][k]) + (meet[2][which][k] + meet[3][which][k]);
    }
}

// Lanes and groups of a row.  As many lanes as the row has pieces of eight, up to 64, so that no wavefront meets another; beyond 512
// columns two groups or more lanes, whichever was faster.  Rows x columns, forward, bf16: two groups of 64 lanes / one of 128, 16384 x 1000
// 15.0 us / 16.0, but backward, where sums take registers, four teams of 128 lanes, 1031 x 1003 in fp32 6.3 us, and of 64 7.6; one
// group of 256 / four of 64, 4096 x 2048 9.7 / 12.5; one of 512 / two of 256, 8192 x 4096 25.0 / 24.1, 64 x 4096 3.4 / 3.9; one of 1024 / two of
// 512, 2048 x 8192 15.5 / 18.4; backward one of 512 / two of 256, 2048 x 4096 14.5 / 15.4.
//
// Workgroups of a launch: enough for every compute unit to hold several at once; each goes through its rows.  Forward 2^19 threads, rows x
// columns: 2^18 / 2^19 / 2^20, 8192 x 4096 28.4 us / 25.0 / 24.4, 1024 x 14336 14.8 / 16.2 / 19.4, 16384 x 1000 14.5 / 14.9 / 16.3.  The gradient's:
// norm_plan.h.
constexpr int64_t kThreadsFwd = 1 << 19;
inline unsigned groups_of(int64_t rows, int teams, int64_t most) {
    const int64_t n = (rows + teams - 1) / teams;
    return (unsigned)(n < most ? n : most);
}

template <typename E, bool W32, int LANES, int GROUPS, int TEAMS>
hipError_t fwd(const NormFwd& a, hipStream_t s) {
    const unsigned groups = groups_of(a.rows, TEAMS, kThreadsFwd / (LANES * TEAMS));
    hipLaunchKernelGGL((norm_fwd_kernel<E, W32, LANES, GROUPS, TEAMS>), dim3(groups), dim3(LANES * TEAMS), 0, s, a);
    return hipGetLastError();
}
template <typename E, bool W32>
hipError_t fwd_by_shape(const NormFwd& a, hipStream_t s) {
    const int c = a.cols;
    if (c <= 64) return fwd<E, W32, 8, 1, 32>(a, s);
    if (c <= 128) return fwd<E, W32, 16, 1, 16>(a, s);
    if (c <= 256) return fwd<E, W32, 32, 1, 8>(a, s);
    if (c <= 512) return fwd<E, W32, 64, 1, 4>(a, s);
    if (c <= 1024) return fwd<E, W32, 64, 2, 4>(a, s);
    if (c <= 2048) return fwd<E, W32, 256, 1, 1>(a, s);
    if (c <= 4096) return fwd<E, W32, 512, 1, 1>(a, s);
    if (c <= 8192) return fwd<E, W32, 1024, 1, 1>(a, s);
    if (c <= 16384) return fwd<E, W32, 1024, 2, 1>(a, s);
    return fwd<E, W32, 512, 8, 1>(a, s);
}

template <typename E, bool W32, int LANES, int GROUPS, int TEAMS>
hipError_t bwd_few_rows(const NormBwd& a, hipStream_t s) {
    const unsigned groups = a.EX ? groups_of(a.rows, TEAMS, kMostNormBwd) : 0, columns = (unsigned)(a.cols + 63) / 64;
    auto launch = [&](unsigned rows, unsigned behind) {
        hipLaunchKernelGGL((norm_bwd_kernel<E, W32, LANES, GROUPS, TEAMS, false>), dim3(rows + behind), dim3(LANES * TEAMS), 0, s, a, rows);
    };
    if (a.EX && (a.EX == a.E || a.EX == a.X)) {       // it would be overwritten while columns are read
        launch(0, columns);
        launch(groups, 0);
    } else {
        launch(groups, columns);
    }
    return hipGetLastError();
}

template <typename E, bool W32, int LANES, int GROUPS, int TEAMS>
hipError_t bwd(const NormBwd& a, hipStream_t s) {
    const bool sums = a.GW || a.GB;
    if (sums && norm_bwd_one_launch(a.rows, a.cols, a.f32)) return bwd_few_rows<E, W32, LANES, GROUPS, TEAMS>(a, s);
    // as many parts as the workspace query counts
    const unsigned groups = sums ? (unsigned)norm_bwd_parts(a.rows, a.cols, a.f32) : groups_of(a.rows, TEAMS, most_norm_bwd(a.cols));
    if (groups && sums) hipLaunchKernelGGL((norm_bwd_kernel<E, W32, LANES, GROUPS, TEAMS, true>), dim3(groups), dim3(LANES * TEAMS), 0, s, a, groups);
    else if (groups) hipLaunchKernelGGL((norm_bwd_kernel<E, W32, LANES, GROUPS, TEAMS, false>), dim3(groups), dim3(LANES * TEAMS), 0, s, a, groups);
    if (sums) return launch_sum_parts(a.part, a.GW, a.part + groups * ((a.cols + 3) / 4 * 4), a.GB, groups, a.cols, (a.cols + 3) / 4 * 4, s);
    return hipGetLastError();
}
// Rows without room for the sums: these in a launch of their own, in parts of the rows.  They go first: EX may be E itself.
template <typename E, bool W32, int GROUPS>
hipError_t bwd_apart(const NormBwd& a, hipStream_t s) {
    if ((a.GW || a.GB) && norm_bwd_one_launch(a.rows, a.cols, a.f32)) return bwd_few_rows<E, W32, 512, GROUPS, 1>(a, s);
    if (a.GW || a.GB) {
        const int64_t tiles = (a.cols + 511) / 512, most = norm_bwd_parts(a.rows, a.cols, a.f32);
        const int64_t per = most ? (a.rows + most - 1) / most : 1, parts = (a.rows + per - 1) / per;
        if (parts) hipLaunchKernelGGL((norm_columns_kernel<E>), dim3((unsigned)tiles, (unsigned)parts), dim3(256), 0, s, a, per);
        const hipError_t e = launch_sum_parts(a.part, a.GW, a.part + parts * ((a.cols + 3) / 4 * 4), a.GB, parts, a.cols,
                                              (a.cols + 3) / 4 * 4, s);
        if (e != hipSuccess) return e;
    }
    if (a.EX && a.rows) {
        const unsigned groups = groups_of(a.rows, 1, kMostNormBwd);
        hipLaunchKernelGGL((norm_bwd_kernel<E, W32, 512, GROUPS, 1, false>), dim3(groups), dim3(512), 0, s, a, groups);
    }
    return hipGetLastError();
}
template <typename E, bool W32>
hipError_t bwd_by_shape(const NormBwd& a, hipStream_t s) {
    const int c = a.cols;
    if (c <= 64) return bwd<E, W32, 8, 1, 32>(a, s);
    if (c <= 128) return bwd<E, W32, 16, 1, 16>(a, s);
    if (c <= 256) return bwd<E, W32, 32, 1, 8>(a, s);
    if (c <= 512) return bwd<E, W32, 64, 1, 4>(a, s);
    if (c <= 1024) return bwd<E, W32, 128, 1, 4>(a, s);
    if (c <= 2048) return bwd<E, W32, 256, 1, 1>(a, s);
    if (c <= 4096) return bwd<E, W32, 512, 1, 1>(a, s);
    if (c <= 8192) return bwd<E, W32, 1024, 1, 1>(a, s);
    if constexpr (!norm_bwd_apart(16384, sizeof(E) == 4)) {
        if (c <= 16384) return bwd<E, W32, 512, 4, 1>(a, s);
    }
    return c <= 16384 ? bwd_apart<E, W32, 4>(a, s) : bwd_apart<E, W32, 8>(a, s);
}

}  // namespace

size_t norm_bwd_workspace_floats(int64_t rows, int64_t cols, int f32) {
    // one part where none is written: a call that wants sums brings a workspace, whatever its rows
    const int64_t parts = norm_bwd_one_launch(rows, cols, f32 != 0) ? 1 : norm_bwd_parts(rows, cols, f32 != 0);
    return 2 * (size_t)parts * (size_t)((cols + 3) / 4 * 4);
}

hipError_t launch_norm_fwd(const NormFwd& a, hipStream_t s) {
    const bool w32 = a.weight_f32 || (!a.weight && !a.bias);
    if (a.f32) return w32 ? fwd_by_shape<float, true>(a, s) : fwd_by_shape<float, false>(a, s);
    return w32 ? fwd_by_shape<uint16_t, true>(a, s) : fwd_by_shape<uint16_t, false>(a, s);
}

hipError_t launch_norm_bwd(const NormBwd& a, hipStream_t s) {
    const bool w32 = a.weight_f32 || !a.weight;
    if (a.f32) return w32 ? bwd_by_shape<float, true>(a, s) : bwd_by_shape<float, false>(a, s);
    return w32 ? bwd_by_shape<uint16_t, true>(a, s) : bwd_by_shape<uint16_t, false>(a, s);
}

}  // namespace halo
