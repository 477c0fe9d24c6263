// Kernels and launches of the INT8 GEMM with the scaling epilogue,  C = diag(row_scale) * (A * op(B)) * diag(col_scale), the
// epilogues that run part of a rotation or add a low-rank product, and small products.  The main loop: gemm_i8_device.h.
#include "gemm_i8_device.h"

namespace halo {
namespace {

// Eight values  x <- x + s * x[partner lane]  for the row stride 2^J inside groups of 16 lanes (row_of_lane), one rounded add or subtract each (the product with
// +-1 is exact).  A DPP read needs two wait states after a vector write of the same register: the leading s_nop supplies
// them for whatever came before; inside a block every register is used once.
template <int J>
__device__ __forceinline__ void lane_butterfly8(float& x0, float& x1, float& x2, float& x3, float& x4, float& x5, float& x6,
                                                float& x7, float s) {
#define HALO_DPP_FMAC8(CTRL)                                                                     \
    asm volatile("s_nop 1\n\t"                                                                   \
                 "v_fmac_f32_dpp %0, %0, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"              \
                 "v_fmac_f32_dpp %1, %1, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"              \
                 "v_fmac_f32_dpp %2, %2, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"              \
                 "v_fmac_f32_dpp %3, %3, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"              \
                 "v_fmac_f32_dpp %4, %4, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"              \
                 "v_fmac_f32_dpp %5, %5, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"              \
                 "v_fmac_f32_dpp %6, %6, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t"              \
                 "v_fmac_f32_dpp %7, %7, %8 " CTRL " row_mask:0xf bank_mask:0xf"                   \
                 : "+v"(x0), "+v"(x1), "+v"(x2), "+v"(x3), "+v"(x4), "+v"(x5), "+v"(x6), "+v"(x7) \
                 : "v"(s))
    if constexpr (J == 0) {
        HALO_DPP_FMAC8("quad_perm:[1,0,3,2]");
    } else if constexpr (J == 1) {
        HALO_DPP_FMAC8("quad_perm:[2,3,0,1]");
    } else if constexpr (J == 3) {
        HALO_DPP_FMAC8("row_ror:8");
    } else {
        HALO_DPP_FMAC8("row_half_mirror");                        // lane ^ 7: see row_of_lane
    }
#undef HALO_DPP_FMAC8
}

// Epilogue of a product whose output is then un-rotated on the left (level 2, E_X = H^T ( ... )): the accumulators are
// scaled, (float(acc) * row_scale[row]) * post_scale, and the eight lowest strides of the left-hand Walsh-Hadamard
// rotation run on the 256 rows of the tile before anything is stored, in ascending order and with every add and
// subtract a separately rounded fp32 operation, exactly as a pass over memory would do them.  Row index inside the
// tile = [wave_m | tile i (3 bits) | row in the tile (4 bits, lanes)], so strides 1 .. 8 pair lanes, 16, 32, 64 pair
// registers and 128 pairs this wavefront with the one holding the other 128 rows of the same columns, through LDS: each of
// the two hands over its second half of register tiles and finishes both rows' results of its first half (half the traffic
// of exchanging everything; the halves are in opposite order in the two, so both run the same code).
// Signs: a lane starts with its values multiplied by (-1)^(ones in its row number), folded into the row scale.  A pair's
// lanes then differ in sign, so the lower lane's own - partner is the wanted sum and the upper lane's own + partner the
// wanted difference, each up to the sign that the lower lane carries; after the fourth stage no sign is left.
// No normalisation: the 1/sqrt(block) of the rotation is applied after its last stride, by whoever runs it.
// N is a multiple of 16, M of 256.  SWAP placement.
template <class Cfg, bool PRE>
__device__ __forceinline__ void epilogue_left8(const GemmArgs& a, const Place<Cfg>& at, int wave, int lane,
                                               unsigned char* smem) {
    static_assert(Cfg::TM == 8 && Cfg::TN % 2 == 0, "256-row tiles");
    constexpr int TM = Cfg::TM, TN = Cfg::TN, HALF = TN / 2;
    static_assert(4 * TM * HALF * 1024 <= Cfg::LDS_BYTES, "exchange buffer");
    const int lrow = row_of_lane(lane & 15);
    const float sign = (__builtin_popcount(lrow) & 1) ? -1.0f : 1.0f;
    float rs[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) rs[i] = ((!PRE && a.row_scale) ? a.row_scale[at.row0 + 16 * i] : 1.0f) * sign;
    const bool scale_more = !PRE && a.post_scale;                 // uniform
    const float post = scale_more ? *a.post_scale : 1.0f;
    float s[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) s[b] = ((lrow >> b) & 1) ? 1.0f : -1.0f;

    // the stages inside the wavefront, on column tile j
    auto stages = [&](auto jj, float (&f)[TM][4]) {
        constexpr int j = decltype(jj)::value;
        __builtin_amdgcn_sched_barrier(0);                        // one column tile at a time
        hold_accumulators<TM * TN>();
        StaticFor<0, TM>::run([&](auto ii) {
            constexpr int i = decltype(ii)::value;
            const v4i x = read_acc<i * TN + j>();
#pragma unroll
            for (int r = 0; r < 4; ++r) f[i][r] = (PRE ? __int_as_float(x[r]) : (float)x[r]) * rs[i];
        });
        if (scale_more) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) f[i][r] *= post;
        }
#pragma unroll
        for (int i = 0; i < TM; i += 2) {
            lane_butterfly8<0>(f[i][0], f[i][1], f[i][2], f[i][3], f[i + 1][0], f[i + 1][1], f[i + 1][2], f[i + 1][3], s[0]);
            lane_butterfly8<1>(f[i][0], f[i][1], f[i][2], f[i][3], f[i + 1][0], f[i + 1][1], f[i + 1][2], f[i + 1][3], s[1]);
            lane_butterfly8<2>(f[i][0], f[i][1], f[i][2], f[i][3], f[i + 1][0], f[i + 1][1], f[i + 1][2], f[i + 1][3], s[2]);
            lane_butterfly8<3>(f[i][0], f[i][1], f[i][2], f[i][3], f[i + 1][0], f[i + 1][1], f[i + 1][2], f[i + 1][3], s[3]);
        }
#pragma unroll
        for (int bit = 0; bit < 3; ++bit)
#pragma unroll
            for (int i = 0; i < TM; ++i)
                if ((i & (1 << bit)) == 0) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = f[i][r], y = f[i | (1 << bit)][r];
                        f[i][r] = x + y;
                        f[i | (1 << bit)][r] = x - y;
                    }
                }
    };
    v4f* xb = reinterpret_cast<v4f*>(smem);                       // [wavefront][j of the half][tile i][lane]
    __syncthreads();                                              // every wavefront is done with the operand stages
    StaticFor<0, HALF>::run([&](auto jj) {
        constexpr int j = decltype(jj)::value;
        float f[TM][4];
        stages(Int<HALF + j>(), f);
#pragma unroll
        for (int i = 0; i < TM; ++i) xb[((wave * HALF + j) * TM + i) * 64 + lane] = (v4f){f[i][0], f[i][1], f[i][2], f[i][3]};
    });
    float kept[HALF][TM][4];
    StaticFor<0, HALF>::run([&](auto jj) { stages(jj, kept[decltype(jj)::value]); });
    __syncthreads();
    const v4f* other = xb + (wave ^ 2) * HALF * TM * 64 + lane;
    const float flip = wave >> 1 ? -1.0f : 1.0f;                  // the lower rows' wavefront: own - other; the upper's: other - own
    const int up = (lane >> 3) & 1;                               // whole lines, as in the plain epilogue
    int32_t* dst = reinterpret_cast<int32_t*>(a.C) + (at.row0 - 8 * up - (wave >> 1) * 128) * a.ldc + at.col_lo + 16 * up;
#pragma unroll
    for (int j = 0; j < HALF; j += 2) {
        __builtin_amdgcn_sched_barrier(0);
        if (at.col_lo + 16 * j < a.N) {
            const bool in = at.col_lo + 16 * (j + up) < a.N;
            int32_t* d = dst + 16 * j;
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                v4i sum[2], dif[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const v4f o = other[((j + h) * TM + i) * 64];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        sum[h][r] = __float_as_int(kept[j + h][i][r] + o[r]);
                        dif[h][r] = __float_as_int((kept[j + h][i][r] - o[r]) * flip);
                    }
                }
                v4i sum_lo, sum_up, dif_lo, dif_up;
                whole_lines(sum[0], sum[1], sum_lo, sum_up);
                whole_lines(dif[0], dif[1], dif_lo, dif_up);
                if (in) {
                    store4(d, sum_lo);
                    store4(d + 8 * a.ldc, sum_up);
                    store4(d + 128 * a.ldc, dif_lo);
                    store4(d + 136 * a.ldc, dif_up);
                }
                d += 16 * a.ldc;
            }
        }
    }
}

// Low-rank side product (a LoRA branch next to the quantised product): turns the int32 accumulators, in place, into the
// fp32 values
//   ((float(acc) * row_scale[row]) * col_scale[col]) * post_scale  +  sum_k lr_a[row, k] * lr_b[k, col],
// the first part rounded exactly as the plain epilogues round it, the sum added by matrix instructions with the scaled
// accumulator as their addend.  The registers then hold float bit patterns and the PRE variants of the epilogues take
// over.
// The low-rank sum, 32 ranks at a time, by bf16 matrix instructions (v_mfma_f32_16x16x32_bf16: lane l supplies column /
// row l % 16, ranks 8 (l / 16) .. + 8; the result layout is that of the int8 instruction).  fp32 operands are split exactly
// into three bf16 pieces (8 + 8 + 8 mantissa bits, x = hi + mid + lo); every product of two pieces is exact and is
// accumulated in fp32.  The products kept are those down to 2^-16 of the full one (all of them when one operand is bf16
// already): what is dropped is below 2^-23 of |a b|, an fp32 rounding.  Smallest terms first.  Every address is clamped into
// its matrix, so that all loads are unconditional; what lies outside is zeroed afterwards.
// What bounds it: the latency of its loads, then its vector instructions.  All of them are requested before the first is used
// (the barriers keep the compiler from moving a load to its use) and land while the accumulators are scaled.
// The s_nop: two wait states between a vector write and a matrix instruction that reads it.
template <int T>
__device__ __forceinline__ void lowrank_mfma(const v8bf& bh, const v8bf& ah, const v8bf& am, const v8bf& al) {
    asm volatile("s_nop 1\n\t"
                 "v_mfma_f32_16x16x32_bf16 a[%4:%5], %0, %3, a[%4:%5]\n\t"
                 "v_mfma_f32_16x16x32_bf16 a[%4:%5], %0, %2, a[%4:%5]\n\t"
                 "v_mfma_f32_16x16x32_bf16 a[%4:%5], %0, %1, a[%4:%5]" ::"v"(bh), "v"(ah), "v"(am), "v"(al), "n"(4 * T),
                 "n"(4 * T + 3));
}
template <int T>
__device__ __forceinline__ void lowrank_mfma(const v8bf& bh, const v8bf& bm, const v8bf& bl, const v8bf& ah, const v8bf& am,
                                             const v8bf& al) {
    asm volatile("s_nop 1\n\t"
                 "v_mfma_f32_16x16x32_bf16 a[%6:%7], %0, %5, a[%6:%7]\n\t"
                 "v_mfma_f32_16x16x32_bf16 a[%6:%7], %2, %3, a[%6:%7]\n\t"
                 "v_mfma_f32_16x16x32_bf16 a[%6:%7], %1, %4, a[%6:%7]\n\t"
                 "v_mfma_f32_16x16x32_bf16 a[%6:%7], %0, %4, a[%6:%7]\n\t"
                 "v_mfma_f32_16x16x32_bf16 a[%6:%7], %1, %3, a[%6:%7]\n\t"
                 "v_mfma_f32_16x16x32_bf16 a[%6:%7], %0, %3, a[%6:%7]" ::"v"(bh), "v"(bm), "v"(bl), "v"(ah), "v"(am), "v"(al),
                 "n"(4 * T), "n"(4 * T + 3));
}
// B_BF16: lr_b is bf16 (the forward product, K-contiguous B) or fp32 (the E product, K-strided B).
template <class Cfg, bool B_BF16>
__device__ __forceinline__ void lowrank_prepare(const GemmArgs& a, const Place<Cfg>& at, int lane) {
    constexpr int TM = Cfg::TM, TN = Cfg::TN;
    const int l16 = lane & 15, g4 = lane >> 4;
    // ---- requests: scales and the first 32 ranks
    float rs[TM];
    v4f cs[TN], pa[TM][2];
    v4u pb[TN][B_BF16 ? 1 : 2];                                   // eight bf16 or fp32 values of lr_b
    auto request = [&](int c0) {
        const int kb = c0 + 8 * g4 < a.lr_rank ? c0 + 8 * g4 : 0; // the rank is a multiple of 8
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t row = at.row0 + 16 * i;
            const v4f* p = reinterpret_cast<const v4f*>(a.lr_a + (row < a.M ? row : a.M - 1) * a.lr_rank + kb);
            pa[i][0] = p[0];
            pa[i][1] = p[1];
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t col = at.col(j) - 4 * g4 + l16, at_b = (col < a.N ? col : a.N - 1) * a.lr_rank + kb;
            if constexpr (B_BF16) {
                pb[j][0] = *reinterpret_cast<const v4u*>(reinterpret_cast<const uint16_t*>(a.lr_b) + at_b);
            } else {
                const v4u* p = reinterpret_cast<const v4u*>(reinterpret_cast<const float*>(a.lr_b) + at_b);
                pb[j][0] = p[0];
                pb[j][1] = p[1];
            }
        }
    };
    const float post = a.post_scale ? *a.post_scale : 1.0f;                          // x * 1.0f is x
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t row = at.row0 + 16 * i;
        rs[i] = a.row_scale ? a.row_scale[row < a.M ? row : a.M - 1] : 1.0f;
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) cs[j] = (v4f){1.0f, 1.0f, 1.0f, 1.0f};
    if (a.col_scale) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const float* p = a.col_scale + (at.col(j) < a.N ? at.col(j) : 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) cs[j][e] = p[e];
        }
    }
    request(0);
    // ---- the scaled accumulators
    StaticFor<0, TN>::run([&](auto jj) {
        constexpr int j = decltype(jj)::value;
        __builtin_amdgcn_sched_barrier(0);
        hold_accumulators<TM * TN>();
        StaticFor<0, TM>::run([&](auto ii) {
            constexpr int t = decltype(ii)::value * TN + j;
            v4i x = read_acc<t>();
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = __float_as_int((((float)x[r] * rs[decltype(ii)::value]) * cs[j][r]) * post);
            write_acc<t>(x);
        });
    });
    // ---- the low-rank sum
    auto hi16 = [](uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); };
    auto split8 = [&](const v4f& x0, const v4f& x1, bool in, v8bf& h, v8bf& m, v8bf& l) {
        uint32_t ph[8], pm[8], pl[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = in ? (e < 4 ? x0[e & 3] : x1[e & 3]) : 0.0f;
            ph[e] = __float_as_uint(x) & 0xFFFF0000u;
            const float r1 = x - __uint_as_float(ph[e]);
            pm[e] = __float_as_uint(r1) & 0xFFFF0000u;
            pl[e] = __float_as_uint(r1 - __uint_as_float(pm[e]));
        }
        h = __builtin_bit_cast(v8bf, (v4u){hi16(ph[0], ph[1]), hi16(ph[2], ph[3]), hi16(ph[4], ph[5]), hi16(ph[6], ph[7])});
        m = __builtin_bit_cast(v8bf, (v4u){hi16(pm[0], pm[1]), hi16(pm[2], pm[3]), hi16(pm[4], pm[5]), hi16(pm[6], pm[7])});
        l = __builtin_bit_cast(v8bf, (v4u){hi16(pl[0], pl[1]), hi16(pl[2], pl[3]), hi16(pl[4], pl[5]), hi16(pl[6], pl[7])});
    };
    for (int c0 = 0;;) {
        const bool k_ok = c0 + 8 * g4 < a.lr_rank;
        v8bf ah[TM], am[TM], al[TM];
        __builtin_amdgcn_sched_barrier(0);
        hold_accumulators<TM * TN>();
#pragma unroll
        for (int i = 0; i < TM; ++i) split8(pa[i][0], pa[i][1], k_ok && at.row0 + 16 * i < a.M, ah[i], am[i], al[i]);
        StaticFor<0, TN>::run([&](auto jj) {
            constexpr int j = decltype(jj)::value;
            const bool in = k_ok && at.col(j) - 4 * g4 + l16 < a.N;
            if constexpr (B_BF16) {
                v4u raw = pb[j][0];
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[e] = in ? raw[e] : 0u;
                const v8bf bh = __builtin_bit_cast(v8bf, raw);
                StaticFor<0, TM>::run([&](auto ii) {
                    constexpr int i = decltype(ii)::value;
                    lowrank_mfma<i * TN + j>(bh, ah[i], am[i], al[i]);
                });
            } else {
                v8bf bh, bm, bl;
                split8(__builtin_bit_cast(v4f, pb[j][0]), __builtin_bit_cast(v4f, pb[j][1]), in, bh, bm, bl);
                StaticFor<0, TM>::run([&](auto ii) {
                    constexpr int i = decltype(ii)::value;
                    lowrank_mfma<i * TN + j>(bh, bm, bl, ah[i], am[i], al[i]);
                });
            }
        });
        hold_accumulators<TM * TN>();
        c0 += 32;
        if (c0 >= a.lr_rank) break;
        request(c0);
    }
    asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");             // as after the main loop
}

// ------------------------------------------------------------------------------------------------ kernel
template <class Cfg, bool TRANSB, bool LEFT, bool LR, bool RAGGED>
__device__ __forceinline__ void one_tile(const GemmArgs& a, int bid, int tiles_m, int tiles_n, unsigned char* smem) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile_m, tile_n;
    tile_of_block<Cfg::GROUP_M>(bid, tiles_m, tiles_n, tile_m, tile_n);
    const int64_t m0 = (int64_t)tile_m * Cfg::BM, n0 = (int64_t)tile_n * Cfg::BN;

    main_loop<Cfg, TRANSB, LEFT>(a, m0, n0, wave, lane, smem);
    const Place<Cfg> at(m0, n0, wave, lane, LEFT);
    if constexpr (LR) lowrank_prepare<Cfg, TRANSB>(a, at, lane);
    if constexpr (LEFT) {
        if (a.left_stages != 0) {          // uniform over the workgroup
            epilogue_left8<Cfg, LR>(a, at, wave, lane, smem);
            return;
        }
    }
    epilogue<Cfg, LR, RAGGED>(a, at, lane);
}

// LEFT: this instance also carries the epilogue that runs the low strides of a left-hand rotation.
// LR: this instance also carries the low-rank side product (lowrank_prepare).
// RAGGED: N (of either product) is not a multiple of 16.
// TN2: the second product of the launch has tiles of that width.
// The alignment: how fast these kernels run depends by up to 2 % on where in memory their instructions lie, whatever they are.  Steps of
// 2048 x 4096 x 4096, the pair of products, the same instructions: 63.8 us where the kernel began on a multiple of 32 KB, 65.2 and 65.6
// elsewhere; on another card 65.8 there, 67.1 in front of other kernels, and beginning on a multiple of 4 KB 66.7, 8 KB 65.9, 16 KB 66.9,
// 32 KB 67.0, 64 KB 66.3.
template <int TM, int TN, bool TRANSB, bool LEFT, bool LR, bool RAGGED, int TN2 = TN>
__global__ void __launch_bounds__(256, 1) __attribute__((aligned(8192)))
gemm_i8_kernel(GemmArgs a, int tiles_m, int tiles_n, GemmArgs a2, int tiles_m2, int tiles_n2, unsigned blocks1) {
    extern __shared__ __align__(16) unsigned char smem[];
    // A second, independent product may ride in the same launch (workgroups from blocks1 on): the tail and the
    // epilogue of one then overlap the main loop of the other.
    int bid = blockIdx.x;
    if (blockIdx.x >= blocks1) {
        bid -= blocks1;
        if constexpr (TN2 != TN) {
            one_tile<GemmCfg<TM, TN2, TRANSB>, TRANSB, LEFT, LR, RAGGED>(a2, bid, tiles_m2, tiles_n2, smem);
            return;
        }
        a = a2;
        tiles_m = tiles_m2;
        tiles_n = tiles_n2;
    }
    one_tile<GemmCfg<TM, TN, TRANSB>, TRANSB, LEFT, LR, RAGGED>(a, bid, tiles_m, tiles_n, smem);
}

// ------------------------------------------------------------------------------------------------ small products
template <int TM, int TN_, bool TRANSB>
__global__ void __launch_bounds__(256)
gemm_i8_small_kernel(GemmArgs a, int tiles_n, GemmArgs a2, int tiles_n2, unsigned blocks1) {
    using Cfg = SmallCfg<TM, TN_, TRANSB>;
    unsigned bid = blockIdx.x;
    if (bid >= blocks1) {                  // the second product of a paired launch
        bid -= blocks1;
        a = a2;
        tiles_n = tiles_n2;
    }
    extern __shared__ __align__(16) unsigned char smem[];
    SmallSums<Cfg> sums;
    small_sums<TM, TN_, TRANSB>(a, bid, tiles_n, smem, sums);
    using vi = typename SmallSums<Cfg>::vi;
    constexpr int EPT = SmallSums<Cfg>::EPT, VW = SmallSums<Cfg>::VW, NV = SmallSums<Cfg>::NV;
    const int64_t row = sums.row, col = sums.col;
    const auto& v = sums.v;
    if (row >= a.M || col >= a.N) return;
    const bool whole = col + EPT <= a.N;
    auto store = [&](int32_t* dst, const vi(&x)[NV]) {
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            if (whole) {
                *reinterpret_cast<vi*>(dst + VW * q) = x[q];
            } else {
#pragma unroll
                for (int e = 0; e < VW; ++e)
                    if (col + VW * q + e < a.N) dst[VW * q + e] = x[q][e];
            }
        }
    };
    if (a.acc_out) store(a.acc_out + row * a.ld_acc + col, v);
    if (!a.C) return;
    const float rs = a.row_scale ? a.row_scale[row] : 1.0f;
    vi f[NV];
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int e = 0; e < VW; ++e) {
            const int64_t c = col + VW * q + e;
            const float cs = a.col_scale ? a.col_scale[c < a.N ? c : a.N - 1] : 1.0f;
            f[q][e] = __float_as_int(((float)v[q][e] * rs) * cs);
        }
    if (a.c_is_f32) {
        store(reinterpret_cast<int32_t*>(a.C) + row * a.ldc + col, f);
        return;
    }
    uint16_t* dst = reinterpret_cast<uint16_t*>(a.C) + row * a.ldc + col;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
        uint32_t w[(VW + 1) / 2];
#pragma unroll
        for (int h = 0; h < VW / 2; ++h) w[h] = pack_bf16x2(__int_as_float(f[q][2 * h]), __int_as_float(f[q][2 * h + 1]));
        if constexpr (VW == 1) w[0] = bf16_bits(__int_as_float(f[q][0]));
        if (VW == 4 && whole) {
            *reinterpret_cast<v2u*>(dst + 4 * q) = (v2u){w[0], w[(VW - 1) / 2]};
        } else if (VW == 2 && whole) {
            *reinterpret_cast<uint32_t*>(dst + 2 * q) = w[0];
        } else {
#pragma unroll
            for (int e = 0; e < VW; ++e)
                if (col + VW * q + e < a.N) dst[VW * q + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
        }
    }
}

// One thread per output, for what the tiles do not take: K = 0 (zeros), and row pitches so large that the rows of a tile do
// not fit one buffer's 4 GiB.
__global__ void __launch_bounds__(256) gemm_i8_plain_kernel(GemmArgs a) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= a.M * a.N) return;
    const int64_t row = at / a.N, col = at % a.N;
    int acc = 0;
    for (int64_t k = 0; k < a.K; ++k)
        acc += (int)a.A[row * a.lda + k] * (int)(a.transB ? a.B[col * a.ldb + k] : a.B[k * a.ldb + col]);
    if (a.acc_out) a.acc_out[row * a.ld_acc + col] = acc;
    if (a.C) {
        const float v = ((float)acc * (a.row_scale ? a.row_scale[row] : 1.0f)) * (a.col_scale ? a.col_scale[col] : 1.0f);
        if (a.c_is_f32) reinterpret_cast<float*>(a.C)[row * a.ldc + col] = v;
        else reinterpret_cast<uint16_t*>(a.C)[row * a.ldc + col] = bf16_bits(v);
    }
}

// ------------------------------------------------------------------------------------------------ ceiling probe
// iters x 32 of the GEMM's matrix instructions per wavefront on operands read once from `operands` (4 KB: 16 bytes per lane
// and fragment, four fragments), nothing else in the loop: the rate the matrix pipes sustain on this machine for this
// operand data.
__global__ void __launch_bounds__(512) mfma_i8_probe_kernel(const int8_t* operands, int iters, int32_t* sink) {
    const int lane = threadIdx.x & 63;
    v4i f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = *reinterpret_cast<const v4i*>(operands + (i * 64 + lane) * 16);
    v4i acc[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = (v4i){0, 0, 0, 0};
    for (int it = 0; it < iters; ++it) {
#pragma unroll
        for (int m = 0; m < 32; ++m)
            acc[m / 2] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f[m % 2], f[2 + (m / 2) % 2], acc[m / 2], 0, 0, 0);
    }
    int s = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) s += acc[i][r];
    if (sink && s == 0x7fffffff) sink[0] = s;      // keeps the loop alive; practically never taken
}

// ------------------------------------------------------------------------------------------------ launch
template <int TM, int TN, bool TRANSB, bool LEFT = false, bool LR = false, bool RAGGED = false>
hipError_t launch_tiles(const GemmArgs& a, hipStream_t s, const GemmArgs* a2 = nullptr) {
    using Cfg = GemmCfg<TM, TN, TRANSB>;
    const bool wants_left = a.left_stages != 0 || (a2 && a2->left_stages != 0);
    const bool wants_lr = a.lr_rank != 0 || (a2 && a2->lr_rank != 0);
    // the left-hand epilogue exists for K-strided B and 256 x 256 tiles
    constexpr bool kLeftShape = TM == 8 && TN == 8 && !TRANSB;
    if constexpr (!LR) {
        if (wants_lr) return launch_tiles<TM, TN, TRANSB, kLeftShape, true>(a, s, a2);
    }
    if constexpr (!LEFT && !LR && kLeftShape) {
        if (wants_left) return launch_tiles<TM, TN, TRANSB, true>(a, s, a2);
    }
    if (wants_left && !LEFT) return hipErrorInvalidValue;
    const bool ragged = a.N % 16 != 0 || (a2 && a2->N % 16 != 0);
    if constexpr (!LEFT && !LR && !RAGGED) {
        if (ragged) return launch_tiles<TM, TN, TRANSB, false, false, true>(a, s, a2);
    }
    if (ragged && !RAGGED) return hipErrorInvalidValue;
    auto lr_ok = [](const GemmArgs& g) {
        if (!LR) return true;
        return g.lr_rank > 0 && g.lr_rank <= kMaxLowRank && g.lr_rank % 8 == 0 && g.lr_a && g.lr_b &&
               (g.lr_b_bf16 != 0) == TRANSB && g.C && !g.acc_out;
    };
    if (!lr_ok(a) || (a2 && !lr_ok(*a2))) return hipErrorInvalidValue;
    static std::once_flag once;
    static hipError_t attr_result = hipSuccess;
    auto kern = gemm_i8_kernel<TM, TN, TRANSB, LEFT, LR, RAGGED>;
    hipError_t e = raise_lds_limit(kern, Cfg::LDS_BYTES, &once, &attr_result);
    if (e != hipSuccess) return e;
    // the epilogue that runs the low strides of a left-hand rotation: 256-row tiles that lie inside the matrix, fp32 out
    auto left_ok = [](const GemmArgs& g) {
        if (g.left_stages == 0) return true;
        return g.left_stages == 8 && g.M % 256 == 0 && g.C && g.c_is_f32 && !g.acc_out && (!g.col_scale || g.lr_rank) &&
               g.K > 0;
    };
    if (!left_ok(a) || (a2 && !left_ok(*a2))) return hipErrorInvalidValue;
    const int tiles_m = (int)((a.M + Cfg::BM - 1) / Cfg::BM), tiles_n = (int)((a.N + Cfg::BN - 1) / Cfg::BN);
    const unsigned blocks1 = (unsigned)(tiles_m * tiles_n);
    int tiles_m2 = 0, tiles_n2 = 0;
    if (a2) {
        tiles_m2 = (int)((a2->M + Cfg::BM - 1) / Cfg::BM);
        tiles_n2 = (int)((a2->N + Cfg::BN - 1) / Cfg::BN);
    }
    GemmArgs g = a, g2 = a2 ? *a2 : a;
    g.whole_lines = bf16_whole_lines(g.M, g.N, g.ldc);
    g2.whole_lines = bf16_whole_lines(g2.M, g2.N, g2.ldc);
    hipLaunchKernelGGL(kern, dim3(blocks1 + (unsigned)(tiles_m2 * tiles_n2)), dim3(Cfg::NT), Cfg::LDS_BYTES, s, g, tiles_m,
                       tiles_n, g2, tiles_m2, tiles_n2, blocks1);
    return hipGetLastError();
}

// The first `wide` columns in tiles of 256 x 256, the others in 256 x 192 (two_widths).
hipError_t launch_two_widths(const GemmArgs& a, int64_t wide, hipStream_t s) {
    if (a.left_stages != 0 || a.lr_rank != 0 || a.N % 16 != 0 || wide % 256 != 0 || wide >= a.N) return hipErrorInvalidValue;
    static std::once_flag once;
    static hipError_t attr_result = hipSuccess;
    constexpr int lds = GemmCfg<8, 8, true>::LDS_BYTES;
    auto kern = gemm_i8_kernel<8, 8, true, false, false, false, 6>;
    hipError_t e = raise_lds_limit(kern, lds, &once, &attr_result);
    if (e != hipSuccess) return e;
    GemmArgs g = a, g2 = a;
    g.whole_lines = bf16_whole_lines(a.M, a.N, a.ldc);
    g2.whole_lines = g.whole_lines;
    g.N = wide;
    g2.N -= wide;
    g2.B += wide * a.ldb;
    if (a.col_scale) g2.col_scale += wide;
    if (a.acc_out) g2.acc_out += wide;
    if (a.C) g2.C = static_cast<char*>(a.C) + wide * (a.c_is_f32 ? 4 : 2);
    const int tiles_m = (int)((a.M + 255) / 256), n1 = (int)(wide / 256), n2 = (int)((g2.N + 191) / 192);
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles_m * (n1 + n2))), dim3(256), lds, s, g, tiles_m, n1, g2, tiles_m, n2,
                       (unsigned)(tiles_m * n1));
    return hipGetLastError();
}

template <int TM, bool TRANSB, int TN = 4>
hipError_t launch_small(const GemmArgs& a, hipStream_t s, const GemmArgs* a2 = nullptr) {
    using Cfg = SmallCfg<TM, TN, TRANSB>;
    if (a.left_stages != 0 || a.lr_rank != 0 || (a2 && (a2->left_stages != 0 || a2->lr_rank != 0))) return hipErrorInvalidValue;
    static std::once_flag once;
    static hipError_t attr_result = hipSuccess;
    auto kern = gemm_i8_small_kernel<TM, TN, TRANSB>;
    hipError_t e = raise_lds_limit(kern, Cfg::LDS_BYTES, &once, &attr_result);
    if (e != hipSuccess) return e;
    auto tiles = [](int64_t n, int t) { return (n + t - 1) / t; };
    const int64_t b1 = tiles(a.M, Cfg::BM) * tiles(a.N, Cfg::BN);
    const int64_t b2 = a2 ? tiles(a2->M, Cfg::BM) * tiles(a2->N, Cfg::BN) : 0;
    if (b1 + b2 > 0x7FFFFFFF) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kern, dim3((unsigned)(b1 + b2)), dim3(256), Cfg::LDS_BYTES, s, a, (int)tiles(a.N, Cfg::BN), a2 ? *a2 : a,
                       (int)(a2 ? tiles(a2->N, Cfg::BN) : 1), (unsigned)b1);
    return hipGetLastError();
}

template <int TM, bool TRANSB>
hipError_t launch_small_by_columns(const GemmArgs& a, hipStream_t s) {
    if constexpr (TRANSB) {
        const int columns = small_tile_columns(a);
        if (columns == 16) return launch_small<TM, true, 1>(a, s);
        if (columns == 32) return launch_small<TM, true, 2>(a, s);
    }
    return launch_small<TM, TRANSB>(a, s);
}

hipError_t launch_plain(const GemmArgs& a, hipStream_t s) {
    if (a.left_stages != 0 || a.lr_rank != 0) return hipErrorInvalidValue;
    const int64_t blocks = (a.M * a.N + 255) / 256;
    if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
    hipLaunchKernelGGL(gemm_i8_plain_kernel, dim3((unsigned)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

// K granularity of the tile configurations 0..3 that the ABI promises to refuse a K for (halo_gemm_config in halo.h).
constexpr int kStepOfConfig[4] = {64, 128, 128, 64};

template <bool TRANSB>
hipError_t launch_by_shape(const GemmArgs& a, hipStream_t s) {
    if constexpr (TRANSB) {
        const int64_t wide = two_widths(a);
        if (wide >= 0) return launch_two_widths(a, wide, s);
    }
    switch (a.config < 0 ? choose_config(a, nullptr) : a.config) {
        case 0:
        case 1: return launch_tiles<8, 8, TRANSB>(a, s);
        case 2: return launch_tiles<8, 4, TRANSB>(a, s);
        case 3:
        case 4: return launch_tiles<4, 4, TRANSB>(a, s);
        case kSmall64: return launch_small<4, TRANSB>(a, s);
        case kSmall32: return a.M <= 16 ? launch_small_by_columns<1, TRANSB>(a, s) : launch_small_by_columns<2, TRANSB>(a, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

bool gemm_config_valid(int cfg, int64_t K) {
    if (cfg == -1 || cfg == 4) return true;
    return cfg >= 0 && cfg <= 3 && K % kStepOfConfig[cfg] == 0;
}

// Two K-strided-B products in one launch (the two backward products of the layer).  Falls back to two launches when
// the shapes do not allow the shared configuration.
hipError_t launch_gemm_i8_pair(const GemmArgs& a1, const GemmArgs& a2, hipStream_t s) {
    const bool ok = !a1.transB && !a2.transB && a1.M > 0 && a1.N > 0 && a2.M > 0 && a2.N > 0 && tiles_can_run(a1) && tiles_can_run(a2) &&
                    a1.config == a2.config && (a1.config == -1 || a1.config == 0 || a1.config == 3);
    if (!ok) {
        hipError_t e = launch_gemm_i8(a1, s);
        return e != hipSuccess ? e : launch_gemm_i8(a2, s);
    }
    switch (a1.config < 0 ? choose_config(a1, &a2) : a1.config) {
        case kSmall32: return launch_small<2, false>(a1, s, &a2);
        case kSmall64: return launch_small<4, false>(a1, s, &a2);
        case kTiles128: return launch_tiles<4, 4, false>(a1, s, &a2);
        default: return launch_tiles<8, 8, false>(a1, s, &a2);
    }
}

hipError_t launch_gemm_i8(const GemmArgs& a, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    if (!tiles_can_run(a)) return launch_plain(a, s);
    return a.transB ? launch_by_shape<true>(a, s) : launch_by_shape<false>(a, s);
}

hipError_t launch_mfma_i8_probe(const int8_t* operands, int iters, int32_t* sink, hipStream_t s) {
    hipLaunchKernelGGL(mfma_i8_probe_kernel, dim3(256), dim3(512), 0, s, operands, iters, sink);
    return hipGetLastError();
}

}  // namespace halo
