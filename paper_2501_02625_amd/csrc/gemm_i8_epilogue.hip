// The INT8 GEMM with bias, activation and residual in its epilogue (halo_gemm_i8_epilogue):  z = (float(acc) * row_scale) * col_scale +
// bias (rounded once with the product),  C = act(z) + residual, and z itself where it is wanted for the backward pass.  Main loop and
// tiles: gemm_i8_device.h.
//
// What bounds it is the product (the chip's power) and then the arithmetic behind it, of which a compute unit does nothing else meanwhile.
// bf16 out, 8192 x 14336 x 4096: without any part of the epilogue 365 us, as the plain product; with silu and Z 386, with gelu and Z 425, on
// other cards 404 to 436 (2.26 POP/s; 8192^3 without an epilogue 2.44); a pass of its own from Z to C would be 92 us at a large copy's
// rate.  2048 x 4096 x 14336 with bias and residual 107 to 110, one row of 4096 x 4096 with them 4.5 (weights in the caches), 777 x 1003 x
// 1008 in fp32 with everything 9.6, without any part 7.8 (the plain product 7.1); there in tiles of 32 x 64 10.9, of 128 x 128 12.0.
#pragma clang fp contract(off)

#include "activation.h"
#include "gemm_i8_device.h"

namespace halo {
namespace {

// 16 bytes of a row: eight bf16 or four fp32 values.
template <bool F32>
struct Piece {
    static constexpr int W = F32 ? 4 : 8;
    __device__ __forceinline__ static float get(const v4u& q, int j) {
        if constexpr (F32) return __uint_as_float(q[j]);
        else return __uint_as_float((j & 1) ? q[j >> 1] & 0xFFFF0000u : q[j >> 1] << 16);
    }
    __device__ __forceinline__ static v4u put(const float* y) {
        v4u q;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (F32) q[i] = __float_as_uint(y[i]);
            else q[i] = pack_bf16x2(y[2 * i], y[2 * i + 1]);
        }
        return q;
    }
    // n of the values (n > 0); p: the first one's address.  PAST: past the caches, for whole lines of large matrices.
    template <bool PAST>
    __device__ __forceinline__ static void store(void* p, const v4u& q, int n) {
        if (n >= W) {
            if constexpr (PAST) __builtin_nontemporal_store(q, reinterpret_cast<v4u*>(p));
            else *reinterpret_cast<v4u*>(p) = q;
            return;
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            if (j >= n) break;
            if constexpr (F32) reinterpret_cast<uint32_t*>(p)[j] = q[j];
            else reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)(q[j >> 1] >> (16 * (j & 1)));
        }
    }
};
template <bool F32>
__device__ __forceinline__ char* address(const void* p, int64_t ld, int64_t row, int64_t col) {
    return reinterpret_cast<char*>(const_cast<void*>(p)) + (row * ld + col) * (F32 ? 4 : 2);
}
__device__ __forceinline__ float bias_at(const EpilogueArgs& e, int64_t col) {
    if (!e.bias) return 0.0f;
    if (e.bias_f32) return reinterpret_cast<const float*>(e.bias)[col];
    return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(e.bias)[col] << 16);
}
template <class F>
__device__ __forceinline__ void with_activation(int act, const F& f) {
    switch (act) {
        case HALO_ACT_RELU: f(Int<HALO_ACT_RELU>()); break;
        case HALO_ACT_GELU: f(Int<HALO_ACT_GELU>()); break;
        case HALO_ACT_GELU_TANH: f(Int<HALO_ACT_GELU_TANH>()); break;
        case HALO_ACT_SILU: f(Int<HALO_ACT_SILU>()); break;
        default: f(Int<HALO_ACT_NONE>()); break;
    }
}

// The accumulators of a wavefront go through LDS, four rows of 16 x 16 tiles at a time, so that a lane has 16 bytes of C, Z and residual
// that lie together, always of the same columns, and the code that computes them is a loop (over the accumulators, which are named
// registers, it would be as long as the tile).  The LDS belongs to the wavefront: no barrier but the first.  One wavefront per SIMD has
// nothing to hide a load behind but its own work: scales and bias are requested in front of the main loop, residuals groups of steps
// ahead.
template <class Cfg, bool F32>
struct Finish {
    using P = Piece<F32>;
    static constexpr int TM = Cfg::TM, TN = Cfg::TN, WN = Cfg::WN, W = P::W;
    static constexpr int LANES = (WN > 64 ? 128 : 64) / W, ROWS = 64 / LANES;             // lanes a row (of 96 columns, a quarter idle), rows a step
    static constexpr int PITCH = WN + 4, PARTS = TM / 4, STEPS = 64 / ROWS, AHEAD = 4, SIZE = F32 ? 4 : 2;
    // groups of steps whose residual is on its way: fp32, one / two / three, 4747 x 4096 x 512 36.2 us / 34.0 / 33.6, 8192 x 14336 x 512 with Z
    // 344 / 329 / 327; bf16, with half the bytes, 28.3 / 29.1 / 29.6 and 180 each way
    static constexpr int GROUPS = F32 ? 2 : 1;
    using Buffer = __amdgpu_buffer_rsrc_t;
    static_assert(TM % 4 == 0 && STEPS % AHEAD == 0 && 4 * 64 * PITCH * 4 <= Cfg::LDS_BYTES, "what a wavefront holds in LDS");
    float rs[TM], cs[W], bias[W];
    int64_t row0, col, col0;                 // of the wavefront's rows, the lane's columns, the tile's
    int at_row, at_col, n;                   // n: columns of the lane inside the matrix; may be negative

    __device__ __forceinline__ Finish(const GemmArgs& a, const EpilogueArgs& e, int64_t m0, int64_t n0, int wave, int lane) {
        at_row = lane / LANES;
        at_col = lane % LANES * W;
        row0 = m0 + (wave >> 1) * Cfg::WM;
        col0 = n0;
        col = n0 + (wave & 1) * 16 * Cfg::LOW_STEP + at_col;
        if (TN % 4 != 0 && at_col >= 16 * Cfg::LOW_STEP) col = n0 + Cfg::high_column(wave & 1) + at_col - 16 * Cfg::LOW_STEP;
        n = at_col >= WN ? 0 : a.N - col < W ? (int)(a.N - col) : W;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t row = row0 + 16 * i + row_of_lane(lane & 15);
            rs[i] = a.row_scale ? a.row_scale[row < a.M ? row : a.M - 1] : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const int64_t c = col + j < a.N ? col + j : a.N - 1;
            cs[j] = a.col_scale ? a.col_scale[c] : 1.0f;
            bias[j] = bias_at(e, c);
        }
        if (at_col >= WN) at_col = 0;                            // an idle lane reads LDS where another does
    }

    // A matrix of C's type from the wavefront's first row and the tile's first column on, as a buffer that ends behind the matrix' last
    // row: loads from rows behind it give zeros, stores to them nothing, and neither needs a branch.  (With branches around them the
    // compiler cannot count what is on its way, and every residual waited for all stores in front of it.)
    __device__ __forceinline__ Buffer buffer(const void* p, int64_t ld, const GemmArgs& a) const {
        const int64_t rows = a.M - row0 < Cfg::WM ? a.M - row0 : Cfg::WM;
        const uint32_t bytes = rows > 0 ? (uint32_t)(rows * ld * SIZE) : 0;
        return __builtin_amdgcn_make_buffer_rsrc(address<F32>(p, ld, row0, col0), 0, (int)bytes, 0x00020000);
    }

    template <int ACT, bool RES>
    __device__ __forceinline__ void run(const GemmArgs& a, const EpilogueArgs& e, int wave, int lane, unsigned char* smem) const {
        float* mine = reinterpret_cast<float*>(smem) + wave * (64 * PITCH);
        constexpr int PAST = 2;                                  // past the caches: 425 us, through them 458 (8192 x 14336 x 4096, gelu, Z)
        const bool partly = n > 0 && n < W, ragged = a.N % W != 0;
        const Buffer to_c = buffer(a.C, a.ldc, a), to_z = buffer(e.Z, e.ld_z, a), from_r = buffer(e.residual, e.ld_res, a);
        // where the lane's 16 bytes of the next row are; those of columns outside the matrix are outside the buffers
        uint32_t at_c = n > 0 ? (uint32_t)((at_row * a.ldc + col - col0) * SIZE) : kOutside;
        uint32_t at_z = n > 0 ? (uint32_t)((at_row * e.ld_z + col - col0) * SIZE) : kOutside;
        uint32_t at_r = n > 0 ? (uint32_t)((at_row * e.ld_res + col - col0) * SIZE) : kOutside;
        const uint32_t more_c = n > 0 ? (uint32_t)(ROWS * a.ldc * SIZE) : 0, more_z = n > 0 ? (uint32_t)(ROWS * e.ld_z * SIZE) : 0;
        const uint32_t more_r = n > 0 ? (uint32_t)(ROWS * e.ld_res * SIZE) : 0;
        v4u res[AHEAD], next[GROUPS][AHEAD];                     // this group's residual, and the following groups'
        auto request = [&](v4u(&to)[AHEAD]) {
            if constexpr (RES) {
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    to[k] = __builtin_amdgcn_raw_buffer_load_b128(from_r, (int)at_r, 0, 0);
                    at_r += more_r;
                }
            }
        };
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) request(next[g]);
        __syncthreads();                                         // every wavefront has read its last operands
#pragma unroll 1
        for (int part = 0; part < PARTS; ++part) {
            auto dump = [&](auto first) {
                StaticFor<0, 4>::run([&](auto ii) {
                    __builtin_amdgcn_sched_barrier(0);
                    hold_accumulators<TM * TN>();
                    StaticFor<0, TN>::run([&](auto jj) {
                        constexpr int i = decltype(ii)::value, j = decltype(jj)::value, row = decltype(first)::value + i;
                        const v4i x = read_acc<row * TN + j>();
                        v4f v;
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = (float)x[k] * rs[row];
                        *reinterpret_cast<v4f*>(mine + (16 * i + row_of_lane(lane & 15)) * PITCH + 16 * j + 4 * (lane >> 4)) = v;
                    });
                });
                __builtin_amdgcn_sched_barrier(0);
                hold_accumulators<TM * TN>();
            };
            if constexpr (PARTS > 1) {
                if (part) dump(Int<4>());
                else dump(Int<0>());
            } else {
                dump(Int<0>());
            }
#pragma unroll 1
            for (int step = 0; step < STEPS; step += AHEAD) {
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    res[k] = next[0][k];
#pragma unroll
                    for (int g = 1; g < GROUPS; ++g) next[g - 1][k] = next[g][k];
                }
                request(next[GROUPS - 1]);                       // behind the last rows: outside the buffer, or rows that nobody uses
                // a group of steps without a branch, so that they cover one another's latencies, and then its stores
                v4f x[AHEAD][W / 4];
                v4u zs[AHEAD], ys[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                    for (int q = 0; q < W / 4; ++q)
                        x[k][q] = *reinterpret_cast<const v4f*>(mine + ((step + k) * ROWS + at_row) * PITCH + at_col + 4 * q);
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    float z[W], y[W];
#pragma unroll
                    for (int j = 0; j < W; ++j) {
                        z[j] = __builtin_fmaf(x[k][j / 4][j % 4], cs[j], bias[j]);
                        y[j] = activation<ACT, !F32 && !RES>(z[j]);
                        if constexpr (RES) y[j] += P::get(res[k], j);
                    }
                    zs[k] = P::put(z);
                    ys[k] = P::put(y);
                }
                if (e.Z) {
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k)
                        __builtin_amdgcn_raw_buffer_store_b128(zs[k], to_z, (int)(partly ? kOutside : at_z + k * more_z), 0, PAST);
                    at_z += AHEAD * more_z;
                }
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
                    __builtin_amdgcn_raw_buffer_store_b128(ys[k], to_c, (int)(partly ? kOutside : at_c + k * more_c), 0, PAST);
                at_c += AHEAD * more_c;
                if (ragged) {                                    // uniform: some tile's columns end inside a lane's 16 bytes
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k) {
                        const int64_t row = row0 + (part * STEPS + step + k) * ROWS + at_row;
                        if (!partly || row >= a.M) continue;
                        if (e.Z) P::template store<false>(address<F32>(e.Z, e.ld_z, row, col), zs[k], n);
                        P::template store<false>(address<F32>(a.C, a.ldc, row, col), ys[k], n);
                    }
                }
            }
        }
    }
};

template <class Cfg, bool F32>
__device__ __forceinline__ void one_tile(const GemmArgs& a, const EpilogueArgs& e, int bid, int tiles_m, int tiles_n, unsigned char* smem) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile_m, tile_n;
    tile_of_block<Cfg::GROUP_M>(bid, tiles_m, tiles_n, tile_m, tile_n);
    // the divisions run in vector registers; what follows from them belongs in scalar ones
    const int64_t m0 = (int64_t)__builtin_amdgcn_readfirstlane(tile_m) * Cfg::BM;
    const int64_t n0 = (int64_t)__builtin_amdgcn_readfirstlane(tile_n) * Cfg::BN;
    const Finish<Cfg, F32> finish(a, e, m0, n0, wave, lane);
    main_loop<Cfg, true, false>(a, m0, n0, wave, lane, smem);
    with_activation(e.act, [&](auto act) {
        if (e.residual) finish.template run<decltype(act)::value, true>(a, e, wave, lane, smem);
        else finish.template run<decltype(act)::value, false>(a, e, wave, lane, smem);
    });
}

template <int TM, int TN, bool F32>
__global__ void __launch_bounds__(256, 1) __attribute__((aligned(8192)))
gemm_i8_epilogue_kernel(GemmArgs a, EpilogueArgs e, int tiles_m, int tiles_n) {
    extern __shared__ __align__(16) unsigned char smem[];
    one_tile<GemmCfg<TM, TN, true>, F32>(a, e, blockIdx.x, tiles_m, tiles_n, smem);
}

// The first columns in tiles of 256 x 256, the others (a2, e2) in 256 x 192: two_widths.
template <bool F32>
__global__ void __launch_bounds__(256, 1) __attribute__((aligned(8192)))
two_widths_gemm_i8_epilogue_kernel(GemmArgs a, EpilogueArgs e, int tiles_n, GemmArgs a2, EpilogueArgs e2, int tiles_n2, int tiles_m,
                                   unsigned blocks1) {
    extern __shared__ __align__(16) unsigned char smem[];
    if (blockIdx.x >= blocks1) one_tile<GemmCfg<8, 6, true>, F32>(a2, e2, blockIdx.x - blocks1, tiles_m, tiles_n2, smem);
    else one_tile<GemmCfg<8, 8, true>, F32>(a, e, blockIdx.x, tiles_m, tiles_n, smem);
}

template <bool F32>
__device__ __forceinline__ float load_one(const char* p) {
    if constexpr (F32) return *reinterpret_cast<const float*>(p);
    else return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
}
template <bool F32>
__device__ __forceinline__ void store_one(char* p, float x) {
    if constexpr (F32) *reinterpret_cast<float*>(p) = x;
    else *reinterpret_cast<uint16_t*>(p) = bf16_bits(x);
}
// One value: z to Z, act(z) + residual to C.
template <bool F32>
__device__ __forceinline__ void finish_one(const GemmArgs& a, const EpilogueArgs& e, int64_t row, int64_t col, float z) {
    float y = 0.0f;
    with_activation(e.act, [&](auto act) {
        if (e.residual) y = activation<decltype(act)::value, false>(z) + load_one<F32>(address<F32>(e.residual, e.ld_res, row, col));
        else y = activation<decltype(act)::value, !F32>(z);
    });
    if (e.Z) store_one<F32>(address<F32>(e.Z, e.ld_z, row, col), z);
    store_one<F32>(address<F32>(a.C, a.ldc, row, col), y);
}

// What a thread of the small kernel needs beside its sums is requested before them, and arrives while they are formed.
template <int TM, int TN, bool F32>
__global__ void __launch_bounds__(256) gemm_i8_epilogue_small_kernel(GemmArgs a, EpilogueArgs e, int tiles_n) {
    using Cfg = SmallCfg<TM, TN, true>;
    using Sums = SmallSums<Cfg>;
    using P = Piece<F32>;
    constexpr int EPT = Sums::EPT, PIECES = EPT / P::W;          // 16 bytes at a time, where there are as many
    extern __shared__ __align__(16) unsigned char smem[];
    const int64_t row = (int64_t)(blockIdx.x / tiles_n) * Cfg::BM + threadIdx.x / Sums::TPR;
    const int64_t col = (int64_t)(blockIdx.x % tiles_n) * Cfg::BN + threadIdx.x % Sums::TPR * EPT;
    const int n = row >= a.M || col >= a.N ? 0 : a.N - col < EPT ? (int)(a.N - col) : EPT;
    float cs[EPT], bias[EPT], res[EPT], rs = 1.0f;
    v4u pieces[PIECES > 0 ? PIECES : 1];
#pragma unroll
    for (int j = 0; j < EPT; ++j) {
        const int64_t c = col + j < a.N ? col + j : a.N - 1;
        cs[j] = a.col_scale ? a.col_scale[c] : 1.0f;
        bias[j] = bias_at(e, c);
        res[j] = 0.0f;
    }
    if (n > 0) {
        if (a.row_scale) rs = a.row_scale[row];
        if (e.residual) {
            if constexpr (PIECES > 0) {
#pragma unroll
                for (int q = 0; q < PIECES; ++q)
                    if (q * P::W < n) pieces[q] = *reinterpret_cast<const v4u*>(address<F32>(e.residual, e.ld_res, row, col + q * P::W));
            } else {
#pragma unroll
                for (int j = 0; j < EPT; ++j)
                    if (j < n) res[j] = load_one<F32>(address<F32>(e.residual, e.ld_res, row, col + j));
            }
        }
    }
    Sums s;
    small_sums<TM, TN, true>(a, blockIdx.x, tiles_n, smem, s);
    if (n <= 0) return;
    if constexpr (PIECES > 0) {
        if (e.residual) {
#pragma unroll
            for (int j = 0; j < EPT; ++j) res[j] = P::get(pieces[j / P::W], j % P::W);
        }
    }
    float z[EPT], y[EPT];
#pragma unroll
    for (int j = 0; j < EPT; ++j) z[j] = __builtin_fmaf((float)s.v[j / Sums::VW][j % Sums::VW] * rs, cs[j], bias[j]);
    with_activation(e.act, [&](auto act) {
        if (e.residual) {
#pragma unroll
            for (int j = 0; j < EPT; ++j) y[j] = activation<decltype(act)::value, false>(z[j]) + res[j];
        } else {
#pragma unroll
            for (int j = 0; j < EPT; ++j) y[j] = activation<decltype(act)::value, !F32>(z[j]);
        }
    });
    auto store = [&](const void* base, int64_t ld, const float* v) {
        if constexpr (PIECES > 0) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q)
                if (q * P::W < n) P::template store<false>(address<F32>(base, ld, row, col + q * P::W), P::put(v + q * P::W), n - q * P::W);
        } else {
#pragma unroll
            for (int j = 0; j < EPT; ++j)
                if (j < n) store_one<F32>(address<F32>(base, ld, row, col + j), v[j]);
        }
    };
    if (e.Z) store(e.Z, e.ld_z, z);
    store(a.C, a.ldc, y);
}

// One thread per output, for what the tiles do not take: K = 0, and row pitches so large that the rows of a tile do not fit one
// buffer.
__global__ void __launch_bounds__(256) gemm_i8_epilogue_plain_kernel(GemmArgs a, EpilogueArgs e) {
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < a.M * a.N; at += (int64_t)gridDim.x * 256) {
        const int64_t row = at / a.N, col = at % a.N;
        int acc = 0;
        for (int64_t k = 0; k < a.K; ++k) acc += (int)a.A[row * a.lda + k] * (int)a.B[col * a.ldb + k];
        const float rs = a.row_scale ? a.row_scale[row] : 1.0f, cs = a.col_scale ? a.col_scale[col] : 1.0f;
        const float z = __builtin_fmaf((float)acc * rs, cs, bias_at(e, col));
        if (a.c_is_f32) finish_one<true>(a, e, row, col, z);
        else finish_one<false>(a, e, row, col, z);
    }
}

inline int64_t tiles(int64_t n, int t) { return (n + t - 1) / t; }

template <int TM, int TN, bool F32>
hipError_t launch_tiled(const GemmArgs& a, const EpilogueArgs& e, hipStream_t s) {
    using Cfg = GemmCfg<TM, TN, true>;
    static std::once_flag once;
    static hipError_t attr_result = hipSuccess;
    auto kern = gemm_i8_epilogue_kernel<TM, TN, F32>;
    const hipError_t err = raise_lds_limit(kern, Cfg::LDS_BYTES, &once, &attr_result);
    if (err != hipSuccess) return err;
    const int tiles_m = (int)tiles(a.M, Cfg::BM), tiles_n = (int)tiles(a.N, Cfg::BN);
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles_m * tiles_n)), dim3(Cfg::NT), Cfg::LDS_BYTES, s, a, e, tiles_m, tiles_n);
    return hipGetLastError();
}

template <bool F32>
hipError_t launch_two_widths(const GemmArgs& a, const EpilogueArgs& e, int64_t wide, hipStream_t s) {
    static std::once_flag once;
    static hipError_t attr_result = hipSuccess;
    constexpr int lds = GemmCfg<8, 8, true>::LDS_BYTES;
    auto kern = two_widths_gemm_i8_epilogue_kernel<F32>;
    const hipError_t err = raise_lds_limit(kern, lds, &once, &attr_result);
    if (err != hipSuccess) return err;
    auto from = [&](const void* p, int bytes) { return p ? const_cast<char*>(static_cast<const char*>(p)) + wide * bytes : nullptr; };
    GemmArgs g = a, g2 = a;
    EpilogueArgs e2 = e;
    g.N = wide;
    g2.N -= wide;
    g2.B += wide * a.ldb;
    if (a.col_scale) g2.col_scale += wide;
    g2.C = from(a.C, F32 ? 4 : 2);
    e2.bias = from(e.bias, e.bias_f32 ? 4 : 2);
    e2.residual = from(e.residual, F32 ? 4 : 2);
    e2.Z = from(e.Z, F32 ? 4 : 2);
    const int tiles_m = (int)tiles(a.M, 256), n1 = (int)(wide / 256), n2 = (int)tiles(g2.N, 192);
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles_m * (n1 + n2))), dim3(256), lds, s, g, e, n1, g2, e2, n2, tiles_m,
                       (unsigned)(tiles_m * n1));
    return hipGetLastError();
}

template <int TM, int TN, bool F32>
hipError_t launch_split(const GemmArgs& a, const EpilogueArgs& e, hipStream_t s) {
    using Cfg = SmallCfg<TM, TN, true>;
    static std::once_flag once;
    static hipError_t attr_result = hipSuccess;
    auto kern = gemm_i8_epilogue_small_kernel<TM, TN, F32>;
    const hipError_t err = raise_lds_limit(kern, Cfg::LDS_BYTES, &once, &attr_result);
    if (err != hipSuccess) return err;
    const int64_t blocks = tiles(a.M, Cfg::BM) * tiles(a.N, Cfg::BN);
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(256), Cfg::LDS_BYTES, s, a, e, (int)tiles(a.N, Cfg::BN));
    return hipGetLastError();
}
template <int TM, bool F32>
hipError_t launch_split_by_columns(const GemmArgs& a, const EpilogueArgs& e, hipStream_t s) {
    const int columns = small_tile_columns(a);
    if (columns == 16) return launch_split<TM, 1, F32>(a, e, s);
    if (columns == 32) return launch_split<TM, 2, F32>(a, e, s);
    return launch_split<TM, 4, F32>(a, e, s);
}
template <bool F32>
hipError_t launch_by_shape(const GemmArgs& a, const EpilogueArgs& e, hipStream_t s) {
    const EpilogueWay way = epilogue_way(a);
    if (way.wide >= 0) return launch_two_widths<F32>(a, e, way.wide, s);
    switch (way.config) {
        case 0:
        case 1: return launch_tiled<8, 8, F32>(a, e, s);
        case 2: return launch_tiled<8, 4, F32>(a, e, s);
        case 3:
        case 4: return launch_tiled<4, 4, F32>(a, e, s);
        case kSmall64: return launch_split<4, 4, F32>(a, e, s);
        case kSmall32: return a.M <= 16 ? launch_split_by_columns<1, F32>(a, e, s) : launch_split_by_columns<2, F32>(a, e, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_gemm_i8_epilogue(const GemmArgs& a, const EpilogueArgs& e, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    if (!a.transB || !a.C || a.acc_out || a.left_stages || a.lr_rank) return hipErrorInvalidValue;
    // offsets from a wavefront's first row are 32-bit numbers
    const int64_t most = int64_t(1) << 22;
    if (!tiles_can_run(a) || a.ldc > most || (e.residual && e.ld_res > most) || (e.Z && e.ld_z > most)) {
        const int64_t blocks = std::min(tiles(a.M * a.N, 256), int64_t(1) << 20);
        hipLaunchKernelGGL(gemm_i8_epilogue_plain_kernel, dim3((unsigned)blocks), dim3(256), 0, s, a, e);
        return hipGetLastError();
    }
    return a.c_is_f32 ? launch_by_shape<true>(a, e, s) : launch_by_shape<false>(a, e, s);
}

}  // namespace halo
