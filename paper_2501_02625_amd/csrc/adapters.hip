// Low-rank adapters of many requests beside a projection that they share, and their gradients.  Token t has the adapter
// a = adapter_of[t] with U_a [rank x m], V_a [n x rank] and the scale s_a:
//   T = drop(X) U_a^T        Y = base + s_a T V_a^T
//   S = s_a E V_a            E_X = base + drop'(S U_a)       G_U = sum over a's tokens of S_t drop(X)_t       G_V = s_a sum of E_t T_t
// All matrices but T, S and the gradients are bf16; bf16 matrix instructions accumulate in fp32.  T and S stay fp32: where they are
// operands they are split exactly into three bf16 pieces, so the sums are those of fp32 products.
//
// Three kernels: thin_kernel (wide times adapter: T, S), wide_kernel (T, S times adapter: Y, E_X) and grad_kernel (sums over tokens).
// The first two take tiles of tokens as they lie; a tile is worked on once for each different adapter among its tokens, so tokens may
// come in any order and nothing has to be sorted for the forward pass.  The third takes the tokens adapter by adapter, in the order
// that group_kernel writes down.  No two adapters meet in one accumulator: what one holds (infinities, NaN) reaches its own tokens only.
#pragma clang fp contract(off)

#include "adapters.h"

namespace halo {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint16_t v2us __attribute__((ext_vector_type(2)));

__device__ __forceinline__ v4f mfma(v4u a, v4u b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// (high half of y) << 16 | (high half of x), and the same for the low halves.
__device__ __forceinline__ uint32_t pack_hi(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); }
__device__ __forceinline__ uint32_t pack_lo(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x05040100u); }

// x = hi + mid + lo exactly, each piece an fp32 value whose low 16 bits are zero (a bf16): the mantissa's top 8 bits, the next 8, the
// last 8.  An infinity is its own top piece.
__device__ __forceinline__ void split3(float x, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
    hi = __float_as_uint(x) & 0xFFFF0000u;
    const float h = __uint_as_float(hi), r = h == x ? 0.0f : x - h;
    mid = __float_as_uint(r) & 0xFFFF0000u;
    lo = __float_as_uint(r - __uint_as_float(mid));
}

__device__ __forceinline__ bool is_adapter(const AdapterPool& p, int a) { return (unsigned)a < (unsigned)p.slots; }
__device__ __forceinline__ int rank_of(const AdapterPool& p, int a) {
    if (!p.ranks) return p.max_rank;
    const int r = p.ranks[a];
    return r < 0 ? 0 : r > p.max_rank ? p.max_rank : r;
}
__device__ __forceinline__ float scale_of(const AdapterPool& p, int a) { return p.scale ? p.scale[a] : 1.0f; }

// Eight bf16 values with the dropped ones set to zero.  Per pair of random 16-bit halves: all ones where the bits are at least `least`
// (saturating difference to least - 1, at most 1, negated).
__device__ __forceinline__ v4u drop_eight(const DropoutMask& d, v4u x, uint32_t row, uint32_t group) {
    const uint4 q = dropout_bits(d, row, group);
    const uint16_t below = (uint16_t)(d.least - 1);
    const uint32_t bits[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const v2us over = __builtin_elementwise_sub_sat(__builtin_bit_cast(v2us, bits[i]), v2us{below, below});
        const v2us one = __builtin_elementwise_min(over, v2us{1, 1});
        x[i] &= __builtin_bit_cast(uint32_t, (v2us)(v2us{0, 0} - one));
    }
    return x;
}

// The tokens of a tile by their adapters.  todo: tokens (a bit each) that have one and are not done; next() takes the adapter of the first
// and all tokens that share it.
struct TileAdapters {
    int id;                  // of the lane's token
    uint64_t todo;
    __device__ __forceinline__ TileAdapters(const AdapterPool& p, int id_, bool in_tile) : id(id_) {
        todo = __ballot(in_tile && is_adapter(p, id));
    }
    __device__ __forceinline__ int next(uint64_t& mine) {
        const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
        mine = __ballot(id == a) & todo;
        todo &= ~mine;
        return a;
    }
};

// ------------------------------------------------------------------------------------------------ T and S
// part[split][t][c] = factor * sum over the split's k of in[t, k] * B_a[k, c]; B_a = U_a^T (K-contiguous) or, with KMAJOR, V_a (rows of
// max_rank).  factor: that of dropout, or with KMAJOR scale_a.  A workgroup owns 16 MT tokens and, of the different adapters among
// them, every gridDim.z-th; its wavefronts and the splits take 64-element chunks of K round robin (a chunk is one 128-byte line of every
// row).  v_mfma_f32_16x16x32_bf16: lane l supplies row (column) l % 16, elements 8 (l / 16) .. + 8; result lane l holds column l % 16,
// rows 4 (l / 16) .. + 4.  Rows of other adapters' tokens are replaced by one of the adapter's own: no line is fetched for them.
// KMAJOR: the lane loads NT neighbouring columns of eight rows at once and packs them, so instruction t covers the columns l % 16 * NT + t.
constexpr int kThinWaves = 8;

struct ThinArgs {
    AdapterPool p;
    const uint16_t* in;
    int64_t ld;
    float* part;             // [splits][b][max_rank]
    DropoutMask drop;
};

template <int NT, bool KMAJOR>
__device__ __forceinline__ void load_b(v4u (&out)[NT], const uint16_t* const (&bp)[NT], int64_t k, int R) {
    if constexpr (!KMAJOR) {
#pragma unroll
        for (int t = 0; t < NT; ++t) out[t] = *reinterpret_cast<const v4u*>(bp[t] + k);
    } else {
        const uint16_t* b = bp[0] + k * R;
        if constexpr (NT == 1) {
            uint32_t e[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) e[u] = b[u * R];
            out[0] = v4u{pack_lo(e[0], e[1]), pack_lo(e[2], e[3]), pack_lo(e[4], e[5]), pack_lo(e[6], e[7])};
        } else {
            uint32_t e[8][NT / 2];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint16_t* q = b + u * R;
                if constexpr (NT == 2) {
                    e[u][0] = *reinterpret_cast<const uint32_t*>(q);
                } else if constexpr (NT == 4) {
                    const uint2 w = *reinterpret_cast<const uint2*>(q);
                    e[u][0] = w.x; e[u][1] = w.y;
                } else {
                    const uint4 w = *reinterpret_cast<const uint4*>(q);
                    e[u][0] = w.x; e[u][1] = w.y; e[u][2] = w.z; e[u][3] = w.w;
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
                out[t] = (t & 1) ? v4u{pack_hi(e[0][t / 2], e[1][t / 2]), pack_hi(e[2][t / 2], e[3][t / 2]),
                                       pack_hi(e[4][t / 2], e[5][t / 2]), pack_hi(e[6][t / 2], e[7][t / 2])}
                                 : v4u{pack_lo(e[0][t / 2], e[1][t / 2]), pack_lo(e[2][t / 2], e[3][t / 2]),
                                       pack_lo(e[4][t / 2], e[5][t / 2]), pack_lo(e[6][t / 2], e[7][t / 2])};
        }
    }
}

template <int NT, int MT, bool KMAJOR, bool DROP>
__global__ void __launch_bounds__(64 * kThinWaves)
thin_kernel(ThinArgs g) {
    constexpr int ROWS = 16 * MT;
    __shared__ float s_part[kThinWaves][NT][4][64];      // [wavefront][rank tile][register][lane]
    __shared__ int s_id[64];
    const AdapterPool& p = g.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lr = lane & 15, kg = lane >> 4;
    const int R = p.max_rank;
    const int64_t K = KMAJOR ? p.n : p.m;
    const int64_t row0 = (int64_t)blockIdx.x * ROWS;
    const int split = blockIdx.y, splits = gridDim.y;
    float* part = g.part + (int64_t)split * p.b * R;
    // read once, so that all wavefronts go the same way
    if (wave == 0) s_id[lane] = lane < ROWS && row0 + lane < p.b ? p.adapter_of[row0 + lane] : -1;
    __syncthreads();
    TileAdapters tile(p, s_id[lane], lane < ROWS);
    if (blockIdx.z == 0) {                               // tokens without an adapter
        for (int i = threadIdx.x; i < ROWS * R; i += 64 * kThinWaves) {
            const int r = i / R;
            if (row0 + r < p.b && !is_adapter(p, s_id[r])) part[row0 * R + i] = 0.0f;
        }
    }
    for (unsigned seen = 0; tile.todo; ++seen) {
        uint64_t mine;
        const int a = tile.next(mine);
        if (seen % gridDim.z != blockIdx.z) continue;
        const int rank = rank_of(p, a);
        const int first = __builtin_ctzll(mine);
        const uint16_t* ap[MT];
        uint32_t token[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int r = i * 16 + lr;
            token[i] = (uint32_t)(row0 + ((mine >> r) & 1 ? r : first));
            ap[i] = g.in + (int64_t)token[i] * g.ld + kg * 8;
        }
        // columns beyond the pool's, or beyond the adapter's own, are replaced by the first one; their results are zero
        const uint16_t* bp[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (KMAJOR) bp[t] = p.V + (int64_t)a * p.n * R + (int64_t)(kg * 8) * R + (lr * NT < R ? lr * NT : 0);
            else bp[t] = p.U + ((int64_t)a * R + (t * 16 + lr < rank ? t * 16 + lr : 0)) * K + kg * 8;
        }
        v4f acc[MT][NT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[i][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        const int64_t step = (int64_t)splits * kThinWaves * 64;
        int64_t k0 = ((int64_t)split * kThinWaves + wave) * 64;
        for (; k0 + 64 <= K; k0 += step) {
            v4u x[MT][2], b[2][NT];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < MT; ++i) x[i][h] = *reinterpret_cast<const v4u*>(ap[i] + k0 + h * 32);
                load_b<NT, KMAJOR>(b[h], bp, k0 + h * 32, R);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (DROP) x[i][h] = drop_eight(g.drop, x[i][h], token[i], (uint32_t)((k0 + h * 32) >> 3) + kg);
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[i][t] = mfma(x[i][h], b[h][t], acc[i][t]);
                }
        }
        if (k0 < K) {                                    // the last chunk, if K is not a multiple of 64: eights beyond K are zero
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t k = k0 + h * 32;
                const bool ok = k + kg * 8 < K;
                const int64_t kc = ok ? k : -(int64_t)kg * 8;
                v4u b[NT];
                load_b<NT, KMAJOR>(b, bp, kc, R);
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (!ok) b[t] = v4u{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    v4u x = *reinterpret_cast<const v4u*>(ap[i] + kc);
                    if (DROP) x = drop_eight(g.drop, x, token[i], (uint32_t)(k >> 3) + kg);
                    if (!ok) x = v4u{0, 0, 0, 0};
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[i][t] = mfma(x, b[t], acc[i][t]);
                }
            }
        }
        const float factor = KMAJOR ? scale_of(p, a) : DROP ? g.drop.factor : 1.0f;
#pragma unroll
        for (int i = 0; i < MT; ++i) {                   // the wavefronts' sums meet in LDS and are added in wavefront order
            __syncthreads();
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) s_part[wave][t][e][lane] = acc[i][t][e];
            __syncthreads();
            for (int idx = threadIdx.x; idx < NT * 256; idx += 64 * kThinWaves) {
                const int t = idx >> 8, e = (idx >> 6) & 3, l = idx & 63;
                float sum = s_part[0][t][e][l];
#pragma unroll
                for (int w = 1; w < kThinWaves; ++w) sum += s_part[w][t][e][l];
                const int r = i * 16 + 4 * (l >> 4) + e;
                const int c = KMAJOR ? (l & 15) * NT + t : t * 16 + (l & 15);
                if (((mine >> r) & 1) && c < R) part[(row0 + r) * R + c] = c < rank ? sum * factor : 0.0f;
            }
        }
    }
}

// out = sum of the splits' parts, in order.
__global__ void __launch_bounds__(256)
thin_join_kernel(const float* part, int splits, int64_t total, float* out) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;       // total is a multiple of 8
    if (i >= total) return;
    float4 sum = *reinterpret_cast<const float4*>(part + i);
    for (int s = 1; s < splits; ++s) {
        const float4 q = *reinterpret_cast<const float4*>(part + s * total + i);
        sum.x += q.x; sum.y += q.y; sum.z += q.z; sum.w += q.w;
    }
    *reinterpret_cast<float4*>(out + i) = sum;
}

// ------------------------------------------------------------------------------------------------ Y and E_X
// out[t, f] = base[t, f] + sum over c of thin[t, c] * B_a[f, c]; B_a = scale_a V_a (c contiguous) or, with BWD, U_a^T with the mask of dropout
// on the sum.  A wavefront owns 16 MT tokens, the columns of its matrix instructions (their thin values stay in registers, split in
// pieces), and goes over blocks of features, the rows: 64 with 16-byte loads of V, or 128 columns of U, loaded eight neighbouring
// columns of eight rank rows at a time and packed, so that instruction v covers the columns 8 i + v.  Either way a lane ends up with
// runs of eight neighbouring features of one token: 16-byte loads of base and stores.
// RC: rank chunks of 32.  RC == 0 (rank up to 16): the halves of the instruction's 32 products hold the pieces (high, middle) and (low,
// nothing), two instructions instead of three.
constexpr int kWideWaves = 4;

struct WideArgs {
    AdapterPool p;
    const float* part;       // [splits][b][max_rank]
    int splits;
    float* thin;             // the sum of the parts is written here if splits > 1
    const void* base;
    int64_t ld_base;
    void* out;
    int64_t ld_out;
    DropoutMask drop;
};

template <bool F32>
__device__ __forceinline__ void add_base_and_store(const WideArgs& g, int64_t token, int64_t f, float (&y)[8]) {
    if constexpr (F32) {
        float* o = reinterpret_cast<float*>(g.out) + token * g.ld_out + f;
        if (g.base) {
            const float* q = reinterpret_cast<const float*>(g.base) + token * g.ld_base + f;
            const v4f lo = *reinterpret_cast<const v4f*>(q), hi = *reinterpret_cast<const v4f*>(q + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { y[j] += lo[j]; y[4 + j] += hi[j]; }
        }
        *reinterpret_cast<v4f*>(o) = v4f{y[0], y[1], y[2], y[3]};
        *reinterpret_cast<v4f*>(o + 4) = v4f{y[4], y[5], y[6], y[7]};
    } else {
        uint16_t* o = reinterpret_cast<uint16_t*>(g.out) + token * g.ld_out + f;
        if (g.base) {
            const v4u q = *reinterpret_cast<const v4u*>(reinterpret_cast<const uint16_t*>(g.base) + token * g.ld_base + f);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[2 * j] += __uint_as_float(q[j] << 16);
                y[2 * j + 1] += __uint_as_float(q[j] & 0xFFFF0000u);
            }
        }
        v4u w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y[2 * j + 1]) << 16;
        *reinterpret_cast<v4u*>(o) = w;
    }
}

template <int RC_, int MT, bool BWD, bool F32>
__global__ void __launch_bounds__(64 * kWideWaves)
wide_kernel(WideArgs g) {
    constexpr bool STACK = RC_ == 0;
    constexpr int RC = STACK ? 1 : RC_, NP = STACK ? 2 : 3, ROWS = 16 * MT;
    constexpr int FB = BWD ? 128 : 64;                   // features per trip
    const AdapterPool& p = g.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lr = lane & 15, kg = lane >> 4;
    const int R = p.max_rank;
    const int64_t wide = BWD ? p.m : p.n;
    const int64_t row0 = (int64_t)blockIdx.x * ROWS;
    const bool lane_token = lane < ROWS && row0 + lane < p.b;
    TileAdapters tile(p, lane_token ? p.adapter_of[row0 + lane] : -1, lane < ROWS);
    const int64_t f_first = ((int64_t)blockIdx.y * kWideWaves + wave) * FB, f_step = (int64_t)gridDim.y * kWideWaves * FB;

    // the thin values of the lane's tokens, in pieces
    const int r_lane = STACK ? 8 * (kg & 1) : 8 * kg;
    v4u bp[MT][RC][NP];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        int64_t t = row0 + i * 16 + lr;
        const bool real = t < p.b;
        if (!real) t = p.b - 1;
        const int a = __shfl(tile.id, i * 16 + lr);
        const float scale = !BWD && is_adapter(p, a) ? scale_of(p, a) : 1.0f;
#pragma unroll
        for (int c = 0; c < RC; ++c) {
            const int r = 32 * c + r_lane;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = 0.0f;
            if (r < R) {                                 // R is a multiple of eight
                const float* q = g.part + t * R + r;
                v4f lo = *reinterpret_cast<const v4f*>(q), hi = *reinterpret_cast<const v4f*>(q + 4);
                for (int s = 1; s < g.splits; ++s) {
                    q += p.b * R;
                    lo += *reinterpret_cast<const v4f*>(q);
                    hi += *reinterpret_cast<const v4f*>(q + 4);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) { x[j] = lo[j]; x[4 + j] = hi[j]; }
                if (g.splits > 1 && blockIdx.y == 0 && blockIdx.z == 0 && wave == 0 && real && !(STACK && kg > 1)) {
                    float* o = g.thin + t * R + r;
                    *reinterpret_cast<v4f*>(o) = lo;
                    *reinterpret_cast<v4f*>(o + 4) = hi;
                }
            }
            uint32_t piece[3][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) split3(x[j] * scale, piece[0][j], piece[1][j], piece[2][j]);
            v4u q[3];
#pragma unroll
            for (int k = 0; k < 3; ++k)
                q[k] = v4u{pack_hi(piece[k][0], piece[k][1]), pack_hi(piece[k][2], piece[k][3]), pack_hi(piece[k][4], piece[k][5]),
                           pack_hi(piece[k][6], piece[k][7])};
            if constexpr (STACK) {
                bp[i][c][0] = kg < 2 ? q[0] : q[1];
                bp[i][c][1] = kg < 2 ? q[2] : v4u{0, 0, 0, 0};
            } else {
#pragma unroll
                for (int k = 0; k < 3; ++k) bp[i][c][k] = q[k];
            }
        }
    }

    if (blockIdx.z == 0 && g.base != g.out) {            // tokens without an adapter: the base as it is
        const uint64_t bare = __ballot(lane_token) & ~tile.todo;
        for (uint64_t todo = bare; todo; todo &= todo - 1) {
            const int64_t t = row0 + __builtin_ctzll(todo);
            for (int64_t f0 = f_first; f0 < wide; f0 += f_step) {
                const int64_t f = f0 + 8 * lane;
                if (8 * lane >= FB || f >= wide) continue;
                float y[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                add_base_and_store<F32>(g, t, f, y);
            }
        }
    }

    for (unsigned seen = 0; tile.todo; ++seen) {
        uint64_t mine;
        const int a = tile.next(mine);
        if (seen % gridDim.z != blockIdx.z) continue;
        const int rank = rank_of(p, a);
        for (int64_t f0 = f_first; f0 < wide; f0 += f_step) {
            if constexpr (!BWD) {
                v4u v[4][RC];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    int64_t f = f0 + 32 * (q >> 1) + 8 * (lr >> 2) + 4 * (q & 1) + (lr & 3);
                    if (f >= wide) f = wide - 1;         // its results are not stored
#pragma unroll
                    for (int c = 0; c < RC; ++c) {
                        const int r = 32 * c + r_lane;
                        v[q][c] = v4u{0, 0, 0, 0};
                        if (r < rank) {
                            v[q][c] = *reinterpret_cast<const v4u*>(p.V + ((int64_t)a * p.n + f) * R + r);
                            if (r + 8 > rank) {          // the adapter's rank ends inside the eight
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    v[q][c][j] &= (r + 2 * j < rank ? 0xFFFFu : 0u) | (r + 2 * j + 1 < rank ? 0xFFFF0000u : 0u);
                            }
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    v4f acc[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        acc[q] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int c = 0; c < RC; ++c)
#pragma unroll
                            for (int k = 0; k < NP; ++k) acc[q] = mfma(v[q][c], bp[i][c][k], acc[q]);
                    }
                    if (!((mine >> (i * 16 + lr)) & 1)) continue;
                    const int64_t t = row0 + i * 16 + lr;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int64_t f = f0 + 32 * h + 8 * kg;
                        if (f >= wide) continue;
                        float y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = acc[2 * h + (j >> 2)][j & 3];
                        add_base_and_store<F32>(g, t, f, y);
                    }
                }
            } else {
                v4f acc[MT][8];
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int v = 0; v < 8; ++v) acc[i][v] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                int64_t col = f0 + 8 * lr;
                if (col >= wide) col = 0;                // its results are not stored
#pragma unroll
                for (int c = 0; c < RC; ++c) {
                    v4u raw[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const int r = 32 * c + r_lane + u;
                        raw[u] = v4u{0, 0, 0, 0};
                        if (r < rank) raw[u] = *reinterpret_cast<const v4u*>(p.U + ((int64_t)a * R + r) * wide + col);
                    }
#pragma unroll
                    for (int v = 0; v < 8; ++v) {
                        const int d = v >> 1;
                        const v4u x = (v & 1) ? v4u{pack_hi(raw[0][d], raw[1][d]), pack_hi(raw[2][d], raw[3][d]),
                                                    pack_hi(raw[4][d], raw[5][d]), pack_hi(raw[6][d], raw[7][d])}
                                              : v4u{pack_lo(raw[0][d], raw[1][d]), pack_lo(raw[2][d], raw[3][d]),
                                                    pack_lo(raw[4][d], raw[5][d]), pack_lo(raw[6][d], raw[7][d])};
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int k = 0; k < NP; ++k) acc[i][v] = mfma(x, bp[i][c][k], acc[i][v]);
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (!((mine >> (i * 16 + lr)) & 1)) continue;
                    const int64_t t = row0 + i * 16 + lr;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t f = f0 + 8 * (4 * kg + e);
                        if (f >= wide) continue;
                        float y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = acc[i][j][e];
                        if (g.drop.least) {
                            const uint4 bits = dropout_bits(g.drop, (uint32_t)t, (uint32_t)(f >> 3));
#pragma unroll
                            for (int j = 0; j < 8; ++j) y[j] = dropout_kept(g.drop, bits, j) ? y[j] * g.drop.factor : 0.0f;
                        }
                        add_base_and_store<F32>(g, t, f, y);
                    }
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ adapter gradients
// Tokens adapter by adapter.  order: the tokens that have an adapter, by adapter and then by index; start[a] .. start[a + 1]: those of a.
// A cut is a multiple of `chunk` in that order; a piece is what one adapter has between cuts, so adapter a's pieces are
// 1 + (cuts strictly inside its range), at least one even without tokens.  Piece i of adapter a has the index
// a + start[a] / chunk + i: at most slots + b / chunk of them, in order, none shared; indices that no adapter takes hold no tokens.
struct Piece {
    int adapter;             // -1: no piece
    int begin, end;          // in `order`
    int part;                // where its sum goes: -1: it is the adapter's only piece, straight to the result
};

// A workgroup per adapter: finds its tokens, writes them down and its pieces.  A piece that is not alone begins or ends at a cut k: its
// sum goes to part k (it begins there) or cuts + k (it is the first one, and ends there).
constexpr int kGroupThreads = 1024;

__global__ void __launch_bounds__(kGroupThreads)
group_kernel(AdapterPool p, int chunk, int* order, int* start, Piece* pieces) {
    __shared__ int s_less[kGroupThreads / 64], s_same[kGroupThreads / 64];
    const int a = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = (int)p.b, cuts = (b + chunk - 1) / chunk;
    int less = 0, same = 0;
    for (int t = tid; t < b; t += kGroupThreads) {
        const int id = p.adapter_of[t];
        less += id >= 0 && id < a;
        same += id == a;
    }
    for (int h = 32; h > 0; h >>= 1) { less += __shfl_xor(less, h); same += __shfl_xor(same, h); }
    if (lane == 0) { s_less[wave] = less; s_same[wave] = same; }
    __syncthreads();
    less = same = 0;
    for (int w = 0; w < kGroupThreads / 64; ++w) { less += s_less[w]; same += s_same[w]; }
    const int begin = less, end = less + same;
    if (tid == 0) {
        start[a] = begin;
        if (a == p.slots - 1) start[p.slots] = end;
    }
    const int count = same ? (end + chunk - 1) / chunk - begin / chunk : 1;
    const int index = a + begin / chunk, next = a == p.slots - 1 ? p.slots + cuts : a + 1 + end / chunk;
    for (int i = tid; index + i < next; i += kGroupThreads) {
        Piece q{-1, 0, 0, -1};
        if (i < count) {
            const int cut = begin / chunk + i;           // the piece lies between this cut and the next
            q.adapter = a;
            q.begin = i == 0 ? begin : cut * chunk;
            q.end = i == count - 1 ? end : (cut + 1) * chunk;
            q.part = count == 1 ? -1 : i == 0 ? cuts + cut + 1 : cut;
        }
        pieces[index + i] = q;
    }
    int at = begin;
    for (int t0 = 0; t0 < b && same > 0; t0 += kGroupThreads) {
        const int t = t0 + tid;
        const bool hit = t < b && p.adapter_of[t] == a;
        const uint64_t hits = __ballot(hit);
        __syncthreads();
        if (lane == 0) s_same[wave] = __builtin_popcountll(hits);
        __syncthreads();
        int before = 0, all = 0;
        for (int w = 0; w < kGroupThreads / 64; ++w) {
            before += w < wave ? s_same[w] : 0;
            all += s_same[w];
        }
        const int to = at + before + __builtin_popcountll(hits & ((1ull << lane) - 1));
        if (hit && to < end) order[to] = t;
        at += all;
    }
}

// The sum over a piece's tokens of big[t, col] * small[t, c]: big bf16 (E for G_V, drop(X) for G_U), small fp32 (T, S).  A workgroup owns 128
// columns of `big`; its four wavefronts take groups of 32 tokens round robin.  v_mfma_f32_16x16x32_bf16 with k = token: lane l supplies,
// for row (A) / column (B) l % 16, the eight tokens 8 (l / 16) .. + 8 of the group.  `big` is read eight neighbouring columns of a token at a
// time; the v-th of them, packed over the eight tokens, is the A operand of the v-th instruction, which covers the columns 8 i + v.
// `small` is split in three pieces.  NT: rank tiles of 16, from column `c_base` on.
constexpr int kGradWaves = 4;

struct GradJob {
    const uint16_t* big;
    int64_t ld;
    const float* small;
    float* out;              // [slots][wide x R], or [slots][R x wide] with rank_major
    float* part;             // [parts] of the same
    int64_t wide;
    int tiles;               // of 128 columns; 0: no such job
    int rank_major;          // G_U
};
struct GradArgs {
    AdapterPool p;
    GradJob job[2];          // G_V, G_U
    const int* order;
    const Piece* pieces;
    DropoutMask drop;
};

template <int NT>
__global__ void __launch_bounds__(64 * kGradWaves)
grad_kernel(GradArgs g) {
    __shared__ float s_sum[kGradWaves][32][64];          // one rank tile of every wavefront: [v * 4 + e][lane]
    const Piece piece = g.pieces[blockIdx.y];
    if (piece.adapter < 0) return;
    const bool second = (int)blockIdx.x >= g.job[0].tiles;
    const GradJob& job = g.job[second ? 1 : 0];
    const AdapterPool& p = g.p;
    const int R = p.max_rank, c_base = blockIdx.z * (16 * NT);
    const int64_t wide = job.wide;
    const int64_t c0 = (int64_t)((int)blockIdx.x - (second ? g.job[0].tiles : 0)) * 128;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i16 = lane & 15, kq = lane >> 4;
    const int64_t col = c0 + 8 * i16;
    const int64_t colc = col < wide ? col : 0;           // columns beyond the matrix are not stored
    const int rank = rank_of(p, piece.adapter);
    const bool masked = second && g.drop.least != 0;
    const uint16_t* big = job.big;
    const float* small = job.small;

    v4f acc[NT][8];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 8; ++v) acc[t][v] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int t0 = piece.begin + wave * 32; t0 < piece.end; t0 += kGradWaves * 32) {
        v4u raw[8];
        float sv[NT][8];
        int token[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int at = t0 + 8 * kq + u;
            const int t = g.order[at < piece.end ? at : piece.end - 1];
            token[u] = (unsigned)t < (unsigned)p.b ? t : 0;      // adapter_of may have changed under way; nothing is read beyond the matrices
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            raw[u] = *reinterpret_cast<const v4u*>(big + token[u] * job.ld + colc);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int c = c_base + t * 16 + i16;
                sv[t][u] = small[(int64_t)token[u] * R + (c < R ? c : 0)];
            }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (masked) raw[u] = drop_eight(g.drop, raw[u], (uint32_t)token[u], (uint32_t)(colc >> 3));
            if (t0 + 8 * kq + u >= piece.end) {          // tokens beyond the piece count as zero
                raw[u] = v4u{0, 0, 0, 0};
#pragma unroll
                for (int t = 0; t < NT; ++t) sv[t][u] = 0.0f;
            }
        }
        v4u bp[NT][3];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            uint32_t q[3][8];
#pragma unroll
            for (int u = 0; u < 8; ++u) split3(sv[t][u], q[0][u], q[1][u], q[2][u]);
#pragma unroll
            for (int k = 0; k < 3; ++k)
                bp[t][k] = v4u{pack_hi(q[k][0], q[k][1]), pack_hi(q[k][2], q[k][3]), pack_hi(q[k][4], q[k][5]), pack_hi(q[k][6], q[k][7])};
        }
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            const int d = v >> 1;
            const v4u a = (v & 1) ? v4u{pack_hi(raw[0][d], raw[1][d]), pack_hi(raw[2][d], raw[3][d]), pack_hi(raw[4][d], raw[5][d]),
                                        pack_hi(raw[6][d], raw[7][d])}
                                  : v4u{pack_lo(raw[0][d], raw[1][d]), pack_lo(raw[2][d], raw[3][d]), pack_lo(raw[4][d], raw[5][d]),
                                        pack_lo(raw[6][d], raw[7][d])};
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int k = 0; k < 3; ++k) acc[t][v] = mfma(a, bp[t][k], acc[t][v]);
        }
    }
    // The wavefronts' sums meet in LDS, one rank tile at a time, and are added in wavefront order; wavefront w then stores the columns
    // v = 2 w, 2 w + 1 of every eight.
    const float factor = second ? (masked ? g.drop.factor : 1.0f) : scale_of(p, piece.adapter);
    float* dst = piece.part < 0 ? job.out + (int64_t)piece.adapter * wide * R : job.part + (int64_t)piece.part * wide * R;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (t > 0) __syncthreads();
#pragma unroll
        for (int v = 0; v < 8; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_sum[wave][v * 4 + e][lane] = acc[t][v][e];
        __syncthreads();
        const int c = c_base + t * 16 + i16;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float o[2];
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const int q = (2 * wave + d) * 4 + e;
                float sum = s_sum[0][q][lane];
#pragma unroll
                for (int w = 1; w < kGradWaves; ++w) sum += s_sum[w][q][lane];
                o[d] = c < rank ? sum * factor : 0.0f;
            }
            const int64_t oc = c0 + 8 * (4 * kq + e) + 2 * wave;
            if (oc >= wide || c >= R) continue;
            if (job.rank_major) {
                *reinterpret_cast<float2*>(dst + (int64_t)c * wide + oc) = make_float2(o[0], o[1]);
            } else {
                dst[oc * R + c] = o[0];
                dst[(oc + 1) * R + c] = o[1];
            }
        }
    }
}

// Adds up the pieces of every adapter that has several, in order; four neighbouring elements per thread.
__global__ void __launch_bounds__(256)
grad_join_kernel(AdapterPool p, int chunk, const int* start, GradJob v, GradJob u) {
    const int a = blockIdx.y;
    const int begin = start[a], end = start[a + 1], cuts = ((int)p.b + chunk - 1) / chunk;
    const int first = begin / chunk, count = end > begin ? (end + chunk - 1) / chunk - first : 1;
    if (count == 1) return;
    const int64_t size_v = v.tiles ? v.wide * p.max_rank : 0, size_u = u.tiles ? u.wide * p.max_rank : 0;
    int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= size_v + size_u) return;
    const bool second = i >= size_v;
    if (second) i -= size_v;
    const GradJob& job = second ? u : v;
    const int64_t size = second ? size_u : size_v;
    float4 sum = *reinterpret_cast<const float4*>(job.part + (int64_t)(cuts + first + 1) * size + i);
    for (int k = 1; k < count; ++k) {
        const float4 q = *reinterpret_cast<const float4*>(job.part + (int64_t)(first + k) * size + i);
        sum.x += q.x; sum.y += q.y; sum.z += q.z; sum.w += q.w;
    }
    *reinterpret_cast<float4*>(job.out + (int64_t)a * size + i) = sum;
}

// ------------------------------------------------------------------------------------------------ launches
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round256(size_t v) { return (v + 255) & ~size_t(255); }

// How thin_kernel is laid over b tokens, a reduction of K and the adapters.
struct ThinPlan {
    int mt;                  // token tiles of 16 per workgroup
    int lanes;               // workgroups that share a tile's different adapters
    int splits;              // of K
};

ThinPlan thin_plan(int64_t b, int64_t K, int slots, int max_rank) {
    ThinPlan q;
    q.mt = b >= 4096 ? (max_rank <= 64 ? 4 : 2) : 1;
    const int64_t tiles = ceil_div(b, 16 * q.mt);
    int64_t most = 16;                                   // different adapters in a tile of 16
    if (b < most) most = b;
    if (slots < most) most = slots;
    q.lanes = b <= 256 ? (int)most : 1;
    const int64_t chunks = ceil_div(K, 64 * kThinWaves);
    int64_t splits = 512 / (tiles * q.lanes > 0 ? tiles * q.lanes : 1);
    if (splits > 8) splits = 8;
    if (splits > chunks) splits = chunks;
    q.splits = splits < 1 ? 1 : (int)splits;
    return q;
}

template <int NT, int MT, bool KMAJOR>
void launch_thin_as(const ThinArgs& g, const ThinPlan& q, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div(g.p.b, 16 * MT), q.splits, q.lanes), block(64 * kThinWaves);
    if (!KMAJOR && g.drop.least)
        hipLaunchKernelGGL((thin_kernel<NT, MT, KMAJOR, !KMAJOR>), grid, block, 0, s, g);
    else
        hipLaunchKernelGGL((thin_kernel<NT, MT, KMAJOR, false>), grid, block, 0, s, g);
}

template <bool KMAJOR>
hipError_t launch_thin(const ThinArgs& g, const ThinPlan& q, hipStream_t s) {
    const int R = g.p.max_rank;
    const bool big = q.mt > 1;
    if (R <= 16) big ? launch_thin_as<1, 4, KMAJOR>(g, q, s) : launch_thin_as<1, 1, KMAJOR>(g, q, s);
    else if (R <= 32) big ? launch_thin_as<2, 4, KMAJOR>(g, q, s) : launch_thin_as<2, 1, KMAJOR>(g, q, s);
    else if (R <= 64) big ? launch_thin_as<4, 4, KMAJOR>(g, q, s) : launch_thin_as<4, 1, KMAJOR>(g, q, s);
    else big ? launch_thin_as<8, 2, KMAJOR>(g, q, s) : launch_thin_as<8, 1, KMAJOR>(g, q, s);
    return hipGetLastError();
}

template <int RC, int MT, bool BWD>
void launch_wide_as(const WideArgs& g, int f32, int lanes, hipStream_t s) {
    const int64_t wide = BWD ? g.p.m : g.p.n, tiles = ceil_div(g.p.b, 16 * MT);
    const int64_t blocks = ceil_div(wide, (BWD ? 128 : 64) * kWideWaves);
    // as many workgroups as fill the chip twice over, each with several blocks of features where there are more
    int64_t y = ceil_div(2048, tiles * lanes);
    if (y > blocks) y = blocks;
    y = ceil_div(blocks, ceil_div(blocks, y));
    const dim3 grid((unsigned)tiles, (unsigned)y, lanes), block(64 * kWideWaves);
    if (f32) hipLaunchKernelGGL((wide_kernel<RC, MT, BWD, true>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((wide_kernel<RC, MT, BWD, false>), grid, block, 0, s, g);
}

template <bool BWD>
hipError_t launch_wide(const WideArgs& g, int f32, int lanes, hipStream_t s) {
    const int R = g.p.max_rank;
    const bool big = g.p.b > 512;
    if (R <= 16) big ? launch_wide_as<0, BWD ? 2 : 4, BWD>(g, f32, lanes, s) : launch_wide_as<0, 1, BWD>(g, f32, lanes, s);
    else if (R <= 32) big ? launch_wide_as<1, BWD ? 2 : 4, BWD>(g, f32, lanes, s) : launch_wide_as<1, 1, BWD>(g, f32, lanes, s);
    else if (R <= 64) big ? launch_wide_as<2, BWD ? 2 : 4, BWD>(g, f32, lanes, s) : launch_wide_as<2, 1, BWD>(g, f32, lanes, s);
    else big ? launch_wide_as<4, 2, BWD>(g, f32, lanes, s) : launch_wide_as<4, 1, BWD>(g, f32, lanes, s);
    return hipGetLastError();
}

// Tokens between two cuts of the gradient sums: few enough that the column tiles fill the chip, so many that the partial sums stay small
// next to what is read for them.
int grad_chunk(int64_t b, int64_t m, int64_t n, int max_rank) {
    const int64_t tiles = ceil_div(m, 128) + ceil_div(n, 128);
    int64_t chunk = ceil_div(b * tiles, 1024), least = 8 * max_rank < 256 ? 256 : 8 * max_rank;
    if (chunk < least) chunk = least;
    return (int)(ceil_div(chunk, 128) * 128);
}

struct BwdLayout {
    size_t part, thin, order, start, pieces, part_v, part_u, total;
    int chunk, cuts;
    ThinPlan plan;
};

BwdLayout bwd_layout(int64_t b, int64_t m, int64_t n, int slots, int R) {
    BwdLayout L;
    L.plan = thin_plan(b, n, slots, R);
    L.chunk = grad_chunk(b, m, n, R);
    L.cuts = (int)ceil_div(b, L.chunk);
    size_t at = 0;
    const auto take = [&at](size_t bytes) { const size_t here = at; at += round256(bytes); return here; };
    L.part = take((size_t)L.plan.splits * b * R * 4);
    L.thin = L.plan.splits > 1 ? take((size_t)b * R * 4) : L.part;
    L.order = take((size_t)b * 4);
    L.start = take(((size_t)slots + 1) * 4);
    L.pieces = take(((size_t)slots + L.cuts) * sizeof(Piece));
    const size_t parts = L.cuts > 1 ? 2 * (size_t)L.cuts + 1 : 0;
    L.part_v = take(parts * n * R * 4);
    L.part_u = take(parts * m * R * 4);
    L.total = at;
    return L;
}

}  // namespace

size_t adapters_fwd_workspace(int64_t b, int64_t m, int64_t, int slots, int max_rank) {
    const ThinPlan q = thin_plan(b, m, slots, max_rank);
    return q.splits > 1 ? round256((size_t)q.splits * b * max_rank * 4) : 0;
}

size_t adapters_bwd_workspace(int64_t b, int64_t m, int64_t n, int slots, int max_rank) {
    return bwd_layout(b, m, n, slots, max_rank).total;
}

hipError_t launch_adapters_fwd(const AdaptersFwd& a, hipStream_t s) {
    const AdapterPool& p = a.pool;
    const ThinPlan q = thin_plan(p.b, p.m, p.slots, p.max_rank);
    float* part = q.splits > 1 ? reinterpret_cast<float*>(a.workspace) : a.T;
    hipError_t e = launch_thin<false>(ThinArgs{p, a.X, a.ld_x, part, a.drop}, q, s);
    if (e != hipSuccess) return e;
    return launch_wide<false>(WideArgs{p, part, q.splits, a.T, a.base, a.ld_base, a.Y, a.ld_y, a.drop}, a.out_f32, q.lanes, s);
}

hipError_t launch_adapters_bwd(const AdaptersBwd& a, hipStream_t s) {
    const AdapterPool& p = a.pool;
    const int64_t b = p.b;
    const BwdLayout L = bwd_layout(b, p.m, p.n, p.slots, p.max_rank);
    unsigned char* ws = reinterpret_cast<unsigned char*>(a.workspace);
    float *part = reinterpret_cast<float*>(ws + L.part), *S = reinterpret_cast<float*>(ws + L.thin);
    hipError_t e = hipSuccess;
    if (b > 0 && (a.EX || a.GU)) {
        e = launch_thin<true>(ThinArgs{p, a.E, a.ld_e, part, DropoutMask{}}, L.plan, s);
        if (e != hipSuccess) return e;
    }
    if (b > 0 && a.EX) {
        e = launch_wide<true>(WideArgs{p, part, L.plan.splits, S, a.base, a.ld_base, a.EX, a.ld_ex, a.drop}, a.out_f32, L.plan.lanes, s);
        if (e != hipSuccess) return e;
    } else if (b > 0 && a.GU && L.plan.splits > 1) {
        const int64_t total = b * p.max_rank;
        hipLaunchKernelGGL(thin_join_kernel, dim3((unsigned)ceil_div(total, 1024)), dim3(256), 0, s, part, L.plan.splits, total, S);
    }
    if (!a.GU && !a.GV) return hipGetLastError();
    int *order = reinterpret_cast<int*>(ws + L.order), *start = reinterpret_cast<int*>(ws + L.start);
    Piece* pieces = reinterpret_cast<Piece*>(ws + L.pieces);
    hipLaunchKernelGGL(group_kernel, dim3(p.slots), dim3(kGroupThreads), 0, s, p, L.chunk, order, start, pieces);
    GradArgs g{};
    g.p = p; g.order = order; g.pieces = pieces; g.drop = a.drop;
    if (a.GV) g.job[0] = GradJob{a.E, a.ld_e, a.T, a.GV, reinterpret_cast<float*>(ws + L.part_v), p.n, (int)ceil_div(p.n, 128), 0};
    if (a.GU) g.job[1] = GradJob{a.X, a.ld_x, S, a.GU, reinterpret_cast<float*>(ws + L.part_u), p.m, (int)ceil_div(p.m, 128), 1};
    const int R = p.max_rank, nt = R <= 16 ? 1 : R <= 32 ? 2 : 4;
    const dim3 grid(g.job[0].tiles + g.job[1].tiles, p.slots + L.cuts, (unsigned)ceil_div(R, 16 * nt)), block(64 * kGradWaves);
    if (nt == 1) hipLaunchKernelGGL(grad_kernel<1>, grid, block, 0, s, g);
    else if (nt == 2) hipLaunchKernelGGL(grad_kernel<2>, grid, block, 0, s, g);
    else hipLaunchKernelGGL(grad_kernel<4>, grid, block, 0, s, g);
    if (L.cuts > 1) {
        const int64_t size = ((a.GV ? p.n : 0) + (a.GU ? p.m : 0)) * R;
        hipLaunchKernelGGL(grad_join_kernel, dim3((unsigned)ceil_div(size, 1024), p.slots), dim3(256), 0, s, p, L.chunk, start, g.job[0], g.job[1]);
    }
    return hipGetLastError();
}

}  // namespace halo
