// What the kernels of the low-rank adapters share (adapters_thin.hip, adapters_wide.hip, adapters_grad.hip).
//
// Token t has the adapter a = adapter_of[t] with U_a [rank x m], V_a [n x rank] and the scale s_a:
//   T = drop(X) U_a^T        Y = base + s_a T V_a^T
//   S = s_a E V_a            E_X = base + drop'(S U_a)       G_U = sum over a's tokens of S_t drop(X)_t       G_V = s_a sum of E_t T_t
// All matrices but T, S and the gradients are bf16; bf16 matrix instructions accumulate in fp32.  T and S stay fp32: where they are
// operands they are split exactly into three bf16 pieces (or four), so the sums are those of fp32 products.
//
// The kernels of T, S, Y and E_X take tiles of tokens as they lie; a tile is worked on once for each different adapter among its tokens, so
// tokens may come in any order and nothing has to be sorted.  The gradients' kernel takes the tokens adapter by adapter, in an order that is
// written down first.  No two adapters meet in one accumulator: what one holds (infinities, NaN) reaches its own tokens only.
//
// v_mfma_f32_16x16x32_bf16: lane l supplies row (first operand) or column (second) l % 16, elements 8 (l / 16) .. + 8 of the 32 that are
// summed over; result lane l holds column l % 16, rows 4 (l / 16) .. + 4.
//
// Loads wait in the order in which they were issued, and where a load may or may not have been issued the compiler waits for all before it.  So
// loads ahead of use always happen, at a place that is clamped to one that exists, and never move from register to register.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "adapters.h"
#include "adapters_plan.h"

namespace halo {
namespace adapters {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4f mfma(v4u a, v4u b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// (high half of y) << 16 | (high half of x), and the same for the low halves.
__device__ __forceinline__ uint32_t pack_hi(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); }
__device__ __forceinline__ uint32_t pack_lo(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x05040100u); }

// Eight rows of four neighbouring bf16 values, two dwords each, become four columns of eight.
__device__ __forceinline__ void columns_of(const uint2 (&x)[8], v4u (&y)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        y[0][e] = pack_lo(x[2 * e].x, x[2 * e + 1].x);
        y[1][e] = pack_hi(x[2 * e].x, x[2 * e + 1].x);
        y[2][e] = pack_lo(x[2 * e].y, x[2 * e + 1].y);
        y[3][e] = pack_hi(x[2 * e].y, x[2 * e + 1].y);
    }
}

// x as the sum of N = 3 or 4 pieces, each an fp32 value whose low 16 bits are zero (a bf16), exactly, but for what lies below 2^-133, the
// least bf16.  The pieces have x's sign, and none of them is zero unless x is (below 2^-110 the last may be): each but the last is the largest
// bf16 whose magnitude lies below what is left.  So a factor that is infinite makes an infinity of every piece, and an infinite x is two
// (three) times the largest bf16 and an infinity.  With pieces cut off at the bits of x, of which all but one may be zero, an infinite factor
// times zero would be NaN.
template <int N>
__device__ __forceinline__ void split(float x, uint32_t (&piece)[N]) {
    x += 0.0f;                                           // -0 becomes 0: below it there is nothing
#pragma unroll
    for (int k = 0; k + 1 < N; ++k) {
        piece[k] = __builtin_elementwise_sub_sat(__float_as_uint(x), 1u) & 0xFFFF0000u;
        x -= __uint_as_float(piece[k]);
    }
    piece[N - 1] = __float_as_uint(x);
}

// The pieces of eight values, as operands.
template <int N>
__device__ __forceinline__ void split_eight(const float (&x)[8], v4u (&q)[N]) {
    uint32_t piece[8][N];
#pragma unroll
    for (int e = 0; e < 8; ++e) split(x[e], piece[e]);
#pragma unroll
    for (int k = 0; k < N; ++k)
        q[k] = v4u{pack_hi(piece[0][k], piece[1][k]), pack_hi(piece[2][k], piece[3][k]), pack_hi(piece[4][k], piece[5][k]),
                   pack_hi(piece[6][k], piece[7][k])};
}

// Loads at a 32-bit byte offset from an address that is the same for the wavefront: one register of address.
template <typename V>
__device__ __forceinline__ V load_at(const void* base, uint32_t offset) {
    return *reinterpret_cast<const V*>(reinterpret_cast<const char*>(base) + offset);
}

__device__ __forceinline__ bool is_adapter(const AdapterPool& p, int a) { return (unsigned)a < (unsigned)p.slots; }
__device__ __forceinline__ int rank_of(const AdapterPool& p, int a) {
    if (!p.ranks) return p.max_rank;
    const int r = p.ranks[a];
    return r < 0 ? 0 : r > p.max_rank ? p.max_rank : r;
}
__device__ __forceinline__ float scale_of(const AdapterPool& p, int a) { return p.scale ? p.scale[a] : 1.0f; }

// Of two random 16-bit halves: 1 where they are at least `least` (saturating difference to least - 1, at most 1).  In assembly, because the
// compiler makes two compares and two selects of it: 14 instructions for the bits of eight elements, or 35.
__device__ __forceinline__ uint32_t kept_pair(uint32_t bits, uint32_t below, uint32_t one) {
    uint32_t r;
    asm("v_pk_sub_u16 %0, %1, %2 clamp\n\tv_pk_min_u16 %0, %0, %3" : "=&v"(r) : "v"(bits), "v"(below), "v"(one));
    return r;
}

// Eight bf16 values with the dropped ones set to zero.
__device__ __forceinline__ v4u drop_eight(const DropoutMask& d, v4u x, uint32_t row, uint32_t group) {
    const uint4 q = dropout_bits(d, row, group);
    const uint32_t below = (d.least - 1) * 0x10001u, bits[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t k = kept_pair(bits[i], below, 0x10001u);
        x[i] &= (k << 16) - k;                          // all ones in the halves that are 1
    }
    return x;
}

// Which of eight elements are kept, a bit each.
__device__ __forceinline__ uint32_t kept_eight(const DropoutMask& d, uint32_t row, uint32_t group) {
    const uint4 q = dropout_bits(d, row, group);
    const uint32_t below = (d.least - 1) * 0x10001u, bits[4] = {q.x, q.y, q.z, q.w};
    uint32_t kept = 0;                                   // of element 2 i in bit 2 i, of element 2 i + 1 in bit 16 + 2 i
#pragma unroll
    for (int i = 0; i < 4; ++i) kept |= kept_pair(bits[i], below, 0x10001u) << (2 * i);
    return (kept | kept >> 15) & 0xFFu;
}

// All ones where bit i is set, else zero.
__device__ __forceinline__ uint32_t bit_mask(uint32_t bits, int i) { return (uint32_t)((int32_t)(bits << (31 - i)) >> 31); }

// The mask's bits for one backward call: [blocks of 64 columns][b] words of 64, so that a token's word is eight bytes times the token from
// the block's beginning.
__host__ __device__ inline int64_t kept_words(int64_t b, int64_t m) { return (m + 63) / 64 * b; }

// Nothing is moved across: loads stay ahead of what would otherwise be drawn in front of them, or pushed behind, to save registers.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// The wavefront's place in its workgroup, in a scalar register: what is decided by it is decided for the wavefront.
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// Where the operand of lane (l % 16 = i, l / 16 = g) lies among an instruction's 64 in LDS: turned by g, so that threads that write neighbouring
// eighths of a row, one g after the other, do not meet in a bank.
__device__ __forceinline__ int operand_slot(int i, int g) { return g * 16 + (i ^ (g * 4)); }

// Of two blocks of four rows of sixteen 16-bit values in LDS, of which lane l of sixteen names the eight bytes l % 4 of row l / 4: column l, the
// first block's rows and then the second's.
__device__ __forceinline__ v4u read_transposed(const char* lo, const char* hi) {
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s* place;
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)(uintptr_t)(__attribute__((address_space(3))) const char*)lo);
    const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)(uintptr_t)(__attribute__((address_space(3))) const char*)hi);
    const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
    return v4u{x.x, x.y, y.x, y.y};
}

// Eight neighbouring values of the parts' sum, the parts in order; four of them on their way at once.
__device__ __forceinline__ void sum_parts(const float* part, int splits, int64_t size, int64_t at, v4f& lo, v4f& hi) {
    lo = hi = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 0; s0 < splits; s0 += 4) {
        v4f l[4], h[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float* q = part + (s0 + u < splits ? s0 + u : s0) * size + at;
            l[u] = *reinterpret_cast<const v4f*>(q);
            h[u] = *reinterpret_cast<const v4f*>(q + 4);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (s0 + u < splits) { lo += l[u]; hi += h[u]; }
    }
}

// ------------------------------------------------------------------------------------------------ tokens by their adapters
// The gradients take the tokens adapter by adapter.  order: places for tokens, adapter a's, by index, from range[a].x on, a multiple of 32, to
// range[a].y; a place without a token holds -1.  With `before` tokens of lower adapters the range begins at before, rounded up to 32, plus
// 32 a: so each finds its own alone, and none overlap.  places: b rounded up to 32, plus 32 slots.
// A cut is a multiple of `chunk` (of 32) of places.  An adapter's range is worked on in equal segments no longer than chunk, at least one even
// without tokens, so it has no more of them but the first than there are cuts in it.  Segment i of adapter a has the index
// a + range[a].x / chunk + i: at most slots + cuts of them, in order, none shared; indices that no adapter takes hold no adapter.  (Segments
// that end where the cuts lie are found as easily, but one may be 64 tokens long and its neighbour 2000.)
struct Segment {
    int adapter;             // -1: none
    int begin, end;          // places
    int part;                // where its sum goes: -1: it is the adapter's only segment, straight to the result
};

// The segments of an adapter with so many tokens: as few as are no longer than chunk, equally long but for the last.
struct Pieces {
    int count, size;
    __device__ __forceinline__ Pieces(int tokens, int chunk) {
        count = tokens > chunk ? (tokens + chunk - 1) / chunk : 1;
        size = ((tokens + 31) / 32 + count - 1) / count * 32;
        if (size > 0) count = (tokens + size - 1) / size;
    }
};

struct GroupArgs {
    int chunk, cuts;         // cuts: ceil(places / chunk)
    int* order;
    int2* range;             // [slots]
    Segment* segments;       // [slots + cuts]
};

// ------------------------------------------------------------------------------------------------ launches of the three files
// What a backward call does besides S in that launch: workgroups that write down the tokens by adapter (one per slot, if wanted), and such
// that draw the mask (if wanted).
struct BackwardExtras {
    GroupArgs group;
    int groups;              // slots, or 0
    uint8_t* kept;           // kept_words(b, m) words of 64 bits; null: no mask
    DropoutMask drop;
};

// T (of drop(X) and U) or, backward, S (of E and V), in `splits` parts [b x max_rank].
struct ThinPlan {
    bool rows;               // the kernel for many tokens
    int lanes;               // workgroups that share a tile's different adapters
    int splits;              // of the reduction
};
ThinPlan thin_plan(int64_t b, int64_t K, int slots);
hipError_t launch_thin(const AdapterPool& p, bool backward, const uint16_t* in, int64_t ld, float* part, const DropoutMask& drop,
                       const ThinPlan& plan, const BackwardExtras& extras, hipStream_t s);
// The extras alone.
hipError_t launch_extras(const AdapterPool& p, const BackwardExtras& extras, hipStream_t s);

struct WideArgs {
    AdapterPool p;
    const float* part;       // [splits][b][max_rank]
    int splits;
    float* thin;             // the sum of the parts is written here (not if null)
    const void* base;
    int64_t ld_base;
    void* out;
    int64_t ld_out;
    const uint8_t* kept;     // backward: BackwardExtras::kept; null: no mask
    float factor;            // and the kept elements' factor
};
hipError_t launch_wide(const WideArgs& g, bool backward, bool f32, hipStream_t s);

struct GradJob {
    const uint16_t* big;
    int64_t ld;
    const float* small;      // [b x max_rank]
    float* out;              // [slots][wide x max_rank], or [slots][max_rank x wide] with rank_major
    float* part;             // [parts] of the same
    int64_t wide;
    int tiles;               // of kGradCols columns; 0: no such job
    int rank_major;          // G_U
};
constexpr int kGradWaves = 4;
constexpr int kGradCols = 64 * kGradWaves;

struct GradArgs {
    AdapterPool p;
    GradJob job[2];          // G_V, G_U
    GroupArgs group;
    const uint8_t* kept;     // for job[1]; null: no mask
    float factor;
};
// Places between two cuts.
int grad_chunk(int64_t b, int64_t places, int64_t m, int64_t n, int max_rank);
// Sums that have a place of their own among a job's parts.
inline int64_t grad_parts(int64_t cuts) { return cuts > 1 ? 2 * cuts + 1 : 0; }
hipError_t launch_grads(const GradArgs& g, hipStream_t s);

}  // namespace adapters
}  // namespace halo
