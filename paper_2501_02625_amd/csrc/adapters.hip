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

#include <type_traits>

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

// Which of eight elements are kept, a bit each.
__device__ __forceinline__ uint32_t kept_eight(const DropoutMask& d, uint32_t row, uint32_t group) {
    const uint4 q = dropout_bits(d, row, group);
    const uint16_t below = (uint16_t)(d.least - 1);
    const uint32_t bits[4] = {q.x, q.y, q.z, q.w};
    uint32_t kept = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const v2us over = __builtin_elementwise_sub_sat(__builtin_bit_cast(v2us, bits[i]), v2us{below, below});
        const uint32_t one = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(over, v2us{1, 1}));
        kept |= ((one | one >> 15) & 3u) << (2 * i);
    }
    return kept;
}

// Four bf16 values of which those with a bit are kept.
__device__ __forceinline__ uint2 keep_four(uint2 x, uint32_t kept) {
    const auto bit = [kept](int i) { return (uint32_t)((int32_t)(kept << (31 - i)) >> 31); };    // all ones, or zero
    return make_uint2(x.x & pack_lo(bit(0), bit(1)), x.y & pack_lo(bit(2), bit(3)));
}

// Nothing is moved across: loads stay ahead of what would otherwise be drawn in front of them, or pushed behind, to save registers.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// The wavefront's place in its workgroup, in a scalar register: what is decided by it is decided for the wavefront.
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

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

// ------------------------------------------------------------------------------------------------ tokens by their adapters
// The gradients take the tokens adapter by adapter.  order: places for tokens, b + 32 (slots + 1) of them; adapter a's tokens, by index, have the
// places from range[a].x on, a multiple of 32, to range[a].y; a place without a token holds -1.  With `before` tokens of lower adapters the
// range begins at before, rounded up to 32, plus 32 a: so each finds its own alone, and none overlap.
// A cut is a multiple of `chunk` (of 32) of places; a segment is what one adapter has between cuts, so adapter a has 1 + (cuts strictly inside
// its range) of them, at least one even without tokens.  Segment i of adapter a has the index a + range[a].x / chunk + i: at most slots + cuts
// of them, in order, none shared; indices that no adapter takes hold no adapter.
struct Segment {
    int adapter;             // -1: none
    int begin, end;          // places
    int part;                // where its sum goes: -1: it is the adapter's only segment, straight to the result
};

struct GroupArgs {
    int chunk, cuts;         // cuts: ceil(places / chunk)
    int* order;
    int2* range;             // [slots]
    Segment* segments;       // [slots + cuts]
};

// One adapter's, by a workgroup.  A segment that is not alone begins or ends at a cut k: its sum goes to part k (it begins there) or cuts + k
// (it is the first one, and ends there).
template <int THREADS>
__device__ __forceinline__ void group_tokens(const AdapterPool& p, const GroupArgs& g, int a) {
    constexpr int WAVES = THREADS / 64;
    __shared__ int s_less[WAVES], s_same[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
    const int b = (int)p.b, chunk = g.chunk;
    int less = 0, same = 0;
    for (int t = tid; t < b; t += THREADS) {
        const int id = p.adapter_of[t];
        less += id >= 0 && id < a;
        same += id == a;
    }
    for (int h = 32; h > 0; h >>= 1) { less += __shfl_xor(less, h); same += __shfl_xor(same, h); }
    if (lane == 0) { s_less[wave] = less; s_same[wave] = same; }
    __syncthreads();
    less = same = 0;
    for (int w = 0; w < WAVES; ++w) { less += s_less[w]; same += s_same[w]; }
    const int begin = (less + 31) / 32 * 32 + 32 * a, end = begin + same;
    if (tid == 0) g.range[a] = make_int2(begin, end);
    const int after = (less + same + 31) / 32 * 32 + 32 * (a + 1);     // where the next adapter begins
    const int count = same ? (end + chunk - 1) / chunk - begin / chunk : 1;
    const int index = a + begin / chunk, next = a == p.slots - 1 ? p.slots + g.cuts : a + 1 + after / chunk;
    for (int i = tid; index + i < next; i += THREADS) {
        Segment q{-1, 0, 0, -1};
        if (i < count) {
            const int cut = begin / chunk + i;           // the segment lies between this cut and the next
            q.adapter = a;
            q.begin = i == 0 ? begin : cut * chunk;
            q.end = i == count - 1 ? end : (cut + 1) * chunk;
            q.part = count == 1 ? -1 : i == 0 ? g.cuts + cut + 1 : cut;
        }
        g.segments[index + i] = q;
    }
    if (tid < after - end) g.order[end + tid] = -1;      // fewer than 64 places
    if (a == 0 && tid < begin) g.order[tid] = -1;
    int at = begin;
    for (int t0 = 0; t0 < b && same > 0; t0 += THREADS) {
        const int t = t0 + tid;
        const bool hit = t < b && p.adapter_of[t] == a;
        const uint64_t hits = __ballot(hit);
        __syncthreads();
        if (lane == 0) s_same[wave] = __builtin_popcountll(hits);
        __syncthreads();
        int before = 0, all = 0;
        for (int w = 0; w < WAVES; ++w) {
            before += w < wave ? s_same[w] : 0;
            all += s_same[w];
        }
        const int to = at + before + __builtin_popcountll(hits & ((1ull << lane) - 1));
        if (hit && to < end) g.order[to] = t;
        at += all;
    }
}

__global__ void __launch_bounds__(512)
group_kernel(AdapterPool p, GroupArgs g) { group_tokens<512>(p, g, blockIdx.x); }

// ------------------------------------------------------------------------------------------------ T and S
// part[split][t][c] = factor * sum over the split's k of in[t, k] * B_a[k, c]; B_a = U_a^T (K-contiguous) or, with KMAJOR, V_a (rows of
// max_rank).  factor: that of dropout, or with KMAJOR scale_a.  A workgroup owns 16 MT tokens and, of the different adapters among
// them, every gridDim.z-th; its wavefronts and the splits take 64-element chunks of K round robin (a chunk is one 128-byte line of every
// row), each tile of tokens beginning at another of them: rows lie whole powers of two apart, and tiles in step would ask the same few
// memory channels at a time.  v_mfma_f32_16x16x32_bf16: lane l supplies row (column) l % 16, elements 8 (l / 16) .. + 8; result lane l holds
// column l % 16, rows 4 (l / 16) .. + 4.  Rows of other adapters' tokens are replaced by one of the adapter's own: no line is fetched
// for them.  KMAJOR: the lane loads NT neighbouring columns of eight rows at once and packs them, so instruction t covers the columns
// l % 16 * NT + t.
constexpr int kThinWaves = 8;

struct ThinArgs {
    AdapterPool p;
    const uint16_t* in;
    int64_t ld;
    float* part;             // [splits][b][max_rank]
    DropoutMask drop;
    int tiles;               // workgroups along x beyond those write down one adapter's tokens each (the backward pass)
    GroupArgs group;
};

template <int NT, bool KMAJOR>
__device__ __forceinline__ void load_b(v4u (&out)[NT], const void* b, const uint32_t (&at)[NT], uint32_t k, uint32_t R) {
    if constexpr (!KMAJOR) {
#pragma unroll
        for (int t = 0; t < NT; ++t) out[t] = load_at<v4u>(b, at[t] + 2 * k);
    } else {
        typedef uint32_t row __attribute__((ext_vector_type(NT > 2 ? NT / 2 : 2)));
        std::conditional_t<NT <= 2, uint32_t, row> e[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const uint32_t o = at[0] + 2 * R * (k + u);
            if constexpr (NT == 1) e[u] = load_at<uint16_t>(b, o);
            else e[u] = load_at<std::conditional_t<NT <= 2, uint32_t, row>>(b, o);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            uint32_t w[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if constexpr (NT <= 2) w[u] = e[u];
                else w[u] = e[u][t / 2];
            }
            out[t] = (t & 1) ? v4u{pack_hi(w[0], w[1]), pack_hi(w[2], w[3]), pack_hi(w[4], w[5]), pack_hi(w[6], w[7])}
                             : v4u{pack_lo(w[0], w[1]), pack_lo(w[2], w[3]), pack_lo(w[4], w[5]), pack_lo(w[6], w[7])};
        }
    }
}

// The operands of one chunk.
template <int NT, int MT>
struct Chunk {
    v4u x[MT][2], b[2][NT];
    template <bool KMAJOR>
    __device__ __forceinline__ void load(const uint16_t* const (&ap)[MT], const void* bbase, const uint32_t (&bat)[NT], uint32_t k0,
                                         uint32_t R) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < MT; ++i) x[i][h] = *reinterpret_cast<const v4u*>(ap[i] + k0 + h * 32);
            load_b<NT, KMAJOR>(b[h], bbase, bat, k0 + h * 32, R);
        }
    }
};

template <int NT, int MT, bool KMAJOR, bool DROP>
__global__ void __launch_bounds__(64 * kThinWaves)
thin_kernel(ThinArgs g) {
    constexpr int ROWS = 16 * MT;
    constexpr bool AHEAD = 16 * (MT + NT) + 4 * MT * NT <= 128;      // registers for two chunks
    __shared__ float s_part[kThinWaves][NT][4][64];      // [wavefront][rank tile][register][lane]
    __shared__ int s_id[64];
    const AdapterPool& p = g.p;
    if (KMAJOR && (int)blockIdx.x >= g.tiles) {
        if (blockIdx.y == 0 && blockIdx.z == 0) group_tokens<64 * kThinWaves>(p, g.group, (int)blockIdx.x - g.tiles);
        return;
    }
    const int lane = threadIdx.x & 63, wave = wave_index();
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
    const int chunk0 = split * kThinWaves + wave, step = splits * kThinWaves, whole = (int)(K >> 6);
    const int count = whole > chunk0 ? (whole - chunk0 + step - 1) / step : 0;      // whole chunks of this wavefront
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
        const uint16_t* b = (KMAJOR ? p.V : p.U) + (int64_t)a * K * R;
        uint32_t bat[NT];                                // bytes from there; an adapter has at most 2^30
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (KMAJOR) bat[t] = 2 * (kg * 8 * R + (lr * NT < R ? lr * NT : 0));
            else bat[t] = 2 * ((uint32_t)(t * 16 + lr < rank ? t * 16 + lr : 0) * (uint32_t)K + kg * 8);
        }
        v4f acc[MT][NT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[i][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        const auto multiply = [&](const Chunk<NT, MT>& q, uint32_t k0) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    v4u x = q.x[i][h];
                    if (DROP) x = drop_eight(g.drop, x, token[i], ((k0 + h * 32) >> 3) + kg);
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[i][t] = mfma(x, q.b[h][t], acc[i][t]);
                }
        };
        if (count > 0) {
            int at = (int)(blockIdx.x % (unsigned)count);
            const auto k_of = [&](int i) { return (uint32_t)(chunk0 + i * step) * 64; };
            const auto after = [&](int i) { return i + 1 < count ? i + 1 : 0; };
            Chunk<NT, MT> now, next;
            now.template load<KMAJOR>(ap, b, bat, k_of(at), R);
#pragma unroll 1
            for (int j = 0; j < count; ++j) {
                if (AHEAD && j + 1 < count) next.template load<KMAJOR>(ap, b, bat, k_of(after(at)), R);
                multiply(now, k_of(at));
                at = after(at);
                if (AHEAD) now = next;
                else if (j + 1 < count) now.template load<KMAJOR>(ap, b, bat, k_of(at), R);
            }
        }
        if ((K & 63) && whole % step == chunk0) {        // the last chunk, if K is not a multiple of 64: eights beyond K are zero
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t k = (int64_t)whole * 64 + h * 32;
                const bool ok = k + kg * 8 < K;          // a lane without elements loads the row's first
                v4u y[NT];
                load_b<NT, KMAJOR>(y, b, bat, (uint32_t)(ok ? k : -(int64_t)kg * 8), R);
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (!ok) y[t] = v4u{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    v4u x = *reinterpret_cast<const v4u*>(ap[i] + (ok ? k : -(int64_t)kg * 8));
                    if (DROP) x = drop_eight(g.drop, x, token[i], (uint32_t)(k >> 3) + kg);
                    if (!ok) x = v4u{0, 0, 0, 0};
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[i][t] = mfma(x, y[t], acc[i][t]);
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

// Where the operand of lane (l % 16 = i, l / 16 = g) lies among an instruction's 64 in LDS: turned by g, so that threads that write neighbouring
// eighths of a row, one g after the other, do not meet in a bank.
__device__ __forceinline__ int operand_slot(int i, int g) { return g * 16 + (i ^ (g * 4)); }

// The same sums for many tokens: a wavefront owns 16 tokens and all of the split's K, in steps of 128; the four of a workgroup share the step's
// part of the adapter, which is staged in LDS as the matrix instructions' operands, two steps in turn.  What a wavefront keeps for itself
// is its rows of the next two steps, on their way: 16 registers a step, so several workgroups fit a compute unit.
constexpr int kRowWaves = 4;
constexpr int kRowTile = 16 * kRowWaves;                 // tokens of a workgroup

template <int NT, bool KMAJOR, bool DROP>
__global__ void __launch_bounds__(64 * kRowWaves, 2)
thin_rows_kernel(ThinArgs g) {
    constexpr int THREADS = 64 * kRowWaves, KS = 128;
    constexpr int UNITS = KMAJOR ? 64 * NT : 256 * NT, PER = (UNITS + THREADS - 1) / THREADS;    // of staging, and per thread
    __shared__ v4u s_b[2][KS / 32][NT][64];
    __shared__ int s_id[kRowTile];
    const AdapterPool& p = g.p;
    if (KMAJOR && (int)blockIdx.x >= g.tiles) {
        if (blockIdx.y == 0) group_tokens<THREADS>(p, g.group, (int)blockIdx.x - g.tiles);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
    const int lr = lane & 15, kg = lane >> 4;
    const int R = p.max_rank;
    const int64_t K = KMAJOR ? p.n : p.m;
    const int64_t row0 = (int64_t)blockIdx.x * kRowTile;
    float* part = g.part + (int64_t)blockIdx.y * p.b * R;
    // read once, so that all wavefronts go the same way
    if (wave == 0) s_id[lane] = row0 + lane < p.b ? p.adapter_of[row0 + lane] : -1;
    __syncthreads();
    TileAdapters tile(p, s_id[lane], true);
    for (uint64_t bare = __ballot(row0 + lane < p.b) & ~tile.todo; bare; bare &= bare - 1)      // tokens without an adapter
        for (int c = tid; c < R; c += THREADS) part[(row0 + __builtin_ctzll(bare)) * R + c] = 0.0f;
    // this split's steps, begun at another one by every tile
    const int steps = (int)((K + KS - 1) / KS), per = (steps + (int)gridDim.y - 1) / (int)gridDim.y;
    const int step0 = (int)blockIdx.y * per, count = steps - step0 < per ? steps - step0 : per;      // count > 0
    const int turn = (int)(blockIdx.x % (unsigned)count);
    const auto k_of = [&](int j) { return (uint32_t)(step0 + (j + turn < count ? j + turn : j + turn - count)) * KS; };
    while (tile.todo) {
        uint64_t mine;
        const int a = tile.next(mine);
        const int rank = rank_of(p, a);
        const int r_own = wave * 16 + lr;
        const uint32_t token = (uint32_t)(row0 + ((mine >> r_own) & 1 ? r_own : __builtin_ctzll(mine)));
        const uint16_t* row = g.in + (int64_t)token * g.ld;
        const uint16_t* b = (KMAJOR ? p.V : p.U) + (int64_t)a * K * R;       // of at most 2^30 bytes

        v4u x[2][4], staged[PER][KMAJOR ? 4 : 1];
        const auto load_x = [&](v4u (&q)[4], int j) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                uint32_t k = k_of(j) + h * 32 + kg * 8;
                q[h] = *reinterpret_cast<const v4u*>(row + (k < (uint32_t)K ? k : 0));
            }
        };
        const auto load_staged = [&](int j) {
            const uint32_t k0 = k_of(j);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t u = (tid + i * THREADS) % UNITS;          // threads beyond load what others do
                if (KMAJOR) {                            // eight rows of four columns
                    const uint32_t c = 4 * (u % (4 * NT)), k = k0 + 8 * (u / (4 * NT));
                    uint32_t at = 2 * ((k < (uint32_t)K ? k : 0) * R + (c < (uint32_t)R ? c : 0));
#pragma unroll
                    for (int e = 0; e < 8; ++e, at += 2 * R) {
                        const uint2 w = load_at<uint2>(b, at);
                        staged[i][e >> 1][2 * (e & 1)] = w.x;
                        staged[i][e >> 1][2 * (e & 1) + 1] = w.y;
                    }
                } else {                                 // eight values of a column: 128 bytes of it by eight neighbouring threads
                    const uint32_t c = (u >> 3) % (16 * NT), k = k0 + 8 * ((u & 7) + 8 * (u / (128 * NT)));
                    staged[i][0] = load_at<v4u>(b, 2 * ((c < (uint32_t)rank ? c : 0) * (uint32_t)K + (k < (uint32_t)K ? k : 0)));
                }
            }
        };
        const auto write_staged = [&](int j) {
            const uint32_t k0 = k_of(j);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t u = tid + i * THREADS;
                if (KMAJOR) {
                    const uint32_t c = 4 * (u % (4 * NT)), k8 = u / (4 * NT);
                    const bool ok = k0 + 8 * k8 < (uint32_t)K;
                    if (UNITS % THREADS == 0 || u < UNITS) {
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const int d = v >> 1;
                            v4u y;
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                y[e] = (v & 1) ? pack_hi(staged[i][e][d], staged[i][e][2 + d]) : pack_lo(staged[i][e][d], staged[i][e][2 + d]);
                            s_b[j & 1][k8 >> 2][c >> 4][operand_slot((c & 15) + v, k8 & 3)] = ok ? y : v4u{0, 0, 0, 0};
                        }
                    }
                } else {
                    const uint32_t c = (u >> 3) % (16 * NT), k8 = (u & 7) + 8 * (u / (128 * NT));
                    s_b[j & 1][k8 >> 2][c >> 4][operand_slot(c & 15, k8 & 3)] = k0 + 8 * k8 < (uint32_t)K ? staged[i][0] : v4u{0, 0, 0, 0};
                }
            }
        };
        v4f acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        const auto multiply = [&](v4u (&x)[4], int j) {
            const uint32_t k0 = k_of(j);
            if (k0 + KS > (uint32_t)K) {
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    if (k0 + h * 32 + kg * 8 >= (uint32_t)K) x[h] = v4u{0, 0, 0, 0};
            }
            v4u q[2][NT];                                // one instruction's operands while the other's are multiplied
            const int slot = operand_slot(lr, kg);
#pragma unroll
            for (int t = 0; t < NT; ++t) q[0][t] = s_b[j & 1][0][t][slot];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                if (h < 3) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) q[(h + 1) & 1][t] = s_b[j & 1][h + 1][t][slot];
                }
                in_order();
                if (DROP) x[h] = drop_eight(g.drop, x[h], token, ((k0 + h * 32) >> 3) + kg);
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = mfma(x[h], q[h & 1][t], acc[t]);
                in_order();
            }
        };
        // Step j: the adapter's part, on its way since the step before, goes to LDS, that of the next step is asked for, and the rows of the
        // step after the next as soon as this one's registers are free.  (Not copied from one to the other: a copy waits for the load.)
        const auto step = [&](v4u (&x)[4], int j) {
            write_staged(j);
            __syncthreads();
            load_staged(j + 1 < count ? j + 1 : j);
            multiply(x, j);
            load_x(x, j + 2 < count ? j + 2 : j);
        };
        __syncthreads();                                 // the adapter before may still be read
        load_staged(0);                                  // first: it is waited for first
        in_order();
        load_x(x[0], 0);
        load_x(x[1], count > 1 ? 1 : 0);
#pragma unroll 1
        for (int j = 0; j < count; j += 2) {
            step(x[0], j);
            if (j + 1 < count) step(x[1], j + 1);
        }
        const float factor = KMAJOR ? scale_of(p, a) : DROP ? g.drop.factor : 1.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][e] = t * 16 + lr < rank ? acc[t][e] * factor : 0.0f;
        in_order();                                      // what is loaded for it is waited for here, not again at each of the stores
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = wave * 16 + 4 * kg + e, c = t * 16 + lr;
                if (((mine >> r) & 1) && c < R) part[(row0 + r) * R + c] = acc[t][e];
            }
    }
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

// The pieces of eight neighbouring values times scale.
__device__ __forceinline__ void split_eight(const v4f& lo, const v4f& hi, float scale, v4u (&q)[3]) {
    uint32_t piece[3][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) split3((e < 4 ? lo[e & 3] : hi[e & 3]) * scale, piece[0][e], piece[1][e], piece[2][e]);
#pragma unroll
    for (int k = 0; k < 3; ++k)
        q[k] = v4u{pack_hi(piece[k][0], piece[k][1]), pack_hi(piece[k][2], piece[k][3]), pack_hi(piece[k][4], piece[k][5]),
                   pack_hi(piece[k][6], piece[k][7])};
}

// ------------------------------------------------------------------------------------------------ pieces of T and S for the gradients
// What grad_kernel multiplies with: for every 32 places of the order, rank tile of 16 and piece the second operand of one matrix
// instruction as the lanes hold it (lane l: column l % 16, places 8 (l / 16) .. + 8), 16 bytes a lane; 0 where a place has no token.  Split here
// once, and not by each of the column tiles that read it.
struct PieceArgs {
    int64_t b, groups;       // groups: of 32 places
    int R, tiles;            // tiles: ceil(R / 16)
    const int* order;
    const float* thin[2];    // T, and the parts of S; null: not wanted
    int splits[2];
    v4u* out[2];             // [places / 32][tiles][3][64]
};

__device__ __forceinline__ void write_pieces(const PieceArgs& g, int64_t group) {
    if (group >= g.groups) return;
    const int lane = threadIdx.x & 63, wave = wave_index(), waves = blockDim.x >> 6;
    const int* order = g.order + group * 32 + 8 * (lane >> 4);
    int token[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) token[u] = order[u];
    for (int i = wave; i < 2 * g.tiles; i += waves) {
        const int job = i >= g.tiles ? 1 : 0, t = i - job * g.tiles, c = t * 16 + (lane & 15);
        if (!g.thin[job]) continue;
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            x[u] = 0.0f;
            if ((uint64_t)(int64_t)token[u] < (uint64_t)g.b && c < g.R) {
                const float* q = g.thin[job] + (int64_t)token[u] * g.R + c;
                for (int s = 0; s < g.splits[job]; ++s) x[u] += q[s * g.b * g.R];
            }
        }
        uint32_t piece[3][8];
#pragma unroll
        for (int u = 0; u < 8; ++u) split3(x[u], piece[0][u], piece[1][u], piece[2][u]);
        v4u* o = g.out[job] + ((group * g.tiles + t) * 3) * 64 + lane;
#pragma unroll
        for (int k = 0; k < 3; ++k)
            o[k * 64] = v4u{pack_hi(piece[k][0], piece[k][1]), pack_hi(piece[k][2], piece[k][3]), pack_hi(piece[k][4], piece[k][5]),
                            pack_hi(piece[k][6], piece[k][7])};
    }
}

__global__ void __launch_bounds__(256)
pieces_kernel(PieceArgs g) { write_pieces(g, blockIdx.x); }

// ------------------------------------------------------------------------------------------------ Y and E_X
// out[t, f] = base[t, f] + sum over c of thin[t, c] * B_a[f, c]; B_a = scale_a V_a (c contiguous) or, with BWD, U_a^T with the mask of dropout
// on the sum.  A workgroup owns 16 MT tokens, the columns of its matrix instructions, whose thin values it keeps in LDS as the operands'
// lanes hold them, split in pieces.  Its wavefronts go over blocks of features, the rows: 64 with 16-byte loads of V, or 64 columns of U,
// loaded four neighbouring columns of eight rank rows at a time and packed, so that instruction v covers the columns 4 i + v.  Either way a
// lane ends up with runs of eight neighbouring features of one token: 16-byte loads of base and stores.  The next block's adapter values and
// base are on their way while one is worked on.
// RC: rank chunks of 32.  RC == 0 (rank up to 16): the halves of the instruction's 32 products hold the pieces (high, middle) and (low,
// nothing), two instructions instead of three.
constexpr int kWideWaves = 4;

struct WideArgs {
    AdapterPool p;
    const float* part;       // [splits][b][max_rank]
    int splits;
    float* thin;             // the sum of the parts is written here (not if null)
    const void* base;
    int64_t ld_base;
    void* out;
    int64_t ld_out;
    DropoutMask drop;
    uint8_t* kept;           // [b][m / 8]: the mask's bits, for the gradients of the same call; null: not wanted
    int tiles;               // workgroups along x beyond those write 32 places' pieces each (the backward pass)
    PieceArgs pieces;
};

// The mask of dropout on eight neighbouring elements of row t; returns its bits.
__device__ __forceinline__ uint32_t drop_run(const DropoutMask& d, int64_t t, int64_t f, float (&y)[8]) {
    const uint32_t kept = kept_eight(d, (uint32_t)t, (uint32_t)(f >> 3));
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (kept >> e) & 1 ? y[e] * d.factor : 0.0f;
    return kept;
}

// Two values rounded to bf16, side by side.
__device__ __forceinline__ uint32_t round_two(float x, float y) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    typedef float v2f __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{x, y}, v2bf));
}

// Eight neighbouring elements of base or result, as they are in memory.
template <bool F32>
struct BaseEight {
    v4u q[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void* base, int64_t at) {
        const v4u* s = reinterpret_cast<const v4u*>(reinterpret_cast<const char*>(base) + at * (F32 ? 4 : 2));
        q[0] = s[0];
        if constexpr (F32) q[1] = s[1];
    }
    __device__ __forceinline__ void store(void* out, int64_t at) const {
        v4u* o = reinterpret_cast<v4u*>(reinterpret_cast<char*>(out) + at * (F32 ? 4 : 2));
        o[0] = q[0];
        if constexpr (F32) o[1] = q[1];
    }
    // keep: all ones, or 0 for nothing
    __device__ __forceinline__ void add(float (&y)[8], uint32_t keep = ~0u) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (F32) {
                y[j] += __uint_as_float(q[0][j] & keep);
                y[4 + j] += __uint_as_float(q[1][j] & keep);
            } else {
                y[2 * j] += __uint_as_float((q[0][j] & keep) << 16);
                y[2 * j + 1] += __uint_as_float(q[0][j] & keep & 0xFFFF0000u);
            }
        }
    }
    __device__ __forceinline__ void set(const float (&y)[8]) {
        if constexpr (F32) {
            q[0] = __builtin_bit_cast(v4u, v4f{y[0], y[1], y[2], y[3]});
            q[1] = __builtin_bit_cast(v4u, v4f{y[4], y[5], y[6], y[7]});
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) q[0][j] = round_two(y[2 * j], y[2 * j + 1]);
        }
    }
    // Of (this, other): even lanes keep this one and odd lanes the other; what they do not keep changes place with the neighbour's.
    __device__ __forceinline__ void exchange(BaseEight& other, bool odd) {
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t give = odd ? q[i][j] : other.q[i][j];
                const uint32_t got = (uint32_t)__builtin_amdgcn_mov_dpp((int)give, 0xB1, 0xF, 0xF, true);   // quad_perm [1,0,3,2]
                q[i][j] = odd ? got : q[i][j];
                other.q[i][j] = odd ? other.q[i][j] : got;
            }
    }
};
template <bool F32>
__device__ __forceinline__ void store_eight(void* out, int64_t at, const float (&y)[8]) {
    BaseEight<F32> x;
    x.set(y);
    x.store(out, at);
}

// A block of 64 features of an adapter, the first operand of the matrix instructions: 16-byte loads of V, or four neighbouring columns of eight
// rank rows of U, packed.  Every lane loads, from a place that exists; what is not the adapter's is cleared in finish().
template <int RC_, bool BWD>
struct AdapterBlock {
    static constexpr bool STACK = RC_ == 0;
    static constexpr int RC = STACK ? 1 : RC_;
    // Features (from the block's first) of a result lane's run q of eight, q = 0, 1, and the e-th of them in the instructions' results.
    __device__ __forceinline__ static int run(int kg, int q) { return BWD ? 16 * kg + 8 * q : 32 * q + 8 * kg; }
    __device__ __forceinline__ static float result(const v4f (&acc)[4], int q, int e) {
        return BWD ? acc[e & 3][2 * q + (e >> 2)] : acc[2 * q + (e >> 2)][e & 3];
    }
    v4u w[RC][4];                                    // as loaded; after finish(): operand q of rank chunk c
    __device__ __forceinline__ void load(const AdapterPool& p, int a, int64_t wide, int64_t f0, int lr, int r_lane) {
        const int R = p.max_rank;
        const uint16_t* b = (BWD ? p.U : p.V) + (int64_t)a * wide * R;   // of at most 2^30 bytes
        if constexpr (!BWD) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t f = (uint32_t)f0 + 32 * (q >> 1) + 8 * (lr >> 2) + 4 * (q & 1) + (lr & 3);
                if (f >= (uint32_t)wide) f = (uint32_t)wide - 1;         // its results are not stored
#pragma unroll
                for (int c = 0; c < RC; ++c) {
                    const int r = 32 * c + r_lane;
                    w[c][q] = load_at<v4u>(b, 2 * (f * R + (r < R ? r : 0)));
                }
            }
        } else {
            uint32_t col = (uint32_t)f0 + 4 * lr;
            if (col >= (uint32_t)wide) col = 0;                          // its results are not stored
#pragma unroll
            for (int c = 0; c < RC; ++c) {
                const int r = 32 * c + r_lane;                           // R is a multiple of eight
                uint32_t at = 2 * ((r < R ? r : 0) * (uint32_t)wide + col);
#pragma unroll
                for (int u = 0; u < 8; ++u, at += 2 * (uint32_t)wide) {
                    const uint2 x = load_at<uint2>(b, at);
                    w[c][u >> 1][2 * (u & 1)] = x.x;
                    w[c][u >> 1][2 * (u & 1) + 1] = x.y;
                }
            }
        }
    }
    __device__ __forceinline__ void finish(int rank, int r_lane) {
        if (rank < (STACK ? 16 : 32 * RC)) {
#pragma unroll
            for (int c = 0; c < RC; ++c) {
                const int r = 32 * c + r_lane;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (!BWD) {            // dword j of every operand: the ranks r + 2 j, r + 2 j + 1
                        const uint32_t keep = (r + 2 * j < rank ? 0xFFFFu : 0u) | (r + 2 * j + 1 < rank ? 0xFFFF0000u : 0u);
#pragma unroll
                        for (int q = 0; q < 4; ++q) w[c][q][j] &= keep;
                    } else {                         // two dwords of the rank row r + 2 j, two of the next
                        const uint32_t even = r + 2 * j < rank ? ~0u : 0u, odd = r + 2 * j + 1 < rank ? ~0u : 0u;
                        w[c][j] &= v4u{even, even, odd, odd};
                    }
                }
            }
        }
        if constexpr (BWD) {                         // eight rows of four columns become four columns
#pragma unroll
            for (int c = 0; c < RC; ++c) {
                v4u y[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int d = v >> 1;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        y[v][j] = (v & 1) ? pack_hi(w[c][j][d], w[c][j][2 + d]) : pack_lo(w[c][j][d], w[c][j][2 + d]);
                }
#pragma unroll
                for (int v = 0; v < 4; ++v) w[c][v] = y[v];
            }
        }
    }
};

template <int RC_, int MT, bool BWD, bool F32>
__global__ void __launch_bounds__(64 * kWideWaves, BWD && RC_ == 4 ? 1 : 2)
wide_kernel(WideArgs g) {
    constexpr bool STACK = RC_ == 0;
    constexpr int RC = STACK ? 1 : RC_, NP = STACK ? 2 : 3, ROWS = 16 * MT;
    constexpr int FB = 64;                               // features per block
    constexpr int NQ = 2;                                // runs of eight features of a lane and token tile
    constexpr bool AHEAD = RC <= 2;                      // registers for two blocks of the adapter
    __shared__ v4u s_thin[MT * RC * NP][64];
    __shared__ int s_id[64];
    if (BWD && (int)blockIdx.x >= g.tiles) {
        if (blockIdx.z == 0) {
            const int64_t group = ((int64_t)blockIdx.x - g.tiles) * gridDim.y + blockIdx.y;
            write_pieces(g.pieces, group);
        }
        return;
    }
    const AdapterPool& p = g.p;
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int lr = lane & 15, kg = lane >> 4;
    const int R = p.max_rank;
    const int64_t wide = BWD ? p.m : p.n;
    const int64_t row0 = (int64_t)blockIdx.x * ROWS;
    if (wave == 0) s_id[lane] = lane < ROWS && row0 + lane < p.b ? p.adapter_of[row0 + lane] : -1;
    __syncthreads();
    TileAdapters tile(p, s_id[lane], lane < ROWS);
    const uint64_t bare = __ballot(lane < ROWS && row0 + lane < p.b) & ~tile.todo;
    // This workgroup's strips of features, one block per wavefront each: a range of them, begun at another one by every tile of tokens.
    const int strips = (int)((wide + FB * kWideWaves - 1) / (FB * kWideWaves)), per = (strips + (int)gridDim.y - 1) / (int)gridDim.y;
    const int strip0 = (int)blockIdx.y * per, count = strips - strip0 < per ? strips - strip0 : per;     // count > 0
    const int turn = (int)(blockIdx.x % (unsigned)count);
    const auto block_at = [&](int j) { return ((int64_t)(strip0 + (j + turn < count ? j + turn : j + turn - count)) * kWideWaves + wave) * FB; };
    const int r_lane = STACK ? 8 * (kg & 1) : 8 * kg;

    // the work of this wavefront: the blocks of features for one adapter after the other
    unsigned seen = 0;
    int a = -1, rank = 0;
    uint64_t mine = 0;
    const auto next_adapter = [&]() {
        a = -1;
        while (tile.todo) {
            uint64_t m;
            const int b = tile.next(m);
            if (seen++ % gridDim.z == blockIdx.z) { a = b; mine = m; rank = rank_of(p, b); return; }
        }
    };
    typedef AdapterBlock<RC_, BWD> Block;
    // feature of run q of the lane in the block at f0
    const auto run_at = [&](int64_t f0, int q) { return f0 + Block::run(kg, q); };
    // a lane whose token has another adapter takes one of this adapter's own
    const auto load_base = [&](BaseEight<F32> (&x)[NQ], int i, int64_t f0) {
        if (!g.base) return;
        const int64_t t = row0 + ((mine >> (i * 16 + lr)) & 1 ? i * 16 + lr : __builtin_ctzll(mine));
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const int64_t f = run_at(f0, q);
            x[q].load(g.base, t * g.ld_base + (f < wide ? f : 0));
        }
    };

    next_adapter();
    Block now;
    if (a >= 0) now.load(p, a, wide, block_at(0), lr, r_lane);

    // the thin values of the tile's tokens, in pieces
    for (int j = wave; j < MT * RC; j += kWideWaves) {
        const int i = j / RC, r = 32 * (j % RC) + r_lane;
        const int64_t t = row0 + i * 16 + lr;
        const int id = s_id[i * 16 + lr];
        const float scale = !BWD && is_adapter(p, id) ? scale_of(p, id) : 1.0f;
        v4f lo = v4f{0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
        if (r < R && t < p.b) {                          // R is a multiple of eight
            sum_parts(g.part, g.splits, p.b * R, t * R + r, lo, hi);
            if (g.thin && blockIdx.y == 0 && blockIdx.z == 0 && !(STACK && kg > 1)) {
                *reinterpret_cast<v4f*>(g.thin + t * R + r) = lo;
                *reinterpret_cast<v4f*>(g.thin + t * R + r + 4) = hi;
            }
        }
        v4u q[3];
        split_eight(lo, hi, scale, q);
        if constexpr (STACK) {
            s_thin[j * NP][lane] = kg < 2 ? q[0] : q[1];
            s_thin[j * NP + 1][lane] = kg < 2 ? q[2] : v4u{0, 0, 0, 0};
        } else {
#pragma unroll
            for (int k = 0; k < NP; ++k) s_thin[j * NP + k][lane] = q[k];
        }
    }
    __syncthreads();

    if (blockIdx.z == 0 && g.base != g.out) {            // tokens without an adapter: the base as it is
        for (uint64_t todo = bare; todo; todo &= todo - 1) {
            const int64_t t = row0 + __builtin_ctzll(todo);
            for (int j = 0; j < count; ++j) {
                const int64_t f = block_at(j) + 8 * lane;
                if (8 * lane >= FB || f >= wide) continue;
                BaseEight<F32> x;
                float y[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                if (g.base) { x.load(g.base, t * g.ld_base + f); x.add(y); }
                store_eight<F32>(g.out, t * g.ld_out + f, y);
            }
        }
    }

    for (; a >= 0; next_adapter()) {
        if (seen > 1 + blockIdx.z) now.load(p, a, wide, block_at(0), lr, r_lane);    // not the first adapter of this wavefront
        BaseEight<F32> base[MT][NQ];
#pragma unroll
        for (int i = 0; i < MT; ++i) load_base(base[i], i, block_at(0));
#pragma unroll 1
        for (int j = 0; j < count; ++j) {
            const int64_t f0 = block_at(j), f1 = block_at(j + 1 < count ? j + 1 : j);
            now.finish(rank, r_lane);
            Block ahead;
            if (AHEAD && j + 1 < count) ahead.load(p, a, wide, f1, lr, r_lane);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if ((mine >> (i * 16)) & 0xFFFF) {
                    v4f acc[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[q] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int c = 0; c < RC; ++c)
#pragma unroll
                        for (int k = 0; k < NP; ++k) {
                            const v4u b = s_thin[(i * RC + c) * NP + k][lane];
#pragma unroll
                            for (int q = 0; q < 4; ++q) acc[q] = mfma(now.w[c][q], b, acc[q]);
                        }
                    if ((mine >> (i * 16 + lr)) & 1) {
                        const int64_t t = row0 + i * 16 + lr;
#pragma unroll
                        for (int q = 0; q < NQ; ++q) {
                            const int64_t f = run_at(f0, q);
                            if (f >= wide) continue;
                            float y[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) y[e] = Block::result(acc, q, e);
                            if (BWD && g.drop.least) {
                                const uint32_t kept = drop_run(g.drop, t, f, y);
                                if (g.kept) g.kept[t * (wide >> 3) + (f >> 3)] = (uint8_t)kept;
                            }
                            if (g.base) base[i][q].add(y);
                            store_eight<F32>(g.out, t * g.ld_out + f, y);
                        }
                    }
                    if (j + 1 < count) load_base(base[i], i, f1);
                }
                __builtin_amdgcn_sched_barrier(0);       // one token tile's values in registers at a time
            }
            if (AHEAD) now = ahead;
            else if (j + 1 < count) now.load(p, a, wide, f1, lr, r_lane);
        }
    }
}

// The same for many tokens: tiles of 16 MT tokens, so that the adapter, which every tile reads once, is little next to base and result.  A step is
// 16 tokens times 64 features; the base of the next steps and the next block of features are on their way meanwhile.  Nothing is exchanged
// once the pieces are in LDS.
constexpr int kTallWaves = 8;

template <int RC_, int MT, bool BWD, bool F32>
__global__ void __launch_bounds__(64 * kTallWaves)
wide_tall_kernel(WideArgs g) {
    constexpr bool STACK = RC_ == 0;
    constexpr int RC = STACK ? 1 : RC_, NP = STACK ? 2 : 3, ROWS = 16 * MT, WORDS = ROWS / 64, DEPTH = F32 ? 2 : 4;
    constexpr bool AHEAD = RC <= 2;                      // registers for two blocks of the adapter
    __shared__ v4u s_thin[MT * RC * NP][64];
    __shared__ int s_id[ROWS];
    const AdapterPool& p = g.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
    const int lr = lane & 15, kg = lane >> 4;
    if (BWD && (int)blockIdx.x >= g.tiles) {
        write_pieces(g.pieces, ((int64_t)blockIdx.x - g.tiles) * gridDim.y + blockIdx.y);
        return;
    }
    const int R = p.max_rank;
    const int64_t wide = BWD ? p.m : p.n;
    const int64_t row0 = (int64_t)blockIdx.x * ROWS;
    typedef AdapterBlock<RC_, BWD> Block;
    const bool odd = lr & 1;
    const int pair = lr & 14, run = Block::run(kg, lr & 1);
    for (int r = tid; r < ROWS; r += 64 * kTallWaves) s_id[r] = row0 + r < p.b ? p.adapter_of[row0 + r] : -1;
    __syncthreads();
    const int r_lane = STACK ? 8 * (kg & 1) : 8 * kg;
    for (int j = wave; j < MT * RC; j += kTallWaves) {   // the thin values of the tile's tokens, in pieces
        const int i = j / RC, r = 32 * (j % RC) + r_lane;
        const int64_t t = row0 + i * 16 + lr;
        const int id = s_id[i * 16 + lr];
        const float scale = !BWD && is_adapter(p, id) ? scale_of(p, id) : 1.0f;
        v4f lo = v4f{0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
        if (r < R && t < p.b) {                          // R is a multiple of eight
            sum_parts(g.part, g.splits, p.b * R, t * R + r, lo, hi);
            if (g.thin && blockIdx.y == 0 && !(STACK && kg > 1)) {
                *reinterpret_cast<v4f*>(g.thin + t * R + r) = lo;
                *reinterpret_cast<v4f*>(g.thin + t * R + r + 4) = hi;
            }
        }
        v4u q[3];
        split_eight(lo, hi, scale, q);
        if constexpr (STACK) {
            s_thin[j * NP][lane] = kg < 2 ? q[0] : q[1];
            s_thin[j * NP + 1][lane] = kg < 2 ? q[2] : v4u{0, 0, 0, 0};
        } else {
#pragma unroll
            for (int k = 0; k < NP; ++k) s_thin[j * NP + k][lane] = q[k];
        }
    }
    __syncthreads();

    // this wavefront's blocks of 64 features: every kTallWaves-th of the workgroup's range
    const int blocks = (int)((wide + 63) >> 6), per = (blocks + (int)gridDim.y - 1) / (int)gridDim.y;
    const int block0 = (int)blockIdx.y * per, end = block0 + per < blocks ? block0 + per : blocks;
    const int count = end - block0 > wave ? (end - block0 - wave + kTallWaves - 1) / kTallWaves : 0;
    if (count <= 0) return;
    const int turn = (int)(blockIdx.x % (unsigned)count);
    const auto f_of = [&](int j) { return (int64_t)(block0 + wave + (j + turn < count ? j + turn : j + turn - count) * kTallWaves) * 64; };

    // without a base: something that is there to be loaded, and nothing of it kept.  (A load that may not happen would have the compiler wait
    // for all of those before it.)
    const void* base_at = g.base ? g.base : g.out;
    const int64_t base_ld = g.base ? g.ld_base : g.ld_out;
    const uint32_t base_keep = g.base ? ~0u : 0u;
    uint64_t todo[WORDS], bare[WORDS];                   // tokens with an adapter that are not done, and tokens without one
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        todo[w] = __ballot(is_adapter(p, s_id[w * 64 + lane]));
        bare[w] = __ballot(row0 + w * 64 + lane < p.b) & ~todo[w];
    }
    if (g.base != g.out) {                               // tokens without an adapter: the base as it is
#pragma unroll
        for (int w = 0; w < WORDS; ++w)
            for (uint64_t left = bare[w]; left; left &= left - 1) {
                const int64_t t = row0 + w * 64 + __builtin_ctzll(left);
                for (int j = 0; j < count; ++j) {
                    const int64_t f = f_of(j) + 8 * lane;
                    if (lane >= 8 || f >= wide) continue;
                    BaseEight<F32> x;
                    float y[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                    if (g.base) { x.load(g.base, t * g.ld_base + f); x.add(y); }
                    store_eight<F32>(g.out, t * g.ld_out + f, y);
                }
            }
    }
#pragma unroll 1
    while (true) {
        int first = -1;                                  // the next adapter's first token
#pragma unroll
        for (int w = WORDS - 1; w >= 0; --w)
            if (todo[w]) first = w * 64 + __builtin_ctzll(todo[w]);
        if (first < 0) break;
        const int a = __builtin_amdgcn_readfirstlane(s_id[first]), rank = rank_of(p, a);
        uint32_t own[2] = {0, 0}, steps = 0;             // bit i: the even (odd) token of the lane's pair in step i is a's; any of the step is
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            const uint64_t mine = __ballot(s_id[w * 64 + lane] == a) & todo[w];
            todo[w] &= ~mine;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t sixteen = (uint32_t)(mine >> (16 * i)) & 0xFFFFu;
                own[0] |= ((sixteen >> pair) & 1u) << (4 * w + i);
                own[1] |= ((sixteen >> (pair + 1)) & 1u) << (4 * w + i);
                steps |= (sixteen ? 1u : 0u) << (4 * w + i);
            }
        }
        struct Place { int j; uint32_t left; };          // block of features, and the steps left in it, this one the lowest
        const auto after = [&](Place q) {
            q.left &= q.left - 1;
            if (!q.left) { ++q.j; q.left = steps; }
            return q;
        };
        // Base and result go a pair of tokens at a time: lane (i, g) has run i % 2 of the even token, then of the odd one, so that eight lanes
        // take 128 bytes of a row at once.  (Token by token, each half of a line was a request of its own.)
        BaseEight<F32> base[DEPTH][2];
        const auto load_base = [&](BaseEight<F32> (&x)[2], const Place& q) {
            const int i = __builtin_ctz(q.left);
            const int64_t f = f_of(q.j < count ? q.j : 0) + run;
#pragma unroll
            for (int k = 0; k < 2; ++k) {                // other adapters' tokens, features beyond: the first of this one's
                const bool ok = (own[k] >> i) & 1 && f < wide;
                x[k].load(base_at, (row0 + (ok ? i * 16 + pair + k : first)) * base_ld + (ok ? f : 0));
            }
        };
        Block now, ahead;
        const auto work = [&](BaseEight<F32> (&x)[2], const Place& q) {
            const int i = __builtin_ctz(q.left);
            v4f acc[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            v4u b[2][NP];                                // one rank chunk's operands while the other's are multiplied
#pragma unroll
            for (int k = 0; k < NP; ++k) b[0][k] = s_thin[i * RC * NP + k][lane];
#pragma unroll
            for (int c = 0; c < RC; ++c) {
                if (c + 1 < RC) {
#pragma unroll
                    for (int k = 0; k < NP; ++k) b[(c + 1) & 1][k] = s_thin[(i * RC + c + 1) * NP + k][lane];
                }
                in_order();
#pragma unroll
                for (int k = 0; k < NP; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[e] = mfma(now.w[c][e], b[c & 1][k], acc[e]);
            }
            x[0].exchange(x[1], odd);
            BaseEight<F32> y[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = Block::result(acc, k, e);
                if (BWD && g.drop.least) {
                    const int64_t f = f_of(q.j) + Block::run(kg, k);
                    const uint32_t kept = drop_run(g.drop, row0 + i * 16 + lr, f, v);
                    if (g.kept && (own[lr & 1] >> i) & 1 && f < wide) g.kept[(row0 + i * 16 + lr) * (wide >> 3) + (f >> 3)] = (uint8_t)kept;
                }
                x[k].add(v, base_keep);
                y[k].set(v);
            }
            y[0].exchange(y[1], odd);
            const int64_t f = f_of(q.j) + run;
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if ((own[k] >> i) & 1 && f < wide) y[k].store(g.out, (row0 + i * 16 + pair + k) * g.ld_out + f);
        };
        Place at{0, steps}, next = at;
        now.load(p, a, wide, f_of(0), lr, r_lane);
#pragma unroll
        for (int k = 0; k < DEPTH; ++k, next = after(next)) load_base(base[k], next);
        if (AHEAD) ahead.load(p, a, wide, f_of(count > 1 ? 1 : 0), lr, r_lane);
        now.finish(rank, r_lane);
#pragma unroll 1
        while (at.j < count) {
#pragma unroll
            for (int k = 0; k < DEPTH; ++k) {
                if (at.j >= count) break;
                work(base[k], at);
                load_base(base[k], next);
                next = after(next);
                const int j = at.j;
                at = after(at);
                if (at.j != j && at.j < count) {
                    if (AHEAD) now = ahead;
                    else now.load(p, a, wide, f_of(at.j), lr, r_lane);
                    now.finish(rank, r_lane);
                    if (AHEAD) ahead.load(p, a, wide, f_of(at.j + 1 < count ? at.j + 1 : at.j), lr, r_lane);
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ adapter gradients
// The sum over a segment's tokens of big[t, col] * small[t, c]: big bf16 (E for G_V, drop(X) for G_U), small fp32 (T, S), given in pieces.  A
// workgroup owns 256 columns of `big`, a wavefront 64, and goes over the places 32 at a time; the step's pieces are staged in LDS for the
// four, two steps in turn.  v_mfma_f32_16x16x32_bf16 with k = place: lane l supplies, for row (A) / column (B) l % 16, the eight places
// 8 (l / 16) .. + 8 of the step.  `big` is read four neighbouring columns of a token at a time; the v-th of them, packed over the eight
// tokens, is the A operand of the v-th instruction, which covers the columns 4 i + v.  NT: rank tiles of 16, from tile blockIdx.z * NT on.
constexpr int kGradWaves = 4;
constexpr int kGradCols = 64 * kGradWaves;

struct GradJob {
    const uint16_t* big;
    int64_t ld;
    const v4u* small;        // PieceArgs::out
    float* out;              // [slots][wide x R], or [slots][R x wide] with rank_major
    float* part;             // [parts] of the same
    int64_t wide;
    int tiles;               // of kGradCols columns; 0: no such job
    int rank_major;          // G_U
};
struct GradArgs {
    AdapterPool p;
    GradJob job[2];          // G_V, G_U
    const int* order;
    const Segment* segments;
    int rank_tiles;
    DropoutMask drop;
    const uint8_t* kept;     // WideArgs::kept
};

// MASK of dropout on X: none, the bits that the E_X kernel left, or drawn here (if E_X is not wanted).
enum GradMask { NO_MASK, KEPT_BITS, DRAWN_MASK };

template <int NT, GradMask MASK>
__global__ void __launch_bounds__(64 * kGradWaves, 2)
grad_kernel(GradArgs g) {
    constexpr int THREADS = 64 * kGradWaves, UNITS = NT * 3 * 64, PER = (UNITS + THREADS - 1) / THREADS;
    __shared__ v4u s_small[2][UNITS];
    const Segment seg = g.segments[blockIdx.y];
    if (seg.adapter < 0) return;
    const bool second = (int)blockIdx.x >= g.job[0].tiles;
    const GradJob& job = g.job[second ? 1 : 0];
    const AdapterPool& p = g.p;
    const int R = p.max_rank, tile0 = blockIdx.z * NT;
    const int64_t wide = job.wide;
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
    const int i16 = lane & 15, kq = lane >> 4;
    const int64_t c0 = (int64_t)((int)blockIdx.x - (second ? g.job[0].tiles : 0)) * kGradCols + wave * 64;
    const int64_t col = c0 + 4 * i16, colc = col < wide ? col : 0;       // columns beyond the matrix are not stored
    const bool masked = MASK != NO_MASK && second;
    const uint16_t* big = job.big + colc;
    // (without a mask the bits of the first place are loaded and not looked at)
    const uint8_t* kept_at = MASK == KEPT_BITS ? g.kept + (masked ? colc >> 3 : 0) : nullptr;
    const int64_t kept_pitch = masked ? wide >> 3 : 0;

    struct Step {
        int token[8];
        uint2 raw[8];
        uint32_t kept[8];
    };
    const int steps = (seg.end - seg.begin + 31) >> 5;
    const auto load_order = [&](int (&token)[8], int j) {
        const int4* o = reinterpret_cast<const int4*>(g.order + seg.begin + 32 * (j < steps ? j : 0) + 8 * kq);
        const int4 lo = o[0], hi = o[1];
        token[0] = lo.x; token[1] = lo.y; token[2] = lo.z; token[3] = lo.w;
        token[4] = hi.x; token[5] = hi.y; token[6] = hi.z; token[7] = hi.w;
    };
    const auto load_rows = [&](Step& q, const int (&token)[8]) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {                    // a place without a token loads the first one, which counts as zero
            const int64_t t = (uint64_t)(int64_t)token[u] < (uint64_t)p.b ? token[u] : 0;
            q.token[u] = token[u];
            q.raw[u] = *reinterpret_cast<const uint2*>(big + t * job.ld);
            if (MASK == KEPT_BITS) q.kept[u] = kept_at[t * kept_pitch];
        }
    };
    v4u staged[PER];
    const auto load_staged = [&](int j) {
        const v4u* small = job.small + ((int64_t)((seg.begin >> 5) + (j < steps ? j : 0)) * g.rank_tiles + tile0) * 3 * 64;
        const int most = (g.rank_tiles - tile0 < NT ? g.rank_tiles - tile0 : NT) * 3 * 64;       // rank tiles that there are
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int u = (tid + i * THREADS) % UNITS;
            staged[i] = small[u < most ? u : 0];
        }
    };
    v4f acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[t][v] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const auto multiply = [&](const Step& q, int j) {
        uint2 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            x[u] = q.raw[u];
            if (masked) {
                const uint32_t kept = MASK == KEPT_BITS ? q.kept[u] >> (colc & 4)
                                                        : kept_eight(g.drop, (uint32_t)q.token[u], (uint32_t)(colc >> 3)) >> (colc & 4);
                x[u] = keep_four(x[u], kept);
            }
            if ((uint64_t)(int64_t)q.token[u] >= (uint64_t)p.b) x[u] = make_uint2(0, 0);
        }
        v4u a[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[0][e] = pack_lo(x[2 * e].x, x[2 * e + 1].x);
            a[1][e] = pack_hi(x[2 * e].x, x[2 * e + 1].x);
            a[2][e] = pack_lo(x[2 * e].y, x[2 * e + 1].y);
            a[3][e] = pack_hi(x[2 * e].y, x[2 * e + 1].y);
        }
        v4u b[2][3];                                     // one rank tile's operands while the other's are multiplied
#pragma unroll
        for (int k = 0; k < 3; ++k) b[0][k] = s_small[j & 1][k * 64 + lane];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (t + 1 < NT) {
#pragma unroll
                for (int k = 0; k < 3; ++k) b[(t + 1) & 1][k] = s_small[j & 1][((t + 1) * 3 + k) * 64 + lane];
            }
            in_order();
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[t][v] = mfma(a[v], b[t & 1][k], acc[t][v]);
            in_order();
        }
    };
    int token[8];                                        // of the step whose rows are asked for next
    Step even, odd;
    // Step j: its pieces, on their way since the step before, go to LDS, those of the next are asked for, and the rows of the step after the
    // next as soon as this one's are used, by places that were asked for a step ago.
    const auto step = [&](Step& q, int j) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (UNITS % THREADS == 0 || tid + i * THREADS < UNITS) s_small[j & 1][tid + i * THREADS] = staged[i];
        __syncthreads();
        load_staged(j + 1);
        multiply(q, j);
        load_rows(q, token);
        load_order(token, j + 3);
        in_order();
    };
    if (steps > 0) {                                     // the same for the workgroup
        load_order(token, 0);
        load_staged(0);
        in_order();
        load_rows(even, token);
        load_order(token, 1);
        in_order();
        load_rows(odd, token);
        load_order(token, 2);
        in_order();
#pragma unroll 1
        for (int j = 0; j < steps; j += 2) {
            step(even, j);
            if (j + 1 < steps) step(odd, j + 1);
        }
    }
    const int rank = rank_of(p, seg.adapter);
    const float factor = second ? (masked ? g.drop.factor : 1.0f) : scale_of(p, seg.adapter);
    float* dst = seg.part < 0 ? job.out + (int64_t)seg.adapter * wide * R : job.part + (int64_t)seg.part * wide * R;
    const bool rank_major = job.rank_major != 0;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][v][e] = (tile0 + t) * 16 + i16 < rank ? acc[t][v][e] * factor : 0.0f;
    in_order();                                          // what is loaded for it is waited for here, not again at each of the stores
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int c = (tile0 + t) * 16 + i16;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t oc = c0 + 4 * (4 * kq + e);
            if (oc >= wide || c >= R) continue;
            if (rank_major) {
                *reinterpret_cast<v4f*>(dst + (int64_t)c * wide + oc) = v4f{acc[t][0][e], acc[t][1][e], acc[t][2][e], acc[t][3][e]};
            } else {
#pragma unroll
                for (int v = 0; v < 4; ++v) dst[(oc + v) * R + c] = acc[t][v][e];
            }
        }
    }
}

// Adds up the segments of every adapter that has several, in order; four neighbouring elements per thread.
__global__ void __launch_bounds__(256)
grad_join_kernel(AdapterPool p, GroupArgs group, GradJob v, GradJob u) {
    const int a = blockIdx.y;
    const int2 range = group.range[a];
    const int first = range.x / group.chunk, count = range.y > range.x ? (range.y + group.chunk - 1) / group.chunk - first : 1;
    if (count == 1) return;
    const int64_t size_v = v.tiles ? v.wide * p.max_rank : 0, size_u = u.tiles ? u.wide * p.max_rank : 0;
    int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= size_v + size_u) return;
    const bool second = i >= size_v;
    if (second) i -= size_v;
    const GradJob& job = second ? u : v;
    const int64_t size = second ? size_u : size_v;
    float4 sum = *reinterpret_cast<const float4*>(job.part + (int64_t)(group.cuts + first + 1) * size + i);
    for (int k = 1; k < count; ++k) {
        const float4 q = *reinterpret_cast<const float4*>(job.part + (int64_t)(first + k) * size + i);
        sum.x += q.x; sum.y += q.y; sum.z += q.z; sum.w += q.w;
    }
    *reinterpret_cast<float4*>(job.out + (int64_t)a * size + i) = sum;
}

// ------------------------------------------------------------------------------------------------ launches
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round256(size_t v) { return (v + 255) & ~size_t(255); }

constexpr int64_t kWideFill = 1024;                   // workgroups of the wide kernels
constexpr int64_t kManyTokens = 1024;                 // from here on thin_rows_kernel
constexpr int64_t kThinFill = 512;                    // its workgroups
constexpr int64_t kManySteps = 8192;                  // from here on wide_tall_kernel
constexpr int64_t kTallFill = 256;                    // its workgroups
constexpr int64_t kGradFill = 768;                    // of grad_kernel

// How the kernels of T and S are laid over b tokens, a reduction of K and the adapters.
struct ThinPlan {
    bool rows;               // thin_rows_kernel
    int lanes;               // workgroups that share a tile's different adapters
    int splits;              // of K
};

ThinPlan thin_plan(int64_t b, int64_t K, int slots) {
    ThinPlan q;
    q.rows = b >= kManyTokens;
    const int64_t tiles = ceil_div(b, q.rows ? kRowTile : 16);
    int64_t most = 16;                                   // different adapters in a tile of 16
    if (b < most) most = b;
    if (slots < most) most = slots;
    q.lanes = b <= 256 ? (int)most : 1;
    const int64_t chunks = ceil_div(K, q.rows ? 128 : 64 * kThinWaves);
    int64_t splits = (q.rows ? kThinFill : 512) / (tiles * q.lanes > 0 ? tiles * q.lanes : 1);
    if (splits > 8) splits = 8;
    if (splits > chunks) splits = chunks;
    if (splits < 1) splits = 1;
    q.splits = (int)ceil_div(chunks, ceil_div(chunks, splits));      // none without a chunk
    return q;
}

template <int NT, bool KMAJOR>
void launch_thin_as(ThinArgs g, int extra, const ThinPlan& q, hipStream_t s) {
    const bool drop = !KMAJOR && g.drop.least;
    g.tiles = (int)ceil_div(g.p.b, q.rows ? kRowTile : 16);
    const dim3 grid((unsigned)(g.tiles + extra), q.splits, q.rows ? 1 : q.lanes), block(64 * (q.rows ? kRowWaves : kThinWaves));
    if (q.rows && drop) hipLaunchKernelGGL((thin_rows_kernel<NT, KMAJOR, !KMAJOR>), grid, block, 0, s, g);
    else if (q.rows) hipLaunchKernelGGL((thin_rows_kernel<NT, KMAJOR, false>), grid, block, 0, s, g);
    else if (drop) hipLaunchKernelGGL((thin_kernel<NT, 1, KMAJOR, !KMAJOR>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((thin_kernel<NT, 1, KMAJOR, false>), grid, block, 0, s, g);
}

// extra: workgroups that write down the tokens by adapter.
template <bool KMAJOR>
hipError_t launch_thin(const ThinArgs& g, int extra, const ThinPlan& q, hipStream_t s) {
    const int R = g.p.max_rank;
    if (R <= 16) launch_thin_as<1, KMAJOR>(g, extra, q, s);
    else if (R <= 32) launch_thin_as<2, KMAJOR>(g, extra, q, s);
    else if (R <= 64) launch_thin_as<4, KMAJOR>(g, extra, q, s);
    else launch_thin_as<8, KMAJOR>(g, extra, q, s);
    return hipGetLastError();
}

// Whether Y (E_X) is made by wide_tall_kernel: enough steps of 16 tokens and 64 features to fill the chip with tall tiles.
bool tall(int64_t b, int64_t wide) { return ceil_div(b, 16) * ceil_div(wide, 64) >= kManySteps; }
int rank_chunks(int R) { return R <= 16 ? 0 : R <= 32 ? 1 : R <= 64 ? 2 : 4; }

// groups: of 32 places, whose pieces are written in the same launch.
template <int RC, bool BWD>
hipError_t launch_wide_as(WideArgs g, int f32, const ThinPlan& q, int64_t groups, hipStream_t s) {
    const int64_t wide = BWD ? g.p.m : g.p.n, blocks = ceil_div(wide, 64 * kWideWaves);
    const dim3 block(64 * kWideWaves);
    if (tall(g.p.b, wide)) {
        constexpr int MT = RC == 4 ? 8 : 16;
        const int64_t tall_tiles = ceil_div(g.p.b, 16 * MT), strips = ceil_div(wide, 64 * kTallWaves);
        int64_t y = ceil_div(kTallFill, tall_tiles);
        if (y > strips) y = strips;
        g.tiles = (int)tall_tiles;
        const dim3 grid((unsigned)(tall_tiles + ceil_div(groups, y)), (unsigned)y);
        if (f32) hipLaunchKernelGGL((wide_tall_kernel<RC, MT, BWD, true>), grid, dim3(64 * kTallWaves), 0, s, g);
        else hipLaunchKernelGGL((wide_tall_kernel<RC, MT, BWD, false>), grid, dim3(64 * kTallWaves), 0, s, g);
        return hipGetLastError();
    }
    const int64_t tiles = ceil_div(g.p.b, 16);
    // as many workgroups as fill the chip, each with several blocks of features where there are more
    int64_t y = ceil_div(kWideFill, tiles * q.lanes);
    if (y > blocks) y = blocks;
    y = ceil_div(blocks, ceil_div(blocks, y));
    g.tiles = (int)tiles;
    const dim3 grid((unsigned)(tiles + ceil_div(groups, y)), (unsigned)y, q.lanes);
    if (f32) hipLaunchKernelGGL((wide_kernel<RC, 1, BWD, true>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((wide_kernel<RC, 1, BWD, false>), grid, block, 0, s, g);
    return hipGetLastError();
}

template <bool BWD>
hipError_t launch_wide(const WideArgs& g, int f32, const ThinPlan& q, int64_t groups, hipStream_t s) {
    switch (rank_chunks(g.p.max_rank)) {
        case 0: return launch_wide_as<0, BWD>(g, f32, q, groups, s);
        case 1: return launch_wide_as<1, BWD>(g, f32, q, groups, s);
        case 2: return launch_wide_as<2, BWD>(g, f32, q, groups, s);
        default: return launch_wide_as<4, BWD>(g, f32, q, groups, s);
    }
}

// Places between two cuts of the gradient sums: few enough that the column tiles fill the chip, so many that the partial sums stay small
// next to what is read for them.
int grad_chunk(int64_t places, int64_t m, int64_t n, int max_rank) {
    const int64_t tiles = ceil_div(m, kGradCols) + ceil_div(n, kGradCols);
    int64_t chunk = ceil_div(places * tiles, kGradFill), least = 8 * max_rank < 256 ? 256 : 8 * max_rank;
    if (chunk < least) chunk = least;
    return (int)(ceil_div(chunk, 128) * 128);
}

struct BwdLayout {
    size_t part, order, range, segments, small_v, small_u, kept, part_v, part_u, total;
    int64_t groups;          // of 32 places
    int chunk, cuts, rank_tiles;
    ThinPlan plan;
};

BwdLayout bwd_layout(int64_t b, int64_t m, int64_t n, int slots, int R, bool drop) {
    BwdLayout L;
    const int64_t places = (b + 31) / 32 * 32 + 32 * (int64_t)slots;
    L.groups = places / 32;
    L.plan = thin_plan(b, n, slots);
    L.chunk = grad_chunk(places, m, n, R);
    L.cuts = (int)ceil_div(places, L.chunk);
    L.rank_tiles = (int)ceil_div(R, 16);
    size_t at = 0;
    const auto take = [&at](size_t bytes) { const size_t here = at; at += round256(bytes); return here; };
    L.part = take((size_t)L.plan.splits * b * R * 4);
    L.order = take((size_t)places * 4);
    L.range = take((size_t)slots * sizeof(int2));
    L.segments = take(((size_t)slots + L.cuts) * sizeof(Segment));
    const size_t small = (size_t)L.groups * L.rank_tiles * 3 * 64 * sizeof(v4u);
    L.small_v = take(small);
    L.small_u = take(small);
    L.kept = take(drop ? (size_t)b * (m / 8) : 0);
    const size_t parts = L.cuts > 1 ? 2 * (size_t)L.cuts + 1 : 0;
    L.part_v = take(parts * n * R * 4);
    L.part_u = take(parts * m * R * 4);
    L.total = at;
    return L;
}

template <int NT>
void launch_grad(const GradArgs& g, GradMask mask, const BwdLayout& L, hipStream_t s) {
    const dim3 grid(g.job[0].tiles + g.job[1].tiles, g.p.slots + L.cuts, (unsigned)ceil_div(L.rank_tiles, NT)), block(64 * kGradWaves);
    if (mask == NO_MASK) hipLaunchKernelGGL((grad_kernel<NT, NO_MASK>), grid, block, 0, s, g);
    else if (mask == KEPT_BITS) hipLaunchKernelGGL((grad_kernel<NT, KEPT_BITS>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((grad_kernel<NT, DRAWN_MASK>), grid, block, 0, s, g);
}

}  // namespace

size_t adapters_fwd_workspace(int64_t b, int64_t m, int64_t, int slots, int max_rank) {
    const ThinPlan q = thin_plan(b, m, slots);
    return q.splits > 1 ? round256((size_t)q.splits * b * max_rank * 4) : 0;
}

size_t adapters_bwd_workspace(int64_t b, int64_t m, int64_t n, int slots, int max_rank, bool drop) {
    return bwd_layout(b, m, n, slots, max_rank, drop).total;
}

hipError_t launch_adapters_fwd(const AdaptersFwd& a, hipStream_t s) {
    const AdapterPool& p = a.pool;
    const ThinPlan q = thin_plan(p.b, p.m, p.slots);
    float* part = q.splits > 1 ? reinterpret_cast<float*>(a.workspace) : a.T;
    ThinArgs t{};
    t.p = p; t.in = a.X; t.ld = a.ld_x; t.part = part; t.drop = a.drop;
    const hipError_t e = launch_thin<false>(t, 0, q, s);
    if (e != hipSuccess) return e;
    WideArgs w{};
    w.p = p; w.part = part; w.splits = q.splits; w.thin = q.splits > 1 ? a.T : nullptr;
    w.base = a.base; w.ld_base = a.ld_base; w.out = a.Y; w.ld_out = a.ld_y;
    return launch_wide<false>(w, a.out_f32, q, 0, s);
}

hipError_t launch_adapters_bwd(const AdaptersBwd& a, hipStream_t s) {
    const AdapterPool& p = a.pool;
    const int64_t b = p.b;
    const BwdLayout L = bwd_layout(b, p.m, p.n, p.slots, p.max_rank, a.drop.least != 0);
    unsigned char* ws = reinterpret_cast<unsigned char*>(a.workspace);
    float* part = reinterpret_cast<float*>(ws + L.part);
    const GroupArgs group{L.chunk, L.cuts, reinterpret_cast<int*>(ws + L.order), reinterpret_cast<int2*>(ws + L.range),
                          reinterpret_cast<Segment*>(ws + L.segments)};
    v4u* small[2] = {reinterpret_cast<v4u*>(ws + L.small_v), reinterpret_cast<v4u*>(ws + L.small_u)};
    const bool grads = a.GU || a.GV, thin = b > 0 && (a.EX || a.GU);
    // the mask's bits go from the E_X kernel to the gradients'
    uint8_t* kept = b > 0 && a.EX && a.GU && a.drop.least ? ws + L.kept : nullptr;
    hipError_t e = hipSuccess;
    // S, and the tokens by their adapters
    if (thin) {
        ThinArgs t{};
        t.p = p; t.in = a.E; t.ld = a.ld_e; t.part = part; t.group = group;
        e = launch_thin<true>(t, grads ? p.slots : 0, L.plan, s);
    } else if (grads) {
        hipLaunchKernelGGL(group_kernel, dim3(p.slots), dim3(512), 0, s, p, group);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    // E_X, and the pieces of T and S
    PieceArgs pieces{};
    pieces.b = b; pieces.groups = L.groups; pieces.R = p.max_rank; pieces.tiles = L.rank_tiles; pieces.order = group.order;
    pieces.thin[0] = a.GV ? a.T : nullptr; pieces.splits[0] = 1; pieces.out[0] = small[0];
    pieces.thin[1] = a.GU ? part : nullptr; pieces.splits[1] = L.plan.splits; pieces.out[1] = small[1];
    if (b > 0 && a.EX) {
        WideArgs w{};
        w.p = p; w.part = part; w.splits = L.plan.splits;
        w.base = a.base; w.ld_base = a.ld_base; w.out = a.EX; w.ld_out = a.ld_ex; w.drop = a.drop; w.kept = kept; w.pieces = pieces;
        e = launch_wide<true>(w, a.out_f32, L.plan, grads ? L.groups : 0, s);
    } else if (grads) {
        hipLaunchKernelGGL(pieces_kernel, dim3((unsigned)L.groups), dim3(256), 0, s, pieces);
        e = hipGetLastError();
    }
    if (e != hipSuccess || !grads) return e;
    GradArgs g{};
    g.p = p; g.order = group.order; g.segments = group.segments; g.rank_tiles = L.rank_tiles; g.drop = a.drop;
    if (a.GV) g.job[0] = GradJob{a.E, a.ld_e, small[0], a.GV, reinterpret_cast<float*>(ws + L.part_v), p.n, (int)ceil_div(p.n, kGradCols), 0};
    if (a.GU) g.job[1] = GradJob{a.X, a.ld_x, small[1], a.GU, reinterpret_cast<float*>(ws + L.part_u), p.m, (int)ceil_div(p.m, kGradCols), 1};
    g.kept = kept;
    const GradMask mask = !a.GU || !a.drop.least ? NO_MASK : kept ? KEPT_BITS : DRAWN_MASK;
    if (L.rank_tiles <= 1) launch_grad<1>(g, mask, L, s);
    else if (L.rank_tiles <= 2) launch_grad<2>(g, mask, L, s);
    else launch_grad<4>(g, mask, L, s);
    if (L.cuts > 1) {
        const int64_t size = ((a.GV ? p.n : 0) + (a.GU ? p.m : 0)) * p.max_rank;
        hipLaunchKernelGGL(grad_join_kernel, dim3((unsigned)ceil_div(size, 1024), p.slots), dim3(256), 0, s, p, group, g.job[0], g.job[1]);
    }
    return hipGetLastError();
}

}  // namespace halo
