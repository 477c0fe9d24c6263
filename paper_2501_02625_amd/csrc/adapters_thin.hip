// The thin results of the low-rank adapters, T = drop(X) U_a^T and S = s_a E V_a, and what a backward call prepares beside them: the tokens by
// their adapters and the mask's bits (adapters_device.h has the formulas).
#pragma clang fp contract(off)

#include <type_traits>

#include "adapters_device.h"

namespace halo {
namespace adapters {
namespace {

// The tokens of a tile by their adapters.  todo: tokens (a bit each) that have one and are not done; next() takes the adapter of the first
// and all tokens that share it.
struct TileAdapters {
    int id;                  // of the lane's token
    uint64_t todo;
    __device__ __forceinline__ TileAdapters(const AdapterPool& p, int id_) : id(id_), todo(__ballot(is_adapter(p, id_))) {}
    __device__ __forceinline__ int next(uint64_t& mine) {
        const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
        mine = __ballot(id == a) & todo;
        todo &= ~mine;
        return a;
    }
};

// One adapter's tokens, written down by a workgroup, which reads all of adapter_of, twice if the adapter has tokens: slots times tokens in
// all.  (S and this at 8192 tokens, 512 columns, rank 8: 10 us up to 1024 slots, 30 at 8192, 104 at 32768, where writing the gradients, zeros
// but for those of four adapters, takes another 344.)  There is a cut at every chunk-th place, and an adapter of several segments, which are
// equally long, has at least as many cuts among its places as segments but the first: these sum into the parts of those cuts k, in order, and
// the first one into cuts + k of the first of them.
template <int THREADS>
__device__ __forceinline__ void group_tokens(const AdapterPool& p, const GroupArgs& g, int a) {
    constexpr int WAVES = THREADS / 64, AHEAD = 8;       // loads on their way at once: there is nothing else to wait for them with
    __shared__ int s_less[WAVES], s_same[WAVES], s_hits[AHEAD * WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
    const int b = (int)p.b, chunk = g.chunk;
    int less = 0, same = 0;
    for (int t0 = 0; t0 < b; t0 += AHEAD * THREADS) {
        int id[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = t0 + i * THREADS + tid;
            id[i] = p.adapter_of[t < b ? t : 0];
            id[i] = t < b ? id[i] : -1;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            less += id[i] >= 0 && id[i] < a;
            same += id[i] == a;
        }
    }
    for (int h = 32; h > 0; h >>= 1) { less += __shfl_xor(less, h); same += __shfl_xor(same, h); }
    if (lane == 0) { s_less[wave] = less; s_same[wave] = same; }
    __syncthreads();
    less = same = 0;
    for (int w = 0; w < WAVES; ++w) { less += s_less[w]; same += s_same[w]; }
    const int begin = (less + 31) / 32 * 32 + 32 * a, end = begin + same;
    if (tid == 0) g.range[a] = make_int2(begin, end);
    const int after = (less + same + 31) / 32 * 32 + 32 * (a + 1);     // where the next adapter begins
    const Pieces pieces(same, chunk);
    const int index = a + begin / chunk, next = a == p.slots - 1 ? p.slots + g.cuts : a + 1 + after / chunk;
    for (int i = tid; index + i < next; i += THREADS) {
        Segment q{-1, 0, 0, -1};
        if (i < pieces.count) {
            const int cut = begin / chunk + i;
            q.adapter = a;
            q.begin = begin + i * pieces.size;
            q.end = i == pieces.count - 1 ? end : q.begin + pieces.size;
            q.part = pieces.count == 1 ? -1 : i == 0 ? g.cuts + cut + 1 : cut;
        }
        g.segments[index + i] = q;
    }
    if (tid < after - end) g.order[end + tid] = -1;      // fewer than 64 places
    int at = begin;
    for (int t0 = 0; t0 < b && same > 0; t0 += AHEAD * THREADS) {
        uint64_t hits[AHEAD];
        int id[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = t0 + i * THREADS + tid;
            id[i] = p.adapter_of[t < b ? t : 0];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) hits[i] = __ballot(t0 + i * THREADS + tid < b && id[i] == a);
        __syncthreads();
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) s_hits[i * WAVES + wave] = __builtin_popcountll(hits[i]);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            int before = 0, all = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                before += w < wave ? s_hits[i * WAVES + w] : 0;
                all += s_hits[i * WAVES + w];
            }
            const int to = at + before + __builtin_popcountll(hits[i] & ((1ull << lane) - 1));
            if (((hits[i] >> lane) & 1) && to < end) g.order[to] = t0 + i * THREADS + tid;
            at += all;
        }
    }
}

// 64 bits of the mask per thread.  Drawn once here and not by both of the kernels that use them: eight elements cost ten rounds of two
// 64-bit products, and those kernels have their own work for the vector units, where the one that this rides with waits for memory.
template <int THREADS>
__device__ __forceinline__ void draw_mask(const AdapterPool& p, const BackwardExtras& x, int64_t block) {
    const int64_t at = block * THREADS + threadIdx.x, word = at / p.b, row = at - word * p.b;
    if (at >= kept_words(p.b, p.m)) return;
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo |= kept_eight(x.drop, (uint32_t)row, (uint32_t)word * 8 + i) << (8 * i);
        hi |= kept_eight(x.drop, (uint32_t)row, (uint32_t)word * 8 + 4 + i) << (8 * i);
    }
    reinterpret_cast<uint2*>(x.kept)[at] = make_uint2(lo, hi);
}

template <int THREADS>
__device__ __forceinline__ void do_extra(const AdapterPool& p, const BackwardExtras& x, int64_t i) {
    if (i < x.groups) group_tokens<THREADS>(p, x.group, (int)i);
    else if (x.kept) draw_mask<THREADS>(p, x, i - x.groups);
}

__global__ void __launch_bounds__(256)
extras_kernel(AdapterPool p, BackwardExtras x) { do_extra<256>(p, x, blockIdx.x); }

// ------------------------------------------------------------------------------------------------ few tokens
// part[split][t][c] = factor * sum over the split's k of in[t, k] * B_a[k, c]; B_a = U_a^T (K-contiguous) or, with KMAJOR, V_a (rows of
// max_rank).  factor: that of dropout, or with KMAJOR scale_a.  A workgroup owns 16 tokens and, of the different adapters among them, every
// lanes-th; its wavefronts and the splits take 64-element chunks of K round robin (a chunk is one 128-byte line of every row), so that a
// single token is read by as many wavefronts as it has lines.  Rows of other adapters' tokens are replaced by one of the adapter's own: no
// line is fetched for them.  KMAJOR: the lane loads NT neighbouring columns of eight rows at once and packs them, so instruction t covers the
// columns l % 16 * NT + t.  Columns beyond the adapter's rank are summed like the others and stored as zero.
constexpr int kFewWaves = 8;

struct ThinArgs {
    AdapterPool p;
    const uint16_t* in;
    int64_t ld;
    float* part;             // [splits][b][max_rank]
    DropoutMask drop;
    int tiles, splits, lanes;
    BackwardExtras extras;
};

// What a workgroup does.  The order in which they begin: the adapters' groups, which wait longest; each tile's first adapter, all splits of it;
// the other adapters, most of which most tiles do not have; and the mask, for which vector units are left over until then.
struct Place { int64_t extra; int tile, split, lane; };

template <bool KMAJOR>
__device__ __forceinline__ Place place_of(const ThinArgs& g) {
    if (!KMAJOR) return Place{-1, (int)blockIdx.x, (int)blockIdx.y, (int)blockIdx.z};      // the same order, and nothing to divide by
    const unsigned groups = g.extras.groups, tiles = (unsigned)(g.tiles * g.splits) * g.lanes, i = blockIdx.x - groups;
    if (blockIdx.x < groups) return Place{(int64_t)blockIdx.x, 0, 0, 0};
    if (i >= tiles) return Place{(int64_t)blockIdx.x - tiles, 0, 0, 0};
    const unsigned j = i / (unsigned)g.tiles;
    return Place{-1, (int)(i - j * g.tiles), (int)(j % (unsigned)g.splits), (int)(j / (unsigned)g.splits)};
}

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

template <int NT, bool KMAJOR, bool DROP>
__global__ void __launch_bounds__(64 * kFewWaves)
thin_few_kernel(ThinArgs g) {
    __shared__ float s_part[kFewWaves][NT][4][64];       // [wavefront][rank tile][register][lane]
    __shared__ int s_id[64];
    const AdapterPool& p = g.p;
    const Place at = place_of<KMAJOR>(g);
    if (KMAJOR && at.extra >= 0) {
        do_extra<64 * kFewWaves>(p, g.extras, at.extra);
        return;
    }
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int lr = lane & 15, kg = lane >> 4;
    const int R = p.max_rank;
    const int64_t K = KMAJOR ? p.n : p.m;
    const int64_t row0 = (int64_t)at.tile * 16;
    const int split = at.split, splits = g.splits;
    float* part = g.part + (int64_t)split * p.b * R;
    // read once, so that all wavefronts go the same way
    if (wave == 0) s_id[lane] = lane < 16 && row0 + lane < p.b ? p.adapter_of[row0 + lane] : -1;
    __syncthreads();
    TileAdapters tile(p, s_id[lane]);
    if (at.lane == 0) {                                  // tokens without an adapter
        for (uint64_t bare = __ballot(lane < 16 && row0 + lane < p.b) & ~tile.todo; bare; bare &= bare - 1)
            for (int c = threadIdx.x; c < R; c += 64 * kFewWaves) part[(row0 + __builtin_ctzll(bare)) * R + c] = 0.0f;
    }
    const int chunks = (int)((K + 63) >> 6), chunk0 = split * kFewWaves + wave, step = splits * kFewWaves;
    const int count = chunks > chunk0 ? (chunks - chunk0 + step - 1) / step : 0;
    for (unsigned seen = 0; tile.todo; ++seen) {
        uint64_t mine;
        const int a = tile.next(mine);
        if (seen % g.lanes != (unsigned)at.lane) continue;
        const uint32_t token = (uint32_t)(row0 + ((mine >> lr) & 1 ? lr : __builtin_ctzll(mine)));
        const uint16_t* row = g.in + (int64_t)token * g.ld;
        // columns beyond the pool's are replaced by the first one and not stored
        const uint16_t* b = (KMAJOR ? p.V : p.U) + (int64_t)a * K * R;       // an adapter has at most 2^30 bytes
        uint32_t bat[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (KMAJOR) bat[t] = 2 * (lr * NT < R ? lr * NT : 0);
            else bat[t] = 2 * ((uint32_t)(t * 16 + lr < R ? t * 16 + lr : 0) * (uint32_t)K);
        }
        v4f acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        struct Chunk { v4u x[2], b[2][NT]; };
        const auto load = [&](Chunk& q, int j) {         // eights beyond K: the row's first, which count as zero
            const uint32_t k0 = (uint32_t)(chunk0 + (j < count ? j : 0) * step) * 64;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t k = k0 + h * 32 + kg * 8, kc = k < (uint32_t)K ? k : 0;
                q.x[h] = *reinterpret_cast<const v4u*>(row + kc);
                load_b<NT, KMAJOR>(q.b[h], b, bat, kc, R);
            }
        };
        const auto multiply = [&](Chunk& q, int j) {
            const uint32_t k0 = (uint32_t)(chunk0 + j * step) * 64;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t k = k0 + h * 32 + kg * 8;
                if (DROP) q.x[h] = drop_eight(g.drop, q.x[h], token, k >> 3);
                if (k0 + 64 > (uint32_t)K && k >= (uint32_t)K) {
                    q.x[h] = v4u{0, 0, 0, 0};
#pragma unroll
                    for (int t = 0; t < NT; ++t) q.b[h][t] = v4u{0, 0, 0, 0};
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = mfma(q.x[h], q.b[h][t], acc[t]);
            }
        };
        if (count > 0) {
            Chunk even, odd;
            load(even, 0);
            if (count > 1) {
                in_order();
                load(odd, 1);
#pragma unroll 1
                for (int j = 0; j + 1 < count; j += 2) {
                    multiply(even, j);
                    load(even, j + 2);
                    multiply(odd, j + 1);
                    load(odd, j + 3);
                }
            }
            if (count & 1) multiply(even, count - 1);
        }
        const int rank = rank_of(p, a);
        const float factor = KMAJOR ? scale_of(p, a) : DROP ? g.drop.factor : 1.0f;
        // the wavefronts' sums meet in LDS and are added in wavefront order
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_part[wave][t][e][lane] = acc[t][e];
        __syncthreads();
        for (int idx = threadIdx.x; idx < NT * 256; idx += 64 * kFewWaves) {
            const int t = idx >> 8, e = (idx >> 6) & 3, l = idx & 63;
            float sum = s_part[0][t][e][l];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) sum += s_part[w][t][e][l];
            const int r = 4 * (l >> 4) + e;
            const int c = KMAJOR ? (l & 15) * NT + t : t * 16 + (l & 15);
            if (((mine >> r) & 1) && c < R) part[(row0 + r) * R + c] = c < rank ? sum * factor : 0.0f;
        }
    }
}

// ------------------------------------------------------------------------------------------------ many tokens
// The same sums: a wavefront owns 16 tokens and all of the split's K, in steps of 128; the four of a workgroup share the step's part of the
// adapter, which is staged in LDS, two steps in turn, that of the next step on its way.  What a wavefront keeps for itself is its rows of the
// next two steps, on their way: 16 registers a step.  Each tile of tokens begins at another step: rows lie whole powers of two apart, and
// tiles in step would ask the same few memory channels at a time.
// The vector memory unit takes as long for an instruction that brings 8 bytes a lane as for one of 16, so both are loaded 16 bytes at a time.
// KMAJOR: the adapter's rows go to LDS as they are and are turned as they are read, for which the hardware has an instruction (eight rows of
// four columns loaded and packed by each thread: 97 us instead of 69 at 6328 tokens, K = 14336, rank 16); and the tokens' rows are loaded by
// whole lines, sixteen lanes 256 bytes, and turned in LDS as well (12.5 -> 9.7 us at 2048 tokens, K = 4096, rank 16; without the adapter's
// work of turning, in the other direction, it costs more than it gives: 15.0 -> 16.4 at 1037 tokens, rank 64).
// Measured: forward, dropout, 8192 tokens, K = 4096, rank 64: 38 us, where drawing as many bits and nothing else takes 8; backward, 6328
// tokens, K = 14336, rank 16: 58 us, 3.1 TB/s; what bounds it is each step's chain of LDS reads and writes, and workgroups of uneven work.
constexpr int kRowWaves = 4;
constexpr int kRowTile = 16 * kRowWaves;                 // tokens of a workgroup

template <int NT, bool KMAJOR, bool DROP>
__global__ void __launch_bounds__(64 * kRowWaves, NT == 8 ? 1 : 2)
thin_rows_kernel(ThinArgs g) {
    constexpr int THREADS = 64 * kRowWaves, KS = 128;
    // KMAJOR: the adapter's rows as they are, 32 bytes for a tile of 16 columns and so many more that four rows of a tile lie in all the banks
    constexpr int PITCH = 32 * NT + (NT > 1 ? 32 : 0);
    __shared__ v4u s_b[2][KMAJOR ? KS * PITCH / 16 : KS / 32 * NT * 64], s_x[KMAJOR ? kRowWaves : 1][16][KS / 8];
    __shared__ int s_id[kRowTile];
    const AdapterPool& p = g.p;
    const Place at = place_of<KMAJOR>(g);
    if (KMAJOR && at.extra >= 0) {
        do_extra<THREADS>(p, g.extras, at.extra);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
    const int lr = lane & 15, kg = lane >> 4;
    const int R = p.max_rank;
    const int64_t K = KMAJOR ? p.n : p.m;
    const int64_t row0 = (int64_t)at.tile * kRowTile;
    float* part = g.part + (int64_t)at.split * p.b * R;
    // read once, so that all wavefronts go the same way
    if (wave == 0) s_id[lane] = row0 + lane < p.b ? p.adapter_of[row0 + lane] : -1;
    __syncthreads();
    TileAdapters tile(p, s_id[lane]);
    if (at.lane == 0) {                                  // tokens without an adapter
        for (uint64_t bare = __ballot(row0 + lane < p.b) & ~tile.todo; bare; bare &= bare - 1)
            for (int c = tid; c < R; c += THREADS) part[(row0 + __builtin_ctzll(bare)) * R + c] = 0.0f;
    }
    const int steps = (int)((K + KS - 1) / KS), per = (steps + g.splits - 1) / g.splits;
    const int step0 = at.split * per, count = steps - step0 < per ? steps - step0 : per;      // count > 0
    const int turn = (int)((unsigned)at.tile % (unsigned)count);
    const auto k_of = [&](int j) { return (uint32_t)(step0 + (j + turn < count ? j + turn : j + turn - count)) * KS; };
    for (unsigned seen = 0; tile.todo; ++seen) {
        uint64_t mine;
        const int a = tile.next(mine);
        if (seen % g.lanes != (unsigned)at.lane) continue;
        const auto token_of = [&](int r) { return (uint32_t)(row0 + ((mine >> r) & 1 ? r : __builtin_ctzll(mine))); };
        const uint32_t token = token_of(wave * 16 + lr);
        const uint16_t* row[4];                          // those that the lane loads, sixteen lanes 256 bytes of each
#pragma unroll
        for (int h = 0; h < 4; ++h) row[h] = g.in + (int64_t)(KMAJOR ? token_of(wave * 16 + 4 * h + kg) : token) * g.ld;
        const uint16_t* b = (KMAJOR ? p.V : p.U) + (int64_t)a * K * R;       // of at most 2^30 bytes

        v4u x[2][4], staged[NT];
        // The adapter's eights that the thread stages, i = 0 .. NT: of a column (128 bytes of it by eight neighbouring threads), or of a row
        uint32_t k8[NT], from[NT], to[NT];               // where it begins along K, in memory (bytes, from the step on) and in LDS
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            uint32_t u = tid + i * THREADS;
            if constexpr (KMAJOR) {
                if (u >= 16u * R) u = 0;                 // more columns than there are: others load the first eight too
                k8[i] = u / (R >> 3);
                from[i] = 16 * u;
                to[i] = k8[i] * (PITCH / 16) + u % (R >> 3);
            } else {
                const uint32_t c = (u >> 3) % (16 * NT), e = (u & 7) + 8 * (u / (128 * NT));
                k8[i] = 8 * e;
                from[i] = 2 * ((c < (uint32_t)R ? c : 0) * (uint32_t)K + k8[i]);
                to[i] = ((e >> 2) * NT + (c >> 4)) * 64 + operand_slot(c & 15, e & 3);
            }
        }
        // of the last step again where there are no more
        const auto load_x = [&](v4u (&x)[4], int j) {
            const uint32_t k0 = k_of(j < count ? j : count - 1);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const uint32_t k = k0 + (KMAJOR ? lr : 4 * h + kg) * 8;
                x[h] = *reinterpret_cast<const v4u*>(row[h] + (k < (uint32_t)K ? k : 0));
            }
        };
        const auto load_staged = [&](int j) {
            const uint32_t k0 = k_of(j < count ? j : count - 1);
#pragma unroll
            for (int i = 0; i < NT; ++i) staged[i] = load_at<v4u>(b, k0 + k8[i] < (uint32_t)K ? 2 * k0 * (KMAJOR ? R : 1) + from[i] : 0);
        };
        const auto write_staged = [&](int j) {
            const uint32_t k0 = k_of(j);
#pragma unroll
            for (int i = 0; i < NT; ++i) s_b[j & 1][to[i]] = k0 + k8[i] < (uint32_t)K ? staged[i] : v4u{0, 0, 0, 0};
        };
        const auto operand = [&](int j, int h, int t) {
            if constexpr (KMAJOR) {                      // sixteen lanes read four rows of the tile, each of them gets a column
                const char* at = reinterpret_cast<const char*>(s_b[j & 1]) + (32 * h + 8 * kg + (lr >> 2)) * PITCH + 32 * t + 8 * (lr & 3);
                return read_transposed(at, at + 4 * PITCH);
            } else return s_b[j & 1][(h * NT + t) * 64 + operand_slot(lr, kg)];
        };
        v4f acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        const auto multiply = [&](v4u (&x)[4], int j) {
            const uint32_t k0 = k_of(j);
            v4u q[2][NT];                                // one instruction's operands while the other's are multiplied
            // from as they are loaded to as they are multiplied, through the wavefront's own part of LDS
            if constexpr (KMAJOR) {
#pragma unroll
                for (int h = 0; h < 4; ++h) s_x[wave][4 * h + kg][lr ^ (kg + 4 * (h & 1))] = x[h];
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int h = 0; h < 4; ++h) x[h] = s_x[wave][lr][(4 * h + kg) ^ (lr & 7)];
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) q[0][t] = operand(j, 0, t);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                if (h < 3) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) q[(h + 1) & 1][t] = operand(j, h + 1, t);
                }
                in_order();
                x[h] = k0 + h * 32 + kg * 8 < (uint32_t)K ? x[h] : v4u{0, 0, 0, 0};
                if (DROP) x[h] = drop_eight(g.drop, x[h], token, ((k0 + h * 32) >> 3) + kg);
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = mfma(x[h], q[h & 1][t], acc[t]);
                in_order();
            }
        };
        __syncthreads();                                 // the adapter before may still be read
        // Step j: the adapter's part, on its way since the step before, goes to LDS, that of the next step is asked for, and the rows of the
        // step after the next as soon as this one's registers are free.
        const auto step = [&](v4u (&x)[4], int j) {
            write_staged(j);
            __syncthreads();
            load_staged(j + 1);
            multiply(x, j);
            load_x(x, j + 2);
            in_order();
        };
        load_staged(0);                                  // first: it is waited for first
        in_order();
        load_x(x[0], 0);
        load_x(x[1], 1);
#pragma unroll 1
        for (int j = 0; j + 1 < count; j += 2) {
            step(x[0], j);
            step(x[1], j + 1);
        }
        if (count & 1) {
            write_staged(count - 1);
            __syncthreads();
            multiply(x[0], count - 1);
        }
        const int rank = rank_of(p, a);
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

// ------------------------------------------------------------------------------------------------ launches
// From here on thin_rows_kernel.  Where the kernels cross depends on K as well, which this rule does not: us of thin_few_kernel and
// thin_rows_kernel, forward, four adapters, requests in turn:
//    tokens       K = 1024, rank 16 and 64       K = 4096, rank 16 and 64
//       512      3.8  5.5      5.4  6.4          3.9  7.4      6.6  9.2
//       777      3.8  5.6      5.5  6.6          5.6  7.5     13.1  9.4
//      1037      3.8  5.5      5.5  6.6          8.0  7.5     18.0  9.4
//      2048      3.9  5.5      6.5  6.7          8.7  7.6     20.3 10.9
//      4096      5.0  5.7     12.4  6.9         12.5  8.9     29.0 12.3
constexpr int64_t kManyTokens = 1024;
constexpr int64_t kFill = 512, kCompute = 256;           // workgroups that fill the chip, and its compute units

int64_t extra_blocks(const AdapterPool& p, const BackwardExtras& x, int threads) {
    return x.groups + (x.kept ? ceil_div(kept_words(p.b, p.m), threads) : 0);
}

template <int NT, bool KMAJOR>
void launch_as(ThinArgs g, const ThinPlan& q, hipStream_t s) {
    const bool drop = !KMAJOR && g.drop.least;
    const int threads = 64 * (q.rows ? kRowWaves : kFewWaves);
    g.tiles = (int)ceil_div(g.p.b, q.rows ? kRowTile : 16);
    g.splits = q.splits;
    g.lanes = q.lanes;
    const int64_t all = (int64_t)g.tiles * q.splits * q.lanes + extra_blocks(g.p, g.extras, threads);
    const dim3 grid = KMAJOR ? dim3((unsigned)all) : dim3(g.tiles, q.splits, q.lanes), block(threads);
    if (q.rows && drop) hipLaunchKernelGGL((thin_rows_kernel<NT, KMAJOR, !KMAJOR>), grid, block, 0, s, g);
    else if (q.rows) hipLaunchKernelGGL((thin_rows_kernel<NT, KMAJOR, false>), grid, block, 0, s, g);
    else if (drop) hipLaunchKernelGGL((thin_few_kernel<NT, KMAJOR, !KMAJOR>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((thin_few_kernel<NT, KMAJOR, false>), grid, block, 0, s, g);
}

template <bool KMAJOR>
void launch_by_rank(const ThinArgs& g, const ThinPlan& q, hipStream_t s) {
    const int R = g.p.max_rank;
    if (R <= 16) launch_as<1, KMAJOR>(g, q, s);
    else if (R <= 32) launch_as<2, KMAJOR>(g, q, s);
    else if (R <= 64) launch_as<4, KMAJOR>(g, q, s);
    else launch_as<8, KMAJOR>(g, q, s);
}

}  // namespace

ThinPlan thin_plan(int64_t b, int64_t K, int slots) {
    ThinPlan q;
    q.rows = b >= kManyTokens;
    const int64_t tiles = ceil_div(b, q.rows ? kRowTile : 16);
    int64_t most = q.rows ? 8 : 16;                      // different adapters in a tile that get a workgroup of their own
    if (b < most) most = b;
    if (slots < most) most = slots;
    const int64_t chunks = ceil_div(K, q.rows ? 128 : 64 * kFewWaves);
    int64_t splits = 0;
    if (q.rows) {
        // One workgroup a compute unit, and room beside it for a tile's other adapters, which are other workgroups' from the beginning: done
        // by one after the other they made the tiles at the requests' borders twice as long as all (58 us instead of 39 at 8192 tokens,
        // K = 4096, rank 64, dropout).  More splits than four cost more where their parts are summed than they give here.
        splits = kCompute / (tiles > 0 ? tiles : 1);
        if (splits > 4) splits = 4;
        if (splits > chunks / 3) splits = chunks / 3;
        if (splits < 1) splits = 1;
        int64_t lanes = kFill / ((tiles > 0 ? tiles : 1) * splits);
        if (lanes < 4) lanes = tiles * splits <= 4 * kFill ? 4 : 1;      // so many tiles are several rounds of workgroups anyway
        q.lanes = (int)(lanes < most ? lanes : most);
    } else {
        // Few tokens: a workgroup for each adapter that there may be in a tile; more than 256: for a second one only.  K = 4096, rank 16, 64
        // adapters, tokens of one adapter after the other and in turn, us with a workgroup each and with two: 5.6 and 10.2, 5.6 and 10.2 at
        // 64 tokens; 5.0 and 6.1, 6.5 and 11.2 at 128; 6.2 and 4.2, 8.8 and 11.2 at 256; 8.8 and 6.0, 12.3 and 12.0 at 272.
        if (b > 256 && most > 2) most = 2;
        q.lanes = (int)(most < 1 ? 1 : most);
        const int64_t busy = b <= 256 ? tiles * q.lanes : tiles;
        splits = kFill / (busy > 0 ? busy : 1);
        if (splits > 8) splits = 8;
        if (splits > chunks) splits = chunks;
        if (splits < 1) splits = 1;
    }
    q.splits = (int)ceil_div(chunks, ceil_div(chunks, splits));      // none without a chunk
    if (q.splits < 1) q.splits = 1;
    return q;
}

hipError_t launch_thin(const AdapterPool& p, bool backward, const uint16_t* in, int64_t ld, float* part, const DropoutMask& drop,
                       const ThinPlan& plan, const BackwardExtras& extras, hipStream_t s) {
    ThinArgs g{};
    g.p = p; g.in = in; g.ld = ld; g.part = part; g.drop = drop; g.extras = extras;
    if (backward) launch_by_rank<true>(g, plan, s);
    else launch_by_rank<false>(g, plan, s);
    return hipGetLastError();
}

hipError_t launch_extras(const AdapterPool& p, const BackwardExtras& extras, hipStream_t s) {
    const int64_t blocks = extra_blocks(p, extras, 256);
    if (blocks > 0) hipLaunchKernelGGL(extras_kernel, dim3((unsigned)blocks), dim3(256), 0, s, p, extras);
    return hipGetLastError();
}

}  // namespace adapters
}  // namespace halo
