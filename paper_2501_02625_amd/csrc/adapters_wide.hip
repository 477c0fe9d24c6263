// The wide results of the low-rank adapters, Y = base + s_a T V_a^T and E_X = base + drop'(S U_a) (adapters_device.h has the formulas).
#pragma clang fp contract(off)

#include "adapters_device.h"

namespace halo {
namespace adapters {
namespace {

// Two values rounded to bf16, side by side.
__device__ __forceinline__ uint32_t round_two(float x, float y) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    typedef float v2f __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{x, y}, v2bf));
}

// Eight neighbouring elements of base or result, as they are in memory.
template <bool F32>
struct Eight {
    v4u q[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void* from) {
        const v4u* s = reinterpret_cast<const v4u*>(from);
        q[0] = s[0];
        if constexpr (F32) q[1] = s[1];
    }
    __device__ __forceinline__ void store(void* to) const {
        v4u* o = reinterpret_cast<v4u*>(to);
        o[0] = q[0];
        if constexpr (F32) o[1] = q[1];
    }
    // keep: all ones, or 0 for nothing
    __device__ __forceinline__ void add_to(float (&y)[8], uint32_t keep) const {
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
    __device__ __forceinline__ void exchange(Eight& other, bool odd) {
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

// A block of 64 features of an adapter, the first operand of the matrix instructions: 16-byte loads of V, or four neighbouring columns of eight
// rank rows of U, packed.  Every lane loads, from a place that exists; what is not the adapter's is cleared in finish().
// RC: rank chunks of 32.  RC == 0 (rank up to 16): the second operand's values are split in four pieces, of which the halves of an
// instruction's 32 products hold two and two, two instructions instead of three, and the first operand twice.
template <int RC_, bool BWD>
struct AdapterBlock {
    static constexpr bool STACK = RC_ == 0;
    static constexpr int RC = STACK ? 1 : RC_;
    v4u w[RC][4];                                        // as loaded; after finish(): operand q of rank chunk c
    // Features (from the block's first) of a result lane's run q of eight, q = 0, 1, and the e-th of them in the instructions' results.
    __device__ __forceinline__ static int run(int kg, int q) { return BWD ? 16 * kg + 8 * q : 32 * q + 8 * kg; }
    __device__ __forceinline__ static float result(const v4f (&acc)[4], int q, int e) {
        return BWD ? acc[e & 3][2 * q + (e >> 2)] : acc[2 * q + (e >> 2)][e & 3];
    }
    // b: the adapter, of at most 2^30 bytes
    __device__ __forceinline__ void load(const uint16_t* b, int R, uint32_t wide, uint32_t f0, int lr, int r_lane) {
        if constexpr (!BWD) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t f = f0 + 32 * (q >> 1) + 8 * (lr >> 2) + 4 * (q & 1) + (lr & 3);
                if (f >= wide) f = wide - 1;             // its results are not stored
#pragma unroll
                for (int c = 0; c < RC; ++c) {
                    const int r = 32 * c + r_lane;
                    w[c][q] = load_at<v4u>(b, 2 * (f * R + (r < R ? r : 0)));
                }
            }
        } else {
            uint32_t col = f0 + 4 * lr;
            if (col >= wide) col = 0;                    // its results are not stored
#pragma unroll
            for (int c = 0; c < RC; ++c) {
                const int r = 32 * c + r_lane;           // R is a multiple of eight
                uint32_t at = 2 * ((r < R ? r : 0) * wide + col);
#pragma unroll
                for (int u = 0; u < 8; ++u, at += 2 * wide) {
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
                    if constexpr (!BWD) {                // dword j of every operand: the ranks r + 2 j, r + 2 j + 1
                        const uint32_t keep = (r + 2 * j < rank ? 0xFFFFu : 0u) | (r + 2 * j + 1 < rank ? 0xFFFF0000u : 0u);
#pragma unroll
                        for (int q = 0; q < 4; ++q) w[c][q][j] &= keep;
                    } else {                             // two dwords of the rank row r + 2 j, two of the next
                        const uint32_t even = r + 2 * j < rank ? ~0u : 0u, odd = r + 2 * j + 1 < rank ? ~0u : 0u;
                        w[c][j] &= v4u{even, even, odd, odd};
                    }
                }
            }
        }
        if constexpr (BWD) {
#pragma unroll
            for (int c = 0; c < RC; ++c) {
                uint2 x[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = make_uint2(w[c][u >> 1][2 * (u & 1)], w[c][u >> 1][2 * (u & 1) + 1]);
                columns_of(x, w[c]);
            }
        }
    }
};

// A workgroup owns a tile of 16 MT tokens, the columns of its matrix instructions, whose thin values it keeps in LDS as the operands' lanes
// hold them, split in pieces; of the different adapters among the tokens it takes every gridDim.z-th.  Its wavefronts go over blocks of 64
// features, the rows: a step is a block times 16 tokens.  The base of the next steps and the next block of the adapter are on their way
// meanwhile; nothing is exchanged once the pieces are in LDS.  Tall tiles (MT 16, above rank 64 MT 8) read the adapter once for 256 (128)
// tokens, little next to base and result; short ones give few tokens more workgroups.
// Measured: forward, 8192 tokens, 14336 features, rank 64, bf16: 117 us, 470 MB of base and result, 4.0 TB/s; a copy of as much takes 92.  At 64
// tokens, 14336 features, 64 adapters of rank 16 it is 14 us for 33 MB: a wavefront has three or four blocks of features and asks for one ahead, so
// that it waits for memory at nearly each of them.
template <int RC_, int MT, int WAVES, bool BWD, bool F32>
__global__ void __launch_bounds__(64 * WAVES, WAVES == 8 || (RC_ == 4 && BWD) ? 1 : 2)
wide_kernel(WideArgs g) {
    constexpr bool STACK = RC_ == 0;
    constexpr int RC = STACK ? 1 : RC_, NP = STACK ? 2 : 3, ROWS = 16 * MT, WORDS = (ROWS + 63) / 64;
    constexpr int DEPTH = MT == 1 || (RC == 2 && BWD && F32) ? 1 : F32 || RC == 4 || (RC == 2 && BWD) ? 2 : 4;     // steps whose base is on its way
    constexpr bool AHEAD = RC <= (MT == 1 ? 1 : 2);      // registers for two blocks of the adapter
    __shared__ v4u s_thin[MT * RC * NP][64];
    __shared__ int s_id[64 * WORDS];
    typedef AdapterBlock<RC_, BWD> Block;
    const AdapterPool& p = g.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
    const int lr = lane & 15, kg = lane >> 4;
    const bool odd = lr & 1;
    const int pair = lr & 14, run = Block::run(kg, lr & 1);
    const int R = p.max_rank;
    const int64_t wide = BWD ? p.m : p.n;
    const int64_t row0 = (int64_t)blockIdx.x * ROWS;
    for (int r = tid; r < 64 * WORDS; r += 64 * WAVES) s_id[r] = r < ROWS && row0 + r < p.b ? p.adapter_of[row0 + r] : -1;
    __syncthreads();
    // this wavefront's blocks of features: every WAVES-th of the workgroup's range, begun at another one by every tile of tokens
    const int blocks = (int)((wide + 63) >> 6), per = (blocks + (int)gridDim.y - 1) / (int)gridDim.y;
    const int block0 = (int)blockIdx.y * per, end = block0 + per < blocks ? block0 + per : blocks;
    const int count = end - block0 > wave ? (end - block0 - wave + WAVES - 1) / WAVES : 0;
    const int turn = count > 0 ? (int)(blockIdx.x % (unsigned)count) : 0;
    const auto f_of = [&](int j) {                       // the first one's where there is no such block
        j = j < count ? j : 0;
        return count > 0 ? (uint32_t)(block0 + wave + (j + turn < count ? j + turn : j + turn - count) * WAVES) * 64 : 0u;
    };
    const int r_lane = STACK ? 8 * (kg & 1) : 8 * kg;
    // without a base: something that is there to be loaded, and nothing of it kept
    const void* base_at = g.base ? g.base : g.out;
    const int64_t base_ld = g.base ? g.ld_base : g.ld_out;
    const uint32_t base_keep = g.base ? ~0u : 0u;
    // and without a mask: something, of which every bit is set
    const uint8_t* kept_at = g.kept ? g.kept : reinterpret_cast<const uint8_t*>(g.part);
    const int64_t kept_block = g.kept ? p.b * 8 : 0;     // bytes from one block of 64 columns to the next
    const uint32_t kept_token = g.kept ? 8 : 0, kept_all = g.kept ? 0u : 0xFFFFu;
    // where the lane's runs of the tile's first pair of tokens begin
    const char* base_lane[2];
    char* out_lane[2];
    constexpr int SIZE = F32 ? 4 : 2;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        base_lane[k] = reinterpret_cast<const char*>(base_at) + ((row0 + pair + k) * base_ld + run) * SIZE;
        out_lane[k] = reinterpret_cast<char*>(g.out) + ((row0 + pair + k) * g.ld_out + run) * SIZE;
    }
    uint64_t todo[WORDS];                                // tokens with an adapter that are not done
#pragma unroll
    for (int w = 0; w < WORDS; ++w) todo[w] = __ballot(is_adapter(p, s_id[w * 64 + lane]));

    // The next adapter of this workgroup: its first token, and bit i of own: the even (odd) token of the lane's pair in step i is its, of steps:
    // any token of step i is.
    unsigned seen = 0;
    int first = -1, a = -1;
    uint32_t own[2] = {0, 0}, steps = 0;
    const auto next_adapter = [&]() {
        a = -1;
        while (true) {
            first = -1;
#pragma unroll
            for (int w = WORDS - 1; w >= 0; --w)
                if (todo[w]) first = w * 64 + __builtin_ctzll(todo[w]);
            if (first < 0) return;
            const int id = __builtin_amdgcn_readfirstlane(s_id[first]);
            own[0] = own[1] = steps = 0;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                const uint64_t mine = __ballot(s_id[w * 64 + lane] == id) & todo[w];
                todo[w] &= ~mine;
#pragma unroll
                for (int i = 0; i < (MT < 4 ? MT : 4); ++i) {
                    const uint32_t sixteen = (uint32_t)(mine >> (16 * i)) & 0xFFFFu;
                    own[0] |= ((sixteen >> pair) & 1u) << (4 * w + i);
                    own[1] |= ((sixteen >> (pair + 1)) & 1u) << (4 * w + i);
                    steps |= (sixteen ? 1u : 0u) << (4 * w + i);
                }
            }
            if (seen++ % gridDim.z == blockIdx.z) { a = id; return; }
        }
    };
    const auto adapter = [&]() { return (BWD ? p.U : p.V) + (int64_t)a * wide * R; };
    Block now, next_block;
    uint64_t bare[WORDS];
#pragma unroll
    for (int w = 0; w < WORDS; ++w) bare[w] = ~todo[w];
    struct Place { int j; uint32_t left; };          // block of features, and the steps left in it, this one the lowest
    const auto after = [&](Place q) {
        q.left &= q.left - 1;
        if (!q.left) { ++q.j; q.left = steps; }
        return q;
    };
    // Base and result go a pair of tokens at a time: lane (i, g) has run i % 2 of the even token, then of the odd one, so that eight lanes
    // take 128 bytes of a row at once.  (Token by token, each half of a line was a request of its own: 137 us instead of 118 at 8192
    // tokens, 14336 features, rank 64.)
    struct Ahead {
        Eight<F32> base[2];
        uint32_t kept;                               // the lane's token's bits of both runs
    };
    Ahead ahead[DEPTH];
    const auto load_ahead = [&](Ahead& x, const Place& q) {
        const int i = __builtin_ctz(q.left);
        const uint32_t f0 = f_of(q.j);
        const int64_t at = (16 * i * base_ld + f0) * SIZE;
        const char* instead = reinterpret_cast<const char*>(base_at) + (row0 + first) * base_ld * SIZE;
#pragma unroll
        for (int k = 0; k < 2; ++k) {                // no base, other adapters' tokens, features and steps beyond: one line for all
            const bool ok = (own[k] & base_keep) >> i & 1 && f0 + run < (uint32_t)wide && q.j < count;
            x.base[k].load(ok ? base_lane[k] + at : instead);
        }
        if constexpr (BWD) {
            const uint32_t t = (uint32_t)(row0 + i * 16 + lr), tc = t < (uint32_t)p.b ? t : (uint32_t)p.b - 1;
            x.kept = kept_all | load_at<uint16_t>(kept_at + (f0 >> 6) * kept_block, tc * kept_token + 2 * kg);
        }
    };
    const auto work = [&](Ahead& x, const Place& q) {
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
        x.base[0].exchange(x.base[1], odd);
        Eight<F32> y[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = Block::result(acc, k, e);
                if (BWD) v[e] = __uint_as_float(__float_as_uint(v[e]) & bit_mask(x.kept, 8 * k + e));
            }
            x.base[k].add_to(v, base_keep);
            y[k].set(v);
        }
        y[0].exchange(y[1], odd);
        const uint32_t f0 = f_of(q.j);
        const int64_t at = (16 * i * g.ld_out + f0) * SIZE;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if ((own[k] >> i) & 1 && f0 + run < (uint32_t)wide) y[k].store(out_lane[k] + at);
    };
    Place at{0, 0}, next{0, 0};
    int rank = 0;
    // What the adapter's first step takes, all on its way at once.
    const auto begin = [&]() {
        at = next = Place{0, steps};
        now.load(adapter(), R, (uint32_t)wide, f_of(0), lr, r_lane);
        rank = rank_of(p, a);
        in_order();
#pragma unroll
        for (int k = 0; k < DEPTH; ++k, next = after(next)) load_ahead(ahead[k], next);
        if (AHEAD) next_block.load(adapter(), R, (uint32_t)wide, f_of(1), lr, r_lane);
    };
    next_adapter();
    if (a < 0 && blockIdx.z > 0) return;                 // the same for the workgroup
    if (a >= 0) begin();
    in_order();

    for (int j = wave; j < MT * RC; j += WAVES) {        // the thin values of the tile's tokens, in pieces
        const int i = j / RC, r = 32 * (j % RC) + r_lane;
        const int64_t t = row0 + i * 16 + lr;
        const int id = s_id[i * 16 + lr];
        const float scale = BWD ? g.factor : is_adapter(p, id) ? scale_of(p, id) : 1.0f;
        v4f lo = v4f{0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
        if (r < R && t < p.b) {                          // R is a multiple of eight
            sum_parts(g.part, g.splits, p.b * R, t * R + r, lo, hi);
            if (g.thin && blockIdx.y == 0 && blockIdx.z == 0 && !(STACK && kg > 1)) {
                *reinterpret_cast<v4f*>(g.thin + t * R + r) = lo;
                *reinterpret_cast<v4f*>(g.thin + t * R + r + 4) = hi;
            }
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (e < 4 ? lo[e & 3] : hi[e & 3]) * scale;
        if (!BWD && !__builtin_isfinite(scale)) {        // beyond the token's own rank there is nothing that it could meet
            const int own_rank = rank_of(p, id);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = r + e < own_rank ? x[e] : 0.0f;
        }
        v4u q[STACK ? 4 : 3];
        split_eight(x, q);
        if constexpr (STACK) {
            s_thin[j * NP][lane] = kg < 2 ? q[0] : q[1];
            s_thin[j * NP + 1][lane] = kg < 2 ? q[2] : q[3];
        } else {
#pragma unroll
            for (int k = 0; k < NP; ++k) s_thin[j * NP + k][lane] = q[k];
        }
    }
    __syncthreads();

    if (count <= 0) return;
    if (blockIdx.z == 0 && g.base != g.out) {            // tokens without an adapter: the base as it is
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            const int r = w * 64 + lane;
            for (uint64_t left = __ballot(r < ROWS && row0 + r < p.b) & bare[w]; left; left &= left - 1) {
                const int64_t t = row0 + w * 64 + __builtin_ctzll(left);
                for (int j = 0; j < count; ++j) {
                    const int64_t f = f_of(j) + 8 * lane;
                    if (lane >= 8 || f >= wide) continue;
                    Eight<F32> x;
                    x.load(reinterpret_cast<const char*>(base_at) + (t * base_ld + f) * SIZE);
                    x.q[0] &= base_keep;
                    if constexpr (F32) x.q[1] &= base_keep;
                    x.store(reinterpret_cast<char*>(g.out) + (t * g.ld_out + f) * SIZE);
                }
            }
        }
    }
#pragma unroll 1
    while (a >= 0) {
        now.finish(rank, r_lane);
#pragma unroll 1
        while (at.j < count) {
#pragma unroll
            for (int k = 0; k < DEPTH; ++k) {
                if (at.j >= count) break;
                work(ahead[k], at);
                load_ahead(ahead[k], next);
                next = after(next);
                const int j = at.j;
                at = after(at);
                if (at.j != j && at.j < count) {
                    if (AHEAD) now = next_block;
                    else now.load(adapter(), R, (uint32_t)wide, f_of(at.j), lr, r_lane);
                    now.finish(rank, r_lane);
                    if (AHEAD) next_block.load(adapter(), R, (uint32_t)wide, f_of(at.j + 1), lr, r_lane);
                }
            }
        }
        next_adapter();
        if (a >= 0) begin();
    }
}

// ------------------------------------------------------------------------------------------------ launches
constexpr int64_t kFill = 256;                           // compute units

template <int RC, int MT, int WAVES, bool BWD>
void launch_as(const WideArgs& g, bool f32, int64_t wanted, hipStream_t s) {
    const int64_t tiles = ceil_div(g.p.b, 16 * MT), blocks = ceil_div(BWD ? g.p.m : g.p.n, 64), strips = ceil_div(blocks, WAVES);
    int64_t lanes = 1;                                   // different adapters of a tile side by side where workgroups are few
    if (MT < 8) {
        int64_t most = 16 * MT < 16 ? 16 * MT : 16;
        if (g.p.b < most) most = g.p.b;
        if (g.p.slots < most) most = g.p.slots;
        // Rank 16, 4096 features, 64 adapters in turn, us with a workgroup for each that there may be in a tile and with as many as fill the chip:
        // 11.2 and 11.7 at 128 tokens, 13.4 and 15.0 at 256, 17.9 and 17.2 at 272; with tokens of one adapter after the other 7.3 and 8.2, 7.5 and
        // 7.4, 9.4 and 9.1.
        lanes = g.p.b <= 256 ? most : wanted / (tiles * strips);
        if (MT == 1 && lanes < 2) lanes = 2;             // for the tiles with a request's border: 16.6 us instead of 19.5 at 2048 x 4096
        if (lanes > most) lanes = most;
        if (lanes < 1) lanes = 1;
    }
    int64_t y = ceil_div(wanted, tiles * lanes);
    if (y > strips) y = strips;
    // As many as one round of workgroups holds, one a compute unit, or several rounds, if that is shorter by the steps of each, its start like
    // four; steps are counted for the workgroup, not for its busiest wavefront.  (To fill the chip at least: 133 us instead of 67 at 6813 x 7096,
    // rank 64, fp32, where that was 270 workgroups.)
    if (MT >= 4) {
        int64_t least = INT64_MAX;
        for (int rounds = 1; rounds <= 8; ++rounds) {
            int64_t k = rounds * kFill / tiles;
            if (k < 1) k = 1;
            if (k > strips) k = strips;
            const int64_t cost = ceil_div(tiles * k, kFill) * (ceil_div(blocks, k) * MT + 4 * WAVES);
            if (cost < least) { least = cost; y = k; }
        }
    }
    y = ceil_div(blocks, ceil_div(blocks, y));
    const dim3 grid((unsigned)tiles, (unsigned)y, (unsigned)lanes), block(64 * WAVES);
    if (f32) hipLaunchKernelGGL((wide_kernel<RC, MT, WAVES, BWD, true>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((wide_kernel<RC, MT, WAVES, BWD, false>), grid, block, 0, s, g);
}

template <int RC, bool BWD>
void launch_by_size(const WideArgs& g, bool f32, hipStream_t s) {
    constexpr int TALL = RC == 4 ? 8 : 16;
    constexpr int WAVES = RC == 4 && BWD ? 4 : 8;        // registers
    const int tokens = wide_tile_tokens(g.p.b, BWD ? g.p.m : g.p.n, g.p.max_rank);
    if (tokens == 16 * TALL) return launch_as<RC, TALL, WAVES, BWD>(g, f32, kFill, s);
    if constexpr (RC < 4) {
        if (tokens == 64) return launch_as<RC, 4, WAVES, BWD>(g, f32, 2 * kFill, s);
    }
    launch_as<RC, 1, 4, BWD>(g, f32, 4 * kFill, s);
}

template <bool BWD>
void launch_by_rank(const WideArgs& g, bool f32, hipStream_t s) {
    const int R = g.p.max_rank;
    if (R <= 16) launch_by_size<0, BWD>(g, f32, s);
    else if (R <= 32) launch_by_size<1, BWD>(g, f32, s);
    else if (R <= 64) launch_by_size<2, BWD>(g, f32, s);
    else launch_by_size<4, BWD>(g, f32, s);
}

}  // namespace

hipError_t launch_wide(const WideArgs& g, bool backward, bool f32, hipStream_t s) {
    if (backward) launch_by_rank<true>(g, f32, s);
    else launch_by_rank<false>(g, f32, s);
    return hipGetLastError();
}

}  // namespace adapters
}  // namespace halo
