// The gradients of the low-rank adapters, G_V = s_a sum of E_t T_t and G_U = sum of S_t drop(X)_t over an adapter's tokens
// (adapters_device.h has the formulas).
#pragma clang fp contract(off)

#include <type_traits>

#include "adapters_device.h"

namespace halo {
namespace adapters {
namespace {

// The sum over a segment's tokens of big[t, col] * small[t, c]: big bf16 (E for G_V, drop(X) for G_U), small fp32 (T, S).  A workgroup owns 256
// columns of `big`, a wavefront 64, and goes over the places 32 at a time; k of the matrix instructions is the place.  Both operands are loaded
// as they lie, 16 bytes a lane, and turned in LDS: a lane has eight columns of four places of `big`, masked before they go to the wavefront's
// own part of LDS, and four columns of places of `small`, which the four wavefronts stage together, in pieces, two steps in turn.  What is
// multiplied is read from there by the instruction that turns four rows of sixteen values.  (Loaded 8 and 4 bytes a lane, as the matrix
// instructions' lanes want them, it was 68 us instead of 41 at 6328 places, 1024 + 14336 columns, rank 16: the vector memory unit takes as long
// for an instruction of 4 bytes a lane as for one of 16.)  NT: rank tiles of 16, from tile blockIdx.z * NT on.
// Measured: rank 16, those sizes, 194 MB of `big`: 4.7 TB/s, memory.  Rank 64, 8192 places, 14336 + 4096 columns, masked, 302 MB: 107 us,
// 2.8 TB/s; matrix instructions (three for each product of fp32 by bf16), LDS and vector instructions each take a quarter of the time, and
// what they do not cover of each other bounds it.  Registers for three workgroups a compute unit: with two it is 114 us.
template <int NT, bool MASK>
__global__ void __launch_bounds__(64 * kGradWaves, 3)
grad_kernel(GradArgs g) {
    constexpr int THREADS = 64 * kGradWaves, UNITS = 128 * NT, PER = (UNITS + THREADS - 1) / THREADS;     // fours of staging, and per thread
    // bytes from one place to the next: so many more than the values that four of a tile lie in all the banks
    constexpr int BIG = 128 + 32, SMALL = 32 * NT + (NT > 1 ? 32 : 0);
    __shared__ v4u s_big[kGradWaves][32 * BIG / 16], s_small[2][3][32 * SMALL / 16];
    const Segment seg = g.group.segments[blockIdx.y];
    if (seg.adapter < 0) return;
    const bool second = (int)blockIdx.x >= g.job[0].tiles;
    const GradJob& job = g.job[second ? 1 : 0];
    const AdapterPool& p = g.p;
    const int R = p.max_rank, tile0 = blockIdx.z * NT;
    const int64_t wide = job.wide;
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
    const int i16 = lane & 15, kq = lane >> 4;
    const int64_t c0 = (int64_t)((int)blockIdx.x - (second ? g.job[0].tiles : 0)) * kGradCols + wave * 64;
    // loading: eight columns of the places 4 (lane / 8) .. + 4; columns beyond the matrix are not stored
    const int c8 = lane & 7, four = lane >> 3;
    const int64_t col = c0 + 8 * c8, colc = col < wide ? col : 0;
    const bool masked = MASK && second;
    const uint16_t* big = job.big + colc;
    const uint8_t* kept_at = MASK && masked ? g.kept + (c0 < wide ? c0 >> 6 : 0) * p.b * 8 + c8 : nullptr;
    const uint32_t last = (uint32_t)p.b - 1, pitch = 2 * (uint32_t)job.ld;       // bytes
    char* const big_put = reinterpret_cast<char*>(s_big[wave]) + 4 * four * BIG + 16 * c8;
    // turning: lane l of sixteen names the four values l % 4 of the place l / 4 and gets the l-th of all four
    const char* const big_get = reinterpret_cast<const char*>(s_big[wave]) + (8 * kq + (i16 >> 2)) * BIG + 8 * (i16 & 3);
    const int small_get = (8 * kq + (i16 >> 2)) * SMALL + 8 * (i16 & 3);

    v4f acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[t][v] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // the sums, with the mask or without; chosen once
    const auto sum = [&](auto with_mask) {
        constexpr bool M = decltype(with_mask)::value;
        struct Step {
            int token[4];
            v4u raw[4];
            uint32_t kept[4];
        };
        const int steps = (seg.end - seg.begin + 31) >> 5;
        const int* order = g.group.order + seg.begin;
        const auto place0 = [&](int j) { return 32 * (j < steps ? j : 0); };
        const auto row_of = [&](int token) { return (uint32_t)token < last ? (uint32_t)token : last; };
        const auto load_order = [&](int4& token, int j) { token = *reinterpret_cast<const int4*>(order + place0(j) + 4 * four); };
        // A place without a token (-1) loads the last one's row.  Only an adapter's last step has such places; there they are set to zero.
        const auto load_rows = [&](Step& q, const int4& token) {
            q.token[0] = token.x; q.token[1] = token.y; q.token[2] = token.z; q.token[3] = token.w;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t t = row_of(q.token[u]);
                q.raw[u] = *reinterpret_cast<const v4u*>(reinterpret_cast<const char*>(big) + (uint64_t)t * pitch);
                if (M) q.kept[u] = kept_at[t * 8];
            }
        };
        // the thread's fours of `small`, i = 0 .. PER
        const int c4 = tid % (4 * NT), staged_c = 16 * tile0 + 4 * c4;
        const uint32_t small_at = 4 * (staged_c < R ? staged_c : 0);     // columns beyond the rank are not stored
        int staged_token[PER];
        v4f staged[PER];
        const auto load_staged_order = [&](int j) {
#pragma unroll
            for (int i = 0; i < PER; ++i) staged_token[i] = order[place0(j) + (tid + i * THREADS) % UNITS / (4 * NT)];
        };
        const auto load_staged = [&](int (&token)[PER]) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                token[i] = staged_token[i];
                staged[i] = load_at<v4f>(job.small, __umul24(row_of(token[i]), 4 * R) + small_at);         // at most 2^31 bytes
            }
        };
        const auto write_staged = [&](const int (&token)[PER], int j) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                v4f x = staged[i];
                if (j == steps - 1) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = token[i] < 0 ? 0.0f : x[e];
                }
                uint32_t piece[4][3];
#pragma unroll
                for (int e = 0; e < 4; ++e) split(x[e], piece[e]);
                const int at = (tid + i * THREADS) / (4 * NT) * SMALL + 8 * c4;
                if (UNITS % THREADS == 0 || tid < UNITS) {
#pragma unroll
                    for (int k = 0; k < 3; ++k)
                        *reinterpret_cast<uint2*>(reinterpret_cast<char*>(s_small[j & 1][k]) + at) =
                            make_uint2(pack_hi(piece[0][k], piece[1][k]), pack_hi(piece[2][k], piece[3][k]));
                }
            }
        };
        const auto operand = [&](int j, int k, int t) {
            const char* at = reinterpret_cast<const char*>(s_small[j & 1][k]) + small_get + 32 * t;
            return read_transposed(at, at + 4 * SMALL);
        };
        const auto multiply = [&](const Step& q, int j) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                v4u x = q.raw[u];
                if (M) {
#pragma unroll
                    for (int d = 0; d < 4; ++d) x[d] &= pack_lo(bit_mask(q.kept[u], 2 * d), bit_mask(q.kept[u], 2 * d + 1));
                }
                if (j == steps - 1) x = q.token[u] < 0 ? v4u{0, 0, 0, 0} : x;
                *reinterpret_cast<v4u*>(big_put + u * BIG) = x;
            }
            __builtin_amdgcn_wave_barrier();
            v4u a[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) a[v] = read_transposed(big_get + 32 * v, big_get + 32 * v + 4 * BIG);
            v4u b[2][3];                                     // one rank tile's operands while the other's are multiplied
#pragma unroll
            for (int k = 0; k < 3; ++k) b[0][k] = operand(j, k, 0);
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (t + 1 < NT) {
#pragma unroll
                    for (int k = 0; k < 3; ++k) b[(t + 1) & 1][k] = operand(j, k, t + 1);
                }
                in_order();
#pragma unroll
                for (int k = 0; k < 3; ++k)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[t][v] = mfma(a[v], b[t & 1][k], acc[t][v]);
                in_order();
            }
        };
        Step even, odd;
        int4 even_next, odd_next;                            // tokens of the steps whose rows are asked for next
        int staged_now[PER];
        // Step j: its part of `small`, on its way since the step before, goes to LDS, that of the next is asked for, and the rows of the step after
        // the next as soon as this one's are used, by tokens that were asked for a step ago, ahead of that step's rows.
        const auto step = [&](Step& q, const int4& q_next, int4& other_next, int j) {
            write_staged(staged_now, j);
            __syncthreads();
            load_staged(staged_now);
            load_staged_order(j + 2);
            multiply(q, j);
            load_order(other_next, j + 3);
            in_order();
            load_rows(q, q_next);
            in_order();
        };
        if (steps > 0) {                                     // the same for the workgroup
            load_staged_order(0);
            load_order(even_next, 0);
            load_order(odd_next, 1);
            load_staged(staged_now);
            load_staged_order(1);
            load_rows(even, even_next);
            in_order();
            load_order(even_next, 2);
            in_order();
            load_rows(odd, odd_next);
            in_order();
#pragma unroll 1
            for (int j = 0; j + 1 < steps; j += 2) {
                step(even, even_next, odd_next, j);
                step(odd, odd_next, even_next, j + 1);
            }
            if (steps & 1) {
                write_staged(staged_now, steps - 1);
                __syncthreads();
                multiply(even, steps - 1);
            }
        }
    };
    if (MASK && second) sum(std::bool_constant<MASK>());
    else sum(std::false_type());
    const int rank = rank_of(p, seg.adapter);
    // Nothing is summed for an adapter without tokens, and its scale, which may be anything, is not used.
    const float scale = scale_of(p, seg.adapter), factor = second ? (masked ? g.factor : 1.0f) : seg.begin < seg.end ? scale : 1.0f;
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
        for (int v = 0; v < 4; ++v) {
            const int64_t oc = c0 + 16 * v + 4 * kq;
            if (oc >= wide || c >= R) continue;
            if (rank_major) {
                *reinterpret_cast<v4f*>(dst + (int64_t)c * wide + oc) = acc[t][v];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) dst[(oc + e) * R + c] = acc[t][v][e];
            }
        }
    }
}

// Adds up the segments of every adapter that has several, in order; four neighbouring elements per thread.
__global__ void __launch_bounds__(256)
grad_join_kernel(AdapterPool p, GroupArgs group, GradJob v, GradJob u) {
    const int a = blockIdx.y;
    const int2 range = group.range[a];
    const int first = range.x / group.chunk, count = Pieces(range.y - range.x, group.chunk).count;
    if (count == 1) return;
    const int64_t size_v = v.tiles ? v.wide * p.max_rank : 0, size_u = u.tiles ? u.wide * p.max_rank : 0;
    int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= size_v + size_u) return;
    const bool second = i >= size_v;
    if (second) i -= size_v;
    const GradJob& job = second ? u : v;
    const int64_t size = second ? size_u : size_v;
    v4f sum = *reinterpret_cast<const v4f*>(job.part + (int64_t)(group.cuts + first + 1) * size + i);
    for (int k0 = 1; k0 < count; k0 += 4) {              // four on their way at once
        v4f q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = *reinterpret_cast<const v4f*>(job.part + (int64_t)(first + (k0 + k < count ? k0 + k : k0)) * size + i);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k0 + k < count) sum += q[k];
    }
    *reinterpret_cast<v4f*>(job.out + (int64_t)a * size + i) = sum;
}

// Workgroups that the segments are cut for, two a compute unit.  Registers leave room for three, but cut for 768 the sums and their joins take
// as long: 8192 tokens, 14336 + 4096 columns, rank 64 110 us and 113, 2048, 4096 + 4096, rank 16 19 and 20.5, 4096 of them, rank 32 29 and 28.
constexpr int64_t kFill = 512;

template <int NT>
void launch_as(const GradArgs& g, hipStream_t s) {
    const int rank_tiles = (int)ceil_div(g.p.max_rank, 16);
    const dim3 grid(g.job[0].tiles + g.job[1].tiles, g.p.slots + g.group.cuts, (unsigned)ceil_div(rank_tiles, NT)), block(64 * kGradWaves);
    if (g.kept) hipLaunchKernelGGL((grad_kernel<NT, true>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((grad_kernel<NT, false>), grid, block, 0, s, g);
}

}  // namespace

// Segments are cut so that together with the column tiles they are kFill workgroups: every further one costs a partial sum that is written and
// read again.  Few tokens have little to be read: a segment of several is at least 64 places, and its partial sum as much as what it reads.
int grad_chunk(int64_t b, int64_t places, int64_t m, int64_t n, int max_rank) {
    const int64_t tiles = ceil_div(m, kGradCols) + ceil_div(n, kGradCols), wanted = kFill > tiles ? kFill / tiles : 1;
    int64_t chunk = ceil_div(places, wanted), least = 2 * max_rank < 64 ? 64 : 2 * max_rank;
    if (chunk < least) chunk = least;
    if (b <= 256) chunk = places;                        // the sums' own launch would cost more
    return (int)(ceil_div(chunk, 32) * 32);
}

hipError_t launch_grads(const GradArgs& g, hipStream_t s) {
    const int R = g.p.max_rank;
    if (R <= 16) launch_as<1>(g, s);
    else if (R <= 32) launch_as<2>(g, s);
    else launch_as<4>(g, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.group.cuts <= 1) return e;
    const int64_t size = ((g.job[0].tiles ? g.p.n : 0) + (g.job[1].tiles ? g.p.m : 0)) * R;
    hipLaunchKernelGGL(grad_join_kernel, dim3((unsigned)ceil_div(size, 1024), g.p.slots), dim3(256), 0, s, g.p, g.group, g.job[0], g.job[1]);
    return hipGetLastError();
}

}  // namespace adapters
}  // namespace halo
