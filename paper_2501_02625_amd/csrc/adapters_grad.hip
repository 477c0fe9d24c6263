// The gradients of the low-rank adapters, G_V = s_a sum of E_t T_t and G_U = sum of S_t drop(X)_t over an adapter's tokens
// (adapters_device.h has the formulas).
#pragma clang fp contract(off)

#include <type_traits>

#include "adapters_device.h"

namespace halo {
namespace adapters {
namespace {

// The sum over a segment's tokens of big[t, col] * small[t, c]: big bf16 (E for G_V, drop(X) for G_U), small fp32 (T, S).  A workgroup owns 256
// columns of `big`, a wavefront 64, and goes over the places 32 at a time.  k of the matrix instructions is the place: lane l supplies the
// eight places 8 (l / 16) .. + 8 of the step.  `big` is read four neighbouring columns of a token at a time; the v-th of them, packed over
// the eight tokens, is the first operand of the v-th instruction, which covers the columns 4 i + v.  The step's part of `small` is fetched by
// the four wavefronts together and staged in LDS in pieces, two steps in turn.  NT: rank tiles of 16, from tile blockIdx.z * NT on.
template <int NT, bool MASK>
__global__ void __launch_bounds__(64 * kGradWaves, 2)
grad_kernel(GradArgs g) {
    constexpr int THREADS = 64 * kGradWaves, UNITS = NT * 64;            // eight values of a column: staging, at most one per thread
    __shared__ v4u s_small[2][NT * 3][64];
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
    const int64_t col = c0 + 4 * i16, colc = col < wide ? col : 0;       // columns beyond the matrix are not stored
    const bool masked = MASK && second;
    const uint16_t* big = job.big + colc;
    const uint8_t* kept_at = MASK && masked ? g.kept + (c0 < wide ? c0 >> 6 : 0) * p.b * 8 + (i16 >> 1) : nullptr;
    const uint32_t last = (uint32_t)p.b - 1, pitch = 2 * (uint32_t)job.ld;       // bytes

    v4f acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[t][v] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // the sums, with the mask or without; chosen once
    const auto sum = [&](auto with_mask) {
        constexpr bool M = decltype(with_mask)::value;
        struct Step {
            int token[8];
            uint2 raw[8];
            uint32_t kept[8];
        };
        const int steps = (seg.end - seg.begin + 31) >> 5;
        const auto load_order = [&](int (&token)[8], int j) {
            const int4* o = reinterpret_cast<const int4*>(g.group.order + seg.begin + 32 * (j < steps ? j : 0) + 8 * kq);
            const int4 lo = o[0], hi = o[1];
            token[0] = lo.x; token[1] = lo.y; token[2] = lo.z; token[3] = lo.w;
            token[4] = hi.x; token[5] = hi.y; token[6] = hi.z; token[7] = hi.w;
        };
        // A place without a token (-1) loads the last one's row.  Only an adapter's last step has such places; there they are set to zero.
        const auto load_rows = [&](Step& q, const int (&token)[8]) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t t = (uint32_t)token[u] < last ? (uint32_t)token[u] : last;
                q.token[u] = token[u];
                q.raw[u] = *reinterpret_cast<const uint2*>(reinterpret_cast<const char*>(big) + (uint64_t)t * pitch);
                if (M) q.kept[u] = kept_at[t * 8];
            }
        };
        // thread (rank tile, lane) stages what that lane multiplies with
        const int unit = tid % UNITS, small_c = (tile0 + (unit >> 6)) * 16 + (unit & 15);
        const uint32_t small_at = 4 * (small_c < R ? small_c : 0);
        float staged[8];
        const auto load_staged = [&](const int (&token)[8]) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t t = (uint32_t)token[u] < last ? (uint32_t)token[u] : last;
                staged[u] = load_at<float>(job.small, __umul24(t, 4 * R) + small_at);        // at most 2^31 bytes
            }
        };
        const auto write_staged = [&](const int (&token)[8], int j) {
            if (j == steps - 1) {
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (token[u] < 0) staged[u] = 0.0f;
            }
            v4u q[3];
            split_eight(staged, q);
            if (UNITS % THREADS == 0 || tid < UNITS) {
#pragma unroll
                for (int k = 0; k < 3; ++k) s_small[j & 1][(unit >> 6) * 3 + k][lane] = q[k];
            }
        };
        const auto multiply = [&](const Step& q, int j) {
            uint2 x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = q.raw[u];
            if (M) {
                const int low = 4 * (i16 & 1);
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const uint32_t kept = q.kept[u] >> low;
                    x[u].x &= pack_lo(bit_mask(kept, 0), bit_mask(kept, 1));
                    x[u].y &= pack_lo(bit_mask(kept, 2), bit_mask(kept, 3));
                }
            }
            if (j == steps - 1) {
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (q.token[u] < 0) x[u] = make_uint2(0, 0);
            }
            v4u a[4];
            columns_of(x, a);
            v4u b[2][3];                                     // one rank tile's operands while the other's are multiplied
#pragma unroll
            for (int k = 0; k < 3; ++k) b[0][k] = s_small[j & 1][k][lane];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (t + 1 < NT) {
#pragma unroll
                    for (int k = 0; k < 3; ++k) b[(t + 1) & 1][k] = s_small[j & 1][(t + 1) * 3 + k][lane];
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
        int even_next[8], odd_next[8];                       // tokens of the steps whose rows are asked for next
        // Step j: its part of `small`, on its way since the step before, goes to LDS, that of the next is asked for, and the rows of the step after
        // the next as soon as this one's are used, by tokens that were asked for a step ago, ahead of that step's rows.
        const auto step = [&](Step& q, const int (&q_next)[8], const Step& other, int (&other_next)[8], int j) {
            write_staged(q.token, j);
            __syncthreads();
            load_staged(other.token);
            multiply(q, j);
            load_order(other_next, j + 3);
            in_order();
            load_rows(q, q_next);
            in_order();
        };
        if (steps > 0) {                                     // the same for the workgroup
            load_order(even_next, 0);
            load_order(odd_next, 1);
            load_rows(even, even_next);
            in_order();
            load_staged(even.token);
            load_order(even_next, 2);
            in_order();
            load_rows(odd, odd_next);
            in_order();
#pragma unroll 1
            for (int j = 0; j + 1 < steps; j += 2) {
                step(even, even_next, odd, odd_next, j);
                step(odd, odd_next, even, even_next, j + 1);
            }
            if (steps & 1) {
                write_staged(even.token, steps - 1);
                __syncthreads();
                multiply(even, steps - 1);
            }
        }
    };
    if (MASK && second) sum(std::bool_constant<MASK>());
    else sum(std::false_type());
    const int rank = rank_of(p, seg.adapter);
    const float factor = second ? (masked ? g.factor : 1.0f) : scale_of(p, seg.adapter);
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

constexpr int64_t kFill = 512;                           // workgroups that the chip holds at once

template <int NT>
void launch_as(const GradArgs& g, hipStream_t s) {
    const int rank_tiles = (int)ceil_div(g.p.max_rank, 16);
    const dim3 grid(g.job[0].tiles + g.job[1].tiles, g.p.slots + g.group.cuts, (unsigned)ceil_div(rank_tiles, NT)), block(64 * kGradWaves);
    if (g.kept) hipLaunchKernelGGL((grad_kernel<NT, true>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((grad_kernel<NT, false>), grid, block, 0, s, g);
}

}  // namespace

// Segments there are as many as adapters with tokens plus cuts, less one; together with the column tiles they should fill the chip once: every
// further one costs a partial sum that is written and read again.  How many adapters have tokens is not known here: as if all had, but cut
// at least half as often as one adapter alone would be.  A segment is at least 256 places and long next to its partial sum.
int grad_chunk(int64_t places, int64_t m, int64_t n, int slots, int max_rank) {
    const int64_t tiles = ceil_div(m, kGradCols) + ceil_div(n, kGradCols), wanted = kFill > tiles ? kFill / tiles : 1;
    int64_t cuts = wanted - slots + 1;
    if (cuts < (wanted + 1) / 2) cuts = (wanted + 1) / 2;
    int64_t chunk = ceil_div(places, cuts), least = 8 * max_rank < 256 ? 256 : 8 * max_rank;
    if (chunk < least) chunk = least;
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
