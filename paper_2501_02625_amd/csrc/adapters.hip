// One pass of the low-rank adapters: how the kernels of adapters_thin.hip, adapters_wide.hip and adapters_grad.hip follow one another, and what
// they keep in the workspace.  Forward: T, then Y.  Backward: S beside the tokens by their adapters and the mask's bits, then E_X, then the
// sums over the tokens, then, where an adapter's tokens were cut, the sums of those.
#include "adapters_device.h"

namespace halo {
using namespace adapters;

namespace {

size_t round256(size_t v) { return (v + 255) & ~size_t(255); }

struct BwdLayout {
    size_t part, thin, order, range, segments, kept, part_v, part_u, total;
    int chunk, cuts;
    ThinPlan plan;
};

BwdLayout bwd_layout(int64_t b, int64_t m, int64_t n, int slots, int R, bool drop) {
    BwdLayout L;
    const int64_t places = (b + 31) / 32 * 32 + 32 * (int64_t)slots;
    L.plan = thin_plan(b, n, slots);
    L.chunk = grad_chunk(b, places, m, n, R);
    L.cuts = (int)ceil_div(places, L.chunk);
    size_t at = 0;
    const auto take = [&at](size_t bytes) { const size_t here = at; at += round256(bytes); return here; };
    L.part = take((size_t)L.plan.splits * b * R * 4);
    L.thin = L.plan.splits > 1 ? take((size_t)b * R * 4) : L.part;
    L.order = take((size_t)places * 4);
    L.range = take((size_t)slots * sizeof(int2));
    L.segments = take(((size_t)slots + L.cuts) * sizeof(Segment));
    L.kept = take(drop ? (size_t)kept_words(b, m) * 8 : 0);
    L.part_v = take((size_t)grad_parts(L.cuts) * n * R * 4);
    L.part_u = take((size_t)grad_parts(L.cuts) * m * R * 4);
    L.total = at;
    return L;
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
    const hipError_t e = launch_thin(p, false, a.X, a.ld_x, part, a.drop, q, BackwardExtras{}, s);
    if (e != hipSuccess) return e;
    return launch_wide(WideArgs{p, part, q.splits, q.splits > 1 ? a.T : nullptr, a.base, a.ld_base, a.Y, a.ld_y, nullptr, 1.0f}, false,
                       a.out_f32 != 0, s);
}

hipError_t launch_adapters_bwd(const AdaptersBwd& a, hipStream_t s) {
    const AdapterPool& p = a.pool;
    const int64_t b = p.b;
    const bool drop = a.drop.least != 0;
    BwdLayout L = bwd_layout(b, p.m, p.n, p.slots, p.max_rank, drop);
    if (!a.EX) L.plan.splits = 1;                        // the kernel of E_X is what adds the parts up
    unsigned char* ws = reinterpret_cast<unsigned char*>(a.workspace);
    float* part = reinterpret_cast<float*>(ws + L.part);
    float* S = L.plan.splits > 1 ? reinterpret_cast<float*>(ws + L.thin) : part;
    const GroupArgs group{L.chunk, L.cuts, reinterpret_cast<int*>(ws + L.order), reinterpret_cast<int2*>(ws + L.range),
                          reinterpret_cast<Segment*>(ws + L.segments)};
    const bool grads = a.GU || a.GV;
    uint8_t* kept = drop && b > 0 && (a.EX || a.GU) ? ws + L.kept : nullptr;
    const BackwardExtras extras{group, grads ? p.slots : 0, kept, a.drop};
    hipError_t e = b > 0 && (a.EX || a.GU) ? launch_thin(p, true, a.E, a.ld_e, part, DropoutMask{}, L.plan, extras, s) : launch_extras(p, extras, s);
    if (e != hipSuccess) return e;
    if (b > 0 && a.EX) {
        e = launch_wide(WideArgs{p, part, L.plan.splits, L.plan.splits > 1 ? S : nullptr, a.base, a.ld_base, a.EX, a.ld_ex, kept,
                                 drop ? a.drop.factor : 1.0f}, true, a.out_f32 != 0, s);
        if (e != hipSuccess) return e;
    }
    if (!grads) return hipSuccess;
    GradArgs g{};
    g.p = p; g.group = group; g.kept = a.GU ? kept : nullptr; g.factor = a.drop.factor;
    if (a.GV) g.job[0] = GradJob{a.E, a.ld_e, a.T, a.GV, reinterpret_cast<float*>(ws + L.part_v), p.n, (int)ceil_div(p.n, kGradCols), 0};
    if (a.GU) g.job[1] = GradJob{a.X, a.ld_x, S, a.GU, reinterpret_cast<float*>(ws + L.part_u), p.m, (int)ceil_div(p.m, kGradCols), 1};
    return launch_grads(g, s);
}

}  // namespace halo
