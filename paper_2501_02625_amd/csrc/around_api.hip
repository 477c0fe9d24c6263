// C ABI of what stands around a layer's products (norm, epilogue, activation's gradient, AdamW): argument checking on the host, then
// kernel launches on the caller's stream.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <memory>
#include <new>

#include "around.h"
#include "halo_internal.h"

using namespace halo;

namespace {

inline bool aligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline halo_status from_hip(hipError_t e) { return e == hipSuccess ? HALO_OK : HALO_EHIP; }
inline bool bad_dtype(int32_t dt) { return dt != HALO_BF16 && dt != HALO_F32; }
constexpr int64_t kMaxDim = int64_t(1) << 22;   // rows / columns of a matrix argument

// A matrix argument of `cols` columns; null pointers are fine.
halo_status check_matrix(const void* p, int64_t ld, int64_t cols, int32_t dt) {
    if (!p) return HALO_OK;
    if (ld < cols) return HALO_ESHAPE;
    return aligned(p, 16) && ld % (dt == HALO_BF16 ? 8 : 4) == 0 ? HALO_OK : HALO_EALIGN;
}
// The same for one that may be `other` itself, with that one's leading dimension.
halo_status check_matrix(const void* p, int64_t ld, int64_t cols, int32_t dt, const void* other, int64_t ld_other) {
    const halo_status st = check_matrix(p, ld, cols, dt);
    return st == HALO_OK && p && p == other && ld != ld_other ? HALO_ESHAPE : st;
}
halo_status first_of(std::initializer_list<halo_status> all) {
    for (const halo_status st : all)
        if (st != HALO_OK) return st;
    return HALO_OK;
}

halo_status check_norm(const halo_norm_desc* d) {
    if (!d || d->rows < 0 || d->cols < 0 || d->reserved != 0) return HALO_EINVAL;
    if (d->kind != HALO_NORM_LAYER && d->kind != HALO_NORM_RMS) return HALO_EINVAL;
    if (bad_dtype(d->dt) || bad_dtype(d->weight_dt) || !(d->eps >= 0.0) || !std::isfinite((float)d->eps)) return HALO_EINVAL;
    if (d->cols > kMaxNormCols || d->rows > INT32_MAX) return HALO_EUNSUPPORTED;
    return HALO_OK;
}

struct Range {
    uintptr_t from, to;
    bool written;
};

}  // namespace

extern "C" {

// ------------------------------------------------------------------------------------------------
size_t halo_activation_bwd_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0 || rows > kMaxDim || cols > kMaxDim) return 0;
    return act_grad_workspace_floats(rows, cols) * 4;
}

halo_status halo_activation_bwd(const void* E, int64_t ld_e, const void* Z, int64_t ld_z, halo_dtype dt, int64_t rows, int64_t cols,
                                halo_activation act, void* EZ, int64_t ld_ez, float* GB, void* workspace, size_t workspace_bytes,
                                void* stream) {
    if (rows < 0 || cols < 0 || bad_dtype(dt)) return HALO_EINVAL;
    if (act < HALO_ACT_NONE || act > HALO_ACT_SILU) return HALO_EINVAL;
    if (cols == 0 || (rows == 0 && !GB)) return HALO_OK;         // also without pointers: what is empty has none
    if (!EZ && !GB) return HALO_EINVAL;
    if (rows > kMaxDim || cols > kMaxDim) return HALO_EUNSUPPORTED;
    if (act == HALO_ACT_NONE) Z = nullptr;
    if (rows > 0) {
        if (!E || (act != HALO_ACT_NONE && !Z)) return HALO_EINVAL;
        const halo_status st = first_of({check_matrix(E, ld_e, cols, dt), check_matrix(Z, ld_z, cols, dt),
                                         check_matrix(EZ, ld_ez, cols, dt, E, ld_e), check_matrix(EZ, ld_ez, cols, dt, Z, ld_z)});
        if (st != HALO_OK) return st;
    }
    if (!aligned(GB, 16)) return HALO_EALIGN;
    const size_t need = GB ? halo_activation_bwd_workspace_bytes(rows, cols) : 0;
    if (need && (!workspace || workspace_bytes < need)) return HALO_EWORKSPACE;
    if (need && !aligned(workspace, 16)) return HALO_EALIGN;
    const ActGrad a{E, ld_e, Z, ld_z, EZ, ld_ez, GB, reinterpret_cast<float*>(workspace), rows, cols, (int)act, dt == HALO_F32 ? 1 : 0};
    return from_hip(launch_act_grad(a, reinterpret_cast<hipStream_t>(stream)));
}

// ------------------------------------------------------------------------------------------------
size_t halo_layer_norm_bwd_workspace_bytes(const halo_norm_desc* desc) {
    if (check_norm(desc) != HALO_OK || desc->rows == 0 || desc->cols == 0) return 0;
    return norm_bwd_workspace_floats(desc->rows, desc->cols, desc->dt == HALO_F32 ? 1 : 0) * 4;
}

halo_status halo_layer_norm_fwd(const halo_norm_desc* desc, const void* X, int64_t ld_x, const void* weight, const void* bias, void* Y,
                                int64_t ld_y, float* mean, float* rstd, void* stream) {
    const halo_status bad = check_norm(desc);
    if (bad != HALO_OK) return bad;
    if (desc->rows == 0 || desc->cols == 0) return HALO_OK;
    if (!X || !Y) return HALO_EINVAL;
    const halo_status st = first_of({check_matrix(X, ld_x, desc->cols, desc->dt), check_matrix(Y, ld_y, desc->cols, desc->dt, X, ld_x)});
    if (st != HALO_OK) return st;
    if (!aligned(weight, 16) || !aligned(bias, 16) || !aligned(mean, 4) || !aligned(rstd, 4)) return HALO_EALIGN;
    const bool rms = desc->kind == HALO_NORM_RMS;
    const NormFwd a{X, ld_x, weight, bias, Y, ld_y, rms ? nullptr : mean, rstd, desc->rows, (int)desc->cols, rms ? 1 : 0,
                    desc->dt == HALO_F32 ? 1 : 0, desc->weight_dt == HALO_F32 ? 1 : 0, (float)desc->eps};
    return from_hip(launch_norm_fwd(a, reinterpret_cast<hipStream_t>(stream)));
}

halo_status halo_layer_norm_bwd(const halo_norm_desc* desc, const void* E, int64_t ld_e, const void* X, int64_t ld_x, const float* mean,
                                const float* rstd, const void* weight, const void* base, int64_t ld_base, void* EX, int64_t ld_ex,
                                float* GW, float* GB, void* workspace, size_t workspace_bytes, void* stream) {
    const halo_status bad = check_norm(desc);
    if (bad != HALO_OK) return bad;
    if (desc->cols == 0 || (desc->rows == 0 && !GW && !GB)) return HALO_OK;
    if (!EX && !GW && !GB) return HALO_EINVAL;
    const bool rms = desc->kind == HALO_NORM_RMS;
    if (rms) mean = nullptr;
    if (!EX) base = nullptr;
    if (desc->rows > 0) {
        if (!E || ((EX || GW) && (!X || !rstd || (!rms && !mean)))) return HALO_EINVAL;
        const int32_t dt = desc->dt;
        const halo_status st = first_of({check_matrix(E, ld_e, desc->cols, dt), check_matrix(EX || GW ? X : nullptr, ld_x, desc->cols, dt),
                                         check_matrix(base, ld_base, desc->cols, dt), check_matrix(EX, ld_ex, desc->cols, dt, E, ld_e),
                                         check_matrix(EX, ld_ex, desc->cols, dt, base, ld_base)});
        if (st != HALO_OK) return st;
    }
    if (!aligned(weight, 16) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(GW, 16) || !aligned(GB, 16)) return HALO_EALIGN;
    const size_t need = GW || GB ? halo_layer_norm_bwd_workspace_bytes(desc) : 0;
    if (need && (!workspace || workspace_bytes < need)) return HALO_EWORKSPACE;
    if (need && !aligned(workspace, 16)) return HALO_EALIGN;
    const NormBwd a{E, ld_e, X, ld_x, mean, rstd, weight, base, ld_base, EX, ld_ex, GW, GB, reinterpret_cast<float*>(workspace), desc->rows,
                    (int)desc->cols, rms ? 1 : 0, desc->dt == HALO_F32 ? 1 : 0, desc->weight_dt == HALO_F32 ? 1 : 0};
    return from_hip(launch_norm_bwd(a, reinterpret_cast<hipStream_t>(stream)));
}

// ------------------------------------------------------------------------------------------------
halo_status halo_adamw(const halo_adamw_desc* desc, const halo_adamw_tensor* tensors, int32_t count, void* stream) {
    if (!desc || count < 0 || (count > 0 && !tensors) || desc->reserved != 0) return HALO_EINVAL;
    const halo_adamw_desc& d = *desc;
    if (bad_dtype(d.param_dt) || bad_dtype(d.grad_dt) || (d.state_bits != 32 && d.state_bits != 8)) return HALO_EINVAL;
    if (!d.step_ptr && d.step < 1) return HALO_EINVAL;
    auto in_unit = [](double b) { return b >= 0.0 && b < 1.0 && (float)b < 1.0f; };
    auto not_negative = [](double x) { return x >= 0.0 && std::isfinite((float)x); };
    if (!in_unit(d.beta1) || !in_unit(d.beta2) || !not_negative(d.eps) || !not_negative(d.weight_decay)) return HALO_EINVAL;
    if (!d.lr_ptr && !not_negative(d.lr)) return HALO_EINVAL;
    if (!d.grad_scale_ptr && !std::isfinite((float)d.grad_scale)) return HALO_EINVAL;
    if (!aligned(d.step_ptr, 8) || !aligned(d.lr_ptr, 4) || !aligned(d.grad_scale_ptr, 4)) return HALO_EALIGN;
    constexpr int kMost = 1024;
    if (count > kMost) return HALO_EUNSUPPORTED;
    const bool eight = d.state_bits == 8;
    const size_t pe = d.param_dt == HALO_BF16 ? 2 : 4, se = eight ? 1 : 4;
    // on the heap: with 1024 tensors they are 246 KB, more than the whole stack of some threads
    const std::unique_ptr<AdamwTensor[]> list(new (std::nothrow) AdamwTensor[count]);
    const std::unique_ptr<Range[]> used(new (std::nothrow) Range[(size_t)count * 7 + 3]);
    if (!list || !used) return from_hip(hipErrorOutOfMemory);
    int n = 0, ranges = 0;
    bool masters = false, plain = false;
    auto add = [&](const void* p, size_t bytes, bool written = true) {
        if (p) used[ranges++] = Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written};
    };
    for (int32_t t = 0; t < count; ++t) {
        const halo_adamw_tensor& x = tensors[t];
        if (x.size < 0) return HALO_EINVAL;
        if (x.size == 0) continue;
        if (!x.param || !x.grad || !x.m || !x.v || (eight && (!x.m_scale || !x.v_scale))) return HALO_EINVAL;
        if (x.master && d.param_dt != HALO_BF16) return HALO_EINVAL;
        (x.master ? masters : plain) = true;
        if (x.size > (int64_t(1) << 34)) return HALO_EUNSUPPORTED;
        if (!aligned(x.param, 16) || !aligned(x.grad, 16) || !aligned(x.m, 16) || !aligned(x.v, 16) || !aligned(x.master, 16)) return HALO_EALIGN;
        if (eight && (!aligned(x.m_scale, 4) || !aligned(x.v_scale, 4))) return HALO_EALIGN;
        const size_t size = (size_t)x.size, blocks = (size + HALO_ADAMW_BLOCK - 1) / HALO_ADAMW_BLOCK;
        add(x.param, size * pe);
        add(x.grad, size * (d.grad_dt == HALO_BF16 ? 2 : 4), false);
        add(x.m, size * se);
        add(x.v, size * se);
        add(x.master, size * 4);
        if (eight) {
            add(x.m_scale, blocks * 4);
            add(x.v_scale, blocks * 4);
        }
        list[n++] = AdamwTensor{x.param, x.grad, x.m, x.v, x.master, x.m_scale, x.v_scale, x.size, t};
    }
    if (masters && plain) return HALO_EINVAL;
    // A tensor given twice would be updated by two workgroups at once, and every workgroup reads the step's numbers.  What is only read may be
    // shared.
    add(d.step_ptr, 8, false);
    add(d.lr_ptr, 4, false);
    add(d.grad_scale_ptr, 4, false);
    std::sort(used.get(), used.get() + ranges, [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t end = 0, written_end = 0;      // of what lies in front
    for (int i = 0; i < ranges; ++i) {
        if (used[i].from < (used[i].written ? end : written_end)) return HALO_EINVAL;
        end = std::max(end, used[i].to);
        if (used[i].written) written_end = std::max(written_end, used[i].to);
    }
    if (n == 0) return HALO_OK;
    AdamwStep s{};
    s.beta1 = (float)d.beta1; s.rest1 = (float)(1.0 - d.beta1); s.beta2 = (float)d.beta2; s.rest2 = (float)(1.0 - d.beta2);
    s.eps = (float)d.eps; s.grad_scale = (float)d.grad_scale;
    s.key0 = (uint32_t)d.seed; s.key1 = (uint32_t)(d.seed >> 32);
    s.step = d.step_ptr ? 1 : d.step;
    s.offset = d.offset + (d.step_ptr ? 0 : (uint64_t)d.step);
    s.lr = d.lr_ptr ? 0.0 : d.lr; s.log_beta1 = std::log2(d.beta1); s.log_beta2 = std::log2(d.beta2); s.weight_decay = d.weight_decay;
    s.step_ptr = d.step_ptr; s.lr_ptr = d.lr_ptr; s.grad_scale_ptr = d.grad_scale_ptr;
    adamw_numbers((double)s.step, s.lr, d.beta1, d.beta2, d.weight_decay, &s.decay, &s.rate, &s.root);
    const int param = d.param_dt == HALO_F32 ? 0 : masters ? 2 : 1;
    return from_hip(launch_adamw(s, list.get(), n, param, d.grad_dt == HALO_F32 ? 1 : 0, eight ? 1 : 0, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
