// C ABI of the sequence layers: argument checks.  The operators and every argument are specified in
// include/scan2d_seq.h.
#include <cmath>
#include <cstdint>

#include "scan2d_seq.hpp"

using namespace scan2d;

namespace {

bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
size_t elem_bytes(int dtype) { return dtype == SCAN2D_BF16 ? 2 : 4; }

// Below 2^26 elements: the kernels address neighbouring rows by 32-bit byte offsets.
bool stride_ok(int64_t stride, int64_t C) { return stride == 0 || (stride >= C && stride < (1LL << 26)); }

int check_recur(const scan2d_recur_desc* d, bool any_layout) {
    if (d == nullptr) return SCAN2D_ERR_NULL_POINTER;
    if (d->T < 0 || d->T >= (1LL << 31) - 4096 || d->C < 1 || d->C >= (1 << 24)) return SCAN2D_ERR_BAD_SHAPE;
    if (any_layout && (d->S < 1 || d->S >= (1 << 24))) return SCAN2D_ERR_BAD_SHAPE;
    if (d->dtype != SCAN2D_F32 && d->dtype != SCAN2D_BF16) return SCAN2D_ERR_BAD_DTYPE;
    if (!(d->scale > 0.0f) || !std::isfinite(d->scale)) return SCAN2D_ERR_BAD_SHAPE;
    const int64_t strides[] = {d->stride_x, d->stride_r, d->stride_i, d->stride_h, d->stride_dh, d->stride_dx, d->stride_dr, d->stride_di};
    for (int64_t s : strides)
        if (!stride_ok(s, d->C)) return SCAN2D_ERR_BAD_SHAPE;
    return SCAN2D_OK;
}

int check_layout(const scan2d_recur_desc* d, const int32_t* offsets, const int32_t* lengths) {
    if (offsets != nullptr && lengths != nullptr) return SCAN2D_ERR_BAD_FLAGS;
    if (offsets == nullptr && d->T % d->S != 0) return SCAN2D_ERR_BAD_SHAPE;
    return SCAN2D_OK;
}

RecurArgs recur_args(const scan2d_recur_desc* d) {
    RecurArgs a = {};
    auto of = [&](int64_t s) { return s == 0 ? (long long)d->C : (long long)s; };
    a.sx = of(d->stride_x); a.sr = of(d->stride_r); a.si = of(d->stride_i); a.sh = of(d->stride_h);
    a.sdh = of(d->stride_dh); a.sdx = of(d->stride_dx); a.sdr = of(d->stride_dr); a.sdi = of(d->stride_di);
    a.T = (int)d->T; a.C = d->C; a.S = d->S; a.scale = d->scale;
    a.per = d->S >= 1 ? (int)(d->T / d->S) : 0;
    return a;
}

int check_norm(const scan2d_group_norm_desc* d) {
    if (d == nullptr) return SCAN2D_ERR_NULL_POINTER;
    if (d->N < 1 || d->P < 1 || d->C < 1 || d->G < 1 || d->C >= (1 << 24) || d->C % d->G != 0) return SCAN2D_ERR_BAD_SHAPE;
    if (d->P >= (1LL << 31) || d->P * d->N >= (1LL << 31) - 4096) return SCAN2D_ERR_BAD_SHAPE;
    if (d->dtype != SCAN2D_F32 && d->dtype != SCAN2D_BF16) return SCAN2D_ERR_BAD_DTYPE;
    if (d->act != SCAN2D_ACT_NONE && d->act != SCAN2D_ACT_SILU && d->act != SCAN2D_ACT_GELU) return SCAN2D_ERR_BAD_FLAGS;
    if (!(d->eps >= 0.0f)) return SCAN2D_ERR_BAD_SHAPE;
    const int64_t strides[] = {d->stride_x, d->stride_y, d->stride_dy, d->stride_dx};
    for (int64_t s : strides)
        if (!stride_ok(s, d->C)) return SCAN2D_ERR_BAD_SHAPE;
    return SCAN2D_OK;
}

GroupNormArgs norm_args(const scan2d_group_norm_desc* d) {
    GroupNormArgs a = {};
    auto of = [&](int64_t s) { return s == 0 ? (long long)d->C : (long long)s; };
    a.sx = of(d->stride_x); a.sy = of(d->stride_y); a.sdy = of(d->stride_dy); a.sdx = of(d->stride_dx);
    a.N = d->N; a.P = (int)d->P; a.C = d->C; a.G = d->G; a.D = d->C / d->G; a.act = d->act; a.eps = d->eps;
    return a;
}

}  // namespace

extern "C" size_t scan2d_seq_recur_saved_bytes(const scan2d_recur_desc* desc) {
    return check_recur(desc, true) == SCAN2D_OK ? recur_saved_bytes(desc) : 0;
}

extern "C" size_t scan2d_seq_recur_workspace_bytes(const scan2d_recur_desc* desc, int pass) {
    if (check_recur(desc, true) != SCAN2D_OK || (pass != SCAN2D_PASS_FWD && pass != SCAN2D_PASS_BWD)) return 0;
    return recur_workspace_bytes(desc, pass);
}

extern "C" int scan2d_seq_recur_fwd(const scan2d_recur_desc* desc, const void* x, const void* r, const void* i, const float* lam,
                                    const int32_t* offsets, const int32_t* lengths, const float* h0, void* h, float* hT, void* saved,
                                    size_t saved_bytes, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_recur(desc, true);
    if (rc == SCAN2D_OK) rc = check_layout(desc, offsets, lengths);
    if (rc != SCAN2D_OK) return rc;
    if (!lam || (desc->T > 0 && (!x || !r || !i || !h))) return SCAN2D_ERR_NULL_POINTER;
    const size_t e = elem_bytes(desc->dtype);
    if (!aligned(x, e) || !aligned(r, e) || !aligned(i, e) || !aligned(h, e) || !aligned(lam, 4) || !aligned(offsets, 4) || !aligned(lengths, 4) ||
        !aligned(h0, 4) || !aligned(hT, 4) || !aligned(saved, 16) || !aligned(workspace, 16))
        return SCAN2D_ERR_MISALIGNED;
    if ((desc->T > 0 && (h == x || h == r || h == i)) || (hT != nullptr && hT == h0)) return SCAN2D_ERR_BAD_SHAPE;
    if (saved != nullptr && saved_bytes < recur_saved_bytes(desc)) return SCAN2D_ERR_WORKSPACE_SMALL;
    const size_t need = recur_workspace_bytes(desc, SCAN2D_PASS_FWD);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return SCAN2D_ERR_WORKSPACE_SMALL;
    rc = check_device();
    if (rc != SCAN2D_OK) return rc;
    RecurArgs a = recur_args(desc);
    a.x = x; a.r = r; a.i = i; a.lam = lam; a.offsets = offsets; a.lengths = lengths; a.h0 = h0; a.h = h; a.hT = hT;
    a.saved = static_cast<float*>(saved); a.workspace = workspace;
    return recur_fwd_launch(desc, a, static_cast<hipStream_t>(stream));
}

extern "C" int scan2d_seq_recur_bwd(const scan2d_recur_desc* desc, const void* x, const void* r, const void* i, const float* lam,
                                    const int32_t* offsets, const int32_t* lengths, const float* h0, const void* dh, const float* dhT,
                                    const void* saved, size_t saved_bytes, void* dx, void* dr, void* di, float* dlam, float* dh0,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_recur(desc, true);
    if (rc == SCAN2D_OK) rc = check_layout(desc, offsets, lengths);
    if (rc != SCAN2D_OK) return rc;
    const bool rows = desc->T > 0;
    const size_t saved_need = recur_saved_bytes(desc);
    if (!lam || !dlam || (rows && (!x || !r || !i || !dh || !dx || !dr || !di)) || (saved_need > 0 && !saved)) return SCAN2D_ERR_NULL_POINTER;
    const size_t e = elem_bytes(desc->dtype);
    const void* const elems[] = {x, r, i, dh, dx, dr, di};
    for (const void* p : elems)
        if (!aligned(p, e)) return SCAN2D_ERR_MISALIGNED;
    const void* const words[] = {lam, offsets, lengths, h0, dhT, dlam, dh0};
    for (const void* p : words)
        if (!aligned(p, 4)) return SCAN2D_ERR_MISALIGNED;
    if (!aligned(saved, 16) || !aligned(workspace, 16)) return SCAN2D_ERR_MISALIGNED;
    if (rows) {
        const void* const in[] = {x, r, i, dh};
        const void* const out[] = {dx, dr, di};
        for (int o = 0; o < 3; ++o) {
            for (const void* p : in)
                if (p == out[o]) return SCAN2D_ERR_BAD_SHAPE;
            for (int q = 0; q < o; ++q)
                if (out[q] == out[o]) return SCAN2D_ERR_BAD_SHAPE;
        }
    }
    if (dh0 != nullptr && dh0 == dhT) return SCAN2D_ERR_BAD_SHAPE;
    if (saved_bytes < saved_need) return SCAN2D_ERR_WORKSPACE_SMALL;
    const size_t need = recur_workspace_bytes(desc, SCAN2D_PASS_BWD);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return SCAN2D_ERR_WORKSPACE_SMALL;
    rc = check_device();
    if (rc != SCAN2D_OK) return rc;
    RecurArgs a = recur_args(desc);
    a.x = x; a.r = r; a.i = i; a.lam = lam; a.offsets = offsets; a.lengths = lengths; a.h0 = h0; a.dh = dh; a.dhT = dhT;
    a.saved = static_cast<float*>(const_cast<void*>(saved)); a.dx = dx; a.dr = dr; a.di = di; a.dlam = dlam; a.dh0 = dh0; a.workspace = workspace;
    return recur_bwd_launch(desc, a, static_cast<hipStream_t>(stream));
}

extern "C" int scan2d_seq_recur_step(const scan2d_recur_desc* desc, const void* x, const void* r, const void* i, const float* lam, float* state,
                                     const int32_t* slots, int64_t slot_count, void* h, void* stream) {
    int rc = check_recur(desc, false);
    if (rc != SCAN2D_OK) return rc;
    if (desc->T < 1 || desc->T > 65535 || !recur_step_fits(desc) || slot_count < 1 || slot_count >= (1LL << 31) || (slots == nullptr && slot_count < desc->T)) return SCAN2D_ERR_BAD_SHAPE;
    if (!x || !r || !i || !lam || !state || !h) return SCAN2D_ERR_NULL_POINTER;
    const size_t e = elem_bytes(desc->dtype);
    if (!aligned(x, e) || !aligned(r, e) || !aligned(i, e) || !aligned(h, e) || !aligned(lam, 4) || !aligned(state, 4) || !aligned(slots, 4))
        return SCAN2D_ERR_MISALIGNED;
    if (h == x || h == r || h == i) return SCAN2D_ERR_BAD_SHAPE;
    rc = check_device();
    if (rc != SCAN2D_OK) return rc;
    RecurArgs a = recur_args(desc);
    a.x = x; a.r = r; a.i = i; a.lam = lam; a.h = h;
    return recur_step_launch(desc, a, state, slots, slot_count, static_cast<hipStream_t>(stream));
}

extern "C" size_t scan2d_group_norm_workspace_bytes(const scan2d_group_norm_desc* desc, int pass) {
    if (check_norm(desc) != SCAN2D_OK || (pass != SCAN2D_PASS_FWD && pass != SCAN2D_PASS_BWD)) return 0;
    return group_norm_workspace_bytes(desc, pass);
}

extern "C" int scan2d_group_norm_fwd(const scan2d_group_norm_desc* desc, const void* x, const float* gamma, const float* beta, const uint8_t* mask,
                                     void* y, float* stats, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_norm(desc);
    if (rc != SCAN2D_OK) return rc;
    if (!x || !y || !stats) return SCAN2D_ERR_NULL_POINTER;
    const size_t e = elem_bytes(desc->dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(stats, 4) || !aligned(workspace, 16))
        return SCAN2D_ERR_MISALIGNED;
    GroupNormArgs a = norm_args(desc);
    if (x == y && a.sx != a.sy) return SCAN2D_ERR_BAD_SHAPE;
    const size_t need = group_norm_workspace_bytes(desc, SCAN2D_PASS_FWD);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return SCAN2D_ERR_WORKSPACE_SMALL;
    rc = check_device();
    if (rc != SCAN2D_OK) return rc;
    a.x = x; a.gamma = gamma; a.beta = beta; a.mask = mask; a.y = y; a.stats = stats; a.workspace = workspace;
    return group_norm_fwd_launch(desc, a, static_cast<hipStream_t>(stream));
}

extern "C" int scan2d_group_norm_bwd(const scan2d_group_norm_desc* desc, const void* x, const float* gamma, const float* beta, const uint8_t* mask,
                                     const float* stats, const void* dy, void* dx, float* dgamma, float* dbeta, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    int rc = check_norm(desc);
    if (rc != SCAN2D_OK) return rc;
    if (!x || !stats || !dy || !dx) return SCAN2D_ERR_NULL_POINTER;
    const size_t e = elem_bytes(desc->dtype);
    if (!aligned(x, e) || !aligned(dy, e) || !aligned(dx, e) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(stats, 4) || !aligned(dgamma, 4) ||
        !aligned(dbeta, 4) || !aligned(workspace, 16))
        return SCAN2D_ERR_MISALIGNED;
    GroupNormArgs a = norm_args(desc);
    if (dx == x || (dx == dy && a.sdx != a.sdy)) return SCAN2D_ERR_BAD_SHAPE;
    const size_t need = group_norm_workspace_bytes(desc, SCAN2D_PASS_BWD);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return SCAN2D_ERR_WORKSPACE_SMALL;
    rc = check_device();
    if (rc != SCAN2D_OK) return rc;
    a.x = x; a.gamma = gamma; a.beta = beta; a.mask = mask; a.stats = const_cast<float*>(stats); a.dy = dy; a.dx = dx; a.dgamma = dgamma;
    a.dbeta = dbeta; a.workspace = workspace;
    return group_norm_bwd_launch(desc, a, static_cast<hipStream_t>(stream));
}
