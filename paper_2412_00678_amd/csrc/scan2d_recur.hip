// The gated linear recurrence on channels-last rows (include/scan2d_seq.h).
#include "scan2d_seq.hpp"

#include "scan2d_block.hpp"
#include "scan2d_common.hpp"

namespace scan2d {
namespace {

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const bf16_t* p) { return __uint_as_float((uint32_t)p->bits << 16); }

__device__ __forceinline__ float sigmoid(float t) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-t * kLog2e)); }

// Per channel: scale * softplus(lam), and sigmoid(lam) / softplus(lam) (-> 1 for lam -> -inf).
__device__ __forceinline__ float decay_of(float lam, float scale) { return scale * (lam > 20.0f ? lam : log1pf(expf(lam))); }
__device__ __forceinline__ float decay_slope(float lam) { return lam < -15.0f ? 1.0f : 1.0f / ((1.0f + expf(-lam)) * (lam > 20.0f ? lam : log1pf(expf(lam)))); }

// 1 - e^z for z <= 0, without the cancellation near 0: the series of (e^z - 1) / z to degree 6 on [-0.5, 0] (the next term is
// below 2e-7); beyond, 1 - e^z >= 0.39.
__device__ __forceinline__ float one_minus_exp(float z, float ez) {
    const float p = 1.0f + z * (0.5f + z * (0.16666667f + z * (0.041666668f + z * (0.008333334f + z * (0.0013888889f + z * 0.0001984127f)))));
    return z > -0.5f ? -z * p : 1.0f - ez;
}

struct Rows { int lo, hi; };
__device__ __forceinline__ Rows rows_of(const RecurArgs& p, int s) {
    if (p.offsets) return {min(max(p.offsets[s], 0), p.T), min(max(p.offsets[s + 1], 0), p.T)};
    const int lo = s * p.per;
    return {lo, lo + (p.lengths ? min(max(p.lengths[s], 0), p.per) : p.per)};
}

template <typename T>
__global__ __launch_bounds__(64) void recur_fwd_kernel(const RecurArgs p) {
    const int c = (blockIdx.x % ((p.C + 63) / 64)) * 64 + threadIdx.x, s = blockIdx.x / ((p.C + 63) / 64);
    if (c >= p.C) return;
    const Rows w = rows_of(p, s);
    const float decay = decay_of(p.lam[c], p.scale);
    float h = p.h0 ? p.h0[(size_t)s * p.C + c] : 0.0f;
    for (int t = w.lo; t < w.hi; ++t) {
        const float x = load1(static_cast<const T*>(p.x) + t * p.sx + c), sr = sigmoid(load1(static_cast<const T*>(p.r) + t * p.sr + c)),
                    si = sigmoid(load1(static_cast<const T*>(p.i) + t * p.si + c));
        const float la = -decay * sr, a = __builtin_amdgcn_exp2f(la * kLog2e);
        if (p.saved) p.saved[(size_t)t * p.C + c] = h;
        h = fmaf(a, h, sqrtf(one_minus_exp(2.0f * la, a * a)) * si * x);
        store_elem(static_cast<T*>(p.h) + t * p.sh + c, h);
    }
    if (p.hT) p.hT[(size_t)s * p.C + c] = h;
}

template <typename T>
__global__ __launch_bounds__(64) void recur_bwd_kernel(const RecurArgs p) {
    const int c = (blockIdx.x % ((p.C + 63) / 64)) * 64 + threadIdx.x, s = blockIdx.x / ((p.C + 63) / 64);
    if (c >= p.C) return;
    const Rows w = rows_of(p, s);
    const float decay = decay_of(p.lam[c], p.scale);
    float e = p.dhT ? p.dhT[(size_t)s * p.C + c] : 0.0f, sum = 0.0f;      // e: gradient that reaches the state behind token t
    for (int t = w.hi - 1; t >= w.lo; --t) {
        const float x = load1(static_cast<const T*>(p.x) + t * p.sx + c), sr = sigmoid(load1(static_cast<const T*>(p.r) + t * p.sr + c)),
                    si = sigmoid(load1(static_cast<const T*>(p.i) + t * p.si + c));
        const float la = -decay * sr, a = __builtin_amdgcn_exp2f(la * kLog2e), b2 = one_minus_exp(2.0f * la, a * a);
        const float ib = b2 > 1.2e-38f ? 1.0f / sqrtf(b2) : 0.0f, b = b2 * ib;
        const float g = load1(static_cast<const T*>(p.dh) + t * p.sdh + c) + e, before = p.saved[(size_t)t * p.C + c];
        e = a * g;
        const float q = la * (e * before - a * a * ib * g * si * x);
        sum += q;
        store_elem(static_cast<T*>(p.dx) + t * p.sdx + c, b * si * g);
        store_elem(static_cast<T*>(p.di) + t * p.sdi + c, b * x * g * si * (1.0f - si));
        store_elem(static_cast<T*>(p.dr) + t * p.sdr + c, q * (1.0f - sr));
    }
    if (p.dh0) p.dh0[(size_t)s * p.C + c] = e;
    static_cast<float*>(p.workspace)[(size_t)s * p.C + c] = sum;
}

__global__ __launch_bounds__(64) void recur_dlam_kernel(const float* parts, int n, int C, const float* lam, float* dlam) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (c >= C) return;
    float sum = 0.0f;
    for (int k = 0; k < n; ++k) sum += parts[(size_t)k * C + c];
    dlam[c] = sum * decay_slope(lam[c]);
}

// One row and 256 channels per workgroup.  A slot that stands at several rows is done by the workgroup of the first of
// them, in the order of the rows.
template <typename T>
__global__ __launch_bounds__(256) void recur_step_kernel(const RecurArgs p, float* state, const int32_t* slots, long long slot_count) {
    const int cols = (p.C + 255) / 256, row = blockIdx.x / cols, c = (blockIdx.x % cols) * 256 + threadIdx.x;
    const int slot = slots ? slots[row] : row;
    if (slot < 0 || slot >= slot_count) return;
    if (slots) {
        int earlier = 0;
        for (int t = threadIdx.x; t < row; t += 256) earlier |= slots[t] == slot;
        if (__syncthreads_or(earlier)) return;
    }
    if (c >= p.C) return;
    const float decay = decay_of(p.lam[c], p.scale);
    float h = state[(size_t)slot * p.C + c];
    for (int t = row; t < (slots ? p.T : row + 1); ++t) {
        if (slots && slots[t] != slot) continue;
        const float x = load1(static_cast<const T*>(p.x) + t * p.sx + c), sr = sigmoid(load1(static_cast<const T*>(p.r) + t * p.sr + c)),
                    si = sigmoid(load1(static_cast<const T*>(p.i) + t * p.si + c));
        const float la = -decay * sr, a = __builtin_amdgcn_exp2f(la * kLog2e);
        h = fmaf(a, h, sqrtf(one_minus_exp(2.0f * la, a * a)) * si * x);
        store_elem(static_cast<T*>(p.h) + t * p.sh + c, h);
    }
    state[(size_t)slot * p.C + c] = h;
}

int launched() { return hipGetLastError() == hipSuccess ? SCAN2D_OK : SCAN2D_ERR_LAUNCH_FAILED; }

}  // namespace

size_t recur_saved_bytes(const scan2d_recur_desc* d) { return (size_t)d->T * d->C * 4; }
size_t recur_workspace_bytes(const scan2d_recur_desc* d, int pass) { return pass == SCAN2D_PASS_BWD ? (size_t)d->S * d->C * 4 : 0; }

int recur_fwd_launch(const scan2d_recur_desc* d, const RecurArgs& a, hipStream_t stream) {
    const long long blocks = (long long)((a.C + 63) / 64) * a.S;
    if (!launch_fits(blocks, 64)) return SCAN2D_ERR_BAD_SHAPE;
    (void)hipGetLastError();
    if (d->dtype == SCAN2D_BF16) hipLaunchKernelGGL(recur_fwd_kernel<bf16_t>, dim3((unsigned)blocks), dim3(64), 0, stream, a);
    else hipLaunchKernelGGL(recur_fwd_kernel<float>, dim3((unsigned)blocks), dim3(64), 0, stream, a);
    return launched();
}

int recur_bwd_launch(const scan2d_recur_desc* d, const RecurArgs& a, hipStream_t stream) {
    const long long blocks = (long long)((a.C + 63) / 64) * a.S;
    if (!launch_fits(blocks, 64)) return SCAN2D_ERR_BAD_SHAPE;
    (void)hipGetLastError();
    if (d->dtype == SCAN2D_BF16) hipLaunchKernelGGL(recur_bwd_kernel<bf16_t>, dim3((unsigned)blocks), dim3(64), 0, stream, a);
    else hipLaunchKernelGGL(recur_bwd_kernel<float>, dim3((unsigned)blocks), dim3(64), 0, stream, a);
    hipLaunchKernelGGL(recur_dlam_kernel, dim3((a.C + 63) / 64), dim3(64), 0, stream, static_cast<const float*>(a.workspace), a.S, a.C, a.lam, a.dlam);
    return launched();
}

int recur_step_launch(const scan2d_recur_desc* d, const RecurArgs& a, float* state, const int32_t* slots, long long slot_count, hipStream_t stream) {
    const long long blocks = (long long)((a.C + 255) / 256) * a.T;
    if (!launch_fits(blocks, 256)) return SCAN2D_ERR_BAD_SHAPE;
    (void)hipGetLastError();
    if (d->dtype == SCAN2D_BF16) hipLaunchKernelGGL(recur_step_kernel<bf16_t>, dim3((unsigned)blocks), dim3(256), 0, stream, a, state, slots, slot_count);
    else hipLaunchKernelGGL(recur_step_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, stream, a, state, slots, slot_count);
    return launched();
}

}  // namespace scan2d
