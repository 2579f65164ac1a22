// Group norm with an activation on channels-last tensors (include/scan2d_seq.h).
#include "scan2d_seq.hpp"

#include "scan2d_block.hpp"
#include "scan2d_common.hpp"

namespace scan2d {
namespace {

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const bf16_t* p) { return __uint_as_float((uint32_t)p->bits << 16); }

__device__ __forceinline__ float act_of(float v, int act) {
    if (act == SCAN2D_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v * kLog2e));
    if (act == SCAN2D_ACT_GELU) return 0.5f * v * (1.0f + erff(v * 0.70710678f));
    return v;
}
__device__ __forceinline__ float act_slope(float v, int act) {
    if (act == SCAN2D_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v * kLog2e));
        return s * (1.0f + v * (1.0f - s));
    }
    if (act == SCAN2D_ACT_GELU) return 0.5f * (1.0f + erff(v * 0.70710678f)) + v * 0.39894228f * __builtin_amdgcn_exp2f(-0.5f * kLog2e * v * v);
    return 1.0f;
}

__device__ __forceinline__ float block_sum(float v, float* red) {
    const int tid = threadIdx.x;
    __syncthreads();
    red[tid] = v;
    __syncthreads();
    for (int d = 128; d > 0; d >>= 1) {
        if (tid < d) red[tid] += red[tid + d];
        __syncthreads();
    }
    return red[0];
}

// One workgroup per item and group, three passes over its values.
template <typename T>
__global__ __launch_bounds__(256) void group_norm_fwd_kernel(const GroupNormArgs p) {
    __shared__ float red[256];
    const int n = blockIdx.x / p.G, g = blockIdx.x % p.G;
    const long long E = (long long)p.P * p.D;
    auto each = [&](auto f) {
        for (long long e = threadIdx.x; e < E; e += 256) {
            const long long row = (long long)n * p.P + e / p.D;
            const int c = g * p.D + (int)(e % p.D);
            f(row, c, p.mask != nullptr && p.mask[row] != 0);
        }
    };
    const T* x = static_cast<const T*>(p.x);
    float cnt = 0.0f, sum = 0.0f, sq = 0.0f;
    each([&](long long row, int c, bool out) { if (!out) { cnt += 1.0f; sum += load1(x + row * p.sx + c); } });
    cnt = block_sum(cnt, red);
    const float mean = cnt > 0.0f ? block_sum(sum, red) / cnt : 0.0f;
    each([&](long long row, int c, bool out) { if (!out) { const float d = load1(x + row * p.sx + c) - mean; sq = fmaf(d, d, sq); } });
    const float rstd = cnt > 0.0f ? 1.0f / sqrtf(block_sum(sq, red) / cnt + p.eps) : 0.0f;
    if (threadIdx.x == 0) { p.stats[2 * (size_t)blockIdx.x] = mean; p.stats[2 * (size_t)blockIdx.x + 1] = rstd; }
    each([&](long long row, int c, bool out) {
        const float xv = load1(x + row * p.sx + c);
        const float v = (xv - mean) * rstd * (p.gamma ? p.gamma[c] : 1.0f) + (p.beta ? p.beta[c] : 0.0f);
        store_elem(static_cast<T*>(p.y) + row * p.sy + c, out ? 0.0f : act_of(v, p.act));
    });
}

template <typename T>
__global__ __launch_bounds__(256) void group_norm_bwd_kernel(const GroupNormArgs p) {
    __shared__ float red[256];
    const int n = blockIdx.x / p.G, g = blockIdx.x % p.G;
    const float mean = p.stats[2 * (size_t)blockIdx.x], rstd = p.stats[2 * (size_t)blockIdx.x + 1];
    const T *x = static_cast<const T*>(p.x), *dy = static_cast<const T*>(p.dy);
    float cnt = 0.0f, s1 = 0.0f, s2 = 0.0f;
    float* part = static_cast<float*>(p.workspace);
    for (int c = g * p.D; c < (g + 1) * p.D; ++c) {
        const float gm = p.gamma ? p.gamma[c] : 1.0f, bt = p.beta ? p.beta[c] : 0.0f;
        float db = 0.0f, dg = 0.0f;
        cnt = 0.0f;
        for (int q = threadIdx.x; q < p.P; q += 256) {
            const long long row = (long long)n * p.P + q;
            if (p.mask != nullptr && p.mask[row] != 0) continue;
            const float xh = (load1(x + row * p.sx + c) - mean) * rstd, dv = load1(dy + row * p.sdy + c) * act_slope(fmaf(xh, gm, bt), p.act);
            db += dv; dg = fmaf(dv, xh, dg);
            cnt += 1.0f;
        }
        db = block_sum(db, red);
        dg = block_sum(dg, red);
        s1 = fmaf(db, gm, s1); s2 = fmaf(dg, gm, s2);
        if (threadIdx.x == 0) {
            part[((size_t)n * p.C + c) * 2] = db;
            part[((size_t)n * p.C + c) * 2 + 1] = dg;
        }
    }
    cnt = block_sum(cnt, red) * p.D;
    const float inv = cnt > 0.0f ? 1.0f / cnt : 0.0f;
    for (int c = g * p.D; c < (g + 1) * p.D; ++c) {
        const float gm = p.gamma ? p.gamma[c] : 1.0f, bt = p.beta ? p.beta[c] : 0.0f;
        for (int q = threadIdx.x; q < p.P; q += 256) {
            const long long row = (long long)n * p.P + q;
            const bool out = p.mask != nullptr && p.mask[row] != 0;
            const float xh = (load1(x + row * p.sx + c) - mean) * rstd, dv = load1(dy + row * p.sdy + c) * act_slope(fmaf(xh, gm, bt), p.act);
            store_elem(static_cast<T*>(p.dx) + row * p.sdx + c, out ? 0.0f : rstd * (dv * gm - (s1 + xh * s2) * inv));
        }
    }
}

__global__ __launch_bounds__(64) void group_norm_params_kernel(const float* part, int N, int C, float* dgamma, float* dbeta) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (c >= C) return;
    float db = 0.0f, dg = 0.0f;
    for (int n = 0; n < N; ++n) { db += part[((size_t)n * C + c) * 2]; dg += part[((size_t)n * C + c) * 2 + 1]; }
    if (dbeta) dbeta[c] = db;
    if (dgamma) dgamma[c] = dg;
}

int launched() { return hipGetLastError() == hipSuccess ? SCAN2D_OK : SCAN2D_ERR_LAUNCH_FAILED; }

}  // namespace

size_t group_norm_workspace_bytes(const scan2d_group_norm_desc* d, int pass) { return pass == SCAN2D_PASS_BWD ? (size_t)d->N * d->C * 8 : 0; }

int group_norm_fwd_launch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, hipStream_t stream) {
    const long long blocks = (long long)a.N * a.G;
    if (!launch_fits(blocks, 256)) return SCAN2D_ERR_BAD_SHAPE;
    (void)hipGetLastError();
    if (d->dtype == SCAN2D_BF16) hipLaunchKernelGGL(group_norm_fwd_kernel<bf16_t>, dim3((unsigned)blocks), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(group_norm_fwd_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, stream, a);
    return launched();
}

int group_norm_bwd_launch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, hipStream_t stream) {
    const long long blocks = (long long)a.N * a.G;
    if (!launch_fits(blocks, 256)) return SCAN2D_ERR_BAD_SHAPE;
    (void)hipGetLastError();
    if (d->dtype == SCAN2D_BF16) hipLaunchKernelGGL(group_norm_bwd_kernel<bf16_t>, dim3((unsigned)blocks), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(group_norm_bwd_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, stream, a);
    hipLaunchKernelGGL(group_norm_params_kernel, dim3((a.C + 63) / 64), dim3(64), 0, stream, static_cast<const float*>(a.workspace), a.N, a.C, a.dgamma, a.dbeta);
    return launched();
}

}  // namespace scan2d
