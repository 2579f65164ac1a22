// Group norm with an activation on channels-last tensors (include/scan2d_seq.h).
//
// Bound: HBM (forward 1 read and 1 write per element, backward 2 and 1) as long as the statistics are there; they need all
// of an item's group first.  Channels go along the lanes, V neighbours each, and what lanes are left over by narrow rows take further
// positions.  A workgroup or wavefront has a slab of whole groups (or a part of one group that is wider than it).
//
// Held form (group_norm_fwd_kernel, group_norm_bwd_kernel): a team of lanes holds all positions of an item's slab in
// registers as they were loaded: one read.  Teams are a power of two of lanes within a wavefront (nothing waits for another
// wavefront; a single token's groups, small maps), or a workgroup.  A team goes on to the next item of its slab with its
// channels' parameters, and in the backward pass its channels' sums, in registers.
// Split form, where an item's slab does not fit: one kernel takes the mean and the squared deviations from it of tiles held in registers,
// one joins the tiles of an item (M2 = sum M2_i + sum n_i (mean_i - mean)^2), one reads the tensor again and writes.
// The variance is always taken from deviations, never from the difference of two large sums.
// All sums run in a fixed order.
#include "scan2d_seq.hpp"

#include "scan2d_block.hpp"
#include "scan2d_common.hpp"

namespace scan2d {
namespace {

template <typename T, int V> struct Pack { uint32_t w[V * Elem<T>::kBytes <= 4 ? 1 : V * Elem<T>::kBytes / 4]; };
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
    Pack<T, V> r;
    if constexpr (V * Elem<T>::kBytes == 2) r.w[0] = p->bits;
    else load_words_any<V * Elem<T>::kBytes / 4>(p, r.w);
    return r;
}
template <typename T, int V>
__device__ __forceinline__ float get(const Pack<T, V>& r, int j) { return get_elem<T, V>(r.w, j); }
template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const float* v) {
    if constexpr (Elem<T>::kBytes == 4) store_words_any<V>(p, reinterpret_cast<const uint32_t*>(v));
    else if constexpr (V == 1) p->bits = (uint16_t)f32_to_bf16_bits(v[0]);
    else {
        uint32_t w[V / 2];
#pragma unroll
        for (int k = 0; k < V / 2; ++k) w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
        store_words_any<V / 2>(p, w);
    }
}

__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v * kLog2e)); }
template <int ACT>
__device__ __forceinline__ float act_of(float v) {
    if constexpr (ACT == SCAN2D_ACT_SILU) return v * sigmoid(v);
    else if constexpr (ACT == SCAN2D_ACT_GELU) return 0.5f * v * (1.0f + erff(v * 0.70710678f));
    else return v;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float v) {
    if constexpr (ACT == SCAN2D_ACT_SILU) {
        const float s = sigmoid(v);
        return s * fmaf(v, 1.0f - s, 1.0f);
    } else if constexpr (ACT == SCAN2D_ACT_GELU) {
        return fmaf(v * 0.39894228f, __builtin_amdgcn_exp2f(-0.5f * kLog2e * v * v), 0.5f * (1.0f + erff(v * 0.70710678f)));
    } else {
        return 1.0f;
    }
}

// How teams of lanes share the work.
struct Geo {
    int ts;                              // lanes of a team
    int width;                           // channels of a slab, at most
    int D;                               // channels of a group within a slab
    int gps;                             // groups of a slab, at most
    int slabs;                           // slabs of a row
    int spg;                             // slabs of a group (1 where a slab has whole groups)
    int lanes;                           // lanes of a row: width / V rounded up
    int slots;                           // rows a team takes at once: ts / lanes
    int tpg;                             // lanes that add up a group, a power of two
};

// A team's slab, and this lane's channels of it.
template <int V>
struct Lane {
    int lt;                              // within the team
    int slot, c;                         // which of the team's rows; first channel
    int lo, hi;                          // the slab's channels
    int groups, D;                       // the slab's groups, their channels (of the slab)
    int g0;                              // its first group
    bool on;                             // has a row at all
    bool own[V];                         // which channels are this lane's
    bool all;
    __device__ Lane(const Geo& q, int C, int G, int slab, int lane) {
        lt = lane;
        if (q.spg > 1) {
            g0 = slab / q.spg;
            const int Dg = C / G, part = slab % q.spg;
            lo = g0 * Dg + part * q.width;
            hi = min(lo + q.width, (g0 + 1) * Dg);
            groups = 1;
            D = hi - lo;
        } else {
            g0 = slab * q.gps;
            groups = min(q.gps, G - g0);
            D = q.D;
            lo = g0 * D;
            hi = lo + groups * D;
        }
        slot = lane / q.lanes;
        const int first = lo + (lane % q.lanes) * V;
        on = slot < q.slots && first < hi;
        c = min(first, C - V);
        all = true;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            own[v] = on && c + v >= first && c + v < hi;
            all = all && own[v];
        }
    }
    __device__ __forceinline__ int group_of(int v) const { return min(max((c + v - lo) / D, 0), groups - 1); }
};

template <bool WAVE>
__device__ __forceinline__ void team_sync() {
    if constexpr (WAVE) {                                  // a team lies within a wavefront, whose LDS accesses keep their order
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
        __syncthreads();
    }
}

// Sums of NR values over a team's rows and the channels of each group of its slab: done(group, sums) is called by one lane of each
// group.  The values of channels that are not the lane's are not looked at.  red: NR x (ts V) floats of the team.
template <int V, int NR, bool WAVE, typename Done>
__device__ __forceinline__ void group_sums(const Geo& q, const Lane<V>& l, float* red, const float (&val)[NR][V], Done done) {
    const int width = l.hi - l.lo, size = q.ts * V;
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (l.own[v]) red[r * size + l.slot * width + l.c + v - l.lo] = val[r][v];
    team_sync<WAVE>();
    const int qq = l.lt & (q.tpg - 1), n = q.slots * l.D, row0 = qq / l.D, d0 = qq % l.D, rowstep = q.tpg / l.D, dstep = q.tpg % l.D;
    for (int g = l.lt / q.tpg; g < l.groups; g += q.ts / q.tpg) {
        float s[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r] = 0.0f;
        for (int e = qq, row = row0, d = d0; e < n; e += q.tpg) {
#pragma unroll
            for (int r = 0; r < NR; ++r) s[r] += red[r * size + row * width + g * l.D + d];
            row += rowstep;
            d += dstep;
            if (d >= l.D) { d -= l.D; ++row; }
        }
        for (int m = 1; m < q.tpg; m <<= 1)
#pragma unroll
            for (int r = 0; r < NR; ++r) s[r] += __shfl_xor(s[r], m);
        if (qq == 0) done(g, s);
    }
    team_sync<WAVE>();
}

// The rows of a team's item that count.
template <bool WAVE>
__device__ __forceinline__ int count_rows(int* cnt, int lt, bool counts, int mine) {
    if (lt == 0) *cnt = 0;
    team_sync<WAVE>();
    if (counts && mine != 0) atomicAdd(cnt, mine);
    team_sync<WAVE>();
    return *cnt;
}

template <int V>
__device__ __forceinline__ void load_params(const GroupNormArgs& p, int c, float* gamma, float* beta) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        gamma[v] = p.gamma ? p.gamma[c + v] : 1.0f;
        beta[v] = p.beta ? p.beta[c + v] : 0.0f;
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_own(T* p, const Lane<V>& l, const float* v) {
    if (l.all) {
        store_pack<T, V>(p, v);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (l.own[k]) store_elem(p + k, v[k]);
    }
}

// ---- held form
template <typename T, int V, int K, int TH, bool WAVE, int ACT>
__global__ __launch_bounds__(TH) void group_norm_fwd_kernel(const GroupNormArgs p, const Geo q, int teams) {
    __shared__ float red[TH * V], res[2][TH * V];
    __shared__ int cnts[WAVE ? TH : 1];
    const int tid = threadIdx.x, lt = WAVE ? tid & (q.ts - 1) : tid, base = tid - lt;
    const int team = WAVE ? (int)((blockIdx.x * (long long)TH + tid) / q.ts) : (int)blockIdx.x;      // teams is a multiple of slabs
    const Lane<V> l(q, p.C, p.G, team % q.slabs, lt);
    float* const myred = red + base * V;
    float *const mean_of = res[0] + base * V, *const rstd_of = res[1] + base * V;
    float gamma[V], beta[V];
    load_params<V>(p, l.c, gamma, beta);
    int gr[V];
#pragma unroll
    for (int v = 0; v < V; ++v) gr[v] = l.group_of(v);
    const int step = teams / q.slabs, rounds = (p.N + step - 1) / step;
    for (int it = 0; it < rounds; ++it) {
        const long long n = team / q.slabs + (long long)it * step;
        const bool real = n < p.N && team < teams;      // the last workgroup may have lanes to spare
        const long long row0 = (real ? n : 0) * p.P;
        Pack<T, V> x[K];
        bool live[K];
        int mine = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int r = l.slot + k * q.slots;
            const long long row = row0 + min(r, p.P - 1);
            x[k] = load_pack<T, V>(static_cast<const T*>(p.x) + row * p.sx + l.c);
            live[k] = real && l.on && r < p.P && (p.mask == nullptr || p.mask[row] == 0);
            mine += live[k];
        }
        int rows = p.P;
        if (p.mask != nullptr) rows = count_rows<WAVE>(&cnts[base], lt, lt % q.lanes == 0, mine);
        const float M = (float)rows * (float)l.D, inv = rows > 0 ? 1.0f / M : 0.0f;
        float s[1][V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            s[0][v] = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) s[0][v] += live[k] ? get<T, V>(x[k], v) : 0.0f;
        }
        group_sums<V, 1, WAVE>(q, l, myred, s, [&](int g, const float* t) { mean_of[g] = t[0] * inv; });
        float mean[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            mean[v] = mean_of[gr[v]];
            s[0][v] = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const float d = live[k] ? get<T, V>(x[k], v) - mean[v] : 0.0f;
                s[0][v] = fmaf(d, d, s[0][v]);
            }
        }
        group_sums<V, 1, WAVE>(q, l, myred, s, [&](int g, const float* t) {
            const float rstd = rows > 0 ? 1.0f / sqrtf(t[0] * inv + p.eps) : 0.0f;
            rstd_of[g] = rstd;
            if (real) {
                float* st = p.stats + ((size_t)n * p.G + l.g0 + g) * 2;
                st[0] = mean_of[g];
                st[1] = rstd;
            }
        });
        float rstd[V];
#pragma unroll
        for (int v = 0; v < V; ++v) rstd[v] = rstd_of[gr[v]];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int r = l.slot + k * q.slots;
            if (real && l.on && r < p.P) {
                float y[V];
#pragma unroll
                for (int v = 0; v < V; ++v) y[v] = live[k] ? act_of<ACT>(fmaf((get<T, V>(x[k], v) - mean[v]) * rstd[v], gamma[v], beta[v])) : 0.0f;
                store_own<T, V>(static_cast<T*>(p.y) + (row0 + r) * p.sy + l.c, l, y);
            }
        }
    }
}

// parts: [..][C][2], the sums for dbeta and dgamma of the items that a team, or a workgroup of teams, had.
template <typename T, int V, int K, int TH, bool WAVE, int ACT>
__global__ __launch_bounds__(TH) void group_norm_bwd_kernel(const GroupNormArgs p, const Geo q, int teams, float2* parts) {
    __shared__ float red[2 * TH * V], res[2][TH * V];
    __shared__ int cnts[WAVE ? TH : 1];
    const int tid = threadIdx.x, lt = WAVE ? tid & (q.ts - 1) : tid, base = tid - lt;
    const int team = WAVE ? (int)((blockIdx.x * (long long)TH + tid) / q.ts) : (int)blockIdx.x;
    const Lane<V> l(q, p.C, p.G, team % q.slabs, lt);
    float* const myred = red + 2 * base * V;
    float *const s1_of = res[0] + base * V, *const s2_of = res[1] + base * V;
    float gamma[V], beta[V], accb[V], accg[V];
    load_params<V>(p, l.c, gamma, beta);
    int gr[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { gr[v] = l.group_of(v); accb[v] = accg[v] = 0.0f; }
    const int step = teams / q.slabs, rounds = (p.N + step - 1) / step;
    for (int it = 0; it < rounds; ++it) {
        const long long n = team / q.slabs + (long long)it * step;
        const bool real = n < p.N && team < teams;      // the last workgroup may have lanes to spare
        const long long row0 = (real ? n : 0) * p.P;
        Pack<T, V> x[K], dy[K];
        bool live[K];
        int mine = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int r = l.slot + k * q.slots;
            const long long row = row0 + min(r, p.P - 1);
            x[k] = load_pack<T, V>(static_cast<const T*>(p.x) + row * p.sx + l.c);
            dy[k] = load_pack<T, V>(static_cast<const T*>(p.dy) + row * p.sdy + l.c);
            live[k] = real && l.on && r < p.P && (p.mask == nullptr || p.mask[row] == 0);
            mine += live[k];
        }
        float mean[V], rstd[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float* st = p.stats + ((size_t)(real ? n : 0) * p.G + l.g0 + gr[v]) * 2;
            mean[v] = st[0];
            rstd[v] = st[1];
        }
        int rows = p.P;
        if (p.mask != nullptr) rows = count_rows<WAVE>(&cnts[base], lt, lt % q.lanes == 0, mine);
        const float inv = rows > 0 ? 1.0f / ((float)rows * (float)l.D) : 0.0f;
        float s[2][V], dv[K][V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float b = 0.0f, g = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const float xh = (get<T, V>(x[k], v) - mean[v]) * rstd[v];
                dv[k][v] = live[k] ? get<T, V>(dy[k], v) * act_slope<ACT>(fmaf(xh, gamma[v], beta[v])) : 0.0f;
                b += dv[k][v];
                g += live[k] ? dv[k][v] * xh : 0.0f;
            }
            accb[v] += b;
            accg[v] += g;
            s[0][v] = b * gamma[v];
            s[1][v] = g * gamma[v];
        }
        group_sums<V, 2, WAVE>(q, l, myred, s, [&](int g, const float* t) { s1_of[g] = t[0] * inv; s2_of[g] = t[1] * inv; });
        float s1[V], s2[V];
#pragma unroll
        for (int v = 0; v < V; ++v) { s1[v] = s1_of[gr[v]]; s2[v] = s2_of[gr[v]]; }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int r = l.slot + k * q.slots;
            if (real && l.on && r < p.P) {
                float dx[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float xh = (get<T, V>(x[k], v) - mean[v]) * rstd[v];
                    dx[v] = live[k] ? rstd[v] * (fmaf(dv[k][v], gamma[v], -s1[v]) - xh * s2[v]) : 0.0f;
                }
                store_own<T, V>(static_cast<T*>(p.dx) + (row0 + r) * p.sdx + l.c, l, dx);
            }
        }
    }
    if (parts == nullptr) return;
    // the rows of a team, or where every team has the one slab of all the workgroup's, together, channel by channel
    const int width = l.hi - l.lo;
    const bool together = !WAVE || q.slabs == 1;
    const int teams_here = WAVE && together ? TH / q.ts : 1, size = teams_here * q.ts * V, slot = (WAVE && together ? tid / q.ts * q.slots : 0) + l.slot;
    float* const sums = WAVE && together ? red : myred;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (l.own[v]) {
            sums[slot * width + l.c + v - l.lo] = accb[v];
            sums[size + slot * width + l.c + v - l.lo] = accg[v];
        }
    __syncthreads();
    if (team >= teams && !together) return;
    float2* const to = parts + (size_t)(together ? (WAVE ? (int)blockIdx.x : team / q.slabs) : team / q.slabs) * p.C + l.lo;
    for (int c = WAVE && together ? tid : lt; c < width; c += WAVE && together ? TH : q.ts) {
        float b = 0.0f, g = 0.0f;
        for (int s = 0; s < teams_here * q.slots; ++s) { b += sums[s * width + c]; g += sums[size + s * width + c]; }
        to[c] = make_float2(b, g);
    }
}

// dbeta and dgamma from E parts of them: 64 channels x 16 shares of the parts per workgroup, joined in order.
__global__ __launch_bounds__(1024) void group_norm_params_kernel(const float2* parts, int E, int C, float* dgamma, float* dbeta) {
    __shared__ float2 red[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float2 s = make_float2(0.0f, 0.0f);
    if (c < C)
        for (int k = w; k < E; k += 16) {
            const float2 t = parts[(size_t)k * C + c];
            s.x += t.x; s.y += t.y;
        }
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < C) {
        for (int k = 1; k < 16; ++k) { s.x += red[k][lane].x; s.y += red[k][lane].y; }
        if (dbeta) dbeta[c] = s.x;
        if (dgamma) dgamma[c] = s.y;
    }
}

// ---- split form.  A workgroup has a tile: slots x K rows of an item's slab.
constexpr int kTileThreads = 256;
struct Tile { long long n; int chunk, slab; };
__device__ __forceinline__ Tile tile_of(const Geo& q, int chunks) {
    Tile t;
    t.slab = blockIdx.x % q.slabs;
    const unsigned r = blockIdx.x / q.slabs;
    t.chunk = r % chunks;
    t.n = r / chunks;
    return t;
}

// part[(n G + g) E + e] = (rows, mean, squared deviations), E = chunks x spg tiles of a group
template <typename T, int V, int K>
__global__ __launch_bounds__(kTileThreads) void group_norm_tiles_kernel(const GroupNormArgs p, const Geo q, int chunks, float4* part) {
    __shared__ float red[kTileThreads * V], mean_of[kTileThreads * V];
    __shared__ int cnt;
    const Tile t = tile_of(q, chunks);
    const Lane<V> l(q, p.C, p.G, t.slab, threadIdx.x);
    const int r0 = t.chunk * q.slots * K;
    const long long row0 = t.n * p.P;
    Pack<T, V> x[K];
    bool live[K];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + l.slot + k * q.slots;
        const long long row = row0 + min(r, p.P - 1);
        x[k] = load_pack<T, V>(static_cast<const T*>(p.x) + row * p.sx + l.c);
        live[k] = l.on && r < p.P && (p.mask == nullptr || p.mask[row] == 0);
        mine += live[k];
    }
    const int rows = p.mask != nullptr ? count_rows<false>(&cnt, l.lt, l.lt % q.lanes == 0, mine) : min(q.slots * K, p.P - r0);
    const float M = (float)rows * (float)l.D, inv = rows > 0 ? 1.0f / M : 0.0f;
    float s[1][V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        s[0][v] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) s[0][v] += live[k] ? get<T, V>(x[k], v) : 0.0f;
    }
    group_sums<V, 1, false>(q, l, red, s, [&](int g, const float* u) { mean_of[g] = u[0] * inv; });
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float mean = mean_of[l.group_of(v)];
        s[0][v] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float d = live[k] ? get<T, V>(x[k], v) - mean : 0.0f;
            s[0][v] = fmaf(d, d, s[0][v]);
        }
    }
    const int E = chunks * q.spg;
    group_sums<V, 1, false>(q, l, red, s, [&](int g, const float* u) {
        part[((size_t)t.n * p.G + l.g0 + g) * E + (size_t)t.chunk * q.spg + t.slab % q.spg] = make_float4(M, mean_of[g], u[0], 0.0f);
    });
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}
// One wavefront per item and group joins its tiles.
__global__ __launch_bounds__(256) void group_norm_join_kernel(const float4* part, long long groups, int E, float eps, float* stats) {
    const long long i = blockIdx.x * 4LL + (threadIdx.x >> 6);
    if (i >= groups) return;
    const int lane = threadIdx.x & 63;
    const float4* mine = part + (size_t)i * E;
    float M = 0.0f, s = 0.0f, m2 = 0.0f;
    for (int e = lane; e < E; e += 64) { M += mine[e].x; s = fmaf(mine[e].x, mine[e].y, s); }
    M = wave_sum(M);
    const float mean = M > 0.0f ? wave_sum(s) / M : 0.0f;
    for (int e = lane; e < E; e += 64) {
        const float4 t = mine[e];
        const float d = t.y - mean;
        m2 += fmaf(t.x * d, d, t.z);
    }
    m2 = wave_sum(m2);
    if (lane == 0) {
        stats[2 * i] = mean;
        stats[2 * i + 1] = M > 0.0f ? 1.0f / sqrtf(m2 / M + eps) : 0.0f;
    }
}

template <typename T, int V, int K, int ACT>
__global__ __launch_bounds__(kTileThreads) void group_norm_apply_kernel(const GroupNormArgs p, const Geo q, int chunks) {
    const Tile t = tile_of(q, chunks);
    const Lane<V> l(q, p.C, p.G, t.slab, threadIdx.x);
    if (!l.on) return;
    const int r0 = t.chunk * q.slots * K;
    const long long row0 = t.n * p.P;
    Pack<T, V> x[K];
    bool live[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + l.slot + k * q.slots;
        const long long row = row0 + min(r, p.P - 1);
        x[k] = load_pack<T, V>(static_cast<const T*>(p.x) + row * p.sx + l.c);
        live[k] = p.mask == nullptr || p.mask[row] == 0;
    }
    float gamma[V], beta[V], mean[V], rstd[V];
    load_params<V>(p, l.c, gamma, beta);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float* st = p.stats + ((size_t)t.n * p.G + l.g0 + l.group_of(v)) * 2;
        mean[v] = st[0];
        rstd[v] = st[1];
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + l.slot + k * q.slots;
        if (r < p.P) {
            float y[V];
#pragma unroll
            for (int v = 0; v < V; ++v) y[v] = live[k] ? act_of<ACT>(fmaf((get<T, V>(x[k], v) - mean[v]) * rstd[v], gamma[v], beta[v])) : 0.0f;
            store_own<T, V>(static_cast<T*>(p.y) + (row0 + r) * p.sy + l.c, l, y);
        }
    }
}

// sums[n][chunk][C] = (sum dv, sum dv xh) of a tile; rows[n][chunk]: its rows that count
template <typename T, int V, int K, int ACT>
__global__ __launch_bounds__(kTileThreads) void group_norm_sums_kernel(const GroupNormArgs p, const Geo q, int chunks, float2* sums, float* counts) {
    __shared__ float red[2][kTileThreads * V];
    __shared__ int cnt;
    const Tile t = tile_of(q, chunks);
    const Lane<V> l(q, p.C, p.G, t.slab, threadIdx.x);
    const int r0 = t.chunk * q.slots * K;
    const long long row0 = t.n * p.P;
    Pack<T, V> x[K], dy[K];
    bool live[K];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + l.slot + k * q.slots;
        const long long row = row0 + min(r, p.P - 1);
        x[k] = load_pack<T, V>(static_cast<const T*>(p.x) + row * p.sx + l.c);
        dy[k] = load_pack<T, V>(static_cast<const T*>(p.dy) + row * p.sdy + l.c);
        live[k] = l.on && r < p.P && (p.mask == nullptr || p.mask[row] == 0);
        mine += live[k];
    }
    float gamma[V], beta[V];
    load_params<V>(p, l.c, gamma, beta);
    const int width = l.hi - l.lo;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float* st = p.stats + ((size_t)t.n * p.G + l.g0 + l.group_of(v)) * 2;
        const float mean = st[0], rstd = st[1];
        float b = 0.0f, g = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float xh = (get<T, V>(x[k], v) - mean) * rstd;
            const float dv = get<T, V>(dy[k], v) * act_slope<ACT>(fmaf(xh, gamma[v], beta[v]));
            b += live[k] ? dv : 0.0f;
            g += live[k] ? dv * xh : 0.0f;
        }
        if (l.own[v]) {
            red[0][l.slot * width + l.c + v - l.lo] = b;
            red[1][l.slot * width + l.c + v - l.lo] = g;
        }
    }
    const int rows = p.mask != nullptr ? count_rows<false>(&cnt, l.lt, l.lt % q.lanes == 0, mine) : min(q.slots * K, p.P - r0);
    __syncthreads();
    for (int c = l.lt; c < width; c += kTileThreads) {
        float b = 0.0f, g = 0.0f;
        for (int s = 0; s < q.slots; ++s) { b += red[0][s * width + c]; g += red[1][s * width + c]; }
        sums[((size_t)t.n * chunks + t.chunk) * p.C + l.lo + c] = make_float2(b, g);
    }
    if (t.slab == 0 && threadIdx.x == 0) counts[(size_t)t.n * chunks + t.chunk] = (float)rows;
}

// 64 channels of an item per workgroup: the tiles' sums joined in order, chan[n][C].
__global__ __launch_bounds__(1024) void group_norm_chan_kernel(const float2* sums, int chunks, int C, float2* chan) {
    __shared__ float2 red[16][64];
    const int cols = (C + 63) / 64, lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = (blockIdx.x % cols) * 64 + lane;
    const size_t n = blockIdx.x / cols;
    float2 s = make_float2(0.0f, 0.0f);
    if (c < C)
        for (int k = w; k < chunks; k += 16) {
            const float2 t = sums[(n * chunks + k) * C + c];
            s.x += t.x; s.y += t.y;
        }
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < C) {
        for (int k = 1; k < 16; ++k) { s.x += red[k][lane].x; s.y += red[k][lane].y; }
        chan[n * C + c] = s;
    }
}
// One wavefront per item and group: coef[n][G] = (sum dv gamma, sum dv gamma xh) / M.
__global__ __launch_bounds__(256) void group_norm_coef_kernel(const float2* chan, const float* counts, int chunks, const float* gamma, long long groups,
                                                              int G, int D, float2* coef) {
    const long long i = blockIdx.x * 4LL + (threadIdx.x >> 6);
    if (i >= groups) return;
    const int lane = threadIdx.x & 63, g = (int)(i % G);
    const long long n = i / G;
    float rows = 0.0f, a = 0.0f, b = 0.0f;
    for (int k = lane; k < chunks; k += 64) rows += counts[n * chunks + k];
    for (int d = lane; d < D; d += 64) {
        const float2 t = chan[((size_t)n * G + g) * D + d];
        const float gm = gamma ? gamma[g * D + d] : 1.0f;
        a = fmaf(t.x, gm, a);
        b = fmaf(t.y, gm, b);
    }
    rows = wave_sum(rows); a = wave_sum(a); b = wave_sum(b);
    const float inv = rows > 0.0f ? 1.0f / (rows * (float)D) : 0.0f;
    if (lane == 0) coef[i] = make_float2(a * inv, b * inv);
}

template <typename T, int V, int K, int ACT>
__global__ __launch_bounds__(kTileThreads) void group_norm_grad_kernel(const GroupNormArgs p, const Geo q, int chunks, const float2* coef) {
    const Tile t = tile_of(q, chunks);
    const Lane<V> l(q, p.C, p.G, t.slab, threadIdx.x);
    if (!l.on) return;
    const int r0 = t.chunk * q.slots * K;
    const long long row0 = t.n * p.P;
    Pack<T, V> x[K], dy[K];
    bool live[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + l.slot + k * q.slots;
        const long long row = row0 + min(r, p.P - 1);
        x[k] = load_pack<T, V>(static_cast<const T*>(p.x) + row * p.sx + l.c);
        dy[k] = load_pack<T, V>(static_cast<const T*>(p.dy) + row * p.sdy + l.c);
        live[k] = p.mask == nullptr || p.mask[row] == 0;
    }
    float gamma[V], beta[V], mean[V], rstd[V], s1[V], s2[V];
    load_params<V>(p, l.c, gamma, beta);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const size_t at = (size_t)t.n * p.G + l.g0 + l.group_of(v);
        mean[v] = p.stats[2 * at];
        rstd[v] = p.stats[2 * at + 1];
        s1[v] = coef[at].x;
        s2[v] = coef[at].y;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + l.slot + k * q.slots;
        if (r < p.P) {
            float dx[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float xh = (get<T, V>(x[k], v) - mean[v]) * rstd[v];
                const float dv = get<T, V>(dy[k], v) * act_slope<ACT>(fmaf(xh, gamma[v], beta[v]));
                dx[v] = live[k] ? rstd[v] * (fmaf(dv, gamma[v], -s1[v]) - xh * s2[v]) : 0.0f;
            }
            store_own<T, V>(static_cast<T*>(p.dx) + (row0 + r) * p.sdx + l.c, l, dx);
        }
    }
}

// ---- shapes
constexpr int kMaxWgs = 2048;            // workgroups of the held form: eight per compute unit
enum { FORM_WAVE = 0, FORM_GROUP = 1, FORM_SPLIT = 2 };
constexpr int kHeldRows = 8, kWaveThreads = 256, kGroupThreads = 512, kTileRows = 8;

int floor_pow2(int v) {
    int r = 1;
    while (2 * r <= v) r *= 2;
    return r;
}
struct NormPlan {
    int form, V, K;                      // K: rows of a lane
    Geo q;
    long long teams, parts;              // held forms; parts of the parameters' sums
    int chunks;                          // split form
};
// Slabs of at most `most` channels for teams of ts lanes; false where a group is wider than that and has to be whole.
bool fill_geo(const scan2d_group_norm_desc* d, int V, int ts, int most, bool whole, Geo* q) {
    const int D = d->C / d->G;
    q->ts = ts;
    q->spg = 1;
    if (D <= most) {
        int slabs = (int)((d->G + most / D - 1) / (most / D));
        q->gps = (d->G + slabs - 1) / slabs;
        q->slabs = (d->G + q->gps - 1) / q->gps;
        q->D = D;
        q->width = q->gps * D;
    } else {
        if (whole) return false;
        q->spg = (D + most - 1) / most;
        q->width = (D + q->spg - 1) / q->spg;
        q->spg = (D + q->width - 1) / q->width;
        q->gps = 1;
        q->slabs = d->G * q->spg;
        q->D = q->width;
    }
    q->lanes = (q->width + V - 1) / V;
    if (q->lanes > ts) return false;
    q->slots = ts / q->lanes;
    q->tpg = floor_pow2(ts / (q->gps < ts ? q->gps : ts));
    if (q->tpg > 64) q->tpg = 64;
    return true;
}
NormPlan plan_of(const scan2d_group_norm_desc* d) {
    NormPlan n = {};
    n.V = d->C >= 4 ? 4 : 1;
    const int D = d->C / d->G;
    const auto held = [&](int form, long long most_teams) {
        n.form = form;
        n.K = n.q.slots >= d->P && n.V > 1 ? 1 : kHeldRows;
        most_teams = most_teams < n.q.slabs ? n.q.slabs : most_teams / n.q.slabs * n.q.slabs;
        n.teams = (long long)d->N * n.q.slabs;
        if (n.teams > most_teams) n.teams = most_teams;
        n.parts = form == FORM_WAVE && n.q.slabs == 1 ? (n.teams * n.q.ts + kWaveThreads - 1) / kWaveThreads : n.teams / n.q.slabs;
        return n;
    };
    // a team within a wavefront: the fewest lanes that hold a row's slab and all positions
    for (int ts = 1; ts <= 64; ts *= 2) {
        const int most = ts * n.V;
        if (D > most || (ts < 64 && d->C > most)) continue;
        if (!fill_geo(d, n.V, ts, most, true, &n.q)) continue;
        if ((long long)n.q.slots * kHeldRows >= d->P) return held(FORM_WAVE, (long long)kMaxWgs * (kWaveThreads / ts));
    }
    // a workgroup: narrower slabs where whole rows do not fit
    for (int most = kGroupThreads * n.V; most >= 32; most /= 2) {
        if (D > most) break;
        if (!fill_geo(d, n.V, kGroupThreads, most, true, &n.q)) continue;
        if ((long long)n.q.slots * kHeldRows >= d->P) return held(FORM_GROUP, kMaxWgs);
    }
    n.form = FORM_SPLIT;
    (void)fill_geo(d, n.V, kTileThreads, kTileThreads * n.V, false, &n.q);
    n.chunks = (int)((d->P + (long long)n.q.slots * kTileRows - 1) / ((long long)n.q.slots * kTileRows));
    return n;
}
size_t up(size_t n) { return (n + 255) / 256 * 256; }
int launched() { return hipGetLastError() == hipSuccess ? SCAN2D_OK : SCAN2D_ERR_LAUNCH_FAILED; }

template <typename T, int V, int ACT>
int fwd(const GroupNormArgs& a, const NormPlan& n, hipStream_t stream) {
    if (n.form != FORM_SPLIT) {
        using Kernel = void (*)(const GroupNormArgs, const Geo, int);
        const bool wave = n.form == FORM_WAVE;
        Kernel k = wave ? group_norm_fwd_kernel<T, V, kHeldRows, kWaveThreads, true, ACT> : group_norm_fwd_kernel<T, V, kHeldRows, kGroupThreads, false, ACT>;
        if constexpr (V > 1)
            if (n.K == 1) k = wave ? group_norm_fwd_kernel<T, V, 1, kWaveThreads, true, ACT> : group_norm_fwd_kernel<T, V, 1, kGroupThreads, false, ACT>;
        const long long blocks = wave ? (n.teams * n.q.ts + kWaveThreads - 1) / kWaveThreads : n.teams;
        hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(wave ? kWaveThreads : kGroupThreads), 0, stream, a, n.q, (int)n.teams);
        return launched();
    }
    const long long blocks = (long long)a.N * n.chunks * n.q.slabs, groups = (long long)a.N * a.G;
    if (!launch_fits(blocks, kTileThreads) || !launch_fits(groups / 4 + 1, 256)) return SCAN2D_ERR_BAD_SHAPE;
    float4* part = static_cast<float4*>(a.workspace);
    hipLaunchKernelGGL((group_norm_tiles_kernel<T, V, kTileRows>), dim3((unsigned)blocks), dim3(kTileThreads), 0, stream, a, n.q, n.chunks, part);
    hipLaunchKernelGGL(group_norm_join_kernel, dim3((unsigned)((groups + 3) / 4)), dim3(256), 0, stream, part, groups, n.chunks * n.q.spg, a.eps, a.stats);
    hipLaunchKernelGGL((group_norm_apply_kernel<T, V, kTileRows, ACT>), dim3((unsigned)blocks), dim3(kTileThreads), 0, stream, a, n.q, n.chunks);
    return launched();
}
template <typename T, int V, int ACT>
int bwd(const GroupNormArgs& a, const NormPlan& n, hipStream_t stream) {
    const bool params = a.dgamma != nullptr || a.dbeta != nullptr;
    const dim3 cols((a.C + 63) / 64);
    if (n.form != FORM_SPLIT) {
        using Kernel = void (*)(const GroupNormArgs, const Geo, int, float2*);
        const bool wave = n.form == FORM_WAVE;
        float2* parts = params ? static_cast<float2*>(a.workspace) : nullptr;
        Kernel k = wave ? group_norm_bwd_kernel<T, V, kHeldRows, kWaveThreads, true, ACT> : group_norm_bwd_kernel<T, V, kHeldRows, kGroupThreads, false, ACT>;
        if constexpr (V > 1)
            if (n.K == 1) k = wave ? group_norm_bwd_kernel<T, V, 1, kWaveThreads, true, ACT> : group_norm_bwd_kernel<T, V, 1, kGroupThreads, false, ACT>;
        const long long blocks = wave ? (n.teams * n.q.ts + kWaveThreads - 1) / kWaveThreads : n.teams;
        hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(wave ? kWaveThreads : kGroupThreads), 0, stream, a, n.q, (int)n.teams, parts);
        if (params) hipLaunchKernelGGL(group_norm_params_kernel, cols, dim3(1024), 0, stream, parts, (int)n.parts, a.C, a.dgamma, a.dbeta);
        return launched();
    }
    const long long blocks = (long long)a.N * n.chunks * n.q.slabs, groups = (long long)a.N * a.G;
    if (!launch_fits(blocks, kTileThreads) || !launch_fits(groups / 4 + 1, 256) || !launch_fits((long long)a.N * cols.x, 1024)) return SCAN2D_ERR_BAD_SHAPE;
    char* w = static_cast<char*>(a.workspace);
    const size_t items = (size_t)a.N * n.chunks;
    float2* sums = reinterpret_cast<float2*>(w);
    w += up(items * a.C * sizeof(float2));
    float* counts = reinterpret_cast<float*>(w);
    w += up(items * sizeof(float));
    float2* chan = reinterpret_cast<float2*>(w);
    w += up((size_t)a.N * a.C * sizeof(float2));
    float2* coef = reinterpret_cast<float2*>(w);
    hipLaunchKernelGGL((group_norm_sums_kernel<T, V, kTileRows, ACT>), dim3((unsigned)blocks), dim3(kTileThreads), 0, stream, a, n.q, n.chunks, sums, counts);
    hipLaunchKernelGGL(group_norm_chan_kernel, dim3((unsigned)(a.N * cols.x)), dim3(1024), 0, stream, sums, n.chunks, a.C, chan);
    hipLaunchKernelGGL(group_norm_coef_kernel, dim3((unsigned)((groups + 3) / 4)), dim3(256), 0, stream, chan, counts, n.chunks, a.gamma, groups, a.G, a.D, coef);
    hipLaunchKernelGGL((group_norm_grad_kernel<T, V, kTileRows, ACT>), dim3((unsigned)blocks), dim3(kTileThreads), 0, stream, a, n.q, n.chunks, coef);
    if (params) hipLaunchKernelGGL(group_norm_params_kernel, cols, dim3(1024), 0, stream, chan, a.N, a.C, a.dgamma, a.dbeta);
    return launched();
}

template <typename T, int V>
int by_act(const GroupNormArgs& a, const NormPlan& n, bool backward, hipStream_t stream) {
    (void)hipGetLastError();
    switch (a.act) {
        case SCAN2D_ACT_SILU: return backward ? bwd<T, V, SCAN2D_ACT_SILU>(a, n, stream) : fwd<T, V, SCAN2D_ACT_SILU>(a, n, stream);
        case SCAN2D_ACT_GELU: return backward ? bwd<T, V, SCAN2D_ACT_GELU>(a, n, stream) : fwd<T, V, SCAN2D_ACT_GELU>(a, n, stream);
        default: return backward ? bwd<T, V, SCAN2D_ACT_NONE>(a, n, stream) : fwd<T, V, SCAN2D_ACT_NONE>(a, n, stream);
    }
}
int dispatch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, bool backward, hipStream_t stream) {
    const NormPlan n = plan_of(d);
    if (d->dtype == SCAN2D_BF16) return n.V == 1 ? by_act<bf16_t, 1>(a, n, backward, stream) : by_act<bf16_t, 4>(a, n, backward, stream);
    return n.V == 1 ? by_act<float, 1>(a, n, backward, stream) : by_act<float, 4>(a, n, backward, stream);
}

}  // namespace

size_t group_norm_workspace_bytes(const scan2d_group_norm_desc* d, int pass) {
    const NormPlan n = plan_of(d);
    if (n.form != FORM_SPLIT) return pass == SCAN2D_PASS_BWD ? (size_t)n.parts * d->C * sizeof(float2) : 0;
    const size_t items = (size_t)d->N * n.chunks;
    if (pass == SCAN2D_PASS_FWD) return items * n.q.spg * d->G * sizeof(float4);
    return up(items * d->C * sizeof(float2)) + up(items * sizeof(float)) + up((size_t)d->N * d->C * sizeof(float2)) + (size_t)d->N * d->G * sizeof(float2);
}
int group_norm_fwd_launch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, hipStream_t stream) { return dispatch(d, a, false, stream); }
int group_norm_bwd_launch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, hipStream_t stream) { return dispatch(d, a, true, stream); }

}  // namespace scan2d
