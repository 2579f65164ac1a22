// Group norm with an activation on channels-last tensors (include/scan2d_seq.h).
//
// Bound: HBM (forward 1 read and 1 write per element, backward 2 and 1) as long as the statistics are there; they need all
// of an item's group first.  Channels go along the lanes, V neighbours each, and what lanes are left over by narrow rows take further
// positions.  A workgroup or wavefront has a slab of whole groups (or a part of one group that is wider than it).
//
// Held form (group_norm_fwd_kernel, group_norm_bwd_kernel): a team of lanes holds all positions of an item's slab in
// registers as they were loaded: one read.  Teams are a power of two of lanes within a wavefront (nothing waits for another
// wavefront; small maps), or a workgroup.  A team goes on to the next items of its slab with its channels' parameters, and in the
// backward pass its channels' sums, in registers; where an item is one row of a lane, a workgroup takes several items at once, so
// that enough bytes are on their way.
// Split form, where an item's slab does not fit: a workgroup has a tile, a share of an item's positions, and goes through it kRows rows
// of a lane at a time.  Forward: each lane keeps mean and squared deviations of its channels (rows in registers: their mean, the deviations
// from it, joined to those before by M2 = M2_1 + M2_2 + n1 n2 / (n1 + n2) (mean_1 - mean_2)^2), which are joined to those of the tile, those
// of the tiles to the item's; then the tensor is read again and written, last rows first, which are the ones still in a cache.
// Backward: the channels' sums of dv and dv xh of a tile, joined to those of the item and with gamma to the groups', then dx from a second read.
// The variance is always taken from deviations, never from the difference of two large sums.
// All sums run in a fixed order.
//
// Measured (forward, backward; a copy reaches 5.2 TB/s, 8.6 where it stays in the Infinity Cache): 16384 tokens x 2048 bf16 31 and 52 us (4.3 and 3.9 TB/s of their
// bytes), held 8 x 196 x 256 bf16 7.4 and 10.7 us, split 65536 x 256 bf16 masked 25 and 40 us, 32 x 3136 x 192 bf16 28 and 45 us, 3 x 4731 x 384 fp32
// 20 and 30 us.  What the split form adds to the bytes' time: the second read, out of the Infinity Cache, and 3 to 5 us per launch.
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
// Outputs are stored non-temporally: nothing reads them again here, and what is read twice stays in the L2 (16384 tokens x 2048 bf16
// forward 36.8 us without, 30.8 with; 2 x 9000 x 771 fp32 40.8 and 37.0).
template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const float* v) {
    if constexpr (V == 1) {
        store_elem(p, v[0]);
    } else {
        constexpr int W = V * Elem<T>::kBytes / 4;
        uint32_t w[W];
#pragma unroll
        for (int k = 0; k < W; ++k) {
            if constexpr (Elem<T>::kBytes == 4) w[k] = __float_as_uint(v[k]);
            else w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
        }
        if constexpr (W == 4) {
            u32x4_a1 q;
            q.x = w[0]; q.y = w[1]; q.z = w[2]; q.w = w[3];
            __builtin_nontemporal_store(q, reinterpret_cast<u32x4_a1*>(p));
        } else {
            static_assert(W == 2, "two or four dwords");
            u32x2_a1 q;
            q.x = w[0]; q.y = w[1];
            __builtin_nontemporal_store(q, reinterpret_cast<u32x2_a1*>(p));
        }
    }
}

__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v * kLog2e)); }
// The normal distribution Phi(v) and e^(-v^2/2): with x = |v| / sqrt(2) and t = 1 / (1 + 0.3 x), Phi(-|v|) = t q(t) e^(-x^2) / 2, q the
// Chebyshev fit of degree 8 to e^(x^2) erfc(x) / t (off by 3.2e-8); one exponential for Phi and its slope, a third of erff's work.
__device__ __forceinline__ float normal_cdf(float v, float& e) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.212132034f, fabsf(v), 1.0f));
    e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * v * v);
    float q = fmaf(t, -0.12841005623340607f, 0.48013120889663696f);
    q = fmaf(t, q, -0.5010061860084534f);
    q = fmaf(t, q, 0.5347656011581421f);
    q = fmaf(t, q, -0.08565600961446762f);
    q = fmaf(t, q, 0.2110726535320282f);
    q = fmaf(t, q, 0.14933134615421295f);
    q = fmaf(t, q, 0.17057515680789948f);
    q = fmaf(t, q, 0.16919629275798798f);
    const float tail = 0.5f * t * q * e;
    return v < 0.0f ? tail : 1.0f - tail;
}
template <int ACT>
__device__ __forceinline__ float act_of(float v) {
    if constexpr (ACT == SCAN2D_ACT_SILU) return v * sigmoid(v);
    else if constexpr (ACT == SCAN2D_ACT_GELU) {
        float e;
        return v * normal_cdf(v, e);
    } else return v;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float v) {
    if constexpr (ACT == SCAN2D_ACT_SILU) {
        const float s = sigmoid(v);
        return s * fmaf(v, 1.0f - s, 1.0f);
    } else if constexpr (ACT == SCAN2D_ACT_GELU) {
        float e;
        const float cdf = normal_cdf(v, e);
        return fmaf(v * 0.39894228f, e, cdf);
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
    float per_lanes, per_D;              // 1 / lanes, 1 / D
};
// a / b for 0 <= a < 2^22, with 1 / b rounded: (a + 1/2) / b is at least 1 / 2b from a whole number, and off by less
__device__ __forceinline__ int quotient(int a, float per_b) { return (int)(((float)a + 0.5f) * per_b); }

// A team's slab, and this lane's channels of it.  ONE: a lane's channels are of one group (V divides the groups' channels).
template <int V, bool ONE>
struct Lane {
    static constexpr int GV = ONE ? 1 : V;                 // values per group of a lane's channels
    int lt;                              // within the team
    int slot, c;                         // which of the team's rows; first channel
    int lo, width;                       // the slab's channels
    int groups, D;                       // the slab's groups, their channels (of the slab)
    int g0;                              // its first group
    int first;                           // the lane's first own channel within the slab
    int gr[GV];                          // the group, within the slab, of each channel
    bool on;                             // has a row at all
    bool own[V];                         // which channels are this lane's
    bool all;
    __device__ Lane(const Geo& q, int C, int G, int slab, int lane) {
        lt = lane;
        int hi;
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
        width = hi - lo;
        slot = quotient(lane, q.per_lanes);
        const int mine = lo + (lane - slot * q.lanes) * V;
        first = mine - lo;
        on = slot < q.slots && mine < hi;
        c = min(mine, C - V);
        all = true;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            own[v] = on && c + v >= mine && c + v < hi;
            all = all && own[v];
        }
#pragma unroll
        for (int v = 0; v < GV; ++v) gr[v] = q.spg > 1 ? 0 : min(quotient(max((ONE ? mine : c + v) - lo, 0), q.per_D), groups - 1);
    }
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
// group.  The values of channels that are not the lane's are not looked at.  red: NR x size floats of the team, size at least
// ts V (ts where a lane's channels are of one group and added up first).
template <int V, bool ONE, int NR, bool WAVE, typename Done>
__device__ __forceinline__ void group_sums(const Geo& q, const Lane<V, ONE>& l, float* red, int size, const float (&val)[NR][V], Done done) {
    const int width = ONE ? q.lanes : l.width, D = ONE ? (l.D + V - 1) / V : l.D;
    if constexpr (ONE) {
        if (l.on) {
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                float s = l.own[0] ? val[r][0] : 0.0f;
#pragma unroll
                for (int v = 1; v < V; ++v) s += l.own[v] ? val[r][v] : 0.0f;
                red[r * size + l.lt] = s;
            }
        }
    } else {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (l.own[v]) red[r * size + l.slot * width + l.c + v - l.lo] = val[r][v];
    }
    team_sync<WAVE>();
    const int qq = l.lt & (q.tpg - 1), n = q.slots * D, row0 = qq / D, d0 = qq % D, rowstep = q.tpg / D, dstep = q.tpg % D;
    for (int g = l.lt / q.tpg; g < l.groups; g += q.ts / q.tpg) {
        float s[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r] = 0.0f;
        for (int e = qq, row = row0, d = d0; e < n; e += q.tpg) {
#pragma unroll
            for (int r = 0; r < NR; ++r) s[r] += red[r * size + row * width + g * D + d];
            row += rowstep;
            d += dstep;
            if (d >= D) { d -= D; ++row; }
        }
        for (int m = 1; m < q.tpg; m <<= 1)
#pragma unroll
            for (int r = 0; r < NR; ++r) s[r] += __shfl_xor(s[r], m);
        if (qq == 0) done(g, s);
    }
    team_sync<WAVE>();
}

// The rows that count of R items of a team, each in a counter of its own (cnts[item][at]): wavefronts read them at different times, so a
// counter is written again only behind another barrier of the team, which the sums of the items are.
template <bool WAVE, int R, int N>
__device__ __forceinline__ void count_rows(int (&cnts)[R][N], int at, int lt, bool counts, const int (&mine)[R], int (&rows)[R]) {
    if (lt == 0) {
#pragma unroll
        for (int i = 0; i < R; ++i) cnts[i][at] = 0;
    }
    team_sync<WAVE>();
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (counts && mine[i] != 0) atomicAdd(&cnts[i][at], mine[i]);
    team_sync<WAVE>();
#pragma unroll
    for (int i = 0; i < R; ++i) rows[i] = cnts[i][at];
}

template <int V>
__device__ __forceinline__ void load_params(const GroupNormArgs& p, int c, float* gamma, float* beta) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        gamma[v] = p.gamma ? p.gamma[c + v] : 1.0f;
        beta[v] = p.beta ? p.beta[c + v] : 0.0f;
    }
}
template <typename T, int V, bool ONE>
__device__ __forceinline__ void store_own(T* p, const Lane<V, ONE>& l, const float* v) {
    if (l.all) {
        store_pack<T, V>(p, v);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (l.own[k]) store_elem(p + k, v[k]);
    }
}

// ---- held form.  R items at once, K rows of each per lane.
template <typename T, int V, bool ONE, int K, int R, int TH, bool WAVE, int ACT>
__global__ __launch_bounds__(TH) void group_norm_fwd_kernel(const GroupNormArgs p, const Geo q, int teams) {
    constexpr int GV = Lane<V, ONE>::GV, PER = ONE ? 1 : V;                  // floats of red per lane
    __shared__ float red[R * TH * PER], res[2][R][TH * GV];
    __shared__ int cnts[R][WAVE ? TH : 1];
    const int tid = threadIdx.x, lt = WAVE ? tid & (q.ts - 1) : tid, base = tid - lt;
    const int team = WAVE ? (int)((blockIdx.x * (long long)TH + tid) / q.ts) : (int)blockIdx.x;      // teams is a multiple of slabs
    const Lane<V, ONE> l(q, p.C, p.G, team % q.slabs, lt);
    float* const myred = red + R * base * PER;
    float gamma[V], beta[V];
    load_params<V>(p, l.c, gamma, beta);
    const int step = teams / q.slabs, rounds = (p.N - 1) / (step * R) + 1;
    for (int it = 0; it < rounds; ++it) {
        Pack<T, V> x[R][K];
        bool live[R][K];
        long long item[R], row0[R];
        int rows[R], mine[R];
        bool real[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long n = team / q.slabs + ((long long)it * R + i) * step;
            real[i] = n < p.N && team < teams;              // the last workgroup may have lanes to spare
            item[i] = n;
            row0[i] = (real[i] ? n : 0) * p.P;
            mine[i] = 0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int r = l.slot + k * q.slots;
                const long long row = row0[i] + min(r, p.P - 1);
                x[i][k] = load_pack<T, V>(static_cast<const T*>(p.x) + row * p.sx + l.c);
                live[i][k] = real[i] && l.on && r < p.P && (p.mask == nullptr || p.mask[row] == 0);
                mine[i] += live[i][k];
            }
            rows[i] = p.P;
        }
        if (p.mask != nullptr) count_rows<WAVE, R>(cnts, WAVE ? base : 0, lt, lt % q.lanes == 0, mine, rows);
        float s[R][V], mean[R][GV], rstd[R][GV];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                s[i][v] = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k) s[i][v] += live[i][k] ? get<T, V>(x[i][k], v) : 0.0f;
            }
        float inv[R];
#pragma unroll
        for (int i = 0; i < R; ++i) inv[i] = rows[i] > 0 ? 1.0f / ((float)rows[i] * (float)l.D) : 0.0f;
        group_sums<V, ONE, R, WAVE>(q, l, myred, q.ts * PER, s, [&](int g, const float* t) {
#pragma unroll
            for (int i = 0; i < R; ++i) res[0][i][base * GV + g] = t[i] * inv[i];
        });
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int v = 0; v < GV; ++v) mean[i][v] = res[0][i][base * GV + l.gr[v]];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                s[i][v] = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const float d = live[i][k] ? get<T, V>(x[i][k], v) - mean[i][ONE ? 0 : v] : 0.0f;
                    s[i][v] = fmaf(d, d, s[i][v]);
                }
            }
        }
        group_sums<V, ONE, R, WAVE>(q, l, myred, q.ts * PER, s, [&](int g, const float* t) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float rs = rows[i] > 0 ? 1.0f / sqrtf(t[i] * inv[i] + p.eps) : 0.0f;
                res[1][i][base * GV + g] = rs;
                if (real[i]) {
                    float* st = p.stats + ((size_t)item[i] * p.G + l.g0 + g) * 2;
                    st[0] = res[0][i][base * GV + g];
                    st[1] = rs;
                }
            }
        });
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int v = 0; v < GV; ++v) rstd[i][v] = res[1][i][base * GV + l.gr[v]];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int r = l.slot + k * q.slots;
                if (real[i] && l.on && r < p.P) {
                    float y[V];
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        y[v] = live[i][k] ? act_of<ACT>(fmaf((get<T, V>(x[i][k], v) - mean[i][ONE ? 0 : v]) * rstd[i][ONE ? 0 : v], gamma[v], beta[v])) : 0.0f;
                    store_own<T, V>(static_cast<T*>(p.y) + (row0[i] + r) * p.sy + l.c, l, y);
                }
            }
        }
    }
}

// parts: [..][C][2], the sums for dbeta and dgamma of the items that a team, or a workgroup of teams, had: the rows of a team, or where every
// team has the one slab of all the workgroup's, together, channel by channel.  red: 2 TH V floats of the workgroup.
template <int V, int TH, bool WAVE, typename L>
__device__ __forceinline__ void write_parts(const GroupNormArgs& p, const Geo& q, const L& l, int team, int teams, float* red, const float* accb,
                                            const float* accg, float2* parts) {
    const int tid = threadIdx.x, base = tid - l.lt;
    const bool together = !WAVE || q.slabs == 1;
    const int teams_here = WAVE && together ? TH / q.ts : 1, size = teams_here * q.ts * V, slot = (WAVE && together ? tid / q.ts * q.slots : 0) + l.slot;
    float* const sums = WAVE && together ? red : red + 2 * base * V;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (l.own[v]) {
            sums[slot * l.width + l.c + v - l.lo] = accb[v];
            sums[size + slot * l.width + l.c + v - l.lo] = accg[v];
        }
    __syncthreads();
    if (team >= teams && !together) return;
    float2* const to = parts + (size_t)(WAVE && together ? (int)blockIdx.x : team / q.slabs) * p.C + l.lo;
    for (int c = WAVE && together ? tid : l.lt; c < l.width; c += WAVE && together ? TH : q.ts) {
        float b = 0.0f, g = 0.0f;
        for (int s = 0; s < teams_here * q.slots; ++s) { b += sums[s * l.width + c]; g += sums[size + s * l.width + c]; }
        to[c] = make_float2(b, g);
    }
}

template <typename T, int V, bool ONE, int K, int R, int TH, bool WAVE, int ACT>
__global__ __launch_bounds__(TH) void group_norm_bwd_kernel(const GroupNormArgs p, const Geo q, int teams, float2* parts) {
    constexpr int GV = Lane<V, ONE>::GV, PER = ONE ? 1 : V;
    constexpr int RED = 2 * R * TH * PER > 2 * TH * V ? 2 * R * TH * PER : 2 * TH * V;       // the channels' sums at the end use it too
    __shared__ float red[RED], res[2][R][TH * GV];
    __shared__ int cnts[R][WAVE ? TH : 1];
    const int tid = threadIdx.x, lt = WAVE ? tid & (q.ts - 1) : tid, base = tid - lt;
    const int team = WAVE ? (int)((blockIdx.x * (long long)TH + tid) / q.ts) : (int)blockIdx.x;
    const Lane<V, ONE> l(q, p.C, p.G, team % q.slabs, lt);
    float* const myred = red + 2 * R * base * PER;
    float gamma[V], beta[V], accb[V], accg[V];
    load_params<V>(p, l.c, gamma, beta);
#pragma unroll
    for (int v = 0; v < V; ++v) accb[v] = accg[v] = 0.0f;
    const int step = teams / q.slabs, rounds = (p.N - 1) / (step * R) + 1;
    for (int it = 0; it < rounds; ++it) {
        Pack<T, V> x[R][K], dy[R][K];
        bool live[R][K], real[R];
        long long row0[R];
        int rows[R], mine[R];
        float mean[R][GV], rstd[R][GV];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long n = team / q.slabs + ((long long)it * R + i) * step;
            real[i] = n < p.N && team < teams;
            row0[i] = (real[i] ? n : 0) * p.P;
            mine[i] = 0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int r = l.slot + k * q.slots;
                const long long row = row0[i] + min(r, p.P - 1);
                x[i][k] = load_pack<T, V>(static_cast<const T*>(p.x) + row * p.sx + l.c);
                dy[i][k] = load_pack<T, V>(static_cast<const T*>(p.dy) + row * p.sdy + l.c);
                live[i][k] = real[i] && l.on && r < p.P && (p.mask == nullptr || p.mask[row] == 0);
                mine[i] += live[i][k];
            }
#pragma unroll
            for (int v = 0; v < GV; ++v) {
                const float* st = p.stats + ((size_t)(real[i] ? n : 0) * p.G + l.g0 + l.gr[v]) * 2;
                mean[i][v] = st[0];
                rstd[i][v] = st[1];
            }
            rows[i] = p.P;
        }
        if (p.mask != nullptr) count_rows<WAVE, R>(cnts, WAVE ? base : 0, lt, lt % q.lanes == 0, mine, rows);
        float s[2 * R][V], dv[R][K][V];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float b = 0.0f, g = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const float xh = (get<T, V>(x[i][k], v) - mean[i][ONE ? 0 : v]) * rstd[i][ONE ? 0 : v];
                    dv[i][k][v] = live[i][k] ? get<T, V>(dy[i][k], v) * act_slope<ACT>(fmaf(xh, gamma[v], beta[v])) : 0.0f;
                    b += dv[i][k][v];
                    g += live[i][k] ? dv[i][k][v] * xh : 0.0f;
                }
                accb[v] += b;
                accg[v] += g;
                s[2 * i][v] = b * gamma[v];
                s[2 * i + 1][v] = g * gamma[v];
            }
        group_sums<V, ONE, 2 * R, WAVE>(q, l, myred, q.ts * PER, s, [&](int g, const float* t) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float inv = rows[i] > 0 ? 1.0f / ((float)rows[i] * (float)l.D) : 0.0f;
                res[0][i][base * GV + g] = t[2 * i] * inv;
                res[1][i][base * GV + g] = t[2 * i + 1] * inv;
            }
        });
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float s1[GV], s2[GV];
#pragma unroll
            for (int v = 0; v < GV; ++v) { s1[v] = res[0][i][base * GV + l.gr[v]]; s2[v] = res[1][i][base * GV + l.gr[v]]; }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int r = l.slot + k * q.slots;
                if (real[i] && l.on && r < p.P) {
                    float dx[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const int w = ONE ? 0 : v;
                        const float xh = (get<T, V>(x[i][k], v) - mean[i][w]) * rstd[i][w];
                        dx[v] = live[i][k] ? rstd[i][w] * (fmaf(dv[i][k][v], gamma[v], -s1[w]) - xh * s2[w]) : 0.0f;
                    }
                    store_own<T, V>(static_cast<T*>(p.dx) + (row0[i] + r) * p.sdx + l.c, l, dx);
                }
            }
        }
        team_sync<WAVE>();                                  // res has been read
    }
    if (parts != nullptr) write_parts<V, TH, WAVE>(p, q, l, team, teams, red, accb, accg, parts);
}

// ---- single rows: a group has a power of two of neighbouring lanes (some may be idle), or a wavefront with J times V channels a lane; the
// sums stay in registers and cross the lanes by DPP and lane swaps (through LDS, as above, they took as long as the memory), and the
// next items are asked for before these are worked on.
constexpr int kTokenThreads = 256;
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true)); }
// NR sums over the `lanes` neighbours (a power of two, aligned) of each lane; all of them get them.
template <int NR>
__device__ __forceinline__ void lane_sums(int lanes, float (&s)[NR]) {
#pragma unroll
    for (int r = 0; r < NR; ++r)
        if (lanes > 1) s[r] += dpp<0xB1>(s[r]);             // quad_perm 1 0 3 2
#pragma unroll
    for (int r = 0; r < NR; ++r)
        if (lanes > 2) s[r] += dpp<0x4E>(s[r]);             // quad_perm 2 3 0 1
#pragma unroll
    for (int r = 0; r < NR; ++r)
        if (lanes > 4) s[r] += dpp<0x141>(s[r]);            // row_half_mirror: the other quad's sum
#pragma unroll
    for (int r = 0; r < NR; ++r)
        if (lanes > 8) s[r] += dpp<0x140>(s[r]);            // row_mirror: the other half row's
    if (lanes > 16) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const auto w = __builtin_amdgcn_permlane16_swap(__float_as_int(s[r]), __float_as_int(s[r]), false, false);
            s[r] = __int_as_float(w[0]) + __int_as_float(w[1]);
        }
    }
    if (lanes > 32) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const auto w = __builtin_amdgcn_permlane32_swap(__float_as_int(s[r]), __float_as_int(s[r]), false, false);
            s[r] = __int_as_float(w[0]) + __int_as_float(w[1]);
        }
    }
}
// q.lanes: lanes of a group, a power of two; q.gps, q.slabs: groups of a team, teams of a row.  ONE: V divides a group's channels.
template <int V, int J, bool ONE>
struct TokenLane {
    int c[J], mine[J], end, g;           // J times: channel to load from, first own channel; behind the group's last; the group
    int lo, width;                       // the team's channels
    bool on, first;                      // has a group; has its first channel
    __device__ TokenLane(const Geo& q, int C, int G, int slab, int lane) {
        const int g0 = slab * q.gps, at = lane / q.lanes, i = lane & (q.lanes - 1);
        lo = g0 * q.D;
        width = min(q.gps, G - g0) * q.D;
        on = at < q.gps && g0 + at < G;
        g = min(g0 + at, G - 1);
        end = (g + 1) * q.D;
        first = on && i == 0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            mine[j] = g * q.D + (j * 64 + i) * V;
            c[j] = min(mine[j], C - V);
        }
    }
    __device__ __forceinline__ bool any(int j) const { return on && mine[j] < end; }
    __device__ __forceinline__ bool own(int j, int v) const { return ONE ? any(j) : any(j) && c[j] + v >= mine[j] && c[j] + v < end; }
    template <typename T>
    __device__ __forceinline__ void load(const void* x, long long at, Pack<T, V>* to) const {
#pragma unroll
        for (int j = 0; j < J; ++j) to[j] = load_pack<T, V>(static_cast<const T*>(x) + at + c[j]);
    }
    template <typename T>
    __device__ __forceinline__ void store(void* to, long long at, int j, const float* v) const {
        T* const p = static_cast<T*>(to) + at + c[j];
        if (ONE || (c[j] == mine[j] && mine[j] + V <= end)) {
            if (any(j)) store_pack<T, V>(p, v);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (own(j, k)) store_elem(p + k, v[k]);
        }
    }
};
template <typename T, int V, int J, bool ONE, int R, int ACT>
__global__ __launch_bounds__(kTokenThreads) void group_norm_tokens_kernel(const GroupNormArgs p, const Geo q, int teams) {
    const int team = (int)((blockIdx.x * (long long)kTokenThreads + threadIdx.x) / q.ts);
    const TokenLane<V, J, ONE> l(q, p.C, p.G, team % q.slabs, threadIdx.x & (q.ts - 1));
    const long long step = teams / q.slabs;
    long long n0 = team < teams ? team / q.slabs : p.N;    // none for lanes to spare
    const auto row = [&](long long n) { return min(n, (long long)p.N - 1) * p.sx; };
    Pack<T, V> x[R][J];
#pragma unroll
    for (int i = 0; i < R; ++i) l.template load<T>(p.x, row(n0 + i * step), x[i]);
    float gamma[J][V], beta[J][V];
#pragma unroll
    for (int j = 0; j < J; ++j) load_params<V>(p, l.c[j], gamma[j], beta[j]);
    const float inv = 1.0f / (float)q.D;
    for (long long it = 0; it * R * step < p.N; ++it, n0 += R * step) {
        Pack<T, V> next[R][J];
        if ((it + 1) * R * step < p.N) {
#pragma unroll
            for (int i = 0; i < R; ++i) l.template load<T>(p.x, row(n0 + (R + i) * step), next[i]);
        }
        float mean[R], rstd[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            mean[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) mean[i] += l.own(j, v) ? get<T, V>(x[i][j], v) : 0.0f;
        }
        lane_sums<R>(q.lanes, mean);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            mean[i] *= inv;
            rstd[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float d = l.own(j, v) ? get<T, V>(x[i][j], v) - mean[i] : 0.0f;
                    rstd[i] = fmaf(d, d, rstd[i]);
                }
        }
        lane_sums<R>(q.lanes, rstd);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long n = n0 + i * step;
            if (n < p.N && l.on) {
                const bool out = p.mask != nullptr && p.mask[n] != 0;
                const float m = out ? 0.0f : mean[i], rs = out ? 0.0f : 1.0f / sqrtf(rstd[i] * inv + p.eps);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    float y[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) y[v] = out ? 0.0f : act_of<ACT>(fmaf((get<T, V>(x[i][j], v) - m) * rs, gamma[j][v], beta[j][v]));
                    l.template store<T>(p.y, n * p.sy, j, y);
                }
                if (l.first) {
                    float* st = p.stats + ((size_t)n * p.G + l.g) * 2;
                    st[0] = m;
                    st[1] = rs;
                }
            }
#pragma unroll
            for (int j = 0; j < J; ++j) x[i][j] = next[i][j];
        }
    }
}
template <typename T, int V, int J, bool ONE, int R, int ACT>
__global__ __launch_bounds__(kTokenThreads) void group_norm_tokens_bwd_kernel(const GroupNormArgs p, const Geo q, int teams, float2* parts) {
    constexpr bool AHEAD = J == 1;                          // several times V channels: no registers left for the next items
    __shared__ float red[2 * kTokenThreads * V * J];
    const int lt = threadIdx.x & (q.ts - 1), team = (int)((blockIdx.x * (long long)kTokenThreads + threadIdx.x) / q.ts);
    const TokenLane<V, J, ONE> l(q, p.C, p.G, team % q.slabs, lt);
    const long long step = teams / q.slabs;
    long long n0 = team < teams ? team / q.slabs : p.N;
    struct Item {
        Pack<T, V> x[J], dy[J];
        float mean, rstd;
    };
    const auto load = [&](long long n, Item& to) {
        n = min(n, (long long)p.N - 1);
        l.template load<T>(p.x, n * p.sx, to.x);
        l.template load<T>(p.dy, n * p.sdy, to.dy);
        const float* st = p.stats + ((size_t)n * p.G + l.g) * 2;
        to.mean = st[0];
        to.rstd = st[1];
    };
    Item w[R];
    if (AHEAD) {
#pragma unroll
        for (int i = 0; i < R; ++i) load(n0 + i * step, w[i]);
    }
    float gamma[J][V], beta[J][V], accb[J][V], accg[J][V];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        load_params<V>(p, l.c[j], gamma[j], beta[j]);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            gamma[j][v] = l.own(j, v) ? gamma[j][v] : 0.0f; // 0 times another group's infinity would count below
            accb[j][v] = accg[j][v] = 0.0f;
        }
    }
    const float inv = 1.0f / (float)q.D;
    for (long long it = 0; it * R * step < p.N; ++it, n0 += R * step) {
        Item next[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (!AHEAD) load(n0 + i * step, w[i]);
            else if ((it + 1) * R * step < p.N) load(n0 + (R + i) * step, next[i]);
        }
        float s1[R], s2[R], dv[R][J][V];
        bool live[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long n = n0 + i * step;
            live[i] = n < p.N && l.on && (p.mask == nullptr || p.mask[n] == 0);
            s1[i] = s2[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const bool counts = live[i] && l.own(j, v);
                    const float xh = (get<T, V>(w[i].x[j], v) - w[i].mean) * w[i].rstd;
                    dv[i][j][v] = counts ? get<T, V>(w[i].dy[j], v) * act_slope<ACT>(fmaf(xh, gamma[j][v], beta[j][v])) : 0.0f;
                    const float g = counts ? dv[i][j][v] * xh : 0.0f;
                    accb[j][v] += dv[i][j][v];
                    accg[j][v] += g;
                    s1[i] = fmaf(dv[i][j][v], gamma[j][v], s1[i]);
                    s2[i] = fmaf(g, gamma[j][v], s2[i]);
                }
        }
        lane_sums<R>(q.lanes, s1);
        lane_sums<R>(q.lanes, s2);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long n = n0 + i * step;
            if (n < p.N && l.on) {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    float dx[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float xh = (get<T, V>(w[i].x[j], v) - w[i].mean) * w[i].rstd;
                        dx[v] = live[i] ? w[i].rstd * (fmaf(dv[i][j][v], gamma[j][v], -s1[i] * inv) - xh * (s2[i] * inv)) : 0.0f;
                    }
                    l.template store<T>(p.dx, n * p.sdx, j, dx);
                }
            }
            if (AHEAD) w[i] = next[i];
        }
    }
    if (parts == nullptr) return;
    // where a row is one team's, the sums of all the workgroup's teams together
    const bool together = q.slabs == 1;
    const int teams_here = together ? kTokenThreads / q.ts : 1, size = teams_here * q.ts * V * J, at = together ? (int)threadIdx.x / q.ts : 0;
    float* const sums = together ? red : red + 2 * (threadIdx.x - lt) * V * J;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (l.own(j, v)) {
                sums[at * l.width + l.c[j] + v - l.lo] = accb[j][v];
                sums[size + at * l.width + l.c[j] + v - l.lo] = accg[j][v];
            }
    __syncthreads();
    if (team >= teams && !together) return;
    float2* const to = parts + (size_t)(together ? (int)blockIdx.x : team / q.slabs) * p.C + l.lo;
    for (int c = together ? threadIdx.x : lt; c < l.width; c += together ? kTokenThreads : q.ts) {
        float b = 0.0f, g = 0.0f;
        for (int k = 0; k < teams_here; ++k) { b += sums[k * l.width + c]; g += sums[size + k * l.width + c]; }
        to[c] = make_float2(b, g);
    }
}

// dbeta and dgamma from E parts of them: 16 channels x 64 shares of the parts per workgroup, joined in order.
__device__ __forceinline__ void join_params(const float2* parts, int E, int C, float* dgamma, float* dbeta, int block, int share, int shares, int lane,
                                            float2 (*red)[16]) {
    const int c = block * 16 + lane;
    float2 s = make_float2(0.0f, 0.0f);
    if (c < C) {
#pragma unroll 8
        for (int k = share; k < E; k += shares) {
            const float2 t = parts[(size_t)k * C + c];
            s.x += t.x; s.y += t.y;
        }
    }
    red[share][lane] = s;
    __syncthreads();
    if (share == 0 && c < C) {
        for (int k = 1; k < shares; ++k) { s.x += red[k][lane].x; s.y += red[k][lane].y; }
        if (dbeta) dbeta[c] = s.x;
        if (dgamma) dgamma[c] = s.y;
    }
}
__global__ __launch_bounds__(1024) void group_norm_params_kernel(const float2* parts, int E, int C, float* dgamma, float* dbeta) {
    __shared__ float2 red[64][16];
    join_params(parts, E, C, dgamma, dbeta, blockIdx.x, threadIdx.x >> 4, 64, threadIdx.x & 15, red);
}

// ---- split form
constexpr int kTileThreads = 512, kRows = 4;
struct Tile {
    long long n;
    int chunk, slab, r0, r1;             // the tile's positions
    __device__ Tile(const Geo& q, int n0, int chunks, int per, int P) {
        slab = blockIdx.x % q.slabs;
        const unsigned r = blockIdx.x / q.slabs;
        chunk = r % chunks;
        n = n0 + (int)(r / chunks);
        r0 = chunk * per;
        r1 = P - r0 < per ? P : r0 + per;                   // r0 + per may pass 2^31
    }
};
// kRows rows of a lane from r on: their masks, and what the ones that count hold (the others are not read: 65536 x 256 bf16 with half of
// the positions masked, forward and backward 74 us where all are read, 64 so).  A batch's masks are asked for a batch ahead.
template <bool MASK>
struct Rows {
    uint8_t mask[kRows];
    bool live[kRows];
    template <typename L>
    __device__ __forceinline__ void ask(const uint8_t* masks, const Geo& q, const L& l, const Tile& t, long long row0, int r) {
        if constexpr (MASK) {
#pragma unroll
            for (int k = 0; k < kRows; ++k) mask[k] = masks[row0 + min(r + l.slot + k * q.slots, t.r1 - 1)];
        }
    }
    template <typename L>
    __device__ __forceinline__ void take(const Geo& q, const L& l, const Tile& t, int r) {
#pragma unroll
        for (int k = 0; k < kRows; ++k) live[k] = l.on && r + l.slot + k * q.slots < t.r1 && (!MASK || mask[k] == 0);
    }
    template <typename T, int V, typename L>
    __device__ __forceinline__ void load(const void* x, long long sx, const Geo& q, const L& l, const Tile& t, long long row0, int r, Pack<T, V>* to) const {
        const T* const at = static_cast<const T*>(x) + l.c;
        if constexpr (MASK) {
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                to[k] = Pack<T, V>();
                if (live[k]) to[k] = load_pack<T, V>(at + (row0 + r + l.slot + k * q.slots) * sx);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kRows; ++k) to[k] = load_pack<T, V>(at + (row0 + min(r + l.slot + k * q.slots, t.r1 - 1)) * sx);
        }
    }
};

// part[(n G + g) E + e] = (values, mean, squared deviations), E = chunks x spg tiles of a group
template <typename T, int V, bool ONE, bool MASK>
__global__ __launch_bounds__(kTileThreads) void group_norm_tiles_kernel(const GroupNormArgs p, const Geo q, int n0, int chunks, int per, float4* part) {
    constexpr int PER = ONE ? 1 : V;
    __shared__ float red[kTileThreads * PER], mean_of[kTileThreads * Lane<V, ONE>::GV];
    __shared__ int cnt[1][1];
    const Tile t(q, n0, chunks, per, p.P);
    const Lane<V, ONE> l(q, p.C, p.G, t.slab, threadIdx.x);
    const long long row0 = t.n * p.P;
    float mean[V], m2[V], n = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) mean[v] = m2[v] = 0.0f;
    int mine[1] = {0};
    const int batch = q.slots * kRows;
    Rows<MASK> rows_at;
    const bool (&live)[kRows] = rows_at.live;
    rows_at.ask(p.mask, q, l, t, row0, t.r0);
    for (int r = t.r0; r < t.r1; r += batch) {
        Pack<T, V> x[kRows];
        rows_at.take(q, l, t, r);
        rows_at.template load<T, V>(p.x, p.sx, q, l, t, row0, r, x);
        if (r + batch < t.r1) rows_at.ask(p.mask, q, l, t, row0, r + batch);
        int here = 0;
#pragma unroll
        for (int k = 0; k < kRows; ++k) here += live[k];
        mine[0] += here;
        const float m = (float)here, inv = here > 0 ? 1.0f / m : 0.0f, share = here > 0 ? m / (n + m) : 0.0f, both = n * share;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float sum = 0.0f, sq = 0.0f;
#pragma unroll
            for (int k = 0; k < kRows; ++k) sum += live[k] ? get<T, V>(x[k], v) : 0.0f;
            sum *= inv;                                     // the mean of these rows
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                const float d = live[k] ? get<T, V>(x[k], v) - sum : 0.0f;
                sq = fmaf(d, d, sq);
            }
            const float d = sum - mean[v];
            mean[v] = here > 0 ? fmaf(d, share, mean[v]) : mean[v];
            m2[v] += here > 0 ? fmaf(d * d, both, sq) : 0.0f;
        }
        n += m;
    }
    int counted[1] = {t.r1 - t.r0};
    if (MASK) count_rows<false, 1>(cnt, 0, l.lt, l.lt % q.lanes == 0, mine, counted);
    const int rows = counted[0];
    const float M = (float)rows * (float)l.D, inv = rows > 0 ? 1.0f / M : 0.0f;
    float s[1][V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[0][v] = n * mean[v];
    group_sums<V, ONE, 1, false>(q, l, red, kTileThreads * PER, s, [&](int g, const float* u) { mean_of[g] = u[0] * inv; });
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float d = n > 0.0f ? mean[v] - mean_of[l.gr[ONE ? 0 : v]] : 0.0f;
        s[0][v] = fmaf(d * d, n, m2[v]);
    }
    const int E = chunks * q.spg;
    group_sums<V, ONE, 1, false>(q, l, red, kTileThreads * PER, s, [&](int g, const float* u) {
        part[((size_t)t.n * p.G + l.g0 + g) * E + (size_t)t.chunk * q.spg + t.slab % q.spg] = make_float4(M, mean_of[g], u[0], 0.0f);
    });
}

// The mean and rstd of a group from its E tiles, by `lanes` lanes (a power of two up to 64, neighbours) of which this is lane `l`.
__device__ __forceinline__ float2 join_tiles(const float4* tiles, int E, float eps, int l, int lanes) {
    float M = 0.0f, s = 0.0f, m2 = 0.0f;
#pragma unroll 8
    for (int e = l; e < E; e += lanes) { const float4 t = tiles[e]; M += t.x; s = fmaf(t.x, t.y, s); }
    for (int m = 1; m < lanes; m <<= 1) { M += __shfl_xor(M, m); s += __shfl_xor(s, m); }
    const float mean = M > 0.0f ? s / M : 0.0f;
#pragma unroll 8
    for (int e = l; e < E; e += lanes) {
        const float4 t = tiles[e];
        const float d = t.y - mean;
        m2 += fmaf(t.x * d, d, t.z);
    }
    for (int m = 1; m < lanes; m <<= 1) m2 += __shfl_xor(m2, m);
    return make_float2(mean, M > 0.0f ? 1.0f / sqrtf(m2 / M + eps) : 0.0f);
}
// One wavefront per item and group, where there are too many tiles for every workgroup of the apply kernel to join them by itself.
__global__ __launch_bounds__(64) void group_norm_join_kernel(const float4* part, int E, float eps, float* stats) {
    const float2 r = join_tiles(part + (size_t)blockIdx.x * E, E, eps, threadIdx.x, 64);
    if (threadIdx.x == 0) { stats[2 * (size_t)blockIdx.x] = r.x; stats[2 * (size_t)blockIdx.x + 1] = r.y; }
}

// part: the tiles, to be joined here, or null: the statistics are there.
template <typename T, int V, bool ONE, bool MASK, int ACT>
__global__ __launch_bounds__(kTileThreads) void group_norm_apply_kernel(const GroupNormArgs p, const Geo q, int n0, int chunks, int per, const float4* part) {
    constexpr int GV = Lane<V, ONE>::GV;
    __shared__ float2 joined[kTileThreads * GV];
    const Tile t(q, n0, chunks, per, p.P);
    const Lane<V, ONE> l(q, p.C, p.G, t.slab, threadIdx.x);
    const long long row0 = t.n * p.P;
    const int batch = q.slots * kRows, last = t.r0 + (t.r1 - 1 - t.r0) / batch * batch;
    Pack<T, V> x[kRows];
    Rows<MASK> rows_at;
    const bool (&live)[kRows] = rows_at.live;
    rows_at.ask(p.mask, q, l, t, row0, last);
    float gamma[V], beta[V], mean[GV], rstd[GV];
    load_params<V>(p, l.c, gamma, beta);
    rows_at.take(q, l, t, last);
    rows_at.template load<T, V>(p.x, p.sx, q, l, t, row0, last, x);
    if (last > t.r0) rows_at.ask(p.mask, q, l, t, row0, last - batch);
    if (part != nullptr) {
        const int E = chunks * q.spg;
        for (int g = l.lt / q.tpg; g < l.groups; g += kTileThreads / q.tpg) {
            const size_t at = (size_t)t.n * p.G + l.g0 + g;
            const float2 r = join_tiles(part + at * E, E, p.eps, l.lt & (q.tpg - 1), q.tpg);
            if ((l.lt & (q.tpg - 1)) == 0) {
                joined[g] = r;
                if (t.chunk == 0 && t.slab % q.spg == 0) { p.stats[2 * at] = r.x; p.stats[2 * at + 1] = r.y; }
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int v = 0; v < GV; ++v) {
        const float* st = p.stats + ((size_t)t.n * p.G + l.g0 + l.gr[v]) * 2;
        mean[v] = part != nullptr ? joined[l.gr[v]].x : st[0];
        rstd[v] = part != nullptr ? joined[l.gr[v]].y : st[1];
    }
    if (!l.on) return;
    for (int r = last; r >= t.r0; r -= batch) {
        if (r < last) {
            rows_at.take(q, l, t, r);
            rows_at.template load<T, V>(p.x, p.sx, q, l, t, row0, r, x);
            if (r > t.r0) rows_at.ask(p.mask, q, l, t, row0, r - batch);
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const int at = r + l.slot + k * q.slots;
            if (at < t.r1) {
                float y[V];
#pragma unroll
                for (int v = 0; v < V; ++v)
                    y[v] = live[k] ? act_of<ACT>(fmaf((get<T, V>(x[k], v) - mean[ONE ? 0 : v]) * rstd[ONE ? 0 : v], gamma[v], beta[v])) : 0.0f;
                store_own<T, V>(static_cast<T*>(p.y) + (row0 + at) * p.sy + l.c, l, y);
            }
        }
    }
}

// sums[n][chunk][C] = (sum dv, sum dv xh) of a tile; counts[n][chunk]: its rows that count
template <typename T, int V, bool ONE, bool MASK, int ACT>
__global__ __launch_bounds__(kTileThreads) void group_norm_sums_kernel(const GroupNormArgs p, const Geo q, int n0, int chunks, int per, float2* sums, float* counts) {
    constexpr int GV = Lane<V, ONE>::GV;
    __shared__ float red[2][kTileThreads * V];
    __shared__ int cnt[1][1];
    const Tile t(q, n0, chunks, per, p.P);
    const Lane<V, ONE> l(q, p.C, p.G, t.slab, threadIdx.x);
    const long long row0 = t.n * p.P;
    const int batch = q.slots * kRows;
    Pack<T, V> x[kRows], dy[kRows];
    Rows<MASK> rows_at;
    const bool (&live)[kRows] = rows_at.live;
    rows_at.ask(p.mask, q, l, t, row0, t.r0);
    float gamma[V], beta[V], mean[GV], rstd[GV], b[V], g[V];
    load_params<V>(p, l.c, gamma, beta);
    const auto load = [&](int r) {
        rows_at.take(q, l, t, r);
        rows_at.template load<T, V>(p.x, p.sx, q, l, t, row0, r, x);
        rows_at.template load<T, V>(p.dy, p.sdy, q, l, t, row0, r, dy);
        if (r + batch < t.r1) rows_at.ask(p.mask, q, l, t, row0, r + batch);
    };
    load(t.r0);
#pragma unroll
    for (int v = 0; v < GV; ++v) {
        const float* st = p.stats + ((size_t)t.n * p.G + l.g0 + l.gr[v]) * 2;
        mean[v] = st[0];
        rstd[v] = st[1];
    }
#pragma unroll
    for (int v = 0; v < V; ++v) b[v] = g[v] = 0.0f;
    int mine[1] = {0};
    for (int r = t.r0; r < t.r1; r += batch) {
        if (r > t.r0) load(r);
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            mine[0] += live[k];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float xh = (get<T, V>(x[k], v) - mean[ONE ? 0 : v]) * rstd[ONE ? 0 : v];
                const float dv = get<T, V>(dy[k], v) * act_slope<ACT>(fmaf(xh, gamma[v], beta[v]));
                b[v] += live[k] ? dv : 0.0f;
                g[v] += live[k] ? dv * xh : 0.0f;
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (l.own[v]) {
            red[0][l.slot * l.width + l.c + v - l.lo] = b[v];
            red[1][l.slot * l.width + l.c + v - l.lo] = g[v];
        }
    int counted[1] = {t.r1 - t.r0};
    if (MASK) count_rows<false, 1>(cnt, 0, l.lt, l.lt % q.lanes == 0, mine, counted);
    const int rows = counted[0];
    __syncthreads();
    for (int c = l.lt; c < l.width; c += kTileThreads) {
        float sb = 0.0f, sg = 0.0f;
        for (int s = 0; s < q.slots; ++s) { sb += red[0][s * l.width + c]; sg += red[1][s * l.width + c]; }
        sums[((size_t)t.n * chunks + t.chunk) * p.C + l.lo + c] = make_float2(sb, sg);
    }
    if (t.slab == 0 && threadIdx.x == 0) counts[(size_t)t.n * chunks + t.chunk] = (float)rows;
}

// Joins the tiles' sums of an item, for `gw` of its groups per workgroup (up to kNarrow channels a group, at least 16 channels, 128 bytes
// a row, together): chan[n][C], and coef[n][G] = (sum dv gamma, sum dv gamma xh) / M.  Where there is only one item, its sums are dbeta and dgamma.
constexpr int kJoinThreads = 1024, kNarrow = 64;
__device__ __forceinline__ float block_rows(const float* counts, size_t n, int chunks, float* rows_of) {
    float rows = 0.0f;
    for (int k = threadIdx.x; k < chunks; k += kJoinThreads) rows += counts[n * chunks + k];
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) rows += __shfl_xor(rows, m);
    if ((threadIdx.x & 63) == 0) rows_of[threadIdx.x >> 6] = rows;
    __syncthreads();
    rows = 0.0f;
    for (int k = 0; k < kJoinThreads / 64; ++k) rows += rows_of[k];
    return rows;
}
__global__ __launch_bounds__(kJoinThreads) void group_norm_chan_kernel(const float2* sums, const float* counts, int chunks, int n0, int C, int G, int D, int gw,
                                                                       const float* gamma, float2* chan, float2* coef, float* dgamma, float* dbeta) {
    __shared__ float2 red[kJoinThreads], total[kJoinThreads];
    __shared__ float rows_of[kJoinThreads / 64];
    const int tid = threadIdx.x, sets = (G + gw - 1) / gw, g0 = (blockIdx.x % sets) * gw;
    const size_t n = n0 + blockIdx.x / sets;
    const int groups = min(gw, G - g0), w = groups * D, lo = g0 * D, shares = kJoinThreads / w, c = tid % w, share = tid / w;
    float2 s = make_float2(0.0f, 0.0f);
    if (share < shares) {
#pragma unroll 8
        for (int k = share; k < chunks; k += shares) {
            const float2 t = sums[(n * chunks + k) * C + lo + c];
            s.x += t.x; s.y += t.y;
        }
    }
    red[tid] = s;
    const float rows = block_rows(counts, n, chunks, rows_of);          // behind its barrier red is there
    if (tid < w) {
        for (int k = 1; k < shares; ++k) { s.x += red[k * w + c].x; s.y += red[k * w + c].y; }
        if (chan) chan[n * C + lo + c] = s;
        if (dbeta) dbeta[lo + c] = s.x;
        if (dgamma) dgamma[lo + c] = s.y;
        const float gm = gamma ? gamma[lo + c] : 1.0f;
        total[tid] = make_float2(s.x * gm, s.y * gm);
    }
    __syncthreads();
    if (tid < groups) {
        const float inv = rows > 0.0f ? 1.0f / (rows * (float)D) : 0.0f;
        float2 t = make_float2(0.0f, 0.0f);
        for (int d = 0; d < D; ++d) { t.x += total[tid * D + d].x; t.y += total[tid * D + d].y; }
        coef[n * G + g0 + tid] = make_float2(t.x * inv, t.y * inv);
    }
}
// Wider groups: 16 channels of an item per workgroup, then one workgroup per item and group.
__global__ __launch_bounds__(kJoinThreads) void group_norm_wide_chan_kernel(const float2* sums, int chunks, int n0, int C, float2* chan, float* dgamma, float* dbeta) {
    __shared__ float2 red[64][16];
    const int cols = (C + 15) / 16, lane = threadIdx.x & 15, share = threadIdx.x >> 4, c = (blockIdx.x % cols) * 16 + lane;
    const size_t n = n0 + blockIdx.x / cols;
    float2 s = make_float2(0.0f, 0.0f);
    if (c < C) {
#pragma unroll 8
        for (int k = share; k < chunks; k += 64) {
            const float2 t = sums[(n * chunks + k) * C + c];
            s.x += t.x; s.y += t.y;
        }
    }
    red[share][lane] = s;
    __syncthreads();
    if (share == 0 && c < C) {
        for (int k = 1; k < 64; ++k) { s.x += red[k][lane].x; s.y += red[k][lane].y; }
        chan[n * C + c] = s;
        if (dbeta) dbeta[c] = s.x;
        if (dgamma) dgamma[c] = s.y;
    }
}
__global__ __launch_bounds__(kJoinThreads) void group_norm_wide_coef_kernel(const float2* chan, const float* counts, int chunks, int n0, int G, int D, const float* gamma,
                                                                            float2* coef) {
    __shared__ float2 red[kJoinThreads / 64];
    __shared__ float rows_of[kJoinThreads / 64];
    const int tid = threadIdx.x, g = blockIdx.x % G;
    const size_t n = n0 + blockIdx.x / G;
    float2 t = make_float2(0.0f, 0.0f);
    for (int d = tid; d < D; d += kJoinThreads) {
        const float2 c = chan[(n * G + g) * D + d];
        const float gm = gamma ? gamma[(size_t)g * D + d] : 1.0f;
        t.x = fmaf(c.x, gm, t.x);
        t.y = fmaf(c.y, gm, t.y);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) { t.x += __shfl_xor(t.x, m); t.y += __shfl_xor(t.y, m); }
    if ((tid & 63) == 0) red[tid >> 6] = t;
    const float rows = block_rows(counts, n, chunks, rows_of);
    if (tid == 0) {
        const float inv = rows > 0.0f ? 1.0f / (rows * (float)D) : 0.0f;
        for (int k = 1; k < kJoinThreads / 64; ++k) { t.x += red[k].x; t.y += red[k].y; }
        coef[n * G + g] = make_float2(t.x * inv, t.y * inv);
    }
}

// The workgroups behind the tiles' join the items' sums to dbeta and dgamma.
template <typename T, int V, bool ONE, bool MASK, int ACT>
__global__ __launch_bounds__(kTileThreads) void group_norm_grad_kernel(const GroupNormArgs p, const Geo q, int n0, int chunks, int per, const float2* coef, unsigned tiles,
                                                                       const float2* chan) {
    constexpr int GV = Lane<V, ONE>::GV;
    __shared__ float2 red[kTileThreads / 16][16];
    if (blockIdx.x >= tiles) {
        join_params(chan, p.N, p.C, p.dgamma, p.dbeta, blockIdx.x - tiles, threadIdx.x >> 4, kTileThreads / 16, threadIdx.x & 15, red);
        return;
    }
    const Tile t(q, n0, chunks, per, p.P);
    const Lane<V, ONE> l(q, p.C, p.G, t.slab, threadIdx.x);
    if (!l.on) return;
    const long long row0 = t.n * p.P;
    const int batch = q.slots * kRows, last = t.r0 + (t.r1 - 1 - t.r0) / batch * batch;
    Pack<T, V> x[kRows], dy[kRows];
    Rows<MASK> rows_at;
    const bool (&live)[kRows] = rows_at.live;
    rows_at.ask(p.mask, q, l, t, row0, last);
    float gamma[V], beta[V], mean[GV], rstd[GV], s1[GV], s2[GV];
    load_params<V>(p, l.c, gamma, beta);
    const auto load = [&](int r) {
        rows_at.take(q, l, t, r);
        rows_at.template load<T, V>(p.x, p.sx, q, l, t, row0, r, x);
        rows_at.template load<T, V>(p.dy, p.sdy, q, l, t, row0, r, dy);
        if (r > t.r0) rows_at.ask(p.mask, q, l, t, row0, r - batch);
    };
    load(last);
#pragma unroll
    for (int v = 0; v < GV; ++v) {
        const size_t at = (size_t)t.n * p.G + l.g0 + l.gr[v];
        mean[v] = p.stats[2 * at];
        rstd[v] = p.stats[2 * at + 1];
        s1[v] = coef[at].x;
        s2[v] = coef[at].y;
    }
    for (int r = last; r >= t.r0; r -= batch) {
        if (r < last) load(r);
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const int at = r + l.slot + k * q.slots;
            if (at < t.r1) {
                float dx[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int w = ONE ? 0 : v;
                    const float xh = (get<T, V>(x[k], v) - mean[w]) * rstd[w];
                    const float dv = get<T, V>(dy[k], v) * act_slope<ACT>(fmaf(xh, gamma[v], beta[v]));
                    dx[v] = live[k] ? rstd[w] * (fmaf(dv, gamma[v], -s1[w]) - xh * s2[w]) : 0.0f;
                }
                store_own<T, V>(static_cast<T*>(p.dx) + (row0 + at) * p.sdx + l.c, l, dx);
            }
        }
    }
}

// ---- shapes
constexpr int kMaxWgs = 2048;            // workgroups of the held form: eight per compute unit
constexpr int kTileWgs = 512;            // tiles of the split form, at least, where there are rows enough: two per compute unit
enum { FORM_WAVE = 0, FORM_GROUP = 1, FORM_SPLIT = 2, FORM_TOKENS = 3 };
constexpr int kHeldRows = 8, kWaveThreads = 256, kGroupThreads = 512;
constexpr int kItems = 4, kItemsBwd = 2;                   // items of a workgroup that takes several at once, one row of a lane each
constexpr int kTokenChannels = 2048;                       // of a group, at most: 32 a lane
constexpr int kTokenWgs = 1024;                            // four workgroups of single rows per compute unit

int floor_pow2(int v) {
    int r = 1;
    while (2 * r <= v) r *= 2;
    return r;
}
struct NormPlan {
    int form, V, K;                      // K: rows of a lane
    bool one;                            // V divides the channels of a group
    Geo q;
    long long teams, parts;              // held forms; parts of the parameters' sums
    int chunks, per;                     // split form: tiles of an item, positions of a tile
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
        q->width = ((D + q->spg - 1) / q->spg + V - 1) / V * V;
        q->spg = (D + q->width - 1) / q->width;
        q->gps = 1;
        q->slabs = d->G * q->spg;
        q->D = q->width;
    }
    q->lanes = (q->width + V - 1) / V;
    if (q->lanes > ts) return false;
    q->slots = ts / q->lanes;
    q->per_lanes = 1.0f / (float)q->lanes;
    q->per_D = 1.0f / (float)q->D;
    q->tpg = floor_pow2(ts / (q->gps < ts ? q->gps : ts));
    if (q->tpg > 64) q->tpg = 64;
    return true;
}
NormPlan plan_of(const scan2d_group_norm_desc* d, bool backward) {
    NormPlan n = {};
    n.V = d->C >= 4 ? 4 : 1;
    const int D = d->C / d->G;
    n.one = D % n.V == 0;
    const auto held = [&](int form, long long most_teams) {
        n.form = form;
        // one row of a lane: a workgroup's only, since the fewest lanes of a wavefront that hold several positions hold them in several rows
        n.K = form == FORM_GROUP && n.q.slots >= d->P && n.V > 1 ? 1 : kHeldRows;
        most_teams = most_teams < n.q.slabs ? n.q.slabs : most_teams / n.q.slabs * n.q.slabs;
        n.teams = (long long)d->N * n.q.slabs;
        if (n.teams > most_teams) n.teams = most_teams;
        n.parts = form == FORM_WAVE && n.q.slabs == 1 ? (n.teams * n.q.ts + kWaveThreads - 1) / kWaveThreads : n.teams / n.q.slabs;
        return n;
    };
    // single rows: the widest loads, and as many groups to a wavefront as it has lanes for
    const int TV = d->dtype == SCAN2D_BF16 && D >= 8 ? 8 : 4;
    if (d->P == 1 && d->C >= 4 && D <= kTokenChannels) {
        n.form = FORM_TOKENS;
        n.V = TV;
        n.K = 1;
        n.one = D % TV == 0;
        n.q = Geo();
        n.q.D = D;
        n.q.lanes = 1;
        while (n.q.lanes < 64 && n.q.lanes * TV < D) n.q.lanes *= 2;
        n.q.ts = n.q.lanes;
        while (n.q.ts < 64 && n.q.ts / n.q.lanes < d->G) n.q.ts *= 2;
        n.q.gps = n.q.ts / n.q.lanes;
        n.q.slabs = (d->G + n.q.gps - 1) / n.q.gps;
        n.q.slots = n.q.spg = 1;
        long long most = (long long)kTokenWgs * (kTokenThreads / n.q.ts);
        n.teams = (long long)d->N * n.q.slabs;
        // backward: at least four items a team while that leaves every SIMD a wavefront, for fewer parts of the parameters'
        // sums (4096 tokens x 600 fp32 18.8 us without, 15.8 with; 300 x 2048 11.7 and 9.5)
        if (backward && most > n.teams / 4) most = n.teams / 4 > 1024 ? n.teams / 4 : 1024;
        most = most < n.q.slabs ? n.q.slabs : most / n.q.slabs * n.q.slabs;
        if (n.teams > most) n.teams = most;
        n.parts = n.q.slabs == 1 ? (n.teams * n.q.ts + kTokenThreads - 1) / kTokenThreads : n.teams / n.q.slabs;
        return n;
    }
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
    // whole rows, or narrower slabs where they keep more lanes busy: 1.2 times (9 x 3000 x 1280 in 32 groups, bf16: 320 of 512 lanes 54 and 103 us, 480 41 and
    // 80), 1.5 times where that cuts a group, whose parts are joined and whose rows share cache lines with another workgroup's (3 x 17280 x 516 in two: 63 and
    // 83 us cut, 41 and 59 whole)
    (void)fill_geo(d, n.V, kTileThreads, kTileThreads * n.V, false, &n.q);
    for (int most = kTileThreads * n.V / 2; most >= 128; most /= 2) {
        Geo q;
        if (fill_geo(d, n.V, kTileThreads, most, false, &q) && q.slots * q.width * 10 >= n.q.slots * n.q.width * (q.spg > n.q.spg ? 15 : 12)) n.q = q;
    }
    const long long batch = (long long)n.q.slots * kRows, batches = (d->P + batch - 1) / batch, each = (long long)d->N * n.q.slabs;
    long long chunks = (kTileWgs + each - 1) / each;
    if (chunks > batches) chunks = batches;
    const long long per = (batches + chunks - 1) / chunks * batch;
    n.per = (int)(per < d->P ? per : d->P);
    n.chunks = (int)((d->P + n.per - 1) / n.per);
    return n;
}
// Whether every workgroup of the apply kernel joins the tiles of its groups by itself: up to 2048 of them, eight to a lane, while
// a kernel of its own costs about 4 us.
bool join_in_apply(const NormPlan& n) { return (long long)n.chunks * n.q.spg * n.q.gps <= 2048; }
size_t up(size_t n) { return (n + 255) / 256 * 256; }
int launched() { return hipGetLastError() == hipSuccess ? SCAN2D_OK : SCAN2D_ERR_LAUNCH_FAILED; }
// `each` workgroups for each of N items: launch(first item, workgroups) for as many items at a time as stay below 2^31 threads, half of what a
// launch may hold, so that the gradient's further workgroups fit beside them.  (16384 tokens of 4096 channels in one group are joined by 2^32
// threads.  Workgroups that go on to further items instead cost shapes of any size: 32 x 3136 x 192 backward 43.8 -> 46.3 us.)
template <typename Launch>
void by_items(int N, int each, int threads, Launch launch) {
    const long long most = (1LL << 31) / ((long long)threads * each);
    for (long long n = 0; n < N; n += most) launch((int)n, (unsigned)((N - n < most ? N - n : most) * each));
}

template <typename T, int V, bool ONE, int ACT>
int fwd_held(const GroupNormArgs& a, const NormPlan& n, hipStream_t stream) {
    using Kernel = void (*)(const GroupNormArgs, const Geo, int);
    const bool wave = n.form == FORM_WAVE;
    Kernel k = wave ? group_norm_fwd_kernel<T, V, ONE, kHeldRows, 1, kWaveThreads, true, ACT> : group_norm_fwd_kernel<T, V, ONE, kHeldRows, 1, kGroupThreads, false, ACT>;
    if constexpr (V > 1)
        if (n.K == 1) {
            // one item per team: none that it could take besides
            if (n.teams >= (long long)a.N * n.q.slabs) k = group_norm_fwd_kernel<T, V, ONE, 1, 1, kGroupThreads, false, ACT>;
            else k = group_norm_fwd_kernel<T, V, ONE, 1, kItems, kGroupThreads, false, ACT>;
        }
    const long long blocks = wave ? (n.teams * n.q.ts + kWaveThreads - 1) / kWaveThreads : n.teams;
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(wave ? kWaveThreads : kGroupThreads), 0, stream, a, n.q, (int)n.teams);
    return launched();
}
template <typename T, int V, bool ONE, int ACT, bool MASK>
int fwd_split(const GroupNormArgs& a, const NormPlan& n, hipStream_t stream) {
    const int each = n.chunks * n.q.slabs;
    const bool in_apply = join_in_apply(n);
    float4* part = static_cast<float4*>(a.workspace);
    by_items(a.N, each, kTileThreads, [&](int n0, unsigned wgs) {
        hipLaunchKernelGGL((group_norm_tiles_kernel<T, V, ONE, MASK>), dim3(wgs), dim3(kTileThreads), 0, stream, a, n.q, n0, n.chunks, n.per, part);
    });
    if (!in_apply)                                          // several tiles an item: fewer than 512 slabs in all, of up to 2048 groups each
        hipLaunchKernelGGL(group_norm_join_kernel, dim3((unsigned)(a.N * a.G)), dim3(64), 0, stream, part, n.chunks * n.q.spg, a.eps, a.stats);
    by_items(a.N, each, kTileThreads, [&](int n0, unsigned wgs) {
        hipLaunchKernelGGL((group_norm_apply_kernel<T, V, ONE, MASK, ACT>), dim3(wgs), dim3(kTileThreads), 0, stream, a, n.q, n0, n.chunks, n.per,
                           in_apply ? part : nullptr);
    });
    return launched();
}
template <typename T, int V, bool ONE, int ACT>
int bwd_held(const GroupNormArgs& a, const NormPlan& n, hipStream_t stream) {
    const bool params = a.dgamma != nullptr || a.dbeta != nullptr;
    const unsigned cols = (a.C + 15) / 16;
    using Kernel = void (*)(const GroupNormArgs, const Geo, int, float2*);
    const bool wave = n.form == FORM_WAVE;
    float2* parts = params ? static_cast<float2*>(a.workspace) : nullptr;
    Kernel k = wave ? group_norm_bwd_kernel<T, V, ONE, kHeldRows, 1, kWaveThreads, true, ACT> : group_norm_bwd_kernel<T, V, ONE, kHeldRows, 1, kGroupThreads, false, ACT>;
    if constexpr (V > 1)
        if (n.K == 1) {
            if (n.teams >= (long long)a.N * n.q.slabs) k = group_norm_bwd_kernel<T, V, ONE, 1, 1, kGroupThreads, false, ACT>;
            else k = group_norm_bwd_kernel<T, V, ONE, 1, kItemsBwd, kGroupThreads, false, ACT>;
        }
    const long long blocks = wave ? (n.teams * n.q.ts + kWaveThreads - 1) / kWaveThreads : n.teams;
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(wave ? kWaveThreads : kGroupThreads), 0, stream, a, n.q, (int)n.teams, parts);
    if (params) hipLaunchKernelGGL(group_norm_params_kernel, dim3(cols), dim3(1024), 0, stream, parts, (int)n.parts, a.C, a.dgamma, a.dbeta);
    return launched();
}
template <typename T, int V, bool ONE, int ACT, bool MASK>
int bwd_split(const GroupNormArgs& a, const NormPlan& n, hipStream_t stream) {
    const bool params = a.dgamma != nullptr || a.dbeta != nullptr;
    const unsigned cols = (a.C + 15) / 16;
    const bool narrow = a.D <= kNarrow;
    const int gw = a.D >= 16 ? 1 : (16 + a.D - 1) / a.D, sets = (a.G + gw - 1) / gw, each = n.chunks * n.q.slabs;
    char* w = static_cast<char*>(a.workspace);
    const size_t items = (size_t)a.N * n.chunks;
    float2* sums = reinterpret_cast<float2*>(w);
    w += up(items * a.C * sizeof(float2));
    float* counts = reinterpret_cast<float*>(w);
    w += up(items * sizeof(float));
    float2* chan = reinterpret_cast<float2*>(w);
    w += up((size_t)a.N * a.C * sizeof(float2));
    float2* coef = reinterpret_cast<float2*>(w);
    const bool several = params && a.N > 1;
    by_items(a.N, each, kTileThreads, [&](int n0, unsigned wgs) {
        hipLaunchKernelGGL((group_norm_sums_kernel<T, V, ONE, MASK, ACT>), dim3(wgs), dim3(kTileThreads), 0, stream, a, n.q, n0, n.chunks, n.per, sums, counts);
    });
    float *const dgamma = several ? nullptr : a.dgamma, *const dbeta = several ? nullptr : a.dbeta;
    if (narrow) {
        by_items(a.N, sets, kJoinThreads, [&](int n0, unsigned wgs) {
            hipLaunchKernelGGL(group_norm_chan_kernel, dim3(wgs), dim3(kJoinThreads), 0, stream, sums, counts, n.chunks, n0, a.C, a.G, a.D, gw, a.gamma,
                               several ? chan : nullptr, coef, dgamma, dbeta);
        });
    } else {
        by_items(a.N, cols, kJoinThreads, [&](int n0, unsigned wgs) {
            hipLaunchKernelGGL(group_norm_wide_chan_kernel, dim3(wgs), dim3(kJoinThreads), 0, stream, sums, n.chunks, n0, a.C, chan, dgamma, dbeta);
        });
        by_items(a.N, a.G, kJoinThreads, [&](int n0, unsigned wgs) {
            hipLaunchKernelGGL(group_norm_wide_coef_kernel, dim3(wgs), dim3(kJoinThreads), 0, stream, chan, counts, n.chunks, n0, a.G, a.D, a.gamma, coef);
        });
    }
    by_items(a.N, each, kTileThreads, [&](int n0, unsigned wgs) {
        hipLaunchKernelGGL((group_norm_grad_kernel<T, V, ONE, MASK, ACT>), dim3(wgs + (several && n0 == 0 ? cols : 0)), dim3(kTileThreads), 0, stream, a, n.q, n0,
                           n.chunks, n.per, coef, wgs, chan);
    });
    return launched();
}

// single rows: J times V channels a lane
template <typename T, int V, int J, bool ONE, int ACT>
int tokens(const GroupNormArgs& a, const NormPlan& n, bool backward, hipStream_t stream) {
    const dim3 blocks((unsigned)((n.teams * n.q.ts + kTokenThreads - 1) / kTokenThreads));
    if (!backward) {
        hipLaunchKernelGGL((group_norm_tokens_kernel<T, V, J, ONE, J == 1 ? 16 / V : 1, ACT>), blocks, dim3(kTokenThreads), 0, stream, a, n.q, (int)n.teams);
        return launched();
    }
    const bool params = a.dgamma != nullptr || a.dbeta != nullptr;
    float2* parts = params ? static_cast<float2*>(a.workspace) : nullptr;
    hipLaunchKernelGGL((group_norm_tokens_bwd_kernel<T, V, J, ONE, J == 1 && V == 4 ? 2 : 1, ACT>), blocks, dim3(kTokenThreads), 0, stream, a, n.q, (int)n.teams, parts);
    if (params) hipLaunchKernelGGL(group_norm_params_kernel, dim3((a.C + 15) / 16), dim3(1024), 0, stream, parts, (int)n.parts, a.C, a.dgamma, a.dbeta);
    return launched();
}
template <typename T, int V, bool ONE, int ACT>
int run(const GroupNormArgs& a, const NormPlan& n, bool backward, hipStream_t stream) {
    if (n.form == FORM_TOKENS) {
        if constexpr (V > 1) {
            const int times = (a.D + 64 * V - 1) / (64 * V);
            if (times == 1) return tokens<T, V, 1, ONE, ACT>(a, n, backward, stream);
            if constexpr (V * Elem<T>::kBytes == 16) {      // 16 bytes a load
                if (times == 2) return tokens<T, V, 2, ONE, ACT>(a, n, backward, stream);
                if (times <= 4) return tokens<T, V, 4, ONE, ACT>(a, n, backward, stream);
                if constexpr (V == 4) return tokens<T, V, 8, ONE, ACT>(a, n, backward, stream);
            }
        }
    } else if constexpr (V <= 4) {                          // eight channels of a lane: single rows only
        if (n.form != FORM_SPLIT) return backward ? bwd_held<T, V, ONE, ACT>(a, n, stream) : fwd_held<T, V, ONE, ACT>(a, n, stream);
        if (a.mask != nullptr) return backward ? bwd_split<T, V, ONE, ACT, true>(a, n, stream) : fwd_split<T, V, ONE, ACT, true>(a, n, stream);
        return backward ? bwd_split<T, V, ONE, ACT, false>(a, n, stream) : fwd_split<T, V, ONE, ACT, false>(a, n, stream);
    }
    return SCAN2D_ERR_BAD_SHAPE;
}

template <typename T, int V, bool ONE>
int by_act(const GroupNormArgs& a, const NormPlan& n, bool backward, hipStream_t stream) {
    (void)hipGetLastError();
    switch (a.act) {
        case SCAN2D_ACT_SILU: return run<T, V, ONE, SCAN2D_ACT_SILU>(a, n, backward, stream);
        case SCAN2D_ACT_GELU: return run<T, V, ONE, SCAN2D_ACT_GELU>(a, n, backward, stream);
        default: return run<T, V, ONE, SCAN2D_ACT_NONE>(a, n, backward, stream);
    }
}
template <typename T>
int by_lane(const GroupNormArgs& a, const NormPlan& n, bool backward, hipStream_t stream) {
    if (n.V == 1) return by_act<T, 1, true>(a, n, backward, stream);
    if constexpr (sizeof(T) == 2)
        if (n.V == 8) return n.one ? by_act<T, 8, true>(a, n, backward, stream) : by_act<T, 8, false>(a, n, backward, stream);
    return n.one ? by_act<T, 4, true>(a, n, backward, stream) : by_act<T, 4, false>(a, n, backward, stream);
}
int dispatch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, bool backward, hipStream_t stream) {
    const NormPlan n = plan_of(d, backward);
    return d->dtype == SCAN2D_BF16 ? by_lane<bf16_t>(a, n, backward, stream) : by_lane<float>(a, n, backward, stream);
}

}  // namespace

size_t group_norm_workspace_bytes(const scan2d_group_norm_desc* d, int pass) {
    const NormPlan n = plan_of(d, pass == SCAN2D_PASS_BWD);
    if (n.form != FORM_SPLIT) return pass == SCAN2D_PASS_BWD ? (size_t)n.parts * d->C * sizeof(float2) : 0;
    const size_t items = (size_t)d->N * n.chunks;
    if (pass == SCAN2D_PASS_FWD) return items * n.q.spg * d->G * sizeof(float4);
    return up(items * d->C * sizeof(float2)) + up(items * sizeof(float)) + up((size_t)d->N * d->C * sizeof(float2)) + (size_t)d->N * d->G * sizeof(float2);
}
int group_norm_fwd_launch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, hipStream_t stream) { return dispatch(d, a, false, stream); }
int group_norm_bwd_launch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, hipStream_t stream) { return dispatch(d, a, true, stream); }

}  // namespace scan2d
