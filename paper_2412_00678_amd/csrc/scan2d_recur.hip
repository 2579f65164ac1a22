// The gated linear recurrence on channels-last rows (include/scan2d_seq.h): per channel
//     a_t = exp(-scale softplus(lam) sigmoid(r_t)),  u_t = sqrt(1 - a_t^2) sigmoid(i_t) x_t,  h_t = a_t h_{t-1} + u_t.
//
// Bound: HBM.  Forward 3 reads and 1 write per element, backward 4 and 3, with six elementary functions per element that
// take about as long as the bytes do in bf16; so every row is read once, and the scan over T is done in one pass.
//
// A sequence of maps h -> A h + S composes to one of the same form: (A1, S1) then (A2, S2) is (A1 A2, A2 S1 + S2).  A
// workgroup takes a chunk of TW x NW consecutive rows (of whatever sequences) x 64 V channels: a wavefront has TW
// rows, a lane V neighbouring channels of them, all in registers.  Each lane forms the map of its rows, the wavefronts' maps
// meet in LDS, and the chunk's map (A, S) goes to the workspace, where the chunks behind it pick it up; the last chunk of a
// team of kTeam writes the team's map instead, and the last of a group of kTeams teams the state behind the group.  The state in front
// of a chunk is the one behind the group before, carried through the maps of the teams and chunks in between, always in this order: the
// same bits every time.  With the state in hand the lane runs its rows once more from registers and writes them.  The first row of a sequence enters as A = -0, S = a h0 + u, rows of
// no sequence as A = -0, S = 0, so sequences of any lengths share chunks; the sign marks a map that does not look at
// what comes before it (0 times a NaN would), where a product of decays that underflows is +0.
// The backward pass is the same scan from the last row to the first for e_t = a_t (dh_t + e_{t+1}); it rebuilds the states from the ones in front of each chunk, which the forward saved.
//
// Measured (a copy reaches 5.2 TB/s): 65536 x 2048 bf16 forward 255 us, 4.2 TB/s of its bytes; 16384 x 2048 bf16 forward 71 us, 3.8, backward
// 136 us, 3.5; 5003 x 771 fp32 21 and 39 us; 37 x 256 bf16 6 and 11 us, one chunk's latency; clearing the workspace 2 us of each, the sum
// for dlam 4 of the backward.
//
// No wait without an end: a workgroup draws its chunk from its column's counter, so every chunk with a smaller number belongs to
// a workgroup that is already running; a chunk's map is written before its workgroup waits for anything, the map of a team and the state
// behind a group wait for chunks with smaller numbers only.  A word in the workspace holds value and flag together (one 64-bit
// store), set to "not written" by a kernel in front of the pass.  A workspace that two calls share at the same time breaks
// all that; for them a wait ends after kSpins looks all the same, with NaN for what did not come, and chunks past the last are none.
#include "scan2d_seq.hpp"

#include "scan2d_block.hpp"
#include "scan2d_common.hpp"

namespace scan2d {
namespace {

constexpr int kTeam = 4, kTeams = 8, kGroup = kTeam * kTeams;     // chunks of a team, teams of a group
constexpr int kSavedRows = 96;           // rows between the states that the forward saves: a chunk of the backward

__device__ __forceinline__ float sigmoid(float t) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-t * kLog2e)); }

// Per channel: scale * softplus(lam) in powers of two, and sigmoid(lam) / softplus(lam) (-> 1 for lam -> -inf).
__device__ __forceinline__ float decay_of(float lam, float scale) { return scale * (lam > 20.0f ? lam : log1pf(expf(lam))) * kLog2e; }
__device__ __forceinline__ float decay_slope(float lam) { return lam < -15.0f ? 1.0f : 1.0f / ((1.0f + expf(-lam)) * (lam > 20.0f ? lam : log1pf(expf(lam)))); }

// 1 - 2^(2y) for y <= 0 without the cancellation near 0, a = 2^y: -y p(y), p the Chebyshev fit of degree 5 to
// (1 - 2^(2y)) / -y on [-0.5, 0] (off by 2.5e-8 with the constants as rounded to fp32); beyond, 1 - a^2 >= 0.5 loses nothing.
__device__ __forceinline__ float one_minus_square(float y, float a) {
    float p = fmaf(y, 0.007358775474131107f, 0.0413372628390789f);
    p = fmaf(y, p, 0.15355470776557922f);
    p = fmaf(y, p, 0.4439942240715027f);
    p = fmaf(y, p, 0.9609044194221497f);
    p = fmaf(y, p, 1.3862943649291992f);
    return y > -0.5f ? -y * p : fmaf(-a, a, 1.0f);
}

// V neighbouring elements as loaded.  The row's address is the same for the whole wavefront (scalar registers), the lane's
// offset in it 32 bits.
typedef __attribute__((address_space(1))) const char* gconst;
typedef __attribute__((address_space(1))) char* gmut;
typedef uint16_t u16_a1 __attribute__((aligned(2)));
template <typename T, int V> struct Pack { uint32_t w[V * Elem<T>::kBytes <= 4 ? 1 : V * Elem<T>::kBytes / 4]; };
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(uint64_t row, uint32_t offset) {
    const gconst p = (gconst)row + offset;
    Pack<T, V> r;
    if constexpr (V * Elem<T>::kBytes == 2) r.w[0] = *reinterpret_cast<__attribute__((address_space(1))) const u16_a1*>(p);
    else if constexpr (V * Elem<T>::kBytes == 4) r.w[0] = *reinterpret_cast<__attribute__((address_space(1))) const u32_a1*>(p);
    else {
        static_assert(V * Elem<T>::kBytes == 8, "two dwords");
        const u32x2_a1 v = *reinterpret_cast<__attribute__((address_space(1))) const u32x2_a1*>(p);
        r.w[0] = v.x; r.w[1] = v.y;
    }
    return r;
}
template <typename T, int V>
__device__ __forceinline__ float get(const Pack<T, V>& r, int j) { return get_elem<T, V>(r.w, j); }
// Outputs go past the L2's keeping (non-temporal): nothing reads them again here, and rows that are still to be read stay
// (5003 x 771 fp32 backward 44.9 us without, 40.6 with; 16384 x 2048 bf16 153 and 142).
template <typename T, int V>
__device__ __forceinline__ void store_pack(uint64_t row, uint32_t offset, const float* v) {
    const gmut p = (gmut)row + offset;
    if constexpr (V * Elem<T>::kBytes == 2) {
        __builtin_nontemporal_store((uint16_t)f32_to_bf16_bits(v[0]), reinterpret_cast<__attribute__((address_space(1))) u16_a1*>(p));
    } else if constexpr (V * Elem<T>::kBytes == 4) {
        uint32_t w;
        if constexpr (V == 1) w = __float_as_uint(v[0]);
        else w = pack_bf16x2(v[0], v[1]);
        __builtin_nontemporal_store(w, reinterpret_cast<__attribute__((address_space(1))) u32_a1*>(p));
    } else {
        u32x2_a1 w;
        w.x = __float_as_uint(v[0]); w.y = __float_as_uint(v[1]);
        __builtin_nontemporal_store(w, reinterpret_cast<__attribute__((address_space(1))) u32x2_a1*>(p));
    }
}

// ---- maps h -> A h + S
constexpr float kCut = -0.0f;            // A of a map that forgets h
__device__ __forceinline__ bool is_cut(float A) { return (int32_t)__float_as_uint(A) < 0; }
__device__ __forceinline__ float apply(float A, float h, float S) { return is_cut(A) ? S : fmaf(A, h, S); }
__device__ __forceinline__ float compose(float first, float then) { return is_cut(then) ? then : first * then; }

// ---- the rows' sequences
struct Span { int lo, hi; };
__device__ __forceinline__ Span span_of(const RecurArgs& p, int s) {
    if (p.offsets) return {min(max(p.offsets[s], 0), p.T), min(max(p.offsets[s + 1], 0), p.T)};
    const int lo = s * p.per;
    return {lo, lo + (p.lengths ? min(max(p.lengths[s], 0), p.per) : p.per)};
}
// What the TW rows of a wavefront from t0 on are, a bit for each, and each row's sequence in lane (row - t0).
struct RowBits {
    uint64_t first, last, inside;
    int seq;
    bool plain;                          // rows of one sequence, neither its first nor its last among them
    __device__ __forceinline__ int seq_of(int j) const { return __builtin_amdgcn_readlane(seq, j); }
};
// Finds a row's sequence, which is the number of ends offsets[1..S] at or before it: 64 of them at a time, evenly spaced
// over what is left.  The first 64 are asked for before the row is known; for up to 64 sequences they are all.
struct SeqSearch {
    int step, end, begin;                // lane l has the last of the l-th `step` ends
    __device__ __forceinline__ explicit SeqSearch(const RecurArgs& p) {
        const int lane = threadIdx.x & 63;
        step = (p.S + 63) / 64;
        end = 0x7fffffff;
        begin = 0;
        if (p.offsets) {
            const int at = (lane + 1) * step - 1;
            if (at < p.S) end = p.offsets[at + 1];
            begin = p.offsets[0];
        }
    }
    __device__ __forceinline__ int at(const RecurArgs& p, int t) const {
        // ends ascend, so the lanes that are past come first; where they do not, this is some number of them
        int lo = __builtin_popcountll(__ballot(end <= t)) * step, n = min(step - 1, max(p.S - lo, 0));
        while (n > 0) {
            const int part = (n + 63) / 64, k = lo + ((int)(threadIdx.x & 63) + 1) * part - 1;
            const int full = __builtin_popcountll(__ballot(k < lo + n && p.offsets[min(k, p.S - 1) + 1] <= t));
            lo += full * part;
            n = min(part - 1, max(p.S - lo, 0));
        }
        return min(lo, p.S);
    }
};
template <int TW>
__device__ __forceinline__ RowBits row_bits(const RecurArgs& p, const SeqSearch& search, int t0) {
    const int lane = threadIdx.x & 63, t = t0 + lane;
    RowBits r;
    int s0 = 0, lo, hi;
    if (p.offsets) {
        s0 = search.at(p, t0);
        if (p.S <= 64) {
            hi = s0 < p.S ? __builtin_amdgcn_readlane(search.end, min(s0, 63)) : -1;
            lo = s0 > 0 ? __builtin_amdgcn_readlane(search.end, s0 - 1) : search.begin;
        } else {
            hi = s0 < p.S ? p.offsets[s0 + 1] : -1;
            lo = p.offsets[s0];
        }
        lo = max(lo, 0);
        hi = min(hi, p.T);
    } else {
        s0 = p.per > 0 ? t0 / p.per : 0;
        lo = s0 * p.per;
        hi = s0 < p.S ? lo + (p.lengths ? min(max(p.lengths[s0], 0), p.per) : p.per) : -1;
    }
    r.plain = lo < t0 && t0 + TW < hi;
    r.seq = s0;
    r.first = r.last = 0;
    r.inside = ~0ull;
    if (!r.plain) {
        int s = s0;                                         // this lane's row's sequence, and its rows
        Span w = {lo, hi};
        if (p.offsets) {
            // 64 ends at a time from the first row's on, in the lanes; the rows' lanes go past them one after the other
            for (int base = p.S <= 64 ? 0 : s0; base < p.S; base += 64) {
                const int end = p.S <= 64 ? search.end : base + lane < p.S ? p.offsets[base + lane + 1] : 0x7fffffff;
                const int last = min(p.S - base, 64);
                int k = max(s0 - base, 0);
                for (; k < last; ++k) {
                    const int e = __builtin_amdgcn_readlane(end, k);
                    if (e >= t0 + TW) break;                // it ends behind the last row
                    if (t >= e) {
                        s = base + k + 1;
                        w.lo = e;
                        w.hi = -1;                          // known once the next end is
                    } else if (s == base + k) {
                        w.hi = e;
                    }
                }
                if (k < last) {
                    const int e = __builtin_amdgcn_readlane(end, k);
                    if (s == base + k) w.hi = e;
                    break;
                }
            }
            w.lo = max(w.lo, 0);
            w.hi = min(w.hi, p.T);
        } else if (p.per > 0) {
            s = t / p.per;
            if (s < p.S) w = span_of(p, s);
        }
        const bool inside = lane < TW && t < p.T && s < p.S && t >= w.lo && t < w.hi;
        r.seq = s;
        r.first = __ballot(inside && t == w.lo);
        r.last = __ballot(inside && t + 1 == w.hi);
        r.inside = __ballot(inside);
    }
    return r;
}
// The rows of a tensor from t0 on: one address for the first of them, 32-bit offsets from there (strides are below 2^26 elements, so
// 15 rows are less than 2^32 bytes).
struct RowPointer {
    uint64_t at;
    uint32_t step;
    int left;                            // rows behind t0
    __device__ __forceinline__ RowPointer(const void* base, long long stride, int bytes, int t0, int T) {
        const int t = min(t0, T - 1);
        step = (uint32_t)stride * (uint32_t)bytes;
        at = (uint64_t)base + (uint64_t)t * step;
        left = T - 1 - t;
    }
    __device__ __forceinline__ uint32_t row(int j) const { return (uint32_t)j * step; }
    __device__ __forceinline__ uint32_t row_or_last(int j) const { return (uint32_t)min(j, left) * step; }     // behind the last row, that one
};

// The states of sequences of no rows go through: to[s] = from[s].  Wavefront `part` of `parts` looks at every parts-th 64 of them.
template <int V>
__device__ __forceinline__ void pass_empty(const RecurArgs& p, const float* from, float* to, int c, long long part, long long parts) {
    for (long long base = part * 64; base < p.S; base += parts * 64) {
        const long long s = base + (threadIdx.x & 63);
        bool empty = false;
        if (s < p.S) {
            const Span w = span_of(p, (int)s);
            empty = w.lo >= w.hi;
        }
        for (uint64_t m = __ballot(empty); m != 0; m &= m - 1) {
            const size_t at = (size_t)(base + __builtin_ctzll(m)) * p.C + c;
#pragma unroll
            for (int v = 0; v < V; ++v) to[at + v] = from ? from[at + v] : 0.0f;
        }
    }
}

// ---- the chain of chunks
// Workspace: a counter per column of workgroups (64 bytes each), then per chunk the maps (A, S) of its channels (behind the last chunk
// of a team: of the whole team), then per group the states behind it.  All bits set: not written.
constexpr uint32_t kUnset = 0xffffffffu;                    // a NaN
constexpr int kSpins = 1 << 20;          // looks at a word before it is given up: a second or two
__host__ __device__ inline size_t chain_counters(int cols) { return (size_t)cols * 8; }               // in 64-bit words
__host__ __device__ inline size_t chain_words(int chunks, int cols, int width) {
    return chain_counters(cols) + ((size_t)chunks + (size_t)(chunks + kGroup - 1) / kGroup) * cols * width;
}

__device__ __forceinline__ uint64_t chain_word(float hi, float lo) {
    uint32_t h = __float_as_uint(hi);
    if (hi != hi) h = 0x7fc00000u;                          // a NaN, but not the one that means "not written"
    return ((uint64_t)h << 32) | __float_as_uint(lo);
}
__device__ __forceinline__ void chain_put(uint64_t* w, uint64_t v) { __hip_atomic_store(w, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t chain_get(const uint64_t* w) { return __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool is_set(uint64_t w) { return (uint32_t)(w >> 32) != kUnset; }

__global__ __launch_bounds__(256) void recur_clear_kernel(uint4* w, size_t n) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) w[i] = make_uint4(kUnset, kUnset, kUnset, kUnset);
}

template <int V, int NW>
struct ChainLds {
    float A[kTeams][64 * V], S[kTeams][64 * V], state[64 * V];
    float decay[64 * V];
    int ticket;
};
// The chunk this workgroup is to do, the next of its column's, and its channels' decays.
template <int V, int NW>
__device__ __forceinline__ int chain_start(const RecurArgs& p, uint64_t* ws, int chunks, int cols, int col, ChainLds<V, NW>& lds) {
    constexpr int WIDTH = 64 * V;
    if (chunks > 1 && threadIdx.x == 0) lds.ticket = (int)(atomicAdd(reinterpret_cast<uint32_t*>(ws + (size_t)col * 8), 1u) + 1u);
    const int c = (int)blockDim.x - 1 - (int)threadIdx.x;   // from the last wavefront on: the first waits for its ticket
    if (c < WIDTH) lds.decay[c] = decay_of(p.lam[min(min(col * WIDTH + c / V * V, p.C - V) + c % V, p.C - 1)], p.scale);
    __syncthreads();
    return chunks > 1 ? __builtin_amdgcn_readfirstlane(lds.ticket) : 0;
}
// Waits for the words of one chunk or group, V per lane.
template <int V>
__device__ __forceinline__ void chain_wait(const uint64_t* w, uint64_t* v) {
    for (int spin = 0;; ++spin) {
        bool all = true;
#pragma unroll
        for (int q = 0; q < V; ++q) {
            v[q] = chain_get(w + q * 64);
            all = all && is_set(v[q]);
        }
        if (__all(all) || spin == kSpins) return;
        __builtin_amdgcn_s_sleep(4);
    }
}
// The value in front of chunk k (in the order of the scan) for this lane's channels, where the map of chunk k itself is (A, S)
// (of the first wavefront; the others need not have it); every wavefront gets it.  kTeam chunks make a team, kTeams teams a group.  A chunk
// reads the maps of its team in front of it (the first wavefront, at most 3), those of the group's teams in front of that (one for
// each further wavefront, at most 7) and the state behind the group before (the last wavefront): 6 reads on average.
// The map of a team does not wait for other teams, nor that of a chunk for anything, so only the states, one per group, are a chain.
// What is left is the way of two words through memory, some 4 us of a workgroup's 13: 65536 x 2048 bf16 forward takes 255 us, 218
// without this function.  (More rows on the way meanwhile need registers that are not there: a workgroup that asks for its next
// chunk's rows before it waits spills; one level of 32 chunks, 16 reads each, takes as long.)
template <int V, int NW>
__device__ __forceinline__ void chain(uint64_t* ws, int chunks, int cols, int col, int k, const float* A, const float* S, float* carry, ChainLds<V, NW>& lds) {
    constexpr int WIDTH = 64 * V;
    static_assert(NW > kTeams - 1, "a wavefront for each team");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int g = k / kGroup, j = k % kGroup, team = j / kTeam, q = j % kTeam;
    uint64_t* maps = ws + chain_counters(cols) + (size_t)col * WIDTH + lane;
    uint64_t* states = maps + (size_t)chunks * cols * WIDTH;
    const size_t step = (size_t)cols * WIDTH;
    const bool end = j == kGroup - 1 || k == chunks - 1;    // nobody reads the map of a group's last chunk
    const bool teller = !end && q == kTeam - 1;             // the last chunk of a team: others wait for the team's map
    // the first wavefront: the maps of the team in front of this chunk, to LDS
    const auto near = [&] {
        uint64_t w[kTeam - 1][V];
        for (int spin = 0;; ++spin) {
            bool all = true;
#pragma unroll
            for (int m = 0; m < kTeam - 1; ++m)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    w[m][v] = 0x3f80000000000000ull;        // h -> 1 h + 0
                    if (m < q) {
                        w[m][v] = chain_get(maps + (size_t)(k - q + m) * step + v * 64);
                        all = all && is_set(w[m][v]);
                    }
                }
            if (__all(all) || spin == kSpins) break;
            __builtin_amdgcn_s_sleep(4);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float tA = 1.0f, tS = 0.0f;
#pragma unroll
            for (int m = 0; m < kTeam - 1; ++m) {
                const float a = __uint_as_float((uint32_t)(w[m][v] >> 32));
                tS = apply(a, tS, __uint_as_float((uint32_t)w[m][v]));
                tA = compose(tA, a);
            }
            lds.A[0][lane * V + v] = tA;
            lds.S[0][lane * V + v] = tS;
            if (teller) chain_put(maps + (size_t)k * step + v * 64, chain_word(compose(tA, A[v]), apply(A[v], tS, S[v])));
        }
    };
    if (wave == 0) {
        if (teller) {
            near();
        } else if (!end) {
#pragma unroll
            for (int v = 0; v < V; ++v) chain_put(maps + (size_t)k * step + v * 64, chain_word(A[v], S[v]));
        }
    }
    if (wave == 0) {
        if (!teller) near();
    } else if (wave <= team) {
        uint64_t w[V];
        chain_wait<V>(maps + (size_t)(g * kGroup + wave * kTeam - 1) * step, w);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            lds.A[wave][lane * V + v] = __uint_as_float((uint32_t)(w[v] >> 32));
            lds.S[wave][lane * V + v] = __uint_as_float((uint32_t)w[v]);
        }
    }
    if (wave == NW - 1) {
        uint64_t w[V];
        if (g > 0) chain_wait<V>(states + (size_t)(g - 1) * step, w);
#pragma unroll
        for (int v = 0; v < V; ++v) lds.state[lane * V + v] = g > 0 ? __uint_as_float((uint32_t)w[v]) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = lds.state[lane * V + v];
    for (int w = 1; w <= team; ++w)
#pragma unroll
        for (int v = 0; v < V; ++v) carry[v] = apply(lds.A[w][lane * V + v], carry[v], lds.S[w][lane * V + v]);
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = apply(lds.A[0][lane * V + v], carry[v], lds.S[0][lane * V + v]);
    if (wave == 0 && j == kGroup - 1 && k != chunks - 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) chain_put(states + (size_t)g * step + v * 64, chain_word(0.0f, apply(A[v], carry[v], S[v])));
    }
}

// The gates of a row's channels: y = log2 a, a, sigmoid(i) and b = sqrt(1 - a^2).
struct Gates { float sr, a, si, b; };
template <typename T, int V>
__device__ __forceinline__ Gates gates(const Pack<T, V>& r, const Pack<T, V>& i, int v, float decay) {
    Gates g;
    g.sr = sigmoid(get<T, V>(r, v));
    g.si = sigmoid(get<T, V>(i, v));
    const float y = -decay * g.sr;
    g.a = __builtin_amdgcn_exp2f(y);
    g.b = __builtin_amdgcn_sqrtf(one_minus_square(y, g.a));
    return g;
}
__device__ __forceinline__ bool bit(uint64_t m, int j) { return ((m >> j) & 1) != 0; }
// The values that the first two of the marked rows read of an [S][C] array (h0 at first rows, dhT at last ones), asked for
// together and ahead; those of further rows, in wavefronts of sequences of a few rows, one by one.
template <int V>
struct Ahead {
    const float* from;
    int row0, row1;
    float val0[V], val1[V];
    __device__ __forceinline__ Ahead(const RecurArgs& p, const RowBits& bits, uint64_t marked, const float* array, int c) : from(array) {
        const uint64_t behind = marked & (marked - 1);
        row0 = array != nullptr && marked != 0 ? __builtin_ctzll(marked) : -1;
        row1 = array != nullptr && behind != 0 ? __builtin_ctzll(behind) : -1;
#pragma unroll
        for (int v = 0; v < V; ++v) val0[v] = val1[v] = 0.0f;
        if (row0 >= 0) {
            const float* q = from + (size_t)bits.seq_of(row0) * p.C + c;
#pragma unroll
            for (int v = 0; v < V; ++v) val0[v] = q[v];
        }
        if (row1 >= 0) {
            const float* q = from + (size_t)bits.seq_of(row1) * p.C + c;
#pragma unroll
            for (int v = 0; v < V; ++v) val1[v] = q[v];
        }
    }
    __device__ __forceinline__ float get(const RecurArgs& p, const RowBits& bits, int j, int c, int v) const {
        if (j != row0 && j != row1) return from[(size_t)bits.seq_of(j) * p.C + c + v];
        float a = val0[v], b = val1[v];
        asm("" : "+v"(a), "+v"(b));                         // values, not the places they are in: those would be in scratch memory
        return j == row0 ? a : b;
    }
};
// A row's map on top of (A, S); PLAIN: known to be neither a first row nor one of no sequence.  A is the product of the other rows' decays.
template <bool PLAIN, int V>
__device__ __forceinline__ void add_row(const RecurArgs& p, const RowBits& bits, int j, int c, const float* a, float* u, float* A, float* S,
                                        const Ahead<V> h0) {
    if (!PLAIN && bit(bits.first, j)) {
        if (p.h0) {
#pragma unroll
            for (int v = 0; v < V; ++v) u[v] = fmaf(a[v], h0.get(p, bits, j, c, v), u[v]);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) S[v] = u[v];
    } else if (!PLAIN && !bit(bits.inside, j)) {
#pragma unroll
        for (int v = 0; v < V; ++v) u[v] = S[v] = 0.0f;
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            S[v] = fmaf(a[v], S[v], u[v]);
            A[v] *= a[v];
        }
    }
}

// the map of a wavefront whose rows are of no sequence, which does nothing else (4 x 395 bf16 forward 6.8 us without, 6.0 with; backward 11.6 and 10.9)
template <int V>
__device__ __forceinline__ void no_rows(float* A) {
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = kCut;
}

// ---- forward
template <int V, int TW, bool PLAIN>
__device__ __forceinline__ void add_rows(const RecurArgs& p, const RowBits& bits, int c, const float (*a)[V], float (*u)[V], float* A, float* S,
                                         const Ahead<V> h0) {
#pragma unroll
    for (int j = 0; j < TW; ++j) add_row<PLAIN, V>(p, bits, j, c, a[j], u[j], A, S, h0);
    // Rows that hold a first one or one of no sequence forget what comes before them, whatever the decays behind are: a product with a NaN
    // among them would not, and the backward pass would carry it to the sequence in front.
    if (!PLAIN && ((bits.first | ~bits.inside) & ((1ull << TW) - 1)) != 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = kCut;
    }
}
template <typename T, int V, int TW, bool PLAIN>
__device__ __forceinline__ void fwd_rows(const RecurArgs& p, const RowBits& bits, int c, uint32_t off, const RowPointer row, const float (*a)[V],
                                         const float (*u)[V], float* h) {
#pragma unroll
    for (int j = 0; j < TW; ++j) {
        const bool cut = !PLAIN && (bit(bits.first, j) || !bit(bits.inside, j));
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = cut ? u[j][v] : fmaf(a[j][v], h[v], u[j][v]);
        if (PLAIN || bit(bits.inside, j)) store_pack<T, V>(row.at, off + row.row(j), h);
        if (!PLAIN && p.hT && bit(bits.last, j)) {
            float* hT = p.hT + (size_t)bits.seq_of(j) * p.C + c;
#pragma unroll
            for (int v = 0; v < V; ++v) hT[v] = h[v];
        }
    }
}

template <typename T, int V, int TW, int NW>
__global__ __launch_bounds__(64 * NW) void recur_fwd_kernel(const RecurArgs p, int chunks, int cols) {
    constexpr int WIDTH = 64 * V, EB = Elem<T>::kBytes;
    __shared__ float mapA[NW][WIDTH], mapS[NW][WIDTH];
    __shared__ ChainLds<V, NW> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), col = blockIdx.x % cols;
    uint64_t* const ws = static_cast<uint64_t*>(p.workspace);
    const SeqSearch search(p);
    const int k = chain_start<V, NW>(p, ws, chunks, cols, col, lds);
    if ((unsigned)k >= (unsigned)chunks) return;
    const int c = min(col * WIDTH + lane * V, p.C - V);     // the lanes past the last channels do those again
    const uint32_t off = (uint32_t)c * EB;
    const int t0 = (k * NW + wave) * TW;
    const RowBits bits = row_bits<TW>(p, search, t0);
    Pack<T, V> xr[TW], rr[TW], ir[TW];
    {
        RowPointer px(p.x, p.sx, EB, t0, p.T), pr(p.r, p.sr, EB, t0, p.T), pi(p.i, p.si, EB, t0, p.T);
#pragma unroll
        for (int j = 0; j < TW; ++j) {
            xr[j] = load_pack<T, V>(px.at, off + px.row_or_last(j));
            rr[j] = load_pack<T, V>(pr.at, off + pr.row_or_last(j));
            ir[j] = load_pack<T, V>(pi.at, off + pi.row_or_last(j));
        }
    }
    const Ahead<V> h0(p, bits, bits.first, p.h0, c);
    float decay[V], A[V], S[V], h[V], a[TW][V], u[TW][V];
#pragma unroll
    for (int v = 0; v < V; ++v) { decay[v] = lds.decay[lane * V + v]; A[v] = 1.0f; S[v] = h[v] = 0.0f; }
#pragma unroll
    for (int j = 0; j < TW; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Gates g = gates<T, V>(rr[j], ir[j], v, decay[v]);
            a[j][v] = g.a;
            u[j][v] = g.b * g.si * get<T, V>(xr[j], v);
        }
    if (bits.plain) add_rows<V, TW, true>(p, bits, c, a, u, A, S, h0);
    else if (bits.inside != 0) add_rows<V, TW, false>(p, bits, c, a, u, A, S, h0);
    else no_rows<V>(A);
#pragma unroll
    for (int v = 0; v < V; ++v) { mapA[wave][lane * V + v] = A[v]; mapS[wave][lane * V + v] = S[v]; }
    __syncthreads();
    if (chunks > 1) {
        if (wave == 0) {
#pragma unroll
            for (int w = 1; w < NW; ++w)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    S[v] = apply(mapA[w][lane * V + v], S[v], mapS[w][lane * V + v]);
                    A[v] = compose(A[v], mapA[w][lane * V + v]);
                }
        }
        chain<V, NW>(ws, chunks, cols, col, k, A, S, h, lds);
    }
    for (int w = 0; w < wave; ++w)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = apply(mapA[w][lane * V + v], h[v], mapS[w][lane * V + v]);
    if (p.saved && t0 % kSavedRows == 0 && t0 < p.T) {
#pragma unroll
        for (int v = 0; v < V; ++v) p.saved[(size_t)(t0 / kSavedRows) * p.C + c + v] = h[v];
    }
    const RowPointer ph(p.h, p.sh, EB, t0, p.T);
    if (bits.plain) fwd_rows<T, V, TW, true>(p, bits, c, off, ph, a, u, h);
    else if (bits.inside != 0) fwd_rows<T, V, TW, false>(p, bits, c, off, ph, a, u, h);
    if (p.hT) pass_empty<V>(p, p.h0, p.hT, c, (long long)k * NW + wave, (long long)chunks * NW);
}

// ---- backward
// The rows' maps and what the second run needs: u gives way to the state in front of each row there.
template <typename T, int V, int TW>
struct BwdRows {
    Pack<T, V> x[TW], dh[TW];
    float a[TW][V], u[TW][V], sr[TW][V], si[TW][V], b[TW][V];
};
template <typename T, int V, int TW, bool PLAIN>
__device__ __forceinline__ void bwd_maps(const RecurArgs& p, const RowBits& bits, int c, BwdRows<T, V, TW>& w, float* A, float* S, float* D,
                                         const Ahead<V> h0, const Ahead<V> dhT) {
    add_rows<V, TW, PLAIN>(p, bits, c, w.a, w.u, A, S, h0);
    // e in front of the rows from the one behind them: D + A e.  Behind a sequence's last row there is another's first, whose e
    // does not come here, or a row of none: D is 0 there.
#pragma unroll
    for (int j = TW - 1; j >= 0; --j) {
        if (!PLAIN && (bit(bits.first, j) || !bit(bits.inside, j))) {
#pragma unroll
            for (int v = 0; v < V; ++v) D[v] = 0.0f;
        } else {
            const bool last = !PLAIN && p.dhT && bit(bits.last, j);
#pragma unroll
            for (int v = 0; v < V; ++v) D[v] = w.a[j][v] * (get<T, V>(w.dh[j], v) + D[v] + (last ? dhT.get(p, bits, j, c, v) : 0.0f));
        }
    }
}
template <typename T, int V, int TW, bool PLAIN>
__device__ __forceinline__ void bwd_rows(const RecurArgs& p, const RowBits& bits, int t0, int c, uint32_t off, const float* decay, BwdRows<T, V, TW>& w,
                                         float* h, float* e, float* sum, const Ahead<V> h0, const Ahead<V> dhT) {
#pragma unroll
    for (int j = 0; j < TW; ++j) {
        const bool first = !PLAIN && bit(bits.first, j), cut = first || (!PLAIN && !bit(bits.inside, j));
        const bool start = first && p.h0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float next = cut ? w.u[j][v] : fmaf(w.a[j][v], h[v], w.u[j][v]);
            w.u[j][v] = cut ? (start ? h0.get(p, bits, j, c, v) : 0.0f) : h[v];
            h[v] = next;
        }
    }
    constexpr int EB = Elem<T>::kBytes;
    const RowPointer px(p.dx, p.sdx, EB, t0, p.T), pr(p.dr, p.sdr, EB, t0, p.T), pi(p.di, p.sdi, EB, t0, p.T);
    float log2a[V];                                         // of an open gate, in natural logarithms
#pragma unroll
    for (int v = 0; v < V; ++v) log2a[v] = -decay[v] * 0.6931471805599453f;
#pragma unroll
    for (int j = TW - 1; j >= 0; --j) {
        if (PLAIN || bit(bits.inside, j)) {
            float dx[V], di[V], dr[V];
            const bool last = !PLAIN && p.dhT && bit(bits.last, j);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float a = w.a[j][v], b = w.b[j][v], si = w.si[j][v], sr = w.sr[j][v], x = get<T, V>(w.x[j], v);
                const float ib = b > 0.0f ? __builtin_amdgcn_rcpf(b) : 0.0f;
                const float g = get<T, V>(w.dh[j], v) + e[v] + (last ? dhT.get(p, bits, j, c, v) : 0.0f), gs = g * si;
                e[v] = a * g;
                const float q = log2a[v] * sr * fmaf(e[v], w.u[j][v], -(a * ib) * (a * gs * x));
                sum[v] += q;
                dx[v] = b * gs;
                di[v] = dx[v] * x * (1.0f - si);
                dr[v] = q * (1.0f - sr);
            }
            store_pack<T, V>(px.at, off + px.row(j), dx);
            store_pack<T, V>(pi.at, off + pi.row(j), di);
            store_pack<T, V>(pr.at, off + pr.row(j), dr);
        }
        if (!PLAIN && bit(bits.first, j) && p.dh0) {
            float* d0 = p.dh0 + (size_t)bits.seq_of(j) * p.C + c;
#pragma unroll
            for (int v = 0; v < V; ++v) d0[v] = e[v];
        }
        if (!PLAIN && (bit(bits.first, j) || !bit(bits.inside, j))) {
#pragma unroll
            for (int v = 0; v < V; ++v) e[v] = 0.0f;
        }
    }
}

template <typename T, int V, int TW, int NW>
__global__ __launch_bounds__(64 * NW) void recur_bwd_kernel(const RecurArgs p, float* parts, int chunks, int cols) {
    constexpr int WIDTH = 64 * V, EB = Elem<T>::kBytes;
    __shared__ float mapA[NW][WIDTH], mapS[NW][WIDTH], mapD[NW][WIDTH];
    __shared__ ChainLds<V, NW> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), col = blockIdx.x % cols;
    uint64_t* const ws = static_cast<uint64_t*>(p.workspace);
    const SeqSearch search(p);
    const int n = chain_start<V, NW>(p, ws, chunks, cols, col, lds), k = chunks - 1 - n;   // the chain runs from the last chunk
    if ((unsigned)n >= (unsigned)chunks) return;
    const int c = min(col * WIDTH + lane * V, p.C - V);
    const uint32_t off = (uint32_t)c * EB;
    const int t0 = (k * NW + wave) * TW;
    const RowBits bits = row_bits<TW>(p, search, t0);
    BwdRows<T, V, TW> rows;
    Pack<T, V> rr[TW], ir[TW];
    {
        RowPointer px(p.x, p.sx, EB, t0, p.T), pr(p.r, p.sr, EB, t0, p.T), pi(p.i, p.si, EB, t0, p.T), pd(p.dh, p.sdh, EB, t0, p.T);
#pragma unroll
        for (int j = 0; j < TW; ++j) {
            rr[j] = load_pack<T, V>(pr.at, off + pr.row_or_last(j));
            ir[j] = load_pack<T, V>(pi.at, off + pi.row_or_last(j));
            rows.x[j] = load_pack<T, V>(px.at, off + px.row_or_last(j));
        }
#pragma unroll
        for (int j = 0; j < TW; ++j) {
            rows.dh[j] = load_pack<T, V>(pd.at, off + pd.row_or_last(j));
        }
    }
    const Ahead<V> h0(p, bits, bits.first, p.h0, c), dhT(p, bits, bits.last, p.dhT, c);
    float decay[V], A[V], S[V], D[V], h[V], e[V], sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        decay[v] = lds.decay[lane * V + v];
        h[v] = p.saved[(size_t)k * p.C + c + v];
        A[v] = 1.0f;
        S[v] = D[v] = e[v] = sum[v] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < TW; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Gates g = gates<T, V>(rr[j], ir[j], v, decay[v]);
            rows.a[j][v] = g.a; rows.sr[j][v] = g.sr; rows.si[j][v] = g.si; rows.b[j][v] = g.b;
            rows.u[j][v] = g.b * g.si * get<T, V>(rows.x[j], v);
        }
    if (bits.plain) bwd_maps<T, V, TW, true>(p, bits, c, rows, A, S, D, h0, dhT);
    else if (bits.inside != 0) bwd_maps<T, V, TW, false>(p, bits, c, rows, A, S, D, h0, dhT);
    else no_rows<V>(A);
#pragma unroll
    for (int v = 0; v < V; ++v) { mapA[wave][lane * V + v] = A[v]; mapS[wave][lane * V + v] = S[v]; mapD[wave][lane * V + v] = D[v]; }
    __syncthreads();
    if (chunks > 1) {
        if (wave == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) { A[v] = 1.0f; D[v] = 0.0f; }
#pragma unroll
            for (int w = NW - 1; w >= 0; --w)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    D[v] = apply(mapA[w][lane * V + v], D[v], mapD[w][lane * V + v]);
                    A[v] = compose(A[v], mapA[w][lane * V + v]);
                }
        }
        chain<V, NW>(ws, chunks, cols, col, n, A, D, e, lds);
    }
    for (int w = NW - 1; w > wave; --w)
#pragma unroll
        for (int v = 0; v < V; ++v) e[v] = apply(mapA[w][lane * V + v], e[v], mapD[w][lane * V + v]);
    for (int w = 0; w < wave; ++w)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = apply(mapA[w][lane * V + v], h[v], mapS[w][lane * V + v]);
    if (bits.plain) bwd_rows<T, V, TW, true>(p, bits, t0, c, off, decay, rows, h, e, sum, h0, dhT);
    else if (bits.inside != 0) bwd_rows<T, V, TW, false>(p, bits, t0, c, off, decay, rows, h, e, sum, h0, dhT);
    if (p.dh0) pass_empty<V>(p, p.dhT, p.dh0, c, (long long)k * NW + wave, (long long)chunks * NW);
    __syncthreads();                                        // the maps have been read
#pragma unroll
    for (int v = 0; v < V; ++v) mapA[wave][lane * V + v] = sum[v];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) total += mapA[w][lane * V + v];
            if (chunks > 1) parts[(size_t)k * p.C + c + v] = total;
            else p.dlam[c + v] = total * decay_slope(p.lam[c + v]);
        }
    }
}

// dlam from the chunks' sums: 16 channels x 64 shares of the chunks per workgroup, the shares joined in order.
__global__ __launch_bounds__(1024) void recur_dlam_kernel(const float* parts, int n, int C, const float* lam, float* dlam) {
    __shared__ float red[64][16];
    const int lane = threadIdx.x & 15, share = threadIdx.x >> 4, c = blockIdx.x * 16 + lane;
    float sum = 0.0f;
    if (c < C) {
#pragma unroll 8
        for (int k = share; k < n; k += 64) sum += parts[(size_t)k * C + c];
    }
    red[share][lane] = sum;
    __syncthreads();
    if (share == 0 && c < C) {
        for (int q = 1; q < 64; ++q) sum += red[q][lane];
        dlam[c] = sum * decay_slope(lam[c]);
    }
}

// No rows at all: the states go through, and nothing adds to dlam.
__global__ __launch_bounds__(256) void recur_none_kernel(const float* from, float* to, long long n, float* zero, int C) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        if (to) to[i] = from ? from[i] : 0.0f;
        if (zero && i < C) zero[i] = 0.0f;
    }
}

// ---- one token per sequence.  One row and 256 V channels per workgroup.  A slot that stands at several rows is done by the
// workgroup of the first of them, in the order of the rows; all rows' slots are looked through while the row's own loads
// are under way.  That hides up to a thousand rows (512 x 2048 bf16 7.4 us, without slots 6.9) and grows with their square behind it
// (4096 x 2048 47 and 36; a table sorted by slot in the workspace would need two more launches, 4 us each).
template <typename T, int V>
__global__ __launch_bounds__(256) void recur_step_kernel(const RecurArgs p, float* state, const int32_t* slots, long long slot_count) {
    __shared__ int seen[4];
    constexpr uint64_t EB = Elem<T>::kBytes;
    const int cols = (p.C + 256 * V - 1) / (256 * V), row = blockIdx.x / cols, first = ((blockIdx.x % cols) * 256 + threadIdx.x) * V;
    const int c = min(first, p.C - V), keep = first - c;    // the last lane may have its channels from `keep` on only
    const int slot = slots ? slots[row] : row;
    if (slot < 0 || slot >= slot_count) return;
    const uint32_t off = (uint32_t)c * (uint32_t)EB;
    float* const st = state + (size_t)slot * p.C + c;
    Pack<T, V> x = load_pack<T, V>((uint64_t)p.x + row * p.sx * EB, off), r = load_pack<T, V>((uint64_t)p.r + row * p.sr * EB, off),
               i = load_pack<T, V>((uint64_t)p.i + row * p.si * EB, off);
    float h[V], decay[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { h[v] = st[v]; decay[v] = p.lam[c + v]; }
    bool again = false;
    if (slots) {
        int found = 0;                                      // 1: at an earlier row, 2: at a later one
        const auto look = [&](int t, int other) {
            if (other == slot && t != row) found |= t < row ? 1 : 2;
        };
        if (p.T <= 256) {
            if ((int)threadIdx.x < p.T) look(threadIdx.x, slots[threadIdx.x]);
        } else {                                            // four at a time, the last four for those past the end: looked at twice, nothing lost
#pragma unroll 4
            for (int t = threadIdx.x * 4; t < p.T; t += 1024) {
                uint32_t w[4];
                const int at = min(t, p.T - 4);
                load_words_any<4>(slots + at, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) look(at + k, (int)w[k]);
            }
        }
        const int all = (__ballot((found & 1) != 0) != 0 ? 1 : 0) | (__ballot((found & 2) != 0) != 0 ? 2 : 0);
        if ((threadIdx.x & 63) == 0) seen[threadIdx.x >> 6] = all;
        __syncthreads();
        const int any = seen[0] | seen[1] | seen[2] | seen[3];
        if (any & 1) return;
        again = (any & 2) != 0;
    }
    if (keep >= V) return;
#pragma unroll
    for (int v = 0; v < V; ++v) decay[v] = decay_of(decay[v], p.scale);
    for (int t = row;;) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Gates g = gates<T, V>(r, i, v, decay[v]);
            h[v] = fmaf(g.a, h[v], g.b * g.si * get<T, V>(x, v));
        }
        const uint64_t to = (uint64_t)p.h + t * p.sh * EB;
        if (keep == 0) {
            store_pack<T, V>(to, off, h);
        } else {
#pragma unroll
            for (int v = 1; v < V; ++v)
                if (v >= keep) store_pack<T, 1>(to, off + v * (uint32_t)EB, h + v);
        }
        if (again)
            do ++t; while (t < p.T && slots[t] != slot);
        if (!again || t >= p.T) break;
        x = load_pack<T, V>((uint64_t)p.x + t * p.sx * EB, off);
        r = load_pack<T, V>((uint64_t)p.r + t * p.sr * EB, off);
        i = load_pack<T, V>((uint64_t)p.i + t * p.si * EB, off);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v >= keep) st[v] = h[v];
}

int launched() { return hipGetLastError() == hipSuccess ? SCAN2D_OK : SCAN2D_ERR_LAUNCH_FAILED; }

// ---- shapes.  One lane per channel up to 64 channels, two channels per lane beyond.
constexpr int kFwdWaves = 8, kBwdWaves = 12;                            // wavefronts of a workgroup
constexpr int kBwdRows = kSavedRows / kBwdWaves;                       // rows of a wavefront in the backward pass
struct RecurPlan {
    int V, chunks, cols;
    int rows, waves;                     // rows of a wavefront, wavefronts of a workgroup
};
RecurPlan plan_of(const scan2d_recur_desc* d, int pass) {
    RecurPlan q;
    q.V = d->C <= 64 ? 1 : 2;
    q.cols = (d->C + 64 * q.V - 1) / (64 * q.V);
    q.waves = pass == SCAN2D_PASS_BWD ? kBwdWaves : kFwdWaves;
    const auto chunks = [&](int rows) { return (d->T + rows * q.waves - 1) / (rows * q.waves); };
    // forward, bf16 or one channel a lane: 16 rows of a wavefront (65536 x 2048 255 us, with 8 rows 298; 65536 x 256 44 and 62; 63200 x 61 fp32
    // 30 and 50), but 8 where that leaves compute units without a workgroup (1000 x 512 10.1 us, with 16 rows 12.7; 37 x 256 6.0 and 9.2), or with
    // registers for too few (fp32)
    const bool deep = d->dtype == SCAN2D_BF16 || q.V == 1;
    q.rows = pass == SCAN2D_PASS_BWD ? kBwdRows : deep && chunks(16) * q.cols >= 256 ? 16 : 8;
    q.chunks = (int)chunks(q.rows);
    return q;
}
size_t chain_bytes(const RecurPlan& q) { return q.chunks > 1 ? (chain_words(q.chunks, q.cols, 64 * q.V) * 8 + 255) / 256 * 256 : 0; }

int clear_chain(const RecurPlan& q, void* workspace, hipStream_t stream) {
    const size_t n = chain_bytes(q) / 16;
    hipLaunchKernelGGL(recur_clear_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, static_cast<uint4*>(workspace), n);
    return launched();
}
// The chunks in as many launches as it takes to stay below 2^32 threads in each: launch(workgroups).  Each does as many chunks of every column and
// goes on where the one before left the counters and the states.
template <typename Launch>
void by_chunks(const RecurPlan& q, Launch launch) {
    const long long most = ((1LL << 32) - 1) / (64LL * q.waves * q.cols);
    for (long long left = q.chunks; left > 0; left -= most) launch((unsigned)((left < most ? left : most) * q.cols));
}

int launch_none(const RecurArgs& a, const float* from, float* to, float* zero, hipStream_t stream) {
    const long long n = (long long)a.S * a.C, blocks = (n + 255) / 256, most = 1 << 16;      // S >= 1: n values are C at least
    hipLaunchKernelGGL(recur_none_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, stream, from, to, n, zero, a.C);
    return launched();
}

}  // namespace

size_t recur_saved_bytes(const scan2d_recur_desc* d) { return (size_t)((d->T + kSavedRows - 1) / kSavedRows) * d->C * 4; }
size_t recur_workspace_bytes(const scan2d_recur_desc* d, int pass) {
    const RecurPlan q = plan_of(d, pass);
    return chain_bytes(q) + (pass == SCAN2D_PASS_BWD && q.chunks > 1 ? (size_t)q.chunks * d->C * 4 : 0);
}

int recur_fwd_launch(const scan2d_recur_desc* d, const RecurArgs& a, hipStream_t stream) {
    const RecurPlan q = plan_of(d, SCAN2D_PASS_FWD);
    (void)hipGetLastError();
    if (q.chunks == 0) return a.hT ? launch_none(a, a.h0, a.hT, nullptr, stream) : SCAN2D_OK;
    if (q.chunks > 1) {
        const int rc = clear_chain(q, a.workspace, stream);
        if (rc != SCAN2D_OK) return rc;
    }
    using Kernel = void (*)(const RecurArgs, int, int);
    Kernel k;
    if (d->dtype != SCAN2D_BF16) k = q.V == 2 ? recur_fwd_kernel<float, 2, 8, kFwdWaves> : q.rows == 8 ? recur_fwd_kernel<float, 1, 8, kFwdWaves> : recur_fwd_kernel<float, 1, 16, kFwdWaves>;
    else if (q.rows == 8) k = q.V == 1 ? recur_fwd_kernel<bf16_t, 1, 8, kFwdWaves> : recur_fwd_kernel<bf16_t, 2, 8, kFwdWaves>;
    else k = q.V == 1 ? recur_fwd_kernel<bf16_t, 1, 16, kFwdWaves> : recur_fwd_kernel<bf16_t, 2, 16, kFwdWaves>;
    by_chunks(q, [&](unsigned wgs) { hipLaunchKernelGGL(k, dim3(wgs), dim3(64 * q.waves), 0, stream, a, q.chunks, q.cols); });
    return launched();
}

int recur_bwd_launch(const scan2d_recur_desc* d, const RecurArgs& a, hipStream_t stream) {
    const RecurPlan q = plan_of(d, SCAN2D_PASS_BWD);
    (void)hipGetLastError();
    if (q.chunks == 0) return launch_none(a, a.dhT, a.dh0, a.dlam, stream);
    float* parts = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + chain_bytes(q));
    if (q.chunks > 1) {
        const int rc = clear_chain(q, a.workspace, stream);
        if (rc != SCAN2D_OK) return rc;
    }
    using Kernel = void (*)(const RecurArgs, float*, int, int);
    const Kernel k = d->dtype == SCAN2D_BF16 ? (q.V == 1 ? recur_bwd_kernel<bf16_t, 1, kBwdRows, kBwdWaves> : recur_bwd_kernel<bf16_t, 2, kBwdRows, kBwdWaves>)
                                             : (q.V == 1 ? recur_bwd_kernel<float, 1, kBwdRows, kBwdWaves> : recur_bwd_kernel<float, 2, kBwdRows, kBwdWaves>);
    by_chunks(q, [&](unsigned wgs) { hipLaunchKernelGGL(k, dim3(wgs), dim3(64 * q.waves), 0, stream, a, parts, q.chunks, q.cols); });
    if (q.chunks > 1)
        hipLaunchKernelGGL(recur_dlam_kernel, dim3((a.C + 15) / 16), dim3(1024), 0, stream, parts, q.chunks, a.C, a.lam, a.dlam);
    return launched();
}

// One channel per lane where a workgroup has the row then.
static int step_channels(const scan2d_recur_desc* d) { return d->C <= 256 ? 1 : 2; }
static long long step_blocks(const scan2d_recur_desc* d) { return (d->C + 256LL * step_channels(d) - 1) / (256 * step_channels(d)) * d->T; }
bool recur_step_fits(const scan2d_recur_desc* d) { return launch_fits(step_blocks(d), 256); }
int recur_step_launch(const scan2d_recur_desc* d, const RecurArgs& a, float* state, const int32_t* slots, long long slot_count, hipStream_t stream) {
    const int V = step_channels(d);
    (void)hipGetLastError();
    using Kernel = void (*)(const RecurArgs, float*, const int32_t*, long long);
    const Kernel k = d->dtype == SCAN2D_BF16 ? (V == 1 ? recur_step_kernel<bf16_t, 1> : recur_step_kernel<bf16_t, 2>)
                                             : (V == 1 ? recur_step_kernel<float, 1> : recur_step_kernel<float, 2>);
    hipLaunchKernelGGL(k, dim3((unsigned)step_blocks(d)), dim3(256), 0, stream, a, state, slots, slot_count);
    return launched();
}

}  // namespace scan2d
