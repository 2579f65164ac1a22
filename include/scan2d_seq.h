/*
 * scan2d_seq.h -- C ABI of the sequence layers of the MI355X (gfx950) 2D selective scan library: operators on
 * channels-last tensors, where a row holds the C channels of one token (or one position of a map).
 *
 * Everything scan2d.h says of its entry points holds here too: device pointers owned by the caller, work only enqueued
 * on `stream` (a hipStream_t, NULL = the default stream), nothing allocated, freed or synchronised, outputs overwritten,
 * SCAN2D_OK or one of its negative codes returned, nothing enqueued and no output touched on an error, calls from several host
 * threads allowed, reductions in a fixed order (bit-reproducible).  The calls can be captured into a HIP graph.  The
 * current device has to be the one that owns the pointers.
 *
 * Rows: element (t, c) of a tensor lies at base + t * stride + c, in elements.  Every tensor has a stride of its own, at
 * least C and below 2^26 (0 stands for C), so that the halves of a projection [T][2 C] are used where they lie.  These tensors need
 * the alignment of their element type only; all others (parameters, states, statistics: dense) that of their type,
 * `saved` and `workspace` 16 bytes.
 *
 * Sizes: what is given at each descriptor.  A launch holds fewer than 2^32 threads; calls that need more are several launches
 * (seq_recur_step alone is always one).
 */
#ifndef SCAN2D_SEQ_H_
#define SCAN2D_SEQ_H_

#include "scan2d.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The gated linear recurrence.  For every sequence s, token t of it and channel c, all arithmetic in fp32:
 *     a_t = exp(-scale * softplus(lam[c]) * sigmoid(r[t,c]))
 *     h_t = a_t * h_{t-1} + sqrt(1 - a_t^2) * sigmoid(i[t,c]) * x[t,c],      h before the first token: h0[s,c], or 0
 *     hT[s,c] = h at the last token of s (h0[s,c] for a sequence of no tokens)
 * r and i are the gates' pre-activations.
 *
 * The T rows hold the sequences in one of three ways:
 *     offsets [S+1] int32: packed, sequence s has the rows offsets[s] .. offsets[s+1] - 1 (ascending, offsets[0] = 0,
 *                  empty sequences allowed; rows from offsets[S] on belong to none)
 *     lengths [S] int32:   padded, sequence s has the first lengths[s] of the rows s T/S .. (s+1) T/S - 1
 *     neither:             every sequence has T/S rows
 * T has to be a multiple of S unless offsets is given.  Rows of no sequence are never written in the outputs and never
 * count.  Values in offsets and lengths outside these rules give wrong results, and no access outside the tensors.
 */
typedef struct {
    int64_t  T;                /* rows, 0 <= T < 2^31 - 4096 */
    int32_t  C, S;             /* channels, sequences: >= 1; C < 2^24, S < 2^24 */
    int32_t  dtype;            /* SCAN2D_F32 or SCAN2D_BF16: type of x, r, i, h, dh, dx, dr, di */
    float    scale;            /* > 0, finite */
    int64_t  stride_x, stride_r, stride_i, stride_h;       /* of the rows, in elements; 0 = C */
    int64_t  stride_dh, stride_dx, stride_dr, stride_di;   /* backward only */
} scan2d_recur_desc;

/*
 *   x, r, i : [T][C] storage type;  lam : [C] fp32;  h0 : [S][C] fp32 or NULL (zero)
 *   h       : [T][C] storage type, written; none of x, r, i (SCAN2D_ERR_BAD_SHAPE)
 *   hT      : [S][C] fp32, written, or NULL; not h0 (SCAN2D_ERR_BAD_SHAPE)
 *   saved   : at least scan2d_seq_recur_saved_bytes(desc) bytes, written: what scan2d_seq_recur_bwd needs of the states
 *             (fp32); NULL where no backward follows
 *   workspace : at least scan2d_seq_recur_workspace_bytes(desc, SCAN2D_PASS_FWD) bytes (NULL if that is 0); contents
 *             undefined before and after; two calls that overlap in time must not share one
 * Not both of offsets and lengths (SCAN2D_ERR_BAD_FLAGS).
 */
int scan2d_seq_recur_fwd(const scan2d_recur_desc* desc, const void* x, const void* r, const void* i, const float* lam,
                         const int32_t* offsets, const int32_t* lengths, const float* h0,
                         void* h, float* hT, void* saved, size_t saved_bytes,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * Backward for given dh = dL/dh and dhT = dL/dhT ([S][C] fp32, or NULL: zero).  With s_r, s_i the sigmoids,
 * l_t = log a_t and b_t = sqrt(1 - a_t^2):
 *     g_t  = dh_t + [t last] dhT + a_{t+1} g_{t+1}
 *     q_t  = l_t * (a_t g_t h_{t-1} - a_t^2 / b_t g_t s_i x_t)         (the second term is 0 where b_t = 0)
 *     dx_t = b_t s_i g_t,   di_t = b_t x_t g_t s_i (1 - s_i),   dr_t = q_t (1 - s_r)
 *     dlam[c] = sum_{s,t} q_t * sigmoid(lam[c]) / softplus(lam[c])
 *     dh0[s,c] = a_t g_t at the first token of s (dhT for a sequence of no tokens)
 *   saved : as scan2d_seq_recur_fwd left it for the same inputs and the same descriptor (not modified)
 *   dh : [T][C] storage type;  dx, dr, di : [T][C] storage type, written, distinct and none of the inputs;
 *   dlam : [C] fp32, written;  dh0 : [S][C] fp32, written, or NULL (it may also be wanted where h0 was NULL); not dhT.
 * The states are recomputed in fp32; the stored h is not read.
 */
int scan2d_seq_recur_bwd(const scan2d_recur_desc* desc, const void* x, const void* r, const void* i, const float* lam,
                         const int32_t* offsets, const int32_t* lengths, const float* h0,
                         const void* dh, const float* dhT, const void* saved, size_t saved_bytes,
                         void* dx, void* dr, void* di, float* dlam, float* dh0,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * One token for each of T sequences (desc.S is not used; T >= 1).  Row t belongs to the state state[slots[t]] (state[t] where slots is
 * NULL; then slot_count >= T), which is replaced by the new one:
 *     state[slot,c] = a_t * state[slot,c] + sqrt(1 - a_t^2) * sigmoid(i) * x,       h[t,c] = state[slot,c]
 *   state : [slot_count][C] fp32;  slots : [T] int32 or NULL.  A row whose slot is negative or not below slot_count is
 *   padding: its h is not written and no state changes.  A slot that stands at several rows takes them in the order of the rows,
 *   as one call after the other would.  1 <= T <= 65535 and T ceil(C / 512) < 2^24 (one launch).
 */
int scan2d_seq_recur_step(const scan2d_recur_desc* desc, const void* x, const void* r, const void* i, const float* lam,
                          float* state, const int32_t* slots, int64_t slot_count, void* h, void* stream);

/* Bytes of `saved`, and of the workspace of a pass (SCAN2D_PASS_FWD, SCAN2D_PASS_BWD); 0 for an invalid descriptor. */
size_t scan2d_seq_recur_saved_bytes(const scan2d_recur_desc* desc);
size_t scan2d_seq_recur_workspace_bytes(const scan2d_recur_desc* desc, int pass);

/*
 * Group norm with an activation on channels-last tensors [N][P][C]: P positions (of a map, or of a sequence; 1 where every
 * token is normalised by itself), the C channels in G groups of C/G neighbours.  mean and var (biased) of item n and group g go over
 * its unmasked positions and the channels of the group:
 *     v[n,p,c] = (x[n,p,c] - mean[n,g]) * rstd[n,g] * gamma[c] + beta[c],    rstd = 1 / sqrt(var + eps),    y = act(v)
 *     SCAN2D_ACT_NONE: v      SCAN2D_ACT_SILU: v / (1 + exp(-v))      SCAN2D_ACT_GELU: v Phi(v), Phi the normal distribution
 * fp32 arithmetic (the variance from squared deviations), one rounding.
 *   mask : [N][P] uint8 or NULL; at a non-zero position x counts for nothing (whatever it holds, NaN included) and y is +0.
 *   An item without an unmasked position has mean 0, rstd 0 and y = 0.
 */
enum { SCAN2D_ACT_NONE = 0, SCAN2D_ACT_SILU = 1, SCAN2D_ACT_GELU = 2 };
typedef struct {
    int32_t  N, C, G;          /* items, channels, groups: >= 1, C a multiple of G; C < 2^24 */
    int64_t  P;                /* positions per item, >= 1; N * P < 2^31 - 4096 */
    int32_t  dtype;            /* SCAN2D_F32 or SCAN2D_BF16: type of x, y, dy, dx */
    int32_t  act;
    float    eps;              /* >= 0 */
    int64_t  stride_x, stride_y, stride_dy, stride_dx;     /* of the N * P rows, in elements; 0 = C */
} scan2d_group_norm_desc;

/*
 *   x : [N][P][C];  gamma, beta : [C] fp32, each may be NULL (1, 0);  y : [N][P][C], written, may be x itself
 *   (same stride then);  stats : [N][G][2] fp32, written: mean and rstd;
 *   workspace : at least scan2d_group_norm_workspace_bytes(desc, SCAN2D_PASS_FWD) bytes (NULL if that is 0).
 */
int scan2d_group_norm_fwd(const scan2d_group_norm_desc* desc, const void* x, const float* gamma, const float* beta,
                          const uint8_t* mask, void* y, float* stats, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Backward for a given dy = dL/dy and the stats that the forward wrote.  With xh = (x - mean) rstd, dv = dy act'(v) (0 where masked), M
 * the number of values of an item's group and sums over them:
 *     dbeta[c] = sum_{n,p} dv      dgamma[c] = sum_{n,p} dv xh
 *     dx = rstd * (dv gamma - (sum dv gamma + xh sum dv gamma xh) / M)          (+0 where masked)
 *   dx : [N][P][C], written, may be dy itself (same stride then) but not x;  dgamma, dbeta : [C] fp32, written, each may be NULL.
 */
int scan2d_group_norm_bwd(const scan2d_group_norm_desc* desc, const void* x, const float* gamma, const float* beta,
                          const uint8_t* mask, const float* stats, const void* dy, void* dx, float* dgamma, float* dbeta,
                          void* workspace, size_t workspace_bytes, void* stream);

size_t scan2d_group_norm_workspace_bytes(const scan2d_group_norm_desc* desc, int pass);

#ifdef __cplusplus
}
#endif
#endif /* SCAN2D_SEQ_H_ */
