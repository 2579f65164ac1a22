// Sequence layers on channels-last tensors (include/scan2d_seq.h): host-side entries used by the C ABI, and what their
// kernels share.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/scan2d_seq.h"

namespace scan2d {

int check_device();                      // scan2d_api.hip: SCAN2D_OK where the current device is a gfx950

// Arguments of the recurrence as the kernels take them; the strides are filled in (never 0).
struct RecurArgs {
    const void *x, *r, *i, *dh;
    const float *lam, *h0, *dhT;
    const int32_t *offsets, *lengths;
    void *h, *dx, *dr, *di;
    float *hT, *dlam, *dh0;
    float* saved;
    void* workspace;
    long long sx, sr, si, sh, sdh, sdx, sdr, sdi;
    int T, C, S, per;                    // per: rows of a sequence where offsets is null
    float scale;
};
size_t recur_saved_bytes(const scan2d_recur_desc* d);
size_t recur_workspace_bytes(const scan2d_recur_desc* d, int pass);
int recur_fwd_launch(const scan2d_recur_desc* d, const RecurArgs& a, hipStream_t stream);
int recur_bwd_launch(const scan2d_recur_desc* d, const RecurArgs& a, hipStream_t stream);
bool recur_step_fits(const scan2d_recur_desc* d);        // below 2^32 threads
int recur_step_launch(const scan2d_recur_desc* d, const RecurArgs& a, float* state, const int32_t* slots, long long slot_count, hipStream_t stream);

struct GroupNormArgs {
    const void *x, *dy;
    const float *gamma, *beta;
    const uint8_t* mask;
    void *y, *dx;
    float *stats, *dgamma, *dbeta;
    void* workspace;
    long long sx, sy, sdy, sdx;
    int N, P, C, G, D, act;              // D = C / G
    float eps;
};
size_t group_norm_workspace_bytes(const scan2d_group_norm_desc* d, int pass);
int group_norm_fwd_launch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, hipStream_t stream);
int group_norm_bwd_launch(const scan2d_group_norm_desc* d, const GroupNormArgs& a, hipStream_t stream);

}  // namespace scan2d
