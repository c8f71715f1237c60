// Arguments of the RMS norm's launchers, as the entry points check them.
#pragma once

#include "masked_load.cuh"
#include "recurrent_b200.h"

namespace conv2d_b200 {

struct RmsArgs {
    const void *x, *residual, *z, *dy, *dh;
    const float *gamma, *rstd_in;
    void *y, *h, *y8, *dx, *dz;
    float *scales, *rstd, *dgamma, *ws;
    int M, C, G, block;
    long long ldx, ldr, ldz, ldy, ldh, ld8, lddy, lddh, lddx, lddz;
    float eps;
};
conv2d_status_t launch_rms_fwd(const RmsArgs& a, conv2d_operand_t type, cudaStream_t stream);
conv2d_status_t launch_rms_bwd(const RmsArgs& a, conv2d_operand_t type, cudaStream_t stream);
size_t rms_bwd_workspace_bytes(int M, int C, int G);
constexpr int kMaxRmsChannels = 16384;                          // of a row, which lies in one block's registers

}  // namespace conv2d_b200
