// The norms between two blocks (llsa_norm_*): the host plan and what the kernels are given.
#pragma once
#include "llsa_internal.h"

namespace llsa {

struct NormShape {
    int tpr, nv;                    // threads a row, 16-byte vectors a thread
    int blocks;                     // workgroups a batch entry
};
struct NormPlan {
    llsa_norm_desc desc;
    NormShape fwd, bwd;
    size_t ws;
};

struct NormArgs {
    const char *x, *branch, *dy, *dx_out;      // backward: x is x'
    char *x_out, *y, *dx, *dbranch;
    const float *gain, *gain_branch;
    const char *gate, *scale, *shift;
    float *stats, *part;                       // part: [batch][workgroup][3][C]
    float *dgain, *dgain_branch, *dgate, *dscale, *dshift;
    int64_t N, mod_stride;
    int32_t C, batch, blocks, mod_f32;
    float eps, alpha, inv_c;
};

void norm_layout(NormPlan &p);
hipError_t launch_norm_forward(const NormPlan &p, NormArgs a, hipStream_t s);
hipError_t launch_norm_backward(const NormPlan &p, NormArgs a, hipStream_t s);

}  // namespace llsa
