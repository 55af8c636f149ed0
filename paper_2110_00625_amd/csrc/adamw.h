// Launch interface of the AdamW step (kavg_adamw).  The boundary (learner_api.hip) has checked every argument.
#pragma once
#include "kavg_internal.h"

namespace kavg {

// A tensor of a launch.  Its rows are cut into pieces of one workgroup each.
struct AdamwTensor {
    float* param; const void* grad; void* m; void* v; float* m_scale; float* v_scale; uint16_t* copy;
    int64_t cols, param_stride, grad_stride, copy_stride;
    uint32_t rows, pieces;                       // pieces of a row
    float decay;
    uint32_t site;                               // number of the tensor in the call
};

struct AdamwRule {
    float beta1, rest1, beta2, rest2, eps;       // rest = 1 - beta
    float rate, root_scale, grad_scale;          // rate = lr / (1 - beta1^t), root_scale = 1 / sqrt(1 - beta2^t)
    uint64_t step, seed;                         // seed: the step added to it (by the kernel, where that is in device memory)
    double lr, exact1, exact2, exact_eps;        // exact: the betas, for a step in device memory, and eps, for one outside of these limits:
    bool wide;                                   // eps is so small or so large that one of eps and 1 / eps is no normal number of fp32
    const int64_t* step_dev; const float* lr_dev; const float* grad_scale_dev;
};

hipError_t launch_adamw(int bits, int grad_dtype, const AdamwRule& rule, const kavg_adamw_tensor* tensors, int count, hipStream_t st);

}  // namespace kavg
