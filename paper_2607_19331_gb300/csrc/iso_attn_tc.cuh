// iso_attn_tc.cuh -- the tensor-core kernels of attention, as its entry points
// (iso_attn.cu) see them.
#pragma once

#include "iso_attn.cuh"

namespace iso {

// the time after which a wait of these kernels gives up, ns
uint64_t attn_wait_ns();

// Forward (iso_attn_fwd.cu).  Parts that the keys are cut into, and the bytes of
// the parts' sums.
struct AttnPlan {
    int parts;
    size_t bytes;
};
AttnPlan attn_plan(long long q_rows, long long k_rows, const iso_attn_cfg& c);
// `part`: AttnPlan::bytes
int attn_tc(const AttnArgs& g, const AttnPlan& p, float* part, cudaStream_t s);

// Backward (iso_attn_grad.cu).  Parts of a key head's query heads that have sums
// of their own, and the bytes of those sums.
struct AttnGradPlan {
    int parts;
    size_t bytes;
};
AttnGradPlan attn_grad_plan(long long q_rows, long long k_rows, const iso_attn_cfg& c);
// `part`: AttnGradPlan::bytes.  delta has been enqueued before.
int attn_grad_tc(const AttnArgs& g, const AttnGradPlan& p, float* part, cudaStream_t s);

}  // namespace iso
