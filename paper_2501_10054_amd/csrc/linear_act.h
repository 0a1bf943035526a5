// The activations of the linear layer's epilogues.
#pragma once
#include "linear.h"
#include "sigma.h"
#include "tiles.h"

namespace {

// GELU for outputs in bf16 to which nothing is added (an activation of its own for the kernels, kActGelu16): z Phi(z) from
// Phi(-|z|) = t exp(P(t) - z^2 / 2), t = 1 / (1 + 0.26 |z|) at every z, with P of degree 4, a minimax fit: Phi(-|z|) is off by 3.4e-5 of itself, a
// hundredth of what the rounding to bf16 moves a value by, so that 0.2 % of the results are the second nearest value (z from N(0, 1.6^2)).  Half the
// instructions of act_flat's, which is for fp32 outputs (2048 x 16384 x 4096, us: without an activation 198.1, with this one 212.7, with act_flat's 216.3).
// A residual may take the result away and leave the error (13 times what act_flat's may be, with residuals of -GELU), so calls with one have act_flat's
// (us: without an activation 243, with act_flat's 275; with this one it was 255).
template <int ACT> __device__ __forceinline__ float linear_act(float z) {
    if constexpr (ACT == kActGelu16) {
        const float u = fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(0.26f, u, 1.0f));
        float p = -0.55232652f;                                     // (in units of log 2)
        p = fmaf(p, t, 1.06301336f);
        p = fmaf(p, t, 0.23485752f);
        p = fmaf(p, t, 1.53103406f);
        p = fmaf(p, t, -3.2766187f);
        const float q = t * __builtin_amdgcn_exp2f(fmaf(u * -0.721347520f, u, p));
        return z * (z > 0.0f ? 1.0f - q : q);
    } else if constexpr (ACT == TARDIS_ACT_RELU) {
        return z <= 0.0f ? 0.0f : z;                                // (a NaN stays one; act_flat has 0 for it)
    } else {
        return act_flat<ACT>(z);
    }
}

template <typename F> __device__ __forceinline__ void with_linear_act(int act, F f) {
    if (act == kActGelu16) f(num<kActGelu16>{});
    else with_act(act, f);
}

}  // namespace
