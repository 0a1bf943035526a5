// The linear layer's large tiles in bf16
#include "linear_quad.h"

namespace {

template <bool GROUPED, int NA, int NB>
__global__ void __launch_bounds__(256, 1) linear_quad_kernel(LinearArgs p) {
    linear_quad<bf16_t, GROUPED, NA, NB>(p);
}

template <typename F> void for_quad_shape(int shape, F f) {
    switch (shape) {
        case 0: f(num<8>{}, num<8>{}); break;
        case 1: f(num<6>{}, num<8>{}); break;
        default: f(num<8>{}, num<4>{}); break;
    }
}

}  // namespace

tardis_status_t td_linear_init_quad() {
    static td_once once;
    return once.run([]() -> tardis_status_t {
        bool ok = true;
        for (int shape = 0; shape < kLinearQuads; ++shape)
            for_quad_shape(shape, [&](auto na, auto nb) {
                typedef LinearQuad<na, nb> G;
                ok &= kLinearQuad[shape].m == G::TM && kLinearQuad[shape].n == G::TN && kLinearQuad[shape].slice == G::SL;
                auto raise = [&](auto kernel) {
                    ok &= hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds) == hipSuccess;
                };
                raise(linear_quad_kernel<false, na, nb>);
                raise(linear_quad_kernel<true, na, nb>);
            });
        return ok ? TARDIS_OK : TARDIS_ERR_HIP;
    });
}

void td_linear_launch_quad(const LinearArgs& p, bool grouped, int shape, int blocks, hipStream_t s) {
    for_quad_shape(shape, [&](auto na, auto nb) {
        constexpr int bytes = LinearQuad<na, nb>::kLds;
        if (grouped) hipLaunchKernelGGL((linear_quad_kernel<true, na, nb>), dim3((unsigned)blocks), dim3(256), bytes, s, p);
        else hipLaunchKernelGGL((linear_quad_kernel<false, na, nb>), dim3((unsigned)blocks), dim3(256), bytes, s, p);
    });
}
