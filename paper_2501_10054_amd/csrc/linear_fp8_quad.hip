// The linear layer's large tiles for x and W in e4m3, outputs in bf16 whose sums need not be exact
#include "linear_quad.h"

namespace {

template <int NA, int NB>
__global__ void __launch_bounds__(256, 1) linear_fp8_quad_kernel(LinearArgs p) {
    linear_quad<e4m3_near_t, false, NA, NB>(p);
}

template <typename F> void for_fp8_quad_shape(int shape, F f) {
    if (shape == 0) f(num<8>{}, num<4>{});
}

}  // namespace

tardis_status_t td_linear_init_fp8_quad() {
    static td_once once;
    return once.run([]() -> tardis_status_t {
        bool ok = true;
        for (int shape = 0; shape < kLinearQuadsFp8; ++shape)
            for_fp8_quad_shape(shape, [&](auto na, auto nb) {
                typedef LinearQuad<na, nb> G;
                ok &= kLinearQuadFp8[shape].m == G::TM && kLinearQuadFp8[shape].n == G::TN && kLinearQuadFp8[shape].slice == G::SL;
                ok &= hipFuncSetAttribute(reinterpret_cast<const void*>(linear_fp8_quad_kernel<na, nb>), hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds) == hipSuccess;
            });
        return ok ? TARDIS_OK : TARDIS_ERR_HIP;
    });
}

void td_linear_launch_fp8_quad(const LinearArgs& p, int shape, int blocks, hipStream_t s) {
    for_fp8_quad_shape(shape, [&](auto na, auto nb) {
        constexpr int bytes = LinearQuad<na, nb>::kLds;
        hipLaunchKernelGGL((linear_fp8_quad_kernel<na, nb>), dim3((unsigned)blocks), dim3(256), bytes, s, p);
    });
}
