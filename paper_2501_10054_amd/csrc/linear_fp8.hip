// The linear layer for x and W in e4m3 with a scale for each row: linear_tile.h's tiles
#include "linear_tile.h"

namespace {

template <typename T, bool DIRECT, int FA, int FB, int WM, int WN, int WK, int KS, int D>
__global__ void __launch_bounds__(64 * WM * WN * WK, 2) linear_fp8_kernel(LinearArgs p) {
    linear_tile<T, false, DIRECT, FA, FB, WM, WN, WK, KS, D>(p);
}

// f(direct, row and column blocks of a wavefront, grid of wavefronts, wavefronts and half-lines of each in K, slices in LDS)
template <typename F> void for_fp8_tile(bool direct, int shape, F f) {
    if (direct) {
        switch (shape) {
            case 0: f(std::true_type{}, num<1>{}, num<1>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<5>{}); break;
            case 1: f(std::true_type{}, num<1>{}, num<2>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<3>{}); break;
            case 2: f(std::true_type{}, num<1>{}, num<1>{}, num<1>{}, num<1>{}, num<8>{}, num<2>{}, num<5>{}); break;
            case 3: f(std::true_type{}, num<2>{}, num<1>{}, num<1>{}, num<2>{}, num<4>{}, num<2>{}, num<5>{}); break;
            case 4: f(std::true_type{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<5>{}); break;
            case 5: f(std::true_type{}, num<4>{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}); break;
            case 6: f(std::true_type{}, num<4>{}, num<4>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<2>{}); break;
            case 7: f(std::true_type{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<2>{}); break;
            case 8: f(std::true_type{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<4>{}, num<2>{}, num<3>{}); break;
            case 9: f(std::true_type{}, num<2>{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<3>{}); break;
            default: f(std::true_type{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<3>{}); break;
        }
    } else {
        switch (shape) {
            case 0: f(std::false_type{}, num<1>{}, num<1>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<6>{}); break;
            case 1: f(std::false_type{}, num<2>{}, num<1>{}, num<1>{}, num<2>{}, num<4>{}, num<1>{}, num<4>{}); break;
            case 2: f(std::false_type{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<4>{}); break;
            default: f(std::false_type{}, num<4>{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}); break;
        }
    }
}

// f(element type, what for_fp8_tile gives)
template <typename F> void for_fp8_shape(bool direct, int shape, bool out_f32, F f) {
    for_fp8_tile(direct, shape, [&](auto d, auto fa, auto fb, auto wm, auto wn, auto wk, auto ks, auto ring) {
        if constexpr (decltype(d)::value && decltype(ks)::value % 2 == 0) {
            if (shape >= kLinearNearFp8 && !out_f32) return f(e4m3_near_t{}, d, fa, fb, wm, wn, wk, ks, ring);
        }
        f(e4m3_t{}, d, fa, fb, wm, wn, wk, ks, ring);
    });
}

}  // namespace

tardis_status_t td_linear_init_fp8() {
    static td_once once;
    return once.run([]() -> tardis_status_t {
        bool ok = true;
        for (int direct = 0; direct < 2; ++direct)
            for (int shape = 0; shape < (direct ? kLinearShapesFp8 : kLinearStagedShapesFp8); ++shape)
                for (int out_f32 = 0; out_f32 < 2; ++out_f32)
                    for_fp8_shape(direct, shape, out_f32, [&](auto type, auto d, auto fa, auto fb, auto wm, auto wn, auto wk, auto ks, auto ring) {
                        typedef LinearTile<decltype(type), decltype(d)::value, fa, fb, wm, wn, wk, ks, ring> G;
                        const LinearShape& is = direct ? kLinearShapeFp8[shape] : kLinearStagedFp8[shape];
                        ok &= is.m == G::TM && is.n == G::TN && is.slice == G::SL;
                        ok &= hipFuncSetAttribute(reinterpret_cast<const void*>(linear_fp8_kernel<decltype(type), decltype(d)::value, fa, fb, wm, wn, wk, ks, ring>),
                                                  hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds) == hipSuccess;
                    });
        return ok ? TARDIS_OK : TARDIS_ERR_HIP;
    });
}

void td_linear_launch_fp8(const LinearArgs& p, bool direct, int shape, int blocks, hipStream_t s) {
    for_fp8_shape(direct, shape, p.out_f32, [&](auto type, auto d, auto fa, auto fb, auto wm, auto wn, auto wk, auto ks, auto ring) {
        typedef LinearTile<decltype(type), decltype(d)::value, fa, fb, wm, wn, wk, ks, ring> G;
        constexpr int bytes = G::kLds, threads = 64 * G::W;
        hipLaunchKernelGGL((linear_fp8_kernel<decltype(type), decltype(d)::value, fa, fb, wm, wn, wk, ks, ring>), dim3((unsigned)blocks), dim3(threads), bytes, s, p);
    });
}
