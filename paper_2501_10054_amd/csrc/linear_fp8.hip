// The linear layer for x and W in e4m3 with a scale for each row: linear_tile.h's tiles.  Weights from HBM: one token 16384 -> 4096 16.2 us, 67 MB, 4.1 TB/s
// (launch and first bytes 5 us); 333 tokens 11008 -> 4096 with a residual 40 us, 0.75 PFLOP/s.  Weights that stay in the 256 MB of cache between calls: 14.5 and 33 us.
#include "linear_tile.h"

namespace {

template <typename T, bool DIRECT, int FA, int FB, int WM, int WN, int WK, int KS, int D>
__global__ void __launch_bounds__(64 * WM * WN * WK, 2) linear_fp8_kernel(LinearArgs p) {
    linear_tile<T, false, DIRECT, FA, FB, WM, WN, WK, KS, D>(p);
}

// f(element type, direct, row and column blocks of a wavefront, grid of wavefronts, wavefronts and half-lines of each in K, slices in LDS)
template <typename F> void for_fp8_shape(bool direct, int shape, bool near, F f) {
    auto use = [&](auto number, auto d, auto... tile) {
        constexpr int s = decltype(number)::value;
        constexpr bool DIRECT = decltype(d)::value;
        if constexpr (DIRECT && s >= kLinearNearFp8) {
            if (near) return f(e4m3_near_t{}, d, tile...);
        }
        if constexpr (linear_has_fp8(DIRECT, !DIRECT || s < kLinearNearFp8, s)) f(e4m3_t{}, d, tile...);
    };
    if (direct) {
        switch (shape) {
            case 0: use(num<0>{}, std::true_type{}, num<1>{}, num<1>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<5>{}); break;
            case 1: use(num<1>{}, std::true_type{}, num<1>{}, num<2>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<3>{}); break;
            case 2: use(num<2>{}, std::true_type{}, num<1>{}, num<1>{}, num<1>{}, num<1>{}, num<8>{}, num<2>{}, num<5>{}); break;
            case 3: use(num<3>{}, std::true_type{}, num<2>{}, num<1>{}, num<1>{}, num<2>{}, num<4>{}, num<2>{}, num<5>{}); break;
            case 4: use(num<4>{}, std::true_type{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<5>{}); break;
            case 5: use(num<5>{}, std::true_type{}, num<4>{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}); break;
            case 6: use(num<6>{}, std::true_type{}, num<4>{}, num<4>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<2>{}); break;
            case 7: use(num<7>{}, std::true_type{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<2>{}); break;
            case 8: use(num<8>{}, std::true_type{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<4>{}, num<2>{}, num<3>{}); break;
            case 9: use(num<9>{}, std::true_type{}, num<2>{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<3>{}); break;
            default: use(num<10>{}, std::true_type{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<3>{}); break;
        }
    } else {
        switch (shape) {
            case 0: use(num<0>{}, std::false_type{}, num<1>{}, num<1>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<6>{}); break;
            case 1: use(num<1>{}, std::false_type{}, num<2>{}, num<1>{}, num<1>{}, num<2>{}, num<4>{}, num<1>{}, num<4>{}); break;
            case 2: use(num<2>{}, std::false_type{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<4>{}); break;
            default: use(num<3>{}, std::false_type{}, num<4>{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}); break;
        }
    }
}

}  // namespace

tardis_status_t td_linear_init_fp8() {
    static td_once once;
    return once.run([]() -> tardis_status_t {
        bool ok = true;
        for (int direct = 0; direct < 2; ++direct)
            for (int shape = 0; shape < (direct ? kLinearShapesFp8 : kLinearStagedShapesFp8); ++shape)
                for (int near = 0; near < 2; ++near)
                    for_fp8_shape(direct, shape, near, [&](auto type, auto d, auto fa, auto fb, auto wm, auto wn, auto wk, auto ks, auto ring) {
                        typedef LinearTile<decltype(type), decltype(d)::value, fa, fb, wm, wn, wk, ks, ring> G;
                        const LinearShape& is = direct ? kLinearShapeFp8[shape] : kLinearStagedFp8[shape];
                        ok &= is.m == G::TM && is.n == G::TN && is.slice == G::SL;
                        ok &= hipFuncSetAttribute(reinterpret_cast<const void*>(linear_fp8_kernel<decltype(type), decltype(d)::value, fa, fb, wm, wn, wk, ks, ring>),
                                                  hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds) == hipSuccess;
                    });
        return ok ? TARDIS_OK : TARDIS_ERR_HIP;
    });
}

void td_linear_launch_fp8(const LinearArgs& p, bool direct, bool near, int shape, int blocks, hipStream_t s) {
    for_fp8_shape(direct, shape, near, [&](auto type, auto d, auto fa, auto fb, auto wm, auto wn, auto wk, auto ks, auto ring) {
        typedef LinearTile<decltype(type), decltype(d)::value, fa, fb, wm, wn, wk, ks, ring> G;
        constexpr int bytes = G::kLds, threads = 64 * G::W;
        hipLaunchKernelGGL((linear_fp8_kernel<decltype(type), decltype(d)::value, fa, fb, wm, wn, wk, ks, ring>), dim3((unsigned)blocks), dim3(threads), bytes, s, p);
    });
}
