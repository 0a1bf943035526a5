// The root-mean-square norm in front of a layer, with the residual's addition in front of it, and rows put into 8 bits:
//     s = x + residual,  y = s / sqrt(mean(s^2) + eps) * weight,  output in bf16, fp32, or e4m3 codes with a scale for each row.
// A row is read once and stays in registers.  What bounds it: HBM (8192 rows of 4096, bf16 with residual to e4m3: 235 MB, 44 us, 5.3 TB/s of reads and writes mixed);
// few rows: the launch (1 row 2.9 us).
#include <algorithm>

#include "tiles.h"

namespace {

struct NormArgs {
    const unsigned char *x, *residual, *weight;   // (null: none)
    unsigned char *sum, *y;                       // (sum null: not asked for)
    float* scales;                                // of outputs in e4m3
    int64_t n, x_pitch;                           // (bytes)
    uint32_t d, units;                            // columns, pieces of 8 of them
    int waves;                                    // of a row
    int norm;                                     // 0: y = s
    double inv_d, eps;
};

constexpr int64_t kBusy = 4096;
constexpr float kE4m3Most = 448.0f, kLeastScale = 0x1p-126f;
// (rows begin at any element's address)
typedef uint32_t norm_u32x4_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t norm_u32x2_t __attribute__((ext_vector_type(2), aligned(1)));

// 8 elements from an element's address; `left` of them are there, the others 0
template <typename T> __device__ __forceinline__ void load8(float (&v)[8], const unsigned char* from, uint32_t left) {
    if (left >= 8) {
        const norm_u32x4_t a = *reinterpret_cast<const norm_u32x4_t*>(from);
        if constexpr (sizeof(T) == 4) {
            const norm_u32x4_t b = *reinterpret_cast<const norm_u32x4_t*>(from + 16);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = __uint_as_float(a[q]), v[4 + q] = __uint_as_float(b[q]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) v[2 * q] = __uint_as_float(a[q] << 16), v[2 * q + 1] = __uint_as_float(a[q] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (uint32_t q = 0; q < 8; ++q) v[q] = q < left ? td_load<T>(reinterpret_cast<const T*>(from) + q) : 0.0f;
    }
}

// f32: as they are; else two in a word, rounded to bf16
template <bool F32> __device__ __forceinline__ void store8(unsigned char* to, const float (&v)[8], uint32_t left) {
    if constexpr (F32) {
        if (left >= 8) {
            norm_u32x4_t a, b;
#pragma unroll
            for (int q = 0; q < 4; ++q) a[q] = __float_as_uint(v[q]), b[q] = __float_as_uint(v[4 + q]);
            *reinterpret_cast<norm_u32x4_t*>(to) = a;
            *reinterpret_cast<norm_u32x4_t*>(to + 16) = b;
        } else {
#pragma unroll
            for (uint32_t q = 0; q < 8; ++q)
                if (q < left) reinterpret_cast<float*>(to)[q] = v[q];
        }
    } else {
        norm_u32x4_t a;
#pragma unroll
        for (int q = 0; q < 4; ++q) a[q] = to_bf16x2(v[2 * q], v[2 * q + 1]);
        if (left >= 8) {
            *reinterpret_cast<norm_u32x4_t*>(to) = a;
        } else {
#pragma unroll
            for (uint32_t q = 0; q < 8; ++q)
                if (q < left) reinterpret_cast<bf16_t*>(to)[q] = (bf16_t)(a[q / 2] >> (16 * (q & 1)));
        }
    }
}

// A row's scale as it divides: 1 / scale in two parts, of which v (high + low) rounded once is v / scale rounded (high alone is off by a rounding, and where
// values have few bits that turns ties: of 960 rows of 4096 in bf16 52 had codes one step off).  low is not negative, so that zeros keep their sign.  Scales above
// 2^64 are made smaller by 2^64, as v is before it comes here, so that the low part has its bits.  It costs one instruction more for an element (2048 rows of 16384 22.5 us, with high alone 21.4).
struct CodeScale {
    float high, low;
    bool large;
};
__device__ __forceinline__ CodeScale code_scale(float scale) {
    CodeScale c;
    c.large = __builtin_amdgcn_readfirstlane(scale > 0x1p64f);
    const float s = c.large ? scale * 0x1p-64f : scale;
    c.high = 1.0f / s;
    if (fmaf(-s, c.high, 1.0f) < 0.0f) c.high = __uint_as_float(__float_as_uint(c.high) - 1);
    c.low = c.high > 0.0f ? fmaf(-s, c.high, 1.0f) * c.high : 0.0f;   // (an infinite scale: codes 0, and NaN of what is infinite)
    return c;
}

__device__ __forceinline__ void store_codes(unsigned char* to, const float (&v)[8], const CodeScale& by, uint32_t left) {
    norm_u32x2_t c = {0, 0};
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = fmaf(v[i], by.high, v[i] * by.low);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int w = 0;
        w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h], q[4 * h + 1], w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h + 2], q[4 * h + 3], w, true);
        c[h] = (uint32_t)w;
    }
    if (left >= 8) {
        *reinterpret_cast<norm_u32x2_t*>(to) = c;
    } else {
#pragma unroll
        for (uint32_t q = 0; q < 8; ++q)
            if (q < left) to[q] = (unsigned char)(c[q / 4] >> (8 * (q & 3)));
    }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// s / rms = ldexp(s, -half) * factor: the squares are summed in 64 bits and the exponent is taken out, so that rows of any magnitude that
// fp32 holds have the norm of the formula (a row of zeros with eps = 0: zeros).
struct RowScale {
    int half;
    float factor;
};
__device__ __forceinline__ RowScale row_scale(double sum, const NormArgs& p) {
    const double v = sum * p.inv_d + p.eps;
    RowScale r;
    r.half = __builtin_amdgcn_frexp_exp(v) >> 1;
    r.factor = v > 0.0 || v != v ? (float)(1.0 / sqrt(__builtin_amdgcn_ldexp(v, -2 * r.half))) : 0.0f;
    return r;
}

// U pieces of 8 elements of a thread stay in registers; U = 0: rows of any length, read again for each step.  OUT: tardis_dtype_t.
template <typename T, int OUT, int U>
__global__ void __launch_bounds__(1024) rms_norm_kernel(NormArgs p) {
    constexpr bool KEPT = U > 0;
    constexpr int N = KEPT ? U : 1;
    __shared__ double sums[16];
    __shared__ float tops[16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), mine = wave % p.waves;
    const int64_t row = (int64_t)blockIdx.x * ((int)(blockDim.x >> 6) / p.waves) + wave / p.waves;
    const bool there = row < p.n;                 // (no return: all wavefronts come to the barriers)
    const uint32_t step = (uint32_t)p.waves * 64u, first = (uint32_t)(mine * 64 + lane), units = there ? p.units : 0u;
    const unsigned char* x = p.x + row * p.x_pitch;
    const int64_t at = row * (int64_t)p.d;
    auto summand = [&](uint32_t u, float (&s)[8]) {
        const uint32_t left = p.d - u * 8u;
        load8<T>(s, x + (size_t)u * 8 * sizeof(T), left);
        if (p.residual) {
            float r[8];
            load8<T>(r, p.residual + (at + (int64_t)u * 8) * sizeof(T), left);
#pragma unroll
            for (int q = 0; q < 8; ++q) s[q] += r[q];
        }
    };
    auto weighed = [&](uint32_t u, float (&s)[8], const RowScale& r) {
        if (p.norm) {
#pragma unroll
            for (int q = 0; q < 8; ++q) s[q] = __builtin_amdgcn_ldexpf(s[q], -r.half) * r.factor;
        }
        if (p.weight) {
            float w[8];
            load8<T>(w, p.weight + (size_t)u * 8 * sizeof(T), p.d - u * 8u);
#pragma unroll
            for (int q = 0; q < 8; ++q) s[q] *= w[q];
        }
    };
    auto over_row = [&](auto f) {                  // f(piece, kept values of it)
        if constexpr (KEPT) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t u = first + (uint32_t)i * step;
                if (u < units) f(u, i);
            }
        } else {
            for (uint32_t u = first; u < units; u += step) f(u, 0);
        }
    };
    float s[N][8];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) s[i][q] = 0.0f;
    RowScale r{0, 1.0f};
    double sum = 0.0;
    if (KEPT || p.norm)
        over_row([&](uint32_t u, int i) {
            summand(u, s[i]);
#pragma unroll
            for (int q = 0; q < 8; ++q) sum += (double)s[i][q] * (double)s[i][q];
        });
    if (p.norm) {
        sum = wave_sum(sum);
        if (p.waves > 1) {
            if (lane == 0) sums[wave] = sum;
            __syncthreads();
            sum = 0.0;
            for (int w = 0; w < p.waves; ++w) sum += sums[wave - mine + w];
        }
        r = row_scale(sum, p);
    }
    if (KEPT && p.sum) over_row([&](uint32_t u, int i) { store8<sizeof(T) == 4>(p.sum + (at + (int64_t)u * 8) * sizeof(T), s[i], p.d - u * 8u); });
    if constexpr (OUT == TARDIS_FP8_E4M3) {
        float top = 0.0f;
        over_row([&](uint32_t u, int i) {
            if (!KEPT) summand(u, s[i]);
            weighed(u, s[i], r);
#pragma unroll
            for (int q = 0; q < 8; ++q) top = fmaxf(top, fabsf(s[i][q]));
        });
        top = td_wave_max(top);
        if (p.waves > 1) {
            if (lane == 0) tops[wave] = top;
            __syncthreads();
            for (int w = 0; w < p.waves; ++w) top = fmaxf(top, tops[wave - mine + w]);
        }
        const float scale = fmaxf(top / kE4m3Most, kLeastScale);
        const CodeScale by = code_scale(scale);
        auto smaller = [&](int i) {
#pragma unroll
            for (int q = 0; q < 8; ++q) s[i][q] *= 0x1p-64f;
        };
        if (KEPT && by.large) over_row([&](uint32_t, int i) { smaller(i); });
        if (there && mine == 0 && lane == 0) p.scales[row] = scale;
        over_row([&](uint32_t u, int i) {
            const uint32_t left = p.d - u * 8u;
            if (!KEPT) {
                summand(u, s[i]);
                if (p.sum) store8<sizeof(T) == 4>(p.sum + (at + (int64_t)u * 8) * sizeof(T), s[i], left);
                weighed(u, s[i], r);
                if (by.large) smaller(i);
            }
            store_codes(p.y + at + (int64_t)u * 8, s[i], by, left);
        });
    } else {
        over_row([&](uint32_t u, int i) {
            const uint32_t left = p.d - u * 8u;
            if (!KEPT) {
                summand(u, s[i]);
                if (p.sum) store8<sizeof(T) == 4>(p.sum + (at + (int64_t)u * 8) * sizeof(T), s[i], left);
            }
            weighed(u, s[i], r);
            store8<OUT == TARDIS_F32>(p.y + (at + (int64_t)u * 8) * (OUT == TARDIS_F32 ? 4 : 2), s[i], left);
        });
    }
}

template <typename T, int OUT> void launch(const NormArgs& p, int each, dim3 grid, dim3 block, hipStream_t s) {
    if (each == 1) hipLaunchKernelGGL((rms_norm_kernel<T, OUT, 1>), grid, block, 0, s, p);
    else if (each == 2) hipLaunchKernelGGL((rms_norm_kernel<T, OUT, 2>), grid, block, 0, s, p);
    else if (each == 4) hipLaunchKernelGGL((rms_norm_kernel<T, OUT, 4>), grid, block, 0, s, p);
    else if (each == 8) hipLaunchKernelGGL((rms_norm_kernel<T, OUT, 8>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((rms_norm_kernel<T, OUT, 0>), grid, block, 0, s, p);
}

template <typename T> void launch(const NormArgs& p, int out, int each, dim3 grid, dim3 block, hipStream_t s) {
    if (out == TARDIS_FP8_E4M3) launch<T, TARDIS_FP8_E4M3>(p, each, grid, block, s);
    else if (out == TARDIS_F32) launch<T, TARDIS_F32>(p, each, grid, block, s);
    else launch<T, TARDIS_BF16>(p, each, grid, block, s);
}

}  // namespace

tardis_status_t td_rms_norm(const void* x, int64_t n, int64_t d, int64_t x_pitch, int32_t dtype, int norm, float eps, const void* weight,
                            const void* residual, void* sum, void* y, float* scales, int32_t out_dtype, hipStream_t s) {
    NormArgs p{};
    p.x = static_cast<const unsigned char*>(x);
    p.residual = static_cast<const unsigned char*>(residual);
    p.weight = static_cast<const unsigned char*>(weight);
    p.sum = static_cast<unsigned char*>(sum);
    p.y = static_cast<unsigned char*>(y);
    p.scales = scales;
    p.n = n;
    p.x_pitch = x_pitch * (int64_t)td_elem_size(dtype);
    p.d = (uint32_t)d;
    p.units = (uint32_t)((d + 7) / 8);
    p.norm = norm;
    p.inv_d = 1.0 / (double)d;
    p.eps = (double)eps;
    // Pieces of a thread and wavefronts of a row.  Outputs in bf16 and fp32: as many wavefronts as the row divides into (8192 rows of 4096 in bf16, us: 1, 2 and 4
    // pieces of a thread 45.2, 47.2, 51.7).  Codes, for which the wavefronts wait for one another a second time: as few as keep 4096 of them
    // busy (16 for each CU), so that fewer rows are divided among more (2048 rows of 4096 with residual, us: 1, 2, 4 and 8 pieces 14.3, 13.3, 12.8, 15.6; 1000 of
    // 11008 17.1, 19.6, 17.2, 20.7); with four times as many rows two pieces in place of four, unless a row then takes more than 8 wavefronts (8192 rows of 4096
    // 47.1, 44.4, 48.1, 50.3; 4096 of 8192 55.0, 45.0, 47.8, 49.9; 16384 of 4096 95.1, 89.5, 97.4, 110; without residual 2048 of 16384 21.3, 23.1,
    // 21.2, 22.9).  8 pieces only for rows that need them.
    const bool codes = out_dtype == TARDIS_FP8_E4M3;
    int each = (int64_t)(p.units + 255) / 256 <= 16 ? 4 : 8;
    auto waves_of = [&](int u) { return (int64_t)(p.units + 64 * u - 1) / (64 * u); };
    while (each > 1 && (!codes || n * waves_of(each) < kBusy) && waves_of(each / 2) <= 16) each /= 2;
    if (codes && each == 4 && n * waves_of(4) >= 4 * kBusy && waves_of(2) <= 8) each = 2;
    p.waves = (int)std::min<int64_t>(16, waves_of(each));
    if (waves_of(each) > 16) each = 0;                                 // (rows that do not fit into registers)
    const int rows = std::max(1, 4 / p.waves), threads = 64 * p.waves * rows;
    const int64_t most = kMostThreads / threads;                       // blocks of a launch
    const int64_t blocks = (n + rows - 1) / rows;
    for (int64_t b = 0; b < blocks; b += most) {
        const dim3 grid((unsigned)std::min(most, blocks - b)), block((unsigned)threads);
        NormArgs q = p;
        const int64_t row = b * rows;
        q.x += row * p.x_pitch;
        if (q.residual) q.residual += row * d * (int64_t)td_elem_size(dtype);
        if (q.sum) q.sum += row * d * (int64_t)td_elem_size(dtype);
        q.y += row * d * (out_dtype == TARDIS_FP8_E4M3 ? 1 : (int64_t)td_elem_size(out_dtype));
        if (q.scales) q.scales += row;
        q.n = n - row;
        if (dtype == TARDIS_F32) launch<float>(q, out_dtype, each, grid, block, s);
        else launch<bf16_t>(q, out_dtype, each, grid, block, s);
    }
    TD_HIP(hipGetLastError());
    return TARDIS_OK;
}
