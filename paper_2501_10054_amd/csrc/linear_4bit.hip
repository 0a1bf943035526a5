// The linear layer with 4-bit weights: y = sigma(sum_G scale_jG sum_(k in G) (q_jk - zero_jG) x_k + b_j) + r.
//
// A code q becomes a bf16 value without a conversion: put under the exponent of 16, with the weight 1 three bits up in the mantissa, it is 16 + q, and
// a word's layout is such that a shift, an and and an or make two neighbouring columns at once.  16 + zero is multiplied with the same tokens by matrix
// instructions that take it away again, so that an accumulator holds sum (q - zero) x of a group, every product exact; the group's scale goes to
// the sum.  Tokens in fp32 are three bf16 parts each, which together hold all of their 24 bits.
#include <algorithm>

#include "linear_act.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));
template <int N> struct words_of { typedef uint32_t type __attribute__((ext_vector_type(N))); };
template <> struct words_of<1> { typedef uint32_t type; };

struct FourArgs {
    const unsigned char* x;
    const uint32_t* W;
    const void *scales, *b, *r;
    const uint8_t* zeros;
    void* y;
    float* part;                   // not null: sums of one range of K each go here, [range][n][N], and nothing else is done
    int64_t n, N, x_pitch;         // (bytes)
    uint32_t k, groups;            // columns; groups of a row
    int act, out_f32, tiles_n, splits;
};

constexpr int kWaves = 8;

__device__ __forceinline__ f32x4_t mma(const td_u32x4& w, const td_u32x4& x, const f32x4_t& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, x), c, 0, 0, 0);
}

// 16 + q of the eight codes of a word, in bf16
__device__ __forceinline__ td_u32x4 sixteen_more(uint32_t w) {
    return {(w << 3 & 0x00780078u) | 0x41804180u, (w >> 1 & 0x00780078u) | 0x41804180u, (w >> 5 & 0x00780078u) | 0x41804180u, (w >> 9 & 0x00780078u) | 0x41804180u};
}
// -(16 + z), twice in a word
__device__ __forceinline__ uint32_t sixteen_less(uint32_t z) {
    return (__float_as_uint(-16.0f - (float)min(z, 128u)) >> 16) * 0x10001u;
}

// The eight columns of a token that a matrix instruction takes of a lane, as parts in bf16 (fp32: head, middle, end)
template <typename T> struct Token {
    static constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    td_u32x4 part[PARTS];
};
__device__ __forceinline__ void split(Token<float>& t, const float (&v)[8]) {
    float rest[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) rest[q] = v[q];
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t w = to_bf16x2(rest[2 * q], rest[2 * q + 1]);
            t.part[i][q] = w;
            rest[2 * q] -= __uint_as_float(w << 16);
            rest[2 * q + 1] -= __uint_as_float(w & 0xffff0000u);
        }
}
template <typename T> __device__ __forceinline__ void load_token(Token<T>& t, const unsigned char* at) {
    const u32x4_any_t a = *reinterpret_cast<const u32x4_any_t*>(at);
    if constexpr (sizeof(T) == 2) {
        t.part[0] = a;
    } else {
        const u32x4_any_t b = *reinterpret_cast<const u32x4_any_t*>(at + 16);
        const float v[8] = {__uint_as_float(a[0]), __uint_as_float(a[1]), __uint_as_float(a[2]), __uint_as_float(a[3]),
                            __uint_as_float(b[0]), __uint_as_float(b[1]), __uint_as_float(b[2]), __uint_as_float(b[3])};
        split(t, v);
    }
}
// `left` of them are there, the others 0
template <typename T> __device__ __forceinline__ void load_token_end(Token<T>& t, const unsigned char* at, int left) {
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = q < left ? td_load<T>(reinterpret_cast<const T*>(at) + q) : 0.0f;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int q = 0; q < 4; ++q) t.part[0][q] = __float_as_uint(v[2 * q]) >> 16 | (__float_as_uint(v[2 * q + 1]) & 0xffff0000u);
    } else {
        split(t, v);
    }
}

// A block has 16 rows of W and 16 TT tokens, its wavefronts every eighth group of a range of K.  GW: words of a group in a lane (32 GW columns a group).
// Lane l holds, of W's row l % 16, the columns 8 GW (l / 16) .. of a group, which is one load, and the same columns of token l % 16.
template <typename T, int GW, int TT>
__global__ void __launch_bounds__(64 * kWaves, 2) linear4_kernel(FourArgs p) {
    typedef typename words_of<GW>::type words_t;
    constexpr int D = 4;                           // groups whose weights are under way together
    __shared__ f32x4_t sums[kWaves * TT * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), low = lane & 15, high = lane >> 4;
    const int tile_n = (int)(blockIdx.x % (uint32_t)p.tiles_n), rest = (int)(blockIdx.x / (uint32_t)p.tiles_n), range = rest % p.splits, tile_m = rest / p.splits;
    const int64_t n0 = (int64_t)tile_n * 16, m0 = (int64_t)tile_m * (16 * TT);
    // (rows and tokens that are not there: the last one's, of which nothing is kept)
    const int64_t row = min(n0 + low, p.N - 1);
    const uint32_t* W = p.W + row * ((int64_t)p.groups * (4 * GW)) + high * GW;
    const uint8_t* zeros = p.zeros ? p.zeros + row * p.groups : nullptr;
    const T* scales[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) scales[q] = static_cast<const T*>(p.scales) + min(n0 + 4 * high + q, p.N - 1) * (int64_t)p.groups;
    const unsigned char* x[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) x[t] = p.x + min(m0 + 16 * t + low, p.n - 1) * p.x_pitch + high * (8 * GW) * sizeof(T);

    f32x4_t acc[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t] = f32x4_t{0, 0, 0, 0};
    auto add = [&](uint32_t g, const words_t& w, uint32_t zero, const float (&scale)[4], auto load) {
        f32x4_t c[TT];
#pragma unroll
        for (int t = 0; t < TT; ++t) c[t] = f32x4_t{0, 0, 0, 0};
        const uint32_t less = sixteen_less(zero);
#pragma unroll
        for (int s = 0; s < GW; ++s) {
            uint32_t word;
            if constexpr (GW == 1) word = w;
            else word = w[s];
            const td_u32x4 codes = sixteen_more(word);
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                Token<T> v;
                load(v, x[t] + ((size_t)g * (32 * GW) + 8 * s) * sizeof(T), (int)p.k - (int)(g * (32 * GW) + high * (8 * GW) + 8 * s));
#pragma unroll
                for (int i = 0; i < Token<T>::PARTS; ++i) {
                    c[t] = mma(codes, v.part[i], c[t]);
                    c[t] = mma(td_u32x4{less, less, less, less}, v.part[i], c[t]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[t][q] = fmaf(scale[q], c[t][q], acc[t][q]);
    };
    const uint32_t step = (uint32_t)(kWaves * p.splits), first = (uint32_t)(range * kWaves + wave), whole = p.k / (32 * GW);
#pragma unroll 1
    for (uint32_t g0 = first; g0 < whole; g0 += D * step) {
        words_t w[D];
        uint32_t zero[D];
        float scale[D][4];
#pragma unroll
        for (int i = 0; i < D; ++i) {                  // (past the last whole group: that one, with scales of 0)
            const uint32_t g = min(g0 + i * step, whole - 1);
            w[i] = __builtin_nontemporal_load(reinterpret_cast<const words_t*>(W + (size_t)g * (4 * GW)));
            zero[i] = zeros ? zeros[g] : 8u;
#pragma unroll
            for (int q = 0; q < 4; ++q) scale[i][q] = g0 + i * step < whole ? td_load<T>(scales[q] + g) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const uint32_t g = min(g0 + i * step, whole - 1);
            add(g, w[i], zero[i], scale[i], [](Token<T>& v, const unsigned char* at, int) { load_token<T>(v, at); });
        }
    }
    if (whole < p.groups && whole % step == first) {   // the last group, which is not whole
        float scale[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) scale[q] = td_load<T>(scales[q] + whole);
        add(whole, *reinterpret_cast<const words_t*>(W + (size_t)whole * (4 * GW)), zeros ? zeros[whole] : 8u, scale,
            [](Token<T>& v, const unsigned char* at, int left) { load_token_end<T>(v, at, left); });
    }
    // the wavefronts' sums, in their order; a thread has four neighbouring columns of a token
#pragma unroll
    for (int t = 0; t < TT; ++t) sums[(wave * TT + t) * 64 + lane] = acc[t];
    __syncthreads();
    if (tid >= TT * 64) return;
    f32x4_t v = sums[tid];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += sums[w * TT * 64 + tid];
    const int64_t m = m0 + (tid >> 6) * 16 + low, n = n0 + 4 * high;
    const int columns = (int)min((int64_t)4, p.N - n);
    if (m >= p.n || columns <= 0) return;
    const int64_t at = m * p.N + n;
    if (p.part) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < columns) p.part[(int64_t)range * p.n * p.N + at + q] = v[q];
        return;
    }
    auto element = [&](const void* from, int64_t i) { return p.out_f32 ? static_cast<const float*>(from)[i] : td_load<bf16_t>(static_cast<const bf16_t*>(from) + i); };
    float bias[4] = {}, r[4] = {};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q >= columns) continue;
        if (p.b) bias[q] = element(p.b, n + q);
        if (p.r) r[q] = element(p.r, at + q);
    }
    with_linear_act(p.act, [&](auto act) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = linear_act<decltype(act)::value>(v[q] + bias[q]) + r[q];
    });
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q >= columns) continue;
        if (p.out_f32) static_cast<float*>(p.y)[at + q] = v[q];
        else td_store<bf16_t>(static_cast<bf16_t*>(p.y) + at + q, v[q]);
    }
}

template <typename T, int GW> void launch(const FourArgs& p, int tokens, dim3 grid, hipStream_t s) {
    const dim3 block(64 * kWaves);
    if (tokens == 1) hipLaunchKernelGGL((linear4_kernel<T, GW, 1>), grid, block, 0, s, p);
    else if (tokens == 2) hipLaunchKernelGGL((linear4_kernel<T, GW, 2>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((linear4_kernel<T, GW, 4>), grid, block, 0, s, p);
}
template <typename T> void launch(const FourArgs& p, int group, int tokens, dim3 grid, hipStream_t s) {
    if (group == 32) launch<T, 1>(p, tokens, grid, s);
    else if (group == 64) launch<T, 2>(p, tokens, grid, s);
    else launch<T, 4>(p, tokens, grid, s);
}

}  // namespace

tardis_status_t td_linear_4bit_work_bytes(const tardis_linear_4bit_desc* d, int64_t n, int64_t x_pitch, int64_t* bytes) {
    *bytes = 0;
    return TARDIS_OK;
}

tardis_status_t td_linear_4bit(const tardis_linear_4bit_desc* d, const void* x, int64_t n, int64_t x_pitch, const void* residual, void* y, void* work,
                               int64_t work_bytes, hipStream_t s) {
    FourArgs p{};
    const int64_t es = (int64_t)td_elem_size(d->dtype), eo = (int64_t)td_elem_size(d->out_dtype);
    p.x = static_cast<const unsigned char*>(x);
    p.W = d->W;
    p.scales = d->scales;
    p.zeros = d->zeros;
    p.b = d->b;
    p.r = residual;
    p.y = y;
    p.n = n;
    p.N = d->n_out;
    p.x_pitch = (n > 1 ? x_pitch : d->n_in) * es;
    p.k = (uint32_t)d->n_in;
    p.groups = (uint32_t)((d->n_in + d->group - 1) / d->group);
    p.act = d->act == TARDIS_ACT_GELU_ERF && d->out_dtype == TARDIS_BF16 && !residual ? kActGelu16 : d->act;
    p.out_f32 = d->out_dtype == TARDIS_F32;
    p.tiles_n = (int)((d->n_out + 15) / 16);
    p.splits = 1;
    const int tokens = n <= 16 ? 1 : n <= 32 ? 2 : 4;                   // (in 16s)
    const int64_t rows = 16 * tokens, most = std::max<int64_t>(1, kMostThreads / (64 * kWaves) / p.tiles_n) * rows;   // tokens of a launch
    for (int64_t at = 0; at < n; at += most) {
        FourArgs q = p;
        q.n = std::min(most, n - at);
        q.x += at * p.x_pitch;
        q.y = static_cast<unsigned char*>(y) + at * p.N * eo;
        if (residual) q.r = static_cast<const unsigned char*>(residual) + at * p.N * eo;
        const dim3 grid((unsigned)(p.tiles_n * ((q.n + rows - 1) / rows)));
        if (d->dtype == TARDIS_F32) launch<float>(q, d->group, tokens, grid, s);
        else launch<bf16_t>(q, d->group, tokens, grid, s);
    }
    TD_HIP(hipGetLastError());
    return TARDIS_OK;
}
