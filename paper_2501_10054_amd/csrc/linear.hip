// A linear layer with its epilogue, y = sigma(x W^T + b) + r, alone or for rows grouped by expert: how a call is done - which tile, in how
// many ranges of K, of which operands a copy with aligned rows is made first.  The kernels are in linear_tile.h and linear_quad.hip.
#include <algorithm>
#include <cmath>

#include "linear_act.h"
#include "tiles.h"

namespace {

bool is_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
typedef uint32_t any16_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t byte16_t __attribute__((ext_vector_type(4), aligned(1)));

// Rows of k bytes, `pitch` apart and at any address, to rows of `units` 16-byte pieces, zeros behind the last element.  (Fewer than 2^32 pieces)
template <typename T>
__global__ void __launch_bounds__(256) linear_pack_kernel(const unsigned char* from, int64_t pitch, uint32_t k, td_u32x4* to, uint32_t rows, uint32_t units) {
    const uint32_t u = blockIdx.x * 256u + threadIdx.x, row = u / units;
    if (row >= rows) return;
    const uint32_t at = (u - row * units) * 16u;
    const unsigned char* p = from + (int64_t)row * pitch + at;
    td_u32x4 v = {0, 0, 0, 0};
    if (at + 16 <= k) {
        if constexpr (sizeof(T) == 1) v = *reinterpret_cast<const byte16_t*>(p);
        else v = *reinterpret_cast<const any16_t*>(p);
    } else {
        const T* el = reinterpret_cast<const T*>(p);
#pragma unroll
        for (uint32_t q = 0; q < 16 / sizeof(T); ++q)
            if (at + q * sizeof(T) < k) {
                if constexpr (sizeof(T) == 1) v[q / 4] |= (uint32_t)el[q].code << (8 * (q & 3));
                else if constexpr (sizeof(T) == 2) v[q / 2] |= (uint32_t)el[q] << (16 * (q & 1));
                else v[q] = __float_as_uint(el[q]);
            }
    }
    to[u] = v;
}

// The sums of the ranges of K, in their order, and the epilogue: a thread has 4 neighbouring columns.
template <typename T>
__global__ void __launch_bounds__(256) linear_join_kernel(LinearArgs p, uint32_t units) {
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = u < (1ll << 32) ? (int64_t)((uint32_t)u / units) : u / units;
    if (row >= p.n) return;
    const int64_t n = (u - row * units) * 4, at = row * p.N + n, range = p.n * p.N;
    const int columns = (int)min((int64_t)4, p.N - n);
    float v[4] = {}, r[4] = {}, bias[4] = {};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q >= columns) continue;
        if constexpr (sizeof(T) == 1) {
            if (p.b) bias[q] = p.out_f32 ? static_cast<const float*>(p.b)[n + q] : td_load<bf16_t>(static_cast<const bf16_t*>(p.b) + n + q);
        } else {
            if (p.b) bias[q] = td_load<T>(static_cast<const T*>(p.b) + n + q);
        }
        if (p.r) r[q] = p.out_f32 ? static_cast<const float*>(p.r)[at + q] : td_load<bf16_t>(static_cast<const bf16_t*>(p.r) + at + q);
    }
    if (columns == 4) {
#pragma unroll 4
        for (int s = 0; s < p.splits; ++s) {
            const td_u32x4 part = *reinterpret_cast<const any16_t*>(p.part + s * range + at);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] += __uint_as_float(part[q]);
        }
    } else {
        for (int s = 0; s < p.splits; ++s)
            for (int q = 0; q < 4; ++q)
                if (q < columns) v[q] += p.part[s * range + at + q];
    }
    if constexpr (sizeof(T) == 1) {
        const float token_scale = p.x_scales ? p.x_scales[row] : 1.0f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] = fmaf(v[q] * token_scale, p.W_scales && q < columns ? p.W_scales[n + q] : 1.0f, bias[q]);
            bias[q] = 0.0f;
        }
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

template <typename T> void join(const LinearArgs& p, hipStream_t s) {
    const int64_t units = (p.N + 3) / 4;
    hipLaunchKernelGGL(linear_join_kernel<T>, dim3((unsigned)((units * p.n + 255) / 256)), dim3(256), 0, s, p, (uint32_t)units);
}

// ---------------------------------------------------------------- how a call is done
// What a tile takes, in us:
//     max(fixed x turns + slices x max(alone x turns, slice x tiles of a CU), 1.5 + bytes / tbs)
// with `blocks` of them at once on a CU, in `turns` turns: alone is a slice's latency, slice its share of the CU.  Bytes: x, y (the ranges'
// sums), W, and for every further row of tiles `again` of W.  The constants are those with which the choice is best: over 581 products and 155
// grouped ones in bf16 (sizes from 64 x 64 to 16384 x 16384, 1 to 5000 rows, weights from HBM; every tile with 1, 2, 4 and 8 ranges) it takes 1.5 and 3.1 % more
// than the best measured, fp32 (185, 39) 0.8 %, staged (179, 28) 1.0 %, staged fp32 (98) 0.3 %.
struct Rate { int blocks; float alone, slice, fixed, tbs; };
// ({}: a tile that is not there, linear_has)
constexpr Rate kRate[] = {{2, 0.244f, 0.223f, 3.80f, 5.50f}, {2, 0.415f, 0.400f, 3.74f, 5.51f}, {1, 0.493f, 0.493f, 4.47f, 5.09f},
                          {2, 0.238f, 0.205f, 4.00f, 4.83f}, {1, 0.321f, 0.321f, 4.01f, 5.09f}, {1, 0.276f, 0.276f, 4.15f, 4.15f},
                          {1, 0.417f, 0.417f, 4.98f, 5.46f}, {2, 0.247f, 0.234f, 4.53f, 5.33f}, {1, 0.376f, 0.376f, 5.14f, 4.27f},
                          {1, 0.512f, 0.512f, 6.21f, 5.25f}, {1, 0.630f, 0.630f, 7.61f, 3.04f}, {1, 0.369f, 0.369f, 4.39f, 5.47f},
                          {1, 0.399f, 0.399f, 4.31f, 4.24f}, {5, 0.489f, 0.262f, 3.07f, 3.94f}, {3, 0.790f, 0.367f, 3.75f, 4.55f},
                          {2, 0.725f, 0.639f, 4.82f, 3.77f}, {1, 0.903f, 0.903f, 14.60f, 3.45f}, {1, 0.770f, 0.770f, 12.50f, 3.95f},
                          {1, 0.788f, 0.788f, 7.70f, 3.77f}};
constexpr Rate kRateF32[] = {{2, 0.266f, 0.238f, 4.14f, 5.61f}, {2, 0.436f, 0.344f, 4.19f, 6.18f}, {}, {2, 0.368f, 0.323f, 3.75f, 4.50f},
                             {}, {}, {}, {}, {}, {}, {1, 3.086f, 3.086f, 8.00f, 3.83f}, {1, 0.483f, 0.483f, 4.53f, 4.86f},
                             {}, {5, 0.689f, 0.540f, 3.88f, 3.38f}, {3, 1.149f, 1.040f, 5.81f, 2.57f}, {2, 2.066f, 2.073f, 7.14f, 5.23f}};
constexpr Rate kRateStaged[] = {{2, 0.246f, 0.231f, 4.77f, 3.34f}, {1, 0.389f, 0.389f, 4.64f, 3.29f}, {2, 0.176f, 0.227f, 4.35f, 4.73f},
                                {2, 0.228f, 0.214f, 4.34f, 2.79f}, {1, 0.560f, 0.560f, 7.05f, 2.77f}};
constexpr Rate kRateStagedF32[] = {{2, 0.104f, 0.250f, 4.45f, 4.01f}, {1, 0.377f, 0.377f, 4.45f, 4.01f}, {2, 0.053f, 0.305f, 4.21f, 4.46f},
                                   {2, 0.556f, 0.550f, 4.53f, 5.00f}, {1, 2.042f, 2.042f, 6.55f, 4.71f}};
// (e4m3, by the faster instruction and with exact sums: 323 and 234 measurements of 15 products each, 3.1 and 1.1 % more than the best; exact ones with outputs in
// fp32; of rows through registers no measurements but estimates)
constexpr Rate kRateFp8[] = {{2, 0.254f, 0.139f, 5.95f, 4.70f}, {3, 0.399f, 0.332f, 4.72f, 3.75f}, {1, 0.382f, 0.350f, 4.64f, 3.47f}, {1, 0.337f, 0.337f, 5.22f, 4.14f},
                             {1, 0.469f, 0.350f, 4.93f, 3.65f}, {1, 1.231f, 0.350f, 5.55f, 2.71f}, {3, 0.784f, 0.450f, 8.51f, 3.86f}, {3, 0.541f, 0.180f, 5.28f, 3.44f},
                             {1, 0.606f, 0.350f, 5.12f, 3.70f}, {2, 0.400f, 0.665f, 9.00f, 4.88f}, {1, 0.495f, 0.709f, 5.36f, 3.32f},
                             {1, 0.691f, 0.350f, 8.92f, 3.16f}};
constexpr Rate kRateFp8Exact[] = {{2, 0.271f, 0.271f, 4.83f, 4.60f}, {3, 0.438f, 0.343f, 4.78f, 4.04f}, {1, 0.280f, 0.280f, 4.98f, 3.63f}, {},
                                {1, 0.647f, 0.350f, 5.48f, 3.08f}, {}, {3, 0.822f, 0.757f, 10.05f, 3.36f}, {3, 0.597f, 0.223f, 5.65f, 3.39f},
                                {1, 0.756f, 0.415f, 5.19f, 3.54f}, {}, {}};
constexpr Rate kRateStagedFp8[] = {{2, 0.320f, 0.300f, 6.30f, 3.30f}, {2, 0.230f, 0.300f, 5.90f, 3.50f}, {2, 0.300f, 0.280f, 5.90f, 2.80f}, {1, 0.750f, 0.750f, 8.50f, 2.60f}};
static_assert(sizeof(kRateFp8) / sizeof(Rate) == kLinearShapesFp8 + kLinearQuadsFp8 && sizeof(kRateFp8Exact) / sizeof(Rate) == kLinearShapesFp8 && sizeof(kRateStagedFp8) / sizeof(Rate) == kLinearStagedShapesFp8, "a rate for each tile");
static_assert(sizeof(kRate) / sizeof(Rate) == kLinearShapes + kLinearQuads && sizeof(kRateF32) / sizeof(Rate) == kLinearShapes &&
              sizeof(kRateStaged) / sizeof(Rate) == kLinearStagedShapes && sizeof(kRateStagedF32) / sizeof(Rate) == kLinearStagedShapes, "a rate for each tile");
// one more launch (2.5 on the GPU; callers that are not a graph wait for their host); a byte copied, of partial sums and outputs joined; sigma of an element of a tile, of eight wavefronts and of four
constexpr double kLaunchUs = 4.0, kCopyUs = 1.0 / 4.5e6, kJoinUs = 1.0 / 5e6, kSigmaUs = 5.0 / 65536, kSigmaQuadUs = 8.0 / 65536;
constexpr double kAgain = 0.34, kAgainF32 = 0.44, kAgainStaged = 0.20, kAgainStagedF32 = 0.43;
constexpr int64_t kMostTiles = 1 << 21;            // of a launch

// What decides: sizes, types, alignment
struct Call {
    int64_t M, N, x_rows, k, pitch;                // rows of y, columns, rows of x; bytes of a row, from row to row of x
    int es, eo, act;
    int experts;                                   // 0: one matrix
    bool gather, x_aligned, W_aligned;             // (addresses)
    bool near;                                     // e4m3: by the faster instruction where tiles are large
};
struct Plan {
    bool direct, pack_x, pack_W;
    int shape, splits, slices;                     // (direct, in bf16: shapes of linear_kernel, then of linear_quad_kernel)
    int64_t k, pitch, at_W, at_part, work;         // of what is multiplied; places in the working memory and its size
    double us;
};

// (es: bytes of an element - 1 e4m3, 2 bf16, 4 fp32)
int shapes_below_quads(bool direct, int es) { return es == 1 ? (direct ? kLinearShapesFp8 : kLinearStagedShapesFp8) : direct ? kLinearShapes : kLinearStagedShapes; }
int shapes_of(bool direct, int es, bool near) { return shapes_below_quads(direct, es) + (!direct || es == 4 ? 0 : es == 2 ? kLinearQuads : near ? kLinearQuadsFp8 : 0); }
bool is_quad(bool direct, int es, int s) { return direct && s >= shapes_below_quads(direct, es); }
const LinearShape& shape_of(bool direct, int es, int s) {
    if (is_quad(direct, es, s)) return (es == 1 ? kLinearQuadFp8 : kLinearQuad)[s - shapes_below_quads(direct, es)];
    return es == 1 ? (direct ? kLinearShapeFp8[s] : kLinearStagedFp8[s]) : direct ? kLinearShape[s] : kLinearStaged[s];
}
const Rate& rate_of(bool direct, int es, bool near, int s) {
    if (es == 1) return !direct ? kRateStagedFp8[s] : near ? kRateFp8[s] : kRateFp8Exact[s];
    return direct ? (es == 2 ? kRate[s] : kRateF32[s]) : es == 2 ? kRateStaged[s] : kRateStagedF32[s];
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Rows of tiles of a launch, at most (of groups: one tile that is not full in each, and no more tiles than rows)
int64_t most_tiles_m(const Call& c, bool quad, const LinearShape& t) {
    const int64_t full = c.experts && quad ? linear_least_rows(t.m) : t.m;
    return c.experts ? std::min(c.M, (c.M + (int64_t)c.experts * (full - 1)) / full) : (c.M + t.m - 1) / t.m;
}

// The least time over the ways that the call allows and that take no more than `room` bytes of working memory (splits = 0: there is none)
Plan make_plan(const Call& c, int64_t room) {
    Plan best{};
    best.us = 1e300;
    // groups: the experts that are hit, if rows fall on them evenly
    const double hit = c.experts ? std::max(1.0, c.experts * (1.0 - std::exp(-(double)c.M / c.experts))) : 1.0;
    const int64_t W_rows = c.N * std::max(c.experts, 1);
    const bool k_whole = c.k % 16 == 0;
    for (int way = 0; way < 2; ++way) {
        Plan p{};
        p.direct = way == 1;
        p.k = c.k;
        p.pitch = c.pitch;
        double before = 0.0;
        if (p.direct) {
            p.pack_W = !(k_whole && c.W_aligned);
            p.pack_x = !(k_whole && c.x_aligned && c.pitch % 16 == 0);
            p.k = round_up(c.k, 16);
            if (p.pack_x) p.pitch = p.k;
            const int64_t bytes_x = p.pack_x ? round_up(c.x_rows * p.k, 256) : 0, bytes_W = p.pack_W ? round_up(W_rows * p.k, 256) : 0;
            p.at_W = bytes_x;
            p.at_part = bytes_x + bytes_W;
            if (p.pack_x) before += kLaunchUs + 2.0 * (double)bytes_x * kCopyUs;
            if (p.pack_W) before += kLaunchUs + 2.0 * (double)bytes_W * kCopyUs;
            if (p.pitch >= 1 << 23 || p.k >= 1 << 23 || (c.gather && (c.x_rows - 1) * p.pitch + p.k >= (int64_t)kNowhere)) continue;
        }
        if (p.at_part > room) continue;
        for (int s = 0; s < shapes_of(p.direct, c.es, c.near); ++s) {
            const bool quad = is_quad(p.direct, c.es, s);
            if (!quad && !(c.es == 1 ? linear_has_fp8(p.direct, c.near, s) : linear_has(c.es, p.direct, c.experts > 0, s))) continue;
            const LinearShape& t = shape_of(p.direct, c.es, s);
            const Rate& r = rate_of(p.direct, c.es, c.near, s);
            const int64_t slices = (p.k + t.slice - 1) / t.slice, tiles_n = (c.N + t.n - 1) / t.n;
            const double tiles_m = c.experts ? hit * std::max(1.0, (double)c.M / hit / t.m + 0.5) : (double)((c.M + t.m - 1) / t.m);
            if (most_tiles_m(c, quad, t) * tiles_n >= kMostTiles) continue;
            for (int splits = 1; splits <= 16; splits *= 2) {
                const double blocks = tiles_m * (double)tiles_n * splits;
                if (splits > 1 && (c.experts || slices / splits < 4 || blocks > 1024 || p.at_part + splits * c.M * c.N * 4 > room)) break;
                // (how many tiles groups have is an estimate)
                const double rounds = c.experts ? std::max(1.0, blocks / 256 + 0.5) : std::ceil(blocks / 256);
                const double turns = c.experts ? std::max(1.0, rounds / r.blocks) : std::ceil(rounds / r.blocks);
                const double per = (double)((slices + splits - 1) / splits);
                const double sigma = c.act == TARDIS_ACT_GELU_ERF || c.act == TARDIS_ACT_GELU_TANH ? (quad ? kSigmaQuadUs : kSigmaUs) * t.m * t.n * rounds : 0.0;
                const double multiply = r.fixed * turns + per * std::max(r.alone * turns, r.slice * rounds) + (splits > 1 ? 0.0 : sigma);
                const double again = p.direct ? (c.es == 4 ? kAgainF32 : kAgain) : (c.es == 4 ? kAgainStagedF32 : kAgainStaged);
                const double bytes = (hit + again * std::max(0.0, tiles_m - hit)) * c.N * p.k + (double)c.M * p.k + (double)c.M * c.N * (splits > 1 ? 4.0 * splits : c.eo);
                double us = before + std::max(multiply, 1.5 + bytes / (r.tbs * 1e6));
                if (splits > 1) us += kLaunchUs + (double)c.M * c.N * (4.0 * splits + c.eo) * kJoinUs;
                if (us < best.us) {
                    best = p;
                    best.us = us;
                    best.shape = s;
                    best.splits = splits;
                    best.slices = (int)((slices + splits - 1) / splits);
                    best.work = p.at_part + (splits > 1 ? splits * c.M * c.N * 4 : 0);
                }
            }
        }
    }
    return best;
}

// make_plan's answer depends on sizes, alignment and working memory alone, of which a program has few: the last plans of a thread, by a hash
// (1.2 us of the 8 that a small call takes of its host)
const Plan& plan_of(const Call& c, int64_t room) {
    struct Kept {
        Call call;
        int64_t room;
        Plan plan;
    };
    static thread_local Kept kept[64];             // (M = 0: none)
    uint64_t h = 0;
    for (const int64_t v : {c.M, c.N, c.k, c.pitch, (int64_t)c.experts}) h = (h ^ (uint64_t)v) * 0x9e3779b97f4a7c15ull;
    Kept& k = kept[h >> 58];
    const Call& o = k.call;
    const bool same = o.M == c.M && o.N == c.N && o.x_rows == c.x_rows && o.k == c.k && o.pitch == c.pitch && o.es == c.es && o.eo == c.eo && o.act == c.act &&
                      o.experts == c.experts && o.gather == c.gather && o.x_aligned == c.x_aligned && o.W_aligned == c.W_aligned && o.near == c.near && k.room == room;
    if (!same) k = {c, room, make_plan(c, room)};
    return k.plan;
}

// p: operands and sizes as the caller gave them; pitches and k in bytes
tardis_status_t run(LinearArgs p, const Call& c, void* work, int64_t work_bytes, hipStream_t s) {
    const Plan& plan = plan_of(c, work_bytes);
    if (plan.splits == 0) return TARDIS_ERR_SHAPE;
    const LinearShape& t = shape_of(plan.direct, c.es, plan.shape);
    const bool grouped = c.experts > 0, quad = is_quad(plan.direct, c.es, plan.shape), f32 = c.es == 4, fp8 = c.es == 1;
    p.tiles_m = (int)((p.n + t.m - 1) / t.m);
    p.tiles_n = (int)((p.N + t.n - 1) / t.n);
    p.tile_rows = (int)std::min<int64_t>(t.m, round_up((p.n + p.tiles_m - 1) / p.tiles_m, 32));
    p.splits = plan.splits;
    p.slices = plan.slices;
    const int64_t tiles = most_tiles_m(c, quad, t) * p.tiles_n * plan.splits;
    if (fp8) TD_TRY(quad ? td_linear_init_fp8_quad() : td_linear_init_fp8());
    else if (f32) TD_TRY(td_linear_init_f32());
    else TD_TRY(quad ? td_linear_init_quad() : td_linear_init_bf16());
    unsigned char* memory = static_cast<unsigned char*>(work);
    auto pack = [&](const unsigned char* from, int64_t pitch, int64_t rows, unsigned char* to) {
        const uint32_t units = (uint32_t)(plan.k / 16);
        const int64_t most = kMostThreads / units;                 // rows of a launch
        for (int64_t row = 0; row < rows; row += most) {
            const uint32_t here = (uint32_t)std::min(most, rows - row);
            const unsigned char* first = from + row * pitch;
            td_u32x4* at = reinterpret_cast<td_u32x4*>(to) + row * units;
            const dim3 grid((here * units + 255) / 256);
            if (fp8) hipLaunchKernelGGL(linear_pack_kernel<e4m3_t>, grid, dim3(256), 0, s, first, pitch, (uint32_t)c.k, at, here, units);
            else if (f32) hipLaunchKernelGGL(linear_pack_kernel<float>, grid, dim3(256), 0, s, first, pitch, (uint32_t)c.k, at, here, units);
            else hipLaunchKernelGGL(linear_pack_kernel<bf16_t>, grid, dim3(256), 0, s, first, pitch, (uint32_t)c.k, at, here, units);
        }
        return to;
    };
    if (plan.pack_x) p.x = pack(p.x, c.pitch, c.x_rows, memory);
    if (plan.pack_W) p.W = pack(p.W, c.k, p.N * std::max(p.experts, 1), memory + plan.at_W);
    p.k = (uint32_t)plan.k;
    p.x_pitch = plan.pitch;
    p.x_bytes = (c.x_rows - 1) * p.x_pitch + p.k;
    LinearArgs q = p;
    if (plan.splits > 1) {
        q.part = reinterpret_cast<float*>(memory + plan.at_part);
        q.act = TARDIS_ACT_IDENTITY;
    }
    const int blocks = (int)((tiles + 7) / 8 * 8);
    if (fp8 && quad) td_linear_launch_fp8_quad(q, plan.shape - kLinearShapesFp8, blocks, s);
    else if (fp8) td_linear_launch_fp8(q, plan.direct, c.near, plan.shape, blocks, s);
    else if (quad) td_linear_launch_quad(q, grouped, plan.shape - kLinearShapes, blocks, s);
    else if (f32) td_linear_launch_f32(q, grouped, plan.direct, plan.shape, blocks, s);
    else td_linear_launch_bf16(q, grouped, plan.direct, plan.shape, blocks, s);
    if (plan.splits > 1) {
        p.part = q.part;
        if (fp8) td_linear_join(p, s);
        else if (f32) join<float>(p, s);
        else join<bf16_t>(p, s);
    }
    TD_HIP(hipGetLastError());
    return TARDIS_OK;
}

const unsigned char* bytes_of(const void* p) { return static_cast<const unsigned char*>(p); }

LinearArgs layer(const tardis_linear_desc* d, bool residual) {
    LinearArgs p{};
    p.W = bytes_of(d->W);
    p.b = d->b;
    p.N = d->n_out;
    p.k = (uint32_t)(d->n_in * (int64_t)td_elem_size(d->dtype));
    p.act = d->act == TARDIS_ACT_GELU_ERF && d->out_dtype == TARDIS_BF16 && !residual ? kActGelu16 : d->act;
    p.out_f32 = d->out_dtype == TARDIS_F32;
    return p;
}

Call call_of(const tardis_linear_desc* d, int64_t experts, const void* x, int64_t x_rows, int64_t x_pitch, bool gather, int64_t rows) {
    const int64_t es = (int64_t)td_elem_size(d->dtype);
    if (x_rows == 1) x_pitch = d->n_in;            // (of one row there is none, and none that is too long)
    return {rows, d->n_out, x_rows, d->n_in * es, x_pitch * es, (int)es, (int)td_elem_size(d->out_dtype), d->act, (int)experts, gather,
            is_aligned16(x), is_aligned16(d->W), false};
}

int act_of(const tardis_linear_fp8_desc* d) { return d->act & ~TARDIS_FP8_EXACT; }

Call call_of(const tardis_linear_fp8_desc* d, const void* x, int64_t n, int64_t x_pitch) {
    if (n == 1) x_pitch = d->n_in;
    return {n, d->n_out, n, d->n_in, x_pitch, 1, (int)td_elem_size(d->out_dtype), act_of(d), 0, false, is_aligned16(x), is_aligned16(d->W),
            d->out_dtype == TARDIS_BF16 && !(d->act & TARDIS_FP8_EXACT)};
}

constexpr int64_t kAnyRoom = (int64_t)1 << 62;

}  // namespace

void td_linear_join(const LinearArgs& p, hipStream_t s) { join<e4m3_t>(p, s); }

tardis_status_t td_linear_work_bytes(const tardis_linear_desc* d, int64_t experts, const void* x, int64_t x_rows, int64_t x_pitch, bool gather, int64_t rows,
                                     int64_t* bytes) {
    const Plan plan = make_plan(call_of(d, experts, x, x_rows, x_pitch, gather, rows), kAnyRoom);
    if (plan.splits == 0) return TARDIS_ERR_SHAPE;
    *bytes = plan.work;
    return TARDIS_OK;
}

tardis_status_t td_linear(const tardis_linear_desc* d, const void* x, int64_t n, int64_t x_pitch, const void* residual, void* y, void* work,
                          int64_t work_bytes, hipStream_t s) {
    LinearArgs p = layer(d, residual != nullptr);
    p.x = bytes_of(x);
    p.r = residual;
    p.y = y;
    p.n = p.x_rows = n;
    return run(p, call_of(d, 0, x, n, x_pitch, false, n), work, work_bytes, s);
}

tardis_status_t td_linear_fp8_work_bytes(const tardis_linear_fp8_desc* d, const void* x, int64_t n, int64_t x_pitch, int64_t* bytes) {
    const Plan plan = make_plan(call_of(d, x, n, x_pitch), kAnyRoom);
    if (plan.splits == 0) return TARDIS_ERR_SHAPE;
    *bytes = plan.work;
    return TARDIS_OK;
}

tardis_status_t td_linear_fp8(const tardis_linear_fp8_desc* d, const void* x, const float* x_scales, int64_t n, int64_t x_pitch, const void* residual,
                              void* y, void* work, int64_t work_bytes, hipStream_t s) {
    LinearArgs p{};
    p.x = bytes_of(x);
    p.W = bytes_of(d->W);
    p.b = d->b;
    p.r = residual;
    p.y = y;
    p.n = p.x_rows = n;
    p.N = d->n_out;
    p.k = (uint32_t)d->n_in;
    p.act = act_of(d) == TARDIS_ACT_GELU_ERF && d->out_dtype == TARDIS_BF16 && !residual ? kActGelu16 : act_of(d);
    p.out_f32 = d->out_dtype == TARDIS_F32;
    p.x_scales = x_scales;
    p.W_scales = d->W_scales;
    return run(p, call_of(d, x, n, x_pitch), work, work_bytes, s);
}

tardis_status_t td_grouped_linear(const tardis_linear_desc* d, int64_t experts, const void* x, int64_t x_rows, int64_t x_pitch, const int32_t* offsets,
                                  const int32_t* order, int64_t per_token, int64_t positions, void* y, void* work, int64_t work_bytes, hipStream_t s) {
    LinearArgs p = layer(d, false);
    p.x = bytes_of(x);
    p.y = y;
    p.n = positions;
    p.x_rows = x_rows;
    p.offsets = offsets;
    p.order = order;
    p.experts = (int)experts;
    p.per_token = (int)per_token;
    p.inv_per_token = per_token > 1 ? (uint32_t)(0x100000000ull / (uint64_t)per_token) : 0xffffffffu;
    return run(p, call_of(d, experts, x, x_rows, x_pitch, order != nullptr, positions), work, work_bytes, s);
}
