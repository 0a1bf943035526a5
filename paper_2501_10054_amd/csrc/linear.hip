// A linear layer with its epilogue, y = sigma(x W^T + b) + r, alone or for rows grouped by expert: which tile a call takes, ranges of K
// and their sum.  The kernel is in linear_tile.h.
#include <algorithm>

#include "linear.h"
#include "sigma.h"
#include "tiles.h"

namespace {

bool is_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The sums of the ranges of K, and the epilogue: a thread has 4 neighbouring columns.
template <typename T>
__global__ void __launch_bounds__(256) linear_join_kernel(LinearArgs p, int64_t units_of_row) {
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, row = u / units_of_row, n = (u - row * units_of_row) * 4, at = row * p.N + n;
    if (row >= p.n) return;
    const int columns = (int)min((int64_t)4, p.N - n);
    float v[4] = {};
    for (int s = 0; s < p.splits; ++s)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < columns) v[q] += p.part[((int64_t)s * p.n) * p.N + at + q];
    with_act(p.act, [&](auto act) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (q >= columns) continue;
            float z = v[q] + (p.b ? td_load<T>(static_cast<const T*>(p.b) + n + q) : 0.0f);
            z = act_flat<decltype(act)::value>(z);
            if (p.r) z += p.out_f32 ? static_cast<const float*>(p.r)[at + q] : td_load<bf16_t>(static_cast<const bf16_t*>(p.r) + at + q);
            if (p.out_f32) static_cast<float*>(p.y)[at + q] = z;
            else td_store<bf16_t>(static_cast<bf16_t*>(p.y) + at + q, z);
        }
    });
}

struct Choice { int shape, splits, slices; };

Choice choose(const LinearArgs& p, int64_t es, bool grouped, bool direct, int64_t work_bytes) {
    Choice best{0, 1, 0};
    if (!direct) best.shape = p.n <= 32 ? 0 : 1;
    else best.shape = p.n <= 16 ? 1 : p.n <= 128 ? 7 : 9;
    const int sl = (direct ? kLinearShape : kLinearStaged)[best.shape].slice;
    const int slices = (int)((p.k + sl - 1) / sl);
    best.slices = (slices + best.splits - 1) / best.splits;
    return best;
}

tardis_status_t run(LinearArgs& p, int32_t dtype, bool grouped, void* work, int64_t work_bytes, hipStream_t s) {
    const int64_t es = (int64_t)td_elem_size(dtype);
    const bool gather = grouped && p.order;
    const bool direct = is_aligned16(p.x) && is_aligned16(p.W) && p.k % 16 == 0 && (p.x_pitch % 16 == 0 || p.n == 1) && p.x_pitch < (1 << 23) &&
                        p.k < (1u << 23) && (!gather || p.x_bytes < (int64_t)kNowhere);
    const Choice c = choose(p, es, grouped, direct, work_bytes);
    const LinearShape& t = (direct ? kLinearShape : kLinearStaged)[c.shape];
    p.tiles_m = (int)((p.n + t.m - 1) / t.m);
    p.tiles_n = (int)((p.N + t.n - 1) / t.n);
    p.splits = c.splits;
    p.slices = c.slices;
    // (of groups: at most one tile that is not full in each, and no more than rows)
    const int64_t tiles_m = grouped ? std::min(p.n, (p.n + (int64_t)p.experts * (t.m - 1)) / t.m) : p.tiles_m;
    const int64_t tiles = tiles_m * p.tiles_n * c.splits;
    if (tiles >= 1 << 21) return TARDIS_ERR_SHAPE;
    if (dtype == TARDIS_F32) TD_TRY(td_linear_init_f32());
    else TD_TRY(td_linear_init_bf16());
    LinearArgs q = p;
    if (c.splits > 1) {
        q.part = static_cast<float*>(work);
        q.act = TARDIS_ACT_IDENTITY;
    }
    const int blocks = (int)((tiles + 7) / 8 * 8);
    if (dtype == TARDIS_F32) td_linear_launch_f32(q, grouped, direct, c.shape, blocks, s);
    else td_linear_launch_bf16(q, grouped, direct, c.shape, blocks, s);
    if (c.splits > 1) {
        p.part = q.part;
        const int64_t units = (p.N + 3) / 4, n = (units * p.n + 255) / 256;
        if (dtype == TARDIS_F32) hipLaunchKernelGGL(linear_join_kernel<float>, dim3((unsigned)n), dim3(256), 0, s, p, units);
        else hipLaunchKernelGGL(linear_join_kernel<bf16_t>, dim3((unsigned)n), dim3(256), 0, s, p, units);
    }
    TD_HIP(hipGetLastError());
    return TARDIS_OK;
}

const unsigned char* bytes_of(const void* p) { return static_cast<const unsigned char*>(p); }

LinearArgs layer(const tardis_linear_desc* d) {
    LinearArgs p{};
    p.W = bytes_of(d->W);
    p.b = d->b;
    p.N = d->n_out;
    p.k = (uint32_t)(d->n_in * (int64_t)td_elem_size(d->dtype));
    p.act = d->act;
    p.out_f32 = d->out_dtype == TARDIS_F32;
    return p;
}

}  // namespace

size_t td_linear_work_bytes(const tardis_linear_desc* d, int64_t n) {
    (void)d;
    (void)n;
    return 0;
}

tardis_status_t td_linear(const tardis_linear_desc* d, const void* x, int64_t n, int64_t x_pitch, const void* residual, void* y, void* work,
                          int64_t work_bytes, hipStream_t s) {
    const int64_t es = (int64_t)td_elem_size(d->dtype);
    LinearArgs p = layer(d);
    p.x = bytes_of(x);
    p.r = residual;
    p.y = y;
    p.n = p.x_rows = n;
    p.x_pitch = x_pitch * es;
    p.x_bytes = (n - 1) * p.x_pitch + p.k;
    return run(p, d->dtype, false, work, work_bytes, s);
}

tardis_status_t td_grouped_linear(const tardis_linear_desc* d, int64_t experts, const void* x, int64_t x_rows, int64_t x_pitch, const int32_t* offsets,
                                  const int32_t* order, int64_t per_token, int64_t positions, void* y, hipStream_t s) {
    const int64_t es = (int64_t)td_elem_size(d->dtype);
    LinearArgs p = layer(d);
    p.x = bytes_of(x);
    p.y = y;
    p.n = positions;
    p.x_rows = x_rows;
    p.x_pitch = x_pitch * es;
    p.x_bytes = (x_rows - 1) * p.x_pitch + p.k;
    p.offsets = offsets;
    p.order = order;
    p.experts = (int)experts;
    p.per_token = (int)per_token;
    p.inv_per_token = per_token > 1 ? (uint32_t)(0x100000000ull / (uint64_t)per_token) : 0xffffffffu;
    return run(p, d->dtype, true, nullptr, 0, s);
}
