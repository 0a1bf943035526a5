// The linear layer's kernels, each by its number, whatever tile the library would take for the sizes: for the test of every one of them.
#include "linear.h"

extern "C" {
int linear_probe_shapes(int f32, int direct) { return direct ? kLinearShapes + (f32 ? 0 : kLinearQuads) : kLinearStagedShapes; }
int linear_probe_has(int f32, int direct, int grouped, int shape) { return (direct && shape >= kLinearShapes) || linear_has(f32 ? 4 : 2, direct, grouped, shape); }
void linear_probe_tile(int direct, int shape, int* out) {
    const LinearShape& s = !direct ? kLinearStaged[shape] : shape < kLinearShapes ? kLinearShape[shape] : kLinearQuad[shape - kLinearShapes];
    out[0] = s.m;
    out[1] = s.n;
    out[2] = s.slice;
}
// experts = 0: one matrix; ranges > 1: y has the sums of the ranges
int linear_probe(int f32, int direct, int shape, const void* x, int64_t x_rows, int64_t pitch, const void* W, const void* b, const void* r, void* y, int64_t rows,
                 int64_t N, int64_t k, int act, int out_f32, int ranges, const int32_t* offsets, const int32_t* order, int experts, int per_token, void* stream) {
    if (!linear_probe_has(f32, direct, experts > 0, shape)) return TARDIS_ERR_SHAPE;
    int t[3];
    linear_probe_tile(direct, shape, t);
    LinearArgs p{};
    p.x = static_cast<const unsigned char*>(x);
    p.W = static_cast<const unsigned char*>(W);
    p.b = b;
    p.r = r;
    p.y = y;
    p.part = ranges > 1 ? static_cast<float*>(y) : nullptr;
    p.n = rows;
    p.N = N;
    p.x_pitch = pitch;
    p.x_rows = x_rows;
    p.x_bytes = (x_rows - 1) * pitch + k;
    p.k = (uint32_t)k;
    p.act = act;
    p.out_f32 = out_f32;
    p.tiles_m = (int)((rows + t[0] - 1) / t[0]);
    p.tiles_n = (int)((N + t[1] - 1) / t[1]);
    const int64_t even = ((rows + p.tiles_m - 1) / p.tiles_m + 31) / 32 * 32;
    p.tile_rows = (int)(even < t[0] ? even : t[0]);
    p.splits = ranges;
    p.slices = (int)(((k + t[2] - 1) / t[2] + ranges - 1) / ranges);
    p.offsets = offsets;
    p.order = order;
    p.experts = experts;
    p.per_token = per_token;
    p.inv_per_token = per_token > 1 ? (uint32_t)(0x100000000ull / (uint64_t)per_token) : 0xffffffffu;
    const int64_t full = direct && shape >= kLinearShapes ? linear_least_rows(t[0]) : t[0];
    const int64_t most = (rows + (int64_t)experts * (full - 1)) / full;
    const int64_t tiles = (experts ? (most < rows ? most : rows) : p.tiles_m) * p.tiles_n * ranges;
    const int blocks = (int)((tiles + 7) / 8 * 8);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool quad = direct && shape >= kLinearShapes;
    const tardis_status_t st = f32 ? td_linear_init_f32() : quad ? td_linear_init_quad() : td_linear_init_bf16();
    if (st != TARDIS_OK) return st;
    if (quad) td_linear_launch_quad(p, experts > 0, shape - kLinearShapes, blocks, s);
    else if (f32) td_linear_launch_f32(p, experts > 0, direct, shape, blocks, s);
    else td_linear_launch_bf16(p, experts > 0, direct, shape, blocks, s);
    return hipGetLastError() == hipSuccess ? TARDIS_OK : TARDIS_ERR_HIP;
}
}
