// What linear.hip (which tile a call takes) and the kernels (linear_tile.h, one translation unit for each element type) share.
#pragma once
#include "common.h"

// C = sigma(x W^T + b) + r.  Pitches and k in bytes.
struct LinearArgs {
    const unsigned char *x, *W;
    const void *b, *r;             // per column (of every group), element type of W; like y (null: none)
    void* y;                       // n x N, bf16 or (out_f32) fp32, rows without a gap
    float* part;                   // not null: sums of one range of K each go here, [range][n][N], and nothing else is done
    int64_t n, N, x_pitch, x_rows;
    int64_t x_bytes;               // up to the end of the last row of x
    uint32_t k;
    int act, out_f32;
    int tiles_m, tiles_n, splits, slices;   // of the whole product; ranges of K, slices in one.  (groups: tiles_n alone)
    int tile_rows;                 // linear_quad_kernel: rows of a tile
    // rows by groups: those of group e are offsets[e] .. offsets[e + 1], with weights W + e N k; row m is row order[m] / per_token of x
    const int32_t *offsets, *order;
    int experts, per_token;
    uint32_t inv_per_token;
};

constexpr int kActGelu16 = 4;                     // behind tardis_act_t's: GELU for outputs in bf16 without a residual
constexpr uint32_t kNowhere = 0xe0000000u;        // an offset past the end of any operand that is loaded by offsets

// The tiles: rows, columns and bytes of K in a slice (64 or 128 for each of the wavefronts that divide it)
struct LinearShape { int m, n, slice; };
constexpr LinearShape kLinearShape[] = {{16, 16, 512}, {16, 32, 512}, {16, 64, 512}, {32, 32, 256}, {32, 64, 256}, {64, 32, 256},
                                        {64, 64, 256}, {64, 64, 128}, {128, 64, 128}, {128, 128, 128}, {192, 128, 128},
                                        {16, 16, 1024}, {32, 32, 512}, {64, 64, 128}, {64, 128, 128}, {128, 128, 128}};
constexpr int kLinearShapes = sizeof(kLinearShape) / sizeof(LinearShape);
constexpr LinearShape kLinearStaged[] = {{16, 16, 512}, {16, 32, 512}, {32, 32, 256}, {64, 64, 128}, {128, 128, 128}};
constexpr int kLinearStagedShapes = sizeof(kLinearStaged) / sizeof(LinearShape);
// The rule in linear.hip has no use for some of them: in fp32 the matrix cores are the limit, where few blocks with long slices gain nothing
// and smaller tiles fill the CUs better; a group's rows are many only where the call has tiles enough for small ones.
constexpr bool linear_has(int es, bool direct, bool grouped, int shape) {
    if (!direct) return !(grouped && shape == 1);
    if (es == 2) return !(grouped && shape == 8);
    return !(shape == 2 || (shape >= 4 && shape <= 9) || shape == 12 || (grouped && (shape == 10 || shape == 15)));
}
// of linear_quad_kernel (bf16, rows in whole pieces)
constexpr LinearShape kLinearQuad[] = {{256, 256, 128}, {192, 256, 128}, {256, 128, 128}};
// (rows with which its tiles of groups are full, if the kernel decides so)
constexpr int linear_least_rows(int m) { return m == 256 ? 192 : m; }
constexpr int kLinearQuads = sizeof(kLinearQuad) / sizeof(LinearShape);

tardis_status_t td_linear_init_quad();
void td_linear_launch_quad(const LinearArgs& p, bool grouped, int shape, int blocks, hipStream_t s);
tardis_status_t td_linear_init_bf16();
tardis_status_t td_linear_init_f32();
void td_linear_launch_bf16(const LinearArgs& p, bool grouped, bool direct, int shape, int blocks, hipStream_t s);
void td_linear_launch_f32(const LinearArgs& p, bool grouped, bool direct, int shape, int blocks, hipStream_t s);
