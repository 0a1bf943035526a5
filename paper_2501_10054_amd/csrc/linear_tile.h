// y = sigma(x W^T + b) + r for one weight matrix, or for one of several by groups of rows (mixture of experts): the kernel, for one
// element type of x, W and b (linear_bf16.hip, linear_f32.hip); which tile a call takes is linear.hip's.
#pragma once
#include "linear_act.h"
#include "tiles.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
// 16 bytes at any element's address
typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ td_u32x4 load_any16(const void* p) { return *static_cast<const u32x4_any_t*>(p); }
__device__ __forceinline__ void store_any16(void* p, const td_u32x4& v) { *static_cast<u32x4_any_t*>(p) = v; }

// One 16 x 16 block of sums: w, x hold 16 bytes of row lane % 16 at piece lane / 16 of 64 bytes of K.  (fp32: element q of all four
// pieces in one instruction, so K is summed in another order, the same for both operands.)
template <typename T> __device__ __forceinline__ void mma_pieces(f32x4_t& c, const td_u32x4& w, const td_u32x4& x);
template <> __device__ __forceinline__ void mma_pieces<bf16_t>(f32x4_t& c, const td_u32x4& w, const td_u32x4& x) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, x), c, 0, 0, 0);
}
template <> __device__ __forceinline__ void mma_pieces<float>(f32x4_t& c, const td_u32x4& w, const td_u32x4& x) {
#pragma unroll
    for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[q]), __uint_as_float(x[q]), c, 0, 0, 0);
}

// n / d for n < 2^21
__device__ __forceinline__ uint32_t divide(uint32_t n, uint32_t d, uint32_t& rest) {
    uint32_t q = (uint32_t)((float)n * __builtin_amdgcn_rcpf((float)d));
    int r = (int)(n - q * d);
    if (r < 0) { --q; r += (int)d; }
    if (r >= (int)d) { ++q; r -= (int)d; }
    rest = (uint32_t)r;
    return q;
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Tile number t of a tiles_m x tiles_n grid: eight tile rows are walked together, column by column, so that the blocks an XCD runs at
// once cover a patch and share the slices of both operands in its L2.
__device__ __forceinline__ void tile_of(uint32_t t, uint32_t tiles_m, uint32_t tiles_n, int& tile_m, int& tile_n) {
    uint32_t in_walk, row;
    const uint32_t walk = divide(t, 8 * tiles_n, in_walk) * 8, rows = min(8u, tiles_m - walk);
    tile_n = uniform((int)divide(in_walk, rows, row));
    tile_m = uniform((int)(walk + row));
}

// What a block computes: rows [first, first + rows) of C, columns from n0 on, slices [s0, s0 + nk) of K, with the weights of `expert`
struct LinearBlock {
    int64_t first, n0;
    int rows, expert, s0, nk, range;
    bool once;                                            // no other block reads its rows of W
};

// The whole slice that a block starts with.  Blocks that share slices start within a window of 8 of them; where each has rows of W to
// itself they spread over the whole row, and W's lines are not kept (16384 x 4096, 16 x 32 tiles, us: 27.3; lines not kept 26.8, spread 25.0, both
// 23.4; 4096 x 11008, 16 x 16: 18.8, 18.1, 19.8, 18.8)
__device__ __forceinline__ int start_of(const LinearBlock& b, int whole) {
    const int xcd = (int)blockIdx.x & 7, local = (int)blockIdx.x >> 3;
    if (!b.once || whole < 8) return first_slice(xcd, local, whole);
    uint32_t at;
    divide((uint32_t)(local + xcd * whole / 8), (uint32_t)whole, at);
    return uniform((int)at);
}

// Number `t` of `all` tiles for block b: an XCD (blocks b, b + 8, ...) has consecutive ones.  false: none
__device__ __forceinline__ bool number_of(uint32_t block, uint32_t all, uint32_t& t) {
    const uint32_t per = (all + 7) / 8, local = block >> 3;
    t = (block & 7) * per + local;
    return local < per && t < all;
}

// inclusive sums over the lanes
__device__ __forceinline__ int wave_scan(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, 64);
        v += lane >= o ? u : 0;
    }
    return v;
}

// Which group's tile this block has: the rows of a group are known on the device alone, so every wavefront adds up the groups' tiles
// (a lane has a group) and looks for its own number.  Offsets outside of 0 .. n count as the nearest of the two.
// EVEN: the tiles of a group have as many rows each, to the next 32; and tiles of 256 rows are full with 192 where that takes the whole launch
// fewer rounds of the CUs (a round takes 7/8 of one with 256), which only the rows of the groups tell: 8 groups of 512 rows on average, 4096 ->
// 8192, us: 3 rounds of 256 rows 320, of 192 rows 282; 8 of 1125, 2048 -> 7168: 5 rounds 305, 6 rounds of 192 rows 320.
template <int TM, bool EVEN> __device__ __forceinline__ bool find_group(const LinearArgs& p, int lane, LinearBlock& b, int& tile_n) {
    const int positions = (int)p.n;
    auto group = [&](int e, int& from) {
        from = e < p.experts ? min(max(p.offsets[e], 0), positions) : 0;
        const int to = e < p.experts ? min(max(p.offsets[e + 1], 0), positions) : 0;
        return max(to - from, 0);
    };
    constexpr int LESS = EVEN ? linear_least_rows(TM) : TM;
    bool less = false;
    auto tiles_of = [&](int rows) { return LESS < TM && less ? (rows + LESS - 1) / LESS : (rows + TM - 1) / TM; };
    auto last = [](int v) { return (uint32_t)__builtin_amdgcn_readlane(v, 63); };
    int from0;
    const int rows0 = group(lane, from0);
    auto count = [&](int& sum0) {
        sum0 = wave_scan(tiles_of(rows0), lane);
        uint32_t all = last(sum0);
        for (int c = 64; c < p.experts; c += 64) {
            int from;
            const int rows = group(c + lane, from);
            all += last(wave_scan(tiles_of(rows), lane));
        }
        return all;
    };
    int sum0;
    uint32_t all = count(sum0);
    if constexpr (LESS < TM) {
        int sum_less;
        less = true;
        const uint32_t all_less = count(sum_less);
        auto rounds = [&](uint32_t tiles) { return (tiles * (uint32_t)p.tiles_n + 255) / 256; };
        less = rounds(all_less) * 7 < rounds(all) * 8;
        if (less) {
            all = all_less;
            sum0 = sum_less;
        }
    }
    uint32_t t;
    if (!number_of(blockIdx.x, all * (uint32_t)p.tiles_n, t)) return false;
    uint32_t before = 0;                              // tiles of the groups before the 64 that are looked at
    for (int c = 0; c < p.experts; c += 64) {
        int from = from0, rows = rows0, sum = sum0;
        if (c > 0) {
            rows = group(c + lane, from);
            sum = wave_scan(tiles_of(rows), lane);
        }
        const uint64_t past = __ballot((before + (uint32_t)sum) * (uint32_t)p.tiles_n > t);
        if (past) {
            const int at = __builtin_ctzll(past);
            from = __builtin_amdgcn_readlane(from, at);
            rows = __builtin_amdgcn_readlane(rows, at);
            const int tiles = tiles_of(rows);
            const uint32_t mine = before + (uint32_t)__builtin_amdgcn_readlane(sum, at) - (uint32_t)tiles;
            int tile_m;
            tile_of(t - mine * (uint32_t)p.tiles_n, (uint32_t)tiles, (uint32_t)p.tiles_n, tile_m, tile_n);
            b.expert = c + at;
            int step = LESS < TM && less ? LESS : TM;
            if constexpr (EVEN) {
                uint32_t rest;
                const int full = step;
                step = uniform((int)divide((uint32_t)rows, (uint32_t)tiles, rest));   // (rows < 2^21 in one group: else the tiles are full)
                step = rows < 1 << 21 ? min((step + (rest > 0) + 31) & ~31, full) : full;
            }
            b.first = from + (int64_t)tile_m * step;
            b.rows = max(0, min(step, rows - tile_m * step));
            b.once = tiles == 1;
            return true;
        }
        before += (uint32_t)__builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// The tile of a block: TM = 16 FA WM rows (tokens) x TN = 16 FB WN columns (rows of W), W wavefronts in a grid of WM x WN, times WK that
// divide K: a slice is 64 WK KS bytes of every row, of which a wavefront multiplies 64 KS, and every fragment of a slice is
// read from LDS by WN (of W: WM) wavefronts only.  D slices are in LDS (DIRECT) or in registers, on their way to two in LDS.
template <typename T, bool DIRECT, int FA, int FB, int WM, int WN, int WK, int KS, int D>
struct LinearTile {
    static constexpr int TM = 16 * FA * WM, TN = 16 * FB * WN, SL = 64 * WK * KS;
    static constexpr int W = WM * WN * WK;
    static constexpr int UA = TM * SL, UB = TN * SL, LA = UA / (1024 * W), LB = UB / (1024 * W);    // bytes of a slice, loads (16 bytes a lane) of a wavefront
    static constexpr int kRing = (DIRECT ? D : 2) * (UA + UB);
    // row blocks of a wavefront that pass through LDS at a time behind the products: as many as the ring has room for
    static constexpr int kRowBytes = WK * WM * 16 * TN * 4;
    static constexpr int fit(int n) { return n == 1 || (FA % n == 0 && n * kRowBytes <= kRing) ? n : fit(n - 1); }
    static constexpr int RB = fit(FA), kLds = RB * kRowBytes > kRing ? RB * kRowBytes : kRing;
    static_assert((W == 8 || W == 4) && UA % (1024 * W) == 0 && UB % (1024 * W) == 0 && kLds <= kLdsBytes, "whole loads");
    static_assert(DIRECT ? D >= 2 && (D - 1) * (LA + LB) <= 63 : D % 2 == 0, "slices under way");
};

// the row of x that is row m of this block's; -1: none
template <bool GROUPED> __device__ __forceinline__ int64_t token_of_row(const LinearArgs& p, const LinearBlock& b, int m) {
    if (m >= b.rows) return -1;
    if (!GROUPED || !p.order) return b.first + m;
    const int32_t at = p.order[b.first + m];
    const uint32_t slot = (uint32_t)at;
    uint32_t token = __umulhi(slot, p.inv_per_token);       // the quotient, or one less
    if (slot - token * (uint32_t)p.per_token >= (uint32_t)p.per_token) ++token;
    return at >= 0 && (int64_t)token < p.x_rows ? (int64_t)token : -1;
}

// What follows the products of W wavefronts in a grid of WM x WN, times WK that divide K.
// acc[i][j][q] = row (WM i + wm) 16 + lane % 16, column (wn FB + j) 16 + 4 (lane / 16) + q of the tile.  RB row blocks of a wavefront at a time
// pass through LDS, where the parts of K meet (WK = 1: every wavefront's own), so that a store covers whole lines of a row and that what
// is done to the elements is a loop; a thread finishes 8 neighbouring columns at once.
// Loads and stores are counted by one counter, in their order: a load in the loop would wait for the stores of the turn before, 1.5 us each
// (behind the products of a 256 x 256 tile with GELU 21.4 us, as here 15.6, of which the activation's instructions are 8.5).  So which rows are
// there is known before the first store, bias is waited for there, and residuals are loaded for several rows at once, in a loop of their own.
template <typename T, bool GROUPED, int W, int FA, int FB, int WM, int WN, int WK, int RB>
__device__ __forceinline__ void finish_linear(const LinearArgs& p, const LinearBlock& b, f32x4_t (&acc)[FA][FB], unsigned char* lds, int tid) {
    static_assert(FA % RB == 0, "all row blocks");
    constexpr bool OWN = WK == 1;
    constexpr int COLS = OWN ? FB * 16 : WN * FB * 16, ROWS = OWN ? RB * 16 : WM * RB * 16, UNITS = COLS / 8, STRIDE = (OWN ? 64 : W * 64) / UNITS;
    static constexpr int TURNS = (ROWS + STRIDE - 1) / STRIDE, kAtOnce = OWN && TURNS % 4 == 0 ? 4 : TURNS % 2 == 0 ? 2 : 1;
    static_assert(TURNS * (FA / RB) <= 32, "a bit for each row of a thread");
    const int lane = tid & 63, wave = uniform(tid >> 6), wk = wave % WK, wn = wave / WK % WN, wm = wave / WK / WN, frow = lane & 15, fp = lane >> 4;
    const int me = OWN ? lane : tid, unit = me % UNITS;
    float* stage = reinterpret_cast<float*>(lds) + (OWN ? wave * ROWS * COLS : 0);
    auto place_of = [&](int part, int row, int piece) { return (part * ROWS + row) * COLS + ((piece ^ (row & 15 & (COLS / 4 - 1))) * 4); };
    auto sync = [&]() {
        if constexpr (OWN) __builtin_amdgcn_wave_barrier();
        else __syncthreads();
    };
    const int64_t n = b.n0 + (OWN ? wn * COLS : 0) + unit * 8;
    const int columns = (int)min((int64_t)8, p.N - n);    // (of this thread; none or less: none)
    // (as 16 bytes of 8 bf16 or 32 of 8 fp32; columns that are not there: 0)
    auto load8 = [&](const void* from, int64_t at, bool f32, td_u32x4 (&w)[2]) {
        if (columns >= 8) {
            w[0] = load_any16(static_cast<const unsigned char*>(from) + at * (f32 ? 4 : 2));
            if (f32) w[1] = load_any16(static_cast<const float*>(from) + at + 4);
        } else {
            w[0] = w[1] = td_u32x4{0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q < columns) {
                    const uint32_t e = f32 ? static_cast<const uint32_t*>(from)[at + q] : (uint32_t)static_cast<const bf16_t*>(from)[at + q] << (16 * (q & 1));
                    const uint32_t as_f32 = f32 ? e : w[q / 4][q % 4], as_bf16 = f32 ? w[0][q / 2] : w[0][q / 2] | e;
                    if (q / 4 != 0 || q % 4 != q / 2) {
                        w[q / 4][q % 4] = as_f32;
                        w[0][q / 2] = as_bf16;
                    } else {
                        w[0][q / 2] = f32 ? as_f32 : as_bf16;
                    }
                }
        }
    };
    auto value = [](const td_u32x4 (&w)[2], bool f32, int q) {
        const uint32_t as_f32 = w[q / 4][q % 4], pair = w[0][q / 2];
        return __uint_as_float(f32 ? as_f32 : q & 1 ? pair & 0xffff0000u : pair << 16);
    };
    float bias[8] = {};
    if (p.b && !p.part && columns > 0) {
        td_u32x4 w[2];
        load8(p.b, (int64_t)b.expert * p.N + n, sizeof(T) == 4, w);
#pragma unroll
        for (int q = 0; q < 8; ++q) bias[q] = value(w, sizeof(T) == 4, q);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) asm volatile("" : "+v"(bias[q]));
    // row of the tile that the thread has in turn t of the row blocks from i0 on
    auto row_of = [&](int i0, int t, int& at) {
        at = me / UNITS + t * STRIDE;
        const int block = OWN ? wm + WM * (at / 16) : at / (RB * 16) + WM * (at / 16 % RB);
        return (i0 * WM + block) * 16 + at % 16;
    };
    uint32_t there = 0;
#pragma unroll
    for (int t = 0; t < TURNS * (FA / RB); ++t) {
        int at;
        const int m = row_of(t / TURNS * RB, t % TURNS, at);
        const bool in = at < ROWS && columns > 0 && (GROUPED ? token_of_row<GROUPED>(p, b, m) >= 0 : m < b.rows);
        there |= in ? 1u << t : 0u;
    }
    asm volatile("" : "+v"(there));
    const bool part = !GROUPED && p.part, residual = !GROUPED && p.r && !part;      // (of groups neither)
    for_constants<FA / RB>([&](auto batch) {
        constexpr int i0 = decltype(batch)::value * RB, first = decltype(batch)::value * TURNS;
        if constexpr (i0 > 0) sync();
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j)
                *reinterpret_cast<f32x4_t*>(stage + place_of(wk, ((OWN ? 0 : wm * RB) + i) * 16 + frow, ((OWN ? 0 : wn * FB) + j) * 4 + fp)) = acc[i0 + i][j];
        sync();
        // (sums of a range of K: act is the identity, without bias and residual)
        with_linear_act(p.act, [&](auto act) {
            auto sum_and_act = [&](int at, float (&v)[8]) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    f32x4_t sum = *reinterpret_cast<const f32x4_t*>(stage + place_of(0, at, unit * 2 + h));
#pragma unroll
                    for (int part = 1; part < WK; ++part) sum += *reinterpret_cast<const f32x4_t*>(stage + place_of(part, at, unit * 2 + h));
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[4 * h + q] = linear_act<decltype(act)::value>(sum[q] + bias[4 * h + q]);
                }
            };
            auto store = [&](int64_t to, const float (&v)[8]) {
                if (part || p.out_f32) {
                    float* y = part ? p.part + (int64_t)b.range * p.n * p.N + to : static_cast<float*>(p.y) + to;
                    if (columns >= 8) {
                        store_any16(y, td_u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
                        store_any16(y + 4, td_u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])});
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (q < columns) y[q] = v[q];
                    }
                } else {
                    bf16_t* y = static_cast<bf16_t*>(p.y) + to;
                    const td_u32x4 o = {to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]), to_bf16x2(v[4], v[5]), to_bf16x2(v[6], v[7])};
                    if (columns >= 8) {
                        store_any16(y, o);
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (q < columns) y[q] = (bf16_t)(o[q / 2] >> (16 * (q & 1)));
                    }
                }
            };
            // (kAtOnce rows side by side; outside of the tile's rows nothing is stored)
            auto turns = [&](auto add) {
#pragma unroll 1
                for (int t0 = 0; t0 < TURNS; t0 += kAtOnce) {
                    td_u32x4 r[kAtOnce][2];
                    int at[kAtOnce];
                    int64_t to[kAtOnce];
                    float v[kAtOnce][8];
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u) {
                        to[u] = (b.first + row_of(i0, t0 + u, at[u])) * p.N + n;
                        if constexpr (decltype(add)::value)
                            if (there >> (first + t0 + u) & 1) load8(p.r, to[u], p.out_f32, r[u]);
                    }
                    if constexpr (decltype(add)::value)
#pragma unroll
                        for (int u = 0; u < kAtOnce; ++u) asm volatile("" : "+v"(r[u][0]), "+v"(r[u][1]));
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u) {
                        sum_and_act(min(at[u], ROWS - 1), v[u]);
                        if constexpr (decltype(add)::value)
#pragma unroll
                            for (int q = 0; q < 8; ++q) v[u][q] += value(r[u], p.out_f32, q);
                    }
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u)
                        if (there >> (first + t0 + u) & 1) store(to[u], v[u]);
                }
            };
            if constexpr (!GROUPED && decltype(act)::value != kActGelu16)   // (alone: linear_act.h)
                if (residual) return turns(std::true_type{});
            turns(std::false_type{});
        });
    });
}

// What bounds it: few rows - the weights' stream from HBM; many - the way from L2 to LDS (tiles below 192 x 128) and the matrix cores.
// DIRECT: x and W in whole, aligned pieces of 16 bytes, which go from memory straight to LDS; D - 1 slices are under way.  Else: through
// registers, D slices ahead, whatever the alignment (odd widths, odd pitches, rows that are 8 MB apart, gathered ones of 3.5 GB; aligned ones where the rule in linear.hip finds
// it faster: 509 x 1500 x 1000 in fp32).
template <typename T, bool GROUPED, bool DIRECT, int FA, int FB, int WM, int WN, int WK, int KS, int D>
__global__ void __launch_bounds__(64 * WM * WN * WK, 2) linear_kernel(LinearArgs p) {
    typedef LinearTile<T, DIRECT, FA, FB, WM, WN, WK, KS, D> G;
    constexpr int TM = G::TM, TN = G::TN, SL = G::SL, LA = G::LA, LB = G::LB, PS = SL / 16, RPL = 64 / PS, SWZ = PS < 16 ? PS - 1 : 15;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int wk = wave % WK, wn = wave / WK % WN, wm = wave / WK / WN, frow = lane & 15, fp = lane >> 4;

    LinearBlock b;
    int tile_n;
    const int slices = (int)((p.k + SL - 1) / SL);
    if constexpr (GROUPED) {
        if (!find_group<TM, false>(p, lane, b, tile_n)) return;
        b.s0 = b.range = 0;
        b.nk = slices;
    } else {
        uint32_t t, in_range;
        if (!number_of(blockIdx.x, (uint32_t)(p.tiles_m * p.tiles_n * p.splits), t)) return;
        int tile_m;
        b.range = uniform((int)divide(t, (uint32_t)(p.tiles_m * p.tiles_n), in_range));
        tile_of(in_range, (uint32_t)p.tiles_m, (uint32_t)p.tiles_n, tile_m, tile_n);
        b.expert = 0;
        b.first = (int64_t)tile_m * TM;
        b.rows = (int)min((int64_t)TM, p.n - b.first);
        b.s0 = b.range * p.slices;
        b.nk = max(0, min(p.slices, slices - b.s0));
        b.once = p.tiles_m == 1;
    }
    b.n0 = (int64_t)tile_n * TN;
    const int rows_w = (int)min((int64_t)TN, p.N - b.n0);
    const unsigned char* W = p.W + ((size_t)b.expert * p.N + b.n0) * p.k;
    // whole slices from a starting point of this block's own, then one that is not whole
    const int whole = max(0, min(b.nk, (int)(p.k / SL) - b.s0));
    const int rot = start_of(b, whole);
    auto slice_of = [&](int t) { return b.s0 + (t >= whole ? t : t + rot >= whole ? t + rot - whole : t + rot); };

    // A load is RPL rows x SL bytes: lane -> row lane / PS, slot lane % PS, which holds piece slot ^ row (so the 16 rows of a fragment
    // hit all banks).  Wavefront w loads the w-th part of the rows of x, of W alike.
    const int row_a = wave * (TM / G::W) + lane / PS, row_b = wave * (TN / G::W) + lane / PS;
    auto piece_of_row = [&](int row) { return (uint32_t)((lane % PS) ^ (row & SWZ)) * 16u; };
    auto token_of = [&](int m) { return token_of_row<GROUPED>(p, b, m); };

    f32x4_t acc[FA][FB];
#pragma unroll
    for (int i = 0; i < FA; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j) acc[i][j] = f32x4_t{0, 0, 0, 0};
    // fragments: lane holds 16 bytes of row lane % 16 at piece 4 (wk + WK step) + lane / 16 of a slice
    uint32_t frag[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) frag[s] = (uint32_t)(frow * SL + (((4 * (wk + WK * s) + fp) ^ (frow & SWZ)) * 16));
    struct Fragments {
        td_u32x4 a[KS][FA], b[KS][FB];
    };
    // (rows: the row blocks of a wavefront that are there, see below)
    auto read = [&](auto rows, Fragments& f, const unsigned char* at_a, const unsigned char* at_b) {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
#pragma unroll
            for (int i = 0; i < decltype(rows)::value; ++i) f.a[s][i] = *reinterpret_cast<const td_u32x4*>(at_a + (WM * i + wm) * (16 * SL) + frag[s]);
#pragma unroll
            for (int j = 0; j < FB; ++j) f.b[s][j] = *reinterpret_cast<const td_u32x4*>(at_b + (wn * FB + j) * (16 * SL) + frag[s]);
        }
    };
    auto multiply = [&](auto rows, const Fragments& f) {
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int i = 0; i < decltype(rows)::value; ++i)
#pragma unroll
                for (int j = 0; j < FB; ++j) mma_pieces<T>(acc[i][j], f.b[s][j], f.a[s][i]);
    };

    if constexpr (DIRECT) {
        const uint32_t base = (uint32_t)uniform((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds);
        const bool gather = GROUPED && p.order;
        // (p.x_bytes: up to the last row's end; offsets of rows that are not there lie past it, where nothing is fetched)
        const i32x4_t ra = gather ? buffer_of(p.x, (uint32_t)p.x_bytes)
                                  : buffer_of(p.x + b.first * p.x_pitch, (uint32_t)((b.rows - 1) * p.x_pitch) + p.k);
        const i32x4_t rb = buffer_of(W, (uint32_t)rows_w * p.k);
        uint32_t off_a[LA], off_b[LB];
#pragma unroll
        for (int i = 0; i < LA; ++i) {
            const int row = row_a + i * RPL;
            uint32_t at;
            if (gather) {
                const int64_t token = token_of(row);
                at = token < 0 ? kNowhere : (uint32_t)token * (uint32_t)p.x_pitch;
            } else {
                at = row < b.rows ? (uint32_t)row * (uint32_t)p.x_pitch : kNowhere;
            }
            off_a[i] = at + piece_of_row(row);
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            const int row = row_b + i * RPL;
            off_b[i] = (row < rows_w ? (uint32_t)row * p.k : kNowhere) + piece_of_row(row);
        }
#pragma unroll
        for (int i = 0; i < LA; ++i) asm volatile("" : "+v"(off_a[i]));   // (waited for here, not between the loads below)
        const uint32_t to_a = base + (uint32_t)wave * (G::UA / G::W), to_b = base + (uint32_t)(D * G::UA) + (uint32_t)wave * (G::UB / G::W);
        auto load_slice = [&](int t, uint32_t slot) {     // (past the last slice: an empty buffer)
            const bool live = t < b.nk;
            const uint32_t soff = live ? (uint32_t)slice_of(t) * SL : 0u;
            i32x4_t a = ra, w = rb;
            a.z = live ? a.z : 0;
            w.z = live ? w.z : 0;
            const uint32_t last = p.k - soff;             // bytes of the row from here on
            if (live && last < (uint32_t)SL) {            // the pieces that the row has not: its first one of this slice
#pragma unroll
                for (int i = 0; i < LB; ++i) {
                    const uint32_t pc = piece_of_row(row_b + i * RPL);
                    load_to_lds(to_b + slot * G::UB + i * 1024u, off_b[i] - (pc < last ? 0u : pc), w, soff);
                }
#pragma unroll
                for (int i = 0; i < LA; ++i) {
                    const uint32_t pc = piece_of_row(row_a + i * RPL);
                    load_to_lds(to_a + slot * G::UA + i * 1024u, off_a[i] - (pc < last ? 0u : pc), a, soff);
                }
            } else {
                if (b.once) {
#pragma unroll
                    for (int i = 0; i < LB; ++i) load_to_lds<true>(to_b + slot * G::UB + i * 1024u, off_b[i], w, soff);
                } else {
#pragma unroll
                    for (int i = 0; i < LB; ++i) load_to_lds(to_b + slot * G::UB + i * 1024u, off_b[i], w, soff);
                }
#pragma unroll
                for (int i = 0; i < LA; ++i) load_to_lds(to_a + slot * G::UA + i * 1024u, off_a[i], a, soff);
            }
        };
        auto arrived = [&](auto behind) {                 // all but the newest D - behind slices; the barrier makes it everybody's
            __builtin_amdgcn_s_waitcnt(0xc07f);           // lgkmcnt(0): the fragments read before are in registers
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - decltype(behind)::value) * (LA + LB)) : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
#pragma unroll 1
        for (int s = 0; s < D; ++s) load_slice(s, (uint32_t)s);
        auto products = [&](auto rows) {
            uint32_t slot = 0;                            // of the slice that is read next
            auto fetch = [&](Fragments& f, int t) {
                read(rows, f, lds + slot * G::UA, lds + D * G::UA + slot * G::UB);
                if (t >= whole) {                         // a slice that is not whole: what the row has not is zero
                    const td_u32x4 zero = {0, 0, 0, 0};
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        const bool in = (uint32_t)slice_of(t) * SL + (uint32_t)(4 * (wk + WK * s) + fp) * 16u < p.k;
#pragma unroll
                        for (int i = 0; i < decltype(rows)::value; ++i) f.a[s][i] = in ? f.a[s][i] : zero;
#pragma unroll
                        for (int j = 0; j < FB; ++j) f.b[s][j] = in ? f.b[s][j] : zero;
                    }
                }
            };
            Fragments f[2];
            auto step = [&](const Fragments& now, Fragments& next, int t) {
                arrived(num<2>{});                        // slice t + 1 is here, and slice t's place is free
                const uint32_t free = slot;
                slot = slot + 1 == D ? 0 : slot + 1;
                load_slice(t + D, free);
                if (t + 1 < b.nk) fetch(next, t + 1);
                multiply(rows, now);
            };
            if (b.nk > 0) {
                arrived(num<1>{});
                fetch(f[0], 0);
            }
#pragma unroll 1
            for (int t = 0; t < b.nk; t += 2) {
                step(f[0], f[1], t);
                if (t + 1 < b.nk) step(f[1], f[0], t + 1);
            }
        };
        // (a tile that is at most half full: its row blocks are dealt out to the wavefronts in turns, so each has half of them)
        if (FA >= 4 && b.rows <= TM / 2) products(num<(FA >= 4 ? FA / 2 : FA)>{});
        else products(num<FA>{});
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    } else {
        // (for rows that are not there the first one's, of which nothing is kept: the loop has no branches, so that a load is waited
        // for when it is used and not where paths meet)
        const unsigned char *from_a[LA], *from_b[LB];
#pragma unroll
        for (int i = 0; i < LA; ++i) from_a[i] = p.x + max(token_of(row_a + i * RPL), (int64_t)0) * p.x_pitch + piece_of_row(row_a + i * RPL);
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            const int row = row_b + i * RPL;
            from_b[i] = W + (size_t)(row < rows_w ? row : 0) * p.k + piece_of_row(row);
        }
        struct Pieces {
            td_u32x4 a[LA], b[LB];
        };
        auto to_lds = [&](const Pieces& v, int place) {
            unsigned char* at = lds + wave * (G::UA / G::W) + place * G::UA + lane * 16;
#pragma unroll
            for (int i = 0; i < LA; ++i) *reinterpret_cast<td_u32x4*>(at + i * 1024) = v.a[i];
            at = lds + 2 * G::UA + wave * (G::UB / G::W) + place * G::UB + lane * 16;
#pragma unroll
            for (int i = 0; i < LB; ++i) *reinterpret_cast<td_u32x4*>(at + i * 1024) = v.b[i];
        };
        auto load_slice = [&](Pieces& v, int t) {         // (past the last whole slice: that one again)
            const uint32_t soff = (uint32_t)slice_of(min(t, whole - 1)) * SL;
#pragma unroll
            for (int i = 0; i < LB; ++i) v.b[i] = load_any16(from_b[i] + soff);
#pragma unroll
            for (int i = 0; i < LA; ++i) v.a[i] = load_any16(from_a[i] + soff);
        };
        Pieces v[D];
        auto step = [&](Pieces& now, int t) {             // (the place in LDS was read two slices ago, before the last barrier)
            const int place = t & 1;
            to_lds(now, place);
            __syncthreads();
            load_slice(now, t + D);
            Fragments f;
            read(num<FA>{}, f, lds + place * G::UA, lds + 2 * G::UA + place * G::UB);
            multiply(num<FA>{}, f);
        };
        if (whole > 0) {
#pragma unroll
            for (int u = 0; u < D; ++u) load_slice(v[u], u);
            int t = 0;
#pragma unroll 1
            for (; t + D <= whole; t += D)
#pragma unroll
                for (int u = 0; u < D; ++u) step(v[u], t + u);
#pragma unroll
            for (int u = 0; u < D; ++u)
                if (t + u < whole) step(v[u], t + u);
        }
        if (whole < b.nk) {                               // a slice that is not whole: element by element, zeros behind the row's end
            const uint32_t soff = (uint32_t)slice_of(whole) * SL;
            auto load_piece = [&](const unsigned char* from, uint32_t pc) {
                td_u32x4 w = {0, 0, 0, 0};
                const T* el = reinterpret_cast<const T*>(from + soff);
                const uint32_t n = soff + pc < p.k ? (p.k - soff - pc) / sizeof(T) : 0u;
#pragma unroll
                for (uint32_t u = 0; u < 16 / sizeof(T); ++u)
                    if (u < n) {
                        if constexpr (sizeof(T) == 2) w[u / 2] |= (uint32_t)el[u] << (16 * (u & 1));
                        else w[u] = __float_as_uint(el[u]);
                    }
                return w;
            };
#pragma unroll
            for (int i = 0; i < LB; ++i) v[0].b[i] = load_piece(from_b[i], piece_of_row(row_b + i * RPL));
#pragma unroll
            for (int i = 0; i < LA; ++i) v[0].a[i] = load_piece(from_a[i], piece_of_row(row_a + i * RPL));
            to_lds(v[0], whole & 1);
            __syncthreads();
            Fragments f;
            read(num<FA>{}, f, lds + (whole & 1) * G::UA, lds + 2 * G::UA + (whole & 1) * G::UB);
            multiply(num<FA>{}, f);
        }
    }
    __syncthreads();

    finish_linear<T, GROUPED, G::W, FA, FB, WM, WN, WK, G::RB>(p, b, acc, lds, tid);
}

}  // namespace

// ---------------------------------------------------------------- launches, for one element type
namespace {

// f(direct, row and column blocks of a wavefront, grid of wavefronts, wavefronts and half-lines of each in K, slices in LDS)
template <typename T, bool GROUPED, typename F> void for_linear_shape(bool direct, int shape, F f) {
    auto use = [&](auto number, auto d, auto... tile) {
        if constexpr (linear_has(sizeof(T), decltype(d)::value, GROUPED, decltype(number)::value)) f(d, tile...);
    };
    if (direct) {
        switch (shape) {
            case 0: use(num<0>{}, std::true_type{}, num<1>{}, num<1>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<5>{}); break;
            case 1: use(num<1>{}, std::true_type{}, num<1>{}, num<2>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<3>{}); break;
            case 2: use(num<2>{}, std::true_type{}, num<1>{}, num<4>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<4>{}); break;
            case 3: use(num<3>{}, std::true_type{}, num<2>{}, num<1>{}, num<1>{}, num<2>{}, num<4>{}, num<1>{}, num<5>{}); break;
            case 4: use(num<4>{}, std::true_type{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<4>{}, num<1>{}, num<6>{}); break;
            case 5: use(num<5>{}, std::true_type{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<4>{}, num<1>{}, num<6>{}); break;
            case 6: use(num<6>{}, std::true_type{}, num<4>{}, num<2>{}, num<1>{}, num<2>{}, num<4>{}, num<1>{}, num<5>{}); break;
            case 7: use(num<7>{}, std::true_type{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<5>{}); break;
            case 8: use(num<8>{}, std::true_type{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<6>{}); break;
            case 9: use(num<9>{}, std::true_type{}, num<4>{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<5>{}); break;
            case 10: use(num<10>{}, std::true_type{}, num<6>{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<4>{}); break;
            case 11: use(num<11>{}, std::true_type{}, num<1>{}, num<1>{}, num<1>{}, num<1>{}, num<8>{}, num<2>{}, num<5>{}); break;
            case 12: use(num<12>{}, std::true_type{}, num<2>{}, num<1>{}, num<1>{}, num<2>{}, num<4>{}, num<2>{}, num<5>{}); break;
            // short rows, whose tiles are mostly beginnings and ends: four wavefronts and two slices, so that 5, 3 and 2 of them are on a CU
            // (3000 x 16384 x 256, us, best of the others / these: 66 / 56; 5000 x 2048 x 256 19.5 / 15.9; 600 x 8000 x 64 9.6 / 7.7)
            case 13: use(num<13>{}, std::true_type{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<2>{}); break;
            case 14: use(num<14>{}, std::true_type{}, num<2>{}, num<4>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<2>{}); break;
            default: use(num<15>{}, std::true_type{}, num<4>{}, num<4>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}, num<2>{}); break;
        }
    } else {
        switch (shape) {
            case 0: use(num<0>{}, std::false_type{}, num<1>{}, num<1>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<6>{}); break;
            case 1: use(num<1>{}, std::false_type{}, num<1>{}, num<2>{}, num<1>{}, num<1>{}, num<8>{}, num<1>{}, num<4>{}); break;
            case 2: use(num<2>{}, std::false_type{}, num<2>{}, num<1>{}, num<1>{}, num<2>{}, num<4>{}, num<1>{}, num<4>{}); break;
            case 3: use(num<3>{}, std::false_type{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<4>{}); break;
            default: use(num<4>{}, std::false_type{}, num<4>{}, num<4>{}, num<2>{}, num<2>{}, num<2>{}, num<1>{}, num<2>{}); break;
        }
    }
}

template <typename T, bool GROUPED> bool linear_raise() {
    bool ok = true;
    for (int direct = 0; direct < 2; ++direct)
        for (int shape = 0; shape < (direct ? kLinearShapes : kLinearStagedShapes); ++shape)
            for_linear_shape<T, GROUPED>(direct, shape, [&](auto d, auto fa, auto fb, auto wm, auto wn, auto wk, auto ks, auto ring) {
                typedef LinearTile<T, decltype(d)::value, fa, fb, wm, wn, wk, ks, ring> G;
                const LinearShape& is = direct ? kLinearShape[shape] : kLinearStaged[shape];
                ok &= is.m == G::TM && is.n == G::TN && is.slice == G::SL;
                ok &= hipFuncSetAttribute(reinterpret_cast<const void*>(linear_kernel<T, GROUPED, decltype(d)::value, fa, fb, wm, wn, wk, ks, ring>),
                                          hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds) == hipSuccess;
            });
    return ok;
}

template <typename T> tardis_status_t linear_init() {
    return linear_raise<T, false>() && linear_raise<T, true>() ? TARDIS_OK : TARDIS_ERR_HIP;
}

template <typename T, bool GROUPED> void linear_launch(const LinearArgs& p, bool direct, int shape, int blocks, hipStream_t s) {
    for_linear_shape<T, GROUPED>(direct, shape, [&](auto d, auto fa, auto fb, auto wm, auto wn, auto wk, auto ks, auto ring) {
        typedef LinearTile<T, decltype(d)::value, fa, fb, wm, wn, wk, ks, ring> G;
        constexpr int bytes = G::kLds, threads = 64 * G::W;
        hipLaunchKernelGGL((linear_kernel<T, GROUPED, decltype(d)::value, fa, fb, wm, wn, wk, ks, ring>), dim3((unsigned)blocks), dim3(threads), bytes, s, p);
    });
}

template <typename T> void linear_launch(const LinearArgs& p, bool grouped, bool direct, int shape, int blocks, hipStream_t s) {
    if (grouped) linear_launch<T, true>(p, direct, shape, blocks, s);
    else linear_launch<T, false>(p, direct, shape, blocks, s);
}

}  // namespace
