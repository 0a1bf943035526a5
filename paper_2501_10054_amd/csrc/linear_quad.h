// The linear layer (and the grouped one) for large tiles, aligned rows, in bf16 (linear_quad.hip) and in e4m3 for outputs in bf16 (linear_fp8_quad.hip).
// 4 wavefronts, one per SIMD, in a 2 x 2 grid: 32 NA rows x 32 NB columns.
//
// Why beside linear_kernel: at 192 x 128 and below its eight wavefronts the LDS is the limit (a slice of 128 bytes takes 960 cycles of LDS reads and
// writes for 768 of MFMA).  A wavefront with 128 x 128 of a 256 x 256 tile reads a slice's fragments from LDS for twice as many MFMAs: 1536 cycles
// for 2048.  Its accumulators fill the second half of the register file, and one wavefront on a SIMD hides nothing behind another one, so
// what stands between two MFMAs (16 cycles, four issue slots) is placed by hand, one thing to a gap: a fragment read in every second gap of
// a half slice; over the whole slice, in equal distances, the loads that refill the ring, m0 in one gap and the load in the next (which
// is also the wait state between them).  The MFMAs are inline assembly, because the compiler, given the builtins, moves accumulators between the halves
// of the register file; so the waits they need are written out here, and the listing's test reads them.
//
// e4m3: a slice has the same bytes and takes the same cycles for twice as many products: an instruction of 32 x 32 results takes 64 bytes of K, in four gaps
// of 16 cycles, from two pieces of a row in a lane.  (One of 16 x 16 takes 128 bytes, both halves of a slice, for which there are not registers twice.)
// Lane l has row l % 32 of two row blocks, pieces 2 (l / 32) and the next of half a slice.  2048 x 4096 -> 16384 on 256 x 128 tiles, weights from HBM: 134 us, 2.05 PFLOP/s; the
// matrix cores work 57 % of the cycles of a slice, the rest waits for the slices' way from L2 (39 bytes a ns and CU).
#pragma once
#include "linear_tile.h"

namespace {

constexpr int kNoLds = 0xc07f;                              // s_waitcnt lgkmcnt(0)

template <int NA, int NB> struct LinearQuad {
    static constexpr int SL = 128, TM = 32 * NA, TN = 32 * NB, UA = TM * SL, UB = TN * SL;
    // slices in LDS; of the rows of x one more where the two do not fit equally often
    static constexpr int SB = kLdsBytes / (UA + UB), SA = SB * (UA + UB) + UA <= kLdsBytes ? SB + 1 : SB;
    static constexpr int kPer = NA + NB;                    // loads of a wavefront per slice, and reads per half slice
    static constexpr int NM = NA * NB, TOT = 2 * NM;        // MFMAs (gaps) of half a slice, of a slice
    static constexpr int kEvery = TOT / kPer;               // gaps from load to load
    static constexpr int kFirst = (NM - 2 + kEvery) / kEvery;   // loads of a period that fall into its first half
    static constexpr int kTurnA = NM - 4, kTurnB = NM - 2;  // (gaps behind the reads)
    static constexpr int kWaitB = NA + (SB - 2) * kPer, kWaitA = (SA - 2) * kPer, kWait = kWaitB < kWaitA ? kWaitB : kWaitA;
    static constexpr int kStart = (SA > SB ? NA : 0) + (SB - 2) * kPer + kFirst;   // loads behind those of slice 0 in the prologue
    static constexpr int kRowBytes = 4 * 16 * NB * 16 * 4;
    static constexpr int kRing = SA * UA + SB * UB;
    // of `rows` row blocks of a wavefront so many at a time behind the products: a part of them that the ring has room for
    static constexpr int fit(int rows, int n) { return n == 1 || (rows % n == 0 && n * kRowBytes <= kRing) ? n : fit(rows, n - 1); }
    static constexpr int kLds = kRing;
    static_assert(kRowBytes <= kRing && SB >= 2 && kWait <= 63 && kStart <= 63 && kLds <= kLdsBytes, "slice buffers");
    static_assert(2 * kPer <= NM - 4 && kFirst * kEvery >= NM && (kPer - 1) * kEvery + 1 < TOT && kEvery * NB > 12, "places of reads and loads");
};

template <typename T, bool GROUPED, int NA, int NB>
__device__ __forceinline__ void linear_quad(const LinearArgs& p) {
    typedef LinearQuad<NA, NB> G;
    constexpr bool WIDE = sizeof(T) == 1;
    static_assert(!WIDE || (NA % 4 == 0 && NB % 4 == 0), "pairs of row blocks, also of half a tile");
    constexpr int SL = G::SL, TM = G::TM, TN = G::TN, SA = G::SA, SB = G::SB, NM = G::NM, TOT = G::TOT;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), wm = wave >> 1, wn = wave & 1;

    LinearBlock b;
    int tile_n;
    const int whole = (int)(p.k / SL);
    if constexpr (GROUPED) {
        if (!find_group<TM, true>(p, lane, b, tile_n) || b.rows == 0) return;
        b.s0 = b.range = 0;
        b.nk = whole;
    } else {
        uint32_t t, in_range;
        if (!number_of(blockIdx.x, (uint32_t)(p.tiles_m * p.tiles_n * p.splits), t)) return;
        int tile_m;
        b.range = uniform((int)divide(t, (uint32_t)(p.tiles_m * p.tiles_n), in_range));
        tile_of(in_range, (uint32_t)p.tiles_m, (uint32_t)p.tiles_n, tile_m, tile_n);
        b.expert = 0;
        b.first = (int64_t)tile_m * p.tile_rows;
        b.rows = (int)min((int64_t)p.tile_rows, p.n - b.first);
        if (b.rows <= 0) return;
        b.s0 = b.range * p.slices;
        b.nk = max(0, min(p.slices, whole - b.s0));
    }
    b.n0 = (int64_t)tile_n * TN;
    const int rows_w = (int)min((int64_t)TN, p.N - b.n0);
    const unsigned char* W = p.W + ((size_t)b.expert * p.N + b.n0) * p.k;
    const int rot = first_slice((int)blockIdx.x & 7, (int)blockIdx.x >> 3, b.nk);

    const bool gather = GROUPED && p.order;
    const i32x4_t ra = gather ? buffer_of(p.x, (uint32_t)p.x_bytes)
                              : buffer_of(p.x + b.first * p.x_pitch, (uint32_t)((b.rows - 1) * p.x_pitch) + p.k);
    const i32x4_t rb = buffer_of(W, (uint32_t)rows_w * p.k);
    // a load is 8 rows of 128 bytes: lane -> row lane / 8, piece (lane % 8) ^ row; wavefront w loads rows [w TM / 4, (w + 1) TM / 4) of x, of W alike
    // (e4m3: ^ 1 more in the second row block of each pair, whose lanes read in one cycle with the first's)
    const uint32_t lrow = (uint32_t)lane >> 3, piece = (((uint32_t)lane & 7u) ^ lrow) * 16u;
    auto piece_a = [&](int i) { return WIDE ? piece ^ ((uint32_t)i / 4 % 2 * 16u) : piece; };
    auto piece_b = [&](int i) { return WIDE ? piece ^ ((uint32_t)i / 2 % 2 * 16u) : piece; };
    uint32_t off_a[NA], off_b[NB];
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        const int row = wave * (TM / 4) + i * 8 + (int)lrow;
        uint32_t at = row < b.rows ? (uint32_t)row * (uint32_t)p.x_pitch : kNowhere;
        if (gather) {
            const int64_t token = token_of_row<GROUPED>(p, b, row);
            at = token < 0 ? kNowhere : (uint32_t)token * (uint32_t)p.x_pitch;
        }
        off_a[i] = at + piece_a(i);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int row = wave * (TN / 4) + i * 8 + (int)lrow;
        off_b[i] = (row < rows_w ? (uint32_t)row * p.k : kNowhere) + piece_b(i);
    }
#pragma unroll
    for (int i = 0; i < NA; ++i) asm volatile("" : "+v"(off_a[i]));
#pragma unroll
    for (int i = 0; i < NB; ++i) asm volatile("" : "+v"(off_b[i]));
    const uint32_t base = (uint32_t)uniform((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds);
    const uint32_t lds_a = (uint32_t)uniform((int)(base + (uint32_t)wave * (G::UA / 4)));
    const uint32_t lds_b = (uint32_t)uniform((int)(base + SA * G::UA + (uint32_t)wave * (G::UB / 4)));

    // The slice that the next loads of x (of W) fetch, found in steps, which stand in different gaps.  Past the last one nothing is to be
    // fetched: an empty buffer, and no offset either (the hardware compares with num_records - soff).
    struct Stream {
        i32x4_t rs;
        uint32_t soff, to;                        // offset in K; ring buffer of this wavefront
        int t, s;                                 // number in the sequence, slice
    };
    auto find = [&](Stream& o, const i32x4_t& r, int step) {
        if (step == 0) o.s = o.t + rot;
        else if (step == 1) o.s += b.s0 - (o.s >= b.nk ? b.nk : 0);
        else if (step == 2) o.soff = o.t < b.nk ? (uint32_t)o.s * SL : 0u;
        else if (step == 3) o.rs.z = o.t < b.nk ? r.z : 0;
        else ++o.t;
        if (step == 2) asm volatile("" : "+s"(o.soff));
        if (step == 3) asm volatile("" : "+s"(o.rs));
    };
    // (m0 and the load are two statements: see the listing's test)
    auto target = [&](uint32_t to, auto n) { asm volatile("s_add_u32 m0, %0, %1" ::"s"(to), "n"(decltype(n)::value * 1024) : "scc"); };
    auto fetch = [&](const Stream& o, uint32_t off) { asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(off), "s"(o.rs), "s"(o.soff)); };
    auto load = [&](auto n, const Stream& o, uint32_t off) {
        target(o.to, n);
        asm volatile("s_nop 0");
        fetch(o, off);
    };
    auto at = [&](Stream& o, const i32x4_t& r, int t, uint32_t to) {
        o.t = t;
        o.to = to;
#pragma unroll
        for (int step = 0; step < 5; ++step) find(o, r, step);
    };
    // In period p (the half of slice p behind the barrier, and the first half of slice p+1) the loads of W(p+SB) and then
    // of x(p+SA) are issued; the prologue issues those of periods -SB .. -2 and the first half of period -1.
    Stream oa, ob;
    oa.rs = ra;
    ob.rs = rb;
    asm volatile("s_nop 4");   // (scalars that vector instructions have written are read by the loads below, which the compiler cannot see)
    if constexpr (SA > SB) {
        at(oa, ra, 0, lds_a);
        for_constants<NA>([&](auto i) { load(i, oa, off_a[decltype(i)::value]); });
    }
    for_constants<SB>([&](auto s) {
        constexpr int n = decltype(s)::value, most = n + 1 < SB ? G::kPer : G::kFirst;
        at(ob, rb, n, lds_b + n * G::UB);
        at(oa, ra, n + SA - SB, lds_a + (n + SA - SB) * G::UA);
        for_constants<NB>([&](auto i) { if constexpr (decltype(i)::value < most) load(i, ob, off_b[decltype(i)::value]); });
        for_constants<NA>([&](auto i) { if constexpr (NB + decltype(i)::value < most) load(i, oa, off_a[decltype(i)::value]); });
    });

    // The products and what follows, of NR row blocks of a wavefront
    auto products = [&](auto rows) {
        constexpr int NR = decltype(rows)::value, PER = WIDE ? 2 : 1;      // row blocks of an instruction, of x and of W
        typedef std::conditional_t<WIDE, f32x16_t, f32x4_t> acc_t;
        acc_t acc[NR / PER][NB / PER];
#pragma unroll
        for (int i = 0; i < NR / PER; ++i)
#pragma unroll
            for (int j = 0; j < NB / PER; ++j)
#pragma unroll
                for (int q = 0; q < 4 * PER * PER; ++q) acc[i][j][q] = 0.0f;
        // fragments: lane holds 16 bytes of row lane % 16 at piece 4 step + lane / 16 (e4m3: of row lane % 32 of two blocks, two pieces from 4 step + 2 (lane / 32) on)
        const int frow = lane & 15, fp = WIDE ? lane >> 5 << 1 : lane >> 4, second = WIDE ? lane >> 4 & 1 : 0;
        uint32_t frag_a[2][PER], frag_b[2][PER];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const uint32_t sw = (uint32_t)(frow * SL + (((s * 4 + fp + u) ^ (frow & 7) ^ second) * 16));
                frag_a[s][u] = (uint32_t)((wm + 2 * second) * 16 * SL) + sw;
                frag_b[s][u] = (uint32_t)(SA * G::UA + (wn * NB + second) * 16 * SL) + sw;
            }
        typedef std::conditional_t<WIDE, i32x8_t, td_u32x4> frag_t;
        frag_t fa[2][NR / PER], fb[2][NB / PER];          // (e4m3: of a pair of blocks two pieces)
        auto put = [](frag_t& f, int piece, const td_u32x4& v) {
#pragma unroll
            for (int q = 0; q < 4; ++q) f[WIDE ? piece * 4 + q : q] = v[q];
        };
        uint32_t xa[PER], xb[PER];                        // where the next half slice's fragments lie
        auto next = [&](uint32_t (&x)[PER], const uint32_t (&frag)[PER], uint32_t ring) {
#pragma unroll
            for (int u = 0; u < PER; ++u) x[u] = frag[u] + ring;
        };
        next(xa, frag_a[0], 0);
        next(xb, frag_b[0], 0);
        auto read_one = [&](int buf, int t) {             // fa[0], all of fb, the rest of fa
            if (t - NB >= NR) return;
            auto a = [&](int i) { put(fa[buf][i / PER], i % PER, *reinterpret_cast<const td_u32x4*>(lds + xa[i % PER] + i / PER * (PER * 2 * 16 * SL))); };
            auto b = [&](int j) { put(fb[buf][j / PER], j % PER, *reinterpret_cast<const td_u32x4*>(lds + xb[j % PER] + j / PER * (PER * 16 * SL))); };
            if (t == 0) a(0);
            else if (t <= NB) b(t - 1);
            else a(t - NB);
        };
        auto multiply = [](auto& c, const auto& w, const auto& x) {
            if constexpr (WIDE) asm volatile("v_mfma_f32_32x32x64_f8f6f4 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
            else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
        };
        // the product that stands in gap h of half a slice
        auto mma = [&](int half, auto gap) {
            constexpr int h = decltype(gap)::value;
            if constexpr (!WIDE) {
                if constexpr (h / NB < NR) multiply(acc[h / NB][h % NB], fb[half][h % NB], fa[half][h / NB]);
            } else if constexpr (h % 4 == 0) {
                constexpr int i = h / 4 / (NB / 2), j = h / 4 % (NB / 2);
                if constexpr (i < NR / 2) multiply(acc[i][j], fb[half][j], fa[half][i]);
            }
        };
        auto hold = [&]() {
            // The compiler does not know how long the products take: every use of the accumulators from here on comes behind the statements
            // before this, a wait among them
#pragma unroll
            for (int i = 0; i < NR / PER; ++i)
#pragma unroll
                for (int j = 0; j < NB / PER; ++j) asm volatile("" : "+a"(acc[i][j])::"memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(G::kStart) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < G::kPer; ++t) read_one(0, t);
        next(xa, frag_a[1], 0);
        next(xb, frag_b[1], 0);
        uint32_t ring_a = 0, ring_b = 0;                  // of the slice that is multiplied
        auto turn = [&](uint32_t o, uint32_t unit, uint32_t ring) { return o + unit == ring ? 0u : o + unit; };
        hold();
        asm volatile("s_nop 7" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        // (a wait that the compiler knows of: what it believes to be under way here it waits for in every turn of the loop)
        __builtin_amdgcn_s_waitcnt(kNoLds);
        __builtin_amdgcn_sched_barrier(0);
        // One slice: the MFMAs of its first half while the fragments of the second are read, the barrier behind which slice kt+1
        // has arrived and this slice's buffers are free, the MFMAs of the second half while slice kt+1's first are read.
        for (int kt = 0; kt < b.nk; ++kt) {
            for_constants<TOT>([&](auto gap) {
                constexpr int q = decltype(gap)::value, half = q / NM, h = q % NM;
                constexpr int since = (q + NM) % TOT;                                     // gaps since the barrier
                constexpr int until_b = NM - 1 - h, until_a = (G::kEvery * NB < NM ? G::kEvery * NB : NM) - 1 - h;
                if constexpr (q == NM) {
                    __builtin_amdgcn_s_waitcnt(kNoLds);
                    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(G::kWait) : "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    oa.to = lds_a + ring_a;
                    ob.to = lds_b + ring_b;
                }
                if constexpr (h % 2 == 0 && h / 2 < G::kPer) read_one(1 - half, h / 2);
                // the loads of this period: m0, the load
                constexpr int n = since / G::kEvery, in = since % G::kEvery;
                if constexpr (n < NB) {
                    if constexpr (in == 0) target(ob.to, num<n>{});
                    if constexpr (in == 1) fetch(ob, off_b[n]);
                } else if constexpr (n < G::kPer) {
                    if constexpr (in == 0) target(oa.to, num<n - NB>{});
                    if constexpr (in == 1) fetch(oa, off_a[n - NB]);
                }
                // the slices of the next period's loads: W's before the barrier, x's while W's are issued
                if constexpr (half == 0 && until_b < 10 && until_b % 2 == 0) find(ob, rb, 4 - until_b / 2);
                if constexpr (half == 1 && until_a >= 0 && until_a < 10 && until_a % 2 == 0) find(oa, ra, 4 - until_a / 2);
                // ring offsets and addresses of the next fragments, once this half's are under way
                if constexpr (half == 0 && h == G::kTurnA) next(xa, frag_a[0], turn(ring_a, G::UA, SA * G::UA));
                if constexpr (half == 0 && h == G::kTurnB) next(xb, frag_b[0], turn(ring_b, G::UB, SB * G::UB));
                if constexpr (half == 1 && h == G::kTurnA) {
                    ring_a = turn(ring_a, G::UA, SA * G::UA);
                    next(xa, frag_a[1], ring_a);
                }
                if constexpr (half == 1 && h == G::kTurnB) {
                    ring_b = turn(ring_b, G::UB, SB * G::UB);
                    next(xb, frag_b[1], ring_b);
                }
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (WIDE ? h % 4 == 0 && h / 4 / (NB / 2) < NR / 2 : h / NB < NR) mma(half, num<h>{});
                else asm volatile("s_nop 0");             // (the wait state between m0 and a load)
                __builtin_amdgcn_sched_barrier(0);
            });
        }
        // the rest of the row, alone: pieces past its end are loaded from its start (in bounds) and zeroed as they are read
        const uint32_t from = (uint32_t)whole * SL, rest = p.k - from;
        if (rest > 0 && b.range == p.splits - 1) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            oa.rs = ra;
            ob.rs = rb;
            oa.soff = ob.soff = from;
            oa.to = lds_a;
            ob.to = lds_b;
            auto back = [&](uint32_t at) { return at < rest ? 0u : at; };
            asm volatile("s_nop 4" : "+s"(oa.rs), "+s"(ob.rs));
            for_constants<NA>([&](auto i) { load(i, oa, off_a[decltype(i)::value] - back(piece_a(decltype(i)::value))); });
            for_constants<NB>([&](auto i) { load(i, ob, off_b[decltype(i)::value] - back(piece_b(decltype(i)::value))); });
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                next(xa, frag_a[s], 0);
                next(xb, frag_b[s], 0);
                auto keep = [&](auto& f) {
#pragma unroll
                    for (int q = 0; q < 4 * PER; ++q) f[q] = (uint32_t)(s * 4 + fp + q / 4) * 16u < rest ? f[q] : 0;
                    asm volatile("" : "+v"(f));
                };
#pragma unroll
                for (int t = 0; t < G::kPer; ++t) read_one(s, t);
#pragma unroll
                for (int i = 0; i < NR / PER; ++i) keep(fa[s][i]);
#pragma unroll
                for (int j = 0; j < NB / PER; ++j) keep(fb[s][j]);
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("s_nop 7" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
                for_constants<NR * NB>([&](auto h) { mma(s, h); });
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // (the products are in inline assembly: their results are waited for here)
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
        __builtin_amdgcn_s_barrier();
        hold();
        finish_linear<T, GROUPED, 4, NR, NB, 2, 2, 1, WIDE && NR % 4 ? 2 : WIDE ? 4 : G::fit(NR, NR), WIDE ? kAccWide : kAccRows>(p, b, acc, lds, tid);
    };
    // The rows of a product or group are divided evenly between its tiles, and the row blocks of a tile are dealt out to the wavefronts in turns, so
    // that a tile which is not full takes fewer MFMAs.  (Each number of row blocks with its own accumulators and epilogue: where loops share them the
    // compiler copies 256 registers from one to the other.)
    if constexpr (NA == 8) {
        if (b.rows <= 128) products(num<4>{});
        else if (b.rows <= 192) products(num<6>{});
        else products(num<8>{});
    } else {
        if (b.rows <= 16 * NA) products(num<NA / 2>{});
        else products(num<NA>{});
    }
}

}  // namespace
