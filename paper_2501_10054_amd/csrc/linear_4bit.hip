// The linear layer with 4-bit weights: y = sigma(sum_G scale_jG sum_(k in G) (q_jk - zero_jG) x_k + b_j) + r.
//
// A code q becomes a bf16 value without a conversion: put under the exponent of 16, with the weight 1 three bits up in the mantissa, it is 16 + q, and
// a word's layout is such that a shift and an and-or make two neighbouring columns at once.  16 + zero is multiplied with the same tokens and taken away
// again (few tokens: by matrix instructions; many: as a product with the sum of the group's columns), so that a group's accumulator ends with
// sum (q - zero) x, every product exact; the group's scale goes to that sum.  Tokens in fp32 are three bf16 parts each, which together hold all of their 24 bits.
// What is raised by 16 is 5 to 10 times what is left of it, and so is its rounding.  Hence every 32 columns' zero points follow their codes into one accumulator, and
// each part has its own: the head's sums have few bits and round little, the others are 2^8 and 2^16 times smaller (fp32 tokens, groups of 128, up to 16 tokens: error of
// the outputs 1.3e-7 of their root mean square, median of 3890 calls; with one sum of codes and one of zero points 2.2e-6.  More tokens 3.0e-7; with one sum for all parts 6.6e-7).
//
// What bounds it: one token - launch, the way of the first bytes, and 0.5 bytes a weight from HBM (16384 -> 4096: 13.7 us, 34.7 MB, and from caches 11.7; the stream alone takes 7 and 5); a
// prompt - vector instructions beside the matrix cores, of which a group's product needs 8 for each 64 bytes of codes and one for each result
// (2048 tokens 4096 -> 16384: 314 us, 0.88 PFLOP/s; 512 tokens 91 us).
#include <algorithm>

#include "linear_tile.h"

namespace {

template <int N> struct words_of { typedef uint32_t type __attribute__((ext_vector_type(N))); };
template <> struct words_of<1> { typedef uint32_t type; };

struct FourArgs {
    const unsigned char* x;
    const uint32_t* W;
    const void *scales, *b, *r;
    const uint8_t* zeros;
    void* y;
    int64_t n, N, x_pitch;         // (bytes)
    uint32_t k, groups, chunk;     // columns; groups of a row; steps whose columns of all tokens are in LDS together
    int act, out_f32;
};

constexpr int kWaves = 8;

__device__ __forceinline__ f32x4_t mma(const td_u32x4& w, const td_u32x4& x, const f32x4_t& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, x), c, 0, 0, 0);
}

// 16 + q of the eight codes of a word, in bf16.  (Both constants in registers: an instruction has room for one, and takes two steps with literals)
struct Sixteen {
    uint32_t mask = 0x00780078u, exponent = 0x41804180u;
    __device__ __forceinline__ Sixteen() { asm("" : "+v"(mask), "+v"(exponent)); }
    __device__ __forceinline__ td_u32x4 more(uint32_t w) const {
        return {(w << 3 & mask) | exponent, (w >> 1 & mask) | exponent, (w >> 5 & mask) | exponent, (w >> 9 & mask) | exponent};
    }
};
// Vector instructions have written the descriptor's registers, and the loads that read them are inline assembly, which the compiler takes for ready: 5 wait states
__device__ __forceinline__ i32x4_t settled(i32x4_t r) {
    asm volatile("s_nop 4" : "+s"(r));
    return r;
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

constexpr int kStep = 128;                          // columns of a step: 64 bytes of a row's codes

// ---------------------------------------------------------------- up to 16 tokens
// A block has 16 RT rows of W and all tokens, which it puts into LDS, with the table of scales and zero points, as many columns at a time as there is room for.
// Its wavefronts are RT times KW: one has 16 rows and a KW-th of the steps, whose codes come straight to a ring of its own in LDS, D - 2 steps ahead of the two
// that are multiplied, without barriers.  The loop is a step long and not unrolled: a block runs through its code once, and what it has to fetch of it counts
// (1 token, 1024 -> 1024: 7.9 us with three batches of four groups in registers, all unrolled; 5.2).
// Lane l multiplies, of W's row l % 16, the columns 8 GW (l / 16) .. of a group, and the same columns of token l % 16.
template <typename T, int RT> struct FourBlock {
    static constexpr int KW = kWaves / RT, PARTS = Token<T>::PARTS, ENTRY = PARTS == 1 ? 4 : 8, D = 8, kRing = kWaves * D * 1024;
    static constexpr int64_t token_pitch(int64_t steps) { return steps * (2 * kStep) + 16; }             // (16 bytes more: other banks)
    static constexpr int64_t lds(int64_t n, int64_t steps, int64_t groups) { return kRing + n * PARTS * token_pitch(steps) + steps * groups * (16 * RT) * ENTRY; }
};
template <typename T, int GW, int RT>
__global__ void __launch_bounds__(64 * kWaves, 4) linear4_kernel(FourArgs p) {
    typedef typename words_of<GW>::type words_t;
    typedef FourBlock<T, RT> S;
    constexpr int D = S::D, KW = S::KW, G = 4 / GW, PARTS = S::PARTS, THREADS = 64 * kWaves;
    constexpr int SUMS = PARTS > 1 ? PARTS : GW > 1 ? 2 : 1;                            // (independent ones, for the matrix cores)
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), low = lane & 15, high = lane >> 4, kw = wave % KW, rt = wave / KW, n = (int)p.n;
    const int64_t block0 = (int64_t)blockIdx.x * (16 * RT), n0 = block0 + rt * 16;
    const uint32_t pitch = p.chunk * (2 * kStep) + 16, part_pitch = pitch * (uint32_t)n;
    unsigned char *tokens = lds + S::kRing, *table = tokens + PARTS * part_pitch;      // table: [group][row of the block]

    // codes: a load is 16 rows of 64 bytes, as they lie.  (What lies behind a row or the last one has tokens of 0 or is kept nowhere)
    const uint32_t row_bytes = p.groups * (16u * GW), base = (uint32_t)uniform((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds);
    const int rows = (int)max((int64_t)0, min((int64_t)16, p.N - n0));
    const i32x4_t rw = settled(buffer_of(reinterpret_cast<const unsigned char*>(p.W) + min(n0, p.N - 1) * row_bytes, (uint32_t)rows * row_bytes));
    const uint32_t off = (uint32_t)(lane >> 2) * row_bytes + (uint32_t)(lane & 3) * 16u, ring = base + (uint32_t)wave * (D * 1024);
    const uint32_t steps = (p.k + kStep - 1) / kStep, share = ((p.chunk + KW - 1) / KW + 1) & ~1u;   // (of a chunk's steps, for a wavefront: even)
    uint32_t ask_chunk = 0, ask = 0, ask_slot = 0;                                            // the step that is asked for next
    auto load_step = [&]() {                       // (past the last one: an empty buffer)
        const uint32_t in = (uint32_t)kw * share + ask, step = ask_chunk + in;
        i32x4_t r = rw;
        r.z = in < p.chunk && step < steps ? r.z : 0;
        const uint32_t soff = r.z ? step * (kStep / 2) : 0u;
        load_to_lds<true>(ring + ask_slot * 1024u, off, r, soff);
        ask_slot = ask_slot + 1 == D ? 0 : ask_slot + 1;
        if (++ask == share) {
            ask = 0;
            ask_chunk += p.chunk;
        }
    };
#pragma unroll 1
    for (int i = 0; i < D - 2; ++i) load_step();

    // what a thread finishes: four neighbouring rows of a token.  (Bias and residual are asked for before the products)
    const int tile = tid >> 6, token = lane >> 2, four = lane & 3;
    const int64_t first_n = block0 + tile * 16 + 4 * four, at_y = (int64_t)token * p.N + first_n;
    const int columns = tid < RT * 64 && token < n ? (int)max((int64_t)0, min((int64_t)4, p.N - first_n)) : 0;
    auto element = [&](const void* from, int64_t i) { return p.out_f32 ? static_cast<const float*>(from)[i] : td_load<bf16_t>(static_cast<const bf16_t*>(from) + i); };
    float bias[4] = {}, r[4] = {};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q >= columns) continue;
        if (p.b) bias[q] = element(p.b, first_n + q);
        if (p.r) r[q] = element(p.r, at_y + q);
    }

    const Sixteen sixteen;
    f32x4_t acc = {0, 0, 0, 0};                     // tokens 4 high + q, row low
    uint32_t slot = 0;
#pragma unroll 1
    for (uint32_t chunk = 0; chunk < steps; chunk += p.chunk) {
        const uint32_t here = min(p.chunk, steps - chunk), units = here * (kStep / 8), entries = here * G, all_units = units * (uint32_t)n, all_entries = entries * (16 * RT);
        if (chunk > 0) __syncthreads();
        // (so many pieces of tokens and entries of the table of a thread side by side: one after the other they would wait for memory each)
        constexpr int X = PARTS == 1 ? 4 : 2, E = 4;
        uint32_t u0 = 0, e0 = 0;
#pragma unroll 1
        do {
            Token<T> v[X];
            uint32_t x_to[X], group[E], e_row[E], zero[E];
            float scale[E];
#pragma unroll
            for (int i = 0; i < X; ++i) {
                uint32_t unit;
                const uint32_t u = min(u0 + i * THREADS + tid, all_units - 1), t = divide(u, units, unit), column = chunk * kStep + unit * 8;
                const unsigned char* at = p.x + t * p.x_pitch + (size_t)column * sizeof(T);
                x_to[i] = t * pitch + unit * 16;
                if (column + 8 <= p.k) load_token<T>(v[i], at);
                else load_token_end<T>(v[i], at, (int)p.k - (int)column);
            }
#pragma unroll
            for (int i = 0; i < E; ++i) {
                e_row[i] = divide(min(e0 + i * THREADS + tid, all_entries - 1), entries, group[i]);
                const int64_t at = min(block0 + e_row[i], p.N - 1) * (int64_t)p.groups + min(chunk * G + group[i], p.groups - 1);
                scale[i] = td_load<T>(static_cast<const T*>(p.scales) + at);
                zero[i] = p.zeros ? p.zeros[at] : 8u;
            }
#pragma unroll
            for (int i = 0; i < X; ++i)
#pragma unroll
                for (int part = 0; part < PARTS; ++part) *reinterpret_cast<td_u32x4*>(tokens + part * part_pitch + x_to[i]) = v[i].part[part];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float less = -16.0f - (float)min(zero[i], 128u);
                unsigned char* to = table + (group[i] * (16 * RT) + e_row[i]) * S::ENTRY;
                if (chunk * G + group[i] >= p.groups) scale[i] = 0.0f;
                if constexpr (PARTS == 1) *reinterpret_cast<uint32_t*>(to) = __float_as_uint(scale[i]) | __float_as_uint(less) >> 16;
                else *reinterpret_cast<f32x2_t*>(to) = f32x2_t{scale[i], less};
            }
            u0 += X * THREADS;
            e0 += E * THREADS;
        } while (u0 < all_units || e0 < all_entries);
        __syncthreads();
        // two steps at a time: a step's instructions wait for one another
#pragma unroll 1
        for (uint32_t in = 0; in < share; in += 2) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(D - 4) : "memory");
            words_t words[2][G];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned char* codes_at = lds + wave * (D * 1024) + (slot + h) * 1024 + low * (kStep / 2) + high * (4 * GW);
#pragma unroll
                for (int g = 0; g < G; ++g) words[h][g] = *reinterpret_cast<const words_t*>(codes_at + g * (16 * GW));
            }
            load_step();                           // (into the slots that were read in the turn before)
            load_step();
            slot = slot + 2 == D ? 0 : slot + 2;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t step = (uint32_t)kw * share + in + h;
                if (step >= here) continue;        // (a place in the ring all the same)
                const unsigned char* x_at = tokens + min(low, n - 1) * pitch + step * (2 * kStep) + high * (16 * GW);
                const unsigned char* entry_at = table + (step * G * (16 * RT) + rt * 16 + low) * S::ENTRY;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    float scale;
                    uint32_t less;
                    if constexpr (PARTS == 1) {
                        const uint32_t e = *reinterpret_cast<const uint32_t*>(entry_at + g * (16 * RT) * S::ENTRY);
                        scale = __uint_as_float(e & 0xffff0000u);
                        less = __builtin_amdgcn_perm(e, e, 0x01000100u);
                    } else {
                        const f32x2_t e = *reinterpret_cast<const f32x2_t*>(entry_at + g * (16 * RT) * S::ENTRY);
                        scale = e[0];
                        less = __builtin_amdgcn_perm(__float_as_uint(e[1]), __float_as_uint(e[1]), 0x03020302u);
                    }
                    f32x4_t c[SUMS];
#pragma unroll
                    for (int i = 0; i < SUMS; ++i) c[i] = f32x4_t{0, 0, 0, 0};
#pragma unroll
                    for (int s = 0; s < GW; ++s) {
                        uint32_t word;
                        if constexpr (GW == 1) word = words[h][g];
                        else word = words[h][g][s];
                        const td_u32x4 codes = sixteen.more(word);
#pragma unroll
                        for (int part = 0; part < PARTS; ++part) {
                            const td_u32x4 x = *reinterpret_cast<const td_u32x4*>(x_at + part * part_pitch + (g * (4 * GW) + s) * 16);
                            f32x4_t& sum = c[PARTS == 1 ? s % SUMS : part];
                            sum = mma(x, codes, sum);
                            sum = mma(x, td_u32x4{less, less, less, less}, sum);
                        }
                    }
#pragma unroll
                    for (int i = SUMS - 1; i > 0; --i) c[i - 1] += c[i];
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[q] = fmaf(scale, c[0][q], acc[q]);
                }
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    // the wavefronts' sums of a row tile, in their order: [row tile][part][token][row]
    float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[((wave * 16) + 4 * high + q) * 16 + low] = acc[q];
    __syncthreads();
    if (columns == 0) return;
    f32x4_t v = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < KW; ++w) v += *reinterpret_cast<const f32x4_t*>(sums + ((tile * KW + w) * 16 + token) * 16 + 4 * four);
    with_linear_act(p.act, [&](auto act) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = linear_act<decltype(act)::value>(v[q] + bias[q]) + r[q];
    });
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q >= columns) continue;
        if (p.out_f32) static_cast<float*>(p.y)[at_y + q] = v[q];
        else td_store<bf16_t>(static_cast<bf16_t*>(p.y) + at_y + q, v[q]);
    }
}

// ---------------------------------------------------------------- many tokens
// What the tiles read beside the codes, made by one launch before theirs:
//   tokens  PARTS parts in bf16, [part][token][units], zeros behind the last column
//   sums    of every group's columns, [part][group][sum_pitch]
//   table   of W's scales and zero points, [group][table_pitch] rows: scale and -(16 + zero), in bf16 side by side (of tokens in bf16) or in fp32
// Groups are as many as whole steps have, those behind the last with scales of 0.
struct FourTokens {
    const unsigned char* x;
    const void* scales;
    const uint8_t* zeros;
    td_u32x4* parts;
    float* sums;
    unsigned char* table;
    int64_t n, N, x_pitch, sum_pitch, table_pitch;
    uint32_t k, units, groups, all_groups, token_blocks;   // columns; pieces of 8 of a row in whole steps
};
template <typename T, int GW>
__global__ void __launch_bounds__(256) linear4_prepare_kernel(FourTokens p) {
    if (blockIdx.x >= p.token_blocks) {            // a thread has 8 groups of a row
        const uint32_t i = (blockIdx.x - p.token_blocks) * 256u + threadIdx.x, first = i / (uint32_t)p.table_pitch * 8, row = i % (uint32_t)p.table_pitch;
        if (first >= p.all_groups) return;
        const int64_t at = (int64_t)row * p.groups + first;
        T scale[8];
        uint8_t zero[8];
        if (row < p.N && first + 8 <= p.groups) {
            typedef T scales_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
            typedef uint8_t zeros_t __attribute__((ext_vector_type(8), aligned(1)));
            const scales_t s = *reinterpret_cast<const scales_t*>(static_cast<const T*>(p.scales) + at);
            zeros_t z = {8, 8, 8, 8, 8, 8, 8, 8};
            if (p.zeros) z = *reinterpret_cast<const zeros_t*>(p.zeros + at);
#pragma unroll
            for (int q = 0; q < 8; ++q) scale[q] = s[q], zero[q] = z[q];
        } else {
#pragma unroll
            for (uint32_t q = 0; q < 8; ++q) {
                const bool in = row < p.N && first + q < p.groups;
                scale[q] = in ? static_cast<const T*>(p.scales)[at + q] : (T)0;
                zero[q] = in && p.zeros ? p.zeros[at + q] : (uint8_t)8;
            }
        }
#pragma unroll
        for (uint32_t q = 0; q < 8; ++q) {
            if (first + q >= p.all_groups) continue;
            const int64_t to = (int64_t)(first + q) * p.table_pitch + row;
            const float less = -16.0f - (float)min((uint32_t)zero[q], 128u);
            if constexpr (sizeof(T) == 2) reinterpret_cast<uint32_t*>(p.table)[to] = (uint32_t)scale[q] << 16 | __float_as_uint(less) >> 16;
            else reinterpret_cast<f32x2_t*>(p.table)[to] = f32x2_t{scale[q], less};
        }
        return;
    }
    const uint32_t u = blockIdx.x * 256u + threadIdx.x;
    const int64_t row = u / p.units;
    const uint32_t unit = u % p.units;
    if (row >= p.n) return;                        // (rows are whole groups: no group is divided)
    const unsigned char* at = p.x + row * p.x_pitch + (size_t)unit * 8 * sizeof(T);
    const int left = (int)p.k - (int)unit * 8;
    Token<T> t;
    if (left >= 8) load_token<T>(t, at);
    else load_token_end<T>(t, at, left);
#pragma unroll
    for (int i = 0; i < Token<T>::PARTS; ++i) {
        double sum = 0.0;
#pragma unroll
        for (int q = 0; q < 4; ++q) sum += (double)__uint_as_float(t.part[i][q] << 16) + (double)__uint_as_float(t.part[i][q] & 0xffff0000u);
#pragma unroll
        for (int o = 1; o < 4 * GW; o *= 2) sum += __shfl_xor(sum, o, 64);
        if (unit % (4 * GW) == 0) p.sums[((int64_t)i * p.all_groups + unit / (4 * GW)) * p.sum_pitch + row] = (float)sum;
    }
#pragma unroll
    for (int i = 0; i < Token<T>::PARTS; ++i) p.parts[((int64_t)i * p.n + row) * p.units + unit] = t.part[i];
}

struct FourTile : LinearArgs {                     // (x: the parts; k: bytes of a row of theirs)
    const float* sums;
    const unsigned char* table;
    int64_t sum_pitch, table_pitch;
    uint32_t groups, all_groups;
};

// D steps in LDS.  The table's and (tokens of one part) the sums' pieces of 1024 bytes are dealt out to the wavefronts, AUX for each; parts have their sums with
// their tokens.
template <int PARTS, int GW, int FA, int FB, int WN, int D> struct FourTileShape {
    static constexpr int TM = 16 * FA, TN = 16 * FB * WN, G = 4 / GW;
    static constexpr int X = TM * 2 * kStep, CODES = TN * kStep / 2, ROW = PARTS == 1 ? 4 : 8, PIECE = TN * ROW < 1024 ? TN * ROW : 1024;   // (of a group's rows in one load)
    static constexpr int TABLE = (G * TN * ROW + 1023) / 1024 * 1024, SUMS = 1024, LX = X / (1024 * WN), LC = CODES / (1024 * WN), LT = TABLE / 1024;
    static constexpr int AUX = (LT + 1 + WN - 1) / WN, LOADS = LX + LC + AUX;
    static constexpr int kLds = D * (X + CODES + TABLE + SUMS), kRowBytes = WN * 16 * FB * 16 * 4;
    static constexpr int RB = FA * kRowBytes <= kLds ? FA : FA % 2 == 0 && 2 * kRowBytes <= kLds ? 2 : 1;   // row blocks behind the products
    static_assert(X % (1024 * WN) == 0 && CODES % (1024 * WN) == 0 && RB * kRowBytes <= kLds && G * TM * 4 <= SUMS && kLds <= kLdsBytes, "slots");
    static_assert(D >= 2 && (D - 2) * LOADS <= 63 && (PARTS == 1 || D == 2), "steps under way");
};

// A tile of TM = 16 FA tokens x TN = 16 FB WN rows of W.  A step of 128 columns - tokens, codes, table, sums - goes to LDS, D - 1 steps ahead, and two blocks
// are on a CU: while one waits for its step the other multiplies.  A wavefront has 16 FB rows to itself, makes the codes of 16 of them into bf16
// and multiplies them with all tokens, group by group: a group's sum begins with -(16 + zero) times the sum of the token's columns, and is
// added to the result with the group's scale.
template <int PARTS, int GW, int FA, int FB, int WN, int D>
__global__ void __launch_bounds__(64 * WN, 2) linear4_tile_kernel(FourTile p) {
    typedef typename words_of<GW>::type words_t;
    typedef FourTileShape<PARTS, GW, FA, FB, WN, D> S;
    constexpr int TM = S::TM, TN = S::TN, G = S::G, LX = S::LX, LC = S::LC, LT = S::LT;
    extern __shared__ __align__(1024) unsigned char lds[];
    unsigned char *at_x = lds, *at_codes = at_x + D * S::X, *at_table = at_codes + D * S::CODES, *at_sums = at_table + D * S::TABLE;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), low = lane & 15, high = lane >> 4;
    uint32_t t, in_range;
    if (!number_of(blockIdx.x, (uint32_t)(p.tiles_m * p.tiles_n * p.splits), t)) return;
    LinearBlock b;
    int tile_m, tile_n;
    const int steps = (int)(p.k / (2 * kStep));
    b.range = uniform((int)divide(t, (uint32_t)(p.tiles_m * p.tiles_n), in_range));
    tile_of(in_range, (uint32_t)p.tiles_m, (uint32_t)p.tiles_n, tile_m, tile_n);
    b.expert = 0;
    b.first = (int64_t)tile_m * TM;
    b.rows = (int)min((int64_t)TM, p.n - b.first);
    b.s0 = b.range * p.slices;
    b.nk = max(0, min(p.slices, steps - b.s0));
    b.n0 = (int64_t)tile_n * TN;
    const int rows_w = (int)min((int64_t)TN, p.N - b.n0);
    const int rot = first_slice((int)blockIdx.x & 7, (int)blockIdx.x >> 3, b.nk);
    auto step_of = [&](int at) { return (uint32_t)(b.s0 + (at + rot >= b.nk ? at + rot - b.nk : at + rot)); };

    // tokens: a load is 4 rows of 256 bytes, lane -> row lane / 16, slot lane % 16, which holds piece slot ^ row; codes: 16 rows of 64 bytes, as they lie; table: 1024
    // bytes of a group's rows; sums: 4 groups of 64 tokens
    const uint32_t base = (uint32_t)uniform((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds);
    const uint32_t row_bytes = p.groups * (16u * GW);
    uint32_t off_x[LX], off_codes[LC];
#pragma unroll
    for (int i = 0; i < LX; ++i) {
        const int row = wave * (TM / WN) + 4 * i + high;
        off_x[i] = (row < b.rows ? (uint32_t)row * p.k : kNowhere) + (uint32_t)((low ^ (row & 15)) * 16);
    }
#pragma unroll
    for (int i = 0; i < LC; ++i) {
        const int row = wave * (TN / WN) + 16 * i + (lane >> 2);
        off_codes[i] = (row < rows_w ? (uint32_t)row * row_bytes : kNowhere) + (uint32_t)(lane & 3) * 16u;
    }
    const uint32_t off_sums = high < G && 4 * low < min(b.rows, TM) ? (uint32_t)(high * p.sum_pitch + 4 * low) * 4u : kNowhere;
    const i32x4_t rc = settled(buffer_of(p.W + b.n0 * row_bytes, (uint32_t)rows_w * row_bytes));
    // (live: past the last step nothing is fetched, from empty buffers)
    auto load_sums = [&](uint32_t step, int part, uint32_t slot, bool live) {
        i32x4_t r = settled(buffer_of(p.sums + ((int64_t)part * p.all_groups + (int64_t)step * G) * p.sum_pitch + b.first,
                                      (uint32_t)((G - 1) * p.sum_pitch + p.sum_pitch - b.first) * 4u));
        r.z = live ? r.z : 0;
        load_to_lds(base + D * (S::X + S::CODES + S::TABLE) + slot * S::SUMS, off_sums, r, 0);
    };
    auto load_x = [&](uint32_t step, int part, uint32_t slot, bool live) {
        i32x4_t r = settled(buffer_of(p.x + ((int64_t)part * p.n + b.first) * p.k, (uint32_t)b.rows * p.k));
        r.z = live ? r.z : 0;
#pragma unroll
        for (int i = 0; i < LX; ++i) load_to_lds(base + slot * S::X + (uint32_t)wave * (S::X / WN) + i * 1024u, off_x[i], r, live ? step * (2 * kStep) : 0u);
        if (PARTS > 1 && wave == 0) load_sums(step, part, slot, live);
    };
    auto load_codes = [&](uint32_t step, uint32_t slot, bool live) {
        i32x4_t r = rc;
        r.z = live ? r.z : 0;
#pragma unroll
        for (int i = 0; i < LC; ++i)
            load_to_lds(base + D * S::X + slot * S::CODES + (uint32_t)wave * (S::CODES / WN) + i * 1024u, off_codes[i], r, live ? step * (kStep / 2) : 0u);
#pragma unroll
        for (int i = 0; i < S::AUX; ++i) {
            const int piece = wave + i * WN;
            if (piece < LT) {
                // lane -> 16 bytes of the step's groups, one behind the other
                const uint32_t in = (uint32_t)piece * 1024u + (uint32_t)lane * 16u, group = in / (TN * S::ROW), at = in % (TN * S::ROW);
                i32x4_t rt = settled(buffer_of(p.table + ((int64_t)step * G * p.table_pitch + b.n0) * S::ROW, (uint32_t)(((G - 1) * p.table_pitch + TN) * S::ROW)));
                rt.z = live ? rt.z : 0;
                load_to_lds((uint32_t)uniform((int)(base + D * (S::X + S::CODES) + slot * S::TABLE + (uint32_t)piece * 1024u)),
                            group < (uint32_t)G ? group * (uint32_t)p.table_pitch * S::ROW + at : kNowhere, rt, 0);
            } else if (PARTS == 1)
                load_sums(step, 0, slot, live);
        }
    };
    const Sixteen sixteen;
    f32x4_t acc[FA][FB];
#pragma unroll
    for (int i = 0; i < FA; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j) acc[i][j] = f32x4_t{0, 0, 0, 0};
    auto products = [&](uint32_t x_slot, uint32_t slot) {
        const unsigned char* from = at_x + x_slot * S::X + low * (2 * kStep);
        const unsigned char* codes_from = at_codes + slot * S::CODES + (wave * FB * 16 + low) * (kStep / 2) + high * (4 * GW);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            td_u32x4 x[FA][GW];
            f32x4_t sum[FA];
#pragma unroll
            for (int i = 0; i < FA; ++i) {
#pragma unroll
                for (int s = 0; s < GW; ++s) x[i][s] = *reinterpret_cast<const td_u32x4*>(from + i * 16 * (2 * kStep) + (((g * (4 * GW) + high * GW + s) ^ low) * 16));
                sum[i] = *reinterpret_cast<const f32x4_t*>(at_sums + x_slot * S::SUMS + (g * 64 + i * 16 + 4 * high) * 4);
            }
#pragma unroll
            for (int j = 0; j < FB; ++j) {
                const words_t words = *reinterpret_cast<const words_t*>(codes_from + j * 16 * (kStep / 2) + g * (16 * GW));
                const unsigned char* entry = at_table + slot * S::TABLE + (g * TN + (wave * FB + j) * 16 + low) * S::ROW;
                float scale, less;
                if constexpr (S::ROW == 4) {
                    const uint32_t e = *reinterpret_cast<const uint32_t*>(entry);
                    scale = __uint_as_float(e & 0xffff0000u);
                    less = __uint_as_float(e << 16);
                } else {
                    const f32x2_t e = *reinterpret_cast<const f32x2_t*>(entry);
                    scale = e[0];
                    less = e[1];
                }
                f32x4_t c[FA];
#pragma unroll
                for (int i = 0; i < FA; ++i) c[i] = sum[i] * less;
#pragma unroll
                for (int s = 0; s < GW; ++s) {
                    uint32_t word;
                    if constexpr (GW == 1) word = words;
                    else word = words[s];
                    const td_u32x4 codes = sixteen.more(word);
#pragma unroll
                    for (int i = 0; i < FA; ++i) c[i] = mma(x[i][s], codes, c[i]);
                }
#pragma unroll
                for (int i = 0; i < FA; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i][j][q] = fmaf(scale, c[i][q], acc[i][j][q]);
            }
        }
    };
    auto arrived = [&]() {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((D - 2) * S::LOADS) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if constexpr (PARTS == 1) {
        auto load_step = [&](int at, uint32_t slot) {
            const bool live = at < b.nk;
            const uint32_t step = live ? step_of(at) : 0u;
            load_x(step, 0, slot, live);
            load_codes(step, slot, live);
        };
#pragma unroll 1
        for (int at = 0; at < D - 1; ++at) load_step(at, (uint32_t)at);
        uint32_t slot = 0, free_slot = D - 1;
#pragma unroll 1
        for (int at = 0; at < b.nk; ++at) {
            arrived();
            load_step(at + D - 1, free_slot);
            products(slot, slot);
            free_slot = slot;
            slot = slot + 1 == D ? 0 : slot + 1;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
        if (b.nk > 0) {
            load_x(step_of(0), 0, 0, true);
            load_codes(step_of(0), 0, true);
        }
        uint32_t x_slot = 0;
#pragma unroll 1
        for (int at = 0; at < b.nk; ++at) {
            const uint32_t slot = (uint32_t)at & 1;
#pragma unroll 1
            for (int part = 0; part < PARTS; ++part) {
                arrived();
                if (part + 1 < PARTS) load_x(step_of(at), part + 1, x_slot ^ 1, true);
                else if (at + 1 < b.nk) load_x(step_of(at + 1), 0, x_slot ^ 1, true);
                if (part == 0 && at + 1 < b.nk) load_codes(step_of(at + 1), slot ^ 1, true);
                products(x_slot, slot);
                x_slot ^= 1;
            }
        }
    }
    __syncthreads();
    finish_linear<four_t, false, WN, FA, FB, 1, WN, 1, S::RB, kAccAcross>(p, b, acc, lds, tid);
}

template <typename T, int GW, int RT> void launch(const FourArgs& p, unsigned blocks, size_t lds, hipStream_t s) {
    hipLaunchKernelGGL((linear4_kernel<T, GW, RT>), dim3(blocks), dim3(64 * kWaves), lds, s, p);
}
// f(element type, group words, row tiles of a block)
template <typename F> void for_four(bool f32, int group, int rows, F f) {
    auto with_rows = [&](auto type, auto gw) {
        if (rows == 1) f(type, gw, num<1>{});
        else if (rows == 2) f(type, gw, num<2>{});
        else f(type, gw, num<4>{});
    };
    auto with_group = [&](auto type) {
        if (group == 32) with_rows(type, num<1>{});
        else if (group == 64) with_rows(type, num<2>{});
        else with_rows(type, num<4>{});
    };
    if (f32) with_group(float{});
    else with_group(bf16_t{});
}

// The tiles: tokens, rows of W, steps in LDS (for tokens in fp32 two)
struct FourShape { int m, n, steps; };
constexpr FourShape kFourShape[] = {{16, 64, 6}, {32, 64, 5}, {64, 64, 3}, {64, 256, 2}};
constexpr int kFourShapes = sizeof(kFourShape) / sizeof(FourShape);
// f(parts of a token, group words, token blocks, row blocks of a wavefront, wavefronts, steps in LDS)
template <typename F> void for_four_tile(bool f32, int group, int shape, F f) {
    auto with_shape = [&](auto parts, auto gw) {
        constexpr bool deep = decltype(parts)::value == 1;
        switch (shape) {
            case 0: f(parts, gw, num<1>{}, num<1>{}, num<4>{}, num<deep ? 6 : 2>{}); break;
            case 1: f(parts, gw, num<2>{}, num<1>{}, num<4>{}, num<deep ? 5 : 2>{}); break;
            case 2: f(parts, gw, num<4>{}, num<1>{}, num<4>{}, num<deep ? 3 : 2>{}); break;
            default: f(parts, gw, num<4>{}, num<4>{}, num<4>{}, num<2>{}); break;
        }
    };
    auto with_parts = [&](auto gw) {
        if (f32) with_shape(num<3>{}, gw);
        else with_shape(num<1>{}, gw);
    };
    if (group == 32) with_parts(num<1>{});
    else if (group == 64) with_parts(num<2>{});
    else with_parts(num<4>{});
}

tardis_status_t init_four() {
    static td_once once;
    return once.run([]() -> tardis_status_t {
        bool ok = true;
        for (int group = 32; group <= 128; group *= 2)
            for (int f32 = 0; f32 < 2; ++f32) {
                for (int rows = 1; rows <= 4; rows *= 2)
                    for_four(f32, group, rows, [&](auto type, auto gw, auto rt) {
                        ok &= hipFuncSetAttribute(reinterpret_cast<const void*>(linear4_kernel<decltype(type), gw, rt>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                  kLdsBytes) == hipSuccess;
                    });
                for (int shape = 0; shape < kFourShapes; ++shape)
                    for_four_tile(f32, group, shape, [&](auto parts, auto gw, auto fa, auto fb, auto wn, auto d) {
                        typedef FourTileShape<parts, gw, fa, fb, wn, d> S;
                        ok &= S::TM == kFourShape[shape].m && S::TN == kFourShape[shape].n;
                        ok &= hipFuncSetAttribute(reinterpret_cast<const void*>(linear4_tile_kernel<parts, gw, fa, fb, wn, d>),
                                                  hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds) == hipSuccess;
                    });
            }
        return ok ? TARDIS_OK : TARDIS_ERR_HIP;
    });
}

// How a call is done, by its sizes and the working memory that it has
struct FourPlan {
    bool tiles;
    int shape, splits, slices;
    int64_t units, all_groups, sum_pitch, table_pitch, at_sums, at_table, at_part, work;
};
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

FourPlan plan_four(const tardis_linear_4bit_desc* d, int64_t n, int64_t room) {
    FourPlan p{};
    const bool f32 = d->dtype == TARDIS_F32;
    // up to 16 tokens: every block of linear4_kernel has them whole, so not where that is long (16 tokens 16384 -> 4096: 512 KB, 29 us; as tiles in 8 ranges 25)
    if (n <= 16 && n * d->n_in * (f32 ? 6 : 2) <= 300 * 1024) return p;
    const int64_t steps = (d->n_in + kStep - 1) / kStep;
    p.units = steps * (kStep / 8);
    p.all_groups = steps * (kStep / d->group);
    p.sum_pitch = round_up(n, 4);
    p.table_pitch = round_up(d->n_out, 256);
    p.at_sums = round_up((f32 ? 3 : 1) * n * p.units * 16, 256);
    p.at_table = p.at_sums + round_up((f32 ? 3 : 1) * p.all_groups * p.sum_pitch * 4, 256);
    p.at_part = p.at_table + p.all_groups * p.table_pitch * (f32 ? 8 : 4);
    // (offsets of a tile's rows, of four groups' sums and of the table are 32 bits)
    if (p.units * 16 * 64 >= kNowhere || 4 * p.sum_pitch * 4 >= kNowhere || n * p.units + p.all_groups * p.table_pitch >= kMostThreads || p.at_part > room) return FourPlan{};
    auto tiles_of = [&](const FourShape& t) { return ((n + t.m - 1) / t.m) * ((d->n_out + t.n - 1) / t.n); };
    // (100 tokens 4096 -> 16384, us: 64 x 64 in one range 37, 64 x 256 in two 42; 300 tokens 84 and 77; 1000 tokens 4096 -> 4096 72 and 61)
    p.shape = n <= 16 ? 0 : n <= 32 ? 1 : n <= 64 || tiles_of(kFourShape[3]) < 256 ? 2 : 3;
    const int64_t tiles = tiles_of(kFourShape[p.shape]);
    if (tiles >= 1 << 21) return FourPlan{};
    // (256 CUs; a range is 8 steps at least, and where it has many a second block on each CU is worth the longer join)
    p.splits = 1;
    while (p.splits < 16 && (tiles * p.splits <= 128 || (tiles * p.splits <= 256 && steps >= 32 * p.splits)) && steps >= 16 * p.splits &&
           p.at_part + 2 * p.splits * n * d->n_out * 4 <= room)
        p.splits *= 2;
    p.slices = (int)((steps + p.splits - 1) / p.splits);
    p.work = p.at_part + (p.splits > 1 ? p.splits * n * d->n_out * 4 : 0);
    p.tiles = true;
    return p;
}

tardis_status_t run_tiles(const tardis_linear_4bit_desc* d, const FourPlan& plan, const void* x, int64_t n, int64_t x_pitch, const void* residual, void* y,
                          unsigned char* work, hipStream_t s) {
    TD_TRY(init_four());
    const bool f32 = d->dtype == TARDIS_F32;
    FourTokens t{};
    t.x = static_cast<const unsigned char*>(x);
    t.scales = d->scales;
    t.zeros = d->zeros;
    t.parts = reinterpret_cast<td_u32x4*>(work);
    t.sums = reinterpret_cast<float*>(work + plan.at_sums);
    t.table = work + plan.at_table;
    t.n = n;
    t.N = d->n_out;
    t.x_pitch = x_pitch * (int64_t)td_elem_size(d->dtype);
    t.sum_pitch = plan.sum_pitch;
    t.table_pitch = plan.table_pitch;
    t.k = (uint32_t)d->n_in;
    t.units = (uint32_t)plan.units;
    t.groups = (uint32_t)((d->n_in + d->group - 1) / d->group);
    t.all_groups = (uint32_t)plan.all_groups;
    t.token_blocks = (uint32_t)((n * plan.units + 255) / 256);
    FourTile p{};
    p.x = work;
    p.W = reinterpret_cast<const unsigned char*>(d->W);
    p.b = d->b;
    p.r = residual;
    p.y = y;
    p.n = p.x_rows = n;
    p.N = d->n_out;
    p.k = (uint32_t)(plan.units * 16);
    p.act = d->act == TARDIS_ACT_GELU_ERF && d->out_dtype == TARDIS_BF16 && !residual ? kActGelu16 : d->act;
    p.out_f32 = d->out_dtype == TARDIS_F32;
    const FourShape& shape = kFourShape[plan.shape];
    p.tiles_m = (int)((n + shape.m - 1) / shape.m);
    p.tiles_n = (int)((d->n_out + shape.n - 1) / shape.n);
    p.splits = plan.splits;
    p.slices = plan.slices;
    p.sums = t.sums;
    p.table = t.table;
    p.sum_pitch = plan.sum_pitch;
    p.table_pitch = plan.table_pitch;
    p.groups = t.groups;
    p.all_groups = t.all_groups;
    FourTile q = p;
    if (plan.splits > 1) {
        q.part = reinterpret_cast<float*>(work + plan.at_part);
        q.act = TARDIS_ACT_IDENTITY;
    }
    const dim3 prepare(t.token_blocks + (unsigned)(((plan.all_groups + 7) / 8 * plan.table_pitch + 255) / 256));
    const int blocks = (int)(((int64_t)p.tiles_m * p.tiles_n * p.splits + 7) / 8 * 8);
    for_four_tile(f32, d->group, plan.shape, [&](auto parts, auto gw, auto fa, auto fb, auto wn, auto deep) {
        constexpr int bytes = FourTileShape<parts, gw, fa, fb, wn, deep>::kLds, threads = 64 * wn;
        if constexpr (decltype(parts)::value == 3) hipLaunchKernelGGL((linear4_prepare_kernel<float, gw>), prepare, dim3(256), 0, s, t);
        else hipLaunchKernelGGL((linear4_prepare_kernel<bf16_t, gw>), prepare, dim3(256), 0, s, t);
        hipLaunchKernelGGL((linear4_tile_kernel<parts, gw, fa, fb, wn, deep>), dim3((unsigned)blocks), dim3(threads), bytes, s, q);
    });
    if (plan.splits > 1) {
        p.part = q.part;
        td_linear_join(p, s);
    }
    TD_HIP(hipGetLastError());
    return TARDIS_OK;
}

}  // namespace

namespace {

// Tokens that are done together: more would take more working memory and nothing less of time
int64_t tokens_at_once(const tardis_linear_4bit_desc* d) {
    const int64_t units = (d->n_in + kStep - 1) / kStep * (kStep / 8);
    return std::max<int64_t>(1, std::min<int64_t>(16384, (kMostThreads / 2) / units));
}

tardis_status_t run_few(const tardis_linear_4bit_desc* d, const void* x, int64_t n, int64_t x_pitch, const void* residual, void* y, hipStream_t s) {
    TD_TRY(init_four());
    FourArgs p{};
    const bool f32 = d->dtype == TARDIS_F32;
    const int64_t es = (int64_t)td_elem_size(d->dtype), eo = (int64_t)td_elem_size(d->out_dtype);
    p.x = static_cast<const unsigned char*>(x);
    p.W = d->W;
    p.scales = d->scales;
    p.zeros = d->zeros;
    p.b = d->b;
    p.r = residual;
    p.y = y;
    p.N = d->n_out;
    p.x_pitch = (n > 1 ? x_pitch : d->n_in) * es;
    p.k = (uint32_t)d->n_in;
    p.groups = (uint32_t)((d->n_in + d->group - 1) / d->group);
    p.act = d->act == TARDIS_ACT_GELU_ERF && d->out_dtype == TARDIS_BF16 && !residual ? kActGelu16 : d->act;
    p.out_f32 = d->out_dtype == TARDIS_F32;
    for (int64_t at = 0; at < n; at += 16) {
        FourArgs q = p;
        q.n = std::min<int64_t>(16, n - at);
        q.x += at * p.x_pitch;
        q.y = static_cast<unsigned char*>(y) + at * p.N * eo;
        if (residual) q.r = static_cast<const unsigned char*>(residual) + at * p.N * eo;
        const int64_t tiles = (p.N + 15) / 16, steps = (d->n_in + kStep - 1) / kStep, groups = kStep / d->group;
        // row tiles of a block: 256 CUs have one or two blocks each, which take about 5 us and what their codes (25 bytes a ns and CU) and tokens (50) take
        int rows = 1;
        double least = 1e300;
        for (int r = 1; r <= 4; r *= 2) {
            const int64_t blocks = (tiles + r - 1) / r, tokens = (f32 ? 3 : 1) * q.n * steps * (2 * kStep), bytes = kWaves * 8 * 1024 + tokens + steps * groups * 16 * r * (f32 ? 8 : 4);
            const int64_t on_cu = std::min<int64_t>(2 * bytes <= kLdsBytes ? 2 : 1, (blocks + 255) / 256);
            const double us = (double)((blocks + 256 * on_cu - 1) / (256 * on_cu)) * (5.0 + (double)on_cu * ((double)(r * 16 * steps * (kStep / 2)) / 25e3 + (double)tokens / 50e3));
            if (us < least) least = us, rows = r;
        }
        for_four(f32, d->group, rows, [&](auto type, auto gw, auto rt) {
            typedef FourBlock<decltype(type), rt> S;
            const int64_t room = kLdsBytes - S::lds(q.n, 0, groups), each = S::lds(q.n, 1, groups) - S::lds(q.n, 0, groups);
            const int64_t fit = room / each;               // (at least 6 steps: 16 tokens in three parts, four groups of 64 rows)
            q.chunk = (uint32_t)std::min(steps, fit >= S::KW ? fit / S::KW * S::KW : fit);
            launch<decltype(type), gw, rt>(q, (unsigned)((tiles + rows - 1) / rows), (size_t)S::lds(q.n, q.chunk, groups), s);
        });
    }
    TD_HIP(hipGetLastError());
    return TARDIS_OK;
}

}  // namespace

tardis_status_t td_linear_4bit_work_bytes(const tardis_linear_4bit_desc* d, int64_t n, int64_t* bytes) {
    *bytes = plan_four(d, std::min(n, tokens_at_once(d)), (int64_t)1 << 62).work;
    return TARDIS_OK;
}

tardis_status_t td_linear_4bit(const tardis_linear_4bit_desc* d, const void* x, int64_t n, int64_t x_pitch, const void* residual, void* y, void* work,
                               int64_t work_bytes, hipStream_t s) {
    const int64_t most = tokens_at_once(d), es = (int64_t)td_elem_size(d->dtype), eo = (int64_t)td_elem_size(d->out_dtype);
    for (int64_t at = 0; at < n; at += most) {
        const int64_t here = std::min(most, n - at);
        const FourPlan plan = plan_four(d, here, work_bytes);
        const unsigned char *from = static_cast<const unsigned char*>(x) + at * x_pitch * es, *add = static_cast<const unsigned char*>(residual);
        unsigned char* to = static_cast<unsigned char*>(y) + at * d->n_out * eo;
        if (add) add += at * d->n_out * eo;
        TD_TRY(plan.tiles ? run_tiles(d, plan, from, here, x_pitch, add, to, static_cast<unsigned char*>(work), s) : run_few(d, from, here, x_pitch, add, to, s));
    }
    return TARDIS_OK;
}
