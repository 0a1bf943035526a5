// A mixture of expert networks around its products (linear.hip): the router's choice with the order of the experts' rows, and the sum of
// the experts' outputs.
#include <algorithm>

#include "common.h"
#include "tiles.h"

namespace {

// ---------------------------------------------------------------- the router's choice
// k times the largest of a token's logits, by G lanes (16 or 64) that hold V logits each; the softmax over the chosen or over all; and the
// slots (token, place in its choice) in the order of their experts, which is a counting sort: its counts and its ranks are sums of whole numbers
// in a fixed order, so the result is the same in every run.
//
// What bounds it: round trips and, for many tokens, the vector instructions of the choice (16384 tokens, 128 experts, 8 chosen, the choice in 64 blocks
// 25.6 us, in 256 8.3, the placement 6.0).  One block does all of a call of few tokens (tokens_of_block); more take two launches, the choice with
// the counts of every block, then the placement, for which every block adds up the counts of those before it (at most kMostBlocks), which
// costs less than a launch of its own for that.
constexpr int kRouteThreads = 1024, kMostBlocks = 256, kRouteWaves = kRouteThreads / 64;

struct RouteArgs {
    const void* logits;
    int64_t n;
    int experts, k, renormalise, tokens;           // tokens of a block
    int32_t *ids, *offsets, *order, *place;
    float* weights;
    int32_t* counts;                               // [block][counts_of_row(experts)]
};

// (rows of whole pieces of 16 bytes)
__host__ __device__ __forceinline__ int counts_of_row(int experts) { return (experts + 3) & ~3; }

template <int CTRL> __device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false); }
template <int CTRL> __device__ __forceinline__ float dpp(float v) { return __int_as_float(dpp<CTRL>(__float_as_int(v))); }
// f over the G lanes of a group, the result in all of them: rotations within 16 lanes, then halves of the wavefront
template <int G, typename V, typename F> __device__ __forceinline__ V over_lanes(V v, F f) {
    v = f(v, dpp<0x128>(v));
    v = f(v, dpp<0x124>(v));
    v = f(v, dpp<0x122>(v));
    v = f(v, dpp<0x121>(v));
    if constexpr (G == 64) {
        v = f(v, __shfl_xor(v, 16, 64));
        v = f(v, __shfl_xor(v, 32, 64));
    }
    return v;
}

template <typename T, int G, int V>
__device__ __forceinline__ void choose_experts(const RouteArgs& p, int64_t first, int tokens, int32_t* counts) {
    const int lane = threadIdx.x % G;
    const auto larger = [](float a, float b) { return fmaxf(a, b); };
    const auto smaller = [](int a, int b) { return min(a, b); };
    const auto add = [](float a, float b) { return a + b; };
#pragma unroll 1
    for (int t = threadIdx.x / G; t < tokens; t += kRouteThreads / G) {
        const T* logits = static_cast<const T*>(p.logits) + (first + t) * p.experts;
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = lane + G * i;
            v[i] = e < p.experts ? td_load<T>(logits + e) : -INFINITY;
            v[i] = v[i] == v[i] ? v[i] : -INFINITY;               // (a NaN is a logit that is not there)
        }
        float most = v[0];
#pragma unroll
        for (int i = 1; i < V; ++i) most = fmaxf(most, v[i]);
        most = over_lanes<G>(most, larger);
        // (the largest is 1 also where it is infinite; where nothing is there no weight is)
        const auto weight = [&](float l) { return l == -INFINITY ? 0.0f : l == most ? 1.0f : expf(l - most); };
        float total = 0.0f;
        if (!p.renormalise) {
#pragma unroll
            for (int i = 0; i < V; ++i) total += weight(v[i]);
            total = over_lanes<G>(total, add);
        }
        int my_id = -1;                                       // lane j has the choice number j
        float my_logit = -INFINITY;
#pragma unroll 1
        for (int j = 0; j < p.k; ++j) {
            float best = v[0];
            int at = 0;
#pragma unroll
            for (int i = 1; i < V; ++i) {
                at = v[i] > best ? i : at;
                best = fmaxf(best, v[i]);
            }
            const float top = over_lanes<G>(best, larger);
            const int id = over_lanes<G>(best == top && top > -INFINITY ? lane + G * at : INT32_MAX, smaller);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = lane + G * i == id ? -INFINITY : v[i];
            my_id = lane == j && id != INT32_MAX ? id : my_id;
            my_logit = lane == j ? top : my_logit;
        }
        const float mine = weight(my_logit);
        if (p.renormalise) total = over_lanes<G>(mine, add);
        if (lane < p.k) {
            const int64_t slot = (first + t) * p.k + lane;
            p.ids[slot] = my_id;
            p.weights[slot] = my_id < 0 ? 0.0f : mine / total;
            if (my_id >= 0) atomicAdd(counts + my_id, 1);
        }
    }
}

__device__ __forceinline__ int scan_of_wave(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, 64);
        v += lane >= o ? u : 0;
    }
    return v;
}

// The slots [begin, end) of a wavefront, of the block's from slot0 on, and the expert of this lane's first one
struct Slots {
    int64_t slot0, slots, begin, end;
    int id;
};
__device__ __forceinline__ Slots slots_of(const RouteArgs& p, int64_t first, int tokens) {
    Slots s;
    s.slots = (int64_t)tokens * p.k;
    s.slot0 = first * p.k;
    const int64_t per_wave = (s.slots + kRouteThreads - 1) / kRouteThreads * 64;
    s.begin = min(s.slots, (threadIdx.x >> 6) * per_wave);
    s.end = min(s.slots, s.begin + per_wave);
    const int64_t i = s.begin + (threadIdx.x & 63);
    s.id = i < s.end ? p.ids[s.slot0 + i] : -1;
    return s;
}

// `all`, `before`: how often an expert is chosen by all blocks, by the blocks before this one; `from`: kRouteWaves x experts zeros
__device__ __forceinline__ void place_slots(const RouteArgs& p, const Slots& s, const int32_t* all, const int32_t* before, int32_t* from, int32_t* sums) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t slot0 = s.slot0, slots = s.slots, begin = s.begin, end = s.end;
    if (s.id >= 0) atomicAdd(from + wave * p.experts + s.id, 1);
    for (int64_t i = begin + 64 + lane; i < end; i += 64) {
        const int id = p.ids[slot0 + i];
        if (id >= 0) atomicAdd(from + wave * p.experts + id, 1);
    }
    // (an expert for a thread)
    const int mine = tid < p.experts ? all[tid] : 0, upto = scan_of_wave(mine, lane);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int offset = upto - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kRouteWaves; ++w) {
        offset += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    if (tid < p.experts) {
        if (blockIdx.x == 0) {
            p.offsets[tid] = offset;
            if (tid == 0) p.offsets[p.experts] = total;
        }
        int at = offset + before[tid], c[kRouteWaves];
#pragma unroll
        for (int w = 0; w < kRouteWaves; ++w) c[w] = from[w * p.experts + tid];
#pragma unroll
        for (int w = 0; w < kRouteWaves; ++w) {
            from[w * p.experts + tid] = at;
            at += c[w];
        }
    }
    __syncthreads();
    const int bits = 32 - __builtin_clz(p.experts);
    volatile int32_t* next = from + wave * p.experts;
    for (int64_t i0 = begin; i0 < end; i0 += 64) {
        const int64_t i = i0 + lane;
        const int id = i0 == begin ? s.id : i < end ? p.ids[slot0 + i] : -1;
        uint64_t same = __ballot(id >= 0);                        // lanes with this one's expert
        for (int bit = 0; bit < bits; ++bit) {
            const uint64_t set = __ballot((id >> bit) & 1);
            same &= (id >> bit) & 1 ? set : ~set;
        }
        if (id >= 0) {
            const int rank = __popcll(same & ((1ull << lane) - 1)), at = next[id] + rank;
            p.order[at] = (int32_t)(slot0 + i);
            p.place[slot0 + i] = at;
            if ((same >> lane) == 1) next[id] = at + 1;           // (the last of them)
        } else if (i < end) {
            p.place[slot0 + i] = -1;
        }
    }
    // what the slots without an expert leave over
    for (int64_t at = slot0 + tid; at < slot0 + slots; at += kRouteThreads)
        if (at >= total) p.order[at] = -1;
}

// ALONE: the call's only block
template <typename T, int G, int V, bool ALONE> __global__ void __launch_bounds__(kRouteThreads) route_choose_kernel(RouteArgs p) {
    extern __shared__ int32_t words[];
    __shared__ int32_t sums[kRouteWaves];
    int32_t *counts = words, *zeros = words + p.experts, *from = zeros + p.experts;
    const int tid = threadIdx.x;
    if (tid < p.experts) {
        counts[tid] = 0;
        if (ALONE) zeros[tid] = 0;
    }
    if (ALONE)
        for (int i = tid; i < kRouteWaves * p.experts; i += kRouteThreads) from[i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * p.tokens;
    const int tokens = (int)min((int64_t)p.tokens, p.n - first);
    choose_experts<T, G, V>(p, first, tokens, counts);
    __syncthreads();
    if constexpr (ALONE) place_slots(p, slots_of(p, first, tokens), counts, zeros, from, sums);
    else if (tid < counts_of_row(p.experts)) p.counts[(int64_t)blockIdx.x * counts_of_row(p.experts) + tid] = tid < p.experts ? counts[tid] : 0;
}

__global__ void __launch_bounds__(kRouteThreads) route_place_kernel(RouteArgs p) {
    extern __shared__ int32_t words[];
    __shared__ int32_t sums[kRouteWaves];
    int32_t *all = words, *before = words + p.experts, *from = before + p.experts;
    const int tid = threadIdx.x, blocks = (int)gridDim.x, mine = (int)blockIdx.x;
    const int64_t first = (int64_t)mine * p.tokens;
    const Slots slots = slots_of(p, first, (int)min((int64_t)p.tokens, p.n - first));
    if (tid < p.experts) all[tid] = before[tid] = 0;
    for (int i = tid; i < kRouteWaves * p.experts; i += kRouteThreads) from[i] = 0;
    __syncthreads();
    // four neighbouring experts for a thread, of every `parts`-th block
    const int pieces = counts_of_row(p.experts) / 4, parts = kRouteThreads / pieces, part = tid / pieces, piece = tid % pieces;
    if (part < parts) {
        typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));   // (working memory begins at any word)
        const i32x4* rows = reinterpret_cast<const i32x4*>(p.counts) + piece;
        i32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
#pragma unroll 8
        for (int i = part; i < blocks; i += parts) {
            const i32x4 c = rows[(int64_t)i * pieces];
            a += c;
            b += i < mine ? c : i32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (piece * 4 + q < p.experts) {
                atomicAdd(all + piece * 4 + q, a[q]);
                atomicAdd(before + piece * 4 + q, b[q]);
            }
    }
    __syncthreads();
    place_slots(p, slots, all, before, from, sums);
}

// f(lanes of a group, logits of a lane)
template <typename F> void for_experts(int64_t experts, F f) {
    if (experts <= 16) f(num<16>{}, num<1>{});
    else if (experts <= 32) f(num<16>{}, num<2>{});
    else if (experts <= 64) f(num<16>{}, num<4>{});
    else if (experts <= 128) f(num<16>{}, num<8>{});
    else if (experts <= 256) f(num<64>{}, num<4>{});
    else if (experts <= 512) f(num<64>{}, num<8>{});
    else f(num<64>{}, num<16>{});
}

// Tokens of a block: all of them where one block does the call, else one for each of its groups of lanes, or so many that the blocks are no more
// than kMostBlocks.  One block where its rounds take less than a second launch and the adding up of counts, 8 us: a round is a load's way and for each
// choice the instructions of V logits and of two sums over lanes (198 tokens, 4 experts, 3 chosen: 8.3 us in one block, 13.8 in two launches; 393
// tokens, 75 experts, 3 chosen 23.7 and 9.7).
int64_t tokens_of_block(int64_t n, int64_t experts, int64_t k) {
    int64_t groups = 1, logits = 1;
    for_experts(experts, [&](auto g, auto v) {
        groups = kRouteThreads / decltype(g)::value;
        logits = decltype(v)::value;
    });
    const int64_t rounds = (n + groups - 1) / groups;
    if (rounds <= 1 || (double)rounds * (0.8 + 0.055 * (double)(k * (logits + 4))) < 8.0) return std::max<int64_t>(1, rounds) * groups;
    return std::max(groups, (n + kMostBlocks - 1) / kMostBlocks);
}

template <typename T> void launch_route(RouteArgs& p, hipStream_t s) {
    const int blocks = (int)std::max<int64_t>(1, (p.n + p.tokens - 1) / p.tokens);   // (no tokens: the offsets alone)
    const size_t bytes = (size_t)(2 + kRouteWaves) * p.experts * 4;
    for_experts(p.experts, [&](auto g, auto v) {
        if (blocks == 1) hipLaunchKernelGGL((route_choose_kernel<T, g, v, true>), dim3(1), dim3(kRouteThreads), bytes, s, p);
        else hipLaunchKernelGGL((route_choose_kernel<T, g, v, false>), dim3(blocks), dim3(kRouteThreads), (size_t)p.experts * 8, s, p);
    });
    if (blocks > 1) hipLaunchKernelGGL(route_place_kernel, dim3(blocks), dim3(kRouteThreads), bytes, s, p);
}

// ---------------------------------------------------------------- the sum of the experts' outputs
// y[t] = r[t] + sum_j w[t, j] z[place[t, j]], in this order, in fp32.  A thread has the columns of 16 bytes of a row; the rows of up to 8
// slots are asked for at once.  Bound: the rows' bytes, each read once (so their lines are not kept).  ALIKE: all threads of a wavefront have the same
// token, whose places and weights are scalar loads.
struct CombineArgs {
    const unsigned char* z;
    const int32_t* place;
    const float* weights;
    const void* r;
    void* y;
    int64_t n, rows, d, units;                     // units: threads of a token
    int k, out_f32;
};

typedef uint32_t any16_t __attribute__((ext_vector_type(4), aligned(2)));

template <typename T, bool ALIKE> __global__ void __launch_bounds__(256) combine_kernel(CombineArgs p) {
    constexpr int C = 16 / (int)sizeof(T);         // columns of a thread
    const uint32_t u = blockIdx.x * 256u + threadIdx.x;
    int64_t t = u / (uint32_t)p.units;
    if (t >= p.n) return;
    if constexpr (ALIKE) t = __builtin_amdgcn_readfirstlane((int)t);
    const int64_t c = (u - t * p.units) * C;
    const int columns = (int)min((int64_t)C, p.d - c);
    float v[C] = {};
    for (int j0 = 0; j0 < p.k; j0 += 8) {
        int at[8];
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            at[j] = j0 + j < p.k ? p.place[t * p.k + j0 + j] : -1;
            w[j] = j0 + j < p.k ? p.weights[t * p.k + j0 + j] : 0.0f;
            at[j] = at[j] < p.rows ? at[j] : -1;
        }
        // (a dropped slot asks for row 0, whose values are not used: a branch around every load would wait for each of them)
        td_u32x4 x[8];
        if (columns == C) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __builtin_nontemporal_load(reinterpret_cast<const any16_t*>(reinterpret_cast<const T*>(p.z) + (int64_t)max(at[j], 0) * p.d + c));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const T* row = reinterpret_cast<const T*>(p.z) + (int64_t)max(at[j], 0) * p.d + c;
                x[j] = td_u32x4{0, 0, 0, 0};
#pragma unroll
                for (int q = 0; q < C; ++q) {
                    if (q >= columns) continue;
                    if constexpr (sizeof(T) == 4) x[j][q] = __float_as_uint(row[q]);
                    else x[j][q / 2] |= (uint32_t)row[q] << (16 * (q & 1));
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int q = 0; q < C; ++q) {
                float z;
                if constexpr (sizeof(T) == 4) z = __uint_as_float(x[j][q]);
                else z = __uint_as_float(q & 1 ? x[j][q / 2] & 0xffff0000u : x[j][q / 2] << 16);
                v[q] = at[j] < 0 ? v[q] : fmaf(w[j], z, v[q]);
            }
    }
    const int64_t to = t * p.d + c;
    if (columns < C) {                             // the end of a row
#pragma unroll
        for (int q = 0; q < C; ++q) {
            if (q >= columns) continue;
            if (p.r) v[q] += p.out_f32 ? static_cast<const float*>(p.r)[to + q] : td_load<bf16_t>(static_cast<const bf16_t*>(p.r) + to + q);
            if (p.out_f32) static_cast<float*>(p.y)[to + q] = v[q];
            else td_store<bf16_t>(static_cast<bf16_t*>(p.y) + to + q, v[q]);
        }
    } else if (p.out_f32) {
#pragma unroll
        for (int h = 0; h < C; h += 4) {
            if (p.r) {
                const td_u32x4 r = *reinterpret_cast<const any16_t*>(static_cast<const float*>(p.r) + to + h);
#pragma unroll
                for (int q = 0; q < 4; ++q) v[h + q] += __uint_as_float(r[q]);
            }
            *reinterpret_cast<any16_t*>(static_cast<float*>(p.y) + to + h) =
                any16_t{__float_as_uint(v[h]), __float_as_uint(v[h + 1]), __float_as_uint(v[h + 2]), __float_as_uint(v[h + 3])};
        }
    } else {
        typedef uint32_t any_t __attribute__((ext_vector_type(C / 2), aligned(2)));
        if (p.r) {
            const any_t r = *reinterpret_cast<const any_t*>(static_cast<const bf16_t*>(p.r) + to);
#pragma unroll
            for (int q = 0; q < C; ++q) v[q] += __uint_as_float(q & 1 ? r[q / 2] & 0xffff0000u : r[q / 2] << 16);
        }
        any_t o;
#pragma unroll
        for (int q = 0; q < C / 2; ++q) o[q] = to_bf16x2(v[2 * q], v[2 * q + 1]);
        *reinterpret_cast<any_t*>(static_cast<bf16_t*>(p.y) + to) = o;
    }
}

}  // namespace

size_t td_route_work_bytes(int64_t n, int64_t experts, int64_t k) {
    const int64_t tokens = tokens_of_block(n, experts, k), blocks = (n + tokens - 1) / tokens;
    return blocks > 1 ? (size_t)blocks * counts_of_row((int)experts) * 4 : 0;
}

tardis_status_t td_moe_route(const void* logits, int64_t n, int64_t experts, int64_t k, int32_t dtype, int renormalise, int32_t* ids, float* weights,
                             int32_t* offsets, int32_t* order, int32_t* place, void* work, hipStream_t s) {
    RouteArgs p{};
    p.logits = logits;
    p.n = n;
    p.experts = (int)experts;
    p.k = (int)k;
    p.renormalise = renormalise;
    p.tokens = (int)tokens_of_block(n, experts, k);
    p.ids = ids;
    p.weights = weights;
    p.offsets = offsets;
    p.order = order;
    p.place = place;
    p.counts = static_cast<int32_t*>(work);
    if (dtype == TARDIS_F32) launch_route<float>(p, s);
    else launch_route<bf16_t>(p, s);
    TD_HIP(hipGetLastError());
    return TARDIS_OK;
}

tardis_status_t td_moe_combine(const void* z, int64_t rows, const int32_t* place, const float* weights, int64_t n, int64_t k, int64_t d, int32_t dtype,
                               const void* residual, void* y, int32_t out_dtype, hipStream_t s) {
    CombineArgs p{};
    p.z = static_cast<const unsigned char*>(z);
    p.rows = rows;
    p.d = d;
    p.k = rows > 0 ? (int)k : 0;
    p.out_f32 = out_dtype == TARDIS_F32;
    const int64_t columns = dtype == TARDIS_F32 ? 4 : 8, eo = (int64_t)td_elem_size(out_dtype);
    p.units = (d + columns - 1) / columns;
    const bool alike = p.units % 64 == 0;
    const int64_t most = kMostThreads / p.units;                   // tokens of a launch
    for (int64_t t = 0; t < n; t += most) {
        p.n = std::min(most, n - t);
        p.place = place + t * k;
        p.weights = weights + t * k;
        p.r = residual ? static_cast<const unsigned char*>(residual) + t * d * eo : nullptr;
        p.y = static_cast<unsigned char*>(y) + t * d * eo;
        auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)((p.units * p.n + 255) / 256)), dim3(256), 0, s, p); };
        if (dtype == TARDIS_F32) launch(alike ? combine_kernel<float, true> : combine_kernel<float, false>);
        else launch(alike ? combine_kernel<bf16_t, true> : combine_kernel<bf16_t, false>);
    }
    TD_HIP(hipGetLastError());
    return TARDIS_OK;
}
