// route.h -- gfx950 device code of the top-k router: for every row the k
// experts with the largest scores, their weights, and the lists that group the
// assignments by expert, the many-way form of the mask unit and its index maps.
//
// Choice.  key = fl32(logit + bias), or the score (softmax or sigmoid, fp32) plus the
// bias; the k largest keys win, ties go to the lowest expert.  An expert whose logit or
// key is NaN or -inf, and every expert of a masked row, is never chosen; a slot without
// an expert holds -1 and weight 0.  Keys are compared as integers that order like the
// floats, so the choice is exact.  Weights are fp32: softmax with the maximum
// subtracted, or sigmoid; a bias never counts in them.
//
// Lists.  Assignment a = row * k + slot.  A counting sort that keeps the order:
// the choosing workgroups count their assignments per expert, k_route_scan adds up
// the counts of the workgroups before each, and the list workgroups rank from there
// (up to 128 rows one workgroup does all three).  Every rank comes
// from ballots and sums of whole numbers, so the lists do not depend on timing.
#pragma once

#include "kernels.h"

namespace dynconv {

constexpr int kMaxExperts = 1024;
constexpr int kMaxTopK = 16;
constexpr int kRouteThreads = 512;
constexpr int kRouteWaves = kRouteThreads / kWave;

constexpr int kRouteSigmoid = 1, kRouteRenormalize = 2, kRouteScoreBias = 8;

// Reductions over G consecutive lanes (16 or 64); every lane gets the result.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u(uint32_t v) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, false));
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;

template <int G, typename F>
__device__ __forceinline__ uint32_t group_reduce(uint32_t v, F op) {
    v = op(v, dpp_u<kDppXor1>(v));
    v = op(v, dpp_u<kDppXor2>(v));
    v = op(v, dpp_u<kDppHalfMirror>(v));
    v = op(v, dpp_u<kDppMirror>(v));
    if constexpr (G == 64) {
        v = op(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), 16)));
        v = op(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), 32)));
    }
    return v;
}
template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
    return group_reduce<G>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int G>
__device__ __forceinline__ uint32_t group_min(uint32_t v) {
    return group_reduce<G>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
template <int G>
__device__ __forceinline__ float group_maxf(float v) {
    return __uint_as_float(group_reduce<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}
template <int G>
__device__ __forceinline__ float group_sumf(float v) {
    return __uint_as_float(group_reduce<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}

// Floats as integers of the same order; 0 stands for NaN and -inf, which no
// other value maps to.  Adding +0 makes the two zeros one.
__device__ __forceinline__ uint32_t order_key(float v) {
    v += 0.0f;
    const uint32_t u = __float_as_uint(v);
    const uint32_t k = (u >> 31) ? ~u : (u | 0x80000000u);
    return v > -__builtin_huge_valf() ? k : 0u;
}

// exp(v - top) where equal infinities count as 1
__device__ __forceinline__ float exp_below(float v, float top) { return v == top ? 1.0f : expf(v - top); }

// 1 / (1 + exp(-v)) by the exponential that does not overflow
__device__ __forceinline__ float sigmoid(float v) {
    const float e = expf(-fabsf(v));
    return (v < 0.0f ? e : 1.0f) / (1.0f + e);
}

// A row of logits on G lanes, V = ceil(E / G) experts a lane (expert v * G + lane).
template <typename T, int G, int V>
__device__ __forceinline__ void load_row(const T *__restrict__ row, bool on, int E, int lane, float (&l)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = v * G + lane;
        l[v] = on && e < E ? static_cast<float>(row[e]) : -__builtin_huge_valf();
    }
}

// Chooses for the row in l.  Lane j < top_k returns slot j: expert (-1: none) and
// weight.
template <typename T, int G, int V>
__device__ __forceinline__ void choose_row(const float (&l)[V], const T *__restrict__ row, int E, int top_k,
                                           const float *__restrict__ bias, int flags, float scale, int lane,
                                           int &expert, float &weight) {
    uint32_t key[V];
    float all_top = -__builtin_huge_valf(), all_sum = 0.0f;
    const bool whole = !(flags & (kRouteSigmoid | kRouteRenormalize));  // softmax over every live expert
    const bool by_score = bias && (flags & kRouteScoreBias);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = v * G + lane;
        key[v] = order_key(bias && !by_score && e < E ? l[v] + bias[e] : l[v]);
    }
    if (whole || (by_score && !(flags & kRouteSigmoid))) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (key[v]) all_top = fmaxf(all_top, l[v]);
        all_top = group_maxf<G>(all_top);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (key[v]) all_sum += exp_below(l[v], all_top);
        all_sum = group_sumf<G>(all_sum);
    }
    if (by_score) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = v * G + lane;
            if (!key[v]) continue;  // e < E
            const float score = (flags & kRouteSigmoid) ? sigmoid(l[v]) : exp_below(l[v], all_top) / all_sum;
            key[v] = order_key(score + bias[e]);
        }
    }
    expert = -1;
    for (int j = 0; j < top_k; ++j) {
        uint32_t m = key[0];
#pragma unroll
        for (int v = 1; v < V; ++v) m = key[v] > m ? key[v] : m;
        m = group_max<G>(m);
        uint32_t at = 0xffffffffu;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) at = key[v] == m ? static_cast<uint32_t>(v * G + lane) : at;
        at = group_min<G>(at);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = at == static_cast<uint32_t>(v * G + lane) ? 0u : key[v];
        if (lane == j && m != 0) expert = static_cast<int>(at);
    }
    weight = 0.0f;
    const float le = expert >= 0 ? static_cast<float>(row[expert]) : -__builtin_huge_valf();
    if (flags & kRouteSigmoid) {
        float s = sigmoid(le), sum = 1.0f;
        if (flags & kRouteRenormalize) {
            // all below 0: relative to the largest's, so that they do not all underflow
            const float top = group_maxf<G>(le);
            if (top < 0.0f) s = exp_below(le, top) * (1.0f + expf(top)) / (1.0f + expf(le));
            sum = group_sumf<G>(expert >= 0 ? s : 0.0f);
        }
        if (expert >= 0) weight = scale * (s / sum);
    } else {
        const float top = whole ? all_top : group_maxf<G>(le);
        const float p = expert >= 0 ? exp_below(le, top) : 0.0f;
        const float sum = whole ? all_sum : group_sumf<G>(p);
        if (expert >= 0) weight = scale * (p / sum);
    }
}

// Lanes of the wave whose value equals this lane's (values below 2^bits).
__device__ __forceinline__ uint64_t equal_lanes(uint32_t v, int bits, uint64_t among) {
    for (int b = 0; b < bits; ++b) {
        const bool bit = (v >> b) & 1u;
        const uint64_t set = __ballot(bit);
        among &= bit ? set : ~set;
    }
    return among;
}

// The exclusive sum over the workgroup's threads (NT of them) of v; total gets
// the whole sum.  sums: NT / 64 words of LDS.
template <int NT>
__device__ __forceinline__ int block_scan_excl(int v, int *sums, int &total) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int incl = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == kWave - 1) sums[wave] = incl;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    __syncthreads();
    return before + incl - v;
}

// Writes the list entries of the `n` assignments starting at a0, whose experts
// (E: none) are ids[0 .. n): base[e] is the list position of the workgroup's
// first assignment of expert e, cnt [waves][E + 1] is scratch.  Each wave takes
// one run of assignments, counts it, and ranks it after the waves before it.
template <int NT>
__device__ __forceinline__ void place_assignments(const uint16_t *ids, int n, int64_t a0, int E, int bits,
                                                  const int *base, uint16_t *cnt, int32_t *__restrict__ rows) {
    constexpr int NW = NT / kWave;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int stride = E + 1;
    for (int i = threadIdx.x; i < NW * stride; i += NT) cnt[i] = 0;
    __syncthreads();
    const int per = (n + NW * kWave - 1) / (NW * kWave) * kWave;
    const int lo = wave * per, hi = lo + per < n ? lo + per : n;
    uint16_t *mine = cnt + wave * stride;
    for (int i0 = lo; i0 < hi; i0 += kWave) {
        const int i = i0 + lane;
        const bool in = i < hi;
        const uint32_t e = in ? ids[i] : 0;
        const uint64_t same = equal_lanes(e, bits, __ballot(in));
        if (in && (same & lanemask_lt(lane)) == 0) mine[e] = static_cast<uint16_t>(mine[e] + __popcll(same));
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (int e = threadIdx.x; e < stride; e += NT) {
        int run = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int c = cnt[w * stride + e];
            cnt[w * stride + e] = static_cast<uint16_t>(run);
            run += c;
        }
    }
    __syncthreads();
    for (int i0 = lo; i0 < hi; i0 += kWave) {
        const int i = i0 + lane;
        const bool in = i < hi;
        const uint32_t e = in ? ids[i] : 0;
        const uint64_t same = equal_lanes(e, bits, __ballot(in));
        const int first = in ? mine[e] : 0;
        __builtin_amdgcn_wave_barrier();
        if (in) {
            const int64_t at = static_cast<int64_t>(base[e]) + first + __popcll(same & lanemask_lt(lane));
            rows[at] = e == static_cast<uint32_t>(E) ? -1 : static_cast<int32_t>(a0 + i);
            if ((same & lanemask_lt(lane)) == 0) mine[e] = static_cast<uint16_t>(first + __popcll(same));
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Rows [t0, t1): choose, write expert and weight, and leave the experts of the
// assignments in ids (LDS).
template <typename T, int G, int V, int NT>
__device__ __forceinline__ void choose_rows(const T *__restrict__ logits, int64_t t0, int64_t t1, int E, int top_k,
                                            const float *__restrict__ bias, const uint8_t *__restrict__ mask, int flags,
                                            float scale, int32_t *__restrict__ expert, float *__restrict__ weight,
                                            uint16_t *ids) {
    const int lane = threadIdx.x % G;
    auto fetch = [&](int64_t t, float (&to)[V]) {
        load_row<T, G, V>(logits + t * E, !mask || mask[t] != 0, E, lane, to);
    };
    float l[V], after[V];
    int64_t t = t0 + threadIdx.x / G;
    if (t < t1) fetch(t, l);
    for (; t < t1; t += NT / G) {
        // the next row comes while this one is chosen from
        if (t + NT / G < t1) fetch(t + NT / G, after);
        int e;
        float w;
        choose_row<T, G, V>(l, logits + t * E, E, top_k, bias, flags, scale, lane, e, w);
        if (lane < top_k) {
            expert[t * top_k + lane] = e;
            weight[t * top_k + lane] = w;
            ids[(t - t0) * top_k + lane] = static_cast<uint16_t>(e < 0 ? E : e);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] = after[v];
    }
}

// Everything in one workgroup, for calls of few rows: 5.4 us for 8 rows of 64
// experts, top 8, the chain of a launch, one load, the rounds and four barriers.
constexpr int kRouteOneThreads = 1024;
constexpr int kRouteOne = 2048;

template <typename T, int G, int V>
__global__ void __launch_bounds__(kRouteOneThreads)
k_route_one(const T *__restrict__ logits, int tokens, int E, int top_k, int bits, const float *__restrict__ bias,
            const uint8_t *__restrict__ mask, int flags, float scale, int32_t *__restrict__ expert,
            float *__restrict__ weight, int32_t *__restrict__ rows, int32_t *__restrict__ starts) {
    __shared__ uint16_t ids[kRouteOne];
    __shared__ int base[kMaxExperts + 1];
    __shared__ int sums[kRouteOneThreads / kWave];
    extern __shared__ uint16_t cnt[];  // [waves][E + 1]
    const int n = tokens * top_k;
    for (int e = threadIdx.x; e <= E; e += kRouteOneThreads) base[e] = 0;
    choose_rows<T, G, V, kRouteOneThreads>(logits, 0, tokens, E, top_k, bias, mask, flags, scale, expert, weight, ids);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kRouteOneThreads) atomicAdd(&base[ids[i]], 1);
    __syncthreads();
    const int e = threadIdx.x;  // E <= kRouteOneThreads: one expert a thread, the slots without one at n
    int total;
    const int c = e < E ? base[e] : 0;
    const int before = block_scan_excl<kRouteOneThreads>(c, sums, total);
    if (e < E) {
        base[e] = before;
        starts[e] = before;
    }
    if (e == 0) {
        base[E] = total;
        starts[E] = total;
    }
    __syncthreads();
    place_assignments<kRouteOneThreads>(ids, n, 0, E, bits, base, cnt, rows);
}

// Longer calls: choose and count, then add the counts up, then the lists; a
// workgroup takes at most kRouteChunk assignments.  Choosing is bound by its vector
// instructions: a round is some 60 of them for 4 rows a wave at 128 experts (the
// largest of a lane's 8 keys, 4 steps over 16 lanes, the place of that key, 4 steps
// for the lowest, its removal).  32768 rows of 128 fp32 logits, top 8: 14.0 us (16.8
// MB: 3.3 us at the rate of a large copy), 7.4 us for the top 1; counts 4.0, lists
// 6.5 us.  16 lanes a row do with a quarter of the steps of a whole wave; a lane's
// experts are 16 apart, so that its loads cover whole lines.
constexpr int kRouteChunk = 2048;

template <typename T, int G, int V, int NT>
__global__ void __launch_bounds__(NT)
k_route_choose(const T *__restrict__ logits, int64_t tokens, int per, int E, int top_k, const float *__restrict__ bias,
               const uint8_t *__restrict__ mask, int flags, float scale, int32_t *__restrict__ expert,
               float *__restrict__ weight, int32_t *__restrict__ hist) {
    __shared__ uint16_t ids[kRouteChunk];
    __shared__ int count[kMaxExperts + 1];
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * per;
    const int64_t t1 = t0 + per < tokens ? t0 + per : tokens;
    for (int e = threadIdx.x; e <= E; e += NT) count[e] = 0;
    choose_rows<T, G, V, NT>(logits, t0, t1, E, top_k, bias, mask, flags, scale, expert, weight, ids);
    __syncthreads();
    const int n = static_cast<int>(t1 - t0) * top_k;
    for (int i = threadIdx.x; i < n; i += NT) atomicAdd(&count[ids[i]], 1);
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += NT)
        hist[static_cast<int64_t>(blockIdx.x) * (E + 1) + e] = count[e];
}

// List positions of every workgroup's first assignment of every expert: one
// wave an expert walks the workgroups' counts, in place; totals[e] gets the sum.
__global__ void __launch_bounds__(kBlock)
k_route_scan(int32_t *__restrict__ hist, int blocks, int stride, int32_t *__restrict__ totals) {
    const int lane = threadIdx.x % kWave;
    const int e = blockIdx.x * kWavesPerBlock + threadIdx.x / kWave;
    if (e >= stride) return;
    constexpr int kOnce = 4;  // loads in flight
    int run = 0;
    for (int b0 = 0; b0 < blocks; b0 += kOnce * kWave) {
        int c[kOnce];
#pragma unroll
        for (int i = 0; i < kOnce; ++i) {
            const int b = b0 + i * kWave + lane;
            c[i] = b < blocks ? hist[static_cast<int64_t>(b) * stride + e] : 0;
        }
#pragma unroll
        for (int i = 0; i < kOnce; ++i) {
            const int b = b0 + i * kWave + lane;
            int incl = c[i];
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const int o = __shfl_up(incl, d);
                if (lane >= d) incl += o;
            }
            if (b < blocks) hist[static_cast<int64_t>(b) * stride + e] = run + incl - c[i];
            run += __shfl(incl, kWave - 1);
        }
    }
    if (lane == 0) totals[e] = run;
}

__global__ void __launch_bounds__(kRouteThreads)
k_route_lists(const int32_t *__restrict__ expert, int64_t n, int per, int E, int bits, const int32_t *__restrict__ hist,
              const int32_t *__restrict__ totals, int32_t *__restrict__ rows, int32_t *__restrict__ starts) {
    __shared__ uint16_t ids[kRouteChunk];
    __shared__ int base[kMaxExperts + 1];
    __shared__ int sums[kRouteWaves];
    extern __shared__ uint16_t cnt[];  // [waves][E + 1]
    const int64_t a0 = static_cast<int64_t>(blockIdx.x) * per;
    const int here = static_cast<int>(a0 + per < n ? per : n - a0);
    for (int i = threadIdx.x; i < here; i += kRouteThreads) {
        const int e = expert[a0 + i];
        ids[i] = static_cast<uint16_t>(e < 0 ? E : e);
    }
    const int32_t *mine = hist + static_cast<int64_t>(blockIdx.x) * (E + 1);
    int run = 0;  // of the experts before this pass's
    for (int e0 = 0; e0 <= E; e0 += kRouteThreads) {
        const int e = e0 + threadIdx.x;
        int total;
        const int before = run + block_scan_excl<kRouteThreads>(e <= E ? totals[e] : 0, sums, total);
        if (e <= E) {
            base[e] = before + mine[e];
            if (blockIdx.x == 0) starts[e] = before;
        }
        run += total;
    }
    __syncthreads();
    place_assignments<kRouteThreads>(ids, here, a0, E, bits, base, cnt, rows);
}

}  // namespace dynconv
