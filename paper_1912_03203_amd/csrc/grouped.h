// grouped.h -- gfx950 device code of the products y = act(W_g x + b_g) of many
// rows with the weights of their groups: experts of a router, or one shared
// projection with low-rank adapters of many requests beside it.
//
// Rows of group g are the list positions [starts[g], starts[g + 1]); lists
// gather the rows that go in (src, divided by src_div) and scatter the rows
// that come out (dst).  The sizes stay on the device: a launch has workgroups
// for the most tiles that any split of its rows can have, and each finds its
// tile from starts.
//
// Everything moves in chunks of 16 bytes along the contraction: 8 entries in
// fp16/bf16, 4 in fp32.  The weights are the matrix cores' A operand and the
// rows the B operand, so a lane ends with 4 consecutive outputs of one row.
#pragma once

#include <type_traits>

#include "kernels.h"
#include "route.h"
#include "wide.h"

namespace dynconv {

constexpr int kMaxGroups = 1024;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// One 16x16 product over a chunk per lane: lane 16 g + r holds chunk g of row
// r, so a step covers 64 bytes of the contraction.
template <typename T>
__device__ __forceinline__ floatx4 chunk_mma(u32x4 a, u32x4 b, floatx4 c) {
    if constexpr (sizeof(T) == 2) {
        typedef typename mma<T>::frag F;
        return mma<T>::run(__builtin_bit_cast(F, a), __builtin_bit_cast(F, b), c);
    } else {
        const floatx4 fa = __builtin_bit_cast(floatx4, a), fb = __builtin_bit_cast(floatx4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[j], fb[j], c, 0, 0, 0);
        return c;
    }
}

// Activations of these calls: none, ReLU, ReLU6, SiLU, GELU.  NaN stays NaN (the
// blocks' clamp is a median of three, which drops it).  GELU by erfc: 1 + erf cancels
// for negative values, 4 % off at -5 and 0 from -5.5 on.
__device__ __forceinline__ float act_any(float v, int kind) {
    if (kind == 0) return v;
    if (kind <= 2) {
        const float low = v < 0.0f ? 0.0f : v;
        return kind == 2 && low > 6.0f ? 6.0f : low;
    }
    if (kind == 3) return v / (1.0f + __expf(-v));
    return 0.5f * v * erfcf(v * -0.70710678118654752f);
}

struct RowsArgs {
    const char *x;         // rows that go in, pitch bytes each
    int64_t x_rows;
    int64_t pitch;         // c_in * sizeof(T)
    const int32_t *src;    // or NULL: list position p reads row p / src_div
    uint32_t src_div;
    const int32_t *starts; // or NULL: one group of all rows
    int groups;
    int64_t rows;          // list positions
    const char *w, *w2;    // [groups][c_out][c_in]; w2: the gate's, or NULL
    const float *b, *b2;   // [groups][c_out], or NULL
    int c_out;
    int act;
    char *y;               // rows that come out, c_out entries each
    int64_t y_rows;
    const int32_t *dst;    // or NULL: list position p writes row p
    bool halves;           // few rows, 16-bit types: a row's entries, then what their rounding left
    // low-rank adapters: y += up[ids[row]] * v[row]
    const char *v;         // [rows][v_pitch bytes], see add_adapters
    int v_pitch;
    const char *up;        // [adapters][c_out][max_rank]
    const int32_t *ids, *ranks;
    int adapters, max_rank, id_bits;  // id_bits: of the numbers below adapters
};

// ---------------------------------------------------------------- tiles
// Work item `id` of the launch: a tile of BM rows of one group (group, row0,
// end) and a slice of the outputs; false past the last one.  Every wave works
// it out by itself, 64 groups a step: the tiles that the groups really have,
// then the item's place among them.  Workgroups go to the 8 XCDs in turn, so
// an XCD gets one run of the items: its L2 then holds the rows and weights of
// neighbouring tiles.  Within a run 8 slices of a row tile come side by side.
struct RowTile {
    int group, slice;
    int64_t row0, end;
};

__device__ __forceinline__ int64_t clamp_row(int64_t v, int64_t rows) { return v < 0 ? 0 : v > rows ? rows : v; }

constexpr int kBand = 8;

// Tiles of group g and its rows; ascends: whether its end is not before its start.
template <int BM>
__device__ __forceinline__ int group_tiles(const int32_t *__restrict__ starts, int groups, int64_t rows, int g, int &lo,
                                           int &hi, bool &ascends) {
    lo = hi = 0;
    ascends = true;
    if (g < groups) {
        const int s = starts[g], e = starts[g + 1];
        ascends = s <= e;
        lo = static_cast<int>(clamp_row(s, rows));
        hi = static_cast<int>(clamp_row(e, rows));
    }
    return hi > lo ? static_cast<int>((static_cast<int64_t>(hi) - lo + BM - 1) / BM) : 0;
}

__device__ __forceinline__ int wave_incl(int v, int lane) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

template <int BM>
__device__ __forceinline__ bool find_tile(const int32_t *__restrict__ starts, int groups, int64_t rows, int id,
                                          int slices, RowTile &t) {
    const int lane = threadIdx.x % kWave;
    int lo = 0, hi = 0, incl = 0, n = 0;
    int64_t total;
    if (!starts) {
        total = (rows + BM - 1) / BM;
    } else {
        int sum = 0;
        for (int g0 = 0; g0 < groups; g0 += kWave) {
            bool ascends;
            n = group_tiles<BM>(starts, groups, rows, g0 + lane, lo, hi, ascends);
            // starts that do not ascend could name more tiles than a launch counts
            if (__ballot(!ascends)) return false;
            incl = wave_incl(n, lane);
            sum += __builtin_amdgcn_readlane(incl, kWave - 1);
        }
        total = sum;
    }
    // fewer than 2^31 items: the host refuses more
    const uint32_t tiles = static_cast<uint32_t>(total), items = tiles * slices, per = (items + 7) / 8;
    const uint32_t place = static_cast<uint32_t>(id) / 8, item = static_cast<uint32_t>(id) % 8 * per + place;
    if (place >= per || item >= items) return false;
    const int band = slices > kBand ? static_cast<int>(item / (tiles * kBand)) : 0;
    const int width = slices - band * kBand < kBand ? slices - band * kBand : kBand;
    const uint32_t in_band = item - tiles * kBand * band;
    const int tile = static_cast<int>(in_band / static_cast<uint32_t>(width));
    t.slice = band * kBand + static_cast<int>(in_band % static_cast<uint32_t>(width));
    if (!starts) {
        t.group = 0;
        t.row0 = static_cast<int64_t>(tile) * BM;
        t.end = rows;
        return true;
    }
    int before = 0;
    for (int g0 = 0; g0 < groups; g0 += kWave) {
        if (groups > kWave) {
            bool ascends;
            n = group_tiles<BM>(starts, groups, rows, g0 + lane, lo, hi, ascends);
            incl = wave_incl(n, lane);
        }
        const uint64_t past = __ballot(before + incl > tile);
        if (past) {
            const int l = __ffsll(static_cast<unsigned long long>(past)) - 1;
            t.group = g0 + l;
            const int first = before + __builtin_amdgcn_readlane(incl - n, l);
            t.row0 = static_cast<int64_t>(__builtin_amdgcn_readlane(lo, l)) + static_cast<int64_t>(tile - first) * BM;
            t.end = __builtin_amdgcn_readlane(hi, l);
            return true;
        }
        before += __builtin_amdgcn_readlane(incl, kWave - 1);
    }
    return false;
}

// The row that list position p reads, or -1 where the list names none.
__device__ __forceinline__ int64_t source_row(const RowsArgs &a, int64_t p) {
    int64_t s = a.src ? static_cast<int64_t>(a.src[p]) : p;
    if (s < 0) return -1;
    if (a.src_div != 1) s = static_cast<uint32_t>(s) / a.src_div;
    return s < a.x_rows ? s : -1;
}

__device__ __forceinline__ int64_t target_row(const RowsArgs &a, int64_t p) {
    const int64_t d = a.dst ? static_cast<int64_t>(a.dst[p]) : p;
    return d >= 0 && d < a.y_rows ? d : -1;
}

template <typename OT>
__device__ __forceinline__ void store_out(OT *p, const float v[4]) {
    io<OT>::store4(p, v);
}

// What is left of v when it is stored as OT; nothing beside NaN and infinities.
template <typename OT>
__device__ __forceinline__ float rest_of(float v) {
    const float high = static_cast<float>(static_cast<OT>(v));
    return fabsf(high) < __builtin_huge_valf() ? v - high : 0.0f;
}

// act(sum + bias) of 4 consecutive outputs, gated: act(gate) * value.
template <bool GATED>
__device__ __forceinline__ void finish4(const RowsArgs &a, int group, int n, floatx4 s, floatx4 s2, float out[4]) {
    float b[4] = {0.0f, 0.0f, 0.0f, 0.0f}, b2[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t at = static_cast<int64_t>(group) * a.c_out + n;
    if (a.b) io<float>::load4(a.b + at, b);
    if (GATED && a.b2) io<float>::load4(a.b2 + at, b2);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const float v = s[u] + b[u];
        out[u] = GATED ? act_any(s2[u] + b2[u], a.act) * v : act_any(v, a.act);
    }
}

// ---------------------------------------------------------------- adapters
__device__ __forceinline__ int adapter_rank(const RowsArgs &a, int ad) {
    const int rank = a.ranks ? a.ranks[ad] : a.max_rank;
    return rank < a.max_rank ? rank : a.max_rank;
}

__device__ __forceinline__ int adapter_of(const RowsArgs &a, int64_t row, bool in) {
    if (!in) return -1;
    const int id = a.ids[row];
    return id >= 0 && id < a.adapters ? id : -1;
}

// The adapter of a row and its rank in one number, or -1 where nothing is added.
constexpr int kAdapterBits = 20;
constexpr int kMaxAdapters = 1 << kAdapterBits;
__device__ __forceinline__ int adapter_key(const RowsArgs &a, int64_t row, bool in) {
    const int id = adapter_of(a, row, in), rank = id < 0 ? 0 : adapter_rank(a, id);
    return rank > 0 ? rank << kAdapterBits | id : -1;
}

// The distinct adapters of a tile of BM rows (row i * 64 + l's key in keys[i] of lane
// l), in the order of their first rows; each wave walks by itself, over numbers that
// all its lanes share.
template <int BM>
struct AdapterWalk {
    uint64_t open[BM / kWave];  // rows of the adapters to come
    uint64_t own;               // this adapter's rows of the 64 that `next` is asked for
    int id, rank, k0;           // k0: its next rank
    __device__ __forceinline__ void start(const int (&keys)[BM / kWave]) {
#pragma unroll
        for (int i = 0; i < BM / kWave; ++i) open[i] = __ballot(keys[i] >= 0);
        own = 0;
        id = rank = k0 = 0;
    }
    __device__ __forceinline__ bool next(const int (&keys)[BM / kWave], int block) {
        int key = -1;
#pragma unroll
        for (int i = 0; i < BM / kWave; ++i)
            if (open[i] && key < 0)
                key = __builtin_amdgcn_readlane(keys[i], __ffsll(static_cast<unsigned long long>(open[i])) - 1);
        if (key < 0) return false;
#pragma unroll
        for (int i = 0; i < BM / kWave; ++i) {
            const uint64_t same = __ballot(keys[i] == key);
            open[i] &= ~same;
            own = i == block ? same : own;
        }
        id = key & (kMaxAdapters - 1);
        rank = key >> kAdapterBits;
        k0 = 0;
        return true;
    }
};

// The distinct adapters of up to 64 rows, row l's (or -1) in lane l: the lanes
// that hold the first row of each.
__device__ __forceinline__ uint64_t distinct_lanes(int id, int bits) {
    const int lane = threadIdx.x % kWave;
    const uint64_t same = equal_lanes(static_cast<uint32_t>(id), bits, __ballot(id >= 0));
    return __ballot(id >= 0 && (same & lanemask_lt(lane)) == 0);
}
__device__ __forceinline__ uint64_t drop_lanes(uint64_t set, int n) {
    for (int i = 0; i < n && set; ++i) set &= set - 1;
    return set;
}

// The second product takes v = scale * down x in the storage type, but a rounded v
// adds a tenth to the result's error (bf16), so 16-bit types keep v as two halves: its
// rounding, and what that left.  They lie chunk by chunk in turn, so a row of v has
// 4 * max_rank bytes in every type, and a step of 64 bytes of it covers 16 ranks: four
// chunks of fp32, or two of the first halves and two of the second, which meet the
// same two chunks of up.
constexpr int kStepRanks = 16;

// The first rank of chunk c of a step's four, and whether it meets a second half.
template <typename T> __device__ __forceinline__ int chunk_rank(int c) { return sizeof(T) == 2 ? c / 2 * 8 : c * 4; }
template <typename T> __device__ __forceinline__ bool chunk_rest(int c) { return sizeof(T) == 2 && c % 2 != 0; }

// A chunk of up without its infinities and NaN; odd gets a bit where there was one.
template <typename T>
__device__ __forceinline__ u32x4 finite_part(u32x4 u, uint32_t &odd) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t m;  // all bits of such an entry
        if constexpr (sizeof(T) == 4) {
            m = static_cast<uint32_t>(static_cast<int32_t>((u[j] & 0x7fffffffu) + 0x00800000u) >> 31);
        } else {
            typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
            constexpr uint32_t kPast = std::is_same<T, half_t>::value ? 0x04000400u : 0x00800080u;
            m = __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, (u[j] & 0x7fff7fffu) + kPast) >> 15);
        }
        u[j] &= ~m;
        odd |= m;
    }
    return u;
}

// Its first `keep` entries, then zeros: the columns past a rank do not count.
template <typename T>
__device__ __forceinline__ u32x4 used_part(u32x4 u, int keep) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) u[j] = keep > j ? u[j] : 0u;
        else u[j] = keep > 2 * j + 1 ? u[j] : keep > 2 * j ? u[j] & 0xffffu : 0u;
    }
    return u;
}

// acc += up[id] * v over the distinct adapters of MF * 16 rows from row0 (row
// l's adapter, or -1, in lane l) and the 16 outputs from n0.  Each adapter is one
// more run of the contraction, whose sums only its own rows take (zeros for the
// others' v would not do: an infinity or NaN in up makes NaN of them); of the
// adapters, every `of`-th from `first` is taken (waves share the work), four at a
// time, so that the loads of four are in flight.
template <typename T, int MF>
__device__ __forceinline__ void add_adapters(const RowsArgs &a, int row_id, int64_t row0, int n0, int first, int of,
                                             floatx4 (&acc)[1][MF]) {
    constexpr int kOnce = 4;
    const int lane = threadIdx.x % kWave, g = lane / 16, r = lane % 16;
    uint64_t left = drop_lanes(distinct_lanes(row_id, a.id_bits), first);
    int id[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) id[f] = __shfl(row_id, f * 16 + r);
    const int n = n0 + r < a.c_out ? n0 + r : a.c_out - 1;
    while (left) {
        int ad[kOnce], rank[kOnce], most = 0;
#pragma unroll
        for (int b = 0; b < kOnce; ++b) {
            ad[b] = left ? __builtin_amdgcn_readlane(row_id, __ffsll(static_cast<unsigned long long>(left)) - 1) : -1;
            rank[b] = ad[b] < 0 ? 0 : adapter_rank(a, ad[b]);
            most = rank[b] > most ? rank[b] : most;
            left = drop_lanes(left, of);
        }
        for (int k0 = 0; k0 < most; k0 += kStepRanks) {
            const int k = k0 + chunk_rank<T>(g);
            const u32x4 none = {0, 0, 0, 0};
            u32x4 rv[MF], uv[kOnce];
#pragma unroll
            for (int b = 0; b < kOnce; ++b)
                uv[b] = k < rank[b] ? *reinterpret_cast<const u32x4 *>(
                                          a.up + ((static_cast<int64_t>(ad[b]) * a.c_out + n) * a.max_rank + k) *
                                                     static_cast<int>(sizeof(T)))
                                    : none;
#pragma unroll
            for (int f = 0; f < MF; ++f)
                rv[f] = k < most && id[f] >= 0
                            ? *reinterpret_cast<const u32x4 *>(a.v + (row0 + f * 16 + r) * a.v_pitch + k0 * 4 + g * 16)
                            : none;
#pragma unroll
            for (int b = 0; b < kOnce; ++b) {
                u32x4 u = uv[b];
                if (rank[b] % (16 / static_cast<int>(sizeof(T))) != 0) u = used_part<T>(u, rank[b] - k);
                uint32_t odd = 0;
                if (chunk_rest<T>(g)) u = finite_part<T>(u, odd);  // the first halves have brought the rest
#pragma unroll
                for (int f = 0; f < MF; ++f) {
                    const floatx4 sum = chunk_mma<T>(u, k < rank[b] ? rv[f] : none, acc[0][f]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[0][f][e] = id[f] == ad[b] ? sum[e] : acc[0][f][e];
                }
            }
        }
    }
}

// more += what the infinities and NaN in up give for one row and N outputs from n.
template <typename T, int N>
__device__ __forceinline__ void odd_products(const RowsArgs &a, int64_t row, int64_t end, int n, float (&more)[N]) {
    const int key = adapter_key(a, row, row < end);
    if (key < 0) return;
    const T *up = reinterpret_cast<const T *>(a.up) +
                  (static_cast<int64_t>(key & (kMaxAdapters - 1)) * a.c_out + n) * a.max_rank;
    const T *v = reinterpret_cast<const T *>(a.v + row * a.v_pitch);
    for (int k = 0; k < key >> kAdapterBits; ++k) {
        const float by = static_cast<float>(v[sizeof(T) == 2 ? k / 8 * 16 + k % 8 : k]);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const float w = static_cast<float>(up[u * a.max_rank + k]);
            if (!(fabsf(w) < __builtin_huge_valf())) more[u] += w * by;
        }
    }
}

// ------------------------------------------------------------ loads to LDS
__device__ const u32x4 kZeroChunk[1] = {u32x4{0, 0, 0, 0}};

// 16 bytes a lane from global memory straight to LDS at `to` + OFF + 16 * lane.  As
// assembly, because the compiler otherwise waits for the loads in flight to
// the other buffer before each read of LDS; loads_barrier does all the waiting.
// The readfirstlanes sit in the operands: without optimisation, variables would
// come back from the stack as vector registers.
#define DC_UNIFORM(v) __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v))
template <int OFF>
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t to) {
    asm volatile("s_add_u32 m0, %0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(DC_UNIFORM(to)), "v"(from),
                 "n"(OFF)
                 : "scc", "m0");
}
#undef DC_UNIFORM

// f(0), f(1), .. f(N - 1) with compile-time numbers
template <int N, typename F>
__device__ __forceinline__ void unrolled(F f) {
    if constexpr (N > 0) {
        unrolled<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// This wave's loads to LDS but the newest N have landed / its reads of LDS are done.
template <int N>
__device__ __forceinline__ void own_loads() {
    static_assert(N < 64, "the counter has 6 bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void own_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Streams of a wave: NF tiles of 16 weight rows times MF tiles of 16 rows, steps
// of 128 bytes through a ring of D steps in LDS that belongs to the wave alone.
// The way through LDS is for the loads' sake: lanes side by side then cover a
// row's whole line, where the matrix cores' layout has them on 16 rows, four
// times the lines for the address unit (17 against 50 bytes a clock and CU, data
// in L2).  Chunk c of a row sits at c ^ row % 8.
constexpr int kStreamStep = 128;
template <int NF, int MF> constexpr int stream_slot() { return 2 * (NF + MF) * 1024; }
// ring steps of NW waves in KB of LDS, 2 to 4
template <int NW, int NF, int MF> constexpr int stream_depth(int kb) {
    const int d = kb * 1024 / (NW * stream_slot<NF, MF>());
    return d < 2 ? 2 : d > 4 ? 4 : d;
}

// The place of this lane in a load: row lane / 8 (and 8 more in the second load of
// a tile), 16-byte chunk stream_chunk() of the step.
__device__ __forceinline__ int stream_row() { return static_cast<int>(threadIdx.x) % kWave / 8; }
__device__ __forceinline__ int stream_chunk() { return static_cast<int>(threadIdx.x) % 8 ^ stream_row(); }

// rows[2 t], rows[2 t + 1]: this lane's rows of tile t (the weights' tiles first),
// at byte 0 of the contraction.
template <typename T, int NF, int MF, int D>
__device__ __forceinline__ void stream_products(const char *const (&rows)[2 * (NF + MF)], int s0, int s1, int64_t pitch,
                                                const char *ring, floatx4 (&acc)[NF][MF]) {
    constexpr int L = 2 * (NF + MF);
    const int lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
    const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char *)(ring)));
    const char *zero = reinterpret_cast<const char *>(kZeroChunk);
    auto load = [&](int step, int slot) {  // zeros past the run and past the row
        const int64_t off = static_cast<int64_t>(step) * kStreamStep + stream_chunk() * 16;
        const bool in = step < s1 && off < pitch;
        unrolled<L>([&](auto i) {
            constexpr int k = decltype(i)::value;
            load_to_lds<k * 1024>(in ? rows[k] + off : zero, at + slot * (L * 1024));
        });
    };
#pragma unroll
    for (int d = 0; d < D; ++d) load(s0 + d, d);
    int slot = 0;
    for (int s = s0; s < s1; ++s) {
        own_loads<(D - 1) * L>();
        u32x4 wv[2][NF], xv[2][MF];
        const char *from = ring + slot * (L * 1024) + r * kStreamStep;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const int chunk = ((kk * 4 + g) ^ (r & 7)) * 16;
#pragma unroll
            for (int i = 0; i < NF; ++i) wv[kk][i] = *reinterpret_cast<const u32x4 *>(from + i * 2048 + chunk);
#pragma unroll
            for (int f = 0; f < MF; ++f) xv[kk][f] = *reinterpret_cast<const u32x4 *>(from + (NF + f) * 2048 + chunk);
        }
        own_reads();
        load(s + D, slot);
        slot = slot + 1 == D ? 0 : slot + 1;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int f = 0; f < MF; ++f) acc[i][f] = chunk_mma<T>(wv[kk][i], xv[kk][f], acc[i][f]);
    }
    own_loads<0>();
}

// ------------------------------------------------------------- few rows
// Groups of a few rows: the time is that of reading the weights.  A workgroup takes
// MF * 16 rows of a group and NF tiles of 16 weight rows (gated: the value's and the
// gate's of 16 outputs); its NW waves split the contraction, stream it, and add up
// through LDS in wave order.  Up to 48 rows 80 KB of LDS leave two workgroups a CU,
// one's loads under way while the other adds up; 64 rows take 96 KB, and adapters 128
// to 160 KB: one workgroup a CU.  64 tokens with 8 of 64 experts, 2048 -> 2 x 1024
// gated, bf16: 537 MB in 98 us, 5.5 TB/s (a large copy: 5.1); the projection back,
// whose contraction is half as long, 268 MB in 65 us, 4.1 TB/s.  A step through one
// 4096 x 4096 projection with 48 rows and 32 adapters of rank 16: 14.8 us, 2.5 TB/s,
// two thirds of it the chain of one workgroup a CU.
template <typename T, typename OT, int NW, int NF, int MF, bool GATED, bool ADAPT>
__global__ void __launch_bounds__(NW * kWave)
k_rows_few(RowsArgs a, int slices) {
    static_assert(!GATED || NF == 2, "value and gate");
    constexpr int BM = MF * 16, kOuts = GATED ? 16 : NF * 16, kTiles = MF * (GATED ? 1 : NF);
    constexpr int D = stream_depth<NW, NF, MF>(ADAPT ? 160 : 80), kRing = D * stream_slot<NF, MF>();
    constexpr int kSums = NF * MF * 1024;  // a wave's, in fp32
    __shared__ __attribute__((aligned(1024))) char lds[NW * (kRing > kSums ? kRing : kSums)];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    RowTile t;
    if (!find_tile<BM>(a.starts, a.groups, a.rows, block_xy(), slices, t)) return;
    const int n0 = t.slice * kOuts;
    int row_id = -1;
    if constexpr (ADAPT) row_id = adapter_of(a, t.row0 + lane, lane < BM && t.row0 + lane < t.end);
    const char *rows[2 * (NF + MF)];
#pragma unroll
    for (int i = 0; i < 2 * NF; ++i) {
        const int n = n0 + (GATED ? 0 : i / 2 * 16) + i % 2 * 8 + stream_row();
        rows[i] = (GATED && i >= 2 ? a.w2 : a.w) +
                  (static_cast<int64_t>(t.group) * a.c_out + (n < a.c_out ? n : a.c_out - 1)) * a.pitch;
    }
#pragma unroll
    for (int f = 0; f < 2 * MF; ++f) {  // past the end the last row again: its lines are there
        const int64_t p = t.row0 + f * 8 + stream_row();
        const int64_t from = source_row(a, p < t.end ? p : t.end - 1);
        rows[2 * NF + f] = a.x + (from < 0 ? 0 : from) * a.pitch;
    }
    floatx4 acc[NF][MF];
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int f = 0; f < MF; ++f) acc[i][f] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = static_cast<int>((a.pitch + kStreamStep - 1) / kStreamStep);
    stream_products<T, NF, MF, D>(rows, steps * wave / NW, steps * (wave + 1) / NW, a.pitch, lds + wave * kRing, acc);
    if constexpr (ADAPT) add_adapters<T, MF>(a, row_id, t.row0, n0, wave, NW, acc);
    __syncthreads();  // the rings are done with
    floatx4 *part = reinterpret_cast<floatx4 *>(lds);  // [wave][i][f][lane]
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int f = 0; f < MF; ++f) part[((wave * NF + i) * MF + f) * kWave + lane] = acc[i][f];
    __syncthreads();
    // a wave for each tile: the rows f * 16 .. f * 16 + 15 of the outputs' tile i
    for (int k = wave; k < kTiles; k += NW) {
        const int f = k % MF, tile = k / MF;
        const int nn = n0 + tile * 16 + 4 * g;
        const int64_t p = t.row0 + f * 16 + r;
        if (nn >= a.c_out || p >= t.end || source_row(a, p) < 0) continue;
        const int64_t to = target_row(a, p);
        if (to < 0) continue;
        floatx4 sum = part[(tile * MF + f) * kWave + lane], sum2 = part[((NF - 1) * MF + f) * kWave + lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            sum += part[((w * NF + tile) * MF + f) * kWave + lane];
            if (GATED) sum2 += part[((w * NF + NF - 1) * MF + f) * kWave + lane];
        }
        float out[4];
        finish4<GATED>(a, t.group, nn, sum, sum2, out);
        if constexpr (sizeof(OT) == 2 && !ADAPT) {
            if (a.halves) {
                OT *row = reinterpret_cast<OT *>(a.y) + to * 2 * a.c_out + nn;
                store_out<OT>(row, out);
#pragma unroll
                for (int u = 0; u < 4; ++u) out[u] = rest_of<OT>(out[u]);
                store_out<OT>(row + a.c_out, out);
                continue;
            }
        }
        store_out<OT>(reinterpret_cast<OT *>(a.y) + to * a.c_out + nn, out);
    }
}

// ------------------------------------------------------------- many rows
// Tiles of BM rows x BN outputs through LDS, 64 bytes of the contraction a
// step, five steps of LDS: the loads run four steps ahead of the products.  A
// row's 4 chunks are stored at chunk ^ (row / 2 % 4), so 8 neighbouring rows at one chunk cover all banks; the loads go straight to
// LDS, which fixes a lane's place there, so the swizzle is applied to the
// address that each lane loads.  Gated: the outputs of a tile are 16 of the
// value's and 16 of the gate's in turn, so a wave holds both.
//
// 256 x 256 tiles run as two groups of four waves (one wave a SIMD each), half a
// step apart: while one group multiplies, the other reads its operands from LDS and
// issues its loads.  8192 x 4096 x 4096 bf16: 218 us, 1260 TFLOP/s (the library's
// product 183 us); with zeros for data 173 us, so the clock that the power allows
// bounds it, then some 8 us a tile for its first loads and its sums.  Smaller tiles
// leave the overlap to the several workgroups of a CU: 64 x 64 for 777 rows 1024 ->
// 2816, 16.2 us, bound by the chain of load, barrier and read of each step.  fp32
// takes four 16x16x4 products where 16-bit types take one 16x16x32: 1499 rows of 12
// groups, 264 -> 520, 16.0 us.
template <int BM, int BN>
struct TileCfg {
    static constexpr int kWavesM = 2, kWavesN = BN >= 256 ? 4 : 2;
    static constexpr int kWaves = kWavesM * kWavesN;
    static constexpr int kThreads = kWaves * kWave;
    static constexpr bool kTwo = kWaves == 8;
    static constexpr int kMF = BM / kWavesM / 16, kNF = BN / kWavesN / 16;
    static constexpr int kLoadsX = BM / 16 / kWaves, kLoadsW = BN / 16 / kWaves;  // of 16 rows, per wave and step
    static constexpr int kLoads = kLoadsX + kLoadsW;
    static constexpr int kSlots = 5, kAhead = kSlots - 1;  // steps in LDS, steps that the loads run ahead
    static constexpr int kSlot = (BM + BN) * 64;
    static constexpr int kWpe = kTwo ? 2 : BM >= 128 ? 2 : 4;  // waves a SIMD that the registers must allow
};

// All but the newest N of this wave's loads have landed, and its reads of LDS
// are done; then the barrier.
template <int N>
__device__ __forceinline__ void loads_barrier() {
    static_assert(N < 64, "the counter has 6 bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
template <typename T, typename OT, int BM, int BN, bool GATED, bool ADAPT>
__global__ void __launch_bounds__((TileCfg<BM, BN>::kThreads))
__attribute__((amdgpu_waves_per_eu(TileCfg<BM, BN>::kWpe, TileCfg<BM, BN>::kWpe)))
k_rows_tile(RowsArgs a, int slices) {
    typedef TileCfg<BM, BN> C;
    constexpr int MF = C::kMF, NF = C::kNF;
    __shared__ __attribute__((aligned(1024))) char lds[C::kSlots * C::kSlot];
    const uint32_t lds0 = static_cast<uint32_t>(
        reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)(lds)));
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    RowTile t;
    if (!find_tile<BM>(a.starts, a.groups, a.rows, block_xy(), slices, t)) return;
    constexpr int kOuts = GATED ? BN / 2 : BN;  // outputs of a tile
    const int n0 = t.slice * kOuts;

    // this lane's next chunks: row 16 i + lane / 4 of the tile, place lane % 4;
    // the rows that go in first, then the weights
    const int lrow = lane / 4, lchunk = (lane % 4) ^ (lrow / 2 % 4);
    const char *next[C::kLoads];
#pragma unroll
    for (int i = 0; i < C::kLoadsX; ++i) {
        const int64_t p = t.row0 + (wave * C::kLoadsX + i) * 16 + lrow;
        const int64_t s = p < t.end ? source_row(a, p) : -1;
        next[i] = a.x + (s < 0 ? 0 : s) * a.pitch + lchunk * 16;
    }
#pragma unroll
    for (int i = 0; i < C::kLoadsW; ++i) {
        const int j = wave * C::kLoadsW + i;  // 16 rows of the weights' tile
        const int n = n0 + (GATED ? j / 2 : j) * 16 + lrow;
        next[C::kLoadsX + i] = (GATED && j % 2 ? a.w2 : a.w) +
                               (static_cast<int64_t>(t.group) * a.c_out + (n < a.c_out ? n : a.c_out - 1)) * a.pitch +
                               lchunk * 16;
    }
    const int own_steps = static_cast<int>((a.pitch + 63) / 64);
    int steps = own_steps, left = static_cast<int>(a.pitch) - lchunk * 16;  // bytes of the row from this lane's chunk on
    const uint32_t xl = lds0 + wave * C::kLoadsX * 1024, wl = lds0 + BM * 64 + wave * C::kLoadsW * 1024;
    const char *zero = reinterpret_cast<const char *>(kZeroChunk);
    // The adapters: each distinct one of the tile's rows is more steps of the
    // contraction, v against up, with the other adapters' rows at zero.  The rows' ids
    // and ranks are read once, here: a read among the steps would wait for the loads
    // that run ahead as well (777 rows of 48 requests in any order: 82 against 95 us).
    int keys[BM / kWave];
    AdapterWalk<BM> ahead, now;  // at the step whose loads are next, at the one that is multiplied
    const int my_rows = wave * C::kLoadsX / 4;  // the 64 rows that this wave's loads belong to
    if constexpr (ADAPT) {
#pragma unroll
        for (int i = 0; i < BM / kWave; ++i) {
            const int64_t p = t.row0 + i * kWave + lane;
            keys[i] = adapter_key(a, p, p < t.end);
        }
        ahead.start(keys);
        while (ahead.next(keys, 0)) steps += (ahead.rank + kStepRanks - 1) / kStepRanks;
        ahead.start(keys);
        now.start(keys);
    }
    // Where the loads of step `step` come from; past the last step zeros.  The
    // steps are taken in order.  own: a step of the rows' own contraction.
    const char *from[C::kLoads];
    auto sources = [&](int step, auto own) {
#pragma unroll
        for (int i = 0; i < C::kLoads; ++i) {
            from[i] = left > 0 ? next[i] : zero;
            next[i] += 64;
        }
        left -= 64;
        if constexpr (ADAPT && !decltype(own)::value) {
            if (step >= own_steps && step < steps) {
                if (ahead.k0 >= ahead.rank) ahead.next(keys, my_rows);
                const int k = ahead.k0 + chunk_rank<T>(lchunk);
                const T *up =
                    reinterpret_cast<const T *>(a.up) + static_cast<int64_t>(ahead.id) * a.c_out * a.max_rank + k;
#pragma unroll
                for (int i = 0; i < C::kLoadsX; ++i) {
                    const int row = (wave * C::kLoadsX + i) * 16 + lrow;
                    const bool in = k < ahead.rank && (ahead.own >> row % kWave & 1) != 0;
                    from[i] = in ? a.v + (t.row0 + row) * a.v_pitch + ahead.k0 * 4 + lchunk * 16 : zero;
                }
#pragma unroll
                for (int i = 0; i < C::kLoadsW; ++i) {
                    int n = n0 + (wave * C::kLoadsW + i) * 16 + lrow;
                    n = n < a.c_out ? n : a.c_out - 1;
                    from[C::kLoadsX + i] = k < ahead.rank
                                               ? reinterpret_cast<const char *>(up + static_cast<int64_t>(n) * a.max_rank)
                                               : zero;
                }
                ahead.k0 += kStepRanks;
            }
        }
    };
    uint32_t to = 0, at = 0;  // the slots that are loaded and read next
    auto after = [](uint32_t slot) { return slot == (C::kSlots - 1) * C::kSlot ? 0u : slot + C::kSlot; };
    auto load = [&](auto which) {  // one of a step's loads
        constexpr int i = decltype(which)::value;
        if constexpr (i < C::kLoadsX) load_to_lds<i * 1024>(from[i], xl + to);
        else load_to_lds<(i - C::kLoadsX) * 1024>(from[i], wl + to);
    };
    auto load_all = [&](int step, auto own) {
        sources(step, own);
        unrolled<C::kLoads>(load);
        to = after(to);
    };

    const int wm = wave % C::kWavesM * (BM / C::kWavesM), wn = wave / C::kWavesM * (BN / C::kWavesN);
    floatx4 acc[NF][MF];
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int f = 0; f < MF; ++f) acc[i][f] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    const int chunk = (g ^ (r / 2 % 4)) * 16;
    const char *xr = lds + (wm + r) * 64 + chunk, *wr = lds + (BM + wn + r) * 64 + chunk;
    u32x4 xv[MF], wv[NF];
    auto read = [&]() {
#pragma unroll
        for (int i = 0; i < NF; ++i) wv[i] = *reinterpret_cast<const u32x4 *>(wr + at + i * 1024);
#pragma unroll
        for (int f = 0; f < MF; ++f) xv[f] = *reinterpret_cast<const u32x4 *>(xr + at + f * 1024);
        at = after(at);
    };
    auto multiply = [&](auto at) {  // one tile of 16 outputs
        constexpr int i = decltype(at)::value;
#pragma unroll
        for (int f = 0; f < MF; ++f) acc[i][f] = chunk_mma<T>(wv[i], xv[f], acc[i][f]);
    };
    unrolled<C::kAhead>([&](auto step) { load_all(decltype(step)::value, std::false_type()); });
    // where the wave's rows go: lane l has rows l, l + 64, .. of them
    constexpr int kTargets = (MF * 16 + kWave - 1) / kWave;
    int target[kTargets];
#pragma unroll
    for (int i = 0; i < kTargets; ++i) {
        const int64_t p = t.row0 + wm + i * kWave + lane;
        const bool have = i * kWave + lane < MF * 16 && p < t.end;
        target[i] = have && source_row(a, p) >= 0 ? static_cast<int>(target_row(a, p)) : -1;
    }
    const bool second = C::kTwo && wave >= C::kWaves / 2;
    if constexpr (C::kTwo) {
        loads_barrier<(C::kAhead - 1) * C::kLoads>();
        if (second) __builtin_amdgcn_s_barrier();
        sources(C::kAhead, std::false_type());
    }
    // A step of an adapter: its own rows' v, and zeros for the others.  Zeros would not
    // keep an infinity or NaN in up from the others, so those entries are taken out
    // here, and odd_products adds what they are to their own rows.
    uint32_t odd = 0;
    auto adapter_products = [&]() {
        if (now.k0 >= now.rank) now.next(keys, 0);
        const int left = now.rank - now.k0;
        now.k0 += kStepRanks;
        if (left < kStepRanks)
#pragma unroll
            for (int i = 0; i < NF; ++i) wv[i] = used_part<T>(wv[i], left - chunk_rank<T>(g));
#pragma unroll
        for (int i = 0; i < NF; ++i) wv[i] = finite_part<T>(wv[i], odd);
        unrolled<NF>(multiply);
    };
    auto run = [&](int s0, int s1, auto own, auto products) {
        for (int s = s0; s < s1; ++s) {
            if constexpr (C::kTwo) {
                // Reading, and the loads of step s + kAhead, into the slot of step
                // s - 1, which both groups have read.  (Among the products the loads
                // hold up: a wave that waits for its turn to load cannot multiply.)
                read();
                unrolled<C::kLoads>(load);
                to = after(to);
                __builtin_amdgcn_sched_barrier(0);
                loads_barrier<(C::kAhead - 1) * C::kLoads>();  // step s + 1 has landed
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(1);
                sources(s + 1 + C::kAhead, own);
                products();
                __builtin_amdgcn_s_setprio(0);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
            } else {
                loads_barrier<(C::kAhead - 1) * C::kLoads>();  // step s has landed, step s - 1 is read
                load_all(s + C::kAhead, own);
                read();
                products();
            }
        }
    };
    auto own_products = [&]() { unrolled<NF>(multiply); };
    if constexpr (ADAPT) {
        // a loop without a choice of sources for as long as the loads are the rows' own
        // (8192 rows of 8 adapters, 4096 x 4096: 250 us against 269 with a choice in each step)
        const int plain = own_steps - (C::kTwo ? 1 : 0) - C::kAhead;
        run(0, plain, std::true_type(), own_products);
        run(plain < 0 ? 0 : plain, own_steps, std::false_type(), own_products);
        run(own_steps, steps, std::false_type(), adapter_products);
    } else {
        run(0, steps, std::true_type(), own_products);
    }
    if constexpr (C::kTwo)
        if (!second) __builtin_amdgcn_s_barrier();
    loads_barrier<0>();  // LDS is free: each wave takes its share for its sums

    // The sums go through LDS in fp32 (16-byte chunk c of a row at c ^ row % 16),
    // so that a lane finishes 16 bytes of one row and a store covers whole lines,
    // in a loop that is short code: every workgroup runs it once.
    constexpr int kCols = NF * 16, kRowBytes = kCols * 4, kChunks = kCols / 4;
    constexpr int kShare = C::kSlots * C::kSlot / C::kWaves;
    constexpr int kRows = MF * 16 < 64 ? MF * 16 : 64;  // of a pass
    static_assert(kRows * kRowBytes <= kShare && MF * 16 % kRows == 0, "a pass fits the wave's share");
    constexpr int kPerLane = 16 / static_cast<int>(sizeof(OT)), kOut = GATED ? kCols / 2 : kCols;
    constexpr int kLanes = kOut / kPerLane, kAtOnce = kWave / kLanes;  // lanes of a row, rows of a store
    char *mine = lds + wave * kShare;
    const int col = lane % kLanes * kPerLane, n = n0 + (GATED ? wn / 2 : wn) + col;
    const int c0 = ((GATED ? col / 16 * 32 + col % 16 : col)) / 4;
    const bool in = n < a.c_out;
    const bool any_odd = ADAPT && __ballot(odd != 0) != 0;
    float bias[kPerLane], bias2[kPerLane];
#pragma unroll
    for (int u = 0; u < kPerLane; u += 4) {
#pragma unroll
        for (int v = 0; v < 4; ++v) bias[u + v] = bias2[u + v] = 0.0f;
        const int64_t at = static_cast<int64_t>(t.group) * a.c_out + n + u;
        if (in && a.b) io<float>::load4(a.b + at, bias + u);
        if (GATED && in && a.b2) io<float>::load4(a.b2 + at, bias2 + u);
    }
    unrolled<MF * 16 / kRows>([&](auto pass) {
        constexpr int f0 = decltype(pass)::value * (kRows / 16);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int f = 0; f < kRows / 16; ++f)
#pragma unroll
            for (int i = 0; i < NF; ++i)
                *reinterpret_cast<floatx4 *>(mine + (f * 16 + r) * kRowBytes +
                                             ((i * 4 + g) ^ (r & (kChunks - 1))) * 16) = acc[i][f0 + f];
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int row = lane / kLanes; row < kRows; row += kAtOnce) {
            const int to = __shfl(target[f0 * 16 / kWave], (f0 * 16 + row) % kWave);
            const char *from_row = mine + row * kRowBytes;
            float out[kPerLane], more[kPerLane];
#pragma unroll
            for (int u = 0; u < kPerLane; ++u) more[u] = 0.0f;
            if constexpr (ADAPT)
                if (any_odd && in) odd_products<T, kPerLane>(a, t.row0 + wm + f0 * 16 + row, t.end, n, more);
#pragma unroll
            for (int u = 0; u < kPerLane; u += 4) {
                const int c = c0 + u / 4;
                const floatx4 v = *reinterpret_cast<const floatx4 *>(from_row + (c ^ (row & 15 & (kChunks - 1))) * 16);
                floatx4 w = v;
                if (GATED)
                    w = *reinterpret_cast<const floatx4 *>(from_row + ((c + 4) ^ (row & 15 & (kChunks - 1))) * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    out[u + e] = GATED   ? act_any(w[e] + bias2[u + e], a.act) * (v[e] + bias[u + e])
                                 : ADAPT ? act_any(v[e] + more[u + e] + bias[u + e], a.act)
                                         : act_any(v[e] + bias[u + e], a.act);
            }
            if (to >= 0 && in) {
                OT *y = reinterpret_cast<OT *>(a.y) + static_cast<int64_t>(to) * a.c_out + n;
                if constexpr (sizeof(OT) == 2) store8<OT>(y, out);
                else io<OT>::store4(y, out);
            }
        }
    });
}

// ------------------------------------------------------- sums of a token
// y[t] = (x[t]) + sum over slots of weight * o[t * k + slot], in slot order, fp32;
// slots without an expert do not count.  o is fp32: rounding it to 16 bits would save
// half of the traffic and add a rounding as large as the result's own to each term.
// Bound by memory: 8192 tokens of 2048, top 4, 50 us for 302 MB, 6 TB/s.
template <typename T>
__global__ void __launch_bounds__(kBlock)
k_combine(const float *__restrict__ o, const int32_t *__restrict__ expert, const float *__restrict__ weight,
          const T *x, T *y, int64_t tokens, int C, int top_k, int experts) {
    const int per = C / 8;
    const int64_t i = static_cast<int64_t>(block_xy()) * kBlock + threadIdx.x;
    if (i >= tokens * per) return;
    const int64_t t = i / per;
    const int c = static_cast<int>(i - t * per) * 8;
    float sum[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) sum[u] = 0.0f;
    for (int s0 = 0; s0 < top_k; s0 += 4) {
        float v[4][8], w[4];
        int e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // past the last slot: the last again, not counted
            const int64_t at = t * top_k + (s0 + j < top_k ? s0 + j : top_k - 1);
            e[j] = s0 + j < top_k ? expert[at] : -1;
            w[j] = weight[at];
            io<float>::load8(o + at * C + c, v[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int u = 0; u < 8; ++u)
                sum[u] = e[j] >= 0 && e[j] < experts ? __builtin_fmaf(w[j], v[j][u], sum[u]) : sum[u];
    }
    if (x) {
        float v[8];
        io<T>::load8(x + t * C + c, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum[u] += v[u];
    }
    io<T>::store4(y + t * C + c, sum);
    io<T>::store4(y + t * C + c + 4, sum + 4);
}

// --------------------------------------------- the second product of few tokens
// y[t] = (x[t]) + sum over slots of weight * (W_e h[t * k + slot] + b_e), e the
// slot's expert, in one launch: for calls of so few tokens that hardly two take
// the same expert, so that nothing is lost by reading the weights for each.  A
// workgroup takes one token and 16 outputs; a wave takes every NW-th slot and
// streams its expert's rows, or with fewer slots than waves several waves a part of
// the contraction each.  Slots and parts are added in their order, in fp32.
//
// Of the 16 rows of a matrix instruction one is needed.  In 16-bit types h comes as
// two halves (its rounding, and what that left) on rows 0 and 8, so h keeps twice the
// storage type's bits for some 0.5 us: the result's own rounding is what remains,
// where a rounded h adds an error as large (few outputs: 1.5 times the error).  One
// token, 8 slots, 1024 -> 2048 bf16: 33.5 MB in 12.0 us, 2.8 TB/s, on 128 workgroups,
// one for every other CU, against 13.5 for the grouped product and the sum; two
// tokens with 8 of 64 experts, whole layer, 44.8 against 49.0.
template <typename T, int NW>
__global__ void __launch_bounds__(NW * kWave)
k_project_tokens(const char *__restrict__ h, int64_t pitch, const int32_t *__restrict__ expert,
                 const float *__restrict__ weight, int top_k, int experts, const char *__restrict__ w,
                 const float *__restrict__ b, const T *x, T *y, int c_out, int slices) {
    constexpr int D = stream_depth<NW, 1, 1>(160), kRing = D * stream_slot<1, 1>();
    __shared__ __attribute__((aligned(1024))) char lds[NW * kRing];
    __shared__ floatx4 part[kMaxTopK > NW ? kMaxTopK : NW][4];  // [slot][part of the contraction][16 outputs]
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t t = blockIdx.x / static_cast<unsigned>(slices);
    const int n0 = static_cast<int>(blockIdx.x % static_cast<unsigned>(slices)) * 16;
    const int steps = static_cast<int>((pitch + kStreamStep - 1) / kStreamStep);
    const int parts = top_k < NW ? NW / top_k : 1, mine = wave % parts;
    constexpr bool kHalves = sizeof(T) == 2;
    for (int s = wave / parts; s < top_k; s += NW) {
        const int e = __builtin_amdgcn_readfirstlane(expert[t * top_k + s]);
        if (e < 0 || e >= experts) continue;
        const char *rows[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int n = n0 + i * 8 + stream_row();
            rows[i] = w + (static_cast<int64_t>(e) * c_out + (n < c_out ? n : c_out - 1)) * pitch;
            rows[2 + i] = h + ((t * top_k + s) * (kHalves ? 2 : 1) + (kHalves ? i : 0)) * pitch;  // rows 0-7, 8-15
        }
        floatx4 acc[1][1] = {{floatx4{0.0f, 0.0f, 0.0f, 0.0f}}};
        stream_products<T, 1, 1, D>(rows, steps * mine / parts, steps * (mine + 1) / parts, pitch, lds + wave * kRing, acc);
        floatx4 v = acc[0][0];
        if constexpr (kHalves) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float rest = __shfl_xor(v[u], 8);
                v[u] = fabsf(v[u]) < __builtin_huge_valf() ? v[u] + rest : v[u];  // infinite weights: the first half says it
            }
        }
        if (lane % 16 == 0) part[s * parts + mine][lane / 16] = v;
    }
    __syncthreads();
    const int n = n0 + 4 * static_cast<int>(threadIdx.x);
    if (threadIdx.x >= 4 || n >= c_out) return;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < top_k; ++s) {
        const int e = expert[t * top_k + s];
        if (e < 0 || e >= experts) continue;
        const float k = weight[t * top_k + s];
        float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (b) io<float>::load4(b + static_cast<int64_t>(e) * c_out + n, bias);
        floatx4 v = part[s * parts][threadIdx.x];
        for (int i = 1; i < parts; ++i) v += part[s * parts + i][threadIdx.x];
#pragma unroll
        for (int u = 0; u < 4; ++u) sum[u] = __builtin_fmaf(k, v[u] + bias[u], sum[u]);
    }
    if (x) {
        float v[4];
        io<T>::load4(x + t * c_out + n, v);
#pragma unroll
        for (int u = 0; u < 4; ++u) sum[u] += v[u];
    }
    io<T>::store4(y + t * c_out + n, sum);
}

// ------------------------------------------------ an adapter's first half
// v[row] = scale * A_id x[row] as add_adapters takes it (16-bit types: in two
// halves), for 16 rows a workgroup: one distinct adapter of the rows at a time, every
// gridDim.z-th from blockIdx.z, NF tiles of 16 of its rows.  The waves split the
// contraction, stream it, and add up through LDS in wave order.  8192 rows of 4096
// bf16, rank 32: 67 MB in 29 us, 2.3 TB/s (an adapter's rows come from L2 for each 16
// rows, four times as much); 32 rows a workgroup were no faster (rank 16 45.1 against
// 41.4 us with the product after it, rank 64 43.3 against 46.7).  48 rows with 32
// adapters: 6.7 us, the chain of one workgroup (48 workgroups, one for each adapter
// that 16 rows can have: most CUs have none).
constexpr int kDownWaves = 8;

template <typename T, int NF>
__global__ void __launch_bounds__(kDownWaves * kWave)
k_adapter_down(const char *__restrict__ x, int64_t rows, int64_t pitch, const char *__restrict__ down,
               const int32_t *__restrict__ ids, const int32_t *__restrict__ ranks, const float *__restrict__ scales,
               int adapters, int id_bits, int max_rank, char *__restrict__ v, int v_pitch) {
    constexpr int NW = kDownWaves, D = stream_depth<NW, NF, 1>(160), kRing = D * stream_slot<NF, 1>();
    static_assert(kRing >= NF * 1024, "a wave's sums fit its ring");
    __shared__ __attribute__((aligned(1024))) char lds[NW * kRing];
    floatx4 *part = reinterpret_cast<floatx4 *>(lds);  // [wave][i][lane]
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int64_t row0 = static_cast<int64_t>(block_xy()) * 16;
    int row_id = lane < 16 && row0 + lane < rows ? ids[row0 + lane] : -1;
    row_id = row_id >= 0 && row_id < adapters ? row_id : -1;
    const char *from[2 * (NF + 1)];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        const int64_t row = row0 + f * 8 + stream_row();
        from[2 * NF + f] = x + (row < rows ? row : rows - 1) * pitch;
    }
    const int steps = static_cast<int>((pitch + kStreamStep - 1) / kStreamStep);
    uint64_t left = drop_lanes(distinct_lanes(row_id, id_bits), static_cast<int>(blockIdx.z));
    while (left) {
        const int ad = __builtin_amdgcn_readlane(row_id, __ffsll(static_cast<unsigned long long>(left)) - 1);
        left = drop_lanes(left, static_cast<int>(gridDim.z));
        int rank = ranks ? ranks[ad] : max_rank;
        rank = rank < max_rank ? rank : max_rank;
        const float scale = scales ? scales[ad] : 1.0f;
        const char *base = down + static_cast<int64_t>(ad) * max_rank * pitch;
        for (int n0 = 0; n0 < rank; n0 += NF * 16) {
#pragma unroll
            for (int i = 0; i < 2 * NF; ++i) {
                const int n = n0 + i * 8 + stream_row();
                from[i] = base + static_cast<int64_t>(n < rank ? n : rank - 1) * pitch;
            }
            floatx4 acc[NF][1];
#pragma unroll
            for (int i = 0; i < NF; ++i) acc[i][0] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            stream_products<T, NF, 1, D>(from, steps * wave / NW, steps * (wave + 1) / NW, pitch, lds + wave * kRing, acc);
            __syncthreads();  // the rings are done with
#pragma unroll
            for (int i = 0; i < NF; ++i) part[(wave * NF + i) * kWave + lane] = acc[i][0];
            __syncthreads();
            if (wave < NF) {  // a wave for each tile of the result
                const int n = n0 + wave * 16 + 4 * g;
                floatx4 sum = part[wave * kWave + lane];
#pragma unroll
                for (int w = 1; w < NW; ++w) sum += part[(w * NF + wave) * kWave + lane];
                if (__shfl(row_id, r) == ad && n < max_rank) {
                    float out[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) out[u] = n + u < rank ? scale * sum[u] : 0.0f;
                    if constexpr (sizeof(T) == 2) {  // chunk n / 8 of the first halves, and of the second
                        T *to = reinterpret_cast<T *>(v + (row0 + r) * v_pitch) + n / 8 * 16 + n % 8;
                        io<T>::store4(to, out);
#pragma unroll
                        for (int u = 0; u < 4; ++u) out[u] = rest_of<T>(out[u]);
                        io<T>::store4(to + 8, out);
                    } else {
                        io<T>::store4(reinterpret_cast<T *>(v + (row0 + r) * v_pitch) + n, out);
                    }
                }
            }
            __syncthreads();
        }
    }
}

}  // namespace dynconv
