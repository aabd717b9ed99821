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

#include "kernels.h"

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
// blocks' clamp is a median of three, which drops it).
__device__ __forceinline__ float act_any(float v, int kind) {
    if (kind == 0) return v;
    if (kind <= 2) {
        const float low = v < 0.0f ? 0.0f : v;
        return kind == 2 && low > 6.0f ? 6.0f : low;
    }
    if (kind == 3) return v / (1.0f + __expf(-v));
    return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
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
    // low-rank adapters: y += up[ids[row]] * v[row]
    const char *v;         // [rows][v_pitch bytes]
    int v_pitch;
    const char *up;        // [adapters][c_out][max_rank]
    const int32_t *ids, *ranks;
    int adapters, max_rank;
};

// ---------------------------------------------------------------- tiles
// Tile `tile` of the groups' rows in tiles of BM: its group and rows, false
// past the last tile.  Every wave works it out by itself, 64 groups a step.
struct RowTile {
    int group;
    int64_t row0, end;
};

__device__ __forceinline__ int64_t clamp_row(int64_t v, int64_t rows) { return v < 0 ? 0 : v > rows ? rows : v; }

template <int BM>
__device__ __forceinline__ bool find_tile(const int32_t *__restrict__ starts, int groups, int64_t rows, int tile,
                                          RowTile &t) {
    if (!starts) {
        t.group = 0;
        t.row0 = static_cast<int64_t>(tile) * BM;
        t.end = rows;
        return t.row0 < rows;
    }
    const int lane = threadIdx.x % kWave;
    int before = 0;
    for (int g0 = 0; g0 < groups; g0 += kWave) {
        const int g = g0 + lane;
        int64_t lo = 0, hi = 0;
        if (g < groups) {
            lo = clamp_row(starts[g], rows);
            hi = clamp_row(starts[g + 1], rows);
        }
        const int n = hi > lo ? static_cast<int>((hi - lo + BM - 1) / BM) : 0;
        int incl = n;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int o = __shfl_up(incl, d);
            if (lane >= d) incl += o;
        }
        const uint64_t past = __ballot(before + incl > tile);
        if (past) {
            const int l = __ffsll(static_cast<unsigned long long>(past)) - 1;
            t.group = g0 + l;
            const int lo32 = __builtin_amdgcn_readlane(static_cast<int>(lo), l);
            const int hi32 = __builtin_amdgcn_readlane(static_cast<int>(hi), l);
            const int first = before + __builtin_amdgcn_readlane(incl - n, l);
            t.row0 = static_cast<int64_t>(lo32) + static_cast<int64_t>(tile - first) * BM;
            t.end = hi32;
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

// acc += up[id] * v over the distinct adapters of the wave's rows (MF tiles of
// 16 from row0; id[f]: the adapter of row f * 16 + lane % 16, or -1) and NF
// tiles of 16 outputs from n0.  Each adapter is one more run of the
// contraction, with the rows of the others at zero.  Only every `of`-th
// adapter from `first` is taken (waves that split the work).
template <typename T, int NF, int MF>
__device__ __forceinline__ void add_adapters(const RowsArgs &a, const int (&id)[MF], int64_t row0, int n0, int first,
                                             int of, floatx4 (&acc)[NF][MF]) {
    const int lane = threadIdx.x % kWave, g = lane / 16, r = lane % 16;
    constexpr int kPer = 16 / static_cast<int>(sizeof(T));
    const char *v = a.v + row0 * a.v_pitch;
    bool open[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) open[f] = id[f] >= 0;
    for (int turn = 0;; ++turn) {
        int ad = -1;
#pragma unroll
        for (int f = MF - 1; f >= 0; --f) {
            const uint64_t left = __ballot(open[f]);
            if (left) ad = __builtin_amdgcn_readlane(id[f], __ffsll(static_cast<unsigned long long>(left)) - 1);
        }
        if (ad < 0) break;
#pragma unroll
        for (int f = 0; f < MF; ++f) open[f] = open[f] && id[f] != ad;
        if (turn % of != first) continue;
        const int rank = adapter_rank(a, ad);
        const T *up = reinterpret_cast<const T *>(a.up) + static_cast<int64_t>(ad) * a.c_out * a.max_rank;
        for (int k0 = 0; k0 < rank; k0 += 4 * kPer) {
            const int k = k0 + g * kPer;
            u32x4 rv[MF], uv[NF];
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                rv[f] = u32x4{0, 0, 0, 0};
                if (id[f] == ad && k < rank)
                    rv[f] = *reinterpret_cast<const u32x4 *>(v + (f * 16 + r) * a.v_pitch + k * static_cast<int>(sizeof(T)));
            }
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                uv[i] = u32x4{0, 0, 0, 0};
                const int n = n0 + i * 16 + r;
                if (k < rank && n < a.c_out)
                    uv[i] = *reinterpret_cast<const u32x4 *>(up + static_cast<int64_t>(n) * a.max_rank + k);
            }
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int f = 0; f < MF; ++f) acc[i][f] = chunk_mma<T>(uv[i], rv[f], acc[i][f]);
        }
    }
}

// ------------------------------------------------------------- few rows
// Groups of a few rows: the time is that of reading the weights.  A workgroup
// takes MF * 16 rows of a group and 16 outputs; its NW waves split the
// contraction, stream the weights straight into the matrix cores' registers,
// and add up through LDS in wave order.
template <typename T, typename OT, int NW, int MF, bool GATED, bool ADAPT>
__global__ void __launch_bounds__(NW * kWave)
k_rows_few(RowsArgs a, int slices) {
    constexpr int BM = MF * 16, NF = GATED ? 2 : 1;
    __shared__ floatx4 part[NW > 1 ? NW - 1 : 1][NF][MF][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int r = lane % 16, g = lane / 16;
    const int id = block_xy();
    RowTile t;
    if (!find_tile<BM>(a.starts, a.groups, a.rows, id / slices, t)) return;
    const int n0 = id % slices * 16;
    const int n = n0 + r < a.c_out ? n0 + r : a.c_out - 1;
    const int64_t woff = (static_cast<int64_t>(t.group) * a.c_out + n) * a.pitch;
    const char *wp[NF];
    wp[0] = a.w + woff;
    if constexpr (GATED) wp[1] = a.w2 + woff;
    const char *xp[MF];
    int64_t from[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int64_t p = t.row0 + f * 16 + r;
        from[f] = p < t.end ? source_row(a, p) : -1;
        xp[f] = a.x + (from[f] < 0 ? 0 : from[f]) * a.pitch;
    }
    floatx4 acc[NF][MF];
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int f = 0; f < MF; ++f) acc[i][f] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    // the waves' runs of the contraction, in steps of 64 bytes
    const int64_t steps = (a.pitch + 63) / 64;
    const int64_t s0 = steps * wave / NW, s1 = steps * (wave + 1) / NW;
    constexpr int U = MF == 1 ? 8 : 4;  // steps in flight
    int64_t s = s0;
    for (; s + U <= s1 && (s + U) * 64 <= a.pitch; s += U) {
        u32x4 wv[U][NF], xv[U][MF];
        const int64_t off = s * 64 + g * 16;
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < NF; ++i) wv[u][i] = *reinterpret_cast<const u32x4 *>(wp[i] + off + u * 64);
#pragma unroll
            for (int f = 0; f < MF; ++f) xv[u][f] = *reinterpret_cast<const u32x4 *>(xp[f] + off + u * 64);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int f = 0; f < MF; ++f) acc[i][f] = chunk_mma<T>(wv[u][i], xv[u][f], acc[i][f]);
    }
    for (; s < s1; ++s) {
        const int64_t off = s * 64 + g * 16;
        const bool in = off < a.pitch;
        u32x4 wv[NF], xv[MF];
#pragma unroll
        for (int i = 0; i < NF; ++i)
            wv[i] = in ? *reinterpret_cast<const u32x4 *>(wp[i] + off) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int f = 0; f < MF; ++f)
            xv[f] = in ? *reinterpret_cast<const u32x4 *>(xp[f] + off) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
            for (int f = 0; f < MF; ++f) acc[i][f] = chunk_mma<T>(wv[i], xv[f], acc[i][f]);
    }
    if constexpr (ADAPT) {
        int ids[MF];
#pragma unroll
        for (int f = 0; f < MF; ++f) ids[f] = adapter_of(a, t.row0 + f * 16 + r, t.row0 + f * 16 + r < t.end);
        add_adapters<T, 1, MF>(a, ids, t.row0, n0, wave, NW, acc);
    }
    if (NW > 1) {
        if (wave > 0) {
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int f = 0; f < MF; ++f) part[wave - 1][i][f][lane] = acc[i][f];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < NW - 1; ++w)
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int f = 0; f < MF; ++f) acc[i][f] += part[w][i][f][lane];
    }
    const int nn = n0 + 4 * g;
    if (nn >= a.c_out) return;
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        if (from[f] < 0) continue;
        const int64_t to = target_row(a, t.row0 + f * 16 + r);
        if (to < 0) continue;
        float out[4];
        finish4<GATED>(a, t.group, nn, acc[0][f], acc[NF - 1][f], out);
        store_out<OT>(reinterpret_cast<OT *>(a.y) + to * a.c_out + nn, out);
    }
}

// ------------------------------------------------------------- many rows
// Tiles of BM rows x BN outputs through LDS, 128 bytes of the contraction a
// step.  A row's 8 chunks are stored at chunk ^ (row % 8), so the 16 rows that
// a wave reads at one chunk spread over all banks; the loads go straight to
// LDS, which fixes a lane's place there, so the swizzle is applied to the
// address that each lane loads.  Two buffers: a step's loads are in flight
// while the step before is multiplied.  Gated: the outputs of a tile are 16 of
// the value's and 16 of the gate's in turn, so a wave holds both.
__device__ const u32x4 kZeroChunk[1] = {u32x4{0, 0, 0, 0}};

template <int BM, int BN>
struct TileCfg {
    static constexpr int kWavesM = 2, kWavesN = BN / 64;
    static constexpr int kWaves = kWavesM * kWavesN;
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int kMF = BM / kWavesM / 16, kNF = BN / kWavesN / 16;
    static constexpr int kLoadsX = BM / 8 / kWaves, kLoadsW = BN / 8 / kWaves;  // of 8 rows, per wave and step
    static constexpr int kBuffer = (BM + BN) * 128;
};

// 16 bytes a lane from global memory straight to LDS at `to` + 16 * lane.  As
// assembly, because the compiler otherwise waits for the loads in flight to
// the other buffer before each read of LDS; loads_barrier does all the waiting.
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from));
}
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base));
}

// Every wave's loads to LDS have landed (they count as vector memory) and its
// reads of LDS are done.
__device__ __forceinline__ void loads_barrier() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// No load to LDS may be under way when a workgroup ends and gives its LDS back.
__device__ __forceinline__ void loads_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <typename P>
__device__ __forceinline__ P uniform_ptr(P p) {
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
    return reinterpret_cast<P>((static_cast<uint64_t>(hi) << 32) | lo);
}

template <typename T, typename OT, int BM, int BN, bool GATED, bool ADAPT>
__global__ void __launch_bounds__((TileCfg<BM, BN>::kThreads)) __attribute__((amdgpu_waves_per_eu(2, 2)))
k_rows_tile(RowsArgs a, int slices) {
    typedef TileCfg<BM, BN> C;
    constexpr int MF = C::kMF, NF = C::kNF;
    __shared__ __attribute__((aligned(1024))) char lds[2 * C::kBuffer];
    const uint32_t lds0 = static_cast<uint32_t>(
        reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)(lds)));
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int id = block_xy();
    RowTile t;
    if (!find_tile<BM>(a.starts, a.groups, a.rows, id / slices, t)) return;
    constexpr int kOuts = GATED ? BN / 2 : BN;  // outputs of a tile
    const int n0 = id % slices * kOuts;

    // this lane's chunks: row 8 i + lane / 8 of the tile, place lane % 8
    const int lrow = lane / 8, lchunk = (lane % 8) ^ lrow;
    const char *xp[C::kLoadsX];
    uint32_t wo[C::kLoadsW];
#pragma unroll
    for (int i = 0; i < C::kLoadsX; ++i) {
        const int64_t p = t.row0 + (wave * C::kLoadsX + i) * 8 + lrow;
        const int64_t s = p < t.end ? source_row(a, p) : -1;
        xp[i] = a.x + (s < 0 ? 0 : s) * a.pitch + lchunk * 16;
    }
#pragma unroll
    for (int i = 0; i < C::kLoadsW; ++i) {
        const int j = (wave * C::kLoadsW + i) * 8 + lrow;
        int n = GATED ? j / 32 * 16 + j % 16 : j;
        n = n0 + n < a.c_out ? n : a.c_out - 1 - n0;
        wo[i] = static_cast<uint32_t>(n) * static_cast<uint32_t>(a.pitch) + lchunk * 16;
    }
    const int64_t woff = (static_cast<int64_t>(t.group) * a.c_out + n0) * a.pitch;
    const char *wb = uniform_ptr(a.w + woff), *wb2 = GATED ? uniform_ptr(a.w2 + woff) : wb;
    const int steps = static_cast<int>((a.pitch + 127) / 128), whole = static_cast<int>(a.pitch / 128);
    const uint32_t xl = lds0 + wave * C::kLoadsX * 1024, wl = lds0 + BM * 128 + wave * C::kLoadsW * 1024;
    const char *zero = reinterpret_cast<const char *>(kZeroChunk);
    // The adapters: each distinct one of the tile's rows is more steps of the
    // contraction, v against up, with the other adapters' rows at zero.
    constexpr int kPer = 16 / static_cast<int>(sizeof(T));
    int open[BM / kWave], ad = -1, rank = 0, k0 = 0;
    if constexpr (ADAPT) {
#pragma unroll
        for (int i = 0; i < BM / kWave; ++i) {
            const int64_t p = t.row0 + i * kWave + lane;
            open[i] = adapter_of(a, p, p < t.end);
        }
    }
    auto next_adapter = [&]() {
        k0 += 8 * kPer;
        while (k0 >= rank) {
            ad = -1;
#pragma unroll
            for (int i = 0; i < BM / kWave; ++i) {
                const uint64_t left = __ballot(open[i] >= 0);
                if (left && ad < 0)
                    ad = __builtin_amdgcn_readlane(open[i], __ffsll(static_cast<unsigned long long>(left)) - 1);
            }
            if (ad < 0) return false;
#pragma unroll
            for (int i = 0; i < BM / kWave; ++i) open[i] = open[i] == ad ? -1 : open[i];
            rank = adapter_rank(a, ad);
            k0 = 0;
        }
        return true;
    };
    // the loads of step `step`; past the last step zeros, and false
    auto load = [&](int step, uint32_t buf) {
        const int64_t off = static_cast<int64_t>(step) * 128;
        if (step < whole) {
#pragma unroll
            for (int i = 0; i < C::kLoadsX; ++i) load_to_lds(xp[i] + off, xl + buf + i * 1024);
#pragma unroll
            for (int i = 0; i < C::kLoadsW; ++i)
                load_to_lds((GATED && ((wave * C::kLoadsW + i) & 2) ? wb2 : wb) + off, wo[i], wl + buf + i * 1024);
            return true;
        }
        if constexpr (ADAPT) {
            if (step >= steps && next_adapter()) {
                const int k = k0 + lchunk * kPer;
                const T *up = reinterpret_cast<const T *>(a.up) + static_cast<int64_t>(ad) * a.c_out * a.max_rank + k;
#pragma unroll
                for (int i = 0; i < C::kLoadsX; ++i) {
                    const int64_t p = t.row0 + (wave * C::kLoadsX + i) * 8 + lrow;
                    const bool in = k < rank && adapter_of(a, p, p < t.end) == ad;
                    load_to_lds(in ? a.v + p * a.v_pitch + k * static_cast<int>(sizeof(T)) : zero, xl + buf + i * 1024);
                }
#pragma unroll
                for (int i = 0; i < C::kLoadsW; ++i) {
                    int n = n0 + (wave * C::kLoadsW + i) * 8 + lrow;
                    n = n < a.c_out ? n : a.c_out - 1;
                    load_to_lds(k < rank ? reinterpret_cast<const char *>(up + static_cast<int64_t>(n) * a.max_rank) : zero,
                                wl + buf + i * 1024);
                }
                return true;
            }
        }
        const bool in = off + lchunk * 16 < a.pitch;
#pragma unroll
        for (int i = 0; i < C::kLoadsX; ++i) load_to_lds(in ? xp[i] + off : zero, xl + buf + i * 1024);
#pragma unroll
        for (int i = 0; i < C::kLoadsW; ++i)
            load_to_lds(in ? (GATED && ((wave * C::kLoadsW + i) & 2) ? wb2 : wb) + off + wo[i] : zero,
                        wl + buf + i * 1024);
        return step < steps;
    };

    const int wm = wave % C::kWavesM * (BM / C::kWavesM), wn = wave / C::kWavesM * (BN / C::kWavesN);
    floatx4 acc[NF][MF];
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int f = 0; f < MF; ++f) acc[i][f] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    const char *xr = lds + (wm + r) * 128, *wr = lds + (BM + wn + r) * 128;
    auto multiply = [&](int buf) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4 xv[MF], wv[NF];
            const int chunk = ((kk * 4 + g) ^ (r & 7)) * 16 + buf;
#pragma unroll
            for (int i = 0; i < NF; ++i) wv[i] = *reinterpret_cast<const u32x4 *>(wr + i * 2048 + chunk);
#pragma unroll
            for (int f = 0; f < MF; ++f) xv[f] = *reinterpret_cast<const u32x4 *>(xr + f * 2048 + chunk);
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int f = 0; f < MF; ++f) acc[i][f] = chunk_mma<T>(wv[i], xv[f], acc[i][f]);
        }
    };
    // two steps a turn; past an odd last step comes one of zeros, so that every
    // product is issued unconditionally
    bool more = load(0, 0);
    for (int s = 0; more; s += 2) {
        loads_barrier();  // this step's loads have landed, the other buffer is read
        load(s + 1, C::kBuffer);
        multiply(0);
        loads_barrier();
        more = load(s + 2, 0);
        multiply(C::kBuffer);
    }
    loads_landed();

#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int64_t p = t.row0 + wm + f * 16 + r;
        if (p >= t.end || source_row(a, p) < 0) continue;
        const int64_t to = target_row(a, p);
        if (to < 0) continue;
        OT *y = reinterpret_cast<OT *>(a.y) + to * a.c_out;
#pragma unroll
        for (int i = 0; i < NF; i += GATED ? 2 : 1) {
            const int n = n0 + (GATED ? (wn + i * 16) / 2 : wn + i * 16) + 4 * g;
            if (n >= a.c_out) continue;
            float out[4];
            finish4<GATED>(a, t.group, n, acc[i][f], acc[GATED ? i + 1 : i][f], out);
            store_out<OT>(y + n, out);
        }
    }
}

// ------------------------------------------------------- sums of a token
// y[t] = (x[t]) + sum over slots of weight * o[t * k + slot], in slot order,
// fp32; slots without an expert do not count.
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
    for (int s = 0; s < top_k; ++s) {
        const int e = expert[t * top_k + s];
        if (e < 0 || e >= experts) continue;
        const float w = weight[t * top_k + s];
        float v[8];
        io<float>::load8(o + (t * top_k + s) * C + c, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum[u] = __builtin_fmaf(w, v[u], sum[u]);
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

// ------------------------------------------------ an adapter's first half
// v[row] = scale * A_id x[row], rounded to the storage type (the matrix cores
// take the second product's operand in it), for 16 rows a workgroup: one
// distinct adapter of the rows at a time, every gridDim.y-th from blockIdx.y;
// the waves split the contraction.
constexpr int kDownWaves = 8;

template <typename T, int NF>
__global__ void __launch_bounds__(kDownWaves * kWave)
k_adapter_down(const char *__restrict__ x, int64_t rows, int64_t pitch, const char *__restrict__ down,
               const int32_t *__restrict__ ids, const int32_t *__restrict__ ranks, const float *__restrict__ scales,
               int adapters, int max_rank, char *__restrict__ v, int v_pitch) {
    __shared__ floatx4 part[kDownWaves - 1][NF][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int r = lane % 16, g = lane / 16;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 16 + r;
    int id = row < rows ? ids[row] : -1;
    if (id >= adapters) id = -1;
    const char *xp = x + (row < rows ? row : rows - 1) * pitch;
    const int64_t steps = (pitch + 63) / 64;
    const int64_t s0 = steps * wave / kDownWaves, s1 = steps * (wave + 1) / kDownWaves;
    bool open = id >= 0;
    for (int turn = 0;; ++turn) {
        const uint64_t left = __ballot(open);
        if (!left) break;
        const int ad = __builtin_amdgcn_readlane(id, __ffsll(static_cast<unsigned long long>(left)) - 1);
        open = open && id != ad;
        if (turn % static_cast<int>(gridDim.y) != static_cast<int>(blockIdx.y)) continue;
        int rank = ranks ? ranks[ad] : max_rank;
        rank = rank < max_rank ? rank : max_rank;
        const float scale = scales ? scales[ad] : 1.0f;
        const char *base = down + static_cast<int64_t>(ad) * max_rank * pitch;
        for (int n0 = 0; n0 < rank; n0 += NF * 16) {
            const char *wp[NF];
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                const int n = n0 + i * 16 + r;
                wp[i] = base + static_cast<int64_t>(n < rank ? n : rank - 1) * pitch;
            }
            floatx4 acc[NF];
#pragma unroll
            for (int i = 0; i < NF; ++i) acc[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            constexpr int U = 4;
            int64_t s = s0;
            for (; s + U <= s1 && (s + U) * 64 <= pitch; s += U) {
                u32x4 wv[U][NF], xv[U];
                const int64_t off = s * 64 + g * 16;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    xv[u] = *reinterpret_cast<const u32x4 *>(xp + off + u * 64);
#pragma unroll
                    for (int i = 0; i < NF; ++i) wv[u][i] = *reinterpret_cast<const u32x4 *>(wp[i] + off + u * 64);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < NF; ++i) acc[i] = chunk_mma<T>(wv[u][i], xv[u], acc[i]);
            }
            for (; s < s1; ++s) {
                const int64_t off = s * 64 + g * 16;
                const bool in = off < pitch;
                const u32x4 none = {0, 0, 0, 0};
                const u32x4 xv = in ? *reinterpret_cast<const u32x4 *>(xp + off) : none;
                u32x4 wv[NF];
#pragma unroll
                for (int i = 0; i < NF; ++i) wv[i] = in ? *reinterpret_cast<const u32x4 *>(wp[i] + off) : none;
#pragma unroll
                for (int i = 0; i < NF; ++i) acc[i] = chunk_mma<T>(wv[i], xv, acc[i]);
            }
            if (wave > 0) {
#pragma unroll
                for (int i = 0; i < NF; ++i) part[wave - 1][i][lane] = acc[i];
            }
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int i = 0; i < NF; ++i) {
#pragma unroll
                    for (int w = 0; w < kDownWaves - 1; ++w) acc[i] += part[w][i][lane];
                    const int n = n0 + i * 16 + 4 * g;
                    if (id == ad && n < max_rank) {
                        float out[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) out[u] = n + u < rank ? scale * acc[i][u] : 0.0f;
                        io<T>::store4(reinterpret_cast<T *>(v + row * v_pitch) + n, out);
                    }
                }
            }
            __syncthreads();
        }
    }
}

}  // namespace dynconv
