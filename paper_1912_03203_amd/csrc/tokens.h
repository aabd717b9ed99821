// tokens.h -- host side of the token operators (router, grouped products,
// expert layers, low-rank adapters): validation, workspace layout, launches.
// Included at the end of dynconv.hip, whose helpers it uses.
#pragma once

namespace {

constexpr int64_t kMaxTokenRows = (int64_t{1} << 31) - 1;  // list entries are int32
constexpr int kMaxWidth = 1 << 16;
constexpr int kMaxRank = 256;

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

dynconv_status check_width(int64_t c) {
    if (c <= 0) return DYNCONV_ERR_SHAPE;
    return c % 8 != 0 || c > kMaxWidth ? DYNCONV_ERR_UNSUPPORTED : DYNCONV_OK;
}

dynconv_status check_act(int32_t act) {
    return act < DYNCONV_ACT_NONE || act > DYNCONV_ACT_GELU ? DYNCONV_ERR_ARG : DYNCONV_OK;
}

// --------------------------------------------------------------- router
int bits_for(int values) {  // of the numbers 0 .. values - 1
    int b = 0;
    while ((1 << b) < values) ++b;
    return b;
}

// Rows per choosing workgroup: as many workgroups as the chip has CUs, 32 rows
// at least (one pass of its groups of lanes), and no more assignments than the
// list workgroup holds.
int route_rows_per_group(int64_t tokens, int top_k) {
    int64_t per = (tokens + 255) / 256;
    per = (per + 31) / 32 * 32;
    return static_cast<int>(std::min<int64_t>(per, kRouteChunk / top_k));
}

// One workgroup does it all up to 128 rows, two passes of its groups of lanes (64
// rows of 64 experts, top 8: 7.5 us against 11.3 in three launches; 128: 11.2
// against 11.4; 256: 18.6 against 11.5).
bool route_is_one(int64_t tokens, int top_k) { return tokens <= 128 && tokens * top_k <= kRouteOne; }

struct RouteLayout {
    int per = 0;
    int64_t blocks = 0;
    size_t hist = 0, totals = 0, bytes = 0;
};

RouteLayout route_layout(int64_t tokens, int experts, int top_k) {
    RouteLayout L;
    if (!route_is_one(tokens, top_k)) {
        L.per = route_rows_per_group(tokens, top_k);
        L.blocks = (tokens + L.per - 1) / L.per;
        L.totals = align_up(sizeof(int32_t) * static_cast<size_t>(L.blocks) * (experts + 1));
    }
    L.bytes = L.totals + align_up(sizeof(int32_t) * (experts + 1));
    return L;
}

dynconv_status check_route_sizes(int64_t tokens, int32_t experts, int32_t top_k) {
    if (tokens < 0 || experts <= 0 || top_k <= 0) return DYNCONV_ERR_SHAPE;
    if (top_k > experts) return DYNCONV_ERR_SHAPE;
    if (experts > kMaxExperts || top_k > kMaxTopK) return DYNCONV_ERR_UNSUPPORTED;
    return tokens > kMaxTokenRows / top_k ? DYNCONV_ERR_SHAPE : DYNCONV_OK;
}

template <typename T, int G, int V>
void launch_route_k(const void *logits, int64_t tokens, int E, int top_k, const float *bias, const uint8_t *mask,
                    int flags, float scale, const dynconv_routes *out, void *ws, hipStream_t st, Marks &mk) {
    const int bits = bits_for(E + 1);
    const RouteLayout L = route_layout(tokens, E, top_k);
    if (L.blocks == 0) {
        launch(mk, k_route_one<T, G, V>, dim3(1), dim3(kRouteOneThreads),
               sizeof(uint16_t) * (kRouteOneThreads / kWave) * (E + 1), st, static_cast<const T *>(logits),
               static_cast<int>(tokens), E, top_k, bits, bias, mask, flags, scale, out->expert, out->weight, out->rows,
               out->starts);
        return;
    }
    int32_t *hist = at<int32_t>(ws, L.hist), *totals = at<int32_t>(ws, L.totals);
    const dim3 grid(static_cast<unsigned>(L.blocks));
    // a row for each group of lanes at least; where there are more (on whole waves
    // always: 32 rows at least), more waves hide each other's waits
    auto choose = [&](auto kern, int threads) {
        launch(mk, kern, grid, dim3(threads), 0, st, static_cast<const T *>(logits), tokens, L.per, E, top_k, bias, mask,
               flags, scale, out->expert, out->weight, hist);
    };
    if (G == kWave || L.per > kRouteThreads / G) choose(k_route_choose<T, G, V, 1024>, 1024);
    else if constexpr (G != kWave) choose(k_route_choose<T, G, V, kRouteThreads>, kRouteThreads);
    launch(mk, k_route_scan, dim3((E + kWavesPerBlock) / kWavesPerBlock), dim3(kBlock), 0, st, hist,
           static_cast<int>(L.blocks), E + 1, totals);
    launch(mk, k_route_lists, grid, dim3(kRouteThreads), sizeof(uint16_t) * kRouteWaves * (E + 1), st, out->expert,
           tokens * top_k, L.per * top_k, E, bits, hist, totals, out->rows, out->starts);
}

template <typename T>
void launch_route(const void *logits, int64_t tokens, int E, int top_k, const float *bias, const uint8_t *mask,
                  int flags, float scale, const dynconv_routes *out, void *ws, hipStream_t st, Marks &mk) {
    auto go = [&](auto f) { f(logits, tokens, E, top_k, bias, mask, flags, scale, out, ws, st, mk); };
    if (E <= 16) go(launch_route_k<T, 16, 1>);
    else if (E <= 32) go(launch_route_k<T, 16, 2>);
    else if (E <= 64) go(launch_route_k<T, 16, 4>);
    else if (E <= 128) go(launch_route_k<T, 16, 8>);
    else if (E <= 256) go(launch_route_k<T, 16, 16>);
    else if (E <= 512) go(launch_route_k<T, 64, 8>);
    else go(launch_route_k<T, 64, 16>);
}

// ------------------------------------------------------ grouped products
// Row tiles of any split of `rows` rows into `groups` groups, at most.
int64_t most_tiles(int64_t rows, int64_t groups, int bm, bool split) {
    return split ? rows / bm + std::min(rows, groups) : (rows + bm - 1) / bm;
}

// The forms of the products: few rows a group (16 to 64 rows a workgroup, the
// contraction split over its waves) or tiles of 64, 128 or 256 rows.
struct RowsPlan {
    int bm = 0;      // rows of a tile
    int slices = 0;  // tiles along the outputs
    bool few = false;
    int64_t blocks = 0;
};

// The form by the mean number of rows a group and the tiles that groups of that
// size make (weight rows = outputs, twice as many when gated); bf16, us, on groups of
// equal size:
//   few rows / 64-row tiles   32 groups 2048 -> 1024, 16 rows each 25.7 / 26.8, 32:
//     28.3 / 28.4, 64: 47.6 / 34.1; 8 groups 1024 -> 2048, 32 rows 10.4 / 9.1.  Few
//     rows up to 16, and beyond where the tiles would leave most CUs idle (a decoding
//     step through one projection).
//   64 / 128  one group of 1024 rows 2048 -> 2048 (128 tiles of 128) 20.1 / 25.0, of
//     2048 rows (256 tiles) 36.6 / 28.3; 12 groups of 125, 1024 -> 1024 (96) 12.7 / 15.9;
//     32 of 96, 2048 -> 1024 (256) 50.5 / 38.0.  The larger tile from 192 on.
//   128 / 256  one group of 2048 rows 2048 -> 4096 (128 tiles of 256) 46.2 / 48.7; 32
//     groups of 256 rows 1024 -> 2048 (256 tiles) 59.9 / 48.2.  Likewise.  fp32 has no
//     256-row tile: its products take 16 times as long, and fill the CUs with less.
// On groups as a router makes them (choices of 2, the experts' logits spread by half
// of the rows' own deviation) half of the groups pass a mean of 16 and take two tiles of
// 16 rows, where the tiles of 64 still take one:
//   few rows / 64-row tiles   32 groups 2048 -> 1024, mean 8 29.2 / 36.2, 16: 34.1 / 38.5,
//     32: 40.0 / 39.5; 64 groups 1024 -> 2048, 8: 58.2 / 58.0, 16: 74.8 / 60.4; 8 groups 1024
//     -> 2048, 16: 11.6 / 9.0: the rule is late for short contractions.
//   128 / 256  32 groups of mean 256, 1024 -> 2048 70.6 / 72.6, of 512, 2048 -> 2048 208 / 186.
RowsPlan rows_plan(int64_t rows, int64_t groups, bool adapt, int c_out, bool gated, dynconv_dtype dt) {
    RowsPlan p;
    const int64_t mean = (rows + groups - 1) / groups, used = std::min(rows, groups);
    const int64_t weights = static_cast<int64_t>(c_out) * (gated ? 2 : 1);
    auto tiles = [&](int bm) { return used * ((mean + bm - 1) / bm) * ((weights + bm - 1) / bm); };
    constexpr int64_t kFill = 192;  // tiles that keep the 256 CUs busy
    p.few = mean <= 16 || (mean <= 64 && tiles(64) < kFill);
    if (p.few) {
        p.bm = static_cast<int>((mean + 15) / 16 * 16);
        const int outs = gated || adapt ? 16 : 32;
        p.slices = (c_out + outs - 1) / outs;
    } else {
        p.bm = dt != DYNCONV_F32 && mean >= 256 && tiles(256) >= kFill ? 256 : tiles(128) >= kFill ? 128 : 64;
        const int outs = gated ? p.bm / 2 : p.bm;
        p.slices = (c_out + outs - 1) / outs;
    }
    // adapters: one group, of all rows; otherwise groups of sizes that only the
    // device knows.  Whole turns of the 8 XCDs.
    p.blocks = (most_tiles(rows, groups, p.bm, !adapt) * p.slices + 7) / 8 * 8;
    return p;
}

template <typename T, typename OT, bool GATED, bool ADAPT>
void launch_rows(const RowsArgs &a, const RowsPlan &p, hipStream_t st, Marks &mk) {
    const dim3 grid = grid_xy(p.blocks);
    if (p.few) {
        constexpr int NW = ADAPT ? 8 : 4, NF = ADAPT ? 1 : 2;
        auto go = [&](auto kern) { launch(mk, kern, grid, dim3(NW * kWave), 0, st, a, p.slices); };
        if (p.bm == 16) go(k_rows_few<T, OT, NW, NF, 1, GATED, ADAPT>);
        else if (p.bm == 32) go(k_rows_few<T, OT, NW, NF, 2, GATED, ADAPT>);
        else if (p.bm == 48) go(k_rows_few<T, OT, NW, NF, 3, GATED, ADAPT>);
        else go(k_rows_few<T, OT, NW, NF, 4, GATED, ADAPT>);
        return;
    }
    if constexpr (sizeof(T) == 2) {
        if (p.bm == 256) {
            launch(mk, k_rows_tile<T, OT, 256, 256, GATED, ADAPT>, grid, dim3(TileCfg<256, 256>::kThreads), 0, st, a,
                   p.slices);
            return;
        }
    }
    if (p.bm == 128)
        launch(mk, k_rows_tile<T, OT, 128, 128, GATED, ADAPT>, grid, dim3(TileCfg<128, 128>::kThreads), 0, st, a, p.slices);
    else
        launch(mk, k_rows_tile<T, OT, 64, 64, GATED, ADAPT>, grid, dim3(TileCfg<64, 64>::kThreads), 0, st, a, p.slices);
}

// out32: the outputs are fp32 whatever the storage type
template <typename T>
void launch_rows_any(const RowsArgs &a, const RowsPlan &p, bool gated, bool out32, hipStream_t st, Marks &mk) {
    if (gated) launch_rows<T, T, true, false>(a, p, st, mk);
    else if (out32) launch_rows<T, float, false, false>(a, p, st, mk);
    else launch_rows<T, T, false, false>(a, p, st, mk);
}

void dispatch_rows(dynconv_dtype dt, const RowsArgs &a, const RowsPlan &p, bool gated, bool out32, hipStream_t st,
                   Marks &mk) {
    if (dt == DYNCONV_F32) launch_rows_any<float>(a, p, gated, out32, st, mk);
    else if (dt == DYNCONV_F16) launch_rows_any<half_t>(a, p, gated, out32, st, mk);
    else launch_rows_any<bf16_t>(a, p, gated, out32, st, mk);
}

// ------------------------------------------------------------- experts
dynconv_status check_experts(const dynconv_experts *e, dynconv_dtype dt, int64_t tokens, int32_t top_k, int32_t flags) {
    if (!e) return DYNCONV_ERR_NULL;
    if (!e->w_expand || !e->w_project) return DYNCONV_ERR_NULL;
    if (!dtype_ok(dt)) return DYNCONV_ERR_DTYPE;
    for (int32_t c : {e->c_in, e->c_hidden, e->c_out})
        if (dynconv_status st = check_width(c)) return st;
    if (dynconv_status st = check_route_sizes(tokens, e->experts, top_k)) return st;
    if (dynconv_status st = check_act(e->act)) return st;
    if (flags & ~DYNCONV_EXPERTS_RESIDUAL) return DYNCONV_ERR_ARG;
    if ((flags & DYNCONV_EXPERTS_RESIDUAL) && e->c_in != e->c_out) return DYNCONV_ERR_SHAPE;
    for (const void *p : {e->w_expand, e->w_gate, e->w_project, static_cast<const void *>(e->b_expand),
                          static_cast<const void *>(e->b_gate), static_cast<const void *>(e->b_project)})
        if (!aligned16(p)) return DYNCONV_ERR_ALIGN;
    return DYNCONV_OK;
}

// Few tokens: one launch for the second product and the sum.  A token's experts
// differ, so one token always gains; more do while their choices seldom meet.  This
// form multiplies one row a matrix instruction, so a second half of the hidden row is
// free there.  Elsewhere it is not: with two halves the second product would read or
// multiply twice the rows (an expert layer of long prompts a third more), so those
// calls round h to the storage type, as this library's blocks do with their
// intermediates, and a token's result is the more exact one in a call of few.
bool few_tokens(int64_t tokens, int top_k, int experts) {
    return tokens == 1 || tokens * top_k * 2 <= experts;
}

struct ExpertsLayout {
    size_t out = 0, bytes = 0;  // hidden rows first, then the experts' outputs in fp32
};

ExpertsLayout experts_layout(const dynconv_experts *e, int64_t tokens, int top_k, dynconv_dtype dt) {
    ExpertsLayout L;
    const size_t rows = static_cast<size_t>(tokens) * top_k;
    if (few_tokens(tokens, top_k, e->experts)) {  // hidden rows alone: two halves in 16-bit types, fp32 as it is
        L.bytes = std::max(kAlign, align_up(rows * e->c_hidden * sizeof(float)));
        return L;
    }
    L.out = align_up(rows * e->c_hidden * dtype_size(dt));
    L.bytes = std::max(kAlign, L.out + align_up(rows * e->c_out * sizeof(float)));
    return L;
}

template <typename T>
void launch_combine(const float *o, const dynconv_routes *r, const void *x, void *y, int64_t tokens, int C, int top_k,
                    int experts, hipStream_t st, Marks &mk) {
    const int64_t items = tokens * (C / 8);
    launch(mk, k_combine<T>, grid_xy((items + kBlock - 1) / kBlock), dim3(kBlock), 0, st, o, r->expert, r->weight,
           static_cast<const T *>(x), static_cast<T *>(y), tokens, C, top_k, experts);
}

template <typename T>
void launch_project_tokens(const RowsArgs &o, const dynconv_routes *r, const void *x, void *y, int64_t tokens, int top_k,
                           int experts, hipStream_t st, Marks &mk) {
    constexpr int NW = 8;
    const int slices = (o.c_out + 15) / 16;
    launch(mk, k_project_tokens<T, NW>, dim3(static_cast<unsigned>(tokens * slices)), dim3(NW * kWave), 0, st, o.x, o.pitch,
           r->expert, r->weight, top_k, experts, o.w, o.b, static_cast<const T *>(x), static_cast<T *>(y), o.c_out, slices);
}

// ------------------------------------------------------------- adapters
dynconv_status check_adapters(const dynconv_linear *l, const dynconv_adapters *a, int64_t rows, dynconv_dtype dt) {
    if (!l || !a) return DYNCONV_ERR_NULL;
    if (!l->w || !a->down || !a->up) return DYNCONV_ERR_NULL;
    if (!dtype_ok(dt)) return DYNCONV_ERR_DTYPE;
    if (rows < 0 || rows > kMaxTokenRows) return DYNCONV_ERR_SHAPE;
    for (int32_t c : {l->c_in, l->c_out})
        if (dynconv_status st = check_width(c)) return st;
    if (dynconv_status st = check_act(l->act)) return st;
    if (a->adapters <= 0 || a->max_rank <= 0) return DYNCONV_ERR_SHAPE;
    if (a->max_rank % 8 != 0 || a->max_rank > kMaxRank || a->adapters > kMaxAdapters) return DYNCONV_ERR_UNSUPPORTED;
    for (const void *p : {l->w, static_cast<const void *>(l->b), a->down, a->up})
        if (!aligned16(p)) return DYNCONV_ERR_ALIGN;
    if (!aligned4(a->ranks) || !aligned4(a->scales)) return DYNCONV_ERR_ALIGN;
    return DYNCONV_OK;
}

// The first halves' results: fp32, or two halves of 16 bits.
size_t adapter_bytes(const dynconv_adapters *a, int64_t rows) {
    return std::max(kAlign, align_up(static_cast<size_t>(rows) * a->max_rank * sizeof(float)));
}

template <typename T>
void launch_adapters(const RowsArgs &args, const RowsPlan &p, const dynconv_linear *l, const dynconv_adapters *ad,
                     void *v, hipStream_t st, Marks &mk) {
    // 16 rows a workgroup, and one for each distinct adapter that 16 rows can have
    // until they fill the CUs
    const int64_t tiles = (args.rows + 15) / 16;
    dim3 grid = grid_xy(tiles);
    grid.z = static_cast<unsigned>(tiles >= 256 ? 1 : std::min<int64_t>({16, args.rows, ad->adapters}));
    auto go = [&](auto kern) {
        launch(mk, kern, grid, dim3(kDownWaves * kWave), 0, st, args.x, args.rows, args.pitch,
               static_cast<const char *>(ad->down), args.ids, ad->ranks, ad->scales, ad->adapters, args.id_bits,
               ad->max_rank, static_cast<char *>(v), args.v_pitch);
    };
    if (ad->max_rank <= 16) go(k_adapter_down<T, 1>);
    else if (ad->max_rank <= 32) go(k_adapter_down<T, 2>);
    else go(k_adapter_down<T, 4>);
    launch_rows<T, T, false, true>(args, p, st, mk);
}

}  // namespace

// ----------------------------------------------------------------- C ABI
extern "C" {

size_t dynconv_route_workspace_bytes(int64_t tokens, int32_t experts, int32_t top_k) {
    if (check_route_sizes(tokens, experts, top_k) != DYNCONV_OK) return 0;
    return route_layout(tokens, experts, top_k).bytes;
}

dynconv_status dynconv_route(const void *logits, int64_t tokens, dynconv_dtype dt, int32_t experts, int32_t top_k,
                             const float *bias, const uint8_t *mask, int32_t flags, float scale,
                             const dynconv_routes *routes, void *ws, size_t ws_bytes, void *stream) {
    if (!routes || !routes->starts) return DYNCONV_ERR_NULL;
    if (!dtype_ok(dt)) return DYNCONV_ERR_DTYPE;
    if (dynconv_status st = check_route_sizes(tokens, experts, top_k)) return st;
    if (tokens > 0 && (!logits || !routes->expert || !routes->weight || !routes->rows)) return DYNCONV_ERR_NULL;
    if (flags & ~(DYNCONV_ROUTE_SIGMOID | DYNCONV_ROUTE_RENORMALIZE | DYNCONV_ROUTE_SCORE_BIAS)) return DYNCONV_ERR_ARG;
    if (routes->capacity < tokens * top_k) return DYNCONV_ERR_CAPACITY;
    if ((reinterpret_cast<uintptr_t>(logits) & (dtype_size(dt) - 1)) != 0) return DYNCONV_ERR_ALIGN;
    for (const void *p : {static_cast<const void *>(bias), static_cast<const void *>(routes->expert),
                          static_cast<const void *>(routes->weight), static_cast<const void *>(routes->rows),
                          static_cast<const void *>(routes->starts), static_cast<const void *>(ws)})
        if (!aligned4(p)) return DYNCONV_ERR_ALIGN;
    if (!ws || ws_bytes < route_layout(tokens, experts, top_k).bytes) return DYNCONV_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    Marks mk;
    auto go = [&](auto f) { f(logits, tokens, experts, top_k, bias, mask, flags, scale, routes, ws, st, mk); };
    if (dt == DYNCONV_F32) go(launch_route<float>);
    else if (dt == DYNCONV_F16) go(launch_route<half_t>);
    else go(launch_route<bf16_t>);
    return launch_status();
}

dynconv_status dynconv_grouped_linear(const void *x, int64_t x_rows, void *y, int64_t y_rows, dynconv_dtype dt,
                                      const dynconv_linear *l, int32_t groups, const int32_t *starts, int64_t rows,
                                      const int32_t *src, int32_t src_div, const int32_t *dst, void *stream) {
    if (!l || !l->w || !starts) return DYNCONV_ERR_NULL;
    if (!dtype_ok(dt)) return DYNCONV_ERR_DTYPE;
    if (x_rows < 0 || y_rows < 0 || rows < 0 || groups <= 0) return DYNCONV_ERR_SHAPE;
    if (x_rows > kMaxTokenRows || y_rows > kMaxTokenRows || rows > kMaxTokenRows) return DYNCONV_ERR_SHAPE;
    for (int32_t c : {l->c_in, l->c_out})
        if (dynconv_status st = check_width(c)) return st;
    if (groups > kMaxGroups) return DYNCONV_ERR_UNSUPPORTED;
    if (dynconv_status st = check_act(l->act)) return st;
    if (src_div < 1 || (!src && src_div != 1)) return DYNCONV_ERR_ARG;
    if ((!src && x_rows < rows) || (!dst && y_rows < rows)) return DYNCONV_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(y) || !aligned16(l->w) || !aligned16(l->b)) return DYNCONV_ERR_ALIGN;
    if (!aligned4(starts) || !aligned4(src) || !aligned4(dst)) return DYNCONV_ERR_ALIGN;
    if (rows == 0 || x_rows == 0 || y_rows == 0) return DYNCONV_OK;
    if (!x || !y) return DYNCONV_ERR_NULL;
    const size_t s = dtype_size(dt);
    if (ranges_overlap(x, static_cast<size_t>(x_rows) * l->c_in * s, y, static_cast<size_t>(y_rows) * l->c_out * s))
        return DYNCONV_ERR_SHAPE;
    RowsArgs a{};
    a.x = static_cast<const char *>(x);
    a.x_rows = x_rows;
    a.pitch = static_cast<int64_t>(l->c_in) * static_cast<int64_t>(s);
    a.src = src;
    a.src_div = static_cast<uint32_t>(src_div);
    a.starts = starts;
    a.groups = groups;
    a.rows = rows;
    a.w = static_cast<const char *>(l->w);
    a.b = l->b;
    a.c_out = l->c_out;
    a.act = l->act;
    a.y = static_cast<char *>(y);
    a.y_rows = y_rows;
    a.dst = dst;
    const RowsPlan p = rows_plan(rows, groups, false, l->c_out, false, dt);
    if (p.blocks > kMaxTokenRows) return DYNCONV_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    Marks mk;
    dispatch_rows(dt, a, p, false, false, static_cast<hipStream_t>(stream), mk);
    return launch_status();
}

size_t dynconv_experts_workspace_bytes(int64_t tokens, const dynconv_experts *e, dynconv_dtype dt, int32_t top_k) {
    if (check_experts(e, dt, tokens, top_k, 0) != DYNCONV_OK) return 0;
    return experts_layout(e, tokens, top_k, dt).bytes;
}

dynconv_status dynconv_experts_forward(const void *x, void *y, int64_t tokens, dynconv_dtype dt,
                                       const dynconv_experts *e, int32_t top_k, const dynconv_routes *routes,
                                       int32_t flags, void *ws, size_t ws_bytes, void *stream) {
    if (dynconv_status st = check_experts(e, dt, tokens, top_k, flags)) return st;
    if (!routes) return DYNCONV_ERR_NULL;
    if (tokens > 0 && (!x || !y || !routes->expert || !routes->weight || !routes->rows || !routes->starts))
        return DYNCONV_ERR_NULL;
    const int64_t rows = tokens * top_k;
    if (routes->capacity < rows) return DYNCONV_ERR_CAPACITY;
    if (!aligned16(x) || !aligned16(y) || !aligned16(ws)) return DYNCONV_ERR_ALIGN;
    if (!aligned4(routes->expert) || !aligned4(routes->weight) || !aligned4(routes->rows) || !aligned4(routes->starts))
        return DYNCONV_ERR_ALIGN;
    const size_t s = dtype_size(dt);
    const size_t in_bytes = static_cast<size_t>(tokens) * e->c_in * s;
    const size_t out_bytes = static_cast<size_t>(tokens) * e->c_out * s;
    if (ranges_overlap(x, in_bytes, y, out_bytes) && !(x == y && e->c_in == e->c_out)) return DYNCONV_ERR_SHAPE;
    const ExpertsLayout L = experts_layout(e, tokens, top_k, dt);
    if (!ws || ws_bytes < L.bytes) return DYNCONV_ERR_WORKSPACE;
    if (tokens == 0) return DYNCONV_OK;
    RowsArgs a{};
    a.x = static_cast<const char *>(x);
    a.x_rows = tokens;
    a.pitch = static_cast<int64_t>(e->c_in) * static_cast<int64_t>(s);
    a.src = routes->rows;
    a.src_div = static_cast<uint32_t>(top_k);
    a.starts = routes->starts;
    a.groups = e->experts;
    a.rows = rows;
    a.w = static_cast<const char *>(e->w_expand);
    a.b = e->b_expand;
    a.w2 = static_cast<const char *>(e->w_gate);
    a.b2 = e->b_gate;
    a.c_out = e->c_hidden;
    a.act = e->act;
    a.y = static_cast<char *>(ws);
    a.y_rows = rows;
    const bool few = few_tokens(tokens, top_k, e->experts);
    if (few) {
        a.dst = routes->rows;  // hidden rows at their assignments, not in list order
        a.halves = dt != DYNCONV_F32;
    }
    const bool gated = e->w_gate != nullptr;
    const RowsPlan p1 = rows_plan(rows, e->experts, false, e->c_hidden, gated, dt);  // few tokens: few rows
    RowsArgs o = a;
    o.halves = false;
    o.x = static_cast<const char *>(ws);
    o.x_rows = rows;
    o.pitch = static_cast<int64_t>(e->c_hidden) * static_cast<int64_t>(s);
    o.src = nullptr;
    o.src_div = 1;
    o.w = static_cast<const char *>(e->w_project);
    o.b = e->b_project;
    o.w2 = nullptr;
    o.b2 = nullptr;
    o.c_out = e->c_out;
    o.act = DYNCONV_ACT_NONE;
    o.y = at(ws, L.out);
    o.dst = routes->rows;
    const RowsPlan p2 = rows_plan(rows, e->experts, false, e->c_out, false, dt);
    if (p1.blocks > kMaxTokenRows || p2.blocks > kMaxTokenRows) return DYNCONV_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    Marks mk;
    const void *res = (flags & DYNCONV_EXPERTS_RESIDUAL) ? x : nullptr;
    dispatch_rows(dt, a, p1, gated, false, st, mk);
    if (few) {
        auto go = [&](auto f) { f(o, routes, res, y, tokens, top_k, e->experts, st, mk); };
        if (dt == DYNCONV_F32) go(launch_project_tokens<float>);
        else if (dt == DYNCONV_F16) go(launch_project_tokens<half_t>);
        else go(launch_project_tokens<bf16_t>);
        return launch_status();
    }
    dispatch_rows(dt, o, p2, false, true, st, mk);
    const float *oo = at<const float>(ws, L.out);
    auto go = [&](auto f) { f(oo, routes, res, y, tokens, e->c_out, top_k, e->experts, st, mk); };
    if (dt == DYNCONV_F32) go(launch_combine<float>);
    else if (dt == DYNCONV_F16) go(launch_combine<half_t>);
    else go(launch_combine<bf16_t>);
    return launch_status();
}

size_t dynconv_adapter_workspace_bytes(int64_t rows, const dynconv_linear *l, const dynconv_adapters *adapters,
                                       dynconv_dtype dt) {
    if (check_adapters(l, adapters, rows, dt) != DYNCONV_OK) return 0;
    return adapter_bytes(adapters, rows);
}

dynconv_status dynconv_adapter_linear(const void *x, void *y, int64_t rows, dynconv_dtype dt, const dynconv_linear *l,
                                      const dynconv_adapters *adapters, const int32_t *ids, void *ws, size_t ws_bytes,
                                      void *stream) {
    if (dynconv_status st = check_adapters(l, adapters, rows, dt)) return st;
    if (rows > 0 && (!x || !y || !ids)) return DYNCONV_ERR_NULL;
    if (!aligned16(x) || !aligned16(y) || !aligned16(ws)) return DYNCONV_ERR_ALIGN;
    if (!aligned4(ids)) return DYNCONV_ERR_ALIGN;
    const size_t s = dtype_size(dt);
    if (ranges_overlap(x, static_cast<size_t>(rows) * l->c_in * s, y, static_cast<size_t>(rows) * l->c_out * s))
        return DYNCONV_ERR_SHAPE;
    if (!ws || ws_bytes < adapter_bytes(adapters, rows)) return DYNCONV_ERR_WORKSPACE;
    if (rows == 0) return DYNCONV_OK;
    RowsArgs a{};
    a.x = static_cast<const char *>(x);
    a.x_rows = rows;
    a.pitch = static_cast<int64_t>(l->c_in) * static_cast<int64_t>(s);
    a.src_div = 1;
    a.groups = 1;
    a.rows = rows;
    a.w = static_cast<const char *>(l->w);
    a.b = l->b;
    a.c_out = l->c_out;
    a.act = l->act;
    a.y = static_cast<char *>(y);
    a.y_rows = rows;
    a.v = static_cast<const char *>(ws);
    a.v_pitch = adapters->max_rank * static_cast<int>(sizeof(float));
    a.up = static_cast<const char *>(adapters->up);
    a.ids = ids;
    a.ranks = adapters->ranks;
    a.adapters = adapters->adapters;
    a.max_rank = adapters->max_rank;
    a.id_bits = bits_for(adapters->adapters);
    const RowsPlan p = rows_plan(rows, 1, true, l->c_out, false, dt);
    if (p.blocks > kMaxTokenRows) return DYNCONV_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    Marks mk;
    auto go = [&](auto f) { f(a, p, l, adapters, ws, st, mk); };
    if (dt == DYNCONV_F32) go(launch_adapters<float>);
    else if (dt == DYNCONV_F16) go(launch_adapters<half_t>);
    else go(launch_adapters<bf16_t>);
    return launch_status();
}

}  // extern "C"
