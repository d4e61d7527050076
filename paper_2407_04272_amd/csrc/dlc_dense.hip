// Host side of the dense operators: argument checks, the choice of kernels, workspace, C ABI.
#include "dlc_dense.h"

using namespace dlc;

namespace {

struct Shape {
    int64_t M, K, N;  // gated: N columns of y, 2 N rows of w
    int64_t ldx, ldw, ldy, ldpre, ldres, lddy, lddx, lddw;
    bool gated, off_boundary;
    int es;
    uint32_t thr;
    float scale;
};

constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxDim = int64_t(1) << 20;
// a launch's threads, work-groups of 256, are counted in 32 bits
constexpr int64_t kMaxGroups = int64_t(1) << 24;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool good_ld(int64_t& ld, int64_t row) {
    if (ld == 0) ld = row;
    return ld >= row && ld <= kMaxDim;
}

bool dropout_params(double p, uint32_t* thr, float* scale) {
    if (!(p >= 0.0 && p <= 1.0)) return false;
    *thr = (uint32_t)(p * 65536.0 + 0.5);
    *scale = *thr < 65536u ? 65536.0f / (float)(65536u - *thr) : 0.0f;
    return true;
}

bool make_shape(const dlc_dense_config* c, bool gated, Shape* s) {
    if (!c) return false;
    if (c->dtype != DLC_F32 && c->dtype != DLC_F16 && c->dtype != DLC_BF16) return false;
    if (c->act < DLC_ACT_NONE || c->act > DLC_ACT_GELU) return false;
    if (c->rows < 0 || c->rows > kMaxRows) return false;
    if (c->in_features < 1 || c->in_features > kMaxDim || c->out_features < 1 || c->out_features > kMaxDim) return false;
    const int64_t wide = gated ? 2 * c->out_features : c->out_features;
    if (wide > kMaxDim) return false;  // (a tile's 256 rows of dz span less than 2^31 bytes)
    s->M = c->rows; s->K = c->in_features; s->N = c->out_features;
    s->ldx = c->ld_x; s->ldw = c->ld_w; s->ldy = c->ld_y; s->ldpre = c->ld_pre;
    s->ldres = c->ld_res; s->lddy = c->ld_dy; s->lddx = c->ld_dx; s->lddw = c->ld_dw;
    if (!good_ld(s->ldx, s->K) || !good_ld(s->ldw, s->K) || !good_ld(s->lddx, s->K) || !good_ld(s->lddw, s->K)) return false;
    if (!good_ld(s->ldy, s->N) || !good_ld(s->ldpre, wide) || !good_ld(s->ldres, s->N) || !good_ld(s->lddy, s->N)) return false;
    if (c->flags & ~(int32_t)DLC_DENSE_OFF_BOUNDARY || c->reserved != 0) return false;
    s->off_boundary = (c->flags & DLC_DENSE_OFF_BOUNDARY) != 0;
    s->gated = gated;
    s->es = c->dtype == DLC_F32 ? 4 : 2;
    // the results of every product fit a launch with the type's largest tile (plan_gemm leaves tiles out that do not)
    const int64_t side = kTileM[s->es == 4 ? 1 : 0], tm = div_up(s->M, side), tk = div_up(s->K, side), tw = div_up(wide, side);
    if (tm * tw >= kMaxGroups || tm * tk >= kMaxGroups || tw * tk >= kMaxGroups) return false;
    return dropout_params(c->dropout_p, &s->thr, &s->scale);
}

bool on(const void* p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }
bool rows16(const void* p, int64_t ld, int es) { return on(p, 16) && (ld * es) % 16 == 0; }

size_t a256(size_t v) { return (v + 255) & ~size_t(255); }

// ---- choice of tile and cut ---------------------------------------------------------------------
struct Plan {
    int tile;
    int split, kper;
    int tiles_m, tiles_n;
    int64_t part_ld;
    size_t bytes;  // of the partial sums
    double t;      // the estimate, us
};

// What a k tile (128 bytes of k) costs with 1, 2 and 3 work-groups on a compute unit, in us, what a work-group costs
// besides, and what it costs more to write partial sums, measured with all three layouts on full and half full cards (0: no
// further work-group fits).  256 x 256 is the fastest per product in half precision (1500 TFLOP/s against 1280 and 850 of
// the other two, all compute units busy) and has the longest start and end; in fp32 128 x 128 and 64 x 128 reach 150 and 138
// TFLOP/s and there is no larger one.
struct TileCost { double tile[3], first, further, part; };
constexpr TileCost kHalfCost[3] = {{{1.38, 0, 0}, 12.0, 9.0, 5.0}, {{0.57, 0.88, 0}, 6.0, 3.0, 0}, {{0.45, 0.64, 1.0}, 4.0, 3.0, 0}};
constexpr TileCost kF32Cost[3] = {{}, {{1.80, 3.58, 0}, 10.0, 4.5, 0}, {{1.25, 1.95, 2.9}, 6.5, 3.0, 0}};
constexpr int kUnits = 256;  // compute units

// cuts of k that are looked at
constexpr int kCuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256, 384, 512};

// a product: M x wide of the result, K the sum's length in k tiles
struct Product {
    int64_t M, wide, steps;
};

// the partial sums' launch, and their way to the caches and back
double join_cost(const Product& p, int64_t split) { return split > 1 ? (double)split * (double)p.M * (double)p.wide * 8.0 / 8.0e6 : 0.0; }

void set_cut(Plan* plan, const Product& p, int tile, int64_t split, int64_t per, int64_t part_ld, int64_t bk) {
    plan->tile = tile;
    plan->split = (int)split;
    plan->kper = (int)(per * bk);
    plan->tiles_m = (int)div_up(p.M, kTileM[tile]);
    plan->tiles_n = (int)div_up(p.wide, kTileN[tile]);
    plan->part_ld = part_ld;
    plan->bytes = split > 1 ? (size_t)split * (size_t)p.M * (size_t)part_ld * 4 : 0;
}

// M x N of the result (gated: N columns of y), K the sum's length: the tile and the cut of K with the smallest estimate
Plan plan_gemm(int64_t M, int64_t N, int64_t K, bool gated, Layout lay, int es) {
    const int64_t bk = kTileBytes / es;
    const Product p{M, gated ? 2 * N : N, div_up(K, bk)};
    const int64_t part_ld = gated ? 2 * round8(N) : round8(N);
    const TileCost* const cost = es == 4 ? kF32Cost : kHalfCost;
    Plan best{};
    best.t = 1e300;
    for (int tile = es == 4 ? 1 : 0; tile < 3; ++tile) {
        const TileCost& c = cost[tile];
        const int64_t tiles = div_up(p.M, kTileM[tile]) * div_up(p.wide, kTileN[tile]);
        if (tiles >= kMaxGroups) continue;
        const int fit = tile == 0 ? 1 : tile == 1 || lay == L_KK ? 2 : 3;  // work-groups that share a compute unit
        for (const int cut : kCuts) {
            if (cut > 1 && (p.steps < 2 * cut || tiles * cut > 4 * kUnits)) break;
            const int64_t per = div_up(p.steps, cut), split = div_up(p.steps, per);
            const int64_t wgs = tiles * split, full = wgs / (kUnits * fit), rest = wgs % (kUnits * fit);
            double t = (double)full * ((double)per * c.tile[fit - 1] + c.further) + c.first - c.further;
            if (rest) t += (double)per * c.tile[(rest - 1) / kUnits] + c.further;
            if (split > 1) t += 4.0 + c.part + join_cost(p, split);
            if (t < best.t) {
                best.t = t;
                set_cut(&best, p, tile, split, per, part_ld, bk);
            }
        }
    }
    return best;
}

// na jobs of `a` us, then nb of `b` us, each on the place that is free first
double makespan(int64_t places, int64_t na, double a, int64_t nb, double b) {
    const int64_t full = na / places, rest = na % places;  // `rest` places take one more of the first kind
    const double late = (double)(full + (rest > 0)) * a, early = (double)full * a;
    double end = late;
    int64_t on_early = 0, on_late = 0;  // jobs of the second kind that one place has taken
    while (nb > 0) {
        const bool to_early = early + (double)on_early * b <= late + (double)on_late * b;
        nb -= to_early ? places - rest : rest;
        const double t = to_early ? early + (double)++on_early * b : late + (double)++on_late * b;
        end = t > end ? t : end;
    }
    return end;
}

// Both products of a backward call in one launch: one tile for both, cut so that no work-group walks over more than a given
// number of k tiles.  True, and the plans, if that is estimated to take less than one launch after the other.
bool plan_pair(const Product& px, const Product& pw, int64_t part_ld, int es, Plan* x, Plan* w) {
    const int64_t bk = kTileBytes / es;
    const TileCost* const cost = es == 4 ? kF32Cost : kHalfCost;
    double best = x->t + w->t;
    bool found = false;
    for (int tile = es == 4 ? 1 : 0; tile < 3; ++tile) {
        const TileCost& c = cost[tile];
        const int fit = tile + 1;
        const int64_t tx = div_up(px.M, kTileM[tile]) * div_up(px.wide, kTileN[tile]);
        const int64_t tw = div_up(pw.M, kTileM[tile]) * div_up(pw.wide, kTileN[tile]);
        for (const int most : kCuts) {
            const int64_t sx = div_up(px.steps, most), sw = div_up(pw.steps, most);
            if (most == 1 || sx > 128 || sw > 128 || tx * sx + tw * sw > 6 * kUnits) continue;
            const int64_t lx = div_up(px.steps, sx), lw = div_up(pw.steps, sw);
            const int64_t wgs = tx * sx + tw * sw;
            const int64_t res = div_up(wgs, kUnits) < fit ? div_up(wgs, kUnits) : fit;
            // dW's work-groups come first, dX's fill the places as they fall free
            const double per_tile = c.tile[res - 1];
            double t = makespan(kUnits * res, tw * sw, (double)lw * per_tile + c.further + (sw > 1 ? c.part : 0.0),
                                tx * sx, (double)lx * per_tile + c.further + (sx > 1 ? c.part : 0.0));
            t += c.first - c.further;
            if (sx > 1 || sw > 1) t += 4.0 + join_cost(px, sx) + join_cost(pw, sw);
            if (t < best) {
                best = t;
                found = true;
                set_cut(x, px, tile, sx, lx, part_ld, bk);
                set_cut(w, pw, tile, sw, lw, part_ld, bk);
            }
        }
    }
    return found;
}

// A matrix of the call that the products read where it stands, or packed (pack_rows)
struct Source {
    const void* p;
    int64_t ld;
};
bool good_rows(int64_t ld, int64_t cols, int es) { return (ld * es) % 16 == 0 && (cols * es) % 16 == 0; }
int64_t packed_ld(int64_t cols, int es) { return div_up(cols * es, 16) * 16 / es; }
size_t packed_bytes(int64_t rows, int64_t cols, int es) { return a256((size_t)rows * (size_t)packed_ld(cols, es) * (size_t)es); }

bool on_boundaries(const Shape& s) { return good_rows(s.ldx, s.K, s.es) && good_rows(s.ldw, s.K, s.es); }

// A forward call that is a pass over the weights, unless pointers are off 16-byte boundaries and the flag did not say so
bool no_plan(const Shape& s) { return s.M <= kSkinnyOddRows || (s.M <= kSkinnyRows && !s.off_boundary && on_boundaries(s)); }

// Room for packed x and w: where their rows are off 16-byte boundaries, or their pointers may be (flags)
size_t pack_room(const Shape& s) {
    const int64_t wide = s.gated ? 2 * s.N : s.N;
    return (s.off_boundary || !good_rows(s.ldx, s.K, s.es) ? packed_bytes(s.M, s.K, s.es) : 0) +
           (s.off_boundary || !good_rows(s.ldw, s.K, s.es) ? packed_bytes(wide, s.K, s.es) : 0);
}

// Where x and w are read by the products, packing those that have to be into `room`; returns the bytes used
size_t place_operands(const Shape& s, const void* x, const void* w, char* room, PackArgs* pk, Source* sx, Source* sw) {
    size_t used = 0;
    const int64_t wide = s.gated ? 2 * s.N : s.N;
    const auto place = [&](int i, const void* p, int64_t ld, int64_t rows, Source* out) {
        *out = Source{p, ld};
        if (!p || (on(p, 16) && good_rows(ld, s.K, s.es))) return;
        pk->src[i] = p; pk->dst[i] = room + used; pk->ld[i] = ld; pk->rows[i] = rows; pk->cols[i] = (int)s.K;
        *out = Source{room + used, packed_ld(s.K, s.es)};
        used += packed_bytes(rows, s.K, s.es);
    };
    place(0, x, s.ldx, s.M, sx);
    place(1, w, s.ldw, wide, sw);
    return used;
}

// workspace of a backward call: dz, the bias gradient's partial sums, one product's partial sums at a time, packed operands
struct BackPlan {
    int64_t ld_dz;
    int row_blocks, rows_per_block;
    int64_t sums_ld;
    Plan x, w;     // one launch after the other, in one piece of the workspace
    bool both;     // in one launch, in two pieces
    Plan bx, bw;
    size_t off_sums, off_part, off_pack, total;
};

BackPlan plan_back(const Shape& s) {
    BackPlan b;
    const int64_t wide = s.gated ? 2 * s.N : s.N;
    b.ld_dz = round8(wide);
    b.sums_ld = b.ld_dz;
    const int64_t cols = div_up(s.N, 256);
    // about eight work-groups of eight wavefronts a compute unit; no more than 256 blocks of rows, whose sums the last launch
    // adds up with all loads in flight
    int64_t blocks = div_up(2048, cols);
    if (blocks > 256) blocks = 256;
    if (blocks > div_up(s.M, kDzRows)) blocks = div_up(s.M, kDzRows);
    if (blocks < 1) blocks = 1;
    b.rows_per_block = (int)(div_up(div_up(s.M, blocks), kDzRows) * kDzRows);
    b.row_blocks = b.rows_per_block ? (int)div_up(s.M, b.rows_per_block) : 0;
    b.off_sums = a256((size_t)s.M * (size_t)b.ld_dz * (size_t)s.es);
    b.off_part = b.off_sums + a256((size_t)b.row_blocks * (size_t)b.sums_ld * 4);
    b.x = plan_gemm(s.M, s.K, wide, false, L_KT, s.es);
    b.w = plan_gemm(wide, s.K, s.M, false, L_TT, s.es);
    b.bx = b.x;
    b.bw = b.w;
    const int64_t bk = kTileBytes / s.es;
    b.both = plan_pair(Product{s.M, s.K, div_up(wide, bk)}, Product{wide, s.K, div_up(s.M, bk)}, round8(s.K), s.es, &b.bx, &b.bw);
    const size_t one = a256(b.x.bytes > b.w.bytes ? b.x.bytes : b.w.bytes), two = b.both ? a256(b.bx.bytes) + a256(b.bw.bytes) : 0;
    b.off_pack = b.off_part + (one > two ? one : two);
    b.total = b.off_pack + pack_room(s);
    return b;
}

void set_plan(GemmArgs* g, const Plan& p, void* part) {
    g->kper = p.kper; g->split = p.split; g->tiles_m = p.tiles_m; g->tiles_n = p.tiles_n;
    g->part = static_cast<float*>(part);
    g->part_ld = p.part_ld;
}

// the product's partial sums to put together (none if k was not cut)
JoinArgs join_of(const GemmArgs& g, bool gated) {
    return g.split > 1 ? JoinArgs{g.part, g.part_ld, g.M, g.split, gated ? 1 : 0, g.e} : JoinArgs{};
}

// The product; sums: what the last launch adds up besides (n = 0: nothing)
template <typename T>
int run_gemm(GemmArgs g, const Plan& p, Layout lay, bool gated, void* part, const SumArgs& sums, hipStream_t st) {
    set_plan(&g, p, part);
    if (DenseOps<T>::gemm(g, lay, gated, p.tile, st) != hipSuccess) return DLC_EHIP;
    if (g.split > 1 || sums.n > 0)
        if (DenseOps<T>::join(join_of(g, gated), JoinArgs{}, sums, st) != hipSuccess) return DLC_EHIP;
    return DLC_OK;
}

template <typename T>
int forward(const dlc_dense_config* c, const Shape& s, const void* x, const void* w, const void* bias, const void* res, void* y,
            void* pre, void* work, size_t work_bytes, Plan plan, hipStream_t st) {
    GemmArgs g{};
    g.a = x; g.b = w; g.lda = s.ldx; g.ldb = s.ldw;
    g.M = (int)s.M; g.N = (int)s.N; g.K = (int)s.K;
    g.split = 1; g.kper = g.K;
    Epi& e = g.e;
    e.y = y; e.pre = pre; e.res = res; e.bias = bias;
    e.ld_y = s.ldy; e.ld_pre = s.ldpre; e.ld_res = s.ldres;
    e.seed = c->seed; e.offset = c->offset; e.d_offset = c->d_offset;
    e.thr = s.thr; e.scale = s.scale; e.act = c->act; e.n = (int)s.N;
    // few rows: a pass over the weights (32 rows of 2048 -> 4096 bf16: 10.3 us in tiles)
    if (s.M <= kSkinnyRows) {
        const bool aligned = on(x, 16) && on(w, 16) && on_boundaries(s);
        if (aligned || s.M <= kSkinnyOddRows) return DenseOps<T>::skinny(g, s.gated, aligned, st) == hipSuccess ? DLC_OK : DLC_EHIP;
        if (no_plan(s)) plan = plan_gemm(s.M, s.N, s.K, s.gated, L_KK, s.es);  // (only the pointers are off, and no flag said so)
    }
    const size_t part = a256(plan.bytes);
    PackArgs pk{};
    Source sx, sw;
    const size_t used = place_operands(s, x, w, static_cast<char*>(work) + part, &pk, &sx, &sw);
    if (part + used > work_bytes) return DLC_ECAPACITY;
    if (used && DenseOps<T>::pack(pk, st) != hipSuccess) return DLC_EHIP;
    g.a = sx.p; g.lda = sx.ld; g.b = sw.p; g.ldb = sw.ld;
    return run_gemm<T>(g, plan, L_KK, s.gated, work, SumArgs{}, st);
}

template <typename T>
int backward(const dlc_dense_config* c, const Shape& s, const void* x, const void* w, const void* pre, const void* dy, void* dx,
             void* dw, void* dbias, void* work, size_t work_bytes, const BackPlan& b, hipStream_t st) {
    char* const wk = static_cast<char*>(work);
    const int64_t wide = s.gated ? 2 * s.N : s.N;
    const bool same = !s.gated && c->act == DLC_ACT_NONE && s.thr == 0;  // dz is dy
    const bool direct = same && rows16(dy, s.lddy, s.es) && (s.N * s.es) % 16 == 0;
    const bool products = (dx || dw) && s.M > 0;
    float* const sums = reinterpret_cast<float*>(wk + b.off_sums);
    PackArgs pk{};
    Source sx{}, sw{};
    size_t used = 0;
    if (products) {
        used = place_operands(s, dw ? x : nullptr, dx ? w : nullptr, wk + b.off_pack, &pk, &sx, &sw);
        if (b.off_pack + used > work_bytes) return DLC_ECAPACITY;
    }
    const bool elementwise = s.M > 0 && (dbias || (products && !direct));
    if (used && !elementwise && DenseOps<T>::pack(pk, st) != hipSuccess) return DLC_EHIP;
    if (elementwise) {
        DzArgs d{};
        d.dy = dy; d.pre = same ? nullptr : pre;
        if (!s.gated && c->act == DLC_ACT_NONE) d.pre = nullptr;
        d.dz = products && !direct ? work : nullptr;
        d.sums = dbias ? sums : nullptr;
        d.ld_dy = s.lddy; d.ld_pre = s.ldpre; d.ld_dz = b.ld_dz; d.sums_ld = b.sums_ld;
        d.M = s.M; d.n = (int)s.N; d.gated = s.gated; d.act = c->act;
        d.row_blocks = b.row_blocks; d.rows_per_block = b.rows_per_block;
        d.thr = s.thr; d.scale = s.scale; d.seed = c->seed; d.offset = c->offset; d.d_offset = c->d_offset;
        if (DenseOps<T>::dz(d, pk, st) != hipSuccess) return DLC_EHIP;
    }
    // the bias gradient's sums are put together by the call's last launch, whichever it is
    const SumArgs sum = dbias ? SumArgs{sums, b.sums_ld, s.M > 0 ? b.row_blocks : 0, (int)wide, dbias} : SumArgs{};
    const void* const dz = direct ? dy : work;
    const int64_t lddz = direct ? s.lddy : b.ld_dz;
    GemmArgs gx{}, gw{};
    gx.a = dz; gx.b = sw.p; gx.lda = lddz; gx.ldb = sw.ld;
    gx.M = (int)s.M; gx.N = (int)s.K; gx.K = (int)wide;
    gx.e.y = dx; gx.e.ld_y = s.lddx; gx.e.n = (int)s.K;
    gw.a = dz; gw.b = sx.p; gw.lda = lddz; gw.ldb = sx.ld;
    gw.M = (int)wide; gw.N = (int)s.K; gw.K = (int)s.M;
    gw.e.y = dw; gw.e.ld_y = s.lddw; gw.e.n = (int)s.K;
    const auto join = [&](const JoinArgs& ja, const JoinArgs& jb) { return DenseOps<T>::join(ja, jb, sum, st) == hipSuccess ? DLC_OK : DLC_EHIP; };
    if (s.M == 0) {  // (an empty sum: a product with no cut at all, as many rows at a time as a launch has threads for)
        const int64_t most = kMaxGroups / 2 * 256 / div_up(s.K, 8);
        for (int64_t r = 0; dw && r < wide; r += most) {
            JoinArgs j{nullptr, 0, (int)(wide - r < most ? wide - r : most), 0, 0, gw.e};
            j.e.y = static_cast<char*>(dw) + r * s.lddw * s.es;
            if (DenseOps<T>::join(j, JoinArgs{}, SumArgs{}, st) != hipSuccess) return DLC_EHIP;
        }
        return dbias ? join(JoinArgs{}, JoinArgs{}) : DLC_OK;
    }
    if (dx && dw && b.both) {
        set_plan(&gx, b.bx, wk + b.off_part);
        set_plan(&gw, b.bw, wk + b.off_part + a256(b.bx.bytes));
        const bool cut = gx.split > 1 || gw.split > 1;
        if (DenseOps<T>::back(gx, gw, cut ? SumArgs{} : sum, b.bx.tile, st) != hipSuccess) return DLC_EHIP;
        return cut ? join(join_of(gx, false), join_of(gw, false)) : DLC_OK;
    }
    if (dx)
        if (const int rc = run_gemm<T>(gx, b.x, L_KT, false, wk + b.off_part, dw ? SumArgs{} : sum, st); rc != DLC_OK) return rc;
    if (dw) return run_gemm<T>(gw, b.w, L_TT, false, wk + b.off_part, sum, st);
    return dbias && !dx ? join(JoinArgs{}, JoinArgs{}) : DLC_OK;
}

// d is there if `need`, and lies on an element's boundary
bool good_ptr(const void* d, int es, bool need) { return d ? on(d, es) : !need; }

// y may take the place of `in` element for element, not with other distances from row to row
bool good_place(const void* in, int64_t ld_in, const void* y, int64_t ld_y, int64_t rows) { return in != y || ld_in == ld_y || rows <= 1; }

// the workspace a forward call needs: the product's partial sums, packed operands (a pass over few rows takes them as they are)
size_t forward_bytes(const Shape& s, const Plan& p) { return no_plan(s) ? 0 : a256(p.bytes) + pack_room(s); }

Plan plan_forward(const Shape& s) { return no_plan(s) ? Plan{} : plan_gemm(s.M, s.N, s.K, s.gated, L_KK, s.es); }

int check_work(size_t need, const void* work, size_t* bytes) {
    if (!on(work, 16)) return DLC_EINVAL;
    if (!work) *bytes = 0;
    return *bytes >= need ? DLC_OK : work ? DLC_ECAPACITY : DLC_EINVAL;
}

int forward_any(const dlc_dense_config* c, bool gated, const void* x, const void* w, const void* bias, const void* res, void* y,
                void* pre, void* work, size_t bytes, void* stream) {
    Shape s;
    if (!make_shape(c, gated, &s)) return DLC_EINVAL;
    const bool need = s.M > 0;
    if (!good_ptr(x, s.es, need) || !good_ptr(w, s.es, need) || !good_ptr(bias, s.es, false) || !good_ptr(res, s.es, false) ||
        !good_ptr(y, s.es, need) || !good_ptr(pre, s.es, false) || !on(c->d_offset, 8)) return DLC_EINVAL;
    if (!need) return DLC_OK;
    if (!good_place(res, s.ldres, y, s.ldy, s.M)) return DLC_EINVAL;
    const Plan p = plan_forward(s);
    if (const int rc = check_work(forward_bytes(s, p), work, &bytes); rc != DLC_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    switch (c->dtype) {
        case DLC_F32: return forward<float>(c, s, x, w, bias, res, y, pre, work, bytes, p, st);
        case DLC_F16: return forward<f16_t>(c, s, x, w, bias, res, y, pre, work, bytes, p, st);
        default: return forward<bf16_t>(c, s, x, w, bias, res, y, pre, work, bytes, p, st);
    }
}

int backward_any(const dlc_dense_config* c, bool gated, const void* x, const void* w, const void* pre, const void* dy, void* dx,
                 void* dw, void* dbias, void* work, size_t bytes, void* stream) {
    Shape s;
    if (!make_shape(c, gated, &s)) return DLC_EINVAL;
    const bool some = s.M > 0;
    if (!good_ptr(x, s.es, some && dw) || !good_ptr(w, s.es, some && dx) || !good_ptr(dy, s.es, some) ||
        !good_ptr(pre, s.es, some && (gated || c->act != DLC_ACT_NONE)) || !good_ptr(dx, s.es, false) || !good_ptr(dw, s.es, false) ||
        !good_ptr(dbias, s.es, false) || !on(c->d_offset, 8)) return DLC_EINVAL;
    const BackPlan p = some ? plan_back(s) : BackPlan{};
    if (const int rc = check_work(p.total, work, &bytes); rc != DLC_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    switch (c->dtype) {
        case DLC_F32: return backward<float>(c, s, x, w, pre, dy, dx, dw, dbias, work, bytes, p, st);
        case DLC_F16: return backward<f16_t>(c, s, x, w, pre, dy, dx, dw, dbias, work, bytes, p, st);
        default: return backward<bf16_t>(c, s, x, w, pre, dy, dx, dw, dbias, work, bytes, p, st);
    }
}

}  // namespace

static size_t workspace(const dlc_dense_config* cfg, bool gated, int backward) {
    Shape s;
    if (!make_shape(cfg, gated, &s) || s.M == 0) return 0;
    return backward ? plan_back(s).total : forward_bytes(s, plan_forward(s));
}
extern "C" size_t dlc_linear_workspace_bytes(const dlc_dense_config* cfg, int backward) { return workspace(cfg, false, backward); }
extern "C" size_t dlc_gated_workspace_bytes(const dlc_dense_config* cfg, int backward) { return workspace(cfg, true, backward); }

extern "C" int dlc_linear_forward(const dlc_dense_config* cfg, const void* x, const void* w, const void* bias, const void* res, void* y,
                                  void* pre, void* work, size_t bytes, void* stream) {
    return forward_any(cfg, false, x, w, bias, res, y, pre, work, bytes, stream);
}

extern "C" int dlc_linear_backward(const dlc_dense_config* cfg, const void* x, const void* w, const void* pre, const void* dy, void* dx,
                                   void* dw, void* dbias, void* work, size_t bytes, void* stream) {
    return backward_any(cfg, false, x, w, pre, dy, dx, dw, dbias, work, bytes, stream);
}

extern "C" int dlc_gated_forward(const dlc_dense_config* cfg, const void* x, const void* w, const void* bias, void* y, void* pre,
                                 void* work, size_t bytes, void* stream) {
    return forward_any(cfg, true, x, w, bias, nullptr, y, pre, work, bytes, stream);
}

extern "C" int dlc_gated_backward(const dlc_dense_config* cfg, const void* x, const void* w, const void* pre, const void* dy, void* dx,
                                  void* dw, void* dbias, void* work, size_t bytes, void* stream) {
    return backward_any(cfg, true, x, w, pre, dy, dx, dw, dbias, work, bytes, stream);
}

extern "C" int dlc_dropout(const dlc_dropout_config* c, const void* x, const void* res, void* y, void* stream) {
    if (!c || (c->dtype != DLC_F32 && c->dtype != DLC_F16 && c->dtype != DLC_BF16) || c->reserved != 0) return DLC_EINVAL;
    if (c->rows < 0 || c->rows > kMaxRows || c->cols < 1 || c->cols > 0x7FFFFFF8ll) return DLC_EINVAL;
    DropArgs d{};
    d.rows = c->rows; d.cols = (int)c->cols;
    d.ld_x = c->ld_x ? c->ld_x : c->cols;
    d.ld_res = c->ld_res ? c->ld_res : c->cols;
    d.ld_y = c->ld_y ? c->ld_y : c->cols;
    if (d.ld_x < c->cols || d.ld_res < c->cols || d.ld_y < c->cols) return DLC_EINVAL;
    if (!dropout_params(c->dropout_p, &d.thr, &d.scale)) return DLC_EINVAL;
    const int es = c->dtype == DLC_F32 ? 4 : 2;
    const int64_t lim = int64_t(1) << 60;  // (a buffer's last byte has a 64-bit address)
    const int64_t ldm = d.ld_x > d.ld_y ? (d.ld_x > d.ld_res ? d.ld_x : d.ld_res) : (d.ld_y > d.ld_res ? d.ld_y : d.ld_res);
    if (c->rows > 0 && ldm > lim / c->rows) return DLC_EINVAL;
    const bool need = c->rows > 0;
    if (!good_ptr(x, es, need) || !good_ptr(res, es, false) || !good_ptr(y, es, need) || !on(c->d_offset, 8)) return DLC_EINVAL;
    if (!need) return DLC_OK;
    if (!good_place(x, d.ld_x, y, d.ld_y, c->rows) || !good_place(res, d.ld_res, y, d.ld_y, c->rows)) return DLC_EINVAL;
    d.x = x; d.res = res; d.y = y;
    d.seed = c->seed; d.offset = c->offset; d.d_offset = c->d_offset;
    hipStream_t st = (hipStream_t)stream;
    hipError_t rc;
    switch (c->dtype) {
        case DLC_F32: rc = DenseOps<float>::drop(d, st); break;
        case DLC_F16: rc = DenseOps<f16_t>::drop(d, st); break;
        default: rc = DenseOps<bf16_t>::drop(d, st); break;
    }
    return rc == hipSuccess ? DLC_OK : DLC_EHIP;
}
