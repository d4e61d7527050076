// Matrices to microscaled form and back, and the host side of the product of microscaled operands.
#include "dlc_mx_gemm.h"

using namespace dlc;

namespace {

struct MxArgs {
    const void* x;       // the ordinary matrix (back: y)
    uint8_t* q;
    uint8_t* scale;
    int64_t rows, ld, tiles;
    int32_t cols, groups;
};

constexpr int kAhead = 4;  // rows of a lane, whose loads are on their way together

// A work-group's tile and a lane's part of it: L lanes have a row, or 512 columns of it; 64 / L rows side by side
template <int L>
struct Part {
    static constexpr int ROWS = 4 * kAhead * 64 / L;  // of a tile
    static constexpr int STEP = 64 / L;               // from a lane's row to its next
    int64_t row;
    int group, col;
    __device__ __forceinline__ Part(int64_t tile, int groups) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int64_t band = L < 64 ? tile : tile / groups;
        row = band * ROWS + wave * (kAhead * STEP) + lane / L;
        group = L < 64 ? 0 : (int)(tile - band * groups);
        col = group * kMxGroup + lane % L * 8;
    }
};

// A tile is a group of 512 columns, eight a lane, of 16 rows: their scales are 256 bytes side by side.  Rows of at most 128
// columns: 64 of them, on 16 lanes each (65536 x 128 bf16 into 8 bits 5.6 us, back 6.1; on 64 lanes 10.4 and 8.4).  Bound by
// memory: 16384 x 4096 bf16 into 4 bits 31 us and back 26 (170 MB, 5.5 and 6.6 TB/s), 8192 x 8192 into 8 bits 32 and 30 (6.3 and
// 6.7 TB/s).  Rows that end inside an eight may be loaded element by element here: the row's last eight instead, as in the norm,
// took as long (8192 x 4099 bf16 20.5 us; with 4096 columns 18.5).  WHOLE: rows end with a whole eight
template <typename T, int ELEM, bool WHOLE, int L>
__global__ __launch_bounds__(256) void k_mx_quantize(const MxArgs a) {
    for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const Part<L> at(tile, a.groups);
        Raw8<T> x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t row = at.row + i * at.STEP;
            const T* const p = static_cast<const T*>(a.x) + row * a.ld + at.col;
            if constexpr (WHOLE) x[i].load_whole(p, row < a.rows && at.col < a.cols);
            else x[i].load(p, row < a.rows ? a.cols - at.col : 0);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t row = at.row + i * at.STEP;
            float f[8];
            x[i].get(f);
            if (row < a.rows) mx_store8<ELEM, (L < 64)>(f, 0, row, at.col, a.cols, a.rows, a.q, a.scale);
        }
    }
}

template <typename T, int ELEM, bool WHOLE, int L>
__global__ __launch_bounds__(256) void k_mx_dequantize(const MxArgs a) {
    const int64_t row_bytes = mx_row_bytes(a.cols, ELEM);
    for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const Part<L> at(tile, a.groups);
        const int cnt = a.cols - at.col;
        if (cnt <= 0) continue;
        MxWords<ELEM> w[kAhead];
        uint32_t byte[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t row = min(at.row + i * at.STEP, a.rows - 1);
            w[i] = *reinterpret_cast<const MxWords<ELEM>*>(a.q + row * row_bytes + at.col * ELEM / 8);
            byte[i] = a.scale[((int64_t)at.group * a.rows + row) * 16 + mx_scale_place(at.col / kMxBlock)];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t row = at.row + i * at.STEP;
            if (row >= a.rows) continue;
            float f[8];
            mx_decode8<ELEM>(w[i], byte[i], f);
            store8(static_cast<T*>(const_cast<void*>(a.x)) + row * a.ld + at.col, WHOLE ? 8 : cnt, f);
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------
constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxDim = int64_t(1) << 20;
constexpr int64_t kMaxGroups = int64_t(1) << 24;  // a launch's threads, work-groups of 256, are counted in 32 bits

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool on(const void* p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }
bool good(const void* p, int es, bool need) { return p ? on(p, es) : !need; }
bool good_type(int t) { return t == DLC_F32 || t == DLC_F16 || t == DLC_BF16; }
bool good_elem(int e) { return e == DLC_MX_E2M1 || e == DLC_MX_E4M3; }

bool good_mx(const dlc_mx_config* c) {
    if (!c || !good_type(c->dtype) || !good_elem(c->elem)) return false;
    if (c->rows < 0 || c->rows > kMaxRows || c->cols < 1 || c->cols > kMaxDim) return false;
    const int64_t lim = c->rows > 0 ? (int64_t(1) << 60) / c->rows : int64_t(1) << 60;  // (a buffer's last byte has a 64-bit address)
    for (const int64_t ld : {c->ld_x, c->ld_y})
        if (ld != 0 && (ld < c->cols || ld > lim)) return false;
    return true;
}

template <typename T, int ELEM, bool WHOLE, int L>
void convert(MxArgs a, bool back, hipStream_t st) {
    a.tiles = div_up(a.rows, Part<L>::ROWS) * a.groups;
    const dim3 grid((unsigned)(a.tiles < (int64_t(1) << 20) ? a.tiles : int64_t(1) << 20)), block(256);
    if (back) k_mx_dequantize<T, ELEM, WHOLE, L><<<grid, block, 0, st>>>(a);
    else k_mx_quantize<T, ELEM, WHOLE, L><<<grid, block, 0, st>>>(a);
}

template <typename T, int ELEM>
void convert(const MxArgs& a, bool back, hipStream_t st) {
    const bool whole = a.cols % 8 == 0;
    if (a.cols <= kMxFill) whole ? convert<T, ELEM, true, 16>(a, back, st) : convert<T, ELEM, false, 16>(a, back, st);
    else whole ? convert<T, ELEM, true, 64>(a, back, st) : convert<T, ELEM, false, 64>(a, back, st);
}

template <typename T>
void convert(const MxArgs& a, int elem, bool back, hipStream_t st) {
    elem == DLC_MX_E4M3 ? convert<T, 8>(a, back, st) : convert<T, 4>(a, back, st);
}

int convert_any(const dlc_mx_config* c, const void* x, const void* q, const void* scale, bool back, void* stream) {
    if (!good_mx(c)) return DLC_EINVAL;
    const int es = c->dtype == DLC_F32 ? 4 : 2;
    const bool need = c->rows > 0;
    if (!good(x, es, need) || !good(q, 16, need) || !good(scale, 16, need)) return DLC_EINVAL;
    if (!need) return DLC_OK;
    MxArgs a{};
    a.x = x; a.q = static_cast<uint8_t*>(const_cast<void*>(q)); a.scale = static_cast<uint8_t*>(const_cast<void*>(scale));
    a.rows = c->rows; a.cols = (int)c->cols;
    a.ld = back ? c->ld_y : c->ld_x;
    if (a.ld == 0) a.ld = c->cols;
    a.groups = (int)mx_groups(c->cols);
    hipStream_t st = (hipStream_t)stream;
    switch (c->dtype) {
        case DLC_F32: convert<float>(a, c->elem, back, st); break;
        case DLC_F16: convert<f16_t>(a, c->elem, back, st); break;
        default: convert<bf16_t>(a, c->elem, back, st); break;
    }
    return hipGetLastError() == hipSuccess ? DLC_OK : DLC_EHIP;
}

// ---- the product ---------------------------------------------------------------------------------
struct Shape {
    int64_t M, K, N, ldy, ldres;
    int elem, es;
};

bool make_shape(const dlc_mx_linear_config* c, Shape* s) {
    if (!c || !good_type(c->dtype) || !good_elem(c->elem_x) || c->act < DLC_ACT_NONE || c->act > DLC_ACT_GELU || c->reserved != 0) return false;
    if (c->rows < 0 || c->rows > kMaxRows) return false;
    if (c->in_features < 1 || c->in_features > kMaxDim || c->out_features < 1 || c->out_features > kMaxDim) return false;
    s->M = c->rows; s->K = c->in_features; s->N = c->out_features;
    s->ldy = c->ld_y ? c->ld_y : s->N;
    s->ldres = c->ld_res ? c->ld_res : s->N;
    if (s->ldy < s->N || s->ldy > kMaxDim || s->ldres < s->N || s->ldres > kMaxDim) return false;
    s->elem = c->elem_x;
    s->es = c->dtype == DLC_F32 ? 4 : 2;
    // (some tile's launch covers the result: the largest, which fp32 results of E4M3 have not)
    const int64_t side = s->elem == DLC_MX_E4M3 && s->es == 4 ? 128 : 256;
    return div_up(s->M, side) * div_up(s->N, side) < kMaxGroups;
}

struct Plan {
    int tile, split, kper, tiles_m, tiles_n;
    int64_t part_ld;
    size_t bytes;  // of the partial sums
};

// What 256 k values cost with 1 and 2 work-groups on a compute unit, in us, what a work-group costs besides, and every
// further one, measured on full cards (0: no second work-group fits; up to half of a card, whose work-groups have more of the
// caches and the power, kHalf of it): E2M1, E4M3, E4M3 with results in fp32.  64 x 128 is the best of the tiles until its tiles no longer fit
// the card at once (1024 x 2048 x 2048 of 4 bits 8.1 us for 10.3 and 22; 2048 x 2048 x 2048 12.3, 11.1 and 22.7, of 8 bits 17.3,
// 13.9 and 29.4), 256 x 256 where there are many (2048 x 8192 x 8192 of 4 bits 120, 98 and 66 us).
struct TileCost { double tile[2], first, further; };
constexpr TileCost kCost[3][3] = {{{{1.66, 0}, 12.8, 11.0}, {{0.64, 0}, 5.8, 3.7}, {{0.46, 0.86}, 4.4, 2.0}},
                                  {{{2.42, 0}, 13.6, 8.3}, {{0.89, 0}, 6.6, 4.2}, {{0.6, 0}, 4.6, 2.6}},
                                  {{}, {{2.2, 0}, 5.5, 3.5}, {{1.45, 0}, 4.2, 2.4}}};
constexpr double kHalf = 0.85;

// Few rows: a round of work-groups (a band of 32 rows and 16 columns each, one on a compute unit) with 1024 k values, what the
// first round costs besides and every further one; the kinds as above.  64 x 2048 -> 2048 of 4 bits 4.0 us, 7.4 the best of the
// tiles; 64 x 8192 -> 2048 5.8 and 10.4; 128 x 8192 -> 2048 in two rounds 9.7 and 12.0; 64 x 65536 -> 2048 22.9 and 19.8.
struct SkinnyCost { double k, first, further; };
constexpr SkinnyCost kSkinnyCost[3] = {{0.30, 3.4, 1.5}, {0.44, 4.1, 1.9}, {0.50, 4.2, 2.2}};
constexpr int kSkinnyRounds = 4;
constexpr int kUnits = 256;  // compute units
constexpr int kCuts[] = {1, 2, 3, 4, 6, 8, 12, 16};

// The tile and the cut of k with the smallest estimate
Plan plan_linear(const Shape& s) {
    Plan best{};
    best.split = 1;
    best.tile = kMxSkinny;
    if (s.M <= kMxSkinnyRows / 2) return best;
    const int64_t groups = mx_groups(s.K);
    const bool exact = s.elem == DLC_MX_E4M3 && s.es == 4;
    const int kind = exact ? 2 : s.elem == DLC_MX_E4M3 ? 1 : 0;
    const TileCost* const cost = kCost[kind];
    double least = 1e300;
    const int64_t rounds = div_up(div_up(s.M, kMxSkinnyRows) * div_up(s.N, 16), kUnits);
    if (rounds <= kSkinnyRounds) {
        const SkinnyCost& c = kSkinnyCost[kind];
        least = c.first + (double)rounds * (double)s.K / 1024.0 * c.k + (double)(rounds - 1) * c.further;
    }
    for (int tile = exact ? 1 : 0; tile < 3; ++tile) {
        const TileCost& c = cost[tile];
        const int64_t tm = div_up(s.M, kMxTileM[tile]), tn = div_up(s.N, kMxTileN[tile]), tiles = tm * tn;
        if (tiles >= kMaxGroups) continue;
        const int fit = c.tile[1] > 0 ? 2 : 1;
        for (const int cut : kCuts) {
            if (cut > 1 && (cut > groups || tiles * cut > 2 * kUnits)) break;
            const int64_t per = div_up(groups, cut), split = div_up(groups, per), wgs = tiles * split;
            const int64_t full = wgs / (kUnits * fit), rest = wgs % (kUnits * fit);
            double t = (double)full * (2.0 * (double)per * c.tile[fit - 1] + c.further) + c.first - c.further;
            if (rest) t += 2.0 * (double)per * c.tile[(rest - 1) / kUnits] * (wgs <= kUnits / 2 ? kHalf : 1.0) + c.further;
            if (split > 1) t += 3.8 + (double)split * (double)s.M * (double)s.N * 8.0 / 6.2e6;  // (the second launch, the sums out and in)
            if (t < least) {
                least = t;
                best.tile = tile;
                best.split = (int)split;
                best.kper = (int)(per * kMxGroup);
                best.tiles_m = (int)tm;
                best.tiles_n = (int)tn;
            }
        }
    }
    best.part_ld = round8(s.N);
    best.bytes = best.split > 1 ? (size_t)best.split * (size_t)s.M * (size_t)best.part_ld * 4 : 0;
    return best;
}

template <typename T>
int product(MxGemmArgs g, const Plan& p, int elem, void* work, hipStream_t st) {
    g.c.split = p.split; g.c.kper = p.kper; g.c.tiles_m = p.tiles_m; g.c.tiles_n = p.tiles_n;
    g.c.part = static_cast<float*>(work);
    g.c.part_ld = p.part_ld;
    if (MxOps<T>::gemm(g, elem, p.tile, st) != hipSuccess) return DLC_EHIP;
    if (p.split == 1) return DLC_OK;
    const JoinArgs j{g.c.part, g.c.part_ld, g.c.M, g.c.split, 0, g.c.e};
    return DenseOps<T>::join(j, JoinArgs{}, SumArgs{}, st) == hipSuccess ? DLC_OK : DLC_EHIP;
}

}  // namespace

extern "C" size_t dlc_mx_data_bytes(const dlc_mx_config* c) { return good_mx(c) ? (size_t)c->rows * (size_t)mx_row_bytes(c->cols, c->elem) : 0; }
extern "C" size_t dlc_mx_scale_bytes(const dlc_mx_config* c) { return good_mx(c) ? (size_t)c->rows * (size_t)mx_groups(c->cols) * 16 : 0; }

extern "C" int dlc_mx_quantize(const dlc_mx_config* cfg, const void* x, void* q, void* scale, void* stream) {
    return convert_any(cfg, x, q, scale, false, stream);
}

extern "C" int dlc_mx_dequantize(const dlc_mx_config* cfg, const void* q, const void* scale, void* y, void* stream) {
    return convert_any(cfg, y, q, scale, true, stream);
}

extern "C" size_t dlc_mx_linear_workspace_bytes(const dlc_mx_linear_config* c) {
    Shape s;
    return make_shape(c, &s) && s.M > 0 ? plan_linear(s).bytes : 0;
}

extern "C" int dlc_mx_linear_forward(const dlc_mx_linear_config* c, const void* xq, const void* xs, const void* wq, const void* ws,
                                     const void* bias, const void* res, void* y, void* work, size_t bytes, void* stream) {
    Shape s;
    if (!make_shape(c, &s)) return DLC_EINVAL;
    const bool need = s.M > 0;
    if (!good(xq, 16, need) || !good(xs, 16, need) || !good(wq, 16, need) || !good(ws, 16, need) || !good(bias, s.es, false) ||
        !good(res, s.es, false) || !good(y, s.es, need) || !on(work, 16)) return DLC_EINVAL;
    if (!need) return DLC_OK;
    if (res == y && s.ldres != s.ldy && s.M > 1) return DLC_EINVAL;
    MxGemmArgs g{};
    g.xs = static_cast<const uint8_t*>(xs); g.ws = static_cast<const uint8_t*>(ws);
    g.c.a = xq; g.c.b = wq;
    g.c.lda = mx_row_bytes(s.K, s.elem); g.c.ldb = mx_row_bytes(s.K, DLC_MX_E2M1);
    g.c.M = (int)s.M; g.c.N = (int)s.N; g.c.K = (int)mx_filled(s.K);
    Epi& e = g.c.e;
    e.y = y; e.res = res; e.bias = bias;
    e.ld_y = s.ldy; e.ld_res = s.ldres; e.act = c->act; e.n = (int)s.N;
    const Plan p = plan_linear(s);
    if (p.bytes > 0 && !work) return DLC_EINVAL;
    if (bytes < p.bytes) return DLC_ECAPACITY;
    hipStream_t st = (hipStream_t)stream;
    switch (c->dtype) {
        case DLC_F32: return product<float>(g, p, s.elem, work, st);
        case DLC_F16: return product<f16_t>(g, p, s.elem, work, st);
        default: return product<bf16_t>(g, p, s.elem, work, st);
    }
}
