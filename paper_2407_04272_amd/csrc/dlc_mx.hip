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
// memory: 16384 x 4096 bf16 into 4 bits 34 us and back 35 (170 MB, 5.0 and 4.9 TB/s, as a copy), 8192 x 8192 into 8 bits 39 and 37
// (5.2 and 5.5 TB/s), eight inputs in turn; 29 and 26, 33 and 30 with one that the last cache still holds in part.  Right behind
// a call whose results are still on their way out of that cache it is slower: 16384 x 4096 there and back 40 + 26.
// Rows that end inside an eight may be loaded element by element here: the row's last eight instead, as in the norm,
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
    MxPlan plan() const { return mx_plan(M, K, N, elem == DLC_MX_E4M3, es == 4); }
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
    return div_up(s->M, side) * div_up(s->N, side) < kMxMaxTiles;
}

template <typename T>
int product(MxGemmArgs g, const MxPlan& p, int elem, void* work, hipStream_t st) {
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
    return make_shape(c, &s) && s.M > 0 ? s.plan().bytes : 0;
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
    const MxPlan p = s.plan();
    if (p.bytes > 0 && !work) return DLC_EINVAL;
    if (bytes < p.bytes) return DLC_ECAPACITY;
    hipStream_t st = (hipStream_t)stream;
    switch (c->dtype) {
        case DLC_F32: return product<float>(g, p, s.elem, work, st);
        case DLC_F16: return product<f16_t>(g, p, s.elem, work, st);
        default: return product<bf16_t>(g, p, s.elem, work, st);
    }
}
