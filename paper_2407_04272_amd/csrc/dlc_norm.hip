// Root-mean-square norm with the residual's addition, forward (results in the type, in microscaled form, or both) and backward.
//
// Bound by memory: every row is read once into registers, its sums are made there, and the results go out.  A team of P lanes
// has a row, U times eight columns a lane; rows longer than 16384 columns are read twice instead.  16384 x 8192 bf16: forward
// with a residual into 8 bits 164-169 us (944 MB, 5.6-5.8 TB/s), backward 193 (1074 MB, 5.6 TB/s).
#include "dlc_mx.h"

using namespace dlc;

namespace {

struct NormArgs {
    const void* x;       // backward: s
    const void* res;     // backward: the gradient along s
    const void* weight;
    const void* dy;
    void* sum;
    void* y;             // backward: dx
    uint8_t* q;
    uint8_t* scale;
    float* part;         // backward: [work-groups][part_ld] partial sums of the weight's gradient
    int64_t part_ld;
    int64_t rows, ld_x, ld_res, ld_sum, ld_y, ld_dy;
    int32_t cols, per;   // per: rows that a team takes one after the other
    float eps, inv_cols;
};

// The sum over a team of P lanes, the same in all of them.  More than a wavefront: over `red`, which is not written again
// before the barrier of the next sum but one.
template <int P, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float (*red)[N]) {
#pragma unroll
    for (int d = 1; d < (P < 64 ? P : 64); d <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d, 64);
    if constexpr (P > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[wave][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = red[0][i];
#pragma unroll
            for (int w = 1; w < P / 64; ++w) v[i] += red[w][i];
        }
    }
}

template <int P>
constexpr int kTeams = P < 256 ? 256 / P : 1;

// How rows end.  Whole: with a whole eight.  Back: not, but they have eight columns: the lane with the last ones takes the last
// eight instead, those that the lane before it has as well among them: they count once, and are stored twice alike.  Short rows
// alone are loaded and stored element by element: as code for all others it took registers and a wait for every element (8192 x
// 4099 bf16: forward 90 us for 47, into 8 bits 92 for 52, backward 93 for 60; with 4096 columns 39, 35 and 46).
enum Ends { kShort, kWhole, kBack };

// ... the first of a lane's columns
template <int E>
__device__ __forceinline__ int first_of(int col, int cols) {
    return E == kBack && col < cols ? min(col, cols - 8) : col;
}

// ... how many of them the lane before has as well
template <int E>
__device__ __forceinline__ int shared_of(int col, int cols) {
    return E == kBack ? max(col + 8 - cols, 0) : 0;
}

template <int E, typename T>
__device__ __forceinline__ void ask(Raw8<T>& q, const void* p, int64_t row, int64_t ld, int col, int cols) {
    const T* const at = static_cast<const T*>(p) + row * ld + first_of<E>(col, cols);
    if constexpr (E == kShort) q.load(at, cols - col);
    else q.load_whole(at, col < cols);
}

template <int E, typename T>
__device__ __forceinline__ void put(void* p, int64_t row, int64_t ld, int col, int cols, const float f[8]) {
    T* const at = static_cast<T*>(p) + row * ld + first_of<E>(col, cols);
    if constexpr (E == kShort) store8(at, cols - col, f);
    else if (col < cols) store8(at, 8, f);
}

template <typename T>
__device__ __forceinline__ void load_weight(const void* weight, int col, int cnt, float w[8]) {
    if (weight) {
        load8(static_cast<const T*>(weight) + col, cnt, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.0f;
    }
}

// s of eight columns, 0 behind the last
template <typename T>
__device__ __forceinline__ void load_sum(const NormArgs& a, int64_t row, int col, int cnt, float s[8]) {
    load8(static_cast<const T*>(a.x) + row * a.ld_x + col, cnt, s);
    if (a.res) {
        float r[8];
        load8(static_cast<const T*>(a.res) + row * a.ld_res + col, cnt, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += r[i];
    }
}

template <typename T, bool MX, int E, bool NARROW = false>
__device__ __forceinline__ void put_row(const NormArgs& a, int64_t row, int col, float r, float s[8], const float w[8]) {
    if (a.sum) put<E, T>(a.sum, row, a.ld_sum, col, a.cols, s);
    if (MX && col >= a.cols) r = 0.0f;  // (a row's NaN stays in its columns)
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = s[i] * r * w[i];
    if (a.y) put<E, T>(a.y, row, a.ld_y, col, a.cols, s);
    if constexpr (MX) mx_store8<8, NARROW>(s, shared_of<E>(col, a.cols), row, col, a.cols, a.rows, a.q, a.scale);
}

template <typename T, int P, int U, bool MX, int E>
__global__ __launch_bounds__(P < 256 ? 256 : P) void k_norm(const NormArgs a) {
    __shared__ float red[2][P > 64 ? P / 64 : 1][1];
    const int t = threadIdx.x % P, team = threadIdx.x / P;
    const int64_t first = ((int64_t)blockIdx.x * kTeams<P> + team) * a.per, last = min(a.rows, first + a.per);
    const int end = !MX ? a.cols : P == 16 ? kMxFill : (int)mx_groups(a.cols) * kMxGroup;
    int odd = 0;
    for (int64_t row = first; row < last; ++row, odd ^= 1) {
        float s[U][8], sq[1] = {0.0f};
        Raw8<T> x[U], res[U], w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (u * P + t) * 8;
            ask<E>(x[u], a.x, row, a.ld_x, col, a.cols);
        }
        if (a.res) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int col = (u * P + t) * 8;
                ask<E>(res[u], a.res, row, a.ld_res, col, a.cols);
            }
        }
        if (a.weight) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int col = (u * P + t) * 8;
                ask<E>(w[u], a.weight, 0, 0, col, a.cols);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u].get(s[u]);
            if (a.res) {
                float r[8];
                res[u].get(r);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[u][i] += r[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (E != kBack || i >= shared_of<E>((u * P + t) * 8, a.cols)) sq[0] += s[u][i] * s[u][i];
        }
        team_sum<P>(sq, red[odd]);
        const float r = __builtin_amdgcn_rsqf(sq[0] * a.inv_cols + a.eps);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (u * P + t) * 8;
            float g[8];
            w[u].get(g);
            if (!a.weight)
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = 1.0f;
            if (col < end) put_row<T, MX, E, P == 16>(a, row, col, r, s[u], g);
        }
    }
}

// ... rows of any length, read twice
template <typename T, bool MX>
__global__ __launch_bounds__(1024) void k_norm_long(const NormArgs a) {
    __shared__ float red[2][16][1];
    const int end = MX ? (int)mx_groups(a.cols) * kMxGroup : a.cols;
    int odd = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, odd ^= 1) {
        float sq[1] = {0.0f}, s[8];
        for (int col = threadIdx.x * 8; col < a.cols; col += 8192) {
            load_sum<T>(a, row, col, a.cols - col, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) sq[0] += s[i] * s[i];
        }
        team_sum<1024>(sq, red[odd]);
        const float r = __builtin_amdgcn_rsqf(sq[0] * a.inv_cols + a.eps);
        for (int col = threadIdx.x * 8; col < end; col += 8192) {
            float w[8];
            load_sum<T>(a, row, col, a.cols - col, s);
            load_weight<T>(a.weight, col, a.cols - col, w);
            put_row<T, MX, kShort>(a, row, col, r, s, w);
        }
    }
}

// dx of eight columns (into g), and dy s r (into s)
template <typename T, int E>
__device__ __forceinline__ void back8(const NormArgs& a, int64_t row, int col, float r, float c, float s[8], float dy[8], const float w[8], const float ds[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float n = dy[i] * (s[i] * r);
        dy[i] = r * (dy[i] * w[i] - s[i] * c) + ds[i];
        s[i] = n;
    }
    if (a.y) put<E, T>(a.y, row, a.ld_y, col, a.cols, dy);
}

template <typename T, int P, int U, int E>
__global__ __launch_bounds__(P < 256 ? 256 : P) void k_norm_back(const NormArgs a) {
    constexpr int TEAMS = kTeams<P>;
    __shared__ float red[2][P > 64 ? P / 64 : 1][2];
    __shared__ float sums[TEAMS > 1 ? TEAMS : 1][TEAMS > 1 ? P * U * 8 : 1];
    const int t = threadIdx.x % P, team = threadIdx.x / P;
    const bool along = a.y && a.res;
    float dw[U][8] = {};
    Raw8<T> rw[U];
    if (a.weight) {
#pragma unroll
        for (int u = 0; u < U; ++u) ask<E>(rw[u], a.weight, 0, 0, (u * P + t) * 8, a.cols);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) rw[u].q[i / Raw8<T>::V][i % Raw8<T>::V] = (T)1.0f;
    }
    int odd = 0;
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < a.rows; row += (int64_t)gridDim.x * TEAMS, odd ^= 1) {
        float s[U][8], dy[U][8], v[2] = {0.0f, 0.0f};
        Raw8<T> rs[U], ry[U], rd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (u * P + t) * 8;
            ask<E>(rs[u], a.x, row, a.ld_x, col, a.cols);
            ask<E>(ry[u], a.dy, row, a.ld_dy, col, a.cols);
        }
        if (along) {
#pragma unroll
            for (int u = 0; u < U; ++u) ask<E>(rd[u], a.res, row, a.ld_res, (u * P + t) * 8, a.cols);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float w[8];
            rs[u].get(s[u]);
            ry[u].get(dy[u]);
            rw[u].get(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (E == kBack && i < shared_of<E>((u * P + t) * 8, a.cols)) continue;
                v[0] += s[u][i] * s[u][i];
                v[1] += dy[u][i] * w[i] * s[u][i];
            }
        }
        team_sum<P>(v, red[odd]);
        const float r = __builtin_amdgcn_rsqf(v[0] * a.inv_cols + a.eps), c = r * r * (v[1] * a.inv_cols);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float w[8], ds[8] = {};
            rw[u].get(w);
            if (along) rd[u].get(ds);
            back8<T, E>(a, row, (u * P + t) * 8, r, c, s[u], dy[u], w, ds);
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[u][i] += s[u][i];
        }
    }
    if (!a.part) return;
    float* const part = a.part + (int64_t)blockIdx.x * a.part_ld;
    if constexpr (TEAMS > 1) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[team][first_of<E>((u * P + t) * 8, a.cols) + i] = dw[u][i];
        __syncthreads();
        for (int col = threadIdx.x; col < a.cols; col += 256) {
            float d = sums[0][col];
#pragma unroll
            for (int m = 1; m < TEAMS; ++m) d += sums[m][col];
            part[col] = d;
        }
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (u * P + t) * 8;
            if (col < a.cols) store8(part + first_of<E>(col, a.cols), 8, dw[u]);  // (the pitch has room for whole chunks)
        }
    }
}

template <typename T>
__global__ __launch_bounds__(1024) void k_norm_back_long(const NormArgs a) {
    __shared__ float red[2][16][2];
    float* const part = a.part ? a.part + (int64_t)blockIdx.x * a.part_ld : nullptr;
    int odd = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, odd ^= 1) {
        float s[8], dy[8], w[8], v[2] = {0.0f, 0.0f};
        const auto load = [&](int col) {
            const int cnt = a.cols - col;
            load8(static_cast<const T*>(a.x) + row * a.ld_x + col, cnt, s);
            load8(static_cast<const T*>(a.dy) + row * a.ld_dy + col, cnt, dy);
            load_weight<T>(a.weight, col, cnt, w);
        };
        for (int col = threadIdx.x * 8; col < a.cols; col += 8192) {
            load(col);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[0] += s[i] * s[i];
                v[1] += dy[i] * w[i] * s[i];
            }
        }
        team_sum<1024>(v, red[odd]);
        const float r = __builtin_amdgcn_rsqf(v[0] * a.inv_cols + a.eps), c = r * r * (v[1] * a.inv_cols);
        for (int col = threadIdx.x * 8; col < a.cols; col += 8192) {
            float ds[8] = {};
            load(col);
            if (a.y && a.res) load8(static_cast<const T*>(a.res) + row * a.ld_res + col, a.cols - col, ds);
            back8<T, kShort>(a, row, col, r, c, s, dy, w, ds);
            if (part) {
                float d[8] = {};
                if (row != blockIdx.x) load8(part + col, 8, d);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] += s[i];
                store8(part + col, 8, d);
            }
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------
constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxCols = int64_t(1) << 20;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool on(const void* p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// Work-groups of a backward call, each with partial sums of its own for the weight's gradient: what the compute units hold at
// once (16384 x 8192 bf16: 256 work-groups of 1024 lanes 196 us, 512 199, 1024 207), no more than there are rows for
int64_t back_groups(int64_t rows, int64_t cols) {
    const int teams = cols <= 128 ? 16 : cols <= 1024 ? 4 : 1;
    const int64_t most = cols <= 2048 ? 1024 : cols <= 6144 ? 512 : 256, want = div_up(rows, teams);
    return want < most ? want : most;
}

template <typename T, int P, int U>
void forward(const NormArgs& a, bool mx, hipStream_t st) {
    const dim3 block(P < 256 ? 256 : P), grid((unsigned)div_up(a.rows, (int64_t)kTeams<P> * a.per));
    const bool whole = a.cols % 8 == 0;
    if constexpr (P < 64) {
        if (a.cols < 8 && mx) return k_norm<T, P, U, true, kShort><<<grid, block, 0, st>>>(a);
        if (a.cols < 8) return k_norm<T, P, U, false, kShort><<<grid, block, 0, st>>>(a);
    }
    if (mx && whole) k_norm<T, P, U, true, kWhole><<<grid, block, 0, st>>>(a);
    else if (mx) k_norm<T, P, U, true, kBack><<<grid, block, 0, st>>>(a);
    else if (whole) k_norm<T, P, U, false, kWhole><<<grid, block, 0, st>>>(a);
    else k_norm<T, P, U, false, kBack><<<grid, block, 0, st>>>(a);
}

template <typename T, int P, int U>
void backward(const NormArgs& a, int64_t groups, hipStream_t st) {
    const dim3 block(P < 256 ? 256 : P), grid((unsigned)groups);
    if constexpr (P < 64)
        if (a.cols < 8) return k_norm_back<T, P, U, kShort><<<grid, block, 0, st>>>(a);
    if (a.cols % 8 == 0) k_norm_back<T, P, U, kWhole><<<grid, block, 0, st>>>(a);
    else k_norm_back<T, P, U, kBack><<<grid, block, 0, st>>>(a);
}

// Teams for a row's length.  Forward, 16384 x 8192 bf16 into 8 bits: 512 lanes of two eights 164 us, 256 of four the same,
// 1024 of one 209; several rows a team one after the other 179 (4) and 191 (8).  8192 x 8195 bf16: 1024 lanes 146 us, 768 120.
// 65536 x 128 bf16 into 8 bits: 16 lanes 11 us, 64 (the group of scales has 512 columns) 27.
template <typename T>
int launch_forward(NormArgs a, bool mx, hipStream_t st) {
    const int64_t wide = mx && a.cols > kMxFill ? mx_groups(a.cols) * kMxGroup : a.cols;
    a.per = (int)div_up(a.rows, int64_t(1) << 20);  // (a launch has fewer than 2^32 threads)
    if (wide <= 128) forward<T, 16, 1>(a, mx, st);
    else if (wide <= 512) forward<T, 64, 1>(a, mx, st);
    else if (wide <= 1024) forward<T, 64, 2>(a, mx, st);
    else if (wide <= 2048) forward<T, 256, 1>(a, mx, st);
    else if (wide <= 4096) forward<T, 256, 2>(a, mx, st);
    else if (wide <= 8192) forward<T, 512, 2>(a, mx, st);
    else if (wide <= 12288) forward<T, 768, 2>(a, mx, st);
    else if (wide <= 16384) forward<T, 1024, 2>(a, mx, st);
    else {
        const dim3 grid((unsigned)(a.rows < (int64_t(1) << 20) ? a.rows : int64_t(1) << 20));
        if (mx) k_norm_long<T, true><<<grid, dim3(1024), 0, st>>>(a);
        else k_norm_long<T, false><<<grid, dim3(1024), 0, st>>>(a);
    }
    return hipGetLastError() == hipSuccess ? DLC_OK : DLC_EHIP;
}

// Backward a lane also keeps its columns' sums: one eight each as long as a work-group has the lanes.  16384 x 8192 bf16: 1024
// lanes of one eight 196 us, 512 of two 199 (two work-groups' worth of registers do not fit a compute unit); asking for the
// next row while one is summed up 199.  8192 x 4099: 1024 lanes 81 us, 768 (two work-groups a compute unit) 60.  4096 x 12288: read
// twice 176 us, 1024 lanes of two eights 110 (registers do not hold them all), 768 82; 16384 columns, 1024 lanes, 138 for 213.
template <typename T>
int launch_backward(const NormArgs& a, int64_t groups, hipStream_t st) {
    if (a.cols <= 128) backward<T, 16, 1>(a, groups, st);
    else if (a.cols <= 512) backward<T, 64, 1>(a, groups, st);
    else if (a.cols <= 1024) backward<T, 64, 2>(a, groups, st);
    else if (a.cols <= 2048) backward<T, 256, 1>(a, groups, st);
    else if (a.cols <= 4096) backward<T, 512, 1>(a, groups, st);
    else if (a.cols <= 6144) backward<T, 768, 1>(a, groups, st);
    else if (a.cols <= 8192) backward<T, 1024, 1>(a, groups, st);
    else if (a.cols <= 12288) backward<T, 768, 2>(a, groups, st);
    else if (a.cols <= 16384) backward<T, 1024, 2>(a, groups, st);
    else k_norm_back_long<T><<<dim3((unsigned)groups), dim3(1024), 0, st>>>(a);
    return hipGetLastError() == hipSuccess ? DLC_OK : DLC_EHIP;
}

// Checks the configuration and fills in what it says
bool make_args(const dlc_norm_config* c, NormArgs* a) {
    if (!c || (c->dtype != DLC_F32 && c->dtype != DLC_F16 && c->dtype != DLC_BF16) || c->reserved != 0) return false;
    if (c->rows < 0 || c->rows > kMaxRows || c->cols < 1 || c->cols > kMaxCols) return false;
    if (!(c->eps >= 0x1p-126 && c->eps <= 0x1p126)) return false;
    const int64_t lim = c->rows > 0 ? (int64_t(1) << 60) / c->rows : int64_t(1) << 60;  // (a buffer's last byte has a 64-bit address)
    for (const int64_t ld : {c->ld_x, c->ld_res, c->ld_sum, c->ld_y, c->ld_dy, c->ld_ds, c->ld_dx})
        if (ld != 0 && (ld < c->cols || ld > lim)) return false;
    a->rows = c->rows;
    a->cols = (int)c->cols;
    a->eps = (float)c->eps;
    a->inv_cols = 1.0f / (float)c->cols;
    return true;
}

int64_t ld_of(int64_t ld, int64_t cols) { return ld ? ld : cols; }
bool good(const void* p, int es, bool need) { return p ? on(p, es) : !need; }
// `out` may take the place of `in` element for element, not with other distances from row to row
bool good_place(const void* in, int64_t ld_in, const void* out, int64_t ld_out, int64_t rows) { return !in || in != out || ld_in == ld_out || rows <= 1; }

size_t back_bytes(int64_t rows, int64_t cols) { return (size_t)back_groups(rows, cols) * (size_t)round8(cols) * 4; }

}  // namespace

extern "C" size_t dlc_norm_workspace_bytes(const dlc_norm_config* c) {
    NormArgs a{};
    return make_args(c, &a) ? back_bytes(a.rows, a.cols) : 0;
}

extern "C" int dlc_norm_forward(const dlc_norm_config* c, const void* x, const void* res, const void* weight, void* sum, void* y, void* q,
                                void* scale, void* stream) {
    NormArgs a{};
    if (!make_args(c, &a)) return DLC_EINVAL;
    const int es = c->dtype == DLC_F32 ? 4 : 2;
    const bool need = a.rows > 0;
    if (!good(x, es, need) || !good(res, es, false) || !good(weight, es, false) || !good(sum, es, false) || !good(y, es, false) ||
        !on(q, 16) || !on(scale, 16) || (q == nullptr) != (scale == nullptr) || (need && !sum && !y && !q)) return DLC_EINVAL;
    if (!need) return DLC_OK;
    a.ld_x = ld_of(c->ld_x, a.cols); a.ld_res = ld_of(c->ld_res, a.cols); a.ld_sum = ld_of(c->ld_sum, a.cols); a.ld_y = ld_of(c->ld_y, a.cols);
    if (!good_place(x, a.ld_x, sum, a.ld_sum, a.rows) || !good_place(res, a.ld_res, sum, a.ld_sum, a.rows) ||
        !good_place(x, a.ld_x, y, a.ld_y, a.rows) || (y && (y == sum || y == res))) return DLC_EINVAL;
    a.x = x; a.res = res; a.weight = weight; a.sum = sum; a.y = y;
    a.q = static_cast<uint8_t*>(q); a.scale = static_cast<uint8_t*>(scale);
    hipStream_t st = (hipStream_t)stream;
    switch (c->dtype) {
        case DLC_F32: return launch_forward<float>(a, q != nullptr, st);
        case DLC_F16: return launch_forward<f16_t>(a, q != nullptr, st);
        default: return launch_forward<bf16_t>(a, q != nullptr, st);
    }
}

extern "C" int dlc_norm_backward(const dlc_norm_config* c, const void* s, const void* weight, const void* dy, const void* ds, void* dx,
                                 void* dweight, void* work, size_t work_bytes, void* stream) {
    NormArgs a{};
    if (!make_args(c, &a)) return DLC_EINVAL;
    const int es = c->dtype == DLC_F32 ? 4 : 2;
    const bool need = a.rows > 0 && (dx || dweight);
    if (!good(s, es, need) || !good(weight, es, false) || !good(dy, es, need) || !good(ds, es, false) || !good(dx, es, false) ||
        !good(dweight, es, false) || !on(work, 16)) return DLC_EINVAL;
    if ((!dx || a.rows == 0) && !dweight) return DLC_OK;
    a.ld_x = ld_of(c->ld_sum, a.cols); a.ld_res = ld_of(c->ld_ds, a.cols); a.ld_dy = ld_of(c->ld_dy, a.cols); a.ld_y = ld_of(c->ld_dx, a.cols);
    if (!good_place(dy, a.ld_dy, dx, a.ld_y, a.rows) || !good_place(ds, a.ld_res, dx, a.ld_y, a.rows) || (dx && dx == s && a.rows > 0)) return DLC_EINVAL;
    const int64_t groups = back_groups(a.rows, a.cols);
    if (dweight && a.rows > 0) {
        if (!work) return DLC_EINVAL;
        if (work_bytes < back_bytes(a.rows, a.cols)) return DLC_ECAPACITY;
        a.part = static_cast<float*>(work);
        a.part_ld = round8(a.cols);
    }
    a.x = s; a.res = ds; a.weight = weight; a.dy = dy; a.y = dx;
    hipStream_t st = (hipStream_t)stream;
    const SumArgs sum{a.part, a.part_ld, (int)groups, a.cols, dweight};
    const auto all = [&](auto one) {
        using T = decltype(one);
        if (a.rows > 0)
            if (const int rc = launch_backward<T>(a, groups, st); rc != DLC_OK) return rc;
        if (!dweight) return (int)DLC_OK;
        return DenseOps<T>::join(JoinArgs{}, JoinArgs{}, sum, st) == hipSuccess ? (int)DLC_OK : (int)DLC_EHIP;
    };
    switch (c->dtype) {
        case DLC_F32: return all(float{});
        case DLC_F16: return all(f16_t{});
        default: return all(bf16_t{});
    }
}
