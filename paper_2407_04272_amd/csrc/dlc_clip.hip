// The norm of all gradients together, and clipping.
//
// Bound by memory: the norm reads every gradient once; clipping reads them again, as far as they did not stay in a cache, and
// writes them.  The tensors' descriptions go with the launch, kTensors of them at a time; a work-group takes a chunk of one
// tensor.  Sums are 64-bit: no gradient's square is lost or too large, whatever the type.  400 million bf16 elements: the norm
// 169 us (4.7 TB/s) and 5 for the chunks' sums, clipping 280 (5.7 TB/s); 2.5 million of fp32 4.5 + 2 + 2.5 us and the gaps between
// three launches.
#include <cfloat>

#include "dlc_dense.h"

using namespace dlc;

namespace {

// Descriptions that go with a launch: kTensors, or kFew where there are no more (a launch's arguments are copied twice on
// their way: 7 tensors and their 2.5 million values 14.6 us a pass with room for 64)
constexpr int kTensors = 64, kFew = 8;
constexpr int64_t kChunk = 8192;       // elements of a chunk, at least: four eights a thread
constexpr int64_t kMaxChunks = 8192;   // ... so many that there are no more than these (and one a tensor)
constexpr int kThreads = 256;
// Elements that one work-group adds up alone, without a second launch: both calls 10.4 us of the host's time for 13.9
constexpr int64_t kOne = 32768;

struct Piece {
    const void* in;
    void* out;
    int64_t n, cols, ld_in, ld_out;   // n elements in all; dense: cols = n
    int32_t dtype;
};

template <int N>
struct ClipArgs {
    Piece t[N];
    uint32_t first[N];                // a tensor's first chunk in this launch; ~0 where there is none
    int64_t chunk;
    int32_t count;
    uint32_t chunks;
    double* part;                     // norm: the chunks' sums
    const double* sum;                // clip
    double max_norm;
    float* norm;
};
static_assert(sizeof(ClipArgs<kTensors>) <= 4096, "what a launch takes along");

// which tensor a chunk is of (all are looked at: their places come in a few wide loads, where a search would wait for one
// after the other)
template <int N>
__device__ __forceinline__ int piece_of(const ClipArgs<N>& a, uint32_t chunk) {
    int n = -1;
#pragma unroll
    for (int i = 0; i < N; ++i) n += a.first[i] <= chunk;
    return n;
}

// f(values, out, elements) for the eights of a chunk (fewer at a row's end), four a thread on their way together
template <typename T, typename F>
__device__ __forceinline__ void each8(const Piece& p, int64_t at, int64_t end, F f) {
    const T* const in = static_cast<const T*>(p.in);
    T* const out = static_cast<T*>(p.out);
    float v[8];
    if (p.cols == p.n) {
        int64_t i = at + threadIdx.x * 8;
        for (int64_t whole = (end - at) / (kThreads * 32); whole > 0; --whole, i += kThreads * 32) {
            Raw8<T> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u].load_whole(in + i + u * (kThreads * 8), true);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                x[u].get(v);
                f(v, out + i + u * (kThreads * 8), 8);
            }
        }
        for (; i < end; i += kThreads * 8) {
            const int cnt = (int)min((int64_t)8, end - i);
            load8(in + i, cnt, v);
            f(v, out + i, cnt);
        }
        return;
    }
    // rows apart: eights of a row, counted through all rows (chunks are whole numbers of them)
    const int64_t per = (p.cols + 7) / 8;
    for (int64_t i = at / 8 + threadIdx.x; i < end / 8; i += kThreads) {
        const int64_t row = i / per, col = (i - row * per) * 8;
        const int cnt = (int)min((int64_t)8, p.cols - col);
        load8(in + row * p.ld_in + col, cnt, v);
        f(v, out + row * p.ld_out + col, cnt);
    }
}

// elements that a chunk counts: rows apart are filled up to eights
__host__ __device__ inline int64_t counted(const Piece& p) { return p.cols == p.n ? p.n : p.n / p.cols * ((p.cols + 7) / 8 * 8); }

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double red[kThreads / 64];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = red[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) s += red[w];
    return s;
}

template <int N>
__global__ __launch_bounds__(kThreads) void k_squares(const ClipArgs<N> a) {
    double s = 0.0;
    for (uint32_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const int piece = piece_of(a, chunk);
        const Piece& p = a.t[piece];
        const int64_t at = (int64_t)(chunk - a.first[piece]) * a.chunk, end = min(counted(p), at + a.chunk);
        const auto run = [&](auto one) {
            using T = decltype(one);
            each8<T>(p, at, end, [&](const float* f, T*, int) {  // (0 past the last)
#pragma unroll
                for (int i = 0; i < 8; ++i) s += (double)f[i] * (double)f[i];
            });
        };
        if (p.dtype == DLC_F32) run(float{});
        else if (p.dtype == DLC_F16) run(f16_t{});
        else run(bf16_t{});
    }
    s = block_sum(s);
    if (threadIdx.x == 0) a.part[blockIdx.x] = s;
}

// The chunks' sums, always in the same order, all loads of a round on their way together
__global__ __launch_bounds__(kThreads) void k_add(const double* part, int64_t n, double* sum) {
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kThreads * 16) {
        double v[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) v[u] = i + u * kThreads < n ? part[i + u * kThreads] : 0.0;
#pragma unroll
        for (int u = 0; u < 16; ++u) s += v[u];
    }
    s = block_sum(s);
    if (threadIdx.x == 0) *sum = s;
}

template <int N>
__global__ __launch_bounds__(kThreads) void k_clip(const ClipArgs<N> a) {
    const double n = sqrt(*a.sum);
    // (finite means that f is what it should be: a finite n past fp32's range is its largest value)
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = n < __builtin_inf() ? (float)fmin(n, (double)FLT_MAX) : (float)n;
    if (a.count == 0) return;
    // (64-bit too: with far gradients and a small limit it lies below fp32's normal range where the results do not)
    const double f = n > a.max_norm && n < __builtin_inf() ? a.max_norm / n : 1.0;
    // from the last chunk on: what the norm read last may still be in the last cache
    const uint32_t chunk = a.chunks - 1 - blockIdx.x;
    const int piece = piece_of(a, chunk);
    const Piece& p = a.t[piece];
    if (f == 1.0 && p.in == p.out) return;
    const int64_t at = (int64_t)(chunk - a.first[piece]) * a.chunk, end = min(counted(p), at + a.chunk);
    const auto run = [&](auto one) {
        using T = decltype(one);
        each8<T>(p, at, end, [&](float* v, T* out, int cnt) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)((double)v[i] * f);
            store8(out, cnt, v);
        });
    };
    if (p.dtype == DLC_F32) run(float{});
    else if (p.dtype == DLC_F16) run(f16_t{});
    else run(bf16_t{});
}

// ---- host ---------------------------------------------------------------------------------------
constexpr int64_t kMaxTensors = int64_t(1) << 20, kMaxElements = int64_t(1) << 40, kMaxAll = int64_t(1) << 44;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct List {
    int64_t chunk = kChunk, all = 0;  // elements of a chunk, elements in all
};

bool good_tensor(const dlc_tensor& t) {
    if (t.dtype != DLC_F32 && t.dtype != DLC_F16 && t.dtype != DLC_BF16) return false;
    if (t.reserved != 0 || t.rows < 0 || t.cols < 0 || (t.ld != 0 && t.ld < t.cols)) return false;
    if (t.rows == 0 || t.cols == 0) return true;
    return t.p && ((uintptr_t)t.p & (t.dtype == DLC_F32 ? 3u : 1u)) == 0;
}

Piece piece(const dlc_tensor& t, const dlc_tensor& o) {
    Piece p{};
    p.in = t.p; p.out = o.p; p.dtype = t.dtype;
    p.n = t.rows * t.cols;
    p.ld_in = t.ld ? t.ld : t.cols;
    p.ld_out = o.ld ? o.ld : o.cols;
    const bool dense = t.rows <= 1 || (p.ld_in == t.cols && p.ld_out == t.cols);
    p.cols = dense ? p.n : t.cols;
    return p;
}

// Checks the tensors and finds the chunks' size and number.  out: as `list`
int look(const dlc_tensor* list, const dlc_tensor* out, int64_t count, List* l) {
    if (count < 0 || count > kMaxTensors || (count > 0 && (!list || !out))) return DLC_EINVAL;
    int64_t all = 0;
    for (int64_t i = 0; i < count; ++i) {
        const dlc_tensor &t = list[i], &o = out[i];
        if (!good_tensor(t) || !good_tensor(o) || t.rows != o.rows || t.cols != o.cols || t.dtype != o.dtype) return DLC_EINVAL;
        if (t.rows == 0 || t.cols == 0) continue;
        if (t.rows > kMaxElements / t.cols || t.ld > (int64_t(1) << 60) / t.rows || o.ld > (int64_t(1) << 60) / t.rows) return DLC_ELIMIT;
        const Piece p = piece(t, o);
        if (t.p == o.p && t.rows > 1 && p.ld_in != p.ld_out) return DLC_EINVAL;
        all += counted(p);
        if (all > kMaxAll) return DLC_ELIMIT;
    }
    l->all = all;
    l->chunk = div_up(div_up(all, kMaxChunks), kChunk) * kChunk;
    if (l->chunk < kChunk) l->chunk = kChunk;
    return DLC_OK;
}

// launch(args): once for up to N tensors
template <int N, typename F>
int each_launch(ClipArgs<N> a, const dlc_tensor* list, const dlc_tensor* out, int64_t count, F launch) {
    int64_t chunks = 0;
    const auto none = [&] {
        a.count = 0;
        chunks = 0;
        for (uint32_t& f : a.first) f = ~0u;
    };
    none();
    for (int64_t i = 0; i < count; ++i) {
        if (list[i].rows == 0 || list[i].cols == 0) continue;
        const Piece p = piece(list[i], out[i]);
        a.first[a.count] = (uint32_t)chunks;
        a.t[a.count++] = p;
        chunks += div_up(counted(p), a.chunk);
        a.chunks = (uint32_t)chunks;
        if (a.count == N) {
            if (launch(a) != hipSuccess) return DLC_EHIP;
            none();
        }
    }
    return a.count == 0 || launch(a) == hipSuccess ? DLC_OK : DLC_EHIP;
}

int64_t all_chunks(const dlc_tensor* list, int64_t count, int64_t chunk) {
    int64_t n = 0;
    for (int64_t i = 0; i < count; ++i)
        if (list[i].rows != 0 && list[i].cols != 0) n += div_up(counted(piece(list[i], list[i])), chunk);
    return n;
}

}  // namespace

extern "C" size_t dlc_gradient_workspace_bytes(const dlc_tensor* list, int64_t count) {
    List l;
    return look(list, list, count, &l) == DLC_OK ? (size_t)all_chunks(list, count, l.chunk) * 8 : 0;
}

extern "C" int dlc_gradient_norm(const dlc_tensor* list, int64_t count, double* d_sum, void* work, size_t bytes, void* stream) {
    List l;
    if (const int rc = look(list, list, count, &l); rc != DLC_OK) return rc;
    if (!d_sum || ((uintptr_t)d_sum & 7) != 0 || ((uintptr_t)work & 15) != 0) return DLC_EINVAL;
    const int64_t chunks = all_chunks(list, count, l.chunk);
    if (chunks > 0 && !work) return DLC_EINVAL;
    if (bytes < (size_t)chunks * 8) return DLC_ECAPACITY;
    hipStream_t st = (hipStream_t)stream;
    const bool one = l.all > 0 && l.all <= kOne && count <= kTensors;
    const auto squares = [&](auto a) {
        a.chunk = l.chunk;
        a.part = one ? d_sum : static_cast<double*>(work);
        return each_launch(a, list, list, count, [&](auto& b) {
            k_squares<<<dim3(one ? 1u : b.chunks), dim3(kThreads), 0, st>>>(b);
            b.part += b.chunks;
            return hipGetLastError();
        });
    };
    const int rc = count <= kFew ? squares(ClipArgs<kFew>{}) : squares(ClipArgs<kTensors>{});
    if (rc != DLC_OK || one) return rc;
    k_add<<<dim3(1), dim3(kThreads), 0, st>>>(static_cast<const double*>(work), chunks, d_sum);
    return hipGetLastError() == hipSuccess ? DLC_OK : DLC_EHIP;
}

extern "C" int dlc_gradient_clip(const dlc_tensor* list, int64_t count, const double* d_sum, double max_norm, float* d_norm,
                                 const dlc_tensor* out, void* stream) {
    List l;
    if (const int rc = look(list, out, count, &l); rc != DLC_OK) return rc;
    if (!d_sum || ((uintptr_t)d_sum & 7) != 0 || ((uintptr_t)d_norm & 3) != 0 || !(max_norm >= 0.0)) return DLC_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const auto clip = [&](auto a) {
        a.chunk = l.chunk;
        a.sum = d_sum;
        a.max_norm = max_norm;
        a.norm = d_norm;
        bool any = false;
        const int rc = each_launch(a, list, out, count, [&](auto& b) {
            k_clip<<<dim3(b.chunks), dim3(kThreads), 0, st>>>(b);
            any = true;
            return hipGetLastError();
        });
        if (rc != DLC_OK || any || !d_norm) return rc;
        k_clip<<<dim3(1), dim3(kThreads), 0, st>>>(a);  // (no tensors: the norm alone)
        return hipGetLastError() == hipSuccess ? (int)DLC_OK : (int)DLC_EHIP;
    };
    return count <= kFew ? clip(ClipArgs<kFew>{}) : clip(ClipArgs<kTensors>{});
}
