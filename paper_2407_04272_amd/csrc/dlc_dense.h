// Internal declarations of the dense operators (linear layers, gated blocks, dropout): arguments of the kernels, the
// device functions that every epilogue shares, and the launches of each element type's source file.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "dlc.h"

namespace dlc {

// What happens to a sum before it is stored: y = drop(act(sum + bias)) + residual, or, gated, y = drop(act(g) * u).  A
// null pointer leaves its part out.  Leading dimensions count elements.
struct Epi {
    void* y;
    void* pre;        // the sum with its bias, before the activation (training: the backward pass reads it)
    const void* res;
    const void* bias;
    int64_t ld_y, ld_pre, ld_res;
    uint64_t seed, offset;
    const uint64_t* d_offset;  // added to offset, read by the kernel
    uint32_t thr;     // an element is dropped if its 16 random bits are below (0: none is, 65536: all are)
    float scale;      // 65536 / (65536 - thr)
    int32_t act;
    int32_t n;        // columns of y (gated: the gate's half of the sums' columns)
};

// One product: C[m][n] = sum over k of A(m, k) B(n, k).
struct GemmArgs {
    const void* a;
    const void* b;
    int64_t lda, ldb;
    int32_t M, N, K;      // gated: N counts the columns of y, B has 2 N rows
    int32_t kper, split;  // the sum is cut into `split` ranges of `kper` (a multiple of the k tile)
    int32_t tiles_m, tiles_n;
    float* part;          // split > 1: [split][M][part_ld] partial sums, put together by join
    int64_t part_ld;
    Epi e;
};

// Adds up the partial sums of a product and does its epilogue (M = 0: nothing)
struct JoinArgs {
    const float* part;
    int64_t part_ld;
    int32_t M, split, gated;
    Epi e;
};

// Up to two matrices whose rows are copied to 16-byte boundaries: dst is [rows][cols rounded up to whole chunks]
struct PackArgs {
    const void* src[2];
    void* dst[2];
    int64_t ld[2], rows[2];
    int32_t cols[2];
};

// dz = drop(dy) * act'(pre) (gated: both halves) and the partial column sums for the bias gradient
struct DzArgs {
    const void* dy;
    const void* pre;
    void* dz;             // null: only the sums
    float* sums;          // [row_blocks][sums_ld], null: no bias
    int64_t ld_dy, ld_pre, ld_dz, sums_ld;
    int64_t M;
    int32_t n, gated, act;
    int32_t row_blocks, rows_per_block;
    uint32_t thr;
    float scale;
    uint64_t seed, offset;
    const uint64_t* d_offset;
};

// Adds up the row blocks' sums: the bias gradient (n = 0: nothing)
struct SumArgs {
    const float* sums;
    int64_t sums_ld;
    int32_t row_blocks, n;
    void* out;
};

struct DropArgs {
    const void* x;
    const void* res;
    void* y;
    int64_t rows, ld_x, ld_res, ld_y;
    int32_t cols;
    uint32_t thr;
    float scale;
    uint64_t seed, offset;
    const uint64_t* d_offset;
};

// operand layouts of a product: both with k along a row (x w'), a with k along a row and b with k down a column (dz w),
// both with k down a column (dz' x)
enum Layout { L_KK = 0, L_KT = 1, L_TT = 2 };

template <typename T>
struct DenseOps {
    static hipError_t gemm(const GemmArgs& g, Layout lay, bool gated, int tile, hipStream_t s);
    static hipError_t skinny(const GemmArgs& g, bool gated, bool aligned, hipStream_t s);
    static hipError_t back(const GemmArgs& gx, const GemmArgs& gw, const SumArgs& a, int tile, hipStream_t s);
    static hipError_t join(const JoinArgs& ja, const JoinArgs& jb, const SumArgs& a, hipStream_t s);
    static hipError_t pack(const PackArgs& p, hipStream_t s);
    static hipError_t dz(const DzArgs& d, const PackArgs& p, hipStream_t s);
    static hipError_t drop(const DropArgs& d, hipStream_t s);
};

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

inline __host__ __device__ int64_t round8(int64_t v) { return (v + 7) & ~int64_t(7); }

// tile sizes (rows, columns, k bytes are 128)
constexpr int kTileM[] = {256, 128, 64};
constexpr int kTileN[] = {256, 128, 128};
constexpr int kTileBytes = 128;  // a cut of k is a multiple of this many bytes of it (a k tile, or two)
constexpr int kSkinnyRows = 32, kSkinnyOddRows = 16;  // most rows of a pass over the weights, and where they stand off boundaries
constexpr int kDzRows = 16;    // rows a work-group of k_dz takes at a time

#if defined(__HIPCC__)

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// ---- random bits: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011) ----
// The ten rounds give 128 bits for eight elements: columns col8*8 .. col8*8+7 of a row.  keep() holds bit v where element
// v stays.  Sixteen bits an element: p is taken to the nearest 1/65536, and a memory-bound pass stays one (32 bits an
// element would double the 64-bit products, which run at a quarter of the add's rate).
__device__ __forceinline__ uint32_t keep_mask(uint32_t col8, uint32_t row, uint64_t seed, uint64_t offset, uint32_t thr) {
    uint32_t c0 = col8, c1 = row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m |= ((w[i] & 0xFFFFu) >= thr ? 1u : 0u) << (2 * i);
        m |= ((w[i] >> 16) >= thr ? 1u : 0u) << (2 * i + 1);
    }
    return m;
}

// ---- activations, in fp32 ----
// FAST (results of half precision): the hardware's exponential and reciprocal, off by a few 2^-24 of the result, and a
// polynomial for erfc, where a full division, expf and erfcf took 8 us of every 256 x 256 tile's epilogue.  An exponential
// that overflows gives 1 / infinity = 0, the limit that is wanted.
template <bool FAST>
__device__ __forceinline__ float sigmoidf(float z) {
    if constexpr (FAST) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
    else return 1.0f / (1.0f + expf(-z));
}

// ... and its slope, which is even: e / (1 + e)^2 with e = exp(-|z|).  (q (1 - q) cancels: 6 % off at z = 16, 0 from 17 on.)
template <bool FAST>
__device__ __forceinline__ float sigmoid_both(float z, float* slope) {
    const float x = __builtin_fabsf(z);
    float e, r;
    if constexpr (FAST) {
        e = __builtin_amdgcn_exp2f(x * -1.44269504f);
        r = __builtin_amdgcn_rcpf(1.0f + e);
    } else {
        e = expf(-x);
        r = 1.0f / (1.0f + e);
    }
    const float p = e * r;  // sigmoid(-|z|)
    *slope = p * r;
    return z < 0.0f ? p : r;
}

// The normal distribution function at z, and (phi) its density.  FAST: erfc(x) = exp(-x^2) t P(t) with t = 1 / (1 + 0.45 x);
// P is a least-squares fit of exp(x^2) erfc(x) / t over all x >= 0, reweighted towards equal relative errors: 1.4e-7 at most.
template <bool FAST>
__device__ __forceinline__ float normal_cdf(float z, float* phi) {
    if constexpr (FAST) {
        const float x = __builtin_fabsf(z) * 0.70710678f;
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.45f, x, 1.0f));
        const float e = __builtin_amdgcn_exp2f(x * x * -1.44269504f);
        float p = -0.04207083582878113f;
        p = __builtin_fmaf(p, t, 0.19364100694656372f);
        p = __builtin_fmaf(p, t, -0.3059483766555786f);
        p = __builtin_fmaf(p, t, 0.14769354462623596f);
        p = __builtin_fmaf(p, t, -0.025435185059905052f);
        p = __builtin_fmaf(p, t, 0.12102247029542923f);
        p = __builtin_fmaf(p, t, 0.17503467202186584f);
        p = __builtin_fmaf(p, t, 0.22829535603523254f);
        p = __builtin_fmaf(p, t, 0.2538819909095764f);
        p = __builtin_fmaf(p, t, 0.25388532876968384f);
        const float h = 0.5f * (e * (t * p));
        if (phi) *phi = e * 0.39894228f;
        return z < 0.0f ? h : 1.0f - h;
    } else {
        if (phi) *phi = expf(-0.5f * z * z) * 0.39894228040143268f;
        return 0.5f * erfcf(z * -0.70710678118654752f);
    }
}

template <bool FAST, int U>
__device__ __forceinline__ void act_values(int act, float (&z)[U][8]) {
    const auto each = [&](auto f) {
#pragma unroll
        for (int r = 0; r < U; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) z[r][i] = f(z[r][i]);
    };
    switch (act) {
        case DLC_ACT_RELU: return each([](float v) { return v < 0.0f ? 0.0f : v; });  // (NaN stays NaN)
        case DLC_ACT_SIGMOID: return each([](float v) { return sigmoidf<FAST>(v); });
        case DLC_ACT_SILU: return each([](float v) { return v * sigmoidf<FAST>(v); });
        case DLC_ACT_GELU: return each([](float v) { return v * normal_cdf<FAST>(v, nullptr); });
        default: break;
    }
}

// A product that is 0 where a factor is, whatever the other one holds; otherwise the ordinary one, subnormals included.  The
// backward pass is made of these: what a dropped or closed element holds does not get out (in half precision a sum past the
// type's range is saved as an infinity), and values and slopes at infinity come out as their limits.  The instruction
// v_mul_legacy_f32 is that product; comparing and selecting takes 72 us for 66 in k_dz of gated 8192 x 4096 bf16.
extern "C" __device__ float dlc_mul_legacy(float a, float b) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float mul0(float a, float b) { return dlc_mul_legacy(a, b); }

// values (into z) and slopes at z
template <bool FAST>
__device__ __forceinline__ void act_both(int act, float z[8], float d[8]) {
    switch (act) {
        case DLC_ACT_RELU:
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] = z[i] <= 0.0f ? 0.0f : 1.0f;
                z[i] = z[i] < 0.0f ? 0.0f : z[i];
            }
            break;
        case DLC_ACT_SIGMOID:
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = sigmoid_both<FAST>(z[i], &d[i]);
            break;
        case DLC_ACT_SILU:
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float slope;
                const float q = sigmoid_both<FAST>(z[i], &slope);
                d[i] = q + mul0(z[i], slope);
                z[i] = mul0(z[i], q);
            }
            break;
        case DLC_ACT_GELU:
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float phi;
                const float c = normal_cdf<FAST>(z[i], &phi);
                d[i] = c + mul0(z[i], phi);
                z[i] = mul0(z[i], c);
            }
            break;
        default:
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = 1.0f;
    }
}

// ---- eight consecutive elements of a row, from an element's boundary ----
// (16 bytes an access wherever they stand: an access that is not on its own boundary costs a little more, element by element
// it costs eight times as many)
template <typename T>
struct Vec8 {
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// reads elements [0, cnt) of p as fp32, 0 behind them
template <typename T>
__device__ __forceinline__ void load8(const T* p, int cnt, float f[8]) {
    constexpr int V = 16 / sizeof(T);
    if (cnt >= 8) {
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            const typename Vec8<T>::type q = *reinterpret_cast<const typename Vec8<T>::type*>(p + i * V);
#pragma unroll
            for (int j = 0; j < V; ++j) f[i * V + j] = (float)q[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < cnt ? (float)p[i] : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, int cnt, const float f[8]) {
    constexpr int V = 16 / sizeof(T);
    if (cnt >= 8) {
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            typename Vec8<T>::type q;
#pragma unroll
            for (int j = 0; j < V; ++j) q[j] = (T)f[i * V + j];
            *reinterpret_cast<typename Vec8<T>::type*>(p + i * V) = q;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < cnt) p[i] = (T)f[i];
    }
}

__device__ __forceinline__ uint64_t full_offset(uint64_t offset, const uint64_t* d_offset) {
    return d_offset ? offset + *d_offset : offset;
}

// Epilogue of eight columns col .. col+7 (col a multiple of 8) of the rows m, m + STEP, ..., of which those below m + rows
// exist: s the sums; gated: s the gate's, u the other's.  Everything is fp32 up to the one rounding at the store.
template <typename T, bool GATED, int U, int STEP>
__device__ __forceinline__ void epilogue8(const Epi& e, uint64_t offset, int64_t m, int rows, int col, float (&s)[U][8], float (&u)[U][8]) {
    const int cnt = e.n - col;
    if (cnt <= 0) return;
    if (e.bias) {
        const T* bias = static_cast<const T*>(e.bias);
        float b[8], c[8];
        load8(bias + col, cnt, b);
        if constexpr (GATED) load8(bias + e.n + col, cnt, c);
#pragma unroll
        for (int r = 0; r < U; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[r][i] += b[i];
                if constexpr (GATED) u[r][i] += c[i];
            }
    }
    if (e.pre) {
#pragma unroll
        for (int r = 0; r < U; ++r) {
            if (r * STEP >= rows) continue;
            T* p = static_cast<T*>(e.pre) + (m + r * STEP) * e.ld_pre;
            store8(p + col, cnt, s[r]);
            if constexpr (GATED) store8(p + e.n + col, cnt, u[r]);
        }
    }
    act_values<sizeof(T) == 2>(e.act, s);
    if constexpr (GATED) {
#pragma unroll
        for (int r = 0; r < U; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[r][i] *= u[r][i];
    }
    if (e.thr) {
#pragma unroll
        for (int r = 0; r < U; ++r) {
            const uint32_t keep = keep_mask((uint32_t)col >> 3, (uint32_t)(m + r * STEP), e.seed, offset, e.thr);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[r][i] = (keep >> i) & 1u ? s[r][i] * e.scale : 0.0f;
        }
    }
    if (e.res) {
        float x[U][8];
#pragma unroll
        for (int r = 0; r < U; ++r)
            if (r * STEP < rows) load8(static_cast<const T*>(e.res) + (m + r * STEP) * e.ld_res + col, cnt, x[r]);
#pragma unroll
        for (int r = 0; r < U; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[r][i] += x[r][i];
    }
#pragma unroll
    for (int r = 0; r < U; ++r)
        if (r * STEP < rows) store8(static_cast<T*>(e.y) + (m + r * STEP) * e.ld_y + col, cnt, s[r]);
}

#endif  // __HIPCC__
}  // namespace dlc
