// Microscaled form (elements E2M1 or E4M3, a scale 2^e for 32 columns; laid out as dlc.h says): what the kernels that write and
// read it share.
#pragma once
#include "dlc_dense.h"
#include "dlc_mx_plan.h"

namespace dlc {

constexpr int kMxBlock = 32, kMxFill = 128;  // columns of a scale, that a row is filled up to

inline __host__ __device__ int64_t mx_groups(int64_t cols) { return (cols + kMxGroup - 1) / kMxGroup; }
inline __host__ __device__ int64_t mx_filled(int64_t cols) { return (cols + kMxFill - 1) / kMxFill * kMxFill; }
inline __host__ __device__ int64_t mx_row_bytes(int64_t cols, int elem) { return mx_filled(cols) * elem / 8; }

#if defined(__HIPCC__)

// Where a block's scale stands in its group of 16
__device__ __forceinline__ int mx_scale_place(int block) { return 4 * (block & 3) + ((block >> 2) & 3); }

// Largest magnitude of a block, as bits (a NaN's are above infinity's, which are above all others: neither gets lost), to the
// scale's byte: e + 127 with e the smallest exponent that the magnitude fits under, 255 where there is none.  The type's
// largest value is 1.75 * 2^8 (E2M1: 1.5 * 2^2), so a magnitude 1.f * 2^k takes k - 8 (k - 2), or one more if f is above.
template <int ELEM>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
    constexpr uint32_t up = ELEM == 8 ? 0x1FFFFFu : 0x3FFFFFu;
    constexpr int less = ELEM == 8 ? 8 : 2;
    const int k = (int)((top + up) >> 23) - less;
    return top >= 0x7F800000u ? 255u : (uint32_t)(k > 0 ? k : 0);
}

// 2^-e, which is a normal number for every e that a finite magnitude gives
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// 2^e; 2^-127 is subnormal
__device__ __forceinline__ float mx_scale(uint32_t byte) {
    return __builtin_bit_cast(float, byte == 0u ? 0x00400000u : byte == 255u ? 0x7FC00000u : byte << 23);
}

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }

// The largest of the four lanes that hold a block
__device__ __forceinline__ uint32_t max_of_quad(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));         // quad_perm 1 0 3 2
    return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));      // quad_perm 2 3 0 1
}

// Eight elements in 8 (or 4) bits each; the conversions round to the nearest, ties to even, and no value is past the largest
template <int ELEM>
struct MxWords;
template <>
struct alignas(8) MxWords<8> { uint32_t w[2]; };
template <>
struct MxWords<4> { uint32_t w[1]; };

template <int ELEM>
__device__ __forceinline__ MxWords<ELEM> mx_encode8(const float f[8], uint32_t byte) {
    const float inv = mx_inverse(byte);
    MxWords<ELEM> q;
    if constexpr (ELEM == 8) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h] * inv, f[4 * h + 1] * inv, 0, false);
            v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2] * inv, f[4 * h + 3] * inv, v, true);
            q.w[h] = byte == 255u ? 0x7F7F7F7Fu : (uint32_t)v;
        }
    } else {
        uint32_t v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, f[0] * inv, f[1] * inv, 1.0f, 0);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, f[2] * inv, f[3] * inv, 1.0f, 1);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, f[4] * inv, f[5] * inv, 1.0f, 2);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, f[6] * inv, f[7] * inv, 1.0f, 3);
        q.w[0] = byte == 255u ? 0x77777777u : v;
    }
    return q;
}

template <int ELEM>
__device__ __forceinline__ void mx_decode8(const MxWords<ELEM>& q, uint32_t byte, float f[8]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const float s = mx_scale(byte);
    f32x2 v[4];
    if constexpr (ELEM == 8) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v[2 * h] = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.w[h], false);
            v[2 * h + 1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.w[h], true);
        }
    } else {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q.w[0], 1.0f, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q.w[0], 1.0f, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q.w[0], 1.0f, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q.w[0], 1.0f, 3);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = v[i][0] * s;
        f[2 * i + 1] = v[i][1] * s;
    }
}

// Stores a lane's eight columns col .. col + 7 of a row (0 behind the last) and, with three lanes beside it, their block's
// scale.  All four lanes of a block come here; col runs to the end of the last group.  `shared` of f stand before col, and so
// many columns are missing behind the last of f: the elements are moved as one word.  NARROW: rows of at most 128 columns,
// whose 16 lanes write the whole group of scales, a word each block, as blocks 0 .. 3 are four bytes apart.
template <int ELEM, bool NARROW>
__device__ __forceinline__ void mx_store8(const float f[8], int shared, int64_t row, int col, int cols, int64_t rows, uint8_t* q, uint8_t* scale) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, i < shared ? 0u : magnitude_bits(f[i]));
    const uint32_t byte = mx_scale_byte<ELEM>(max_of_quad(top));
    if (col < (int)mx_filled(cols)) {
        const MxWords<ELEM> w = mx_encode8<ELEM>(f, byte);
        uint8_t* const p = q + row * mx_row_bytes(cols, ELEM) + col * ELEM / 8;
        const int by = byte == 255u ? 0 : (shared & 7) * ELEM;  // (a NaN block's are all alike)
        if constexpr (ELEM == 8) {
            const uint64_t v = ((uint64_t)w.w[1] << 32 | w.w[0]) >> by;
            *reinterpret_cast<uint2*>(p) = uint2{(uint32_t)v, (uint32_t)(v >> 32)};
        } else {
            *reinterpret_cast<uint32_t*>(p) = w.w[0] >> by;
        }
    }
    if ((col & (kMxBlock - 1)) == 0) {
        const int block = col / kMxBlock;
        if constexpr (NARROW) *reinterpret_cast<uint32_t*>(scale + row * 16 + mx_scale_place(block)) = byte;
        else scale[((int64_t)(col / kMxGroup) * rows + row) * 16 + mx_scale_place(block)] = (uint8_t)byte;
    }
}

#endif  // __HIPCC__
}  // namespace dlc
