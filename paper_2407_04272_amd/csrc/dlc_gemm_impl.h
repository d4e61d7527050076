// The matrix products of the dense operators, one template for three element types and three operand layouts.
//
// C[m][n] = sum over k of A(m, k) B(n, k), tile by tile: a work-group takes BM x BN of C and walks k tile by tile.  The
// tiles of A and B go from memory to a ring of slots in LDS, several tiles ahead, without passing through registers; a
// wavefront holds a part of C in registers as 16 x 16 blocks and takes its fragments of a tile from LDS.
//
// 256 x 256 in half precision, 128 x 128 in fp32 (gemm_wide): four wavefronts, each with a quarter, read a step's fragments
// while they multiply the one before.  Half precision has one of them on each SIMD with 128 x 128: a byte read from LDS is
// used for twice the products of a 64 x 64 part, which leaves LDS idle four fifths of the time and the clock higher than
// eight wavefronts of 128 x 64 in two alternating groups did (the card is bound by power, 1.9 to 2.0 GHz here, with the
// matrix cores busy 75 % of the time).  bf16, without an epilogue, k along both rows, down one's and down both's columns:
// 8192 x 2048 x 8192 184, 186 and 187 us = 1495, 1478 and 1465 TFLOP/s (eight wavefronts: 193, 204 and 206; a library 171 to
// 185), 16384 x 8192 x 2048 400, 405 and 408 (421, 439 and 446).  fp32 4096 x 4096 x 4096 926, 941 and 945 us = 148, 146 and
// 145 TFLOP/s, the matrix cores busy 94 % at 2.4 GHz (reads and products in turn: 970, 1004 and 984); 4096 x 1024 x 1664,
// one work-group a compute unit, 104, 107 and 108 us with warm clocks (116 to 122 over the first hundred calls from idle; reads
// and products in turn took 7, 15 and 24 % longer).
// 128 x 128 in half precision and 64 x 128, four wavefronts: two or three work-groups share a compute unit and fill each
// other's gaps (gemm_tile).
//
// LDS layouts (16-byte chunks):
//   k along a row     rows of TB bytes of k, chunk c of row r at place c ^ (r >> 1): what the 16 lanes of a quarter of a
//                     16-byte read touch lies in 16 different sixteenths of the banks (no conflicts counted)
//   k down a column   k row r of BM (BN) elements, units of 16 elements u at u ^ f(r).  Half precision is read with the
//                     transposing read: 16 lanes take 4 k rows of 16 elements, every lane gets the 4 k values of one
//                     element.  fp32 is read element by element.
// A load to LDS writes 64 consecutive chunks per wavefront, so the permutation is applied to the address that is read.
#pragma once
#include "dlc_dense.h"

namespace dlc {

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// One 16 x 16 block times 64 bytes of k: rows from `r`, columns from `c`; lane l gives row (column) l % 16 and the 16 bytes
// of k from (l / 16) * 16 on, and holds D[(l / 16) * 4 + i][l % 16].  (32 x 32 blocks read half the operands and were 8 %
// slower on 8192 x 2048 x 8192: large products run at the clock that the power allows, and theirs was lower.)
template <typename T>
__device__ __forceinline__ f32x4 mma(const u32x4_t& r, const u32x4_t& c, f32x4 acc) {
    if constexpr (std::is_same<T, float>::value) {
        const f32x4 rf = __builtin_bit_cast(f32x4, r), cf = __builtin_bit_cast(f32x4, c);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(rf[j], cf[j], acc, 0, 0, 0);
        return acc;
    } else if constexpr (std::is_same<T, f16_t>::value) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, r), __builtin_bit_cast(f16x8, c), acc, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r), __builtin_bit_cast(bf16x8, c), acc, 0, 0, 0);
    }
}

// 16 bytes from an element's boundary
typedef uint32_t u32x4_by2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));

// elements 0 .. cnt - 1 of a chunk, 0 behind them
template <typename T>
__device__ __forceinline__ u32x4_t load_chunk(const char* p, int cnt) {
    constexpr int EPC = 16 / sizeof(T);
    if (cnt >= EPC) {
        if constexpr (sizeof(T) == 2) return *reinterpret_cast<const u32x4_by2*>(p);
        else return *reinterpret_cast<const u32x4_by4*>(p);
    }
    u32x4_t q = {0u, 0u, 0u, 0u};
    if (cnt > 0) {
#pragma unroll
        for (int j = 0; j < EPC - 1; ++j) {
            if (j < cnt) {
                if constexpr (sizeof(T) == 4) q[j] = reinterpret_cast<const uint32_t*>(p)[j];
                else q[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
            }
        }
    }
    return q;
}

// ---- fragments from LDS ----
// They are read in blocks that wait for their own results.  To the compiler's knowledge a read may touch whatever a load to
// LDS in flight writes, and it would wait for all of those before the read; the kernel's own waits and barriers order the two.

// k along a row: N rows PITCH bytes apart, 16 bytes each
template <int N, int PITCH, int OFF>
__device__ __forceinline__ void read_rows(u32x4_t* o, uint32_t a) {
    if constexpr (N == 2) {
        asm volatile(
            "ds_read_b128 %0, %2 offset:%3\n\t"
            "ds_read_b128 %1, %2 offset:%4\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(o[0]), "=&v"(o[1])
            : "v"(a), "i"(OFF + 0 * PITCH), "i"(OFF + 1 * PITCH) : "memory");
    } else if constexpr (N == 4) {
        asm volatile(
            "ds_read_b128 %0, %4 offset:%5\n\t"
            "ds_read_b128 %1, %4 offset:%6\n\t"
            "ds_read_b128 %2, %4 offset:%7\n\t"
            "ds_read_b128 %3, %4 offset:%8\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3])
            : "v"(a), "i"(OFF + 0 * PITCH), "i"(OFF + 1 * PITCH), "i"(OFF + 2 * PITCH), "i"(OFF + 3 * PITCH) : "memory");
    } else if constexpr (N == 8) {
        asm volatile(
            "ds_read_b128 %0, %8 offset:%9\n\t"
            "ds_read_b128 %1, %8 offset:%10\n\t"
            "ds_read_b128 %2, %8 offset:%11\n\t"
            "ds_read_b128 %3, %8 offset:%12\n\t"
            "ds_read_b128 %4, %8 offset:%13\n\t"
            "ds_read_b128 %5, %8 offset:%14\n\t"
            "ds_read_b128 %6, %8 offset:%15\n\t"
            "ds_read_b128 %7, %8 offset:%16\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]), "=&v"(o[4]), "=&v"(o[5]), "=&v"(o[6]), "=&v"(o[7])
            : "v"(a), "i"(OFF + 0 * PITCH), "i"(OFF + 1 * PITCH), "i"(OFF + 2 * PITCH), "i"(OFF + 3 * PITCH), "i"(OFF + 4 * PITCH), "i"(OFF + 5 * PITCH), "i"(OFF + 6 * PITCH), "i"(OFF + 7 * PITCH) : "memory");
    }
}

// ... of both operands
template <int NA, int NB, int PITCH, int OFF>
__device__ __forceinline__ void read_rows2(u32x4_t* x, uint32_t a, u32x4_t* y, uint32_t b) {
    static_assert((NA == 2 || NA == 4) && NB == 4, "");
    if constexpr (NA == 2) {
        asm volatile(
            "ds_read_b128 %2, %7 offset:%8\n\t"
            "ds_read_b128 %3, %7 offset:%9\n\t"
            "ds_read_b128 %4, %7 offset:%10\n\t"
            "ds_read_b128 %5, %7 offset:%11\n\t"
            "ds_read_b128 %0, %6 offset:%8\n\t"
            "ds_read_b128 %1, %6 offset:%9\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(x[0]), "=&v"(x[1]), "=&v"(y[0]), "=&v"(y[1]), "=&v"(y[2]), "=&v"(y[3])
            : "v"(a), "v"(b), "i"(OFF + 0 * PITCH), "i"(OFF + 1 * PITCH), "i"(OFF + 2 * PITCH), "i"(OFF + 3 * PITCH) : "memory");
    } else {
        asm volatile(
            "ds_read_b128 %4, %9 offset:%10\n\t"
            "ds_read_b128 %5, %9 offset:%11\n\t"
            "ds_read_b128 %6, %9 offset:%12\n\t"
            "ds_read_b128 %7, %9 offset:%13\n\t"
            "ds_read_b128 %0, %8 offset:%10\n\t"
            "ds_read_b128 %1, %8 offset:%11\n\t"
            "ds_read_b128 %2, %8 offset:%12\n\t"
            "ds_read_b128 %3, %8 offset:%13\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(y[0]), "=&v"(y[1]), "=&v"(y[2]), "=&v"(y[3])
            : "v"(a), "v"(b), "i"(OFF + 0 * PITCH), "i"(OFF + 1 * PITCH), "i"(OFF + 2 * PITCH), "i"(OFF + 3 * PITCH) : "memory");
    }
}

// ... both halves of N slots' rows, PITCH bytes apart (at a and b)
template <int N, int PITCH>
__device__ __forceinline__ void read_halves(u32x4_t* o, uint32_t a, uint32_t b) {
    if constexpr (N == 2) {
        asm volatile(
            "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\t"
            "ds_read_b128 %2, %4 offset:%6\n\tds_read_b128 %3, %5 offset:%6\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]) : "v"(a), "v"(b), "i"(PITCH) : "memory");
    } else if constexpr (N == 4) {
        asm volatile(
            "ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\t"
            "ds_read_b128 %2, %8 offset:%10\n\tds_read_b128 %3, %9 offset:%10\n\t"
            "ds_read_b128 %4, %8 offset:%11\n\tds_read_b128 %5, %9 offset:%11\n\t"
            "ds_read_b128 %6, %8 offset:%12\n\tds_read_b128 %7, %9 offset:%12\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]), "=&v"(o[4]), "=&v"(o[5]), "=&v"(o[6]), "=&v"(o[7])
            : "v"(a), "v"(b), "i"(PITCH), "i"(2 * PITCH), "i"(3 * PITCH) : "memory");
    } else {
        static_assert(N == 3, "");
        asm volatile(
            "ds_read_b128 %0, %6\n\tds_read_b128 %1, %7\n\t"
            "ds_read_b128 %2, %6 offset:%8\n\tds_read_b128 %3, %7 offset:%8\n\t"
            "ds_read_b128 %4, %6 offset:%9\n\tds_read_b128 %5, %7 offset:%9\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]), "=&v"(o[4]), "=&v"(o[5])
            : "v"(a), "v"(b), "i"(PITCH), "i"(2 * PITCH) : "memory");
    }
}

__device__ __forceinline__ u32x4_t join_halves(s16x4 lo, s16x4 hi) {
    return __builtin_bit_cast(u32x4_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// k down a column, half precision: the transposing read, 4 k rows and the next 4, K4 bytes on
template <int N, int OFF, int K4>
__device__ __forceinline__ void read_cols(u32x4_t* o, const uint32_t* a) {
    if constexpr (N == 2) {
        s16x4 v0, v1, v2, v3;
        asm volatile(
            "ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
            "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v0), "=&v"(v1), "=&v"(v2), "=&v"(v3)
            : "v"(a[0]), "v"(a[1]), "i"(OFF), "i"(OFF + K4) : "memory");
        o[0] = join_halves(v0, v1);
        o[1] = join_halves(v2, v3);
    } else if constexpr (N == 4) {
        s16x4 v0, v1, v2, v3, v4, v5, v6, v7;
        asm volatile(
            "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
            "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
            "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
            "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v0), "=&v"(v1), "=&v"(v2), "=&v"(v3), "=&v"(v4), "=&v"(v5), "=&v"(v6), "=&v"(v7)
            : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "i"(OFF), "i"(OFF + K4) : "memory");
        o[0] = join_halves(v0, v1);
        o[1] = join_halves(v2, v3);
        o[2] = join_halves(v4, v5);
        o[3] = join_halves(v6, v7);
    } else if constexpr (N == 8) {
        s16x4 v0, v1, v2, v3, v4, v5, v6, v7, v8, v9, v10, v11, v12, v13, v14, v15;
        asm volatile(
            "ds_read_b64_tr_b16 %0, %16 offset:%24\n\tds_read_b64_tr_b16 %1, %16 offset:%25\n\t"
            "ds_read_b64_tr_b16 %2, %17 offset:%24\n\tds_read_b64_tr_b16 %3, %17 offset:%25\n\t"
            "ds_read_b64_tr_b16 %4, %18 offset:%24\n\tds_read_b64_tr_b16 %5, %18 offset:%25\n\t"
            "ds_read_b64_tr_b16 %6, %19 offset:%24\n\tds_read_b64_tr_b16 %7, %19 offset:%25\n\t"
            "ds_read_b64_tr_b16 %8, %20 offset:%24\n\tds_read_b64_tr_b16 %9, %20 offset:%25\n\t"
            "ds_read_b64_tr_b16 %10, %21 offset:%24\n\tds_read_b64_tr_b16 %11, %21 offset:%25\n\t"
            "ds_read_b64_tr_b16 %12, %22 offset:%24\n\tds_read_b64_tr_b16 %13, %22 offset:%25\n\t"
            "ds_read_b64_tr_b16 %14, %23 offset:%24\n\tds_read_b64_tr_b16 %15, %23 offset:%25\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v0), "=&v"(v1), "=&v"(v2), "=&v"(v3), "=&v"(v4), "=&v"(v5), "=&v"(v6), "=&v"(v7), "=&v"(v8), "=&v"(v9), "=&v"(v10), "=&v"(v11), "=&v"(v12), "=&v"(v13), "=&v"(v14), "=&v"(v15)
            : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7]), "i"(OFF), "i"(OFF + K4) : "memory");
        o[0] = join_halves(v0, v1);
        o[1] = join_halves(v2, v3);
        o[2] = join_halves(v4, v5);
        o[3] = join_halves(v6, v7);
        o[4] = join_halves(v8, v9);
        o[5] = join_halves(v10, v11);
        o[6] = join_halves(v12, v13);
        o[7] = join_halves(v14, v15);
    }
}

// k down a column, fp32: element by element, 4 k rows ROW bytes apart
template <int OFF, int ROW>
__device__ __forceinline__ void read_cols_f32(u32x4_t& o, uint32_t a) {
    uint32_t v0, v1, v2, v3;
    asm volatile(
        "ds_read_b32 %0, %4 offset:%5\n\tds_read_b32 %1, %4 offset:%6\n\t"
        "ds_read_b32 %2, %4 offset:%7\n\tds_read_b32 %3, %4 offset:%8\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(v0), "=&v"(v1), "=&v"(v2), "=&v"(v3)
        : "v"(a), "i"(OFF), "i"(OFF + ROW), "i"(OFF + 2 * ROW), "i"(OFF + 3 * ROW) : "memory");
    o = u32x4_t{v0, v1, v2, v3};
}

// ---- the inner loop of the 256 x 256 tile ----
// 16 products of 16 x 16 x 32, while four fragments of the next step are read from LDS and two loads to LDS are started.  It
// is one block of assembly because a wavefront has its SIMD to itself: whatever else it issues has to stand between the
// products, or the matrix cores wait.  The block waits for its own reads; the loads write no register.  The sums are kept
// in the second half of the register file ("a"), which leaves the first to two steps' fragments.
struct LoadTo {
    uint32_t v0, v1;  // offsets
    u32x4_t s0, s1;   // sources
    uint32_t at;      // where in LDS the wavefront's first load of the tile goes
};

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is the compiler's to set before each use: none lives across)
#define DLC_MFMA(TY, ACC, B, A) "v_mfma_f32_16x16x32_" TY " %" #ACC ", %" #B ", %" #A ", %" #ACC "\n\t"
#define DLC_CHUNK_ROWS(TY) \
    asm volatile( \
    DLC_MFMA(TY, 4, 22, 20) "ds_read_b128 %0, %30 offset:%31\n\t" DLC_MFMA(TY, 5, 23, 20) \
    "ds_read_b128 %1, %30 offset:%32\n\t" DLC_MFMA(TY, 6, 24, 20) "ds_read_b128 %2, %30 offset:%33\n\t" \
    DLC_MFMA(TY, 7, 25, 20) "ds_read_b128 %3, %30 offset:%34\n\t" DLC_MFMA(TY, 8, 26, 20) DLC_MFMA(TY, 9, 27, 20) \
    "s_add_u32 m0, %39, %40\n\t" DLC_MFMA(TY, 10, 28, 20) "buffer_load_dwordx4 %35, %37, 0 offen lds\n\t" \
    DLC_MFMA(TY, 11, 29, 20) DLC_MFMA(TY, 12, 22, 21) DLC_MFMA(TY, 13, 23, 21) DLC_MFMA(TY, 14, 24, 21) \
    "s_add_u32 m0, %39, %41\n\t" DLC_MFMA(TY, 15, 25, 21) "buffer_load_dwordx4 %36, %38, 0 offen lds\n\t" \
    DLC_MFMA(TY, 16, 26, 21) DLC_MFMA(TY, 17, 27, 21) DLC_MFMA(TY, 18, 28, 21) DLC_MFMA(TY, 19, 29, 21) \
    "s_waitcnt lgkmcnt(0)" \
    : "=&v"(next[0]), "=&v"(next[1]), "=&v"(next[2]), "=&v"(next[3]), \
      "+a"(acc0[0]), "+a"(acc0[1]), "+a"(acc0[2]), "+a"(acc0[3]), "+a"(acc0[4]), "+a"(acc0[5]), "+a"(acc0[6]), "+a"(acc0[7]), \
      "+a"(acc1[0]), "+a"(acc1[1]), "+a"(acc1[2]), "+a"(acc1[3]), "+a"(acc1[4]), "+a"(acc1[5]), "+a"(acc1[6]), "+a"(acc1[7]) \
    : "v"(a0), "v"(a1), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(b[4]), "v"(b[5]), "v"(b[6]), "v"(b[7]), \
      "v"(from[0]), "i"(OFF), "i"(OFF + STEP), "i"(OFF + 2 * STEP), "i"(OFF + 3 * STEP), \
      "v"(to.v0), "v"(to.v1), "s"(to.s0), "s"(to.s1), "s"(to.at), "i"(I * 8192), "i"(I * 8192 + 4096) \
    : "memory", "m0", "scc")
#define DLC_CHUNK_COLS(TY) \
    asm volatile( \
    DLC_MFMA(TY, 8, 26, 24) "ds_read_b64_tr_b16 %0, %34 offset:%38\n\t" DLC_MFMA(TY, 9, 27, 24) \
    "ds_read_b64_tr_b16 %1, %34 offset:%39\n\t" DLC_MFMA(TY, 10, 28, 24) "ds_read_b64_tr_b16 %2, %35 offset:%38\n\t" \
    DLC_MFMA(TY, 11, 29, 24) "ds_read_b64_tr_b16 %3, %35 offset:%39\n\t" DLC_MFMA(TY, 12, 30, 24) \
    "ds_read_b64_tr_b16 %4, %36 offset:%38\n\t" DLC_MFMA(TY, 13, 31, 24) "ds_read_b64_tr_b16 %5, %36 offset:%39\n\t" \
    DLC_MFMA(TY, 14, 32, 24) "ds_read_b64_tr_b16 %6, %37 offset:%38\n\t" DLC_MFMA(TY, 15, 33, 24) \
    "ds_read_b64_tr_b16 %7, %37 offset:%39\n\t" DLC_MFMA(TY, 16, 26, 25) "s_add_u32 m0, %44, %45\n\t" \
    DLC_MFMA(TY, 17, 27, 25) "buffer_load_dwordx4 %40, %42, 0 offen lds\n\t" DLC_MFMA(TY, 18, 28, 25) \
    DLC_MFMA(TY, 19, 29, 25) "s_add_u32 m0, %44, %46\n\t" DLC_MFMA(TY, 20, 30, 25) \
    "buffer_load_dwordx4 %41, %43, 0 offen lds\n\t" DLC_MFMA(TY, 21, 31, 25) DLC_MFMA(TY, 22, 32, 25) \
    DLC_MFMA(TY, 23, 33, 25) "s_waitcnt lgkmcnt(0)" \
    : "=&v"(h0), "=&v"(h1), "=&v"(h2), "=&v"(h3), "=&v"(h4), "=&v"(h5), "=&v"(h6), "=&v"(h7), \
      "+a"(acc0[0]), "+a"(acc0[1]), "+a"(acc0[2]), "+a"(acc0[3]), "+a"(acc0[4]), "+a"(acc0[5]), "+a"(acc0[6]), "+a"(acc0[7]), \
      "+a"(acc1[0]), "+a"(acc1[1]), "+a"(acc1[2]), "+a"(acc1[3]), "+a"(acc1[4]), "+a"(acc1[5]), "+a"(acc1[6]), "+a"(acc1[7]) \
    : "v"(a0), "v"(a1), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(b[4]), "v"(b[5]), "v"(b[6]), "v"(b[7]), \
      "v"(from[0]), "v"(from[1]), "v"(from[2]), "v"(from[3]), "i"(OFF), "i"(OFF + STEP), \
      "v"(to.v0), "v"(to.v1), "s"(to.s0), "s"(to.s1), "s"(to.at), "i"(I * 8192), "i"(I * 8192 + 4096) \
    : "memory", "m0", "scc")

// acc0, acc1: rows of blocks, a0 and a1 times b.  COLS: the fragments read have k down a column (from: four addresses, STEP
// to the second half), else along a row (from: one, STEP from block to block).  I: the loads are numbers 2 I and 2 I + 1.
template <typename T, bool COLS, int OFF, int STEP, int I>
__device__ __forceinline__ void chunk16(f32x4* acc0, f32x4* acc1, const u32x4_t& a0, const u32x4_t& a1, const u32x4_t* b, u32x4_t* next,
                                        const uint32_t* from, const LoadTo& to) {
    constexpr bool F16 = std::is_same<T, f16_t>::value;
    if constexpr (!COLS) {
        if constexpr (F16) DLC_CHUNK_ROWS("f16");
        else DLC_CHUNK_ROWS("bf16");
    } else {
        s16x4 h0, h1, h2, h3, h4, h5, h6, h7;
        if constexpr (F16) DLC_CHUNK_COLS("f16");
        else DLC_CHUNK_COLS("bf16");
        next[0] = join_halves(h0, h1);
        next[1] = join_halves(h2, h3);
        next[2] = join_halves(h4, h5);
        next[3] = join_halves(h6, h7);
    }
}
#undef DLC_CHUNK_ROWS
#undef DLC_CHUNK_COLS
#undef DLC_MFMA

#define DLC_MFMA_F32(ACC, B, A) "v_mfma_f32_16x16x4_f32 %" #ACC ", %" #B ", %" #A ", %" #ACC "\n\t"
#define DLC_CHUNK_ROWS_F32 \
    asm volatile( \
    DLC_MFMA_F32(2, 22, 18) "ds_read_b128 %0, %26 offset:%27\n\t" DLC_MFMA_F32(3, 23, 18) \
    "ds_read_b128 %1, %26 offset:%28\n\t" DLC_MFMA_F32(4, 24, 18) DLC_MFMA_F32(5, 25, 18) DLC_MFMA_F32(6, 22, 19) \
    "s_add_u32 m0, %31, %32\n\t" DLC_MFMA_F32(7, 23, 19) "buffer_load_dwordx4 %29, %30, 0 offen lds\n\t" \
    DLC_MFMA_F32(8, 24, 19) DLC_MFMA_F32(9, 25, 19) DLC_MFMA_F32(10, 22, 20) DLC_MFMA_F32(11, 23, 20) \
    DLC_MFMA_F32(12, 24, 20) DLC_MFMA_F32(13, 25, 20) DLC_MFMA_F32(14, 22, 21) DLC_MFMA_F32(15, 23, 21) \
    DLC_MFMA_F32(16, 24, 21) DLC_MFMA_F32(17, 25, 21) "s_waitcnt lgkmcnt(0)" \
    : "=&v"(next[0]), "=&v"(next[1]), \
      "+a"(acc[0][0]), "+a"(acc[0][1]), "+a"(acc[0][2]), "+a"(acc[0][3]), \
      "+a"(acc[1][0]), "+a"(acc[1][1]), "+a"(acc[1][2]), "+a"(acc[1][3]), \
      "+a"(acc[2][0]), "+a"(acc[2][1]), "+a"(acc[2][2]), "+a"(acc[2][3]), \
      "+a"(acc[3][0]), "+a"(acc[3][1]), "+a"(acc[3][2]), "+a"(acc[3][3]) \
    : "v"(a[0][K]), "v"(a[1][K]), "v"(a[2][K]), "v"(a[3][K]), "v"(b[0][K]), "v"(b[1][K]), "v"(b[2][K]), "v"(b[3][K]), \
      "v"(from[0]), "i"(OFF), "i"(OFF + STEP), "v"(to.v0), "s"(to.s0), "s"(to.at), "i"(I * 4096) \
    : "memory", "m0", "scc")
#define DLC_CHUNK_COLS_F32 \
    asm volatile( \
    DLC_MFMA_F32(8, 28, 24) "ds_read_b32 %0, %32 offset:%34\n\t" DLC_MFMA_F32(9, 29, 24) \
    "ds_read_b32 %1, %32 offset:%35\n\t" DLC_MFMA_F32(10, 30, 24) "ds_read_b32 %2, %32 offset:%36\n\t" \
    DLC_MFMA_F32(11, 31, 24) "ds_read_b32 %3, %32 offset:%37\n\t" DLC_MFMA_F32(12, 28, 25) \
    "ds_read_b32 %4, %33 offset:%34\n\t" DLC_MFMA_F32(13, 29, 25) "ds_read_b32 %5, %33 offset:%35\n\t" \
    DLC_MFMA_F32(14, 30, 25) "ds_read_b32 %6, %33 offset:%36\n\t" DLC_MFMA_F32(15, 31, 25) \
    "ds_read_b32 %7, %33 offset:%37\n\t" DLC_MFMA_F32(16, 28, 26) DLC_MFMA_F32(17, 29, 26) \
    "s_add_u32 m0, %40, %41\n\t" DLC_MFMA_F32(18, 30, 26) "buffer_load_dwordx4 %38, %39, 0 offen lds\n\t" \
    DLC_MFMA_F32(19, 31, 26) DLC_MFMA_F32(20, 28, 27) DLC_MFMA_F32(21, 29, 27) DLC_MFMA_F32(22, 30, 27) \
    DLC_MFMA_F32(23, 31, 27) "s_waitcnt lgkmcnt(0)" \
    : "=&v"(h0), "=&v"(h1), "=&v"(h2), "=&v"(h3), "=&v"(h4), "=&v"(h5), "=&v"(h6), "=&v"(h7), \
      "+a"(acc[0][0]), "+a"(acc[0][1]), "+a"(acc[0][2]), "+a"(acc[0][3]), \
      "+a"(acc[1][0]), "+a"(acc[1][1]), "+a"(acc[1][2]), "+a"(acc[1][3]), \
      "+a"(acc[2][0]), "+a"(acc[2][1]), "+a"(acc[2][2]), "+a"(acc[2][3]), \
      "+a"(acc[3][0]), "+a"(acc[3][1]), "+a"(acc[3][2]), "+a"(acc[3][3]) \
    : "v"(a[0][K]), "v"(a[1][K]), "v"(a[2][K]), "v"(a[3][K]), "v"(b[0][K]), "v"(b[1][K]), "v"(b[2][K]), "v"(b[3][K]), \
      "v"(from[0]), "v"(from[1]), "i"(OFF), "i"(OFF + STEP), "i"(OFF + 2 * STEP), "i"(OFF + 3 * STEP), "v"(to.v0), "s"(to.s0), "s"(to.at), "i"(I * 4096) \
    : "memory", "m0", "scc")

// fp32: 16 products of 16 x 16 x 4, of value K of every fragment; two fragments are read and load I is started
template <bool COLS, int K, int OFF, int STEP, int I>
__device__ __forceinline__ void chunk16_f32(f32x4 (&acc)[4][4], const u32x4_t* a, const u32x4_t* b, u32x4_t* next, const uint32_t* from,
                                            const LoadTo& to) {
    if constexpr (!COLS) {
        DLC_CHUNK_ROWS_F32;
    } else {
        uint32_t h0, h1, h2, h3, h4, h5, h6, h7;
        DLC_CHUNK_COLS_F32;
        next[0] = u32x4_t{h0, h1, h2, h3};
        next[1] = u32x4_t{h4, h5, h6, h7};
    }
}
#undef DLC_CHUNK_ROWS_F32
#undef DLC_CHUNK_COLS_F32
#undef DLC_MFMA_F32
#pragma clang diagnostic pop

// The sums are in their registers: products that assembly started are not known to the compiler
template <int MI, int NJ>
__device__ __forceinline__ void settle(f32x4 (&acc)[MI][NJ]) {
    asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) asm volatile("" : "+a"(acc[i][j]));
}

// Permutation of a k row's units where k runs down a column, UNITS of them in a row: the k rows that are read together
// (half precision: 4 consecutive ones and the 4 that stand 8 further; fp32: 4 that are 4 apart) get different values.
template <typename T, int UNITS>
__device__ __forceinline__ int unit_swizzle(int krow) {
    const int f = sizeof(T) == 4 ? (krow >> 2) & 3 : (krow & 3) | (((krow >> 3) & 1) << 2);
    return f & (UNITS - 1);
}

// One operand's path into LDS.  KT: k runs down a column.  R: rows (columns of C) of the tile.  TB: bytes of k of a tile.
// DUAL: the tile's rows are those of two matrices one behind the other, 32 of the first and 32 of the second in turn.
// Rows start on 16-byte boundaries, and what stands between a row's end and the next boundary is zeros or outside the sum.
template <typename T, bool KT, int R, int TB, int THREADS, bool DUAL>
struct Operand {
    static constexpr int EPC = 16 / sizeof(T);           // elements of a chunk
    static constexpr int BK = TB / sizeof(T);            // k values of a tile
    static constexpr int CPR = KT ? R / EPC : TB / 16;   // chunks of a row in LDS
    static constexpr int ROWS = KT ? BK : R;             // rows in LDS
    static constexpr int PASSES = ROWS * CPR / THREADS;  // chunks a thread moves
    static constexpr int RSTEP = THREADS / CPR;          // rows between them
    static constexpr int BYTES = ROWS * CPR * 16;
    static_assert(PASSES * THREADS == ROWS * CPR, "tile and work-group");
    static_assert(KT || RSTEP % 16 == 0, "a thread's chunks are at one place of their rows");

    // An offset past the buffer's range: the load gives 0.  (The range ends here; a tile's rows span no more than
    // 256 * 2^22 bytes = 2^30.)
    static constexpr uint32_t kOut = 0x7FFFFFF0u;

    const char* base;       // of the tile's first row and the current k tile
    int64_t step;           // bytes to the next k tile
    int64_t ld;             // bytes
    int64_t half_off;       // DUAL: bytes from a row of the first matrix to the same row of the second
    int k_left;             // k values from the current tile on
    int key;                // the k value in a tile of a thread's first chunk (k along a row: of the chunk's first element)
    int row0, slot;         // the thread's first row and its place in it
    uint32_t voff[PASSES];  // offsets of the thread's chunks from base, kOut outside the matrix

    // the chunk that stands at place `s` of row r
    __device__ __forceinline__ static int chunk_at(int r, int s) {
        if constexpr (KT) {
            constexpr int UB = sizeof(T) == 4 ? 2 : 1;  // log2 of a unit's chunks
            return (((s >> UB) ^ unit_swizzle<T, (CPR >> UB)>(r)) << UB) | (s & ((1 << UB) - 1));
        } else {
            return s ^ ((r >> 1) & (CPR - 1));
        }
    }
    __device__ __forceinline__ int chunk_of(int i) const { return chunk_at(row0 + i * RSTEP, slot); }
    // DUAL: row r of the tile is row f of its matrix
    __device__ __forceinline__ static int source_row(int r) { return DUAL ? ((r >> 6) << 5) | (r & 31) : r; }

    // row: first row (column) of the tile; rows: of the matrix (DUAL: of one of the two)
    __device__ __forceinline__ void init(const void* p, int64_t ld_elems, int row, int rows, int k0, int k1, int tid) {
        ld = ld_elems * (int64_t)sizeof(T);
        row0 = tid / CPR;
        slot = tid % CPR;
        const int rows_left = rows - row;
        k_left = k1 - k0;
        const int64_t down = KT ? k0 : row, along = KT ? row : k0;
        base = static_cast<const char*>(p) + down * ld + along * (int64_t)sizeof(T);
        step = KT ? (int64_t)BK * ld : (int64_t)TB;
        half_off = (int64_t)rows * ld;
        key = KT ? row0 : chunk_of(0) * EPC;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int r = row0 + i * RSTEP, c = chunk_of(i), f = source_row(r);
            const bool in = KT ? c * EPC < rows_left : f < rows_left;
            voff[i] = in ? (uint32_t)f * (uint32_t)ld + (uint32_t)c * 16u : kOut;
        }
    }

    // Before a k tile's loads: what lies outside the matrix becomes 0, and so do tiles past the last.
    __device__ __forceinline__ void mask() {
        if (k_left < BK) {  // (the last tile; those behind it stay empty)
#pragma unroll
            for (int i = 0; i < PASSES; ++i) voff[i] = key + (KT ? i * RSTEP : 0) < k_left ? voff[i] : kOut;
        }
    }
    // What a thread's chunks i with i % 2 = odd are loaded from (DUAL: its rows 32 .. 63 of each 64 are the second matrix's)
    __device__ __forceinline__ u32x4_t source(int odd) const {
        static_assert(!DUAL || RSTEP == 32, "a pass's rows are all of one matrix");
        const uint64_t p = (uint64_t)(uintptr_t)(base + (DUAL && odd ? half_off : 0));
        return u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32) & 0xFFFFu), kOut,
                       0x00020000u};
    }
    // Behind them: on to the next k tile
    __device__ __forceinline__ void advance() {
        k_left -= BK;
        base += step;
    }
    // Starts loads FROM .. FROM + N - 1 of the current k tile to `lds`
    template <int FROM, int N>
    __device__ __forceinline__ void load(char* lds, int tid) const {
        const int wave_lds = (tid & ~63) * 16;
#pragma unroll
        for (int i = FROM; i < FROM + N; ++i) {
            char* const dst = lds + wave_lds + i * THREADS * 16;
            const char* const src = base + (DUAL && i % 2 ? half_off : 0);
            const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)src, 0, kOut, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)dst, 16, voff[i], 0, 0, 0);
        }
    }
    // All of them
    __device__ __forceinline__ void fetch(char* lds, int tid) {
        mask();
        load<0, PASSES>(lds, tid);
        advance();
    }

    // Where a lane reads in a tile: row (column) `row` + l % 16 of N blocks of 16, its k values (l / 16) * 16 bytes on in
    // each 64 bytes of k (k along a row: block i stands 16 rows on)
    template <int N>
    struct Place {
        static constexpr int COUNT = KT ? N : TB / 64;
        uint32_t a[COUNT];
    };
    template <int N>
    __device__ __forceinline__ static void place(Place<N>& p, uint32_t at, int row, int lane) {
        const int g = lane >> 4, j = lane & 15;
        if constexpr (!KT) {
#pragma unroll
            for (int h = 0; h < TB / 64; ++h)
                p.a[h] = at + (uint32_t)((row + j) * TB + (((h * 4 + g) ^ ((j >> 1) & (CPR - 1))) << 4));
        } else if constexpr (sizeof(T) == 2) {
            const int k = g * 8 + (j >> 2), f = unit_swizzle<T, CPR / 2>(k);  // (the same for k + 4)
#pragma unroll
            for (int v = 0; v < N; ++v) p.a[v] = at + (uint32_t)(k * (CPR * 16) + (j & 3) * 8 + ((((row >> 4) + v) ^ f) << 5));
        } else {
            const int f = unit_swizzle<T, CPR / 4>(g * 4);  // (the same for the four k rows)
#pragma unroll
            for (int v = 0; v < N; ++v) p.a[v] = at + (uint32_t)(g * 4 * (CPR * 16) + j * 4 + ((((row >> 4) + v) ^ f) << 6));
        }
    }
    // Fragments of the N blocks from the tile OFF bytes on (TB = 64)
    template <int N, int OFF>
    __device__ __forceinline__ static void frags(u32x4_t (&out)[N], const Place<N>& p) {
        static_assert(TB == 64, "one block of k");
        if constexpr (!KT) {
            read_rows<N, 16 * TB, OFF>(out, p.a[0]);
        } else if constexpr (sizeof(T) == 2) {
            read_cols<N, OFF, 4 * CPR * 16>(out, p.a);
        } else {
#pragma unroll
            for (int v = 0; v < N; ++v) read_cols_f32<OFF, CPR * 16>(out[v], p.a[v]);
        }
    }
};

// orders a wavefront's LDS accesses before the ones after it (its own lanes only)
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A barrier that nothing is moved across, and that waits for nothing itself: what has to be there is waited for before it.
__device__ __forceinline__ void bare_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// waits until no more than N of this wavefront's loads are in flight
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
    asm volatile("" ::: "memory");
}

// Work-group -> tile.  Consecutive work-groups go to the 8 XCDs in turn; each XCD gets a stretch of consecutive tiles, and
// those run down 4 tile rows before the next column, so that the 32 tiles an XCD works on at a time share rows and columns
// in its L2 (nine requests in ten hit) and rows of up to 8 tiles are read once (8 and 16 tile rows: 3 and 5 % slower where
// there are several rounds of tiles).
__device__ __forceinline__ void tile_of(int wg, int total, int tiles_m, int tiles_n, int& tm, int& tn, int& sp) {
    const int q = total / 8, r = total % 8, x = wg % 8, i = wg / 8;
    int t = x < r ? x * (q + 1) + i : r * (q + 1) + (x - r) * q + i;
    const int per = tiles_m * tiles_n;
    sp = t / per;
    t -= sp * per;
    const int band = 4 * tiles_n, b0 = t / band;
    const int h = min(4, tiles_m - b0 * 4);
    t -= b0 * band;
    tm = b0 * 4 + t % h;
    tn = t / h;
}

// RM x 64 of a wavefront's sums (acc[RM / 16][j0 .. j0 + 3]) through a piece of LDS of its own, so that a lane gets eight
// consecutive columns, and the epilogue.  The 16-byte units of a row are permuted by the row.  m0, n0: the first row and
// column of y
template <typename T, bool GATED, int RM, int NJ>
__device__ __forceinline__ void write_block(const GemmArgs& ga, const f32x4 (*acc)[NJ], int j0, char* buf, int m0, int n0, int sp, int lane) {
    const uint64_t offset = full_offset(ga.e.offset, ga.e.d_offset);
    const int g = lane >> 4, c16 = lane & 15;
    constexpr int CH = GATED ? 4 : 8;  // chunks of eight columns in a row
#pragma unroll
    for (int i = 0; i < RM / 16; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *reinterpret_cast<f32x4*>(buf + (i * 16 + c16) * 256 + (((j * 4 + g) ^ c16) << 4)) = acc[i][j0 + j];
    wave_sync();
    constexpr int STEP = 64 / CH;  // a lane's rows are so far apart, its columns the same
    // Rows at a time, whose residuals and results are on their way together: one by one, 16384 x 2048 x 2048 backward took 260
    // us for 247, 8192 x 1024 x 512 41 for 37 (gated, four: too many registers on the small tiles, 20 us for 17.5)
    constexpr int AT_ONCE = GATED ? 2 : 4;
    const int ch = lane % CH, row0 = lane / CH, col = n0 + ch * 8;
#pragma unroll 1
    for (int q = 0; q < RM; q += STEP * AT_ONCE) {
        float s[AT_ONCE][8], u[AT_ONCE][8];
        const int m = m0 + q + row0;
#pragma unroll
        for (int r = 0; r < AT_ONCE; ++r) {
            const int row = q + r * STEP + row0;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                *reinterpret_cast<f32x4*>(s[r] + v * 4) = *reinterpret_cast<const f32x4*>(buf + row * 256 + (((ch * 2 + v) ^ (row & 15)) << 4));
                if constexpr (GATED)
                    *reinterpret_cast<f32x4*>(u[r] + v * 4) = *reinterpret_cast<const f32x4*>(buf + row * 256 + (((8 + ch * 2 + v) ^ (row & 15)) << 4));
            }
        }
        if (m >= ga.M) continue;
        if (ga.split == 1) {
            epilogue8<T, GATED, AT_ONCE, STEP>(ga.e, offset, m, ga.M - m, col, s, u);
        } else if (col < ga.N) {  // (the pitch of the partial sums has room for whole chunks)
#pragma unroll
            for (int r = 0; r < AT_ONCE; ++r) {
                if (m + r * STEP >= ga.M) continue;
                float* p = ga.part + ((int64_t)sp * ga.M + m + r * STEP) * ga.part_ld + col;
                *reinterpret_cast<f32x4*>(p) = *reinterpret_cast<f32x4*>(s[r]);
                *reinterpret_cast<f32x4*>(p + 4) = *reinterpret_cast<f32x4*>(s[r] + 4);
                if constexpr (GATED) {
                    float* p2 = p + ((ga.N + 7) & ~7);
                    *reinterpret_cast<f32x4*>(p2) = *reinterpret_cast<f32x4*>(u[r]);
                    *reinterpret_cast<f32x4*>(p2 + 4) = *reinterpret_cast<f32x4*>(u[r] + 4);
                }
            }
        }
    }
    wave_sync();
}

// a lane's places are kept in registers, not made again
template <typename P>
__device__ __forceinline__ void keep(P& p) {
#pragma unroll
    for (int i = 0; i < P::COUNT; ++i) asm volatile("" : "+v"(p.a[i]));
}

// ... and of gemm_wide's: all of a compute unit's, in fp32 half of it
template <typename T>
constexpr int wide_lds() {
    return sizeof(T) == 2 ? 160 * 1024 : 80 * 1024;
}

// LDS of a work-group: with k along the rows three slots for A and two or three for B, otherwise four for both
template <typename T, int LAY, int BM, int BN>
constexpr int gemm_lds() {
    return LAY == L_KK ? 3 * BM * 128 + (BM == 64 ? 3 : 2) * BN * 128 : 4 * (BM + BN) * 64;
}

// Tile `wg` of `total` of a product (the tiles of every cut of k), 128 x 128 (half precision) or 64 x 128
template <typename T, int LAY, int BM, int BN, bool GATED>
__device__ __forceinline__ void gemm_tile(const GemmArgs& ga, int wg, int total, char* const lds) {
    constexpr int WAVES = 4, THREADS = 256;
    constexpr int WM = BM / 2, WN = BN / 2, MI = WM / 16, NJ = WN / 16;
    // With k along both operands' rows a tile has 128 bytes of them: whole cache lines, half the requests.  With k down a
    // column a row is long anyway, and tiles of 64 bytes in four slots spread the loads over the phases.
    constexpr int TB = LAY == L_KK ? 128 : 64;
    constexpr int BK = TB / sizeof(T);
    using OpA = Operand<T, LAY == L_TT, BM, TB, THREADS, false>;
    using OpB = Operand<T, LAY != L_KK, BN, TB, THREADS, GATED>;
    static_assert(WN == 64, "a wavefront's columns (gated: 32 of the gate and 32 of the other)");
    constexpr int STAGE = OpA::BYTES + OpB::BYTES;
    constexpr int A3 = 3 * OpA::BYTES;  // k along the rows: where B's slots start
    constexpr bool DEEP = BM == 64;     // there is room for a third (128 x 4096 x 4096 in bf16 19.0 -> 16.4 us)
    constexpr int LDS = gemm_lds<T, LAY, BM, BN>();
    static_assert(LDS == (LAY == L_KK ? A3 + (DEEP ? 3 : 2) * OpB::BYTES : 4 * STAGE), "slots");

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int tm, tn, sp;
    tile_of(wg, total, ga.tiles_m, ga.tiles_n, tm, tn, sp);
    const int m0 = tm * BM, n0 = tn * (GATED ? BN / 2 : BN);
    const int k0 = sp * ga.kper, k1 = min(ga.K, k0 + ga.kper);
    OpA oa;
    OpB ob;
    oa.init(ga.a, ga.lda, m0, ga.M, k0, k1, tid);
    ob.init(ga.b, ga.ldb, n0, ga.N, k0, k1, tid);
    const int steps = (k1 - k0 + BK - 1) / BK;
    const int wm = (wave / 2) * WM, wn = (wave % 2) * WN;

    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct { u32x4_t a[MI], b[NJ]; } f;
    auto multiply = [&] {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] = mma<T>(f.b[j], f.a[i], acc[i][j]);
    };
    constexpr std::integral_constant<int, 0> i0{};
    constexpr std::integral_constant<int, 1> i1{};
    constexpr std::integral_constant<int, 2> i2{};
    constexpr std::integral_constant<int, 3> i3{};
    const uint32_t at = (uint32_t)(uintptr_t)(const lds_char*)lds;

    if constexpr (LAY == L_KK) {
        typename OpA::template Place<MI> pa;
        typename OpB::template Place<NJ> pb;
        OpA::template place<MI>(pa, at, wm, lane);
        OpB::template place<NJ>(pb, at + A3, wn, lane);
        uint32_t sa = 0, sb = 0;  // slots of the current tiles, in bytes
        auto read = [&](auto half) {
            constexpr int H = decltype(half)::value;
            read_rows2<MI, NJ, 16 * TB, 0>(f.a, pa.a[H] + sa, f.b, pb.a[H] + sb);
            __builtin_amdgcn_sched_barrier(0);  // (the reads first, the loads behind them)
        };
        oa.fetch(lds, tid);
        ob.fetch(lds + A3, tid);
        oa.fetch(lds + OpA::BYTES, tid);
        if constexpr (DEEP) ob.fetch(lds + A3 + OpB::BYTES, tid);
        for (int s = 0; s < steps; ++s) {
            // tiles are started when all have read those whose places they take: two ahead, of B one ahead if it has two slots
            wait_loads<OpA::PASSES + (DEEP ? OpB::PASSES : 0)>();
            bare_barrier();
            read(i0);
            ob.fetch(lds + A3 + (!DEEP ? OpB::BYTES - sb : sb == 0 ? 2 * OpB::BYTES : sb - OpB::BYTES), tid);
            multiply();
            read(i1);
            oa.fetch(lds + (sa == 0 ? 2 * OpA::BYTES : sa - OpA::BYTES), tid);
            multiply();
            sa = sa == 2 * OpA::BYTES ? 0 : sa + OpA::BYTES;
            sb = !DEEP ? OpB::BYTES - sb : sb == 2 * OpB::BYTES ? 0 : sb + OpB::BYTES;
        }
    } else {
        // four slots, each with a tile of A and one of B; a lane's places in the first and in the third
        typename OpA::template Place<MI> pa[2];
        typename OpB::template Place<NJ> pb[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            OpA::template place<MI>(pa[h], at + h * 2 * STAGE, wm, lane);
            OpB::template place<NJ>(pb[h], at + h * 2 * STAGE + OpA::BYTES, wn, lane);
            keep(pa[h]);
            keep(pb[h]);
        }
        auto load = [&](int slot) {
            oa.fetch(lds + slot * STAGE, tid);
            ob.fetch(lds + slot * STAGE + OpA::BYTES, tid);
        };
        load(0);
        load(1);
        load(2);
        auto step = [&](auto slot) {
            constexpr int S = decltype(slot)::value, H = S / 2, OFF = S % 2 * STAGE;
            wait_loads<2 * (OpA::PASSES + OpB::PASSES)>();
            bare_barrier();
            OpB::template frags<NJ, OFF>(f.b, pb[H]);
            OpA::template frags<MI, OFF>(f.a, pa[H]);
            __builtin_amdgcn_sched_barrier(0);
            load((S + 3) % 4);
            multiply();
        };
        for (int s = 0; s < steps; s += 4) {  // (tiles past the last are zeros)
            step(i0);
            step(i1);
            step(i2);
            step(i3);
        }
    }
    wait_loads<0>();  // (tiles past the last may still be on their way)

    constexpr int FIT = LDS / WAVES / 256;                    // rows a wavefront has room for
    constexpr int RM = FIT >= WM ? WM : FIT >= 64 ? 64 : 32;  // rows at a time
    static_assert(RM <= FIT && WM % RM == 0, "room for the epilogue");
    __syncthreads();
#pragma unroll
    for (int h = 0; h < WM / RM; ++h)
        write_block<T, GATED, RM>(ga, &acc[h * (RM / 16)], 0, lds + wave * RM * 256, m0 + wm + h * RM, n0 + (GATED ? wn / 2 : wn), sp, lane);
}

// The same with 256 x 256 of C in half precision, 128 x 128 in fp32: four wavefronts, each with a quarter.  While a step's (64
// bytes of k) fragments are multiplied the next step's are read; a step's loads go to the slots that all have read.  One
// barrier a step (k along both rows: every two): it stands behind a wait for the tile that is read next, whose loads were
// started two to four steps before.
template <typename T, int LAY, bool GATED>
__device__ __forceinline__ void gemm_wide(const GemmArgs& ga, int wg, int total, char* const lds) {
    constexpr bool F32 = std::is_same<T, float>::value;
    constexpr int THREADS = 256, W = F32 ? 128 : 256, P = W / 2, MI = P / 16, NJ = MI;
    constexpr int D = F32 ? 1 : 2;  // loads a chunk
    // k along a row: tiles of 128 bytes of it (whole cache lines), two steps each; down a column: of 64
    constexpr bool CA = LAY == L_TT, CB = LAY != L_KK;
    constexpr int TA = CA ? 64 : 128, TBB = CB ? 64 : 128;
    using OpA = Operand<T, CA, W, TA, THREADS, false>;
    using OpB = Operand<T, CB, W, TBB, THREADS, GATED>;
    constexpr int SLOTS_A = CA ? 4 : 3, SLOTS_B = CB ? 4 : 2;
    constexpr int A0 = 0, B0 = SLOTS_A * OpA::BYTES;
    static_assert(B0 + SLOTS_B * OpB::BYTES <= wide_lds<T>(), "slots");
    static_assert((CA ? 2 : 4) * D == OpA::PASSES && (CB ? 2 : 4) * D == OpB::PASSES, "loads");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tm, tn, sp;
    tile_of(wg, total, ga.tiles_m, ga.tiles_n, tm, tn, sp);
    const int m0 = tm * W, n0 = tn * (GATED ? W / 2 : W);
    const int k0 = sp * ga.kper, k1 = min(ga.K, k0 + ga.kper);
    OpA oa;
    OpB ob;
    oa.init(ga.a, ga.lda, m0, ga.M, k0, k1, tid);
    ob.init(ga.b, ga.ldb, n0, ga.N, k0, k1, tid);
    const int wm = (wave >> 1) * P, wn = (wave & 1) * P;

    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct { u32x4_t a[MI], b[NJ]; } f[2];
    const uint32_t at = (uint32_t)(uintptr_t)(const lds_char*)lds, mine = at + (uint32_t)wave * 1024u;
    constexpr int SA = CA ? (F32 ? 1 : 4) * OpA::CPR * 16 : 16 * TA, SB = CB ? (F32 ? 1 : 4) * OpB::CPR * 16 : 16 * TBB;
    constexpr int R = MI / 2;  // blocks whose fragments a chunk reads; to the next ones: (columns: at addresses of their own)
    constexpr int RA = CA ? 0 : R * SA, RB = CB ? 0 : R * SB, NA = CA ? R : 0, NB = CB ? R : 0;
    typename OpA::template Place<MI> pa[CA ? 2 : 1];
    typename OpB::template Place<NJ> pb[CB ? 2 : 1];
#pragma unroll
    for (int h = 0; h < (CA ? 2 : 1); ++h) {
        OpA::template place<MI>(pa[h], at + A0 + h * 2 * OpA::BYTES, wm, lane);
        keep(pa[h]);
    }
#pragma unroll
    for (int h = 0; h < (CB ? 2 : 1); ++h) {
        OpB::template place<NJ>(pb[h], at + B0 + h * 2 * OpB::BYTES, wn, lane);
        keep(pb[h]);
    }
    // A step's products with c's fragments, while n's are read from ra and rb; l0 .. l3: where the four chunks' loads go, w0 .. w3:
    // which of their tile's they are
    auto multiply = [&](auto& c, auto& n, const uint32_t* ra, const uint32_t* rb, auto off_a, auto off_b, const auto& l0, const auto& l1,
                        const auto& l2, const auto& l3, auto w0, auto w1, auto w2, auto w3) {
        constexpr int OA = decltype(off_a)::value, OB = decltype(off_b)::value;
        if constexpr (F32) {
            chunk16_f32<CB, 0, OB, SB, decltype(w0)::value>(acc, c.a, c.b, n.b, rb, l0);
            chunk16_f32<CB, 1, OB + RB, SB, decltype(w1)::value>(acc, c.a, c.b, n.b + R, rb + NB, l1);
            chunk16_f32<CA, 2, OA, SA, decltype(w2)::value>(acc, c.a, c.b, n.a, ra, l2);
            chunk16_f32<CA, 3, OA + RA, SA, decltype(w3)::value>(acc, c.a, c.b, n.a + R, ra + NA, l3);
        } else {
            chunk16<T, CB, OB, SB, decltype(w0)::value>(acc[0], acc[1], c.a[0], c.a[1], c.b, n.b, rb, l0);
            chunk16<T, CB, OB + RB, SB, decltype(w1)::value>(acc[2], acc[3], c.a[2], c.a[3], c.b, n.b + R, rb + NB, l1);
            chunk16<T, CA, OA, SA, decltype(w2)::value>(acc[4], acc[5], c.a[4], c.a[5], c.b, n.a, ra, l2);
            chunk16<T, CA, OA + RA, SA, decltype(w3)::value>(acc[6], acc[7], c.a[6], c.a[7], c.b, n.a + R, ra + NA, l3);
        }
    };
    constexpr std::integral_constant<int, 0> i0{};
    constexpr std::integral_constant<int, 1> i1{};
    constexpr std::integral_constant<int, 2> i2{};
    constexpr std::integral_constant<int, 3> i3{};
    // a chunk's loads, D i to D i + D - 1 of the operand's current tile, to the slot at `slot` (fp32: one, of either source)
    auto to = [&](const auto& o, int i, uint32_t slot) {
        return LoadTo{o.voff[D * i], o.voff[D * i + D - 1], o.source(D == 1 ? i % 2 : 0), o.source(1), mine + slot};
    };

    if constexpr (LAY == L_KK) {
        const int tiles = (k1 - k0 + OpA::BK - 1) / OpA::BK;
        uint32_t sa = 0, sb = 0;  // slots of the current tiles, in bytes
        oa.fetch(lds, tid);
        ob.fetch(lds + B0, tid);
        oa.fetch(lds + OpA::BYTES, tid);
        ob.fetch(lds + B0 + OpB::BYTES, tid);
        wait_loads<OpA::PASSES + OpB::PASSES>();
        bare_barrier();
        read_rows<NJ, SB, 0>(f[0].b, pb[0].a[0]);
        read_rows<MI, SA, 0>(f[0].a, pa[0].a[0]);
        settle(acc);
        for (int s = 0; s < tiles; ++s) {
            // the tile's first half; A's tile after the next goes where the one before was
            const uint32_t slot_a = sa == 0 ? 2 * OpA::BYTES : sa - OpA::BYTES;
            uint32_t ra = pa[0].a[1] + sa, rb = pb[0].a[1] + sb;
            oa.mask();
            multiply(f[0], f[1], &ra, &rb, i0, i0, to(oa, 0, slot_a), to(oa, 1, slot_a), to(oa, 2, slot_a), to(oa, 3, slot_a), i0, i1, i2, i3);
            oa.advance();
            // the next tiles have come, and all have read this one: B's after the next takes its place
            wait_loads<OpA::PASSES>();
            bare_barrier();
            const uint32_t slot_b = B0 + sb;
            sa = sa == 2 * OpA::BYTES ? 0 : sa + OpA::BYTES;
            sb = OpB::BYTES - sb;
            ra = pa[0].a[0] + sa;
            rb = pb[0].a[0] + sb;
            ob.mask();
            multiply(f[1], f[0], &ra, &rb, i0, i0, to(ob, 0, slot_b), to(ob, 1, slot_b), to(ob, 2, slot_b), to(ob, 3, slot_b), i0, i1, i2, i3);
            ob.advance();
        }
    } else if constexpr (LAY == L_KT) {
        // a tile of A lasts two steps, half of its loads in each
        const int steps = (k1 - k0 + OpB::BK - 1) / OpB::BK;
        uint32_t sa = 0;
        oa.mask();
        oa.template load<0, 2 * D>(lds, tid);
        ob.fetch(lds + B0, tid);
        oa.template load<2 * D, 2 * D>(lds, tid);
        oa.advance();
        ob.fetch(lds + B0 + OpB::BYTES, tid);
        oa.mask();
        oa.template load<0, 2 * D>(lds + OpA::BYTES, tid);
        ob.fetch(lds + B0 + 2 * OpB::BYTES, tid);
        oa.template load<2 * D, 2 * D>(lds + OpA::BYTES, tid);
        oa.advance();
        ob.fetch(lds + B0 + 3 * OpB::BYTES, tid);
        wait_loads<10 * D>();
        bare_barrier();
        OpB::template frags<NJ, 0>(f[0].b, pb[0]);
        read_rows<MI, SA, 0>(f[0].a, pa[0].a[0]);
        settle(acc);
        auto step = [&](auto slot) {
            constexpr int S = decltype(slot)::value, X = (S + 1) % 4;
            constexpr std::integral_constant<int, X % 2 * OpB::BYTES> off{};
            constexpr uint32_t slot_b = B0 + S * OpB::BYTES;
            if constexpr (S % 2 == 0) {
                wait_loads<8 * D>();
                bare_barrier();
                const uint32_t slot_a = sa == 0 ? 2 * OpA::BYTES : sa - OpA::BYTES;
                const uint32_t ra = pa[0].a[1] + sa;
                oa.mask();
                ob.mask();
                multiply(f[0], f[1], &ra, pb[X / 2].a, i0, off, to(oa, 0, slot_a), to(oa, 1, slot_a), to(ob, 0, slot_b), to(ob, 1, slot_b), i0, i1, i0, i1);
            } else {
                wait_loads<6 * D>();
                bare_barrier();
                const uint32_t slot_a = sa == 0 ? 2 * OpA::BYTES : sa - OpA::BYTES;
                sa = sa == 2 * OpA::BYTES ? 0 : sa + OpA::BYTES;
                const uint32_t ra = pa[0].a[0] + sa;
                ob.mask();
                multiply(f[1], f[0], &ra, pb[X / 2].a, i0, off, to(oa, 2, slot_a), to(oa, 3, slot_a), to(ob, 0, slot_b), to(ob, 1, slot_b), i2, i3, i0, i1);
                oa.advance();
            }
            ob.advance();
        };
        for (int s = 0; s < steps; s += 4) {  // (tiles past the last are zeros)
            step(i0);
            step(i1);
            step(i2);
            step(i3);
        }
    } else {
        const int steps = (k1 - k0 + OpB::BK - 1) / OpB::BK;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            oa.fetch(lds + i * OpA::BYTES, tid);
            ob.fetch(lds + B0 + i * OpB::BYTES, tid);
        }
        constexpr int LOADS = OpA::PASSES + OpB::PASSES;
        wait_loads<3 * LOADS>();
        bare_barrier();
        OpB::template frags<NJ, 0>(f[0].b, pb[0]);
        OpA::template frags<MI, 0>(f[0].a, pa[0]);
        settle(acc);
        auto step = [&](auto slot) {
            constexpr int S = decltype(slot)::value, X = (S + 1) % 4;
            constexpr std::integral_constant<int, X % 2 * OpA::BYTES> off_a{};
            constexpr std::integral_constant<int, X % 2 * OpB::BYTES> off_b{};
            wait_loads<2 * LOADS>();
            bare_barrier();
            oa.mask();
            ob.mask();
            multiply(f[S % 2], f[1 - S % 2], pa[X / 2].a, pb[X / 2].a, off_a, off_b, to(oa, 0, S * OpA::BYTES), to(oa, 1, S * OpA::BYTES),
                     to(ob, 0, B0 + S * OpB::BYTES), to(ob, 1, B0 + S * OpB::BYTES), i0, i1, i0, i1);
            oa.advance();
            ob.advance();
        };
        for (int s = 0; s < steps; s += 4) {
            step(i0);
            step(i1);
            step(i2);
            step(i3);
        }
    }
    wait_loads<0>();  // (tiles past the last may still be on their way)
    settle(acc);
    __syncthreads();
    static_assert(4 * P * 256 <= wide_lds<T>(), "room for the epilogue");
#pragma unroll
    for (int h = 0; h < P / 64; ++h)
        write_block<T, GATED, P>(ga, acc, h * 4, lds + wave * P * 256, m0 + wm, n0 + (GATED ? wn / 2 + h * 32 : wn + h * 64), sp, lane);
}

// which of the tiles are gemm_wide's
template <typename T, int TILE>
constexpr bool kWide = TILE == (sizeof(T) == 2 ? 0 : 1);

template <typename T, int LAY, int BM, int BN, bool GATED>
__global__ __launch_bounds__(256, 2) void k_gemm(const GemmArgs ga) {
#if defined(__HIP_DEVICE_COMPILE__)  // (the host's pass has no use for the body, and does not know its assembly)
    __shared__ __attribute__((aligned(16))) char lds[gemm_lds<T, LAY, BM, BN>()];
    gemm_tile<T, LAY, BM, BN, GATED>(ga, blockIdx.x, gridDim.x, lds);
#endif
}

template <typename T, int LAY, bool GATED>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 1 : 2) void k_gemm_wide(const GemmArgs ga) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ __attribute__((aligned(16))) char lds[wide_lds<T>()];
    gemm_wide<T, LAY, GATED>(ga, blockIdx.x, gridDim.x, lds);
#endif
}

// kSumCols columns of the bias gradient from the row blocks' sums, added up in a fixed order by 256 threads with all loads in
// flight
constexpr int kSumCols = 16;

template <typename T>
__device__ __forceinline__ void sum_columns(const SumArgs& sa, int wg, float (*red)[17]) {
    const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
    const int c = wg * kSumCols + cx;
    float s = 0.f;
    if (c < sa.n) {
        const float* const p = sa.sums + c;
        for (int i = ry; i < sa.row_blocks; i += 256) {
            float v[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) v[u] = i + 16 * u < sa.row_blocks ? p[(int64_t)(i + 16 * u) * sa.sums_ld] : 0.f;
#pragma unroll
            for (int u = 0; u < 16; ++u) s += v[u];
        }
    }
    red[ry][cx] = s;
    __syncthreads();
    if (ry == 0 && c < sa.n) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) t += red[w][cx];
        static_cast<T*>(sa.out)[c] = (T)t;
    }
}

// Both products of a backward call in one launch, and the bias gradient if nothing comes behind: small products leave most
// compute units idle one by one, and of large ones the last round of tiles is shared.  dW's work-groups come first: they are
// the longer ones.  Each product's start at a multiple of 8, so that tile_of's XCDs are the real ones.  bf16, rows x in x
// out, the whole call against one launch after the other: 64 x 1024 x 1024 15.3 us for 20.1, 2048 x 512 x 2048 28 for 46,
// 8192 x 8192 x 1024 244 for 301; 16384 x 2048 x 2048 takes 205 us in this kernel, 1340 TFLOP/s.
template <typename T, int TILE>
__global__ __launch_bounds__(256, TILE == 0 ? 1 : 2) void k_back(const GemmArgs gx, const GemmArgs gw, const SumArgs sa, int nx, int nw) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int BM = kTileM[TILE], BN = kTileN[TILE];
    __shared__ __attribute__((aligned(16))) char lds[kWide<T, TILE> ? wide_lds<T>() : gemm_lds<T, L_TT, BM, BN>()];
    const int nw8 = (nw + 7) & ~7, nx8 = (nx + 7) & ~7;
    int b = blockIdx.x;
    if (b < nw8) {
        if (b >= nw) return;
        if constexpr (kWide<T, TILE>) gemm_wide<T, L_TT, false>(gw, b, nw, lds);
        else gemm_tile<T, L_TT, BM, BN, false>(gw, b, nw, lds);
        return;
    }
    b -= nw8;
    if (b < nx8) {
        if (b >= nx) return;
        if constexpr (kWide<T, TILE>) gemm_wide<T, L_KT, false>(gx, b, nx, lds);
        else gemm_tile<T, L_KT, BM, BN, false>(gx, b, nx, lds);
        return;
    }
    sum_columns<T>(sa, b - nx8, reinterpret_cast<float(*)[17]>(lds));
#endif
}


// The wavefronts' sums of 16 x 16 elements (gated: of both halves) added up in order, and the epilogue
constexpr int kSkinnyWaves = 8;

template <typename T, bool GATED>
__device__ __forceinline__ void skinny_end(const GemmArgs& ga, int m0, int n0, const float (*sums)[GATED ? 2 : 1][16][20], int tid) {
    const int row = tid >> 1, ch = tid & 1;
    if (tid >= 32 || m0 + row >= ga.M) return;
    float s[1][8], u[1][8];
#pragma unroll
    for (int v = 0; v < 8; ++v) {
        s[0][v] = 0.f;
        u[0][v] = 0.f;
#pragma unroll
        for (int w = 0; w < kSkinnyWaves; ++w) {
            s[0][v] += sums[w][0][row][ch * 8 + v];
            if constexpr (GATED) u[0][v] += sums[w][1][row][ch * 8 + v];
        }
    }
    epilogue8<T, GATED, 1, 1>(ga.e, full_offset(ga.e.offset, ga.e.d_offset), m0 + row, 1, n0 + ch * 8, s, u);
}

// Few rows (at most 32): the product is a pass over B.  A work-group takes 16 columns of C (gated: and the 16 of the other
// half); its wavefronts take 128 bytes of k in turn, each on its own, and their sums meet in LDS.
//
// A wavefront loads 8 rows of 128 bytes at a time, whole cache lines from neighbouring lanes, to its two slots in LDS and
// reads its fragments from there; with two slots two work-groups share a compute unit (more slots were slower).  Fragments
// loaded straight from memory take 16 bytes of 16 rows from neighbouring lanes: 16 rows of 8192 -> 1024 bf16 16.7 us that
// way, 7.7 us (2.2 TB/s) this way; 2048 -> 8192 12.4 and 10.4 us (3.2 TB/s), gated 2048 -> 4096 13.0 and 11.0 us.

// One operand of a wavefront: 16 rows, 128 bytes of k of each in a slot, chunk c of row r at place c ^ (r >> 1)
template <typename T>
struct SkinnyRows {
    static constexpr int EPC = 16 / sizeof(T), BK = 128 / sizeof(T);
    static constexpr uint32_t kOut = 0x7FFFFFF0u;
    static constexpr int BYTES = 2048, LOADS = 2;
    const char* base;  // of the first row and the wavefront's next 128 bytes
    uint32_t voff[2];
    int k[2];          // first k value of the lane's chunks
    __device__ __forceinline__ void init(const void* p, int64_t ld, int row, int rows, int k0, int lane) {
        base = static_cast<const char*>(p) + ((int64_t)row * ld + k0) * (int64_t)sizeof(T);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = (lane >> 3) + 8 * i, c = (lane & 7) ^ ((r >> 1) & 7);
            voff[i] = row + r < rows ? (uint32_t)r * (uint32_t)(ld * (int64_t)sizeof(T)) + (uint32_t)c * 16u : kOut;
            k[i] = c * EPC;
        }
    }
    __device__ __forceinline__ void fetch(char* lds, int k_left, int step) {
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, kOut, 0x00020000);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(lds + i * 1024), 16, k[i] < k_left ? voff[i] : kOut, 0, 0, 0);
        base += step;
    }
};

// MT: blocks of 16 rows of A
template <typename T, bool GATED, int MT>
__global__ __launch_bounds__(64 * kSkinnyWaves) void k_skinny(const GemmArgs ga) {
#if defined(__HIP_DEVICE_COMPILE__)
    using Rows = SkinnyRows<T>;
    constexpr int OB = GATED ? 2 : 1, OPS = OB + MT, SLOT = OPS * Rows::BYTES, SLOTS = 2, LOADS = OPS * Rows::LOADS;
    constexpr int BK = Rows::BK;
    __shared__ __attribute__((aligned(16))) char lds[kSkinnyWaves * SLOTS * SLOT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, j = lane & 15;
    const int n0 = blockIdx.x * 16, k0 = wave * BK;
    char* const mine = lds + wave * (SLOTS * SLOT);
    Rows op[OPS];  // B (gated: both halves), then A's blocks
#pragma unroll
    for (int i = 0; i < OPS; ++i) {
        if (i < OB) op[i].init(static_cast<const T*>(ga.b) + (int64_t)i * ga.N * ga.ldb, ga.ldb, n0, ga.N, k0, lane);
        else op[i].init(ga.a, ga.lda, (i - OB) * 16, ga.M, k0, lane);
    }
    f32x4 acc[OB][MT];
#pragma unroll
    for (int i = 0; i < OB; ++i)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[i][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    int ahead = ga.K - k0;  // k values from the next tile to fetch on
    auto fetch = [&](char* slot) {
#pragma unroll
        for (int i = 0; i < OPS; ++i) op[i].fetch(slot + i * Rows::BYTES, ahead, kSkinnyWaves * 128);
        ahead -= kSkinnyWaves * BK;
    };
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) fetch(mine + i * SLOT);
    const uint32_t at = (uint32_t)(uintptr_t)(const lds_char*)mine + (uint32_t)(j * 128);
    const uint32_t c0 = (uint32_t)((g ^ ((j >> 1) & 7)) << 4), c1 = c0 ^ 64u;  // the lane's chunk in each half
    int slot = 0;
    for (int k = k0; k < ga.K; k += kSkinnyWaves * BK) {
        wait_loads<(SLOTS - 1) * LOADS>();
        u32x4_t f[2 * OPS];
        const uint32_t s = at + (uint32_t)(slot * SLOT);
        read_halves<OPS, Rows::BYTES>(f, s + c0, s + c1);
        fetch(mine + slot * SLOT);
        slot ^= 1;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < OB; ++i)
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[i][m] = mma<T>(f[2 * i + h], f[2 * (OB + m) + h], acc[i][m]);
    }
    wait_loads<0>();
    __syncthreads();
    typedef float Sums[OB][16][20];
    Sums* const sums = reinterpret_cast<Sums*>(lds);  // [MT][wavefronts]
    static_assert(sizeof(Sums) * MT * kSkinnyWaves <= sizeof(lds), "room for the sums");
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < OB; ++i) *reinterpret_cast<f32x4*>(&sums[m * kSkinnyWaves + wave][i][j][g * 4]) = acc[i][m];
    __syncthreads();
    if (wave < MT) skinny_end<T, GATED>(ga, wave * 16, n0, sums + wave * kSkinnyWaves, lane);
#endif
}

// ... at most 16 rows, of operands that are off 16-byte boundaries: fragments straight from memory (8 rows of 2047 -> 2047 f16
// 13 us, no slower than to copy the weights first; 7 us on boundaries)
template <typename T, bool GATED>
__global__ __launch_bounds__(64 * kSkinnyWaves) void k_skinny_odd(const GemmArgs ga) {
    constexpr int EPC = 16 / sizeof(T), KS = 64 / sizeof(T), UN = 8;
    __shared__ __attribute__((aligned(16))) float sums[kSkinnyWaves][GATED ? 2 : 1][16][20];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, j = lane & 15;
    const int n0 = blockIdx.x * 16;
    const int64_t ldb = ga.ldb;
    const T* pa = static_cast<const T*>(ga.a) + (int64_t)min(j, ga.M - 1) * ga.lda + g * EPC;
    const T* pb = static_cast<const T*>(ga.b) + (int64_t)min(n0 + j, ga.N - 1) * ldb + g * EPC;
    const T* pu = pb + (int64_t)ga.N * ldb;
    const bool row_ok = j < ga.M;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f}, accu = {0.f, 0.f, 0.f, 0.f};
    auto chunk = [&](const T* p, int k) {  // elements k .. k + EPC - 1 of a row, 0 past its end
        return load_chunk<T>(reinterpret_cast<const char*>(p + k), ga.K - k - g * EPC);
    };
    for (int k = wave * KS * UN; k < ga.K; k += kSkinnyWaves * KS * UN) {
        u32x4_t fa[UN], fb[UN], fu[UN];
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            fb[i] = chunk(pb, k + i * KS);
            if constexpr (GATED) fu[i] = chunk(pu, k + i * KS);
            fa[i] = u32x4_t{0u, 0u, 0u, 0u};
            if (row_ok) fa[i] = chunk(pa, k + i * KS);
        }
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            acc = mma<T>(fb[i], fa[i], acc);
            if constexpr (GATED) accu = mma<T>(fu[i], fa[i], accu);
        }
    }
    *reinterpret_cast<f32x4*>(&sums[wave][0][j][g * 4]) = acc;
    if constexpr (GATED) *reinterpret_cast<f32x4*>(&sums[wave][1][j][g * 4]) = accu;
    __syncthreads();
    skinny_end<T, GATED>(ga, 0, n0, sums, tid);
}

// eight columns of a product whose k was cut: the partial sums added up in the order of the cuts, and the epilogue
template <typename T, bool GATED>
__device__ __forceinline__ void join_chunk(const JoinArgs& ja, int64_t idx) {
    const int chunks = (ja.e.n + 7) / 8;
    if (idx >= (int64_t)chunks * ja.M) return;
    const int m = (int)(idx / chunks), col = (int)(idx % chunks) * 8;
    float s[1][8] = {}, u[1][8] = {};
    const float* p = ja.part + (int64_t)m * ja.part_ld + col;
    const int64_t slab = (int64_t)ja.M * ja.part_ld;
    const int up = (ja.e.n + 7) & ~7;
#pragma unroll 4
    for (int i = 0; i < ja.split; ++i, p += slab) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(p + h * 4);
#pragma unroll
            for (int v = 0; v < 4; ++v) s[0][h * 4 + v] += q[v];
            if constexpr (GATED) {
                const f32x4 r = *reinterpret_cast<const f32x4*>(p + up + h * 4);
#pragma unroll
                for (int v = 0; v < 4; ++v) u[0][h * 4 + v] += r[v];
            }
        }
    }
    epilogue8<T, GATED, 1, 1>(ja.e, full_offset(ja.e.offset, ja.e.d_offset), m, 1, col, s, u);
}

// The last launch of a call: the bias gradient, then the partial sums of up to two products, which come from the caches for
// the most part (two cuts of 2048 x 2048: 8.7 us, 4.9 TB/s).  Always in the same order: no result depends on which
// work-group was first.
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_join(const JoinArgs ja, const JoinArgs jb, const SumArgs sa, int sum_wgs, int ja_wgs) {
    __shared__ float red[16][17];
    int b = blockIdx.x;
    if (b < sum_wgs) return sum_columns<T>(sa, b, red);
    b -= sum_wgs;
    if (b < ja_wgs) return join_chunk<T, GATED>(ja, (int64_t)b * 256 + threadIdx.x);
    if constexpr (!GATED) join_chunk<T, false>(jb, (int64_t)(b - ja_wgs) * 256 + threadIdx.x);
}

// Rows that do not start on 16-byte boundaries, or end inside a chunk, copied to rows that do, zeros behind their ends: the
// products load whole chunks straight to LDS.  (Products that took such rows through registers cost 1.6 times as much with
// k along the rows, 4 times with k down a column: 4096 x 2047 -> 2047 f16.)
template <typename T>
__device__ __forceinline__ void pack_rows(const PackArgs& pk, int64_t first, int64_t step) {
    constexpr int EPC = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t cpr = (uint32_t)(pk.cols[i] + EPC - 1) / EPC;
        const int64_t total = (int64_t)cpr * pk.rows[i];
        for (int64_t c = first; c < total; c += step) {
            // (a 64-bit division takes longer than the copy)
            const int64_t r = total < (int64_t(1) << 32) ? (int64_t)((uint32_t)c / cpr) : c / cpr;
            const int k = (int)(c - r * cpr) * EPC;
            const char* const p = static_cast<const char*>(pk.src[i]) + (r * pk.ld[i] + k) * (int64_t)sizeof(T);
            static_cast<u32x4_t*>(pk.dst[i])[c] = load_chunk<T>(p, pk.cols[i] - k);
        }
    }
}

// (16384 x 2047 and 2047 x 2047 in half precision 38 us, 4.0 TB/s)
template <typename T>
__global__ __launch_bounds__(256) void k_pack(const PackArgs pk) {
    pack_rows<T>(pk, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

// dz and the bias gradient's partial sums: a work-group takes 256 columns and rows_per_block rows, 32 lanes side by side
// with eight columns each, kDzRows rows at a time.  The work-groups behind those copy rows for the products (pack_rows).
// Bound by memory: 16384 x 2048 in bf16 with dropout 41 us (4.9 TB/s), gated 8192 x 4096 67 (5.0).  (128 row blocks for the
// first: 32, 16 and 8 rows at a time 59, 52 and 47 us.)
template <typename T, bool GATED>
__global__ __launch_bounds__(32 * kDzRows) void k_dz(const DzArgs da, const PackArgs pk) {
    __shared__ float red[kDzRows][256 + 8];
    if ((int)blockIdx.y >= da.row_blocks) {
        const int64_t wg = (int64_t)(blockIdx.y - da.row_blocks) * gridDim.x + blockIdx.x, wgs = (int64_t)(gridDim.y - da.row_blocks) * gridDim.x;
        pack_rows<T>(pk, wg * (32 * kDzRows) + threadIdx.x, wgs * (32 * kDzRows));
        return;
    }
    const int tid = threadIdx.x, cx = tid & 31, ry = tid >> 5;
    const int col = (blockIdx.x * 32 + cx) * 8;
    const int64_t r0 = (int64_t)blockIdx.y * da.rows_per_block, r1 = min(da.M, r0 + da.rows_per_block);
    const uint64_t offset = full_offset(da.offset, da.d_offset);
    const int cnt = da.n - col;
    // the other half's columns follow at once, as the weight's rows do: the products take [g | u] as one matrix
    const int last = GATED ? 2 * da.n : da.n;
    float sum[GATED ? 2 : 1][8] = {};
    if (cnt > 0) {
        for (int64_t r = r0 + ry; r < r1; r += kDzRows) {
            float d[8], z[8], u[8];
            load8(static_cast<const T*>(da.dy) + r * da.ld_dy + col, cnt, d);
            if (da.thr) {
                const uint32_t keep = keep_mask((uint32_t)col >> 3, (uint32_t)r, da.seed, offset, da.thr);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = (keep >> i) & 1u ? d[i] * da.scale : 0.0f;
            }
            if (da.pre) {
                const T* p = static_cast<const T*>(da.pre) + r * da.ld_pre + col;
                load8(p, cnt, z);
                if constexpr (GATED) load8(p + da.n, cnt, u);
                float slope[8];
                act_both<sizeof(T) == 2>(da.act, z, slope);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (GATED) {
                        const float dh = d[i];
                        d[i] = mul0(mul0(dh, u[i]), slope[i]);
                        u[i] = mul0(dh, z[i]);
                    } else {
                        d[i] = mul0(d[i], slope[i]);
                    }
                }
            }
            // columns past the last are 0: the products read whole chunks
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i >= cnt) { d[i] = 0.0f; if constexpr (GATED) u[i] = 0.0f; }
                sum[0][i] += d[i];
                if constexpr (GATED) sum[1][i] += u[i];
            }
            if (da.dz) {
                T* q = static_cast<T*>(da.dz) + r * da.ld_dz + col;
                if constexpr (GATED) {
                    store8(q, cnt, d);
                    store8(q + da.n, cnt, u);
                    if (cnt <= 8)
                        for (int i = cnt; i < cnt + (8 - last % 8) % 8; ++i) q[da.n + i] = (T)0.0f;
                } else {
                    store8(q, 8, d);
                }
            }
        }
    }
    if (da.sums) {
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) red[ry][cx * 8 + i] = sum[h][i];
            __syncthreads();
            const int c = blockIdx.x * 256 + tid;
            if (tid < 256 && c < da.n) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < kDzRows; ++w) s += red[w][tid];
                da.sums[(int64_t)blockIdx.y * da.sums_ld + (h ? da.n : 0) + c] = s;
            }
        }
    }
}

// y = drop(x) + residual, eight columns a thread: one Philox block each.  Bound by memory: 16384 x 8192 bf16 with a residual
// 134 us, 6.0 TB/s; 256 x 16 is all launch (1.9 us in the kernel).
template <typename T>
__global__ __launch_bounds__(256) void k_drop(const DropArgs da) {
    const int64_t chunks = ((int64_t)da.cols + 7) / 8, total = chunks * da.rows;
    const uint64_t offset = full_offset(da.offset, da.d_offset);
    for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (int64_t)gridDim.x * 256) {
        const int64_t row = idx / chunks;
        const int col = (int)(idx - row * chunks) * 8, cnt = da.cols - col;
        float s[8];
        load8(static_cast<const T*>(da.x) + row * da.ld_x + col, cnt, s);
        if (da.thr) {
            const uint32_t keep = keep_mask((uint32_t)(col >> 3), (uint32_t)row, da.seed, offset, da.thr);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = (keep >> i) & 1u ? s[i] * da.scale : 0.0f;
        }
        if (da.res) {
            float r[8];
            load8(static_cast<const T*>(da.res) + row * da.ld_res + col, cnt, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += r[i];
        }
        store8(static_cast<T*>(da.y) + row * da.ld_y + col, cnt, s);
    }
}

// ---- launches -----------------------------------------------------------------------------------
template <typename T, int LAY, bool GT>
static hipError_t gemm_pick(const GemmArgs& g, int tile, hipStream_t s) {
    const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * g.split)), block(256);
    if (tile == (sizeof(T) == 2 ? 0 : 1)) k_gemm_wide<T, LAY, GT><<<grid, block, 0, s>>>(g);
    else if (tile == 2) k_gemm<T, LAY, kTileM[2], kTileN[2], GT><<<grid, block, 0, s>>>(g);
    else if constexpr (sizeof(T) == 2) k_gemm<T, LAY, kTileM[1], kTileN[1], GT><<<grid, block, 0, s>>>(g);
    return hipGetLastError();
}

template <typename T>
hipError_t DenseOps<T>::gemm(const GemmArgs& g, Layout lay, bool gated, int tile, hipStream_t s) {
    if (gated) return gemm_pick<T, L_KK, true>(g, tile, s);
    if (lay == L_KK) return gemm_pick<T, L_KK, false>(g, tile, s);
    if (lay == L_KT) return gemm_pick<T, L_KT, false>(g, tile, s);
    return gemm_pick<T, L_TT, false>(g, tile, s);
}

template <typename T, bool GT>
static void skinny_go(const GemmArgs& g, bool aligned, hipStream_t s) {
    const dim3 grid((unsigned)((g.N + 15) / 16)), block(64 * kSkinnyWaves);
    if (!aligned) k_skinny_odd<T, GT><<<grid, block, 0, s>>>(g);
    else if (g.M <= 16) k_skinny<T, GT, 1><<<grid, block, 0, s>>>(g);
    else k_skinny<T, GT, 2><<<grid, block, 0, s>>>(g);
}

template <typename T>
hipError_t DenseOps<T>::skinny(const GemmArgs& g, bool gated, bool aligned, hipStream_t s) {
    if (gated) skinny_go<T, true>(g, aligned, s);
    else skinny_go<T, false>(g, aligned, s);
    return hipGetLastError();
}

template <typename T>
hipError_t DenseOps<T>::back(const GemmArgs& gx, const GemmArgs& gw, const SumArgs& a, int tile, hipStream_t s) {
    const int nx = gx.tiles_m * gx.tiles_n * gx.split, nw = gw.tiles_m * gw.tiles_n * gw.split;
    const dim3 grid((unsigned)(((nx + 7) & ~7) + ((nw + 7) & ~7) + (a.n + kSumCols - 1) / kSumCols));
    if (tile == 1) k_back<T, 1><<<grid, dim3(256), 0, s>>>(gx, gw, a, nx, nw);
    else if (tile == 2) k_back<T, 2><<<grid, dim3(256), 0, s>>>(gx, gw, a, nx, nw);
    else if constexpr (sizeof(T) == 2) k_back<T, 0><<<grid, dim3(256), 0, s>>>(gx, gw, a, nx, nw);
    return hipGetLastError();
}

template <typename T>
hipError_t DenseOps<T>::join(const JoinArgs& ja, const JoinArgs& jb, const SumArgs& a, hipStream_t s) {
    const auto wgs = [](const JoinArgs& j) { return ((int64_t)((j.e.n + 7) / 8) * j.M + 255) / 256; };
    const int sum_wgs = (a.n + kSumCols - 1) / kSumCols;
    const dim3 grid((unsigned)(sum_wgs + wgs(ja) + wgs(jb)));
    if (ja.gated) k_join<T, true><<<grid, dim3(256), 0, s>>>(ja, jb, a, sum_wgs, (int)wgs(ja));
    else k_join<T, false><<<grid, dim3(256), 0, s>>>(ja, jb, a, sum_wgs, (int)wgs(ja));
    return hipGetLastError();
}

// work-groups of `threads` for the chunks to copy, at most `most`
template <typename T>
static int pack_wgs(const PackArgs& pk, int threads, int most) {
    constexpr int EPC = 16 / sizeof(T);
    int64_t n = 0;
    for (int i = 0; i < 2; ++i) n += (pk.cols[i] + EPC - 1) / EPC * pk.rows[i];
    const int64_t w = (n + threads - 1) / threads;
    return (int)(w < most ? w : most);
}

template <typename T>
hipError_t DenseOps<T>::pack(const PackArgs& pk, hipStream_t s) {
    const int wgs = pack_wgs<T>(pk, 256, 4096);
    if (wgs == 0) return hipSuccess;
    k_pack<T><<<dim3((unsigned)wgs), dim3(256), 0, s>>>(pk);
    return hipGetLastError();
}

template <typename T>
hipError_t DenseOps<T>::dz(const DzArgs& d, const PackArgs& pk, hipStream_t s) {
    const unsigned cols = (unsigned)((d.n + 255) / 256);
    const unsigned more = ((unsigned)pack_wgs<T>(pk, 32 * kDzRows, 1024) + cols - 1) / cols;
    const dim3 grid(cols, (unsigned)d.row_blocks + more);
    if (d.gated) k_dz<T, true><<<grid, dim3(32 * kDzRows), 0, s>>>(d, pk);
    else k_dz<T, false><<<grid, dim3(32 * kDzRows), 0, s>>>(d, pk);
    return hipGetLastError();
}

template <typename T>
hipError_t DenseOps<T>::drop(const DropArgs& d, hipStream_t s) {
    const int64_t n = (((int64_t)d.cols + 7) / 8) * d.rows;
    const int64_t want = (n + 255) / 256;
    k_drop<T><<<dim3((unsigned)(want < (1 << 20) ? want : (1 << 20))), dim3(256), 0, s>>>(d);
    return hipGetLastError();
}

}  // namespace dlc
