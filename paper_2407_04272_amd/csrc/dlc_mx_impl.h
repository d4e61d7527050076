// The product of microscaled operands on the matrix cores, one template for three types of the result.
//
// C[m][n] = sum over k of x(m, k) w(n, k), in steps of 128 k values: one instruction multiplies 16 x 128 by 128 x 16 elements
// and applies the scales of both, which every lane gives for the 32 k values that it stands for.
#pragma once
#include "dlc_gemm_impl.h"
#include "dlc_mx_gemm.h"

namespace dlc {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// How the products are made:
//   ELEM 4, E2M1 times E2M1: the scaled instruction, exact products (whole numbers of quarters up to 36), fp32 sums.
//   ELEM 8, E4M3 times E2M1, results of half precision: the scaled instruction.  It lines up the eight products of a lane's
//     consecutive elements at 2^E, E the largest sum of two factors' exponents (0.5 has that of 1; products of 0 do not count), and
//     drops what lies more than 13 binary places below (towards zero); their sums are fp32.  That is below 7 2^-13 of the
//     largest's magnitude (2^-12 if its weight is 0.5), in the norm some 2^-14 of a result, against its own rounding of 2^-11 or
//     2^-8, and taken where the matrix cores set the time.  Up to 16 rows, where memory does, mx_mma_split keeps all.
//   ELEM 8, results in fp32 (EXACT): elements times scales as bf16, which holds all from 2^-126 on exactly, and the bf16
//     instruction, whose sums are fp32 throughout.  2048 x 8192 -> 8192 292-305 us, 940 TFLOP/s, bound by the conversions,
//     which every wavefront makes for itself (the scaled instruction 91 us).  Their order does not matter: all of a quarter
//     in front of its products 310, between those of the quarter before 330.
template <typename T, int ELEM>
constexpr bool kMxExact = ELEM == 8 && std::is_same<T, float>::value;

// One 16 x 16 block times 128 k values.  w: rows, E2M1, lane l row l % 16, k values (l / 16) * 32 on (16 bytes).  x: columns,
// lane l column l % 16; E2M1 the same, E4M3 two chunks of 16 bytes: EXACT k values (l / 16) * 32 on, otherwise (l / 16) * 16
// on and 64 further.  A lane's scales are those of the 32 k values from (l / 16) * 32 on: byte S of sw and sx.
template <int ELEM, bool EXACT, int S>
__device__ __forceinline__ f32x4 mx_mma(const u32x4_t& w, const u32x4_t& x0, const u32x4_t& x1, uint32_t sw, uint32_t sx, f32x4 acc) {
    if constexpr (EXACT) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const float fw = mx_scale((sw >> (8 * S)) & 255u), fx = mx_scale((sx >> (8 * S)) & 255u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // 8 of the lane's k values each
            bf16x8 a, b;
            const uint32_t lo = i < 2 ? x0[2 * i] : x1[2 * i - 4], hi = i < 2 ? x0[2 * i + 1] : x1[2 * i - 3];
            const bf16x2 p[8] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], fw, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], fw, 1),
                                 __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], fw, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], fw, 3),
                                 __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, fx, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, fx, true),
                                 __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, fx, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, fx, true)};
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                a[v] = p[v >> 1][v & 1];
                b[v] = p[4 + (v >> 1)][v & 1];
            }
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
        }
        return acc;
    }
    const i32x8 wv = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    i32x8 xv = {(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], 0, 0, 0, 0};
    if constexpr (ELEM == 8) xv = i32x8{(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, acc, 4, ELEM == 8 ? 0 : 4, S, (int)sw, S, (int)sx);
}

// ... E4M3 times E2M1 by the scaled instruction with nothing cut off: x's elements from 2 on, whose codes have bit 6, then the
// others.  From 2 on the largest sum of exponents is 8 + 2 and a product's last place 2^-3; below 2, 0 + 2 and 2^-10.
template <int S>
__device__ __forceinline__ f32x4 mx_mma_split(const u32x4_t& w, const u32x4_t& x0, const u32x4_t& x1, uint32_t sw, uint32_t sx, f32x4 acc) {
    u32x4_t big[2], rest[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t x = i < 4 ? x0[i] : x1[i - 4];
        const uint32_t mask = __builtin_amdgcn_perm(x << 9, x << 1, 0x090B080Au);  // bit 6 in all of its byte
        big[i >> 2][i & 3] = x & mask;
        rest[i >> 2][i & 3] = x & ~mask;
    }
    acc = mx_mma<8, false, S>(w, big[0], big[1], sw, sx, acc);
    return mx_mma<8, false, S>(w, rest[0], rest[1], sw, sx, acc);
}

// The loads before it are asked for before those behind it: waits that leave some on their way count on the order
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }

// Both chunks of N blocks' rows, STEP bytes apart
template <int N, int STEP = 2048>
__device__ __forceinline__ void read_frags(u32x4_t* o, uint32_t a, uint32_t b) {
    if constexpr (N == 1) {
        asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)" : "=&v"(o[0]), "=&v"(o[1]) : "v"(a), "v"(b) : "memory");
    } else {
        read_halves<N, STEP>(o, a, b);
    }
}

// ---- few rows ----
// The product is a pass over w for a band of 32 rows (16, if there are no more).  A work-group takes 16 columns of C; its
// wavefronts take groups of 512 k values in turn, each on its own, and their sums meet in LDS.  A wavefront loads 8 rows of 128 bytes at a time, whole cache
// lines, to its two slots in LDS and reads its fragments from there.  Bound by the latency of memory, one call after the other in
// a graph: 1 x 1664 -> 1024 3.5 us (0.9 MB, fp16), 16 x 8192 -> 2048 5.9 us (8.9 MB: 1.5 TB/s with 128 work-groups), of which an
// empty launch is 2; with E4M3 products that are cut 3.2 and 5.4.  MT: blocks of 16 rows of x
template <typename T, int ELEM, int MT>
__global__ __launch_bounds__(64 * kSkinnyWaves) void k_mx_skinny(const MxGemmArgs mx) {
#if defined(__HIP_DEVICE_COMPILE__)
    using Rows = SkinnyRows<uint8_t>;
    constexpr bool EXACT = kMxExact<T, ELEM>;
    constexpr int XT = ELEM / 4, OPS = 1 + XT * MT;  // 128-byte tiles of x for one of w; 256 k values of both
    constexpr int SLOT = OPS * Rows::BYTES, SLOTS = 2, LOADS = OPS * Rows::LOADS;
    constexpr int WSTEP = kSkinnyWaves * 256, XSTEP = WSTEP * XT;  // bytes to the wavefront's next group
    __shared__ __attribute__((aligned(16))) char lds[kSkinnyWaves * SLOTS * SLOT];
    const GemmArgs& ga = mx.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, j = lane & 15;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * kMxSkinnyRows, k0 = wave * kMxGroup;
    char* const mine = lds + wave * (SLOTS * SLOT);
    Rows w, x[XT * MT];  // (x: [block][tile])
    w.init(ga.b, ga.ldb, n0, ga.N, k0 / 2, lane);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < XT; ++t) x[m * XT + t].init(ga.a, ga.lda, m0 + m * 16, ga.M, k0 * ELEM / 8 + t * 128, lane);
    int left = ga.K - k0;  // k values from the next tile to fetch on
    const auto fetch = [&](char* slot, bool second) {  // a group's first 256 values, its second
        w.fetch(slot, left / 2, second ? WSTEP - 128 : 128);
#pragma unroll
        for (int i = 0; i < XT * MT; ++i) x[i].fetch(slot + (1 + i) * Rows::BYTES, left * ELEM / 8 - (i % XT) * 128, second ? XSTEP - 128 * XT : 128 * XT);
        left -= second ? kSkinnyWaves * kMxGroup - 256 : 256;
    };
    // a lane's scales of a group, whose rows past the last are the last's
    const uint8_t* qw = mx.ws + (int64_t)min(n0 + j, ga.N - 1) * 16 + g * 4 + (int64_t)wave * ga.N * 16;
    const uint8_t* qx[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) qx[m] = mx.xs + (int64_t)min(m0 + m * 16 + j, ga.M - 1) * 16 + g * 4 + (int64_t)wave * ga.M * 16;
    uint32_t sw = 0, sx[MT] = {};
    const auto scales = [&](int k) {
        if (k >= ga.K) return;
        sw = *reinterpret_cast<const uint32_t*>(qw);
        qw += (int64_t)kSkinnyWaves * ga.N * 16;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            sx[m] = *reinterpret_cast<const uint32_t*>(qx[m]);
            qx[m] += (int64_t)kSkinnyWaves * ga.M * 16;
        }
    };
    f32x4 acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
    scales(k0);
    fetch(mine, false);
    fetch(mine + SLOT, true);
    const uint32_t at = (uint32_t)(uintptr_t)(const lds_char*)mine + (uint32_t)(j * 128);
    const int key = (j >> 1) & 7;
    const uint32_t c0 = (uint32_t)((g ^ key) << 4), c1 = c0 ^ 64u;  // the lane's chunk in each half of 128 bytes
    // ... of x: where products are exact two that stand side by side
    const uint32_t d0 = EXACT ? (uint32_t)(((2 * g) ^ key) << 4) : c0, d1 = EXACT ? (uint32_t)(((2 * g + 1) ^ key) << 4) : c1;
    for (int k = k0; k < ga.K; k += kSkinnyWaves * kMxGroup) {
        const uint32_t tw = sw;
        uint32_t tx[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) tx[m] = sx[m];
        const auto half = [&](auto which) {
            constexpr int H = decltype(which)::value;
            wait_loads<(SLOTS - 1) * LOADS>();
            u32x4_t fw[2], fx[2 * XT * MT];
            const uint32_t s = at + (uint32_t)(H * SLOT);
            read_frags<1>(fw, s + c0, s + c1);
            read_frags<XT * MT>(fx, s + Rows::BYTES + d0, s + Rows::BYTES + d1);
            fetch(mine + H * SLOT, H == 1);
            if constexpr (H == 0) scales(k + kSkinnyWaves * kMxGroup);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if constexpr (ELEM == 4) {
                    acc[m] = mx_mma<4, false, 2 * H>(fw[0], fx[2 * m], fx[2 * m], tw, tx[m], acc[m]);
                    acc[m] = mx_mma<4, false, 2 * H + 1>(fw[1], fx[2 * m + 1], fx[2 * m + 1], tw, tx[m], acc[m]);
                } else if constexpr (MT == 1 && !EXACT) {
                    acc[m] = mx_mma_split<2 * H>(fw[0], fx[0], fx[1], tw, tx[m], acc[m]);
                    acc[m] = mx_mma_split<2 * H + 1>(fw[1], fx[2], fx[3], tw, tx[m], acc[m]);
                } else {
                    acc[m] = mx_mma<8, EXACT, 2 * H>(fw[0], fx[4 * m], fx[4 * m + 1], tw, tx[m], acc[m]);
                    acc[m] = mx_mma<8, EXACT, 2 * H + 1>(fw[1], fx[4 * m + 2], fx[4 * m + 3], tw, tx[m], acc[m]);
                }
            }
        };
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, 1>{});
    }
    wait_loads<0>();
    __syncthreads();
    typedef float Sums[1][16][20];
    Sums* const sums = reinterpret_cast<Sums*>(lds);  // [MT][wavefronts]
    static_assert(sizeof(Sums) * MT * kSkinnyWaves <= sizeof(lds), "room for the sums");
#pragma unroll
    for (int m = 0; m < MT; ++m) *reinterpret_cast<f32x4*>(&sums[m * kSkinnyWaves + wave][0][j][g * 4]) = acc[m];
    __syncthreads();
    if (wave < MT) skinny_end<T, false>(ga, m0 + wave * 16, n0, sums + wave * kSkinnyWaves, lane);
#endif
}

// ---- tiles of 128 x 128 and 64 x 128 ----
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
#define DLC_MX(OP, BL, ACC, B, A, SB, SA) "v_mfma_scale_f32_16x16x128_f8f6f4 %" #ACC ", %" #B ", %" #A ", %" #ACC ", %" #SB ", %" #SA " " OP " cbsz:4 blgp:" BL "\n\t"
#define DLC_MX_BYTE0 "op_sel_hi:[0,0,0]"
#define DLC_MX_BYTE1 "op_sel:[1,1,0] op_sel_hi:[0,0,0]"
#define DLC_MX_BYTE2 "op_sel_hi:[1,1,0]"
#define DLC_MX_BYTE3 "op_sel:[1,1,0] op_sel_hi:[1,1,0]"
#define DLC_MX_PAIR4(OP, BL) \
    asm volatile("s_nop 1\n\t" \
    DLC_MX(OP, BL, 4, 14, 12, 20, 18) "ds_read_b128 %0, %24 offset:%28\n\t" DLC_MX(OP, BL, 5, 15, 12, 21, 18) "ds_read_b128 %1, %25 offset:%29\n\t" \
    DLC_MX(OP, BL, 6, 16, 12, 22, 18) "ds_read_b128 %2, %26 offset:%30\n\t" DLC_MX(OP, BL, 7, 17, 12, 23, 18) "ds_read_b128 %3, %27 offset:%31\n\t" \
    DLC_MX(OP, BL, 8, 14, 13, 20, 19) DLC_MX(OP, BL, 9, 15, 13, 21, 19) \
    DLC_MX(OP, BL, 10, 16, 13, 22, 19) DLC_MX(OP, BL, 11, 17, 13, 23, 19) \
    "s_waitcnt lgkmcnt(0)" \
    : "=&v"(next[0]), "=&v"(next[1]), "=&v"(next[2]), "=&v"(next[3]), \
      "+a"(acc0[0]), "+a"(acc0[1]), "+a"(acc0[2]), "+a"(acc0[3]), "+a"(acc1[0]), "+a"(acc1[1]), "+a"(acc1[2]), "+a"(acc1[3]) \
    : "v"(a0), "v"(a1), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(sa0), "v"(sa1), "v"(sb[0]), "v"(sb[1]), "v"(sb[2]), "v"(sb[3]), \
      "v"(from[Next::source(0)]), "v"(from[Next::source(1)]), "v"(from[Next::source(2)]), "v"(from[Next::source(3)]), \
      "i"(Next::offset(0)), "i"(Next::offset(1)), "i"(Next::offset(2)), "i"(Next::offset(3)) \
    : "memory")
#define DLC_MX_PAIR6(OP, BL) \
    asm volatile("s_nop 1\n\t" \
    DLC_MX(OP, BL, 6, 16, 14, 22, 20) "ds_read_b128 %0, %26 offset:%32\n\t" DLC_MX(OP, BL, 7, 17, 14, 23, 20) "ds_read_b128 %1, %27 offset:%33\n\t" \
    DLC_MX(OP, BL, 8, 18, 14, 24, 20) "ds_read_b128 %2, %28 offset:%34\n\t" DLC_MX(OP, BL, 9, 19, 14, 25, 20) "ds_read_b128 %3, %29 offset:%35\n\t" \
    DLC_MX(OP, BL, 10, 16, 15, 22, 21) "ds_read_b128 %4, %30 offset:%36\n\t" DLC_MX(OP, BL, 11, 17, 15, 23, 21) "ds_read_b128 %5, %31 offset:%37\n\t" \
    DLC_MX(OP, BL, 12, 18, 15, 24, 21) DLC_MX(OP, BL, 13, 19, 15, 25, 21) \
    "s_waitcnt lgkmcnt(0)" \
    : "=&v"(next[0]), "=&v"(next[1]), "=&v"(next[2]), "=&v"(next[3]), "=&v"(next[4]), "=&v"(next[5]), \
      "+a"(acc0[0]), "+a"(acc0[1]), "+a"(acc0[2]), "+a"(acc0[3]), "+a"(acc1[0]), "+a"(acc1[1]), "+a"(acc1[2]), "+a"(acc1[3]) \
    : "v"(a0), "v"(a1), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(sa0), "v"(sa1), "v"(sb[0]), "v"(sb[1]), "v"(sb[2]), "v"(sb[3]), \
      "v"(from[Next::source(0)]), "v"(from[Next::source(1)]), "v"(from[Next::source(2)]), "v"(from[Next::source(3)]), "v"(from[Next::source(4)]), "v"(from[Next::source(5)]), \
      "i"(Next::offset(0)), "i"(Next::offset(1)), "i"(Next::offset(2)), "i"(Next::offset(3)), "i"(Next::offset(4)), "i"(Next::offset(5)) \
    : "memory")
#define DLC_MX_PAIR8(OP, BL) \
    asm volatile("s_nop 1\n\t" \
    DLC_MX(OP, BL, 8, 18, 16, 24, 22) "ds_read_b128 %0, %28 offset:%36\n\t" DLC_MX(OP, BL, 9, 19, 16, 25, 22) "ds_read_b128 %1, %29 offset:%37\n\t" \
    DLC_MX(OP, BL, 10, 20, 16, 26, 22) "ds_read_b128 %2, %30 offset:%38\n\t" DLC_MX(OP, BL, 11, 21, 16, 27, 22) "ds_read_b128 %3, %31 offset:%39\n\t" \
    DLC_MX(OP, BL, 12, 18, 17, 24, 23) "ds_read_b128 %4, %32 offset:%40\n\t" DLC_MX(OP, BL, 13, 19, 17, 25, 23) "ds_read_b128 %5, %33 offset:%41\n\t" \
    DLC_MX(OP, BL, 14, 20, 17, 26, 23) "ds_read_b128 %6, %34 offset:%42\n\t" DLC_MX(OP, BL, 15, 21, 17, 27, 23) "ds_read_b128 %7, %35 offset:%43\n\t" \
    "s_waitcnt lgkmcnt(0)" \
    : "=&v"(next[0]), "=&v"(next[1]), "=&v"(next[2]), "=&v"(next[3]), "=&v"(next[4]), "=&v"(next[5]), "=&v"(next[6]), "=&v"(next[7]), \
      "+a"(acc0[0]), "+a"(acc0[1]), "+a"(acc0[2]), "+a"(acc0[3]), "+a"(acc1[0]), "+a"(acc1[1]), "+a"(acc1[2]), "+a"(acc1[3]) \
    : "v"(a0), "v"(a1), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(sa0), "v"(sa1), "v"(sb[0]), "v"(sb[1]), "v"(sb[2]), "v"(sb[3]), \
      "v"(from[Next::source(0)]), "v"(from[Next::source(1)]), "v"(from[Next::source(2)]), "v"(from[Next::source(3)]), "v"(from[Next::source(4)]), "v"(from[Next::source(5)]), "v"(from[Next::source(6)]), "v"(from[Next::source(7)]), \
      "i"(Next::offset(0)), "i"(Next::offset(1)), "i"(Next::offset(2)), "i"(Next::offset(3)), "i"(Next::offset(4)), "i"(Next::offset(5)), "i"(Next::offset(6)), "i"(Next::offset(7)) \
    : "memory")

// A step's fragments, in the order of their reads: four of w, those of x (E4M3: two of each block).  FIRST: of some of them
template <int ELEM, int FIRST, int STEP>
struct MxNext {
    static constexpr int place(int i) { return FIRST + i - 4; }                                                    // among x's
    static constexpr int source(int i) { return place(i) < 0 ? 0 : ELEM == 4 ? 1 : 1 + place(i) % 2; }             // of {w, x, x's second chunk}
    static constexpr int offset(int i) { return place(i) < 0 ? (FIRST + i) * STEP : place(i) * 4 / ELEM * STEP; }  // blocks STEP bytes apart
};

// Rows of blocks acc0 and acc1 += a0 and a1 times b, with byte S of the scales, while R fragments are read
template <int ELEM, int S, int R, typename Next, typename A>
__device__ __forceinline__ void mx_pair(f32x4* acc0, f32x4* acc1, const A& a0, const A& a1, const u32x4_t* b, uint32_t sa0, uint32_t sa1,
                                        const uint32_t* sb, u32x4_t* next, const uint32_t (&from)[3]) {
#define DLC_MX_PAIR(OP) \
    if constexpr (R == 4) DLC_MX_PAIR4(OP, "4"); \
    else if constexpr (R == 6 && ELEM == 4) DLC_MX_PAIR6(OP, "4"); \
    else if constexpr (R == 6) DLC_MX_PAIR6(OP, "0"); \
    else DLC_MX_PAIR8(OP, "0")
    static_assert(R == 4 ? ELEM == 4 : R == 6 || (R == 8 && ELEM == 8), "reads of a pair");
    if constexpr (S == 0) { DLC_MX_PAIR(DLC_MX_BYTE0); }
    else if constexpr (S == 1) { DLC_MX_PAIR(DLC_MX_BYTE1); }
    else if constexpr (S == 2) { DLC_MX_PAIR(DLC_MX_BYTE2); }
    else { DLC_MX_PAIR(DLC_MX_BYTE3); }
#undef DLC_MX_PAIR
}
#undef DLC_MX_PAIR4
#undef DLC_MX_PAIR6
#undef DLC_MX_PAIR8

// Four wavefronts, each with a quarter; tiles of 256 k values in three slots.  While a step (half a tile) is multiplied, the
// next one's fragments are read from LDS, between the products of one block of assembly; between a tile's two steps stands
// the only barrier, behind which the third tile from there is on its way to this one's place.  Where products are exact the
// compiler has the inner loop, and reading and multiplying take turns.
// For results that 256 x 256 tiles would leave most of the card without: 512 x 8192 -> 2048 of 4 bits 17 us (23 with reads and
// products in turn), 1024 x 8192 18 (27), 2048 x 8192 25 (36); 777 x 515 -> 1023, E4M3 rows, bias, gelu and residual 8.5 us.
// Where the tiles fill the card, bound by the way from L2 to LDS (128 x 128: 32 KB a tile on every unit in 0.64 us, 13 TB/s); where
// they do not, by what one unit gets (512 x 8192 -> 2048: 128 work-groups, 24 KB a tile in 0.39-0.44 us, 7-8 TB/s together; a cut
// of k that gives the others work costs a second launch and the sums' way, 4 us and more); at small sizes by the start and
// the epilogue, 4.4 us.  More slots were no faster.  Two work-groups of 64 x 128 and 4 bits fit a compute unit.  A group's
// scales are asked for two tiles ahead: one tile ahead they cost a fifth (2048 x 8192 33 us for 28), now a tenth.
template <int ELEM, int BM>
constexpr int mx_tile_lds() {
    const int ring = 3 * (BM * 32 * ELEM + 128 * 128), out = BM / 2 * 256 * 4;
    return ring > out ? ring : out;
}

template <typename T, int ELEM, int BM>
__global__ __launch_bounds__(256) void k_mx_tile(const MxGemmArgs mx) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool EXACT = kMxExact<T, ELEM>;
    constexpr int BN = 128, WM = BM / 2, WN = 64, MI = WM / 16, NJ = WN / 16, XT = ELEM / 4, STEP = 16 * 128;
    using OpA = Operand<uint8_t, false, BM, 128, 256, false>;
    using OpB = Operand<uint8_t, false, BN, 128, 256, false>;
    constexpr int SLOT = XT * OpA::BYTES + OpB::BYTES, LOADS = XT * OpA::PASSES + OpB::PASSES;
    __shared__ __attribute__((aligned(16))) char lds[mx_tile_lds<ELEM, BM>()];
    const GemmArgs& ga = mx.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, j = lane & 15;
    int tm, tn, sp;
    tile_of(blockIdx.x, gridDim.x, ga.tiles_m, ga.tiles_n, tm, tn, sp);
    const int m0 = tm * BM, n0 = tn * BN, k0 = sp * ga.kper, k1 = min(ga.K, k0 + ga.kper);
    const int wm = (wave >> 1) * WM, wn = (wave & 1) * WN;
    OpA oa;
    OpB ob;
    oa.init(ga.a, ga.lda, m0, ga.M, k0 * ELEM / 8, k1 * ELEM / 8, tid);
    ob.init(ga.b, ga.ldb, n0, ga.N, k0 / 2, k1 / 2, tid);
    const auto fetch = [&](int slot) {
        char* const to = lds + slot * SLOT;
#pragma unroll
        for (int t = 0; t < XT; ++t) oa.fetch(to + t * OpA::BYTES, tid);
        ob.fetch(to + XT * OpA::BYTES, tid);
    };
    // a lane's scales of a group, whose rows past the last are the last's
    uint32_t px[MI], pw[NJ];
    struct { uint32_t x[MI], w[NJ]; } sc[2];
#pragma unroll
    for (int i = 0; i < MI; ++i) px[i] = (uint32_t)(min(m0 + wm + i * 16 + j, ga.M - 1) - m0) * 16 + g * 4;
#pragma unroll
    for (int n = 0; n < NJ; ++n) pw[n] = (uint32_t)(min(n0 + wn + n * 16 + j, ga.N - 1) - n0) * 16 + g * 4;
    const uint8_t* bx = mx.xs + ((int64_t)(k0 / kMxGroup) * ga.M + m0) * 16;
    const uint8_t* bw = mx.ws + ((int64_t)(k0 / kMxGroup) * ga.N + n0) * 16;
    const auto scales = [&](auto& to, int k) {  // of the group at k, or the last once more: always as many loads
        if (k > k0 && k < k1) {
            bx += (int64_t)ga.M * 16;
            bw += (int64_t)ga.N * 16;
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) to.x[i] = *reinterpret_cast<const uint32_t*>(bx + px[i]);
#pragma unroll
        for (int n = 0; n < NJ; ++n) to.w[n] = *reinterpret_cast<const uint32_t*>(bw + pw[n]);
    };
    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int n = 0; n < NJ; ++n) acc[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    const uint32_t at = (uint32_t)(uintptr_t)(const lds_char*)lds;
    const int key = (j >> 1) & 7;
    const uint32_t c0 = (uint32_t)((g ^ key) << 4), c1 = c0 ^ 64u;
    const uint32_t d0 = EXACT ? (uint32_t)(((2 * g) ^ key) << 4) : c0, d1 = EXACT ? (uint32_t)(((2 * g + 1) ^ key) << 4) : c1;
    const uint32_t ra = at + (uint32_t)((wm + j) * 128), rb = at + (uint32_t)(XT * OpA::BYTES + (wn + j) * 128);
    if constexpr (!EXACT) {
        struct { u32x4_t f[NJ + XT * MI]; } f[2];
        constexpr int WORDS = MI + NJ;  // loads of scales
        const int tiles = (k1 - k0 + 255) / 256;
        scales(sc[0], k0);
        fetch(0);
        fetch(1);
        fetch(2);
        in_order();
        scales(sc[1], k0 + kMxGroup);
        wait_loads<2 * LOADS + WORDS>();
        bare_barrier();
        read_rows<NJ, STEP, 0>(f[0].f, rb + c0);
        if constexpr (ELEM == 4) read_rows<MI, STEP, 0>(f[0].f + NJ, ra + c0);
        else read_halves<MI, STEP>(f[0].f + NJ, ra + d0, ra + d1);
        settle(acc);
        // a step's products with c while n is read; `first` and `second` behind their halves
        const auto multiply = [&](auto step, const auto& sc, const auto& c, auto& n, const uint32_t (&from)[3], auto first, auto second) {
            constexpr int S = decltype(step)::value;
            const auto a = [&](int i) {
                if constexpr (ELEM == 4) return c.f[NJ + i];
                else {
                    const u32x4_t &x = c.f[NJ + 2 * i], &y = c.f[NJ + 2 * i + 1];
                    return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
                }
            };
            constexpr int R = (NJ + XT * MI) * 2 / MI;
            mx_pair<ELEM, S, R, MxNext<ELEM, 0, STEP>>(acc[0], acc[1], a(0), a(1), c.f, sc.x[0], sc.x[1], sc.w, n.f, from);
            first();
            if constexpr (MI == 4) mx_pair<ELEM, S, R, MxNext<ELEM, R, STEP>>(acc[2], acc[3], a(2), a(3), c.f, sc.x[2], sc.x[3], sc.w, n.f + R, from);
            second();
        };
        uint32_t s = 0;  // the current tile's slot, in bytes
        const auto tile = [&](auto s0, auto s1, const auto& sc, auto last) {
            const uint32_t now = s;
            s = s == 2 * SLOT ? 0 : s + SLOT;
            const uint32_t mid[3] = {rb + now + c1, ra + now + (ELEM == 8 ? OpA::BYTES + d0 : c1), ra + now + OpA::BYTES + d1};
            const uint32_t end[3] = {rb + s + c0, ra + s + (ELEM == 8 ? d0 : c0), ra + s + d1};
            multiply(s0, sc, f[0], f[1], mid, [] {}, [] {});
            // the next tile has come, the one after it and the next scales but one need not have; all have read this one, whose
            // place the third from here takes
            wait_loads<LOADS + WORDS>();
            bare_barrier();
            char* const to = lds + now;
            multiply(s1, sc, f[1], f[0], end,
                     [&] {
#pragma unroll
                         for (int t = 0; t < XT; ++t) oa.fetch(to + t * OpA::BYTES, tid);
                     },
                     [&] {
                         ob.fetch(to + XT * OpA::BYTES, tid);
                         in_order();
                         last();
                     });
        };
        // Two groups in turn, each with its scales in registers of its own, which are asked for two tiles before their first use.
        // (One path through the loop: the compiler waits for what any path to a use may have left on its way.)
        constexpr std::integral_constant<int, 0> s0{};
        constexpr std::integral_constant<int, 1> s1{};
        constexpr std::integral_constant<int, 2> s2{};
        constexpr std::integral_constant<int, 3> s3{};
        int t = 0;
        for (; t + 4 <= tiles; t += 4) {
            const int k = k0 + t * 256 + 2 * kMxGroup;
            tile(s0, s1, sc[0], [] {});
            tile(s2, s3, sc[0], [&] { scales(sc[0], k); });
            tile(s0, s1, sc[1], [] {});
            tile(s2, s3, sc[1], [&] { scales(sc[1], k + kMxGroup); });
        }
        if (t < tiles) tile(s0, s1, sc[0], [] {});
        if (t + 1 < tiles) tile(s2, s3, sc[0], [] {});
        if (t + 2 < tiles) tile(s0, s1, sc[1], [] {});
        settle(acc);
    } else {
        int slot = 0;
        scales(sc[0], k0);
        fetch(0);
        fetch(1);
        for (int k = k0; k < k1; k += kMxGroup) {
            uint32_t tx[MI], tw[NJ];
#pragma unroll
            for (int i = 0; i < MI; ++i) tx[i] = sc[0].x[i];
#pragma unroll
            for (int n = 0; n < NJ; ++n) tw[n] = sc[0].w[n];
            const auto half = [&](auto which) {
                constexpr int H = decltype(which)::value;
                // this tile has come; all have read the one before, whose place the tile after the next takes
                wait_loads<LOADS>();
                bare_barrier();
                const uint32_t s = (uint32_t)(slot * SLOT);
                u32x4_t fw[2 * NJ], fx[XT][2 * MI];
                read_frags<NJ, STEP>(fw, rb + s + c0, rb + s + c1);
#pragma unroll
                for (int t = 0; t < XT; ++t) read_frags<MI, STEP>(fx[t], ra + s + t * OpA::BYTES + d0, ra + s + t * OpA::BYTES + d1);
                fetch(slot == 0 ? 2 : slot - 1);
                slot = slot == 2 ? 0 : slot + 1;
                if constexpr (H == 0) scales(sc[0], k + kMxGroup);
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int n = 0; n < NJ; ++n) {
                        acc[i][n] = mx_mma<8, true, 2 * H>(fw[2 * n], fx[0][2 * i], fx[0][2 * i + 1], tw[n], tx[i], acc[i][n]);
                        acc[i][n] = mx_mma<8, true, 2 * H + 1>(fw[2 * n + 1], fx[1][2 * i], fx[1][2 * i + 1], tw[n], tx[i], acc[i][n]);
                    }
            };
            half(std::integral_constant<int, 0>{});
            if (k + 256 < k1) half(std::integral_constant<int, 1>{});
        }
    }
    wait_loads<0>();  // (tiles past the last may still be on their way)
    __syncthreads();
    write_block<T, false, WM>(ga, acc, 0, lds + wave * WM * 256, m0 + wm, n0 + wn, sp, lane);
#endif
}

// ---- 256 x 256 tiles ----
// The pipeline of the half-precision products' widest tile (gemm_wide): four wavefronts, each with 128 x 128 of C in the second
// half of the register file; while a step (128 k values) is multiplied, the next one's fragments are read from LDS, and tiles
// of 128 bytes of a row are on their way there.  16 products of 16 x 16 x 128 are one block of assembly, with the reads
// between them: a wavefront has its SIMD to itself.  Loads, scales' among them, stand between the blocks; their waits are the
// compiler's and wait_loads'.
// The main loop is bound by the matrix cores and the card's power: with its scales the instruction takes 24 cycles (without, 16; one
// of 32 x 32 x 64, which does twice as much, 33; with an E4M3 operand 32), and on random elements it reaches 5640 TFLOP/s on the
// whole card.  16384 x 8192 -> 4096 274 us, 4020 TFLOP/s: with 2048, 4096 and 8192 k values 105, 157 and 262 us in one session, so
// that 208 are the main loop, 5290 TFLOP/s, and 53 the starts and ends of four rounds of tiles, which all units reach at the same
// time.  E4M3 rows 358 us, 3070 TFLOP/s.  Measured and left: blocks of 32 x 32 (280 us where this took 254), work-groups that stay and ask for the next
// tile's operands during the epilogue (the same), results stored from the registers without LDS (265-286 for 254), no masks
// on the loads (268 for 270).
#define DLC_MX_MOST4(OP, BL) \
    asm volatile("s_nop 1\n\t" \
    DLC_MX(OP, BL, 4, 18, 16, 28, 26) "ds_read_b128 %0, %36 offset:%37\n\t" DLC_MX(OP, BL, 5, 19, 16, 29, 26) "ds_read_b128 %1, %36 offset:%38\n\t" \
    DLC_MX(OP, BL, 6, 20, 16, 30, 26) "ds_read_b128 %2, %36 offset:%39\n\t" DLC_MX(OP, BL, 7, 21, 16, 31, 26) "ds_read_b128 %3, %36 offset:%40\n\t" \
    DLC_MX(OP, BL, 8, 22, 16, 32, 26) DLC_MX(OP, BL, 9, 23, 16, 33, 26) DLC_MX(OP, BL, 10, 24, 16, 34, 26) DLC_MX(OP, BL, 11, 25, 16, 35, 26) \
    DLC_MX(OP, BL, 12, 18, 17, 28, 27) DLC_MX(OP, BL, 13, 19, 17, 29, 27) DLC_MX(OP, BL, 14, 20, 17, 30, 27) DLC_MX(OP, BL, 15, 21, 17, 31, 27) \
    "s_waitcnt lgkmcnt(0)" \
    : "=&v"(next[0]), "=&v"(next[1]), "=&v"(next[2]), "=&v"(next[3]), \
      "+a"(acc0[0]), "+a"(acc0[1]), "+a"(acc0[2]), "+a"(acc0[3]), "+a"(acc0[4]), "+a"(acc0[5]), "+a"(acc0[6]), "+a"(acc0[7]), \
      "+a"(acc1[0]), "+a"(acc1[1]), "+a"(acc1[2]), "+a"(acc1[3]) \
    : "v"(a0), "v"(a1), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(b[4]), "v"(b[5]), "v"(b[6]), "v"(b[7]), "v"(sa0), "v"(sa1), \
      "v"(sb[0]), "v"(sb[1]), "v"(sb[2]), "v"(sb[3]), "v"(sb[4]), "v"(sb[5]), "v"(sb[6]), "v"(sb[7]), "v"(from), "i"(OFF), "i"(OFF + STEP), "i"(OFF + 2 * STEP), "i"(OFF + 3 * STEP) \
    : "memory")
#define DLC_MX_MOST8(OP, BL) \
    asm volatile("s_nop 1\n\t" \
    DLC_MX(OP, BL, 6, 20, 18, 30, 28) "ds_read_b128 %0, %38 offset:%41\n\t" DLC_MX(OP, BL, 7, 21, 18, 31, 28) "ds_read_b128 %1, %39 offset:%41\n\t" \
    DLC_MX(OP, BL, 8, 22, 18, 32, 28) "ds_read_b128 %2, %38 offset:%42\n\t" DLC_MX(OP, BL, 9, 23, 18, 33, 28) "ds_read_b128 %3, %39 offset:%42\n\t" \
    DLC_MX(OP, BL, 10, 24, 18, 34, 28) "ds_read_b128 %4, %40 offset:%43\n\t" DLC_MX(OP, BL, 11, 25, 18, 35, 28) "ds_read_b128 %5, %40 offset:%44\n\t" \
    DLC_MX(OP, BL, 12, 26, 18, 36, 28) DLC_MX(OP, BL, 13, 27, 18, 37, 28) DLC_MX(OP, BL, 14, 20, 19, 30, 29) DLC_MX(OP, BL, 15, 21, 19, 31, 29) \
    DLC_MX(OP, BL, 16, 22, 19, 32, 29) DLC_MX(OP, BL, 17, 23, 19, 33, 29) \
    "s_waitcnt lgkmcnt(0)" \
    : "=&v"(na[0]), "=&v"(na[1]), "=&v"(na[2]), "=&v"(na[3]), "=&v"(nb[0]), "=&v"(nb[1]), \
      "+a"(acc0[0]), "+a"(acc0[1]), "+a"(acc0[2]), "+a"(acc0[3]), "+a"(acc0[4]), "+a"(acc0[5]), "+a"(acc0[6]), "+a"(acc0[7]), \
      "+a"(acc1[0]), "+a"(acc1[1]), "+a"(acc1[2]), "+a"(acc1[3]) \
    : "v"(a0), "v"(a1), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(b[4]), "v"(b[5]), "v"(b[6]), "v"(b[7]), "v"(sa0), "v"(sa1), \
      "v"(sb[0]), "v"(sb[1]), "v"(sb[2]), "v"(sb[3]), "v"(sb[4]), "v"(sb[5]), "v"(sb[6]), "v"(sb[7]), "v"(from0), "v"(from1), "v"(from_b), "i"(OFF_A), "i"(OFF_A + STEP), "i"(OFF_B), "i"(OFF_B + STEP) \
    : "memory")
#define DLC_MX_REST(OP, BL) \
    asm volatile( \
    DLC_MX(OP, BL, 0, 5, 4, 10, 9) DLC_MX(OP, BL, 1, 6, 4, 11, 9) DLC_MX(OP, BL, 2, 7, 4, 12, 9) DLC_MX(OP, BL, 3, 8, 4, 13, 9) \
    : "+a"(acc1[4]), "+a"(acc1[5]), "+a"(acc1[6]), "+a"(acc1[7]) \
    : "v"(a1), "v"(b[4]), "v"(b[5]), "v"(b[6]), "v"(b[7]), "v"(sa1), "v"(sb[4]), "v"(sb[5]), "v"(sb[6]), "v"(sb[7]) \
    : "memory")
// Rows of blocks acc0 and acc1 += a0 and a1 times b, with byte S of the scales: twelve products and four reads, STEP bytes
// apart, `then` (one load), the other four products
template <int S, int OFF, int STEP, typename F>
__device__ __forceinline__ void mx_chunk4(f32x4* acc0, f32x4* acc1, const u32x4_t& a0, const u32x4_t& a1, const u32x4_t* b, uint32_t sa0,
                                          uint32_t sa1, const uint32_t* sb, u32x4_t* next, uint32_t from, F then) {
    if constexpr (S == 0) DLC_MX_MOST4(DLC_MX_BYTE0, "4");
    else if constexpr (S == 1) DLC_MX_MOST4(DLC_MX_BYTE1, "4");
    else if constexpr (S == 2) DLC_MX_MOST4(DLC_MX_BYTE2, "4");
    else DLC_MX_MOST4(DLC_MX_BYTE3, "4");
    then();
    if constexpr (S == 0) DLC_MX_REST(DLC_MX_BYTE0, "4");
    else if constexpr (S == 1) DLC_MX_REST(DLC_MX_BYTE1, "4");
    else if constexpr (S == 2) DLC_MX_REST(DLC_MX_BYTE2, "4");
    else DLC_MX_REST(DLC_MX_BYTE3, "4");
}

// ... a0 and a1 of 8 bits an element; two rows' fragments of two chunks each (at from0 and from1) and two of b are read
template <int S, int OFF_A, int OFF_B, int STEP, typename F>
__device__ __forceinline__ void mx_chunk8(f32x4* acc0, f32x4* acc1, const i32x8& a0, const i32x8& a1, const u32x4_t* b, uint32_t sa0,
                                          uint32_t sa1, const uint32_t* sb, u32x4_t* na, u32x4_t* nb, uint32_t from0, uint32_t from1,
                                          uint32_t from_b, F then) {
    if constexpr (S == 0) DLC_MX_MOST8(DLC_MX_BYTE0, "0");
    else if constexpr (S == 1) DLC_MX_MOST8(DLC_MX_BYTE1, "0");
    else if constexpr (S == 2) DLC_MX_MOST8(DLC_MX_BYTE2, "0");
    else DLC_MX_MOST8(DLC_MX_BYTE3, "0");
    then();
    if constexpr (S == 0) DLC_MX_REST(DLC_MX_BYTE0, "0");
    else if constexpr (S == 1) DLC_MX_REST(DLC_MX_BYTE1, "0");
    else if constexpr (S == 2) DLC_MX_REST(DLC_MX_BYTE2, "0");
    else DLC_MX_REST(DLC_MX_BYTE3, "0");
}
#undef DLC_MX
#undef DLC_MX_MOST4
#undef DLC_MX_MOST8
#undef DLC_MX_REST
#undef DLC_MX_BYTE0
#undef DLC_MX_BYTE1
#undef DLC_MX_BYTE2
#undef DLC_MX_BYTE3
#pragma clang diagnostic pop

// One operand's scales: a lane's words for N blocks of 16 rows, four steps each
template <int N>
struct Scales {
    const uint8_t* base;  // of the tile's first row in the next group
    int64_t left;         // bytes from there to the end
    int64_t step;
    uint32_t voff;
    uint32_t now[N], next[N];
    // row: the tile's first; mine: the wavefront's first row in it
    __device__ __forceinline__ void init(const uint8_t* p, int row, int mine, int rows, int group, int groups, int lane) {
        step = (int64_t)rows * 16;
        base = p + (int64_t)group * step + (int64_t)row * 16;
        left = (int64_t)(groups - group) * step - (int64_t)row * 16;
        voff = (uint32_t)((mine + (lane & 15)) * 16 + (lane >> 4) * 4);
    }
    // The next group's (past the last: zeros; rows past the last get others' scales, and their sums are not stored)
    __device__ __forceinline__ void load() {
        const uint32_t range = left <= 0 ? 0u : left < 8192 ? (uint32_t)left : 8192u;
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, range, 0x00020000);
#pragma unroll
        for (int i = 0; i < N; ++i) next[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, voff + i * 256, 0, 0);
        base += step;
        left -= step;
    }
    // (to the compiler all of them are used, and none of the loads that waits count can go)
    __device__ __forceinline__ void turn() {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            now[i] = next[i];
            asm volatile("" : "+v"(now[i]));
        }
    }
};

template <typename T, int ELEM>
__global__ __launch_bounds__(256, 1) void k_mx_wide(const MxGemmArgs mx) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int THREADS = 256, W = 256, P = W / 2, MI = P / 16, NJ = MI, TB = 128;
    using OpA = Operand<uint8_t, false, W, TB, THREADS, false>;
    using OpB = OpA;
    constexpr int B0 = 3 * OpA::BYTES, STEP = 16 * TB;
    __shared__ __attribute__((aligned(16))) char lds[5 * OpA::BYTES];
    const GemmArgs& ga = mx.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tm, tn, sp;
    tile_of(blockIdx.x, gridDim.x, ga.tiles_m, ga.tiles_n, tm, tn, sp);
    const int m0 = tm * W, n0 = tn * W;
    const int k0 = sp * ga.kper, k1 = min(ga.K, k0 + ga.kper), groups = (ga.K + kMxGroup - 1) / kMxGroup;
    const int wm = (wave >> 1) * P, wn = (wave & 1) * P;
    OpA oa;
    OpB ob;
    oa.init(ga.a, ga.lda, m0, ga.M, k0 * ELEM / 8, k1 * ELEM / 8, tid);
    ob.init(ga.b, ga.ldb, n0, ga.N, k0 / 2, k1 / 2, tid);
    Scales<MI> sa;
    Scales<NJ> sb;
    sa.init(mx.xs, m0, wm, ga.M, k0 / kMxGroup, groups, lane);
    sb.init(mx.ws, n0, wn, ga.N, k0 / kMxGroup, groups, lane);

    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const uint32_t at = (uint32_t)(uintptr_t)(const lds_char*)lds;
    typename OpA::template Place<MI> pa;
    typename OpB::template Place<NJ> pb;
    OpA::template place<MI>(pa, at, wm, lane);
    OpB::template place<NJ>(pb, at + B0, wn, lane);
    keep(pa);
    keep(pb);
    char* const mine = lds + wave * 1024;  // where the wavefront's first load of a tile in the first slot goes
    uint32_t slot_a = 0, slot_b = 0;       // slots of the current tiles, in bytes
    const auto after = [](uint32_t s) { return s == 2 * OpA::BYTES ? 0u : s + (uint32_t)OpA::BYTES; };
    const auto before = [](uint32_t s) { return s == 0 ? 2u * OpA::BYTES : s - (uint32_t)OpA::BYTES; };
    sa.load();
    sb.load();
    sa.turn();
    sb.turn();

    if constexpr (ELEM == 4) {
        const int tiles = (k1 - k0 + 255) / 256;
        struct { u32x4_t a[MI], b[NJ]; } f[2];
        oa.fetch(lds, tid);
        ob.fetch(lds + B0, tid);
        oa.fetch(lds + OpA::BYTES, tid);
        ob.fetch(lds + B0 + OpB::BYTES, tid);
        wait_loads<2 * OpA::PASSES>();
        bare_barrier();
        read_rows<NJ, STEP, 0>(f[0].b, pb.a[0]);
        read_rows<MI, STEP, 0>(f[0].a, pa.a[0]);
        settle(acc);
        // A step's products with c's fragments while n's are read; behind each of the four blocks two loads
        const auto multiply = [&](auto step, auto& c, auto& n, uint32_t ra, uint32_t rb, const auto& o, char* to) {
            constexpr int S = decltype(step)::value;
            mx_chunk4<S, 0, STEP>(acc[0], acc[1], c.a[0], c.a[1], c.b, sa.now[0], sa.now[1], sb.now, n.b, rb, [&] { o.template load<0, 1>(to, 0); });
            o.template load<1, 1>(to, 0);
            mx_chunk4<S, 4 * STEP, STEP>(acc[2], acc[3], c.a[2], c.a[3], c.b, sa.now[2], sa.now[3], sb.now, n.b + 4, rb, [&] { o.template load<2, 1>(to, 0); });
            o.template load<3, 1>(to, 0);
            mx_chunk4<S, 0, STEP>(acc[4], acc[5], c.a[4], c.a[5], c.b, sa.now[4], sa.now[5], sb.now, n.a, ra, [&] { o.template load<4, 1>(to, 0); });
            o.template load<5, 1>(to, 0);
            mx_chunk4<S, 4 * STEP, STEP>(acc[6], acc[7], c.a[6], c.a[7], c.b, sa.now[6], sa.now[7], sb.now, n.a + 4, ra, [&] { o.template load<6, 1>(to, 0); });
            o.template load<7, 1>(to, 0);
        };
        const auto tile = [&](auto first, auto second) {
            // the tile's first half; A's tile after the next goes where the one before was
            oa.mask();
            multiply(first, f[0], f[1], pa.a[1] + slot_a, pb.a[1] + slot_b, oa, mine + before(slot_a));
            oa.advance();
            // the next tiles have come (scales need not have, behind which are A's loads), and all have read this one: B's after
            // the next takes its place
            wait_loads<OpA::PASSES + (decltype(first)::value == 0 ? MI + NJ : 0)>();
            bare_barrier();
            slot_a = after(slot_a);
            const uint32_t free_b = slot_b;
            slot_b = OpB::BYTES - slot_b;
            ob.mask();
            multiply(second, f[1], f[0], pa.a[0] + slot_a, pb.a[0] + slot_b, ob, mine + B0 + free_b);
            ob.advance();
        };
        for (int s = 0; s < tiles; s += 2) {
            in_order();
            sa.load();
            sb.load();
            tile(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
            if (s + 1 < tiles) tile(std::integral_constant<int, 2>{}, std::integral_constant<int, 3>{});
            sa.turn();
            sb.turn();
        }
    } else {
        const int steps = (k1 - k0 + 127) / 128;
        u32x4_t a[2][4], b[2][NJ];  // two rows' fragments of A, two chunks each, and the next two's
        oa.fetch(lds, tid);
        ob.fetch(lds + B0, tid);
        oa.fetch(lds + OpA::BYTES, tid);
        ob.fetch(lds + B0 + OpB::BYTES, tid);
        wait_loads<2 * OpA::PASSES>();
        bare_barrier();
        read_rows<NJ, STEP, 0>(b[0], pb.a[0]);
        read_halves<2, STEP>(a[0], pa.a[0], pa.a[1]);
        settle(acc);
        const auto wide = [](const u32x4_t& x, const u32x4_t& y) {
            return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
        };
        // Step n, S of its group: multiplies A's tile n and half H of a tile of B, reads what comes next.  Behind the barrier
        // before its last block all have read tile n, and n + 1 has come: tile n + 3 takes n's place, in eight loads until the
        // middle of the next step.  Behind an odd step's barrier B's tile after the next goes before them.
        const auto step = [&](auto which) {
            constexpr int S = decltype(which)::value, H = S & 1;
            const uint32_t ra = slot_a, nx = after(slot_a), free_b = slot_b;
            const uint32_t rb = H == 0 ? pb.a[1] + slot_b : pb.a[0] + (OpB::BYTES - slot_b);
            char* const early = mine + before(slot_a);
            char* const late = mine + slot_a;
            char* const late_b = mine + B0 + free_b;
            u32x4_t* const nb = b[1 - H];
            const u32x4_t* const cb = b[H];
            mx_chunk8<S, 2 * STEP, 0, STEP>(acc[0], acc[1], wide(a[0][0], a[0][1]), wide(a[0][2], a[0][3]), cb, sa.now[0], sa.now[1], sb.now, a[1], nb,
                                            pa.a[0] + ra, pa.a[1] + ra, rb, [&] { oa.template load<H == 0 ? 0 : 4, H == 0 ? 2 : 1>(early, 0); });
            oa.template load<H == 0 ? 2 : 5, H == 0 ? 2 : 1>(early, 0);
            mx_chunk8<S, 4 * STEP, 2 * STEP, STEP>(acc[2], acc[3], wide(a[1][0], a[1][1]), wide(a[1][2], a[1][3]), cb, sa.now[2], sa.now[3], sb.now, a[0],
                                                   nb + 2, pa.a[0] + ra, pa.a[1] + ra, rb, [&] { oa.template load<H == 0 ? 4 : 6, H == 0 ? 2 : 1>(early, 0); });
            oa.template load<H == 0 ? 6 : 7, H == 0 ? 2 : 1>(early, 0);
            oa.advance();
            oa.mask();
            mx_chunk8<S, 6 * STEP, 4 * STEP, STEP>(acc[4], acc[5], wide(a[0][0], a[0][1]), wide(a[0][2], a[0][3]), cb, sa.now[4], sa.now[5], sb.now, a[1],
                                                   nb + 4, pa.a[0] + ra, pa.a[1] + ra, rb, [] {});
            wait_loads<OpA::PASSES>();
            bare_barrier();
            if constexpr (H == 1) {
                if constexpr (S == 1) {
                    sa.load();
                    sb.load();
                }
                ob.mask();
                ob.template load<0, 2>(late_b, 0);
            } else {
                oa.template load<0, 1>(late, 0);
            }
            mx_chunk8<S, 0, 6 * STEP, STEP>(acc[6], acc[7], wide(a[1][0], a[1][1]), wide(a[1][2], a[1][3]), cb, sa.now[6], sa.now[7], sb.now, a[0],
                                            nb + 6, pa.a[0] + nx, pa.a[1] + nx, rb, [&] {
                                                if constexpr (H == 0) oa.template load<1, 2>(late, 0);
                                                else ob.template load<2, 3>(late_b, 0);
                                            });
            if constexpr (H == 0) {
                oa.template load<3, 1>(late, 0);
            } else {
                ob.template load<5, 3>(late_b, 0);
                ob.advance();
                slot_b = OpB::BYTES - slot_b;
            }
            slot_a = nx;
        };
        oa.mask();
        for (int n = 0; n < steps; n += 4) {
            step(std::integral_constant<int, 0>{});
            if (n + 1 < steps) step(std::integral_constant<int, 1>{});
            if (n + 2 < steps) step(std::integral_constant<int, 2>{});
            if (n + 3 < steps) step(std::integral_constant<int, 3>{});
            sa.turn();
            sb.turn();
        }
    }
    wait_loads<0>();  // (tiles past the last may still be on their way)
    settle(acc);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < P / 64; ++h) write_block<T, false, P>(ga, acc, h * 4, lds + wave * P * 256, m0 + wm, n0 + wn + h * 64, sp, lane);
#endif
}

template <typename T, int ELEM>
static void mx_go(const MxGemmArgs& g, int tile, hipStream_t s) {
    const dim3 skinny((unsigned)((g.c.N + 15) / 16), (unsigned)((g.c.M + kMxSkinnyRows - 1) / kMxSkinnyRows)), grid((unsigned)(g.c.tiles_m * g.c.tiles_n * g.c.split));
    if (tile == kMxSkinny && g.c.M <= 16) k_mx_skinny<T, ELEM, 1><<<skinny, dim3(64 * kSkinnyWaves), 0, s>>>(g);
    else if (tile == kMxSkinny) k_mx_skinny<T, ELEM, 2><<<skinny, dim3(64 * kSkinnyWaves), 0, s>>>(g);
    else if (tile == 2) k_mx_tile<T, ELEM, 64><<<grid, dim3(256), 0, s>>>(g);
    else if (tile == 1) k_mx_tile<T, ELEM, 128><<<grid, dim3(256), 0, s>>>(g);
    else if constexpr (!kMxExact<T, ELEM>) k_mx_wide<T, ELEM><<<grid, dim3(256), 0, s>>>(g);
}

template <typename T>
hipError_t MxOps<T>::gemm(const MxGemmArgs& g, int elem_x, int tile, hipStream_t s) {
    if (elem_x == DLC_MX_E4M3) mx_go<T, 8>(g, tile, s);
    else mx_go<T, 4>(g, tile, s);
    return hipGetLastError();
}

}  // namespace dlc
