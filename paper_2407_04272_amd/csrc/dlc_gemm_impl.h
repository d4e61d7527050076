// The matrix products of the dense operators, one template for three element types and three operand layouts.
//
// C[m][n] = sum over k of A(m, k) B(n, k), tile by tile: a work-group takes BM x BN of C and walks k in tiles of 128 bytes
// (64 half precision or 32 fp32 elements).  Each k tile of A and B goes from memory to one of two buffers in LDS while the
// matrix cores work on the other.  A wavefront holds a WM x WN part of C in registers as 16 x 16 blocks.
//
// LDS layouts (16-byte chunks; chosen so that 16 lanes that read together touch 16 different sixteenths of the banks):
//   k along a row     row r, chunk c of its 8 at r * 128 + (c ^ ((r >> 1) & 7)) * 16
//   k down a column   k row r of BM (BN) elements, 32-byte (fp32: 64-byte) units u at u ^ f(r): half precision reads these
//                     with the transposing LDS read (a group of 16 lanes takes 4 k rows of 16 elements and hands every lane
//                     the 4 k values of its element), fp32 element by element
// A load to LDS writes 64 consecutive chunks per wavefront, so the permutation is applied to the address that is read.
#pragma once
#include "dlc_dense.h"

namespace dlc {

typedef __attribute__((address_space(3))) void lds_void;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// One 16 x 16 block times 64 bytes of k: rows from `r`, columns from `c`; lane l holds D[(l / 16) * 4 + i][l % 16].
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
template <int ES>
__device__ __forceinline__ u32x4_t load_part(const char* p) {
    if constexpr (ES == 2) return *reinterpret_cast<const u32x4_by2*>(p);
    else return *reinterpret_cast<const u32x4_by4*>(p);
}

// permutation of a k row's units where k runs down a column; UNITS of them in a row
template <typename T, int UNITS>
__device__ __forceinline__ int unit_swizzle(int krow) {
    const int f = sizeof(T) == 4 ? (krow >> 2) & 3 : (krow & 3) | (((krow >> 3) & 1) << 2);
    return f & (UNITS - 1);
}

// One operand's path into LDS.  KT: k runs down a column.  R: rows (columns of C) of the tile.  DUAL: the tile's rows are
// those of two matrices of `half` rows each, 32 of the first and 32 of the second in turn.
template <typename T, bool KT, int R, int THREADS, bool ALIGNED, bool DUAL>
struct Operand {
    static constexpr int EPC = 16 / sizeof(T);          // elements of a chunk
    static constexpr int BK = kTileBytes / sizeof(T);   // elements of a k tile
    static constexpr int CPR = KT ? R / EPC : 8;        // chunks of a row in LDS
    static constexpr int ROWS = KT ? BK : R;            // rows in LDS
    static constexpr int PASSES = ROWS * CPR / THREADS; // chunks a thread moves
    static constexpr int RSTEP = THREADS / CPR;         // rows between them
    static constexpr bool SAME = RSTEP % 16 == 0;       // ... which all have the same permutation
    static constexpr int BYTES = ROWS * CPR * 16;
    static_assert(PASSES * THREADS == ROWS * CPR , "tile and work-group");

    const char* base;      // of the tile's first row and the current k tile
    int64_t ld;            // bytes
    int row0, slot;        // this thread's first row and its place in it
    int chunk;             // the chunk that stands there
    int rows_left;         // rows of the matrix from the tile's first on (columns, where k runs down)
    int k_left;            // k values from the current tile on
    uint32_t voff;         // byte offset of the thread's first chunk
    int64_t half_off;      // DUAL: bytes from a row of the first half to the same row of the second
    u32x4_t reg[ALIGNED ? 1 : PASSES];

    __device__ __forceinline__ static int chunk_at(int r, int slot) {
        if constexpr (KT) {
            constexpr int UB = sizeof(T) == 4 ? 2 : 1;  // log2 of a unit's chunks
            return (((slot >> UB) ^ unit_swizzle<T, (CPR >> UB)>(r)) << UB) | (slot & ((1 << UB) - 1));
        } else {
            return slot ^ ((r >> 1) & 7);
        }
    }

    __device__ __forceinline__ int chunk_of(int i) const { return SAME ? chunk : chunk_at(row0 + i * RSTEP, slot); }

    // row: first row (column) of the tile; rows: of the matrix (DUAL: of one half)
    __device__ __forceinline__ void init(const void* p, int64_t ld_elems, int row, int rows, int k0, int k1, int tid) {
        ld = ld_elems * (int64_t)sizeof(T);
        row0 = tid / CPR;
        slot = tid % CPR;
        chunk = chunk_at(row0, slot);
        rows_left = rows - row;
        k_left = k1 - k0;
        if constexpr (KT) base = static_cast<const char*>(p) + (int64_t)row * sizeof(T) + (int64_t)k0 * ld;
        else base = static_cast<const char*>(p) + (int64_t)row * ld + (int64_t)k0 * sizeof(T);
        if constexpr (DUAL) half_off = (int64_t)rows * ld;
        voff = (uint32_t)row0 * (uint32_t)ld + chunk * 16u;
    }

    // Copies the current k tile to `lds` (ALIGNED), or to registers; then steps to the next.  What lies outside the
    // matrix becomes 0: by the buffer's range check where rows or k rows end, by an offset past any range where a row does.
    __device__ __forceinline__ void fetch(char* lds, int tid) {
        if constexpr (ALIGNED) {
            // (a tile's rows span no more than 256 * 2^22 bytes = 2^30: no range reaches kOut)
            constexpr uint32_t kOut = 0x7FFFFFF0u;
            const int wave_lds = (tid & ~63) * 16;
            // rows run to the last valid one; where k runs along them its end is the range's end for the last row only
            const int nrow = KT ? k_left : rows_left, ncol = KT ? rows_left : k_left;
            // (whole chunks: a row that ends inside one is a row of dz, which is padded with zeros)
            const int64_t bytes = nrow > 0 && ncol > 0 ? (int64_t)(nrow - 1) * ld + (int64_t)((ncol + EPC - 1) / EPC) * 16 : 0;
            const int range = bytes < (int64_t)kOut ? (int)bytes : (int)kOut;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                char* const dst = lds + wave_lds + i * THREADS * 16;
                if constexpr (DUAL) {
                    const int r = row0 + i * RSTEP;
                    // (a wavefront's 8 rows are all of one matrix)
                    const bool second = __builtin_amdgcn_readfirstlane(r >> 5) & 1;
                    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)(base + (second ? half_off : 0)), 0, range, 0x00020000);
                    const uint32_t f = (uint32_t)(((r >> 6) << 5) | (r & 31));
                    const uint32_t v = chunk * EPC < ncol ? f * (uint32_t)ld + chunk * 16u : kOut;
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)dst, 16, v, 0, 0, 0);
                } else {
                    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, range, 0x00020000);
                    const int ch = chunk_of(i);
                    const uint32_t v = ch * EPC < ncol ? voff + (uint32_t)(i * RSTEP) * (uint32_t)ld + (uint32_t)(ch - chunk) * 16u : kOut;
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)dst, 16, v, 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int r = row0 + i * RSTEP, chunk = chunk_of(i);
                const char* p;
                int cnt;  // elements of the chunk inside the matrix
                if constexpr (KT) {
                    p = base + (int64_t)r * ld + chunk * 16;
                    cnt = r < k_left ? rows_left - chunk * EPC : 0;
                } else if constexpr (DUAL) {
                    const int f = ((r >> 6) << 5) | (r & 31);
                    p = base + ((r >> 5) & 1 ? half_off : 0) + (int64_t)f * ld + chunk * 16;
                    cnt = f < rows_left ? k_left - chunk * EPC : 0;
                } else {
                    p = base + (int64_t)r * ld + chunk * 16;
                    cnt = r < rows_left ? k_left - chunk * EPC : 0;
                }
                reg[i] = load_chunk(p, cnt);
            }
        }
        k_left -= BK;
        base += KT ? (int64_t)BK * ld : (int64_t)kTileBytes;
    }

    __device__ __forceinline__ static u32x4_t load_chunk(const char* p, int cnt) {
        if (cnt >= EPC) return load_part<sizeof(T)>(p);
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

    __device__ __forceinline__ void put(char* lds, int tid) const {
        if constexpr (!ALIGNED) {
#pragma unroll
            for (int i = 0; i < PASSES; ++i) *reinterpret_cast<u32x4_t*>(lds + (tid + i * THREADS) * 16) = reg[i];
        }
    }

    // 64 bytes of k (half a k tile, kk = 0, 1) of the 16 rows from `row` on: lane l gets row l % 16, its k values
    // (l / 16) * 16 bytes on
    __device__ __forceinline__ static u32x4_t frag(const char* lds, int row, int kk, int lane) {
        const int g = lane >> 4, j = lane & 15;
        if constexpr (!KT) {
            const int r = row + j;
            return *reinterpret_cast<const u32x4_t*>(lds + r * 128 + (((kk * 4 + g) ^ ((r >> 1) & 7)) << 4));
        } else if constexpr (sizeof(T) == 2) {
            const int k = kk * 32 + g * 8 + (j >> 2);
            const int u0 = (row >> 4) ^ unit_swizzle<T, CPR / 2>(k);  // (the same for k + 4)
            const char* p = lds + k * (CPR * 16) + u0 * 32 + (j & 3) * 8;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * CPR * 16));
            return __builtin_bit_cast(u32x4_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            u32x4_t q;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = kk * 16 + g * 4 + i;
                const int u0 = (row >> 4) ^ unit_swizzle<T, CPR / 4>(k);
                q[i] = *reinterpret_cast<const uint32_t*>(lds + k * (CPR * 16) + u0 * 64 + j * 4);
            }
            return q;
        }
    }
};

// orders a wavefront's LDS accesses before the ones after it (its own lanes only)
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Work-group -> tile.  Consecutive work-groups go to the 8 XCDs in turn; each XCD gets a stretch of consecutive tiles, and
// those run down 8 tile rows before the next column, so that the tiles an XCD works on at a time share rows and columns in
// its L2.
__device__ __forceinline__ void tile_of(int wg, int total, int tiles_m, int tiles_n, int& tm, int& tn, int& sp) {
    const int q = total / 8, r = total % 8, x = wg % 8, i = wg / 8;
    int t = x < r ? x * (q + 1) + i : r * (q + 1) + (x - r) * q + i;
    const int per = tiles_m * tiles_n;
    sp = t / per;
    t -= sp * per;
    const int band = 8 * tiles_n, b0 = t / band;
    const int h = min(8, tiles_m - b0 * 8);
    t -= b0 * band;
    tm = b0 * 8 + t % h;
    tn = t / h;
}

template <typename T, int LAY, int BM, int BN, int WAVES_M, int WAVES_N, bool ALIGNED, bool GATED>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) void k_gemm(const GemmArgs ga) {
    constexpr int THREADS = 64 * WAVES_M * WAVES_N;
    constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, MI = WM / 16, NJ = WN / 16;
    constexpr int BK = kTileBytes / sizeof(T);
    using OpA = Operand<T, LAY == L_TT, BM, THREADS, ALIGNED, false>;
    using OpB = Operand<T, LAY != L_KK, BN, THREADS, ALIGNED, GATED>;
    static_assert(!GATED || WN == 64, "a wavefront's columns are 32 of the gate and 32 of the other");
    constexpr int STAGE = OpA::BYTES + OpB::BYTES;
    __shared__ __attribute__((aligned(16))) char lds0[STAGE];
    __shared__ __attribute__((aligned(16))) char lds1[STAGE];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int tm, tn, sp;
    tile_of(blockIdx.x, gridDim.x, ga.tiles_m, ga.tiles_n, tm, tn, sp);
    const int m0 = tm * BM, n0 = tn * (GATED ? BN / 2 : BN);
    const int k0 = sp * ga.kper, k1 = min(ga.K, k0 + ga.kper);
    OpA oa;
    OpB ob;
    oa.init(ga.a, ga.lda, m0, ga.M, k0, k1, tid);
    ob.init(ga.b, ga.ldb, n0, ga.N, k0, k1, tid);
    const int steps = (k1 - k0 + BK - 1) / BK;
    const int wm = (wave / WAVES_N) * WM, wn = (wave % WAVES_N) * WN;

    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto compute = [&](const char* lds) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4_t fa[MI], fb[NJ];
#pragma unroll
            for (int j = 0; j < NJ; ++j) fb[j] = OpB::frag(lds + OpA::BYTES, wn + j * 16, kk, lane);
#pragma unroll
            for (int i = 0; i < MI; ++i) fa[i] = OpA::frag(lds, wm + i * 16, kk, lane);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] = mma<T>(fb[j], fa[i], acc[i][j]);
        }
    };
    // one k tile: wait for it, let the other buffer's readers finish, start the next tile's loads into that buffer
    auto step = [&](char* cur, char* nxt, bool more) {
        if constexpr (ALIGNED) {
            __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
            if (more) { oa.fetch(nxt, tid); ob.fetch(nxt + OpA::BYTES, tid); }
            compute(cur);
        } else {
            oa.put(cur, tid);
            ob.put(cur + OpA::BYTES, tid);
            __syncthreads();
            if (more) { oa.fetch(nullptr, tid); ob.fetch(nullptr, tid); }
            compute(cur);
        }
    };
    if (steps > 0) {
        oa.fetch(lds0, tid);
        ob.fetch(lds0 + OpA::BYTES, tid);
    }
    for (int s = 0; s < steps; s += 2) {
        step(lds0, lds1, s + 1 < steps);
        if (s + 1 < steps) step(lds1, lds0, s + 2 < steps);
    }

    // Epilogue: a wavefront's part goes through its own piece of LDS, so that a lane gets eight consecutive columns; the
    // 16-byte units of a row are permuted by the row
    constexpr int RM = WM < 64 ? WM : 64;  // rows at a time
    static_assert(WN == 64 && WM % RM == 0, "a row of the piece has 16 units");
    static_assert(WAVES_M * WAVES_N * RM * 256 <= 2 * STAGE, "room for the epilogue");
    constexpr int PER = STAGE / (RM * 256);  // wavefronts whose pieces are in the first buffer
    __syncthreads();
    char* const buf = (wave < PER ? lds0 + wave * RM * 256 : lds1 + (wave - PER) * RM * 256);
    const uint64_t offset = full_offset(ga.e.offset, ga.e.d_offset);
    const int g = lane >> 4, c16 = lane & 15;
    constexpr int CH = GATED ? 4 : 8;  // chunks of eight columns in a row
#pragma unroll
    for (int h = 0; h < WM / RM; ++h) {
#pragma unroll
        for (int i = 0; i < RM / 16; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                *reinterpret_cast<f32x4*>(buf + (i * 16 + c16) * 256 + (((j * 4 + g) ^ c16) << 4)) = acc[h * (RM / 16) + i][j];
        wave_sync();
#pragma unroll 1
        for (int q = 0; q < RM * CH / 64; ++q) {
            const int idx = q * 64 + lane, row = idx / CH, ch = idx % CH;
            const int m = m0 + wm + h * RM + row, col = n0 + (GATED ? wn / 2 : wn) + ch * 8;
            float s[8], u[8];
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                *reinterpret_cast<f32x4*>(s + v * 4) = *reinterpret_cast<const f32x4*>(buf + row * 256 + (((ch * 2 + v) ^ (row & 15)) << 4));
                if constexpr (GATED)
                    *reinterpret_cast<f32x4*>(u + v * 4) = *reinterpret_cast<const f32x4*>(buf + row * 256 + (((8 + ch * 2 + v) ^ (row & 15)) << 4));
            }
            if (m < ga.M) {
                if (ga.split > 1) {
                    if (col < ga.N) {  // (the pitch of the partial sums has room for whole chunks)
                        float* p = ga.part + ((int64_t)sp * ga.M + m) * ga.part_ld + col;
                        *reinterpret_cast<f32x4*>(p) = *reinterpret_cast<f32x4*>(s);
                        *reinterpret_cast<f32x4*>(p + 4) = *reinterpret_cast<f32x4*>(s + 4);
                        if constexpr (GATED) {
                            float* p2 = p + ((ga.N + 7) & ~7);
                            *reinterpret_cast<f32x4*>(p2) = *reinterpret_cast<f32x4*>(u);
                            *reinterpret_cast<f32x4*>(p2 + 4) = *reinterpret_cast<f32x4*>(u + 4);
                        }
                    }
                } else {
                    epilogue8<T, GATED>(ga.e, offset, m, col, s, u);
                }
            }
        }
        wave_sync();
    }
}

// Few rows (at most 16): the product is a pass over B.  A work-group takes 16 columns of C (gated: and the 16 of the other
// half), its wavefronts take stretches of k in turn straight from memory, and their sums meet in LDS.
constexpr int kSkinnyWaves = 8;

template <typename T, bool ALIGNED, bool GATED>
__global__ __launch_bounds__(64 * kSkinnyWaves) void k_skinny(const GemmArgs ga) {
    constexpr int EPC = 16 / sizeof(T), KS = 64 / sizeof(T), UN = 4;
    __shared__ __attribute__((aligned(16))) float sums[kSkinnyWaves][GATED ? 2 : 1][16][20];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, j = lane & 15;
    const int n0 = blockIdx.x * 16;
    const int64_t ldb = ga.ldb;
    const T* pa = static_cast<const T*>(ga.a) + (int64_t)min(j, ga.M - 1) * ga.lda + g * EPC;
    const T* pb = static_cast<const T*>(ga.b) + (int64_t)min(n0 + j, ga.N - 1) * ldb + g * EPC;
    const T* pu = pb + (int64_t)ga.N * ldb;
    const bool row_ok = j < ga.M;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f}, accu = {0.f, 0.f, 0.f, 0.f};
    using Op = Operand<T, false, 128, 256, false, false>;
    auto chunk = [&](const T* p, int k) {  // elements k .. k + EPC - 1 of a row, 0 past its end
        const int cnt = ga.K - k - g * EPC;
        if constexpr (ALIGNED) {
            u32x4_t q = {0u, 0u, 0u, 0u};
            if (cnt > 0) q = *reinterpret_cast<const u32x4_t*>(p + k);
            return q;
        } else {
            return Op::load_chunk(reinterpret_cast<const char*>(p + k), cnt);
        }
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
    if (tid < 32) {
        const int row = tid >> 1, ch = tid & 1;
        if (row < ga.M) {
            float s[8], u[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                s[v] = 0.f;
                u[v] = 0.f;
                for (int w = 0; w < kSkinnyWaves; ++w) {
                    s[v] += sums[w][0][row][ch * 8 + v];
                    if constexpr (GATED) u[v] += sums[w][1][row][ch * 8 + v];
                }
            }
            epilogue8<T, GATED>(ga.e, full_offset(ga.e.offset, ga.e.d_offset), row, n0 + ch * 8, s, u);
        }
    }
}

// Adds up the partial sums of a product whose k was cut, in the order of the cuts, and does the epilogue
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_join(const JoinArgs ja) {
    const int chunks = (ja.e.n + 7) / 8;
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (int64_t)chunks * ja.M) return;
    const int m = (int)(idx / chunks), col = (int)(idx % chunks) * 8;
    float s[8] = {}, u[8] = {};
    const float* p = ja.part + (int64_t)m * ja.part_ld + col;
    const int64_t slab = (int64_t)ja.M * ja.part_ld;
    const int up = (ja.e.n + 7) & ~7;
    for (int i = 0; i < ja.split; ++i, p += slab) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(p + h * 4);
#pragma unroll
            for (int v = 0; v < 4; ++v) s[h * 4 + v] += q[v];
            if constexpr (GATED) {
                const f32x4 r = *reinterpret_cast<const f32x4*>(p + up + h * 4);
#pragma unroll
                for (int v = 0; v < 4; ++v) u[h * 4 + v] += r[v];
            }
        }
    }
    epilogue8<T, GATED>(ja.e, full_offset(ja.e.offset, ja.e.d_offset), m, col, s, u);
}

// dz and the bias gradient's partial sums: a work-group takes 256 columns and rows_per_block rows, 32 lanes side by side
// with eight columns each, 8 rows at a time
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_dz(const DzArgs da) {
    __shared__ float red[8][256 + 8];
    const int tid = threadIdx.x, cx = tid & 31, ry = tid >> 5;
    const int col = (blockIdx.x * 32 + cx) * 8;
    const int64_t r0 = (int64_t)blockIdx.y * da.rows_per_block, r1 = min(da.M, r0 + da.rows_per_block);
    const uint64_t offset = full_offset(da.offset, da.d_offset);
    const int cnt = da.n - col;
    // the other half's columns follow at once, as the weight's rows do: the products take [g | u] as one matrix
    const int last = GATED ? 2 * da.n : da.n;
    float sum[GATED ? 2 : 1][8] = {};
    if (cnt > 0) {
        for (int64_t r = r0 + ry; r < r1; r += 8) {
            float d[8], z[8], u[8];
            load8(static_cast<const T*>(da.dy) + r * da.ld_dy + col, cnt, da.vec & 1, d);
            if (da.thr) {
                const uint32_t keep = keep_mask((uint32_t)col >> 3, (uint32_t)r, da.seed, offset, da.thr);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = (keep >> i) & 1u ? d[i] * da.scale : 0.0f;
            }
            if (da.pre) {
                const T* p = static_cast<const T*>(da.pre) + r * da.ld_pre + col;
                load8(p, cnt, da.vec & 2, z);
                if constexpr (GATED) load8(p + da.n, cnt, (da.vec & 2) && da.n % 8 == 0, u);
                float slope[8];
                act_both(da.act, z, slope);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (GATED) {
                        const float dh = d[i];
                        d[i] = dh * u[i] * slope[i];
                        u[i] = dh * z[i];
                    } else {
                        d[i] = slope[i] == 0.0f ? 0.0f : d[i] * slope[i];  // (a gradient that is not finite does not pass a closed unit)
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
                    store8(q, cnt, true, d);
                    store8(q + da.n, cnt, da.n % 8 == 0, u);
                    if (cnt <= 8)
                        for (int i = cnt; i < cnt + (8 - last % 8) % 8; ++i) q[da.n + i] = (T)0.0f;
                } else {
                    store8(q, 8, true, d);
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
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) s += red[w][tid];
            const int c = blockIdx.x * 256 + tid;
            if (c < da.n) da.sums[(int64_t)blockIdx.y * da.sums_ld + (h ? da.n : 0) + c] = s;
        }
    }
}

// bias gradient: the row blocks' sums added up in order
template <typename T>
__global__ __launch_bounds__(256) void k_sum(const SumArgs sa) {
    __shared__ float red[8][33];
    const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + cx, total = sa.n;
    float s = 0.f;
    if (c < total)
        for (int i = ry; i < sa.row_blocks; i += 8) s += sa.sums[(int64_t)i * sa.sums_ld + c];
    red[ry][cx] = s;
    __syncthreads();
    if (ry == 0 && c < total) {
        s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += red[w][cx];
        static_cast<T*>(sa.out)[c] = (T)s;
    }
}

// y = drop(x) + residual, eight columns a thread
template <typename T>
__global__ __launch_bounds__(256) void k_drop(const DropArgs da) {
    const int64_t chunks = ((int64_t)da.cols + 7) / 8, total = chunks * da.rows;
    const uint64_t offset = full_offset(da.offset, da.d_offset);
    for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (int64_t)gridDim.x * 256) {
        const int64_t row = idx / chunks;
        const int col = (int)(idx - row * chunks) * 8, cnt = da.cols - col;
        float s[8];
        load8(static_cast<const T*>(da.x) + row * da.ld_x + col, cnt, da.vec & 1, s);
        if (da.thr) {
            const uint32_t keep = keep_mask((uint32_t)(col >> 3), (uint32_t)row, da.seed, offset, da.thr);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = (keep >> i) & 1u ? s[i] * da.scale : 0.0f;
        }
        if (da.res) {
            float r[8];
            load8(static_cast<const T*>(da.res) + row * da.ld_res + col, cnt, da.vec & 4, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += r[i];
        }
        store8(static_cast<T*>(da.y) + row * da.ld_y + col, cnt, da.vec & 2, s);
    }
}

// ---- launches -----------------------------------------------------------------------------------
template <typename T, int LAY, int BM, int BN, int WM, int WN, bool AL, bool GT>
static hipError_t gemm_go(const GemmArgs& g, hipStream_t s) {
    k_gemm<T, LAY, BM, BN, WM, WN, AL, GT><<<dim3((unsigned)(g.tiles_m * g.tiles_n * g.split)), dim3(64 * WM * WN), 0, s>>>(g);
    return hipGetLastError();
}

template <typename T, int LAY, bool GT>
static hipError_t gemm_tile(const GemmArgs& g, int tile, bool aligned, hipStream_t s) {
    if (!aligned) return tile == 2 ? gemm_go<T, LAY, 64, 128, 2, 2, false, GT>(g, s) : gemm_go<T, LAY, 128, 128, 2, 2, false, GT>(g, s);
    if (tile == 0) return gemm_go<T, LAY, 256, 256, 2, 4, true, GT>(g, s);
    if (tile == 1) return gemm_go<T, LAY, 128, 128, 2, 2, true, GT>(g, s);
    return gemm_go<T, LAY, 64, 128, 2, 2, true, GT>(g, s);
}

template <typename T>
hipError_t DenseOps<T>::gemm(const GemmArgs& g, Layout lay, bool gated, int tile, bool aligned, hipStream_t s) {
    if (gated) return gemm_tile<T, L_KK, true>(g, tile, aligned, s);
    if (lay == L_KK) return gemm_tile<T, L_KK, false>(g, tile, aligned, s);
    if (lay == L_KT) return gemm_tile<T, L_KT, false>(g, tile, aligned, s);
    return gemm_tile<T, L_TT, false>(g, tile, aligned, s);
}

template <typename T>
hipError_t DenseOps<T>::skinny(const GemmArgs& g, bool gated, bool aligned, hipStream_t s) {
    const dim3 grid((unsigned)((g.N + 15) / 16)), block(64 * kSkinnyWaves);
    if (gated) {
        if (aligned) k_skinny<T, true, true><<<grid, block, 0, s>>>(g);
        else k_skinny<T, false, true><<<grid, block, 0, s>>>(g);
    } else {
        if (aligned) k_skinny<T, true, false><<<grid, block, 0, s>>>(g);
        else k_skinny<T, false, false><<<grid, block, 0, s>>>(g);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t DenseOps<T>::join(const JoinArgs& j, hipStream_t s) {
    const int64_t n = (int64_t)((j.e.n + 7) / 8) * j.M;
    const dim3 grid((unsigned)((n + 255) / 256));
    if (j.gated) k_join<T, true><<<grid, dim3(256), 0, s>>>(j);
    else k_join<T, false><<<grid, dim3(256), 0, s>>>(j);
    return hipGetLastError();
}

template <typename T>
hipError_t DenseOps<T>::dz(const DzArgs& d, hipStream_t s) {
    const dim3 grid((unsigned)((d.n + 255) / 256), (unsigned)d.row_blocks);
    if (d.gated) k_dz<T, true><<<grid, dim3(256), 0, s>>>(d);
    else k_dz<T, false><<<grid, dim3(256), 0, s>>>(d);
    return hipGetLastError();
}

template <typename T>
hipError_t DenseOps<T>::sum(const SumArgs& a, hipStream_t s) {
    k_sum<T><<<dim3((unsigned)((a.n + 31) / 32)), dim3(256), 0, s>>>(a);
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
