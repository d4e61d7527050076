// The product of microscaled operands: arguments and the launches of each element type's source file.
#pragma once
#include "dlc_mx.h"

namespace dlc {

struct MxGemmArgs {
    GemmArgs c;           // lda, ldb in bytes, K in elements (filled rows)
    const uint8_t* xs;    // scales of x and of w
    const uint8_t* ws;
};

template <typename T>
struct MxOps {
    // tile: of kMxTileM (0: not with E4M3 and results in fp32) or kMxSkinny (bands of kMxSkinnyRows rows)
    static hipError_t gemm(const MxGemmArgs& g, int elem_x, int tile, hipStream_t s);
};

}  // namespace dlc
