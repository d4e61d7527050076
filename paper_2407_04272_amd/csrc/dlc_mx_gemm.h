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
    static hipError_t gemm(const MxGemmArgs& g, int elem_x, hipStream_t s);
};

}  // namespace dlc
