#include "dlc_gemm_impl.h"
namespace dlc { template struct DenseOps<f16_t>; }
