#include "dlc_gemm_impl.h"
namespace dlc { template struct DenseOps<bf16_t>; }
