#include "dlc_mx_impl.h"
namespace dlc { template struct MxOps<bf16_t>; }
