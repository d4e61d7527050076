#include "dlc_mx_impl.h"
namespace dlc { template struct MxOps<f16_t>; }
