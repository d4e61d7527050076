#include "dlc_mx_impl.h"
namespace dlc { template struct MxOps<float>; }
