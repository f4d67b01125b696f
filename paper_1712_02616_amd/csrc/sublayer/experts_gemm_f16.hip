// The products of routed experts in IABN_F16 (experts_gemm.h).
#include "experts_gemm.h"

namespace iabn_impl {
template void launch_grouped<IABN_F16>(int, const GroupArgs&, int, hipStream_t);
template void launch_grouped_few<IABN_F16>(int, const GroupArgs&, hipStream_t);
}  // namespace iabn_impl
