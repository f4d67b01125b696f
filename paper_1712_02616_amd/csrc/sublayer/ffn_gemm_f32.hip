// The gated feed-forward block's products in IABN_F32 (ffn_gemm.h).
#include "ffn_gemm.h"

namespace iabn_impl {
template bool launch_gemm<IABN_F32>(GemmKind, const GemmArgs&, int, hipStream_t);
}  // namespace iabn_impl
