// The gated feed-forward block's products in IABN_BF16 (ffn_gemm.h).
#include "ffn_gemm.h"

namespace iabn_impl {
template bool launch_gemm<IABN_BF16>(GemmKind, const GemmArgs&, int, hipStream_t);
}  // namespace iabn_impl
