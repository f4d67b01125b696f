// The gated feed-forward block for few tokens in IABN_BF16 (ffn_few.h).
#include "ffn_few.h"

namespace iabn_impl {
template bool launch_few<IABN_BF16>(GemmKind, const GemmArgs&, hipStream_t);
}  // namespace iabn_impl
