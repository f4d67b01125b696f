// The gated feed-forward block for few tokens in IABN_F32 (ffn_few.h).
#include "ffn_few.h"

namespace iabn_impl {
template bool launch_few<IABN_F32>(GemmKind, const GemmArgs&, hipStream_t);
}  // namespace iabn_impl
