// Attention over a paged cache in mx4, queries in bf16.
#include <algorithm>

#include "mx4_attention_launch.h"

namespace mx4 {
int launch_attention_bf16(adadim_ctx* ctx, const Attention& a);
int launch_attention_bf16(adadim_ctx* ctx, const Attention& a) { return launch_attention<__bf16>(ctx, a); }
}  // namespace mx4
