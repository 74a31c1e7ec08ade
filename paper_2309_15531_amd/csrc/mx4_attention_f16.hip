// Attention over a paged cache in mx4, queries in f16.
#include <algorithm>

#include "mx4_attention_launch.h"

namespace mx4 {
int launch_attention_f16(adadim_ctx* ctx, const Attention& a);
int launch_attention_f16(adadim_ctx* ctx, const Attention& a) { return launch_attention<_Float16>(ctx, a); }
}  // namespace mx4
