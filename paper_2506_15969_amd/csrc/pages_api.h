// What the two host files share.
#pragma once
#include "lazyev.h"

#include "kernels.h"

namespace lazyev {
// The arguments of an attention over these pages but for the pointers of the call; false: refused.
bool attend_args(const lazyev_pages *pages, int32_t length, int32_t n_tokens, int32_t n_q_heads, AttendArgs *a);
}  // namespace lazyev
