// The paged key-value cache's argument check, shared by the entry points that
// take one (include/mixfp4.h).
#pragma once
#include "mixfp4.h"

namespace mixfp4 {

int check_kv_cache(const mixfp4_kv_cache* c);

}  // namespace mixfp4
