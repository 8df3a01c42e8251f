// Rotary positions between the C entry points and their kernels.
#pragma once

#include "common.h"

namespace rs {

// Checks a call's rope and one of its parts (rope_api.cpp).
rs_status check_rope(const rs_rope *rope, int d);
rs_status check_rope_part(const rs_rope_part *p, int dtype, int d, int n, const char *what);

// Launches of calls whose arguments are checked (rope.hip).
struct CacheView;
rs_status rope_launch(const rs_rope &rope, const rs_rope_rows &rows, bool transpose, hipStream_t st);
rs_status append_rope_launch(const CacheView &c, int dtype, int d, const rs_rope &rope, const void *kn, const void *vn,
                             int64_t skt, int64_t skh, int64_t svt, int64_t svh, const rs_rope_part *q, const int32_t *pos,
                             const int32_t *start, int nrows, int max_rows, hipStream_t st);

}  // namespace rs
