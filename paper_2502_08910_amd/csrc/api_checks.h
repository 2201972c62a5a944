// Argument checks that the entry points share (api.hip).
#pragma once

#include "common.h"

namespace ihip {

inline bool pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }

int32_t check_shape(const ihip_shape *s, const char *who);
int32_t check_tensor(const ihip_tensor &t, const char *who, const char *name);
int32_t check_tensor8(const ihip_tensor &t, const char *who, const char *name);      // strides in bytes
int32_t check_paged(const char *who, const ihip_shape *shape, const ihip_paged_kv *pg, KvFormat *fmt);
int32_t check_scales(const char *who, float k_scale, float v_scale);

// Not negative, and finite as a factor for powers of two.  0 becomes the smallest number there is: products times it are close to 0 as well
// (2^127 * 2^-149), and -infinity stays it.
inline int32_t check_sm_scale(const char *who, float sm_scale, float *log2_scale)
{
    const float s = sm_scale * 1.44269504088896340736f;
    if (!(sm_scale >= 0.0f) || s > 3.4028234e38f) return fail(IHIP_ERR_INVALID_ARG, "%s: sm_scale = %g", who, sm_scale);
    *log2_scale = s > 0.0f ? s : 0x1p-149f;
    return IHIP_OK;
}

}  // namespace ihip
