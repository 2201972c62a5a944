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

}  // namespace ihip
