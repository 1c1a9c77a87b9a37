#include "ops.h"
extern "C" dt_status dt_packed_attn(const dt_packed_config *, const void *, const int64_t *, const void *, const int64_t *, const void *, const int64_t *, const int32_t *,
                         const int32_t *, const int32_t *, const int32_t *, const int32_t *, const float *, const float *, void *, const int64_t *, float *, void *) {
    return dt::ops_fail(DT_ERR_UNSUPPORTED, "not yet");
}
