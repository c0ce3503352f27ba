#include "cct_internal.h"
extern "C" int cct_moe_workspace_bytes(const cct_moe_desc_t*, size_t*) { return CCT_EUNSUPPORTED; }
extern "C" int cct_moe_forward(const cct_moe_desc_t*, const void*, int64_t, const void*, int64_t, const void*, int64_t, int64_t, const void*, int64_t, int64_t, const void*, int64_t,
                    int64_t, const void*, int64_t, void*, int64_t, int32_t*, float*, void*, size_t, void*) { return CCT_EUNSUPPORTED; }
