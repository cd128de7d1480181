// Checks shared by the calls on the paged cache.
#pragma once
#include "cascade_internal.h"

// Status of a paged cache's host-side fields (pointers, alignment, strides, sizes) for this context.
int check_paged_cache(const cascade_ctx* ctx, const cascade_paged_cache* cache);
// CASCADE_ERR_INVALID_ARG unless the context's device is the current one.
int check_current_device(const cascade_ctx* ctx);
