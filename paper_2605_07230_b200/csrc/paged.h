// Checks shared by the calls on the paged cache.
#pragma once
#include "cascade_internal.h"

// Status of a paged cache's host-side fields (pointers, alignment, strides, sizes) for this context.
int check_paged_cache(const cascade_ctx* ctx, const cascade_paged_cache* cache);
// Whether 32-bit arrays (null: not given) all start on 4-byte boundaries.
template <typename... P>
bool aligned4(const P*... p) {
  return ((... | reinterpret_cast<uintptr_t>(p)) & 3u) == 0;
}
// CASCADE_ERR_INVALID_ARG unless the context's device is the current one.
int check_current_device(const cascade_ctx* ctx);

// Bits of cascade_ctx.paged_configured.
enum : uint32_t { PAGED_CFG_TABLES = 1, PAGED_CFG_ATTN_TC = 2, PAGED_CFG_SAMPLE = 4, PAGED_CFG_SAMPLE_BF16 = 8 };
// Lets kernel `f` use `bytes` of dynamic shared memory, once per context and bit.
template <typename F>
int configure_smem(cascade_ctx* ctx, uint32_t bit, F* f, int bytes) {
  if (ctx->paged_configured & bit) return CASCADE_OK;
  CASCADE_CUDA_TRY(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  ctx->paged_configured |= bit;
  return CASCADE_OK;
}
