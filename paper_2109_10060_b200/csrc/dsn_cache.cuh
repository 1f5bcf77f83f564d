// Parameters and launchers of the 4-bit cache: plan and write (dsn_cache.cu), attention over the pages (dsn_cache_attention.cu).
#pragma once

#include "dsn_transformer.cuh"

// Bytes of a block of 16 tokens in one head, per group of 64 elements: k codes, k pairs, v codes, v pairs.
#define DSN_CACHE_BLOCK 16
__host__ __device__ constexpr uint32_t dsn_cache_block_bytes(int D) { return 18u * (uint32_t)D; }

struct CachePlanParams {
  int32_t B, R, page, n_pages, max_pages;
  FastDiv by_page;
  const int32_t* new_tokens;
  const int32_t* lengths;
  const int32_t* pool_state;
  int32_t* lengths_out;
  int32_t* pool_state_out;
  int32_t* table;
  int32_t* placed;
  int32_t* slots;
  int32_t* pool;
  int32_t* status;
};
cudaError_t dsn_launch_cache_plan(const CachePlanParams& p, cudaStream_t s);
cudaError_t dsn_launch_cache_reset(int32_t B, int32_t n_pages, int32_t* lengths, int32_t* pool, int32_t* pool_state, cudaStream_t s);

struct CacheWriteParams {
  int16_t heads[DSN_MAX_SLICES];
  int32_t B, R, H, D, group, G, T, page, max_heads, grouped;
  int64_t n_slots;      // tokens that the pages hold
  FastDiv by_R, by_page;
  const int32_t* offsets;
  const int32_t* perm;
  const int32_t* group_slice;
  const int32_t* slots;
  const __nv_bfloat16* qkv;
  int64_t ld_qkv;
  __nv_bfloat16* values;
  int64_t ld_values;
  uint8_t* pages;
  int32_t* status;
};
cudaError_t dsn_launch_cache_write(const CacheWriteParams& p, int sm_count, cudaStream_t s);

struct CacheAttParams {
  int16_t heads[DSN_MAX_SLICES];
  int32_t B, R, H, group, G, T, page, n_pages, max_pages, max_heads, grouped, window;
  float scale_log2;     // scale of the scores times log2(e)
  FastDiv by_page;
  const int32_t* offsets;
  const int32_t* perm;
  const int32_t* group_slice;
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* placed;   // or nullptr: R rows each
  const __nv_bfloat16* qkv;
  int64_t ld_qkv;
  __nv_bfloat16* out;
  int64_t ld_out;
  const uint8_t* pages;
  int32_t* status;
};
cudaError_t dsn_launch_cache_attention(const CacheAttParams& p, int D, int sm_count, cudaStream_t s);
