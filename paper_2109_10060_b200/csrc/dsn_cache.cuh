// Parameters and launchers of the 4-bit cache: plan and write (dsn_cache.cu), attention over the pages (dsn_cache_attention.cu).
#pragma once

#include "dsn_transformer.cuh"

// Bytes of a block of 16 tokens in one head, per group of 64 elements: k codes, k pairs, v codes, v pairs.
#define DSN_CACHE_BLOCK 16
__host__ __device__ constexpr uint32_t dsn_cache_block_bytes(int D) { return 18u * (uint32_t)D; }

// The window as the kernels get it.  One that reaches over all tokens a request can hold hides nothing: 0, so that windows are below 2^30 there and their
// difference to a token's number, which is above -2^24 (rows in front of a request's first token), stays in 32 bits.
__host__ __device__ constexpr int32_t dsn_cache_window(int32_t window, int32_t max_pages, int32_t page) {
  return window >= (int64_t)max_pages * page ? 0 : window;
}
// First token that token `me` sees.
__host__ __device__ constexpr int32_t dsn_cache_first_seen(int32_t me, int32_t window) { return window && me - window + 1 > 0 ? me - window + 1 : 0; }

struct CachePlanParams {
  int32_t B, R, page, n_pages, max_pages;
  FastDiv by_page, by_R;
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
  int32_t B, R, H, D, group, G, T, page, max_heads, grouped, split;   // split: warps a row
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
cudaError_t dsn_launch_cache_write(CacheWriteParams& p, int sm_count, cudaStream_t s);

// A request of the line of steps.
struct __align__(16) CacheEntry {
  int64_t first;       // its first step in the line
  int32_t sample, pos;
  int32_t heads, steps, len, rows;
};
// What a warp (in shared memory) or a CTA (in the workspace) has to say about the items at the ends of its stretch.
struct __align__(16) CachePart {
  int32_t head_state;  // 0: the stretch begins with an item of its own; 1: an earlier one's item ends here; 2: all of it lies inside one item; 3: it is empty
  int32_t tail;        // 1: its last item began here and goes on
  int32_t sample, pos, head, rows;   // of that last item
  int32_t head_far;    // (warp) the first item's part went through the workspace and lies behind the last one's in the ring
  int32_t pad;
};

struct CacheAttParams {
  int16_t heads[DSN_MAX_SLICES];
  int32_t B, R, H, group, G, T, page, n_pages, max_pages, max_heads, grouped, window;
  float scale_log2;     // scale of the scores times log2(e)
  FastDiv by_page, by_group;
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
  // in the workspace
  CachePart* parts;      // [CTAs]
  CacheEntry* list;      // [B]
  float* warp_data;
  float* cta_data;
};
#define DSN_CACHE_MAX_CTAS 148   // a B200's SMs: the workspace query has no context to ask
// Query vectors of a head (rows * group) up to which the form for a few of them runs.  It reads the cache once for every 16, the many-rows form turns it into
// fp16 tiles once for 256: 64 requests of up to 8192 tokens, 8 heads of 128: 121 us for 8, 185 for 16, 340 for 20 (442 in the many-rows form), 463 in that form for 64.
#define DSN_CACHE_FEW 32
size_t dsn_cache_attention_ws_bytes(int D, int cols, int64_t B);
cudaError_t dsn_launch_cache_attention(CacheAttParams& p, int D, int sm_count, void* workspace, cudaStream_t s);
size_t dsn_cache_rows_ws_bytes(int D, int64_t B);
cudaError_t dsn_launch_cache_attention_rows(CacheAttParams& p, int D, int sm_count, void* workspace, cudaStream_t s);
