// The many-rows attention with copies that never come: bulk loads from an address range are not issued, so the wait for their tile runs out; and what the
// loader waits for before its CTA ends is noted.  Built and driven by test_gpu_cache_withheld.py.
#include <string.h>

#include "dsn_cache_line.cuh"

int dsn_pdl_enabled() { return 0; }

namespace {
__device__ uint64_t g_range[2];
__device__ int g_drain[DSN_CACHE_MAX_CTAS][2];
__device__ __forceinline__ void load_unless_withheld(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  const uint64_t at = reinterpret_cast<uint64_t>(src);
  if (at < g_range[0] || at >= g_range[1]) dsn_bulk_load(dst, src, bytes, bar);
}
__device__ __forceinline__ void drain_noted(uint32_t bars, int depth, int first, int asked) {
  if ((threadIdx.x & 31) == 0) g_drain[blockIdx.x][0] = first, g_drain[blockIdx.x][1] = asked;
  dsn_drain(bars, depth, first, asked);
}
__device__ int g_ended[DSN_CACHE_MAX_CTAS];
__device__ __forceinline__ void products_noted(uint32_t bar) {
  const bool ok = dsn_q4::products_end(bar);
  if ((threadIdx.x & 31) == 0) atomicAdd(&g_ended[blockIdx.x], ok ? 1 : 100);
}
}  // namespace
#define products_end products_noted
#define dsn_bulk_load load_unless_withheld
#define dsn_drain drain_noted
#include "dsn_cache_attention_rows.cu"

// One request of one path and one head of 64, pages of 64 tokens in a row; drain: host [148][2], -1 where a CTA waited for nothing.
// ended: host [148], warps of a CTA whose products had ended when they left early (100: had not).  Returns a cudaError_t.
extern "C" int cache_rows_withheld(const void* qkv, void* out, const uint8_t* pages, const int32_t* table, const int32_t* lengths, const int32_t* offsets, const int32_t* perm,
                                   int rows, int n_pages, const void* from, const void* to, int32_t* status, int sm_count, void* workspace, int32_t* drain, int32_t* ended) {
  const uint64_t range[2] = {reinterpret_cast<uint64_t>(from), reinterpret_cast<uint64_t>(to)};
  cudaError_t e = cudaMemcpyToSymbol(g_range, range, sizeof(range));
  memset(drain, 0xff, sizeof(g_drain));
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_drain, drain, sizeof(g_drain));
  memset(ended, 0, sizeof(g_ended));
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_ended, ended, sizeof(g_ended));
  if (e != cudaSuccess) return e;
  CacheAttParams p;
  memset(&p, 0, sizeof(p));
  p.heads[0] = 1;
  p.B = 1; p.R = rows; p.H = 1; p.group = 1; p.G = 1; p.T = 1; p.page = 64; p.n_pages = n_pages; p.max_pages = n_pages; p.max_heads = 1;
  p.scale_log2 = 0.125f * 1.44269504f;
  p.by_page = dsn_fast_div(64); p.by_group = dsn_fast_div(1);
  p.offsets = offsets; p.perm = perm; p.table = table; p.lengths = lengths; p.pages = pages; p.status = status;
  p.qkv = static_cast<const __nv_bfloat16*>(qkv); p.ld_qkv = 192;
  p.out = static_cast<__nv_bfloat16*>(out); p.ld_out = 64;
  e = dsn_launch_cache_attention_rows(p, 64, sm_count, workspace, nullptr);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(drain, g_drain, sizeof(g_drain));
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(ended, g_ended, sizeof(g_ended));
  return e;
}
extern "C" long cache_rows_ws_bytes() { return (long)dsn_cache_rows_ws_bytes(64, 1); }
