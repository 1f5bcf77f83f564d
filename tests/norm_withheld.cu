// The norm's ring with copies that never come: bulk loads from an address range are not issued, so the wait for their row runs out.
// Built and driven by test_gpu_norm_withheld.py.
#include "dsn_transformer.cuh"

int dsn_pdl_enabled() { return 0; }

namespace {
__device__ uint64_t g_range[2];
__device__ __forceinline__ void load_unless_withheld(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  const uint64_t at = reinterpret_cast<uint64_t>(src);
  if (at < g_range[0] || at >= g_range[1]) dsn_bulk_load(dst, src, bytes, bar);
}
}  // namespace
#define dsn_bulk_load load_unless_withheld
#include "dsn_norm_quant.cu"

// One path, input order, residual; sum in place of x; q and scale may be NULL (the sum alone).  Returns a cudaError_t.
extern "C" int norm_withheld(void* x, const void* residual, int8_t* q, float* scale, int rows, int k, int ld, int f32, const void* from, const void* to,
                             const int32_t* offsets, const int32_t* perm, int32_t* status, int sm_count, void* stream) {
  const uint64_t range[2] = {reinterpret_cast<uint64_t>(from), reinterpret_cast<uint64_t>(to)};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaMemcpyToSymbolAsync(g_range, range, sizeof(range), 0, cudaMemcpyHostToDevice, s);
  if (e != cudaSuccess) return e;
  NormParams p;
  memset(&p, 0, sizeof(p));
  p.k[0] = (int16_t)k;
  p.R = 1; p.B = rows; p.G = 1; p.T = 1; p.max_k = k;
  p.by_R = dsn_fast_div(1);
  p.in_input_order = p.out_input_order = 1;
  p.offsets = offsets; p.perm = perm;
  p.x = x; p.residual = residual; p.sum = x; p.q = q; p.scale = scale;
  p.ldx = p.ld_res = p.ld_sum = p.ldq = p.ldy = ld;
  p.eps = 1e-6f; p.minus_zero = -0.0f; p.status = status;
  return dsn_launch_norm_quant(p, f32, sm_count, s);
}
