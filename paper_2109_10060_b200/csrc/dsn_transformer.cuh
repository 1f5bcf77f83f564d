// Parameters and launchers of the 8-bit transformer operators: residual + norm + codes (dsn_norm_quant.cu),
// linear layers on codes (dsn_gemm_i8_pair.cu, dsn_rows_i8.cu), rotary positions (dsn_rotary.cu).
#pragma once

#include "dsn_gemm_device.cuh"
#include "dsn_internal.cuh"

// Bounded wait that polls for a while before it takes the library's slow path: that one starts with a read of the wait limit from
// global memory and of the global timer, a microsecond that a wait for the next row or tile should not cost.
__device__ __forceinline__ bool dsn_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, int32_t* status, int where) {
#pragma unroll 1
  for (int i = 0; i < 64; ++i)
    if (dsn_gemm::mbar_try_wait(bar, parity)) return true;
  return dsn_gemm::mbar_wait_slow(bar, parity, abort_flag, status, where);
}

// After a wait that ran out: the copies that a group asked for, units first .. asked - 1 of its ring of `depth` barriers, get a last bounded
// chance to land before the group's shared memory goes to another CTA.
__device__ __forceinline__ void dsn_drain(uint32_t bars, int depth, int first, int asked) {
  for (int i = first; i < asked; ++i)
    for (int j = 0; j < (1 << 14) && !dsn_gemm::mbar_try_wait(bars + 8u * (uint32_t)(i % depth), (uint32_t)(i / depth) & 1u); ++j) {}
}

// Quotient of n < 2^31 by a divisor fixed on the host: (umulhi(n, mul) + n) >> shift.
struct FastDiv {
  uint32_t mul, shift, d;
};
inline FastDiv dsn_fast_div(uint32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  return FastDiv{(uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1), l, d};
}
__device__ __forceinline__ uint32_t dsn_div(uint32_t n, const FastDiv& f) { return (__umulhi(n, f.mul) + n) >> f.shift; }

// Where a grouped position lies: its sample and the slice of its group.  Up to 32 groups take one load per lane, more
// a binary search.  All lanes of the warp call this with the same arguments; slice < 0: no work at this position.
struct PosInfo {
  int sample;
  int slice;
};
__device__ __forceinline__ PosInfo dsn_locate_warp(int p, int G, int T, const int32_t* __restrict__ offsets,
                                                   const int32_t* __restrict__ perm, const int32_t* __restrict__ group_slice) {
  const int lane = threadIdx.x & 31;
  int g;
  if (G <= 32) {
    const int end = lane < G ? offsets[lane + 1] : 0x7fffffff;
    g = __popc(__ballot_sync(0xffffffffu, end <= p));   // groups that end at or before p, empty ones among them
  } else {
    if (p >= offsets[G]) return PosInfo{0, -1};
    int lo = 0, hi = G;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (offsets[mid] <= p) lo = mid; else hi = mid;
    }
    g = lo;
  }
  if (g >= G) return PosInfo{0, -1};
  PosInfo i;
  i.sample = perm[p];
  i.slice = group_slice ? group_slice[g] : g;
  if (i.sample < 0 || i.slice >= T) i.slice = -1;
  return i;
}

// The same for one thread on its own.
__device__ __forceinline__ PosInfo dsn_locate(int p, int G, int T, const int32_t* __restrict__ offsets, const int32_t* __restrict__ perm,
                                              const int32_t* __restrict__ group_slice) {
  if (p >= offsets[G]) return PosInfo{0, -1};
  int lo = 0, hi = G;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= p) lo = mid; else hi = mid;
  }
  PosInfo i;
  i.sample = perm[p];
  i.slice = group_slice ? group_slice[lo] : lo;
  if (i.sample < 0 || i.slice >= T) i.slice = -1;
  return i;
}

// Every lane a position of its own (p < B, or not below 0 and past the end of all groups); all lanes of the warp call this.  One trip to memory for
// up to 32 groups, whose ends go round the warp, instead of one a step of a search.
__device__ __forceinline__ PosInfo dsn_locate_lanes(int p, int B, int G, int T, const int32_t* __restrict__ offsets, const int32_t* __restrict__ perm,
                                                    const int32_t* __restrict__ group_slice) {
  if (G > 32) return p < B ? dsn_locate(p, G, T, offsets, perm, group_slice) : PosInfo{0, -1};
  const int lane = threadIdx.x & 31;
  const int end = lane < G ? offsets[lane + 1] : 0x7fffffff;
  const int slice = lane < G ? (group_slice ? group_slice[lane] : lane) : -1;
  PosInfo i;
  i.sample = p < B ? perm[p] : -1;
  int g = 0;
  for (int j = 0; j < G; ++j) g += __shfl_sync(0xffffffffu, end, j) <= p;
  i.slice = __shfl_sync(0xffffffffu, slice, g & 31);
  if (g >= G || i.sample < 0 || i.slice >= T) i.slice = -1;
  return i;
}

// Untiled bulk copies between global and shared memory: both ends on 16 bytes, whole 16 bytes.
__device__ __forceinline__ void dsn_bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void dsn_bulk_store(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(reinterpret_cast<uint64_t>(dst)), "r"(src), "r"(bytes)
               : "memory");
}
// Barrier `id` of `n` threads (whole warps) that also tells all of them whether `ok` holds in every one.
__device__ __forceinline__ bool dsn_group_all(bool ok, int id, int n) {
  int all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbar.red.and.pred q, %2, %3, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
               : "=r"(all)
               : "r"((int)ok), "r"(id), "r"(n)
               : "memory");
  return all != 0;
}
// Resident CTAs per SM of a kernel form on the current device, asked once.
template <typename K>
inline cudaError_t dsn_ctas_per_sm(K kernel, int threads, size_t smem, int* per_device /* [DSN_MAX_DEVICES] */, int* out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= DSN_MAX_DEVICES) return cudaErrorInvalidDevice;
  if (per_device[dev] == 0) {
    int n = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem);
    if (e != cudaSuccess) return e;
    per_device[dev] = n > 0 ? n : 1;
  }
  *out = per_device[dev];
  return cudaSuccess;
}

struct NormParams {
  int16_t k[DSN_MAX_SLICES];
  int32_t R, B, G, T, max_k;
  FastDiv by_R;
  int32_t in_input_order, out_input_order;
  const int32_t* offsets;
  const int32_t* perm;
  const int32_t* group_slice;
  const void* x;
  const void* residual;
  void* sum;
  int8_t* q;
  float* scale;
  void* y;
  int64_t ldx, ld_res, ld_sum, ldq, ldy;
  const float* weight;
  float eps, minus_zero;
  int32_t* status;
};
cudaError_t dsn_launch_norm_quant(const NormParams& p, int f32, int sm_count, cudaStream_t s);

struct RotaryParams {
  uint64_t freq[128];   // turns per unit of position, in units of 2^-64
  uint8_t axis[128];
  int16_t heads[DSN_MAX_SLICES];
  int32_t N, D, vectors, rotated, pairs, n_axes, max_heads;
  FastDiv by_N;
  int32_t B, G, T, grouped;
  int32_t n_pos;        // rows of one axis of `positions`
  int32_t shared, interleaved, inverse, in_place, whole_rows;
  const int32_t* offsets;
  const int32_t* perm;
  const int32_t* group_slice;
  const int32_t* positions;
  const void* x;
  void* y;
  int64_t ldx, ldy;
  int32_t* status;
};
cudaError_t dsn_launch_rotary(const RotaryParams& p, int f32, int aligned, int sm_count, cudaStream_t s);

// 8-bit linear layer on CTA pairs: `g` as in the bf16 pair kernel (maps on bytes, 128 a chunk; y, residual of either type)
struct GemmI8Params {
  GemmParams g;
  const float* x_scale;   // one per row of x
  const float* w_scale;   // one per output channel
  int32_t scale_input_order;  // rows of x_scale by sample (else by grouped position)
  FastDiv by_R;
};
size_t dsn_gemm_i8_smem_bytes(int BN, int stages, int G);
cudaError_t dsn_launch_gemm_i8(const GemmI8Params& p, int f32, int clusters, size_t smem_bytes, cudaStream_t s);

// 8-bit linear layer of at most DSN_ROWS_I8_MAX rows in all
#define DSN_ROWS_I8_MAX 32
struct RowsI8Params {
  int16_t k_in[DSN_MAX_SLICES];
  int16_t k_out[DSN_MAX_SLICES];
  int32_t B, R, G, T, C_in, max_ki, max_ko;
  int32_t in_input_order, out_input_order;
  const int32_t* offsets;
  const int32_t* perm;
  const int32_t* group_slice;
  const int8_t* x;
  const float* x_scale;
  const int8_t* W;
  const float* w_scale;
  const float* bias;
  const float* bn_scale;
  const float* bn_shift;
  int32_t bn_ld, act;
  const void* residual;
  void* y;
  int64_t ldx, ldw, ldy;
};
cudaError_t dsn_launch_rows_i8(const RowsI8Params& p, int f32, cudaStream_t s);
// rows of x, in input order, to rows of `ld` bytes in grouped order
cudaError_t dsn_launch_gather_i8(const RowsI8Params& p, int8_t* dst, int64_t ld, cudaStream_t s);
