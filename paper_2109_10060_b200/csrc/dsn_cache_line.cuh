// The line of steps that the attention kernels over the 4-bit cache deal out: the steps of all (request, head) items, one request after the other,
// cut into equal stretches, one a CTA.  Every CTA scans the requests' lengths on its own and keeps the requests of its stretch.
#pragma once

#include <cuda_fp16.h>

#include "dsn_cache.cuh"

namespace dsn_q4 {

constexpr int kListSmem = 64;      // requests that a CTA keeps in shared memory; further ones are read from the workspace
constexpr float kLowest = -1e38f;  // reference before any score: finite, so that differences are

// One look at a barrier that may put the thread to sleep for up to 20 us until the phase ends: a warp that only looks again and again takes issue slots from
// those that work (a third of all instructions of the many-rows kernel).
__device__ __forceinline__ bool patient_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity), "r"(20000u)
      : "memory");
  return ok != 0;
}
// Bounded wait of a whole warp, whose lanes all get the same answer: a wait that runs out while the barrier completes must not part them.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, int32_t* status, int where) {
#pragma unroll 1
  for (int i = 0; i < 64; ++i)
    if (__all_sync(0xffffffffu, patient_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, dsn_gemm::mbar_wait_slow(bar, parity, abort_flag, status, where));
}

// After a wait that ran out: the products that this warp issued get a last bounded chance to end before the CTA gives TMEM and shared memory back.
__device__ __forceinline__ bool products_end(uint32_t bar) {
  if (dsn_gemm::elect_one()) dsn_gemm::umma_commit(bar);
  __syncwarp();
  for (int j = 0; j < (1 << 14); ++j)
    if (__all_sync(0xffffffffu, dsn_gemm::mbar_try_wait(bar, 0))) return true;
  return false;
}

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Codes as fp16 numbers, two at a time: 1024 + code from the low half of a byte in each 16 bits, 1024 + 16 code from its high half.  One instruction each as
// long as the 1024 is in a register: the compiler, which knows the constant, would rather spend a second instruction (304 -> 180 logic instructions for
// 32 tokens of 128 elements); hence a value that it cannot know.
__device__ __forceinline__ uint32_t opaque_1024() { return 0x64006400u | (threadIdx.x >> 16); }
__device__ __forceinline__ uint32_t low_codes(uint32_t w, uint32_t k1024) {
  uint32_t r;
  asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xEA;" : "=r"(r) : "r"(w), "r"(k1024));
  return r;
}
__device__ __forceinline__ uint32_t high_codes(uint32_t w, uint32_t k1024) {
  uint32_t r;
  asm("lop3.b32 %0, %1, 0x00f000f0, %2, 0xEA;" : "=r"(r) : "r"(w), "r"(k1024));
  return r;
}
__device__ __forceinline__ uint32_t code_of_low(uint32_t h) {   // code - 8
  const __half2 r = __hadd2(*reinterpret_cast<const __half2*>(&h), __float2half2_rn(-1032.f));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t code_of_high(uint32_t h) {
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&h), __float2half2_rn(0.0625f), __float2half2_rn(-72.f));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}

__device__ __forceinline__ void lds128(uint32_t a, uint32_t (&v)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(a));
}
__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Exclusive sums over the CTA of two numbers at once (s_warp: two numbers a warp).
template <int THREADS>
__device__ __forceinline__ void block_scan(uint64_t& v, uint32_t& w, uint64_t* s_warp, uint64_t& v_total, uint32_t& w_total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t incl = v;
  uint32_t count = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t u = __shfl_up_sync(0xffffffffu, (unsigned long long)incl, o);
    const uint32_t c = __shfl_up_sync(0xffffffffu, count, o);
    if (lane >= o) incl += u, count += c;
  }
  __syncthreads();
  if (lane == 31) s_warp[2 * warp] = incl, s_warp[2 * warp + 1] = count;
  __syncthreads();
  uint64_t before = 0;
  uint32_t before_w = 0;
  v_total = 0;
  w_total = 0;
#pragma unroll
  for (int k = 0; k < THREADS / 32; ++k) {
    const uint64_t u = s_warp[2 * k];
    const uint32_t c = (uint32_t)s_warp[2 * k + 1];
    if (k < warp) before += u, before_w += c;
    v_total += u;
    w_total += c;
  }
  v = before + incl - v;
  w = before_w + count - w;
}

// Where share i of n of a line of `total` begins: shares differ by one at most.
__device__ __forceinline__ uint64_t dsn_share(uint64_t total, uint32_t i, uint32_t n) {
  if (total >> 32) return total / n * i + min((uint64_t)i, total % n);
  const uint32_t t = (uint32_t)total, q = t / n, r = t - q * n;
  return (uint64_t)q * i + min(i, r);
}

// One request's place in the line: what it needs to know, the items it has (its heads, pieces(rows) times each) and how many steps each of them makes,
// steps(len, rows).
template <typename Steps, typename Pieces>
__device__ __forceinline__ CacheEntry look_up(const CacheAttParams& p, int pos, bool report, Steps steps, Pieces pieces) {
  const PosInfo at = dsn_locate_lanes(pos, p.B, p.G, p.T, p.offsets, p.perm, p.group_slice);
  CacheEntry e;
  e.first = 0;
  e.sample = at.sample; e.pos = pos; e.heads = 0; e.steps = 0; e.len = 0; e.rows = 0;
  if (pos >= p.B || at.slice < 0 || at.sample >= p.B) return e;
  const int most = p.max_pages * p.page;
  const int len = p.lengths[at.sample], rows = p.placed ? p.placed[at.sample] : p.R;
  e.len = min(max(len, 0), most);
  e.rows = min(max(rows, 0), p.R);
  if (report && (len != e.len || rows != e.rows)) dsn_set_status(p.status, DSN_ERR_BAD_INDEX, at.sample);
  if (e.rows == 0) return e;
  e.heads = p.heads[at.slice] * pieces(e.rows);
  e.steps = steps(e.len, e.rows);
  return e;
}

// The CTA's stretch A .. Z - 1 and the requests in it: number i of them in s_list[i], from kListSmem on in p.list[first_order + i].
struct Stretch {
  uint64_t A, Z;
  int first_order, count;
};
template <int THREADS, typename Steps, typename Pieces>
__device__ __forceinline__ Stretch find_stretch(const CacheAttParams& p, CacheEntry* s_list, uint64_t* s_scan, uint32_t workers, Steps steps, Pieces pieces) {
  __shared__ int s_first_order, s_count;
  const int tid = threadIdx.x;
  if (tid == 0) s_first_order = 0, s_count = 0;
  const CacheEntry e0 = look_up(p, tid, blockIdx.x == 0, steps, pieces);
  uint64_t sum0, first0 = (uint64_t)e0.heads * e0.steps;
  uint32_t ones0, order0 = e0.heads > 0;
  block_scan<THREADS>(first0, order0, s_scan, sum0, ones0);
  uint64_t total = sum0;
  for (int b = THREADS; b < p.B; b += THREADS) {
    const CacheEntry e = look_up(p, b + tid, blockIdx.x == 0, steps, pieces);
    uint64_t sum, first = (uint64_t)e.heads * e.steps;
    uint32_t ones, order = e.heads > 0;
    block_scan<THREADS>(first, order, s_scan, sum, ones);
    total += sum;
  }
  Stretch st;
  // a short line goes to as few CTAs as give each of their `workers` a step: what one CTA cuts it joins by itself
  const uint32_t in_use = total >= (uint64_t)gridDim.x * workers ? gridDim.x : max(1u, ((uint32_t)total + workers - 1) / workers);
  st.A = dsn_share(total, min(blockIdx.x, in_use), in_use);
  st.Z = dsn_share(total, min(blockIdx.x + 1, in_use), in_use);
  uint64_t at_first = 0;
  uint32_t at_order = 0;
  for (int b = 0; b < p.B; b += THREADS) {
    CacheEntry e = e0;
    uint64_t first = first0, sum = sum0;
    uint32_t order = order0, ones = ones0;
    if (b > 0) {
      e = look_up(p, b + tid, false, steps, pieces);
      first = (uint64_t)e.heads * e.steps;
      order = e.heads > 0;
      block_scan<THREADS>(first, order, s_scan, sum, ones);
      first += at_first;
      order += at_order;
    }
    at_first += sum;
    at_order += ones;
    const bool here = e.heads > 0 && first < st.Z && first + (uint64_t)e.heads * e.steps > st.A;
    if (here && first <= st.A) s_first_order = (int)order;   // one thread of all: the request that holds step A
    __syncthreads();
    if (here) {
      const int i = (int)order - s_first_order;
      e.first = (int64_t)first;
      if (i < kListSmem) s_list[i] = e; else p.list[order] = e;
      atomicMax(&s_count, i + 1);
    }
    __syncthreads();
  }
  st.first_order = s_first_order;
  st.count = s_count;
  return st;
}

}  // namespace dsn_q4
