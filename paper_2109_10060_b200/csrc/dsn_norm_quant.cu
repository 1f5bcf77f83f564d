// Residual addition, root-mean-square norm on elastic widths and 8-bit codes with a scale per row, in one pass:
//   h = x + residual;  n = h / sqrt(mean h^2 + eps) * w;  s = max|n| / 127;  q = round(h w * (127 * (1 / max|h w|))).
// The factor 1 / sqrt(...) is common to a row, so it drops out of the code: the sum of squares and the maximum of |h w|
// come out of ONE reduction, and the codes do not depend on the order of the sum.
// Bound by memory, once the bytes in flight do not depend on the registers of the threads that work and the instructions per element are
// few.  Ring form: a group of 16 .. 256 threads has a ring of shared-memory slots of its own, which bulk copies fill with the rows to
// come (rows are looked up 32 at a time, one a lane); it takes a row into registers, eight columns a thread and step, asks for the row
// that goes into the free slot, and works two columns an instruction.  (One fetching warp for all groups was the bottleneck
// of short rows: 59 us on 50,432 rows of 384 columns.)  The weights of a thread's columns stay in its registers.  Direct form
// (few rows, where the ring's start-up is longer than the rows; rows too long for a ring): the same arithmetic on rows read
// straight into registers.

#include "dsn_transformer.cuh"

namespace {

using dsn_gemm::fadd2;
using dsn_gemm::ffma2;
using dsn_gemm::pack2;
using dsn_gemm::unpack2;

__device__ __forceinline__ uint64_t fmul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_abs3_nan(float m, uint64_t v2) {
  float a, b, r;
  unpack2(v2, a, b);
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(fabsf(a)), "f"(fabsf(b)));
  return r;
}

// Eight columns as four pairs of fp32.
template <bool F32>
struct Elem;
template <>
struct Elem<false> {
  typedef __nv_bfloat16 type;
  static __device__ __forceinline__ void load(const type* p, uint64_t (&v)[4]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ void store(type* p, const uint64_t (&v)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      unpack2(v[i], a, b);
      __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
      w[i] = *reinterpret_cast<uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float load1(const type* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void store1(type* p, float v) { *p = __float2bfloat16_rn(v); }
};
template <>
struct Elem<true> {
  typedef float type;
  static __device__ __forceinline__ void load(const type* p, uint64_t (&v)[4]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = pack2(a.x, a.y); v[1] = pack2(a.z, a.w); v[2] = pack2(b.x, b.y); v[3] = pack2(b.z, b.w);
  }
  static __device__ __forceinline__ void store(type* p, const uint64_t (&v)[4]) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(v[i], f[2 * i], f[2 * i + 1]);
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
  static __device__ __forceinline__ float load1(const type* p) { return *p; }
  static __device__ __forceinline__ void store1(type* p, float v) { *p = v; }
};
// A step of which only the first n columns belong to the row (n < 8, none or fewer than none included).
template <bool F32>
__device__ __forceinline__ void load_part(const typename Elem<F32>::type* p, const typename Elem<F32>::type* res, int n, uint64_t (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = 0.f, b = 0.f;
    if (2 * i < n) a = Elem<F32>::load1(p + 2 * i) + (res ? Elem<F32>::load1(res + 2 * i) : 0.f);
    if (2 * i + 1 < n) b = Elem<F32>::load1(p + 2 * i + 1) + (res ? Elem<F32>::load1(res + 2 * i + 1) : 0.f);
    v[i] = pack2(a, b);
  }
}
template <bool F32>
__device__ __forceinline__ void store_part(typename Elem<F32>::type* p, int n, const uint64_t (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    unpack2(v[i], a, b);
    if (2 * i < n) Elem<F32>::store1(p + 2 * i, a);
    if (2 * i + 1 < n) Elem<F32>::store1(p + 2 * i + 1, b);
  }
}

struct RowAt {
  int k;             // 0: no such row
  int part;          // the bytes behind the last whole 16 are not in shared memory
  int64_t in, out;   // row numbers
};
__device__ __forceinline__ RowAt locate_row(const NormParams& p, uint32_t row) {
  const int pos = (int)dsn_div(row, p.by_R), r = (int)(row - (uint32_t)pos * (uint32_t)p.R);
  RowAt a{0, 0, 0, 0};
  if (pos < p.B) {
    const PosInfo at = dsn_locate_warp(pos, p.G, p.T, p.offsets, p.perm, p.group_slice);
    if (at.slice >= 0) {
      a.k = p.k[at.slice];
      a.in = (int64_t)(p.in_input_order ? at.sample : pos) * p.R + r;
      a.out = (int64_t)(p.out_input_order ? at.sample : pos) * p.R + r;
    }
  }
  return a;
}

// (sum, maximum) over the TPR threads of a row, and whether `ok` holds in all of them: a group with its own named barrier `id` where
// it is more than a warp.  `part` holds two sets of one entry a warp, taken in turn: one barrier a call is enough then.
template <int TPR>
__device__ __forceinline__ bool row_reduce(float& ss, float& mx, float2* part, int& turn, int id, bool ok) {
#pragma unroll
  for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) {
    ss += __shfl_xor_sync(0xffffffffu, ss, o);
    mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  }
  if constexpr (TPR > 32) {
    constexpr int NW = TPR / 32;
    float2* mine = part + turn * NW;
    if ((threadIdx.x & 31) == 0) mine[(threadIdx.x >> 5) % NW] = make_float2(ss, mx);
    ok = dsn_group_all(ok, id, TPR);
    ss = 0.f;
    mx = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float2 v = mine[i];
      ss += v.x;
      mx = max_nan(mx, v.y);
    }
    turn ^= 1;
    return ok;
  }
  return (bool)__all_sync(0xffffffffu, ok);
}

template <int TPR, int VPT>
__device__ __forceinline__ void load_weights(const NormParams& p, int t, uint64_t (&w)[VPT][4]) {
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int c = 8 * (t + j * TPR);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[j][i] = pack2(1.f, 1.f);
    if (p.weight) {
      if (c + 8 <= p.max_k) Elem<true>::load(p.weight + c, w[j]);
      else if (c < p.max_k) load_part<true>(p.weight + c, nullptr, p.max_k - c, w[j]);
    }
  }
}

constexpr float kSmallMax = 7.52316385e-37f;   // 2^-120: 127 / a maximum below it would leave fp32

// A row that lies in the registers of its TPR threads (h, zero at and beyond k) -> everything that is written for it.  False where `ok`
// does not hold in all threads of the row (those have k = 0: what precedes the agreement, the stream, is stored by threads with ok alone); then
// they all leave.  When it returns, all of them have the row in registers.
template <bool F32, int TPR, int VPT>
__device__ __forceinline__ bool finish_row(const NormParams& p, const RowAt& cur, int t, uint64_t (&h)[VPT][4], const uint64_t (&w)[VPT][4], float2* part,
                                           int& turn, int id, bool ok) {
  typedef Elem<F32> E;
  typedef typename E::type elem;
  const int k = cur.k;
  // product with the weights; columns at and beyond k count as zero whatever the weight there
  auto product = [&](int j, uint64_t (&v)[4]) {
    const int c = 8 * (t + j * TPR);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fmul2(h[j][i], w[j][i]);
    if (c + 8 > k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a, b;
        unpack2(v[i], a, b);
        v[i] = pack2(c + 2 * i < k ? a : 0.f, c + 2 * i + 1 < k ? b : 0.f);
      }
    }
  };
  float ss, mx;
  auto measure = [&]() {
    uint64_t s2 = 0ull;
    mx = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      uint64_t v[4];
      product(j, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s2 = ffma2(h[j][i], h[j][i], s2);
        mx = max_abs3_nan(mx, v[i]);
      }
    }
    float a, b;
    unpack2(s2, a, b);
    ss = a + b;
    ok = row_reduce<TPR>(ss, mx, part, turn, id, ok);
  };
  if (p.sum) {
    elem* d = static_cast<elem*>(p.sum) + cur.in * p.ld_sum;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = 8 * (t + j * TPR);
      if (c + 8 <= k) E::store(d + c, h[j]);
      else if (c < k) store_part<F32>(d + c, k - c, h[j]);
    }
    if (!p.q && !p.y) return TPR > 32 ? dsn_group_all(ok, id, TPR) : (bool)__all_sync(0xffffffffu, ok);
  }
  measure();
  if (!ok) return false;
  // n = h w rs.  Where the squares (or a product with the weight) left the range of fp32, 127 / max would, or the row holds something
  // that is no number, the row is looked at again (rare; the same decision in all threads of the row).
  const float rk = __fdividef(1.f, (float)k);
  float rs = rsqrtf(ss * rk + p.eps);
  const bool redo = !(ss < INFINITY) || !(mx < INFINITY) || (mx < kSmallMax && mx > 0.f);
  if (TPR < 32 ? __any_sync(0xffffffffu, redo) : redo) {
    const float ss1 = ss;
    float top = 0.f, none = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max_abs3_nan(top, h[j][i]);
    row_reduce<TPR>(none, top, part, turn, id, true);
    // h times a power of two (exact; what underflows is below 2^-120 of the row's largest value), so that its largest is 1 .. 4
    float f = 1.f;
    if (redo && top < INFINITY && top > 0.f) {
      const int e = (int)(__float_as_uint(top) >> 23);
      f = __uint_as_float((uint32_t)(e > 252 ? 1 : (e < 1 ? 253 : 254 - e)) << 23);
    }
    auto scale_row = [&](float f) {
      const uint64_t f2 = pack2(f, f);
#pragma unroll
      for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) h[j][i] = fmul2(h[j][i], f2);
      measure();
    };
    scale_row(f);
    if (f < 1.f) rs = rsqrtf(ss * rk + p.eps * f * f);
    else if (f > 1.f) rs = rsqrtf(ss1 * rk + p.eps) / f;               // eps outweighs squares this small
    // Weights that take a row of this size out of the range: another power of two, of which the sum of squares knows nothing.  (As a loop of two
    // rounds this block cost the rows that never come here: 37 x 121 rows of 1000 fp32 columns 9.4 -> 9.9 us.)
    f = !redo || !(top < INFINITY) ? 1.f : (mx < kSmallMax && mx > 0.f ? 0x1p100f : (mx == INFINITY ? 0x1p-8f : 1.f));
    if (TPR < 32 ? __any_sync(0xffffffffu, f != 1.f) : f != 1.f) {
      scale_row(f);
      rs *= 1.f / f;
    }
    if (!(top < INFINITY)) mx = __uint_as_float(0x7fffffffu);          // NaN or infinity in the row: NaN comes out
  }
  if (k == 0) return true;
  elem* y = p.y ? static_cast<elem*>(p.y) + cur.out * p.ldy : nullptr;
  if (p.q) {
    const float inv = mx > 0.f ? __fmul_rn(__frcp_rn(mx), 127.f) : mx;   // a row of zeros: 0; NaN stays
    const float scale = mx * rs * (1.f / 127.f);
    const uint32_t keep = mx < INFINITY ? 0xffffffffu : 0u;             // a row that is no number has the codes 0
    const uint64_t inv2 = pack2(inv, inv), scale2 = pack2(scale, scale);
    const uint64_t none = pack2(p.minus_zero, p.minus_zero);
    const uint64_t magic = pack2(12582912.f, 12582912.f), nmagic = pack2(-12582912.f, -12582912.f);
    int8_t* q = p.q + cur.out * p.ldq;
    if (t == 0) p.scale[cur.out] = scale;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = 8 * (t + j * TPR);
      if (c >= k) continue;
      uint64_t v[4];
      uint32_t b[8];
      product(j, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // The sum with 1.5 * 2^23 rounds to the nearest integer, ties to even, and leaves its low byte in the low byte.  The product in front
        // of it is rounded too, as the definition says: it is a fused one with a -0 that comes from the host, because the compiler joins a
        // packed product, or a fused one with a -0 that it can see, with the sum.
        const uint64_t m = fadd2(ffma2(v[i], inv2, none), magic);
        b[2 * i] = (uint32_t)m;
        b[2 * i + 1] = (uint32_t)(m >> 32);
        v[i] = fmul2(fadd2(m, nmagic), scale2);
      }
      const uint32_t lo = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410) & keep;
      const uint32_t hi = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410) & keep;
      if (c + 8 <= k) {
        *reinterpret_cast<uint2*>(q + c) = make_uint2(lo, hi);
        if (y) E::store(y + c, v);
      } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
          if (c + i < k) q[c + i] = (int8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
        if (y) store_part<F32>(y + c, k - c, v);
      }
    }
  } else {
    const float f = mx >= 0.f ? rs : mx;
    const uint64_t f2 = pack2(f, f);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = 8 * (t + j * TPR);
      if (c >= k) continue;
      uint64_t v[4];
      product(j, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = fmul2(v[i], f2);
      if (c + 8 <= k) E::store(y + c, v);
      else store_part<F32>(y + c, k - c, v);
    }
  }
  return true;
}

// Direct form: rows read straight into registers, TPR threads (at least a warp) a row.  Two CTAs of 512 threads an SM, which 68 registers would not
// allow (197 fp32 rows of up to 5140 columns with residual: 5.4 us, 6.9 with one).
template <bool F32, bool RES, int TPR, int VPT, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 512 ? 2 : 0) norm_quant_kernel(const __grid_constant__ NormParams p) {
  typedef Elem<F32> E;
  typedef typename E::type elem;
  __shared__ float2 part[TPR > 32 ? 2 * TPR / 32 : 1];
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  constexpr int RPC = THREADS / TPR;                     // more than one only where a row is a warp's
  const uint32_t rows = (uint32_t)p.B * (uint32_t)p.R;   // below 2^31
  const uint32_t stride = gridDim.x * RPC;
  const int t = threadIdx.x % TPR;
  uint32_t row = blockIdx.x * RPC + threadIdx.x / TPR;
  RowAt next = locate_row(p, row);
  uint64_t w[VPT][4];
  load_weights<TPR, VPT>(p, t, w);
  int turn = 0;
  for (; row < rows; row += stride) {
    const RowAt cur = next;
    const int k = cur.k;
    uint64_t h[VPT][4];
    const elem* x = static_cast<const elem*>(p.x) + cur.in * p.ldx;
    const elem* res = RES ? static_cast<const elem*>(p.residual) + cur.in * p.ld_res : nullptr;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = 8 * (t + j * TPR);
      if (c + 8 <= k) {
        E::load(x + c, h[j]);
        if (RES) {
          uint64_t b[4];
          E::load(res + c, b);
#pragma unroll
          for (int i = 0; i < 4; ++i) h[j][i] = fadd2(h[j][i], b[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) h[j][i] = 0ull;
        if (c < k) load_part<F32>(x + c, res ? res + c : nullptr, k - c, h[j]);
      }
    }
    next = locate_row(p, row + stride < rows ? row + stride : rows);
    finish_row<F32, TPR, VPT>(p, cur, t, h, w, part, turn, 0, true);
  }
}

// Ring form.
constexpr int kRingThreads = 256;
constexpr int kRingDepth = 8;               // most slots of a group

template <bool F32, bool RES, int TPR, int VPT>
__global__ void __launch_bounds__(kRingThreads, 2) norm_quant_ring_kernel(const __grid_constant__ NormParams p, int depth, uint32_t row_bytes) {
  typedef Elem<F32> E;
  typedef typename E::type elem;
  constexpr int RB = TPR < 32 ? 32 / TPR : 1;                       // rows a group (at least a warp) works on at once: a unit
  constexpr int GT = TPR < 32 ? 32 : TPR, GROUPS = kRingThreads / GT;
  constexpr int UB = 32 / RB;                                       // units that the lanes of a warp look up at once
  constexpr int ES = F32 ? 4 : 2;
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ uint64_t s_full[GROUPS][kRingDepth];
  __shared__ RowAt s_at[GROUPS][kRingDepth][RB];
  __shared__ float2 s_part[GROUPS][TPR > 32 ? 2 * TPR / 32 : 1];
  __shared__ uint32_t s_abort;
  const int g = threadIdx.x / GT, lane = threadIdx.x & 31;
  const int sub = TPR < 32 ? lane / TPR : 0, t = threadIdx.x % TPR;
  const bool fetches = (threadIdx.x % GT) < 32;                     // the group's first warp asks for rows
  if (threadIdx.x < GROUPS * kRingDepth) dsn_gemm::mbar_init(dsn_gemm::smem_u32(&s_full[0][0] + threadIdx.x), 1);
  if (threadIdx.x == 0) {
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const uint32_t rows = (uint32_t)p.B * (uint32_t)p.R, units = (rows + RB - 1) / RB;
  const uint32_t gid = blockIdx.x * GROUPS + g, ngroups = gridDim.x * GROUPS;
  const int mine = gid < units ? (int)((units - gid + ngroups - 1) / ngroups) : 0;   // units of this group
  const uint32_t copies = RES ? 2u : 1u, slot_bytes = RB * copies * row_bytes;
  uint8_t* slots = ring + (size_t)g * depth * slot_bytes;
  volatile uint32_t* abort_flag = &s_abort;

  RowAt ahead{0, 0, 0, 0};   // this lane's row of the units being asked for
  int asked = 0;             // units asked for
  auto ask = [&](int slot) {
    __syncwarp();            // the slot's former row has been taken by all lanes
    if (asked % UB == 0) {   // the next units' rows, one a lane
      ahead = RowAt{0, 0, 0, 0};
      const uint64_t wide = ((uint64_t)(asked + lane / RB) * ngroups + gid) * RB + lane % RB;
      const uint32_t row = wide < rows ? (uint32_t)wide : rows;   // rows / R = B: no position
      const int pos = (int)dsn_div(row, p.by_R), r = (int)(row - (uint32_t)pos * (uint32_t)p.R);
      const PosInfo at = dsn_locate_lanes(pos, p.B, p.G, p.T, p.offsets, p.perm, p.group_slice);
      if (at.slice >= 0) {
        ahead.k = p.k[at.slice];
        ahead.in = (int64_t)(p.in_input_order ? at.sample : pos) * p.R + r;
        ahead.out = (int64_t)(p.out_input_order ? at.sample : pos) * p.R + r;
        ahead.part = ahead.in + 1 == (int64_t)rows;   // behind the last row's columns nothing need be allocated
      }
      __syncwarp();
    }
    const uint32_t bytes = ahead.part ? (uint32_t)(ahead.k * ES) & ~15u : (uint32_t)(ahead.k * ES + 15) & ~15u;
    const bool turn_of = lane / RB == asked % UB;
    uint32_t all = bytes;
#pragma unroll
    for (int o = 1; o < RB; o <<= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    const uint32_t bar = dsn_gemm::smem_u32(&s_full[g][slot]);
    if (turn_of) {
      s_at[g][slot][lane % RB] = ahead;
      __threadfence_block();
    }
    if (RB > 1) __syncwarp();   // every row's place is written before the barrier can complete
    if (turn_of && lane % RB == 0) dsn_gemm::mbar_expect_tx(bar, copies * all);
    if (RB > 1) __syncwarp();
    if (turn_of && bytes) {
      const uint32_t dst = dsn_gemm::smem_u32(slots) + (uint32_t)slot * slot_bytes + (uint32_t)(lane % RB) * copies * row_bytes;
      dsn_bulk_load(dst, static_cast<const elem*>(p.x) + ahead.in * p.ldx, bytes, bar);
      if (RES) dsn_bulk_load(dst + row_bytes, static_cast<const elem*>(p.residual) + ahead.in * p.ld_res, bytes, bar);
    }
    ++asked;
  };
  if (fetches)
    for (int i = 0; i < depth && i < mine; ++i) ask(i);

  uint64_t w[VPT][4];
  load_weights<TPR, VPT>(p, t, w);
  int turn = 0, slot = 0;
  uint32_t phase = 0;
  int n = 0;
  for (; n < mine; ++n) {
    const bool ok = dsn_wait(dsn_gemm::smem_u32(&s_full[g][slot]), phase, abort_flag, p.status, 71);
    // a thread whose wait ran out has no row: its slot holds an earlier one, or nothing yet, and the stream may be written in place
    const RowAt cur = ok ? s_at[g][slot][sub] : RowAt{0, 0, 0, 0};
    const int k = cur.k;
    const elem* xs = reinterpret_cast<const elem*>(slots + (size_t)slot * slot_bytes + (size_t)sub * copies * row_bytes);
    const elem* rsd = reinterpret_cast<const elem*>(reinterpret_cast<const uint8_t*>(xs) + row_bytes);
    uint64_t h[VPT][4];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = 8 * (t + j * TPR);
#pragma unroll
      for (int i = 0; i < 4; ++i) h[j][i] = 0ull;
      if (c < k) {
        if (c + 8 <= k || !cur.part) {
          E::load(xs + c, h[j]);
          if (RES) {
            uint64_t b[4];
            E::load(rsd + c, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) h[j][i] = fadd2(h[j][i], b[i]);
          }
          if (c + 8 > k) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float a, b;
              unpack2(h[j][i], a, b);
              h[j][i] = pack2(c + 2 * i < k ? a : 0.f, c + 2 * i + 1 < k ? b : 0.f);
            }
          }
        } else {
          load_part<F32>(static_cast<const elem*>(p.x) + cur.in * p.ldx + c, RES ? static_cast<const elem*>(p.residual) + cur.in * p.ld_res + c : nullptr,
                         k - c, h[j]);
        }
      }
    }
    // a group leaves together when a wait ran out anywhere in it
    if (!finish_row<F32, TPR, VPT>(p, cur, t, h, w, s_part[g], turn, 1 + g, ok)) break;
    if (fetches && asked < mine) ask(slot);
    if (++slot == depth) { slot = 0; phase ^= 1u; }
  }
  if (fetches && n < mine) dsn_drain(dsn_gemm::smem_u32(&s_full[g][0]), depth, n, asked);
}

template <bool F32, bool RES, int TPR, int VPT>
cudaError_t launch(const NormParams& p, int sm_count, cudaStream_t s) {
  constexpr int THREADS = TPR > 32 ? TPR : 128;
  static int resident[DSN_MAX_DEVICES] = {};
  auto kernel = norm_quant_kernel<F32, RES, TPR, VPT, THREADS>;
  int n = 0;
  const cudaError_t e = dsn_ctas_per_sm(kernel, THREADS, 0, resident, &n);
  if (e != cudaSuccess) return e;
  const int64_t rows = (int64_t)p.B * p.R, ctas = (rows + THREADS / TPR - 1) / (THREADS / TPR), most = (int64_t)sm_count * n;
  return dsn_launch(kernel, dim3((unsigned)(ctas < most ? ctas : most)), dim3(THREADS), 0, s, 1, p);
}

// Rings of at most 64 KB a CTA (more bytes in flight only crowd the writes: 100.6 us at 96 KB, 78 against 81 us without y) where two CTAs
// share an SM, of up to 200 KB where one takes it alone (two slots of long rows).
template <bool F32, bool RES, int TPR, int VPT>
cudaError_t launch_ring(const NormParams& p, int sm_count, cudaStream_t s) {
  static size_t configured[DSN_MAX_DEVICES] = {};
  auto kernel = norm_quant_ring_kernel<F32, RES, TPR, VPT>;
  constexpr int RB = TPR < 32 ? 32 / TPR : 1, GROUPS = kRingThreads / (TPR < 32 ? 32 : TPR);
  const uint32_t row = (uint32_t)((p.max_k + 7) / 8 * (F32 ? 32 : 16));   // whole steps of eight columns
  const uint32_t one = GROUPS * RB * (RES ? 2u : 1u) * row;               // a slot of every group
  int per_sm = 2, depth = (int)(64 * 1024 / one);
  if (depth < 2) depth = (int)(96 * 1024 / one);
  if (depth < 2) {
    per_sm = 1;
    depth = (int)(200 * 1024 / one);
  }
  if (depth < 2) return cudaErrorInvalidConfiguration;
  if (depth > kRingDepth) depth = kRingDepth;
  const size_t smem = (size_t)depth * one;
  const cudaError_t e = dsn_ensure_dynamic_smem(kernel, smem, configured);
  if (e != cudaSuccess) return e;
  const int64_t units = ((int64_t)p.B * p.R + RB - 1) / RB, ctas = (units + GROUPS - 1) / GROUPS, most = (int64_t)sm_count * per_sm;
  return dsn_launch(kernel, dim3((unsigned)(ctas < most ? ctas : most)), dim3(kRingThreads), smem, s, 1, p, depth, row);
}

template <bool F32, bool RES>
cudaError_t pick(const NormParams& p, int sm_count, cudaStream_t s) {
  const int steps = (p.max_k + 7) / 8;
  const int64_t rows = (int64_t)p.B * p.R;
  // Rows beyond 8192 columns have the direct form alone, whose 32 weights and 32 columns a thread do not fit the registers (2000 rows bf16 with residual, codes
  // and stream: 8192 columns 25 us, 12,000 68, 30,000 131 against 17, 26, 64 for the bytes).
  // The ring's start-up costs a microsecond (us, ring and direct form, with residual and codes: 1024 rows of 4096 9.5, 8.5; 2400 of 4096 18.6, 20.0; 4800 of
  // 768 8.6, 8.7; 4800 of 384 6.0, 5.6).
  if (rows >= 8 * sm_count && rows * p.max_k >= 5 << 20 && steps <= 1024) {
    if (steps <= 16) return launch_ring<F32, RES, 16, 1>(p, sm_count, s);
    if (steps <= 32) return launch_ring<F32, RES, 16, 2>(p, sm_count, s);
    if (steps <= 48) return launch_ring<F32, RES, 16, 3>(p, sm_count, s);
    if (steps <= 96) return launch_ring<F32, RES, 32, 3>(p, sm_count, s);
    if (steps <= 128) return launch_ring<F32, RES, 32, 4>(p, sm_count, s);
    if (steps <= 256) return launch_ring<F32, RES, 64, 4>(p, sm_count, s);
    // 2056 .. 4096 columns, 128 or 256 threads a row (us with either).  bf16, 16,384 rows: where the stream and y are both written, memory bounds
    // the pass from some 3400 columns on and fewer rows being written at a time suit it better (3200 columns 78.0, 92.9; 3456 97.1, 94.8; 4096 113.5,
    // 95.9, without codes 98.9, 85.1); with less to write, the time a row takes from its wait to its stores does, and more rows do (4096 without the
    // stream 82.8, 89.0, without y 78.1, 91.8).  fp32, 8192 rows with residual, codes and y: with the stream either way within a tenth (2816: 72.9, 64.4;
    // 3584: 82.4, 90.9; 4096: 102.9, 105.2), without it 256 threads (3200: 71.7, 56.8; 4096: 76.8, 69.9).
    if (steps <= 512 && RES && p.y && (F32 ? p.q != nullptr : p.sum != nullptr && steps > 424)) return launch_ring<F32, RES, 256, 2>(p, sm_count, s);
    if (steps <= 512) return launch_ring<F32, RES, 128, 4>(p, sm_count, s);
    return launch_ring<F32, RES, 256, 4>(p, sm_count, s);
  }
  if (steps <= 32) return launch<F32, RES, 32, 1>(p, sm_count, s);
  if (steps <= 64) return launch<F32, RES, 32, 2>(p, sm_count, s);
  if (steps <= 128) return launch<F32, RES, 64, 2>(p, sm_count, s);
  if (steps <= 256) return launch<F32, RES, 128, 2>(p, sm_count, s);
  if (steps <= 512) return launch<F32, RES, 256, 2>(p, sm_count, s);
  if (steps <= 1024) return launch<F32, RES, 512, 2>(p, sm_count, s);
  if (steps <= 2048) return launch<F32, RES, 1024, 2>(p, sm_count, s);
  return launch<F32, RES, 1024, 4>(p, sm_count, s);
}

}  // namespace

cudaError_t dsn_launch_norm_quant(const NormParams& p, int f32, int sm_count, cudaStream_t s) {
  if (p.residual) return f32 ? pick<true, true>(p, sm_count, s) : pick<false, true>(p, sm_count, s);
  return f32 ? pick<true, false>(p, sm_count, s) : pick<false, false>(p, sm_count, s);
}
