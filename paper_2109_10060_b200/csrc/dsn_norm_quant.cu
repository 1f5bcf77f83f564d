// Residual addition, root-mean-square norm on elastic widths and 8-bit codes with a scale per row, in one pass:
//   h = x + residual;  n = h / sqrt(mean h^2 + eps) * w;  s = max|n| / 127;  q = round(h w * 127 / max|h w|).
// The factor 1 / sqrt(...) is common to a row, so it drops out of the code: the sum of squares and the maximum of |h w|
// come out of ONE reduction, and the codes do not depend on the order of the sum.
// Bound by memory: a row lives in the registers of 32 .. 1024 threads between its only read and its writes; eight
// columns (16 bytes of bf16, 32 of fp32) a thread and step.
#include "dsn_transformer.cuh"

namespace {

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

template <bool F32>
struct Elem;
template <>
struct Elem<false> {
  typedef __nv_bfloat16 type;
  static __device__ __forceinline__ void load8(const type* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store8(type* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
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
  static __device__ __forceinline__ void load8(const type* p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  static __device__ __forceinline__ void store8(type* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
  static __device__ __forceinline__ float load1(const type* p) { return *p; }
  static __device__ __forceinline__ void store1(type* p, float v) { *p = v; }
};

// (sum, maximum) over the TPR threads of a row; every thread of the CTA calls this.
template <int TPR, int THREADS>
__device__ __forceinline__ void row_reduce(float& ss, float& mx) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    ss += __shfl_xor_sync(0xffffffffu, ss, o);
    mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  }
  if constexpr (TPR > 32) {
    __shared__ float2 part[THREADS / 32];
    const int warp = threadIdx.x >> 5;
    __syncthreads();   // an earlier reduction's reads are done
    if ((threadIdx.x & 31) == 0) part[warp] = make_float2(ss, mx);
    __syncthreads();
    const int w0 = warp & ~(TPR / 32 - 1);
    ss = 0.f;
    mx = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) {
      const float2 v = part[w0 + i];
      ss += v.x;
      mx = max_nan(mx, v.y);
    }
  }
}

// TPR threads a row, VPT steps of eight columns a thread, THREADS a CTA.
template <bool F32, int TPR, int VPT, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_quant_kernel(const __grid_constant__ NormParams p) {
  typedef Elem<F32> E;
  typedef typename E::type elem;
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const uint32_t row = blockIdx.x * (uint32_t)(THREADS / TPR) + threadIdx.x / TPR;   // B * R < 2^31
  const int t = threadIdx.x % TPR;
  const int pos = (int)(row / (uint32_t)p.R), r = (int)(row - (uint32_t)pos * (uint32_t)p.R);
  PosInfo at{0, -1};
  if (pos < p.B) at = dsn_locate_warp(pos, p.G, p.T, p.offsets, p.perm, p.group_slice);
  const int k = at.slice < 0 ? 0 : p.k[at.slice];   // 0: this row does not exist; its threads only take part in the barriers
  const int64_t in_row = (int64_t)(p.in_input_order ? at.sample : pos) * p.R + r;
  const int64_t out_row = (int64_t)(p.out_input_order ? at.sample : pos) * p.R + r;
  const elem* x = static_cast<const elem*>(p.x) + in_row * p.ldx;
  const elem* res = p.residual ? static_cast<const elem*>(p.residual) + in_row * p.ld_res : nullptr;

  float h[VPT][8], w[VPT][8];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int c = 8 * (t + j * TPR);
    if (c + 8 <= k) {
      E::load8(x + c, h[j]);
      if (res) {
        float b[8];
        E::load8(res + c, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[j][i] += b[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[j][i] = 0.f;
        if (c + i < k) h[j][i] = E::load1(x + c + i) + (res ? E::load1(res + c + i) : 0.f);
      }
    }
  }
  float ss = 0.f, mx = 0.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int c = 8 * (t + j * TPR);
    if (p.weight && c + 8 <= k) {
      Elem<true>::load8(p.weight + c, w[j]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[j][i] = (p.weight && c + i < k) ? p.weight[c + i] : 1.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      ss = fmaf(h[j][i], h[j][i], ss);
      mx = max_nan(mx, fabsf(h[j][i] * w[j][i]));
    }
  }
  if (p.sum) {
    elem* d = static_cast<elem*>(p.sum) + in_row * p.ld_sum;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = 8 * (t + j * TPR);
      if (c + 8 <= k) {
        E::store8(d + c, h[j]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < k) E::store1(d + c + i, h[j][i]);
      }
    }
  }
  if (!p.q && !p.y) return;
  row_reduce<TPR, THREADS>(ss, mx);
  float eps = p.eps;
  // The squares (or a product with the weight) left the range of fp32, or the row holds something that is no number.  Rare, and the
  // same for all threads of a row, but not for all rows of the CTA: the second reduction is entered by all when one row asks.
  const bool redo = !(ss < INFINITY) || !(mx < INFINITY);
  if (TPR > 32 ? __syncthreads_or(redo) : __any_sync(0xffffffffu, redo)) {
    float top = 0.f, any = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max_nan(top, fabsf(h[j][i]));
    row_reduce<TPR, THREADS>(any, top);
    // h is scaled by a power of two to less than 4 (exact; what underflows is below 2^-120 of the row's largest value)
    const uint32_t top_exp = __float_as_uint(top) >> 23;
    const float f = (redo && top < INFINITY && top > 2.f) ? __uint_as_float((top_exp < 253u ? 254u - top_exp : 1u) << 23) : 1.f;
    float ss2 = 0.f, mx2 = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[j][i] *= f;
        ss2 = fmaf(h[j][i], h[j][i], ss2);
        mx2 = max_nan(mx2, fabsf(h[j][i] * w[j][i]));
      }
    row_reduce<TPR, THREADS>(ss2, mx2);
    ss = ss2;
    mx = mx2;
    eps = eps * f * f;
    if (!(top < INFINITY)) mx = __uint_as_float(0x7fffffffu);   // NaN or infinity in the row: NaN comes out
  }
  if (k == 0) return;
  const float rs = rsqrtf(ss / (float)k + eps);
  if (p.q) {
    // a maximum below 2^-120 would overflow 127 / max: such a row is scaled up first (exact)
    const float up = mx < 7.52316385e-37f ? 1.32922800e36f : 1.f;
    const float inv = mx > 0.f ? __fdiv_rn(127.f, mx * up) : (mx == 0.f ? 0.f : mx);
    const float scale = __fdiv_rn(mx * rs, 127.f);
    int8_t* q = p.q + out_row * p.ldq;
    elem* y = p.y ? static_cast<elem*>(p.y) + out_row * p.ldy : nullptr;
    if (t == 0) p.scale[out_row] = scale;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = 8 * (t + j * TPR);
      uint32_t code[2] = {0u, 0u};
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int n = __float2int_rn(__fmul_rn(__fmul_rn(h[j][i], w[j][i]) * up, inv));   // NaN gives 0
        code[i >> 2] |= (uint32_t)(n & 0xff) << (8 * (i & 3));
        v[i] = (float)n * scale;
      }
      if (c + 8 <= k) {
        *reinterpret_cast<uint2*>(q + c) = make_uint2(code[0], code[1]);
        if (y) E::store8(y + c, v);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < k) {
            q[c + i] = (int8_t)(code[i >> 2] >> (8 * (i & 3)));
            if (y) E::store1(y + c + i, v[i]);
          }
      }
    }
  } else {
    elem* y = static_cast<elem*>(p.y) + out_row * p.ldy;
    const float f = mx >= 0.f ? rs : mx;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = 8 * (t + j * TPR);
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = h[j][i] * w[j][i] * f;
      if (c + 8 <= k) {
        E::store8(y + c, v);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < k) E::store1(y + c + i, v[i]);
      }
    }
  }
}

template <bool F32, int TPR, int VPT>
cudaError_t launch(const NormParams& p, cudaStream_t s) {
  constexpr int THREADS = TPR > 128 ? TPR : 128;
  const int64_t rows = (int64_t)p.B * p.R;
  const int per = THREADS / TPR;
  return dsn_launch(norm_quant_kernel<F32, TPR, VPT, THREADS>, dim3((unsigned)((rows + per - 1) / per)), dim3(THREADS), 0, s, 1, p);
}

template <bool F32>
cudaError_t pick(const NormParams& p, int max_k, cudaStream_t s) {
  const int steps = (max_k + 7) / 8;
  if (steps <= 32) return launch<F32, 32, 1>(p, s);
  if (steps <= 64) return launch<F32, 32, 2>(p, s);
  if (steps <= 128) return launch<F32, 64, 2>(p, s);
  if (steps <= 256) return launch<F32, 128, 2>(p, s);
  if (steps <= 512) return launch<F32, 256, 2>(p, s);
  if (steps <= 1024) return launch<F32, 512, 2>(p, s);
  if (steps <= 2048) return launch<F32, 1024, 2>(p, s);
  return launch<F32, 1024, 4>(p, s);
}

}  // namespace

cudaError_t dsn_launch_norm_quant(const NormParams& p, int f32, int max_k, cudaStream_t s) {
  return f32 ? pick<true>(p, max_k, s) : pick<false>(p, max_k, s);
}
