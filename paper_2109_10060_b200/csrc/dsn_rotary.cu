// Rotary positions with one to three axes on the heads of a row (q and k of a [head][q|k|v][D] row, or plain heads):
//   (u, v) -> (u cos a - v sin a, u sin a + v cos a),  a = position[axis] * frequency of the pair.
// The frequency of a pair is held as turns per unit of position in 64-bit fixed point; position * frequency modulo 2^64 IS
// the angle modulo a full turn, exactly, whatever the position, and its top 32 bits go to sincospi in fp32.
// Bound by memory: a token's sines and cosines are computed once into shared memory and serve all of its heads;
// 16-byte pieces, every element read and written once.
#include "dsn_transformer.cuh"

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void turn_of(const RotaryParams& p, int i, int position, float& c, float& s) {
  const uint64_t a = (uint64_t)(int64_t)position * p.freq[i];
  const float half_turns = (float)(int32_t)(a >> 32) * 4.656612873077393e-10f;   // 2^-31: -1 .. 1 half turns
  sincospif(half_turns, &s, &c);
  if (p.inverse) s = -s;
}

template <bool F32>
struct Vec;
template <>
struct Vec<false> {
  typedef __nv_bfloat16 type;
  static constexpr int n = 8;
  static __device__ __forceinline__ void load(const type* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(type* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float get(const type* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void put(type* p, float v) { *p = __float2bfloat16_rn(v); }
};
template <>
struct Vec<true> {
  typedef float type;
  static constexpr int n = 4;
  static __device__ __forceinline__ void load(const type* p, float (&v)[4]) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  }
  static __device__ __forceinline__ void store(type* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
  static __device__ __forceinline__ float get(const type* p) { return *p; }
  static __device__ __forceinline__ void put(type* p, float v) { *p = v; }
};

// VEC: rows, vectors and the turned part are made of whole 16-byte pieces; otherwise element by element.
// A CTA takes kThreads / TPT tokens, TPT threads each.
template <bool F32, bool VEC, int TPT>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ RotaryParams p) {
  typedef Vec<F32> E;
  typedef typename E::type elem;
  extern __shared__ float2 s_turn[];   // [kThreads / TPT][pairs]
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const uint32_t row = blockIdx.x * (uint32_t)(kThreads / TPT) + threadIdx.x / TPT;   // B * N < 2^31
  const int t = threadIdx.x % TPT;
  const int pos = (int)(row / (uint32_t)p.N), r = (int)(row - (uint32_t)pos * (uint32_t)p.N);
  PosInfo at{0, -1};
  if (pos < p.B) at = dsn_locate_warp(pos, p.G, p.T, p.offsets, p.perm, p.group_slice);
  const int heads = at.slice < 0 ? 0 : p.heads[at.slice];
  const int64_t xrow = (int64_t)(p.grouped ? pos : at.sample) * p.N + r;
  float2* turn = s_turn + (threadIdx.x / TPT) * p.pairs;
  if (heads > 0) {
    const int64_t prow = p.shared ? r : xrow;
    for (int i = t; i < p.pairs; i += TPT) {
      float c, s;
      turn_of(p, i, p.positions[(int64_t)p.axis[i] * p.n_pos + prow], c, s);
      turn[i] = make_float2(c, s);
    }
  }
  if constexpr (TPT > 32) __syncthreads(); else __syncwarp();
  if (heads == 0) return;
  const elem* x = static_cast<const elem*>(p.x) + xrow * p.ldx;
  elem* y = static_cast<elem*>(p.y) + xrow * p.ldy;
  const int P = p.pairs, D = p.D;
  const int turned = heads * p.rotated;   // vectors that turn
  constexpr int W = VEC ? E::n : 1;
  if constexpr (VEC) {
    if (!p.interleaved) {
      const int per = P / W;   // pieces of a half
      for (int u = t; u < turned * per; u += TPT) {
        const int v = u / per, i = (u - v * per) * W;
        const int hd = v / p.rotated;
        const int64_t o = (int64_t)(hd * p.vectors + (v - hd * p.rotated)) * D + i;
        float a[W], b[W];
        E::load(x + o, a);
        E::load(x + o + P, b);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float2 cs = turn[i + e];
          const float n = a[e] * cs.x - b[e] * cs.y;
          b[e] = a[e] * cs.y + b[e] * cs.x;
          a[e] = n;
        }
        E::store(y + o, a);
        E::store(y + o + P, b);
      }
    } else {
      const int per = 2 * P / W;
      for (int u = t; u < turned * per; u += TPT) {
        const int v = u / per, i = (u - v * per) * W;
        const int hd = v / p.rotated;
        const int64_t o = (int64_t)(hd * p.vectors + (v - hd * p.rotated)) * D + i;
        float a[W];
        E::load(x + o, a);
#pragma unroll
        for (int e = 0; e < W; e += 2) {
          const float2 cs = turn[(i + e) >> 1];
          const float n = a[e] * cs.x - a[e + 1] * cs.y;
          a[e + 1] = a[e] * cs.y + a[e + 1] * cs.x;
          a[e] = n;
        }
        E::store(y + o, a);
      }
    }
  } else {
    for (int u = t; u < turned * P; u += TPT) {
      const int v = u / P, i = u - v * P;
      const int hd = v / p.rotated;
      const int64_t o = (int64_t)(hd * p.vectors + (v - hd * p.rotated)) * D;
      const int64_t oa = o + (p.interleaved ? 2 * i : i), ob = o + (p.interleaved ? 2 * i + 1 : i + P);
      const float a = E::get(x + oa), b = E::get(x + ob);
      const float2 cs = turn[i];
      E::put(y + oa, a * cs.x - b * cs.y);
      E::put(y + ob, a * cs.y + b * cs.x);
    }
  }
  if (p.in_place) return;
  // what does not turn is copied: the rest of the turned vectors, then the vectors that stay as they are
  const int rest = (D - 2 * P) / W;
  for (int u = t; u < turned * rest; u += TPT) {
    const int v = u / rest, i = 2 * P + (u - v * rest) * W;
    const int hd = v / p.rotated;
    const int64_t o = (int64_t)(hd * p.vectors + (v - hd * p.rotated)) * D + i;
    if constexpr (VEC) *reinterpret_cast<uint4*>(y + o) = *reinterpret_cast<const uint4*>(x + o); else y[o] = x[o];
  }
  const int still = (p.vectors - p.rotated) * D / W;   // contiguous pieces of a head
  for (int u = t; u < heads * still; u += TPT) {
    const int hd = u / still;
    const int64_t o = (int64_t)(hd * p.vectors + p.rotated) * D + (int64_t)(u - hd * still) * W;
    if constexpr (VEC) *reinterpret_cast<uint4*>(y + o) = *reinterpret_cast<const uint4*>(x + o); else y[o] = x[o];
  }
}

template <bool F32, bool VEC, int TPT>
cudaError_t launch(const RotaryParams& p, cudaStream_t s) {
  const int per = kThreads / TPT;
  const int64_t rows = (int64_t)p.B * p.N;
  return dsn_launch(rotary_kernel<F32, VEC, TPT>, dim3((unsigned)((rows + per - 1) / per)), dim3(kThreads), per * p.pairs * sizeof(float2),
                    s, 1, p);
}
template <bool F32, bool VEC>
cudaError_t pick(const RotaryParams& p, int max_heads, cudaStream_t s) {
  const int64_t pieces = (int64_t)max_heads * p.vectors * p.D / (VEC ? Vec<F32>::n : 1);
  if (pieces <= 128) return launch<F32, VEC, 32>(p, s);
  if (pieces <= 512) return launch<F32, VEC, 128>(p, s);
  return launch<F32, VEC, 256>(p, s);
}

}  // namespace

cudaError_t dsn_launch_rotary(const RotaryParams& p, int f32, int max_heads, int aligned, cudaStream_t s) {
  const int n = f32 ? 4 : 8;
  const bool vec = aligned && p.D % n == 0 && (p.interleaved ? 2 * p.pairs : p.pairs) % n == 0;
  if (f32) return vec ? pick<true, true>(p, max_heads, s) : pick<true, false>(p, max_heads, s);
  return vec ? pick<false, true>(p, max_heads, s) : pick<false, false>(p, max_heads, s);
}
