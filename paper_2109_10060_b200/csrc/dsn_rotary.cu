// Rotary positions with one to three axes on the heads of a row (q and k of a [head][q|k|v][D] row, or plain heads):
//   (u, v) -> (u cos a - v sin a, u sin a + v cos a),  a = position[axis] * frequency of the pair.
// The frequency of a pair is held as turns per unit of position in 64-bit fixed point; position * frequency modulo 2^64 IS
// the angle modulo a full turn, exactly, whatever the position, and its top 32 bits go to sincospi in fp32.
// Bound by memory.  A token's sines and cosines are computed once into shared memory, one pair a lane; a thread then owns
// one 16-byte place of a vector, keeps its factors in registers and walks the heads with them, two elements an instruction, several
// heads' loads in flight.  Every element is read and written once.
#include <type_traits>

#include "dsn_gemm_device.cuh"
#include "dsn_transformer.cuh"

namespace {

using dsn_gemm::ffma2;
using dsn_gemm::pack2;
using dsn_gemm::unpack2;

__device__ __forceinline__ uint64_t fmul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t neg2(uint64_t a) { return a ^ 0x8000000080000000ull; }
__device__ __forceinline__ uint64_t swap2(uint64_t a) { return (a >> 32) | (a << 32); }

// 16 bytes as pairs of fp32.
template <bool F32>
struct Vec;
template <>
struct Vec<false> {
  typedef __nv_bfloat16 type;
  static constexpr int n = 8;
  static __device__ __forceinline__ void widen(const uint4& a, uint64_t (&v)[4]) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ uint4 narrow(const uint64_t (&v)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      unpack2(v[i], a, b);
      __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
      w[i] = *reinterpret_cast<uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float get(const type* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void put(type* p, float v) { *p = __float2bfloat16_rn(v); }
};
template <>
struct Vec<true> {
  typedef float type;
  static constexpr int n = 4;
  static __device__ __forceinline__ void widen(const uint4& a, uint64_t (&v)[2]) {
    v[0] = (uint64_t)a.x | ((uint64_t)a.y << 32);
    v[1] = (uint64_t)a.z | ((uint64_t)a.w << 32);
  }
  static __device__ __forceinline__ uint4 narrow(const uint64_t (&v)[2]) {
    return make_uint4((uint32_t)v[0], (uint32_t)(v[0] >> 32), (uint32_t)v[1], (uint32_t)(v[1] >> 32));
  }
  static __device__ __forceinline__ float get(const type* p) { return *p; }
  static __device__ __forceinline__ void put(type* p, float v) { *p = v; }
};

// first element of turned vector v: vectors lie [head][vectors][D], the first `rotated` of a head turn
__device__ __forceinline__ int vec_at(const RotaryParams& p, int v) {
  const int hd = p.rotated == 1 ? v : (p.rotated == 2 ? v >> 1 : v / p.rotated);
  return (hd * p.vectors + (v - hd * p.rotated)) * p.D;
}

// Copies 16-byte pieces (or elements) [i0, i1) of the vectors [v0, v1), which lie `at(v)` elements into the row.
template <typename T, typename At>
__device__ __forceinline__ void copy_pieces(const T* x, T* y, int per, int count, int t, int tpt, At at) {
  if (per <= 0) return;
  const int step = tpt >= per ? tpt / per : 1;
  if (tpt >= per) {
    const int v0 = t / per, i = t - v0 * per;
    if (v0 < step)
#pragma unroll 4
      for (int v = v0; v < count; v += step) y[at(v) + i] = x[at(v) + i];
  } else {
    for (int v = 0; v < count; ++v)
      for (int i = t; i < per; i += tpt) y[at(v) + i] = x[at(v) + i];
  }
}

// VEC: rows, vectors and the turned part are made of whole 16-byte pieces; otherwise element by element.
// TPT threads a token, THREADS a CTA; a CTA walks tokens with the stride of the grid.
template <bool F32, bool VEC, bool INTER, int TPT, int THREADS>
__global__ void __launch_bounds__(THREADS) rotary_kernel(const __grid_constant__ RotaryParams p) {
  typedef Vec<F32> E;
  typedef typename E::type elem;
  constexpr int TPC = THREADS / TPT;
  __shared__ __align__(16) float s_cos[TPC][128], s_sin[TPC][128];
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const int mine = threadIdx.x / TPT, t = threadIdx.x % TPT;
  const uint32_t rows = (uint32_t)p.B * (uint32_t)p.N;   // below 2^31
  const uint32_t stride = gridDim.x * TPC;
  const int P = p.pairs, D = p.D;
  // this thread's place: piece i of the turned part (VEC halves: of each half), vectors v0, v0 + step, ...
  constexpr int W = VEC ? E::n : 1;
  const int per = VEC && INTER ? 2 * P / W : P / W;
  const int step = TPT >= per ? TPT / per : 1;
  const int v0 = TPT >= per ? t / per : 0, first = TPT >= per ? t - v0 * per : t;

  for (uint32_t base = blockIdx.x * TPC; base < rows; base += stride) {
    const uint32_t row = base + mine;
    const int pos = (int)dsn_div(row, p.by_N), r = (int)(row - (uint32_t)pos * (uint32_t)p.N);
    PosInfo at{0, -1};
    if (pos < p.B) at = dsn_locate_warp(pos, p.G, p.T, p.offsets, p.perm, p.group_slice);
    const int heads = at.slice < 0 ? 0 : p.heads[at.slice];
    const int64_t xrow = (int64_t)(p.grouped ? pos : at.sample) * p.N + r;
    if (heads > 0) {
      const int32_t* at_pos = p.positions + (p.shared ? (int64_t)r : xrow);
      for (int i = t; i < P; i += TPT) {
        const uint64_t a = (uint64_t)(int64_t)at_pos[(int64_t)p.axis[i] * p.n_pos] * p.freq[i];
        float c, s;
        sincospif((float)(int32_t)(a >> 32) * 4.656612873077393e-10f, &s, &c);   // 2^-31: -1 .. 1 half turns
        s_cos[mine][i] = c;
        s_sin[mine][i] = p.inverse ? -s : s;
      }
    }
    if constexpr (TPT > 32) __syncthreads(); else __syncwarp();
    const elem* x = static_cast<const elem*>(p.x) + xrow * p.ldx;
    elem* y = static_cast<elem*>(p.y) + xrow * p.ldy;
    const int turned = heads * p.rotated;   // vectors that turn (0: no such row)
    if constexpr (VEC) {
      constexpr int NP = W / 2;             // pairs of fp32 in 16 bytes
      if (v0 < step) {
        for (int pc = first; pc < per; pc += TPT) {   // one round unless a vector has more pieces than the token has threads
          const int i = pc * W;
          if constexpr (!INTER) {
            uint64_t c[NP], s[NP];
#pragma unroll
            for (int e = 0; e < NP; ++e) {
              c[e] = *reinterpret_cast<const uint64_t*>(&s_cos[mine][i + 2 * e]);
              s[e] = *reinterpret_cast<const uint64_t*>(&s_sin[mine][i + 2 * e]);
            }
#pragma unroll 3
            for (int v = v0; v < turned; v += step) {
              const int o = vec_at(p, v) + i;
              uint64_t a[NP], b[NP], na[NP], nb[NP];
              E::widen(*reinterpret_cast<const uint4*>(x + o), a);
              E::widen(*reinterpret_cast<const uint4*>(x + o + P), b);
#pragma unroll
              for (int e = 0; e < NP; ++e) {
                na[e] = ffma2(neg2(b[e]), s[e], fmul2(a[e], c[e]));
                nb[e] = ffma2(b[e], c[e], fmul2(a[e], s[e]));
              }
              *reinterpret_cast<uint4*>(y + o) = E::narrow(na);
              *reinterpret_cast<uint4*>(y + o + P) = E::narrow(nb);
            }
          } else {
            uint64_t c[NP], s[NP];   // (cos, cos) and (-sin, sin) of each pair of the piece
#pragma unroll
            for (int e = 0; e < NP; ++e) {
              const float ce = s_cos[mine][i / 2 + e], se = s_sin[mine][i / 2 + e];
              c[e] = pack2(ce, ce);
              s[e] = pack2(-se, se);
            }
#pragma unroll 4
            for (int v = v0; v < turned; v += step) {
              const int o = vec_at(p, v) + i;
              uint64_t a[NP];
              E::widen(*reinterpret_cast<const uint4*>(x + o), a);
#pragma unroll
              for (int e = 0; e < NP; ++e) a[e] = ffma2(swap2(a[e]), s[e], fmul2(a[e], c[e]));
              *reinterpret_cast<uint4*>(y + o) = E::narrow(a);
            }
          }
        }
      }
    } else if (v0 < step) {
      for (int i = first; i < P; i += TPT) {
        const float c = s_cos[mine][i], s = s_sin[mine][i];
        const int ia = INTER ? 2 * i : i, ib = INTER ? 2 * i + 1 : i + P;
        for (int v = v0; v < turned; v += step) {
          const int o = vec_at(p, v);
          const float a = E::get(x + o + ia), b = E::get(x + o + ib);
          E::put(y + o + ia, a * c - b * s);
          E::put(y + o + ib, a * s + b * c);
        }
      }
    }
    if (!p.in_place) {
      // what does not turn is copied: the rest of the turned vectors, then the vectors that stay as they are
      typedef typename std::conditional<VEC, uint4, elem>::type piece;
      const piece* xs = reinterpret_cast<const piece*>(x);
      piece* ys = reinterpret_cast<piece*>(y);
      copy_pieces(xs, ys, (D - 2 * P) / W, turned, t, TPT, [&](int v) { return (vec_at(p, v) + 2 * P) / W; });
      copy_pieces(xs, ys, (p.vectors - p.rotated) * D / W, heads, t, TPT, [&](int hd) { return (hd * p.vectors + p.rotated) * D / W; });
    }
    if constexpr (TPT > 32) __syncthreads(); else __syncwarp();   // the factors are rewritten for the next token
  }
}

template <bool F32, bool VEC, bool INTER, int TPT>
cudaError_t launch(const RotaryParams& p, int sm_count, cudaStream_t s) {
  constexpr int THREADS = TPT > 128 ? TPT : 128;
  static int resident[DSN_MAX_DEVICES] = {};   // CTAs per SM of this form
  auto kernel = rotary_kernel<F32, VEC, INTER, TPT, THREADS>;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= DSN_MAX_DEVICES) return cudaErrorInvalidDevice;
  if (resident[dev] == 0) {
    int n = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, THREADS, 0);
    if (e != cudaSuccess) return e;
    resident[dev] = n > 0 ? n : 1;
  }
  const int64_t ctas = ((int64_t)p.B * p.N + THREADS / TPT - 1) / (THREADS / TPT), most = (int64_t)sm_count * resident[dev];
  return dsn_launch(kernel, dim3((unsigned)(ctas < most ? ctas : most)), dim3(THREADS), 0, s, 1, p);
}
template <bool F32, bool VEC, bool INTER>
cudaError_t pick(const RotaryParams& p, int sm_count, cudaStream_t s) {
  // a warp a token where there are tokens enough to fill the GPU, else 256 threads
  return (int64_t)p.B * p.N >= 16 * sm_count ? launch<F32, VEC, INTER, 32>(p, sm_count, s) : launch<F32, VEC, INTER, 256>(p, sm_count, s);
}
template <bool F32>
cudaError_t pick_form(const RotaryParams& p, bool vec, int sm_count, cudaStream_t s) {
  if (vec) return p.interleaved ? pick<F32, true, true>(p, sm_count, s) : pick<F32, true, false>(p, sm_count, s);
  return p.interleaved ? pick<F32, false, true>(p, sm_count, s) : pick<F32, false, false>(p, sm_count, s);
}

}  // namespace

cudaError_t dsn_launch_rotary(const RotaryParams& p, int f32, int aligned, int sm_count, cudaStream_t s) {
  const int n = f32 ? 4 : 8;
  const bool vec = aligned && p.D % n == 0 && (p.interleaved ? 2 * p.pairs : p.pairs) % n == 0;
  return f32 ? pick_form<true>(p, vec, sm_count, s) : pick_form<false>(p, vec, sm_count, s);
}
