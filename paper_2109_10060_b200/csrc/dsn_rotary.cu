// Rotary positions with one to three axes on the heads of a row (q and k of a [head][q|k|v][D] row, or plain heads):
//   (u, v) -> (u cos a - v sin a, u sin a + v cos a),  a = position[axis] * frequency of the pair.
// The frequency of a pair is held as turns per unit of position in 64-bit fixed point; position * frequency modulo 2^64 IS
// the angle modulo a full turn, exactly, whatever the position, and its top 32 bits go to sincospi in fp32.
// Bound by memory; two elements an instruction, a token's sines and cosines computed once, one pair a lane, into shared memory.
// Ring form: a group of 32 .. 256 threads has a ring of shared-memory slots of its own, which bulk copies fill with the rows to come
// (tokens and their positions are looked up 32 at a time, one a lane); it turns a row where it lies and one bulk copy takes it out, so
// what does not turn (v, the rest of a head) costs no instruction at all, and the bytes in flight do not depend on registers.
// Where rows are whole 16-byte pieces but vectors or the turned part are not, the ring's threads turn a pair at a time in shared memory (5096 rows of up
// to 31 heads x 256 bf16 with 67 pairs: 32 us; element by element in global memory, the direct form: 100 us).
// Direct form (few tokens, rows that are not made of 16-byte pieces or too long for a ring): a thread owns one place of a vector (an element pair if need be),
// keeps its factors in registers and walks the heads with them.
// Measured in a graph: 32,766 rows of 16 heads x 80 fp32, three axes: 58 us (5.8 TB/s of 6.6 for a copy); q and k of 25,216 rows of up to 12 heads x 64
// bf16: 32 us (5.4 TB/s), and 33 us in place, where v need not move but does: rows pass whole (the q and k alone would take 18).
#include <type_traits>

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

// Ring form.
constexpr int kRingThreads = 256;
constexpr int kRingDepth = 8;    // most slots of a group
struct TokenAt {
  int heads;       // 0: no such token
  int pos[3];
  int64_t row;
};

template <bool F32, bool VEC, bool INTER, int TPT>
__global__ void __launch_bounds__(kRingThreads, 2) rotary_ring_kernel(const __grid_constant__ RotaryParams p, int depth, uint32_t slot_bytes) {
  typedef Vec<F32> E;
  constexpr int GROUPS = kRingThreads / TPT, ES = F32 ? 4 : 2, W = VEC ? E::n : 1, NP = E::n / 2;
  typedef typename E::type elem;
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ uint64_t s_full[GROUPS][kRingDepth];
  __shared__ TokenAt s_at[GROUPS][kRingDepth];
  // the factors of a token as the places take them: halves cos and sin, neighbours (cos, cos) and (-sin, sin) of every pair
  constexpr int NS = VEC && INTER ? 256 : 128;
  __shared__ __align__(16) float s_cos[GROUPS][NS], s_sin[GROUPS][NS];
  __shared__ uint32_t s_abort;
  const int g = threadIdx.x / TPT, t = threadIdx.x % TPT, lane = threadIdx.x & 31;
  const bool fetches = t < 32;   // the group's first warp asks for rows and sends them off
  if (threadIdx.x < GROUPS * kRingDepth) dsn_gemm::mbar_init(dsn_gemm::smem_u32(&s_full[0][0] + threadIdx.x), 1);
  if (threadIdx.x == 0) {
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const uint32_t rows = (uint32_t)p.B * (uint32_t)p.N;
  const uint32_t gid = blockIdx.x * GROUPS + g, ngroups = gridDim.x * GROUPS;
  const int mine = gid < rows ? (int)((rows - gid + ngroups - 1) / ngroups) : 0;   // tokens of this group
  uint8_t* slots = ring + (size_t)g * depth * slot_bytes;
  volatile uint32_t* abort_flag = &s_abort;

  TokenAt ahead{0, {0, 0, 0}, 0};   // this lane's token of those being asked for
  int asked = 0;
  auto ask = [&](int slot) {
    __syncwarp();   // the slot's former token has been looked at by all lanes
    if (asked % 32 == 0) {
      ahead = TokenAt{0, {0, 0, 0}, 0};
      const uint64_t wide = (uint64_t)(asked + lane) * ngroups + gid;
      const uint32_t row = wide < rows ? (uint32_t)wide : rows;   // rows / N = B: no position
      const int pos = (int)dsn_div(row, p.by_N), r = (int)(row - (uint32_t)pos * (uint32_t)p.N);
      const PosInfo at = dsn_locate_lanes(pos, p.B, p.G, p.T, p.offsets, p.perm, p.group_slice);
      if (at.slice >= 0) {
        ahead.heads = p.heads[at.slice];
        ahead.row = (int64_t)(p.grouped ? pos : at.sample) * p.N + r;
        const int32_t* at_pos = p.positions + (p.shared ? (int64_t)r : ahead.row);
        ahead.pos[0] = at_pos[0];
        if (p.n_axes > 1) ahead.pos[1] = at_pos[p.n_pos];
        if (p.n_axes > 2) ahead.pos[2] = at_pos[2 * (int64_t)p.n_pos];
      }
      __syncwarp();
    }
    if (lane == asked % 32) {
      const uint32_t bytes = (uint32_t)(ahead.heads * p.vectors * p.D * ES), bar = dsn_gemm::smem_u32(&s_full[g][slot]);
      s_at[g][slot] = ahead;
      dsn_gemm::mbar_expect_tx(bar, bytes);
      if (bytes) dsn_bulk_load(dsn_gemm::smem_u32(slots) + (uint32_t)slot * slot_bytes, static_cast<const uint8_t*>(p.x) + ahead.row * p.ldx * ES, bytes, bar);
    }
    __syncwarp();
    ++asked;
  };
  if (fetches)
    for (int i = 0; i < depth && i < mine; ++i) ask(i);

  const int P = p.pairs, D = p.D;
  const int per = VEC && INTER ? 2 * P / W : P / W;   // places of a vector that this kernel's threads take (one pair each where places are not whole)
  const int dv = TPT / per, di = TPT - dv * per;    // from one of a thread's places to its next
  const int v0 = t / per, i0 = t - v0 * per;
  // the pairs whose angle this thread computes
  constexpr int NF = TPT < 128 ? 128 / TPT : 1;
  uint64_t freq[NF];
  int axis[NF];
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    const int i = t + j * TPT;
    freq[j] = i < P ? p.freq[i] : 0;
    axis[j] = i < P ? p.axis[i] : 0;
  }
  int slot = 0;
  uint32_t phase = 0;
  int n = 0;
  for (; n < mine; ++n) {
    bool ok = dsn_wait(dsn_gemm::smem_u32(&s_full[g][slot]), phase, abort_flag, p.status, 73);
    ok = TPT > 32 ? dsn_group_all(ok, 1 + g, TPT) : (bool)__all_sync(0xffffffffu, ok);   // a group leaves together
    if (!ok) break;
    const TokenAt cur = s_at[g][slot];
    uint8_t* row = slots + (size_t)slot * slot_bytes;
    if (cur.heads > 0) {
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        const int i = t + j * TPT;
        if (i < P) {
          const int at = axis[j] == 0 ? cur.pos[0] : (axis[j] == 1 ? cur.pos[1] : cur.pos[2]);
          const uint64_t a = (uint64_t)(int64_t)at * freq[j];
          float c, s;
          sincospif((float)(int32_t)(a >> 32) * 4.656612873077393e-10f, &s, &c);   // 2^-31: -1 .. 1 half turns
          s = p.inverse ? -s : s;
          if constexpr (VEC && INTER) {
            *reinterpret_cast<float2*>(&s_cos[g][2 * i]) = make_float2(c, c);
            *reinterpret_cast<float2*>(&s_sin[g][2 * i]) = make_float2(-s, s);
          } else {
            s_cos[g][i] = c;
            s_sin[g][i] = s;
          }
        }
      }
      if (TPT > 32) asm volatile("bar.sync %0, %1;" ::"r"(1 + g), "n"(TPT) : "memory"); else __syncwarp();
      const int turned = cur.heads * p.rotated;
      auto factors = [&](int i, uint64_t (&c)[NP], uint64_t (&s)[NP]) {   // of the place that begins at element i
#pragma unroll
        for (int e = 0; e < NP; e += 2) {
          const ulonglong2 cc = *reinterpret_cast<const ulonglong2*>(&s_cos[g][i + 2 * e]), ss = *reinterpret_cast<const ulonglong2*>(&s_sin[g][i + 2 * e]);
          c[e] = cc.x;
          c[e + 1] = cc.y;
          s[e] = ss.x;
          s[e + 1] = ss.y;
        }
      };
      auto turn_place = [&](uint8_t* at, const uint64_t (&c)[NP], const uint64_t (&s)[NP]) {
        uint64_t a[NP];
        E::widen(*reinterpret_cast<const uint4*>(at), a);
        if constexpr (!INTER) {
          uint64_t b[NP], na[NP], nb[NP];
          E::widen(*reinterpret_cast<const uint4*>(at + P * ES), b);
#pragma unroll
          for (int e = 0; e < NP; ++e) {
            na[e] = ffma2(neg2(b[e]), s[e], fmul2(a[e], c[e]));
            nb[e] = ffma2(b[e], c[e], fmul2(a[e], s[e]));
          }
          *reinterpret_cast<uint4*>(at) = E::narrow(na);
          *reinterpret_cast<uint4*>(at + P * ES) = E::narrow(nb);
        } else {
#pragma unroll
          for (int e = 0; e < NP; ++e) a[e] = ffma2(swap2(a[e]), s[e], fmul2(a[e], c[e]));
          *reinterpret_cast<uint4*>(at) = E::narrow(a);
        }
      };
      if constexpr (VEC) {
        uint64_t c[NP], s[NP];
        if (di == 0) {   // this thread's place is the same in all of its vectors
          factors(i0 * W, c, s);
#pragma unroll 4
          for (int v = v0; v < turned; v += dv) turn_place(row + (size_t)(vec_at(p, v) + i0 * W) * ES, c, s);
        } else {
          int v = v0, pc = i0;
#pragma unroll 2
          while (v < turned) {
            factors(pc * W, c, s);
            turn_place(row + (size_t)(vec_at(p, v) + pc * W) * ES, c, s);
            v += dv;
            pc += di;
            if (pc >= per) { pc -= per; ++v; }
          }
        }
      } else {
        int v = v0, pc = i0;
#pragma unroll 2
        while (v < turned) {
          elem* at = reinterpret_cast<elem*>(row) + vec_at(p, v);
          const int ia = INTER ? 2 * pc : pc, ib = INTER ? 2 * pc + 1 : pc + P;
          const float a = E::get(at + ia), b = E::get(at + ib), c = s_cos[g][pc], s = s_sin[g][pc];
          E::put(at + ia, a * c - b * s);
          E::put(at + ib, a * s + b * c);
          v += dv;
          pc += di;
          if (pc >= per) { pc -= per; ++v; }
        }
      }
      dsn_gemm::fence_async_smem();   // the turned elements are visible to the copy that takes them out
    }
    if (TPT > 32) asm volatile("bar.sync %0, %1;" ::"r"(1 + g), "n"(TPT) : "memory"); else __syncwarp();
    if (fetches) {
      if (t == 0) {
        if (cur.heads > 0) dsn_bulk_store(static_cast<uint8_t*>(p.y) + cur.row * p.ldy * ES, dsn_gemm::smem_u32(row), (uint32_t)(cur.heads * p.vectors * D * ES));
        dsn_gemm::bulk_commit();
        asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");   // the token before has left its slot
      }
      __syncwarp();
      if (n > 0 && asked < mine) ask(slot == 0 ? depth - 1 : slot - 1);  // which takes the next row
    }
    if (++slot == depth) { slot = 0; phase ^= 1u; }
  }
  if (t == 0) dsn_gemm::bulk_wait0();
  if (fetches && n < mine) dsn_drain(dsn_gemm::smem_u32(&s_full[g][0]), depth, n, asked);
}

template <bool F32, bool VEC, bool INTER, int TPT>
cudaError_t launch_ring(const RotaryParams& p, uint32_t row_bytes, int per_sm, int sm_count, cudaStream_t s) {
  static size_t configured[DSN_MAX_DEVICES] = {};
  auto kernel = rotary_ring_kernel<F32, VEC, INTER, TPT>;
  constexpr int GROUPS = kRingThreads / TPT;
  int depth = (int)((per_sm == 2 ? 92 : 184) * 1024 / (GROUPS * row_bytes));
  if (depth < 2) return cudaErrorInvalidConfiguration;
  if (depth > kRingDepth) depth = kRingDepth;
  const size_t smem = (size_t)depth * GROUPS * row_bytes;
  const cudaError_t e = dsn_ensure_dynamic_smem(kernel, smem, configured);
  if (e != cudaSuccess) return e;
  const int64_t ctas = ((int64_t)p.B * p.N + GROUPS - 1) / GROUPS, most = (int64_t)sm_count * per_sm;
  return dsn_launch(kernel, dim3((unsigned)(ctas < most ? ctas : most)), dim3(kRingThreads), smem, s, 1, p, depth, row_bytes);
}

template <bool F32, bool VEC, bool INTER, int TPT>
cudaError_t launch(const RotaryParams& p, int sm_count, cudaStream_t s) {
  constexpr int THREADS = TPT > 128 ? TPT : 128;
  static int resident[DSN_MAX_DEVICES] = {};
  auto kernel = rotary_kernel<F32, VEC, INTER, TPT, THREADS>;
  int n = 0;
  const cudaError_t e = dsn_ctas_per_sm(kernel, THREADS, 0, resident, &n);
  if (e != cudaSuccess) return e;
  const int64_t ctas = ((int64_t)p.B * p.N + THREADS / TPT - 1) / (THREADS / TPT), most = (int64_t)sm_count * n;
  return dsn_launch(kernel, dim3((unsigned)(ctas < most ? ctas : most)), dim3(THREADS), 0, s, 1, p);
}
template <bool F32, bool VEC, bool INTER>
cudaError_t pick(const RotaryParams& p, int sm_count, cudaStream_t s) {
  const int64_t bytes = (int64_t)p.max_heads * p.vectors * p.D * (F32 ? 4 : 2);
  // whole_rows: every path's rows are whole 16-byte pieces, whatever their vectors are
  // (us, ring and direct form, 4.6 KB rows: 300 rows 4.4, 3.7; 600 rows 4.4, 5.3; 4800 rows 9.3, 12.1)
  if (p.whole_rows && (int64_t)p.B * p.N >= 4 * sm_count && bytes <= 92 * 1024) {
    // the fewest threads a row with which two slots a group fit
    if (bytes <= 5888) return launch_ring<F32, VEC, INTER, 32>(p, (uint32_t)bytes, 2, sm_count, s);
    if (bytes <= 11776) return launch_ring<F32, VEC, INTER, 64>(p, (uint32_t)bytes, 2, sm_count, s);
    if (bytes <= 23552) return launch_ring<F32, VEC, INTER, 128>(p, (uint32_t)bytes, 2, sm_count, s);
    return launch_ring<F32, VEC, INTER, 256>(p, (uint32_t)bytes, bytes <= 47104 ? 2 : 1, sm_count, s);
  }
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
