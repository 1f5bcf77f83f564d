// 4-bit cache of keys and values: which pages and slots the new tokens of a batch take (plan), and the write that rounds k and v into them.
#include "dsn_cache.cuh"

namespace {

using dsn_gemm::fadd2;
using dsn_gemm::ffma2;
using dsn_gemm::pack2;
using dsn_gemm::unpack2;

// ------------------------------------------------------------------------------------------------ plan
// One cluster of CTAs (one CTA for few rows); every CTA scans all requests on its own (8 bytes each), one a thread and THREADS at a time, and then the threads of
// the cluster share the slots.  A slot needs no other thread's result: a token's page stands in the table already or
// is the ring's entry at a place that the scan gives.  What a CTA of the cluster still has to read (lengths, ring counters) is overwritten only behind the
// cluster's barrier.  Pages taken and pages returned are different entries of the ring, so those need no order.
// Bound by trips to memory: lengths, then pages, then the stores; rows are looked up eight a thread, or four neighbours a lane, at once (128 x 2048 rows: 8.0 us, one after the other 18; 64 x 1 row 2.4).
struct PlanRequest {
  int32_t held, placed;   // placed < 0: the request ends
  uint32_t start;         // new pages of the requests before it; or returned pages of the requests before it
};

// Place i of the ring: what is taken or given back together does not pass the whole ring.
__device__ __forceinline__ uint32_t ring(uint32_t i, uint32_t N) { return i >= N ? (i - N < N ? i - N : (i - N) % N) : i; }

template <int THREADS, bool LONG>   // LONG: many rows a request
__global__ void __launch_bounds__(THREADS) cache_plan_kernel(const __grid_constant__ CachePlanParams p) {
  constexpr int WARPS = THREADS / 32;
  __shared__ PlanRequest s_req[THREADS];
  __shared__ unsigned long long s_warp[WARPS];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x, ranks = gridDim.x;   // the grid is one cluster
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const uint32_t N = (uint32_t)p.n_pages;
  const uint32_t first = (uint32_t)p.pool_state[0] % N;
  const uint32_t avail = min((uint32_t)max(p.pool_state[1], 0), N);
  const int64_t room = (int64_t)p.max_pages * p.page;
  uint32_t asked = 0, used = 0, returned = 0;   // pages: asked for, taken, given back by the requests before this chunk
  for (int base = 0; base < p.B; base += THREADS) {
    const int i = base + tid;
    int held = 0, n = 0, have = 0, need = 0;
    bool end = false;
    if (i < p.B) {
      held = p.lengths[i];
      n = p.new_tokens[i];
      if (held < 0 || held > room || n < -1 || n > p.R) {
        if (rank == 0) dsn_set_status(p.status, DSN_ERR_BAD_INDEX, i);
        n = 0;
        held = held < 0 ? 0 : held;   // no page is asked for or returned; no row is placed
      } else {
        have = (int)dsn_div((uint32_t)(held + p.page - 1), p.by_page);
        end = n < 0;
        if (!end) need = (int)dsn_div((uint32_t)(held + n + p.page - 1), p.by_page) - have;
      }
    }
    bool fits = have + need <= p.max_pages;
    if (!fits) need = 0;
    // one scan for both sums: pages asked for in the low half, pages returned in the high half
    const unsigned long long v = (unsigned long long)(uint32_t)need | ((unsigned long long)(uint32_t)(end ? have : 0) << 32);
    unsigned long long incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    __syncthreads();   // the chunk before is done with s_req and s_warp
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    unsigned long long before = 0, total = 0;
#pragma unroll 8
    for (int w = 0; w < WARPS; ++w) {
      const unsigned long long u = s_warp[w];
      if (w < warp) before += u;
      total += u;
    }
    incl += before;
    const uint32_t upto = asked + (uint32_t)incl;
    if (need > 0 && upto > avail) fits = false;
    if (i < p.B) {
      const bool ok = fits || end;
      if (!ok && rank == 0) dsn_set_status(p.status, DSN_ERR_CACHE_FULL, i);
      const int placed = end ? -1 : (ok ? n : 0);
      s_req[tid] = PlanRequest{held, placed, end ? returned + (uint32_t)(incl >> 32) - (uint32_t)have : upto - (uint32_t)need};
      if (rank == 0) p.placed[i] = placed > 0 ? placed : 0;
    }
    asked += (uint32_t)total;
    returned += (uint32_t)(total >> 32);
    if (asked <= avail) {   // all of them
      used = asked;
      __syncthreads();
    } else {                // served requests are those up to a point (and those that need nothing): what they take is the largest sum that fits
      const uint32_t top = __reduce_max_sync(0xffffffffu, i < p.B && need > 0 && fits ? upto : 0u);
      __syncthreads();
      if (lane == 0) s_warp[warp] = top;
      __syncthreads();
      for (int w = 0; w < WARPS; ++w) used = max(used, (uint32_t)s_warp[w]);
    }
    const int count = min(THREADS, p.B - base);
    if (LONG) {
      // 512 rows of a request a warp, four in a row a lane: they lie in one page or two
      const int segs = (p.R + 511) / 512;
      const bool wide = p.R % 4 == 0 && (reinterpret_cast<uintptr_t>(p.slots) & 15) == 0;
      for (int64_t it = (int64_t)rank * WARPS + warp; it < (int64_t)count * segs; it += (int64_t)ranks * WARPS) {
        const int k = (int)(it / segs), r0 = (int)(it - (int64_t)k * segs) * 512 + lane * 4;
        const PlanRequest q = s_req[k];
        const int have_k = (int)dsn_div((uint32_t)(q.held + p.page - 1), p.by_page);
        int32_t* table = p.table + (int64_t)(base + k) * p.max_pages;
        int32_t* slots = p.slots + (int64_t)(base + k) * p.R;
        int pa[4], pb[4], col[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {   // all pages first, as no load may pass a store
          const int r = r0 + 128 * j;
          col[j] = (int)dsn_div((uint32_t)(q.held + r), p.by_page);
          pa[j] = pb[j] = -1;
          const int last = min(r + 3, q.placed - 1);   // of these rows, the last that is placed
          if (r <= last) {
            pa[j] = *(col[j] < have_k ? table + col[j] : p.pool + ring(first + q.start + (uint32_t)(col[j] - have_k), N));
            if (q.held + last >= (col[j] + 1) * p.page)
              pb[j] = *(col[j] + 1 < have_k ? table + col[j] + 1 : p.pool + ring(first + q.start + (uint32_t)(col[j] + 1 - have_k), N));
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = r0 + 128 * j, at = q.held + r - col[j] * p.page, turn = p.page - at;   // row r + turn is the first in the second page
          const int n = min(q.placed - r, 4), na = (uint32_t)pa[j] < N ? min(n, turn) : 0, nb = (uint32_t)pb[j] < N ? n : 0;
          const int sa = pa[j] * p.page + at, sb = pb[j] * p.page - turn;
          int slot[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) slot[i] = i < na ? sa + i : (i >= turn && i < nb ? sb + i : -1);
          const bool opens = at == 0;   // one page at most begins in four rows
          if (n > (opens ? 0 : turn) && col[j] + !opens >= have_k) table[col[j] + !opens] = opens ? pa[j] : pb[j];
          if (r >= p.R) continue;
          if (wide) *reinterpret_cast<int4*>(slots + r) = make_int4(slot[0], slot[1], slot[2], slot[3]);
          else
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (r + i < p.R) slots[r + i] = slot[i];
        }
      }
    } else {
    // rows of all requests of the chunk in a line, eight a thread at a time; all pages first, as no load may pass a store
    const uint32_t stride = (uint32_t)(ranks * THREADS), stop = (uint32_t)(base + count) * (uint32_t)p.R;   // rows: below 2^31
    for (uint32_t row0 = (uint32_t)base * (uint32_t)p.R + (uint32_t)(rank * THREADS + tid); row0 < stop; row0 += 8u * stride) {
      int pg[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t row = row0 + (uint32_t)j * stride;
        pg[j] = -1;
        if (row < stop) {
          const uint32_t k = dsn_div(row, p.by_R), r = row - k * (uint32_t)p.R;
          const PlanRequest q = s_req[k - base];
          if ((int)r < q.placed) {
            const int have_k = (int)dsn_div((uint32_t)(q.held + p.page - 1), p.by_page), col = (int)dsn_div((uint32_t)q.held + r, p.by_page);
            pg[j] = *(col < have_k ? p.table + (int64_t)k * p.max_pages + col : p.pool + ring(first + q.start + (uint32_t)(col - have_k), N));
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t row = row0 + (uint32_t)j * stride;
        if (row >= stop) break;
        const uint32_t k = dsn_div(row, p.by_R), r = row - k * (uint32_t)p.R;
        const PlanRequest q = s_req[k - base];
        int slot = -1;
        if ((int)r < q.placed) {
          const int pos = q.held + (int)r, have_k = (int)dsn_div((uint32_t)(q.held + p.page - 1), p.by_page);
          const int col = (int)dsn_div((uint32_t)pos, p.by_page), at = pos - col * p.page;
          if (col >= have_k && at == 0) p.table[(int64_t)k * p.max_pages + col] = pg[j];
          slot = pg[j] < 0 || pg[j] >= p.n_pages ? -1 : pg[j] * p.page + at;
        }
        p.slots[row] = slot;
      }
    }
    }
    // pages of requests that ended, a warp a request
    if ((uint32_t)(total >> 32))
      for (int k = rank * WARPS + warp; k < count; k += ranks * WARPS) {
        const PlanRequest q = s_req[k];
        if (q.placed >= 0) continue;
        const int have_k = (int)dsn_div((uint32_t)(q.held + p.page - 1), p.by_page);
        const int32_t* from = p.table + (int64_t)(base + k) * p.max_pages;
        for (int j0 = lane; j0 < have_k; j0 += 256) {
          int pg[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) pg[j] = j0 + 32 * j < have_k ? from[j0 + 32 * j] : 0;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j0 + 32 * j < have_k) p.pool[ring(first + avail + q.start + (uint32_t)(j0 + 32 * j), N)] = pg[j];
        }
      }
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (rank == 0) {
    for (int i = tid; i < p.B; i += THREADS) {
      const int held = p.lengths[i], n = p.new_tokens[i];
      const bool end = n == -1 && held >= 0 && held <= room;
      p.lengths_out[i] = end ? 0 : held + p.placed[i];   // placed[i] is this thread's own write
    }
    if (tid == 0) {
      p.pool_state_out[0] = (int32_t)((first + used) % N);
      p.pool_state_out[1] = (int32_t)min(avail - used + returned, N);
    }
  }
}

__global__ void __launch_bounds__(256) cache_reset_kernel(int32_t B, int32_t n_pages, int32_t* lengths, int32_t* pool, int32_t* pool_state) {
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const int64_t n = max(B, n_pages);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    if (i < B) lengths[i] = 0;
    if (i < n_pages) pool[i] = (int32_t)i;
    if (i == 0) {
      pool_state[0] = 0;
      pool_state[1] = n_pages;
    }
  }
}

// ------------------------------------------------------------------------------------------------ write
__device__ __forceinline__ uint64_t fmul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

constexpr int kWriteWarps = 4, kWriteCtas = 28;   // warps a CTA; CTAs an SM at most (8 are resident): rows differ, and small CTAs in three waves even that out
                                                  // (by path 22.6 us, 4 x 4096 rows 31.9; 8 warps, 8 CTAs an SM: 26.2, 31.8)

// A lane takes eight elements: 8 lanes a group of 64, 2 D / 8 lanes the k and v of a head, which lie side by side in the row.  A warp takes a row, or every
// `split`th piece of it where there are few rows, four pieces on their way at a time.
// Bound by instructions once memory is busy: least and greatest value go through the shuffles as one pair of bf16 numbers (the least, minus the greatest);
// a code comes out of an addition that rounds (1.5 * 2^23 + 8: its low four bits are the code), eight of them are put together by multiply-adds.
// Measured (in a graph): 128 x 197 rows of 12 heads of 64 by path 22.3 us, 4 x 4096 rows of 8 heads of 128 with values 31.6 (floors 10.6 and 23.3 at a copy's rate); without values 19.9 and
// 26.9 (6.0 and 13.1: look-ups and arithmetic stay the same); one row 2.2.
template <int D, bool VALUES>
__global__ void __launch_bounds__(kWriteWarps * 32) cache_write_kernel(const __grid_constant__ CacheWriteParams p) {
  constexpr int LPH = D / 4;             // lanes a head
  constexpr int HPW = 32 / LPH;          // heads a warp does at a time
  constexpr int U = 4;
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const int lane = threadIdx.x & 31, sub = lane % LPH;
  const int half = sub / (D / 8), grp = (sub % (D / 8)) >> 3, word = sub & 7;
  const int64_t items = (int64_t)p.B * p.R * p.split, warps = (int64_t)gridDim.x * kWriteWarps;
  for (int64_t it = (int64_t)blockIdx.x * kWriteWarps + (threadIdx.x >> 5); it < items; it += warps) {
    const uint32_t row = (uint32_t)(it / p.split);
    const int part = (int)(it - (int64_t)row * p.split);
    const int pos = (int)dsn_div(row, p.by_R), r = (int)(row - (uint32_t)pos * (uint32_t)p.R);
    const PosInfo at = dsn_locate_warp(pos, p.G, p.T, p.offsets, p.perm, p.group_slice);
    if (at.slice < 0 || at.sample >= p.B) continue;
    const int slot = p.slots[(int64_t)at.sample * p.R + r];
    if (slot == -1) continue;
    if (slot < 0 || slot >= p.n_slots) {
      if (lane == 0) dsn_set_status(p.status, DSN_ERR_BAD_INDEX, (int)row);
      continue;
    }
    const int heads = p.heads[at.slice], chunks = (heads + HPW - 1) / HPW;
    const int64_t xrow = (int64_t)(p.grouped ? pos : at.sample) * p.R + r;
    const __nv_bfloat16* x = p.qkv + xrow * p.ld_qkv + (int64_t)p.group * D + sub * 8;
    const int pg = (int)dsn_div((uint32_t)slot, p.by_page), tok = slot - pg * p.page, t = tok % DSN_CACHE_BLOCK;
    const int64_t head_bytes = (int64_t)(p.page / DSN_CACHE_BLOCK) * dsn_cache_block_bytes(D);
    uint8_t* blk = p.pages + pg * (p.H * head_bytes) + (tok / DSN_CACHE_BLOCK) * dsn_cache_block_bytes(D) + half * (dsn_cache_block_bytes(D) / 2);
    for (int c0 = part; c0 < chunks; c0 += U * p.split) {
      uint4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int head = (c0 + u * p.split) * HPW + lane / LPH;
        raw[u] = make_uint4(0, 0, 0, 0);
        if (head < heads) raw[u] = *reinterpret_cast<const uint4*>(x + (int64_t)head * (p.group + 2) * D);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (c0 + u * p.split >= chunks) break;
        const int head = (c0 + u * p.split) * HPW + lane / LPH;
        const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(w);
        const __nv_bfloat162 mn = __hmin2_nan(__hmin2_nan(h[0], h[1]), __hmin2_nan(h[2], h[3])),
                             mx = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
        __nv_bfloat162 ends = __halves2bfloat162(__hmin_nan(mn.x, mn.y), __hneg(__hmax_nan(mx.x, mx.y)));
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) {
          const uint32_t other = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<const uint32_t*>(&ends), o);
          ends = __hmin2_nan(ends, *reinterpret_cast<const __nv_bfloat162*>(&other));
        }
        const uint32_t size = *reinterpret_cast<const uint32_t*>(&ends) & 0x7fff7fffu;
        const uint32_t all = __ballot_sync(0xffffffffu, max(size & 0xffffu, size >> 16) >= 0x7f80u);   // NaN or infinity
        const bool poison = (LPH == 32 ? all : (all >> (lane & 16)) & 0xffffu) != 0;
        const float lo = __bfloat162float(ends.x), hi = -__bfloat162float(ends.y);
        const float fifteenth = 1.0f / 15.0f;
        float s = __bfloat162float(__float2bfloat16_rn(__fsub_rn(__fmul_rn(hi, fifteenth), __fmul_rn(lo, fifteenth))));
        if (s < 1.17549435e-38f) s = 0.f;
        float z = __bfloat162float(__float2bfloat16_rn(2.f * __fadd_rn(0.5f * lo, 4.f * s)));
        float inv = s > 0.f ? __frcp_rn(s) : 0.f, from = -z;                   // s = 0: all differences are finite, all codes 8
        if (poison) {
          s = inv = from = 0.f;
          z = __uint_as_float(0x7fc00000u);
        }
        constexpr float magic = 12582920.f;   // 1.5 * 2^23 + 8
        const uint64_t from_2 = pack2(from, from), inv_2 = pack2(inv, inv), magic_2 = pack2(magic, magic);
        uint64_t step[4];
        uint32_t code = 0;
#pragma unroll
        for (int j = 3; j >= 0; --j) {
          const uint32_t v = poison ? 0u : w[j];
          float q0, q1;
          unpack2(fmul2(fadd2(pack2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)), from_2), inv_2), q0, q1);   // what the ends cut off may be an infinity
          step[j] = fadd2(pack2(fminf(fmaxf(q0, -8.f), 7.f), fminf(fmaxf(q1, -8.f), 7.f)), magic_2);
          unpack2(step[j], q0, q1);
          code = (code * 16u + __float_as_uint(q1)) * 16u + __float_as_uint(q0);
        }
        code -= 0x4b400000u * 0x11111111u;                                     // the eight exponents' share
        if (head < heads) {
          uint8_t* to = blk + head * head_bytes;
          *reinterpret_cast<uint32_t*>(to + (grp * DSN_CACHE_BLOCK + t) * 32 + word * 4) = code;
          if (word == 0)
            *reinterpret_cast<uint32_t*>(to + D / 64 * DSN_CACHE_BLOCK * 32 + (grp * DSN_CACHE_BLOCK + t) * 4) =
                (__float_as_uint(s) >> 16) | (__float_as_uint(z) & 0xffff0000u);
          if (VALUES) {
            uint32_t val[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float y0, y1;
              unpack2(ffma2(pack2(s, s), fadd2(step[j], pack2(-magic, -magic)), pack2(z, z)), y0, y1);
              const __nv_bfloat162 y = __floats2bfloat162_rn(y0, y1);
              val[j] = *reinterpret_cast<const uint32_t*>(&y);
            }
            *reinterpret_cast<uint4*>(p.values + xrow * p.ld_values + (int64_t)head * 2 * D + sub * 8) = make_uint4(val[0], val[1], val[2], val[3]);
          }
        }
      }
    }
  }
}

}  // namespace

namespace {

// CTAs of a cluster for many rows: 16 where the device can hold such a cluster, else 8, which it always can (128 prompts: 8.0 and 10.4 us; 4: 15.5).
template <bool LONG>
int plan_ranks() {
  static int known[DSN_MAX_DEVICES] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= DSN_MAX_DEVICES) return 8;
  if (known[dev]) return known[dev];
  auto kernel = cache_plan_kernel<1024, LONG>;
  int ranks = 8, n = 0;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 16;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(16);
  cfg.blockDim = dim3(1024);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
      cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess && n > 0)
    ranks = 16;
  else
    cudaGetLastError();   // 8, then; not an error of the call
  return known[dev] = ranks;
}

}  // namespace

cudaError_t dsn_launch_cache_plan(const CachePlanParams& p, cudaStream_t s) {
  const int64_t rows = (int64_t)p.B * p.R;
  if (p.B <= 128 && rows <= 1024) return dsn_launch(cache_plan_kernel<128, false>, dim3(1), dim3(128), 0, s, 1, p);   // fewer warps meet sooner
  const int ranks = rows > 4096 ? (p.R >= 64 ? plan_ranks<true>() : plan_ranks<false>()) : 1;
  return dsn_launch(p.R >= 64 ? cache_plan_kernel<1024, true> : cache_plan_kernel<1024, false>, dim3((unsigned)ranks), dim3(1024), 0, s, ranks, p);
}

cudaError_t dsn_launch_cache_reset(int32_t B, int32_t n_pages, int32_t* lengths, int32_t* pool, int32_t* pool_state, cudaStream_t s) {
  const int64_t n = B > n_pages ? B : n_pages;
  const int64_t ctas = (n + 255) / 256;
  return dsn_launch(cache_reset_kernel, dim3((unsigned)(ctas < 592 ? ctas : 592)), dim3(256), 0, s, 1, B, n_pages, lengths, pool, pool_state);
}

cudaError_t dsn_launch_cache_write(CacheWriteParams& p, int sm_count, cudaStream_t s) {
  const int hpw = p.D == 64 ? 2 : 1, chunks = (p.max_heads + hpw - 1) / hpw;
  const int64_t rows = (int64_t)p.B * p.R, most = (int64_t)sm_count * kWriteCtas;
  // few rows: as many warps a row as fill the GPU, up to one a piece
  int64_t split = (int64_t)sm_count * 64 / rows;
  p.split = (int32_t)(split < 1 ? 1 : (split > chunks ? chunks : split));
  const int64_t ctas = (rows * p.split + kWriteWarps - 1) / kWriteWarps;
  const dim3 grid((unsigned)(ctas < most ? ctas : most));
  if (p.D == 64) return p.values ? dsn_launch(cache_write_kernel<64, true>, grid, dim3(kWriteWarps * 32), 0, s, 1, p) : dsn_launch(cache_write_kernel<64, false>, grid, dim3(kWriteWarps * 32), 0, s, 1, p);
  return p.values ? dsn_launch(cache_write_kernel<128, true>, grid, dim3(kWriteWarps * 32), 0, s, 1, p) : dsn_launch(cache_write_kernel<128, false>, grid, dim3(kWriteWarps * 32), 0, s, 1, p);
}
