// Ragged grouped sliced linear layer on 8-bit integers, CTA pairs (tcgen05 cta_group::2, kind::i8, 32-bit integer sums):
//   y = act((sum_c x[c] W[o][c]) * sx[row] * sw[o] + bias, per-path affine, + skip features).
// Tiles, barriers and roles are those of the bf16 pair kernel: a cluster of two CTAs owns a 256-row x BN-column tile, each
// CTA loads its 128 rows and half of the weight tile, the even CTA issues the products of both.  A 128-byte
// row piece holds 128 columns here, an instruction takes 32 of them, and at twice the products per byte the main loop of a
// tile is half as long, so the epilogue weighs twice as much.  A warp of its own prepares tiles ahead: it decodes the tile, folds sw and the
// affine into one factor and one addend a column, and puts them with the rows' scales and places into shared memory (done by the
// epilogue warps themselves, decoding and fetching took 1.7 of their 5.8 thousand cycles a tile); what is left to an element is
// a conversion, a multiplication and a packed multiply-add.
// Bound by the tensor cores where the reduction is long (16,384 rows, 4096 -> 4096: 166 us and 3.3 POP/s, twice the measured bf16 rate, while the power
// allows it, 176 to 195 us in longer runs), by the epilogue where it is short (50,432 rows, 768 -> 2304: 76 us, 2.3 POP/s; the bf16 kernel
// without a bias takes 129 us).  Times are those of calls in a graph.
// Barriers (every CTA has the same layout):
//   full[s]    even CTA only: one arrival (expect_tx for the bytes of both CTAs), completed by the loads of both
//   empty[s]   both CTAs: the multicast commit frees the stage
//   tfull[a]   both CTAs: the accumulator is complete
//   tempty[a]  even CTA only, 2 x 8 arrivals: the epilogue warps of both CTAs
//   ready[a], done[a]  each CTA its own: the prepared tile's hand-over to the epilogue warps and back
// Every wait is bounded; on a timeout the CTA flags DSN_ERR_TIMEOUT and leaves its loops.
#include "dsn_gemm_pair_device.cuh"
#include "dsn_transformer.cuh"

namespace {

using namespace dsn_gemm;

constexpr int kBKB = 128;                          // bytes (= columns) of a chunk
constexpr int kPieces = 4;                         // pieces of 32 columns that an epilogue warp takes of a tile, at most
constexpr int kI8Threads = kThreads + 32;          // one more warp: the tiles' preparation

__device__ __forceinline__ uint32_t mbar_test_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok;
}
__device__ __forceinline__ float relu_nan(float v) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(0.f));
  return r;
}
// GELU for fp32 outputs.  The distribution function by Abramowitz and Stegun's formula 7.1.26 (erf within 1.5e-7):
// erf(z) = 1 - (a1 t + ... + a5 t^5) exp(-z^2), t = 1 / (1 + p z), z >= 0; x Phi(x) = max(x, 0) - |x| q / 2 with q the product.  A fifth of the
// instructions of erff, whose code for a tile's 32 columns kept the warps waiting for instructions.
__device__ __forceinline__ float gelu_f32(float x) {
  const float z = fabsf(x) * 0.70710678118654752f;
  const float t = __fdividef(1.f, fmaf(0.3275911f, z, 1.f));
  float q = fmaf(t, 1.061405429f, -1.453152027f);
  q = fmaf(t, q, 1.421413741f);
  q = fmaf(t, q, -0.284496736f);
  q = fmaf(t, q, 0.254829592f) * t;
  q *= __expf(-z * z);
  return relu_nan(x) - 0.5f * fminf(fabsf(x), 1e30f) * q;   // (infinity: 0 times it would be no number)
}

// What the epilogue reads for a tile besides the accumulator.
struct Prepared {
  float mul[256], add[256];   // per column: sw (and the affine's scale), bias (and the affine's shift)
  float sx[BM];               // per row
  int64_t row[BM];            // output row, -1: not part of the result
  int n0, ncols, map, ko;
};
static_assert(sizeof(Prepared) % 16 == 0, "two in a row, whose factors are read 16 bytes at a time");

// D[tmem] (+)= A[smem] * B[smem]^T on both CTAs' tensor cores, signed 8-bit operands, 32-bit integer sums
__device__ __forceinline__ void umma_i8_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Instruction descriptor: D 32-bit integer, A and B signed 8-bit, both K-major, M x N tile.
__device__ __forceinline__ uint32_t make_idesc_i8(int M, int N) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// first column of piece j of a warp (bf16 rows are stored 64 columns at a time, fp32 rows 32; two warps share a lane quarter)
template <bool F32>
__device__ __forceinline__ int piece_col(int first, int j) {
  return F32 ? 32 * first + 64 * j : 64 * first + 128 * (j >> 1) + 32 * (j & 1);
}

// Skip features, fp32: eight columns of this thread's row.
__device__ __forceinline__ void add_residual(const void* res_row, int c, int ncols, float (&f)[8]) {
  const float* rp = static_cast<const float*>(res_row) + c;
  if (c + 8 <= ncols) {
    const float4 r0 = __ldg(reinterpret_cast<const float4*>(rp)), r1 = __ldg(reinterpret_cast<const float4*>(rp) + 1);
    f[0] += r0.x; f[1] += r0.y; f[2] += r0.z; f[3] += r0.w;
    f[4] += r1.x; f[5] += r1.y; f[6] += r1.z; f[7] += r1.w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < ncols) f[e] += __ldg(rp + e);
  }
}
// Skip features, bf16: 32 columns of this thread's row as they lie in memory, all loads of a piece in flight at once (one after the other they cost a
// trip to memory for every eight columns: 724 samples of 7 rows, 1227 -> 1696 with GELU, 35 -> 31 us; the 32 registers that fp32 takes are not there).
struct Skip {
  uint4 v[4];
  __device__ __forceinline__ void fetch(const void* row, int cb, int ncols) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = cb + 8 * i;
      const uint16_t* at = static_cast<const uint16_t*>(row) + c;
      v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (row == nullptr) continue;
      if (c + 8 <= ncols) {
        v[i] = __ldg(reinterpret_cast<const uint4*>(at));
      } else {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < ncols) w[e >> 1] |= (uint32_t)at[e] << (16 * (e & 1));
        v[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  __device__ __forceinline__ void add(int j, float (&f)[8]) const {   // columns 8 * j .. 8 * j + 7
    const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] += __uint_as_float(w[e] << 16);
      f[2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u);
    }
  }
};

// 32 accumulator columns of this thread's row -> scales, affine, skip features, activation -> the row's 16-byte places from `place` on
// in the warp's staging tile.
template <bool F32, int ACT, bool RES>
__device__ __forceinline__ void epilogue_i8_piece(const uint32_t (&v)[32], int cb, int ncols, float sx, const float* s_mul, const float* s_add,
                                                  const void* res_row, const Skip& skip, uint8_t* stage_w, int lane, int place) {
  const uint64_t sx2 = pack2(sx, sx), zero2 = pack2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < 4; ++j) {   // eight columns at a time
    float f[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 m = reinterpret_cast<const float4*>(s_mul)[2 * j + h], d = reinterpret_cast<const float4*>(s_add)[2 * j + h];
      const int c = 8 * j + 4 * h;
      uint64_t a = ffma2(pack2((float)(int)v[c], (float)(int)v[c + 1]), sx2, zero2);
      uint64_t b = ffma2(pack2((float)(int)v[c + 2], (float)(int)v[c + 3]), sx2, zero2);
      a = ffma2(a, pack2(m.x, m.y), pack2(d.x, d.y));
      b = ffma2(b, pack2(m.z, m.w), pack2(d.z, d.w));
      unpack2(a, f[4 * h], f[4 * h + 1]);
      unpack2(b, f[4 * h + 2], f[4 * h + 3]);
    }
    if (RES && F32 && res_row) add_residual(res_row, cb + 8 * j, ncols, f);
    if (RES && !F32) skip.add(j, f);
#pragma unroll
    for (int c = 0; c < 8; c += 2) {
      if (ACT == DSN_ACT_RELU) {
        f[c] = relu_nan(f[c]);
        f[c + 1] = relu_nan(f[c + 1]);
      } else if (ACT == DSN_ACT_GELU) {
        if (F32) {
          f[c] = gelu_f32(f[c]);
          f[c + 1] = gelu_f32(f[c + 1]);
        } else {
          gelu_pair(f[c], f[c + 1], f[c], f[c + 1]);
        }
      }
    }
    if (F32) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<float4*>(stage_w + lane * 128 + (((place + 2 * j + h) ^ (lane & 7)) << 4)) =
            make_float4(f[4 * h], f[4 * h + 1], f[4 * h + 2], f[4 * h + 3]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
        w[e] = *reinterpret_cast<uint32_t*>(&b);
      }
      *reinterpret_cast<uint4*>(stage_w + lane * 128 + (((place + j) ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// The staged piece (32 rows x 128 bytes, swizzled; columns c0 .. of the tile) leaves: one TMA store where the rows are consecutive, else
// eight lanes a row.  Columns that a TMA store cannot clip (its granule is 16 bytes) are written by every lane for its own row.
template <bool F32>
__device__ __forceinline__ void store_piece(uint8_t* stage_w, char* yrow, int c0, int ncols, int n0, int lane, bool contig, const CUtensorMap* mapY, int base_row) {
  constexpr int W = F32 ? 32 : 64;          // columns of a staged piece
  constexpr int G = F32 ? 4 : 8;            // columns of 16 bytes
  constexpr int ES = F32 ? 4 : 2;
  const int last = ncols - c0 < W ? ncols - c0 : W;
  if (contig) {
    fence_async_smem();
    __syncwarp();
    if (elect_one()) {
      tma_store_2d(mapY, n0 + c0, base_row, smem_u32(stage_w));
      bulk_commit();
    }
    const int whole = last & ~(G - 1);
    if (whole != last) {
      const uint8_t* sp = stage_w + lane * 128 + (((whole / G) ^ (lane & 7)) << 4);
      for (int e = 0; e < last - whole; ++e) {
        if (F32) reinterpret_cast<float*>(yrow)[c0 + whole + e] = reinterpret_cast<const float*>(sp)[e];
        else reinterpret_cast<uint16_t*>(yrow)[c0 + whole + e] = reinterpret_cast<const uint16_t*>(sp)[e];
      }
    }
  } else {
    __syncwarp();
    const int j = lane & 7;
#pragma unroll
    for (int i = 0; i < 8; ++i) {          // eight lanes a row, 16 bytes each
      const int row = 4 * i + (lane >> 3);
      char* rp = reinterpret_cast<char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(yrow), row));
      if (rp != nullptr && G * j < last) {
        const uint8_t* sp = stage_w + row * 128 + ((j ^ (row & 7)) << 4);
        char* dst = rp + (int64_t)(c0 + G * j) * ES;
        if (G * j + G <= last) {
          *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(sp);
        } else {
          for (int e = 0; e < last - G * j; ++e) {
            if (F32) reinterpret_cast<float*>(dst)[e] = reinterpret_cast<const float*>(sp)[e];
            else reinterpret_cast<uint16_t*>(dst)[e] = reinterpret_cast<const uint16_t*>(sp)[e];
          }
        }
      }
    }
    __syncwarp();
  }
}

// Epilogue of one tile for one warp.  The next piece's columns are on their way from TMEM while a piece is worked on, and the accumulator
// goes back to the issuing warp (`tempty`, in the even CTA) as soon as the last of them have arrived.
template <bool F32, int ACT, bool RES>
__device__ __forceinline__ void epilogue_i8_tile(uint32_t taddr, int ncols, int n0, int first, float sx, const void* res_row,
                                                 uint8_t* stage_w, const Prepared* prep, char* yrow, int lane, bool contig, const CUtensorMap* mapY, int base_row,
                                                 uint32_t tempty, int bn) {
  // Loads run whether a piece exists or not (a missing one reads the tile's last columns again): straight code keeps the two blocks of 32
  // registers in place.
  auto load = [&](int j, uint32_t (&v)[32]) {
    const int cb = piece_col<F32>(first, j);
    tmem_ld_32x32(taddr + (cb + 32 <= bn ? cb : bn - 32), v);
  };
  Skip skip;   // (left alone where there are no bf16 skip features)
  auto work = [&](const int j, const uint32_t (&v)[32]) {
    const int cb = piece_col<F32>(first, j);
    if (cb < ncols) {
      if (F32 || !(j & 1)) {                  // a new staging tile: an earlier store of this warp has read it
        if (elect_one()) bulk_wait_read0();
        __syncwarp();
      }
      epilogue_i8_piece<F32, ACT, RES>(v, cb, ncols, sx, prep->mul + cb, prep->add + cb, res_row, skip, stage_w, lane, (F32 || !(j & 1)) ? 0 : 4);
      if (F32 || (j & 1) || piece_col<F32>(first, j + 1) >= ncols)
        store_piece<F32>(stage_w, yrow, F32 ? cb : (cb & ~63), ncols, n0, lane, contig, mapY, base_row);
    }
  };
  if constexpr (RES && !F32) {
    uint32_t v[32];
#pragma unroll 1   // one block of accumulator columns beside one of skip features: the registers do not hold two of both
    for (int j = 0; j < kPieces; ++j) {
      load(j, v);
      if (piece_col<F32>(first, j) < ncols) skip.fetch(res_row, piece_col<F32>(first, j), ncols);
      tmem_ld_wait();
      if (j + 1 == kPieces) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(tempty);
      }
      work(j, v);
    }
    return;
  }
  uint32_t va[32], vb[32];
  load(0, va);
#pragma unroll 1   // two pieces a round: the code of four side by side waited for instructions
  for (int j = 0; j < kPieces; j += 2) {
    tmem_ld_wait();
    load(j + 1, vb);
    work(j, va);
    tmem_ld_wait();
    if (j + 2 < kPieces) {
      load(j + 2, va);
    } else {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(tempty);
    }
    work(j + 1, vb);
  }
}

template <bool F32, bool RES>
__global__ void __launch_bounds__(kI8Threads, 1) gemm_i8_pair_kernel(const __grid_constant__ GemmI8Params P) {
  extern __shared__ uint8_t smem_raw[];
  const GemmParams& p = P.g;
  const GemmGeom& g = p.g;
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw);

  const uint32_t bar_full = base;
  const uint32_t bar_empty = base + 8 * kMaxStages;
  const uint32_t bar_tfull = base + 16 * kMaxStages;
  const uint32_t bar_tempty = bar_tfull + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 16 * kMaxStages + 32);
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + 16 * kMaxStages + 36);
  const uint32_t bar_ready = base + 16 * kMaxStages + 48, bar_done = bar_ready + 16;

  const int stages = g.stages;
  const uint32_t bh_bytes = (uint32_t)(g.BN / 2) * kBKB;  // this CTA's half of the weight tile
  const uint32_t stage_bytes = kABytes + bh_bytes;        // kABytes: 128 rows of 128 bytes
  const uint32_t tiles_base = base + kCtrlBytes;
  uint8_t* out_stage = smem + kCtrlBytes + (size_t)stages * stage_bytes;
  Prepared* prepared = reinterpret_cast<Prepared*>(out_stage + kStageOutBytes);
  int32_t* s_prefix = reinterpret_cast<int32_t*>(prepared + 2);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const uint32_t tmem_cols = 2u * (uint32_t)g.BN;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(bar_tfull + 8 * a, 1);
      mbar_init(bar_tempty + 8 * a, 2 * kEpiWarps);
      mbar_init(bar_ready + 8 * a, 1);
      mbar_init(bar_done + 8 * a, kEpiWarps);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(tmem_slot), tmem_cols);
    tmem_relinquish_pair();
  }

  // The CTAs of the pair meet in two halves: what they announce (initialised barriers) is taken up only after the tile table, which hides
  // the 700 cycles of the meeting.
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  // barriers and TMEM are set up; everything below reads what earlier kernels wrote
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  // s_prefix[0..G]: tile prefix; [G+1 .. 2G+1]: group offsets; [2G+2 .. 3G+1]: slice of each group (one trip to memory for all three)
  dsn_build_tile_prefix(p.G, s_prefix, [&](int grp) {
    const int sl = p.group_slice ? p.group_slice[grp] : grp;
    const int lo = p.offsets[grp], hi = p.offsets[grp + 1];
    const bool known = sl >= 0 && sl < p.T;
    s_prefix[p.G + 1 + grp] = lo;
    if (grp == p.G - 1) s_prefix[2 * p.G + 1] = hi;
    s_prefix[2 * p.G + 2 + grp] = known ? sl : 0;
    if (!known || p.map_id[sl] == 0xFF || hi <= lo) return 0;
    const int mt = g.flat ? ((hi - lo) * g.R + BM - 1) / BM : ((hi - lo + g.nb - 1) / g.nb) * g.tiles_x * g.tiles_y;
    return ((mt + 1) / 2) * ((p.k_out[sl] + g.BN - 1) / g.BN);
  });
  tc_fence_before();
  __syncthreads();
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");  // the peer's barriers are initialised before anything can arrive on them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int total = s_prefix[p.G];
  PairCursor cursor;  // every role walks its own tile sequence

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer (both CTAs)
    int stage = 0;
    uint32_t phase = 0;
    const uint32_t a_box_bytes = (uint32_t)(g.bw * g.bh * g.nb) * kBKB;
    const uint32_t tx_bytes = 2u * (a_box_bytes + bh_bytes);
    bool ok = true;
    for (int tile = pair; ok && tile < total; tile += npairs) {
      const PairTile t = decode_pair_tile(p, s_prefix, tile, rank, cursor);
      const CUtensorMap* mA = &p.mapA[t.map];
      const CUtensorMap* mB = &p.mapB[t.map];
      const int nkc = (t.ki + kBKB - 1) / kBKB;
      const int n_inst = (t.ncols + 31) & ~31;
      const int brow0 = t.n0 + rank * (n_inst >> 1);  // first weight row of this CTA's half
      int bsel = t.b0;
      if (g.a_input_order) bsel = t.b0 < t.p_end ? p.perm[t.b0] : p.B;  // past the group: out of range, zeros
      const int cx = g.flat ? t.row0 : t.x0, cb = g.flat ? 0 : bsel;
      for (int kc = 0; kc < nkc; ++kc) {
        ok = __all_sync(0xffffffffu, dsn_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, p.status, 61));
        if (!ok) break;
        if (elect_one()) {
          const uint32_t full_lead = leader_addr(bar_full + 8 * stage);  // the even CTA's barrier
          if (rank == 0) mbar_expect_tx(bar_full + 8 * stage, tx_bytes);
          const uint32_t sa = tiles_base + stage * stage_bytes;
          tma_load_4d_pair(sa, mA, kc * kBKB, cx, 0, cb, full_lead);
          tma_load_3d_pair(sa + kABytes, mB, kc * kBKB, 0, brow0, full_lead);
        }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (even CTA only)
    if (rank == 0) {
      int stage = 0;
      uint32_t phase = 0;
      int it = 0;
      bool ok = true;
      const uint64_t da0 = make_smem_desc(tiles_base), db0 = make_smem_desc(tiles_base + kABytes);
      const uint64_t dstep = (uint64_t)(stage_bytes >> 4);
      uint64_t da = da0, db = db0;
      for (int tile = pair; ok && tile < total; tile += npairs, ++it) {
        const PairTile t = decode_pair_tile(p, s_prefix, tile, 0, cursor);
        const int acc = it & 1;
        const uint32_t acc_phase = (uint32_t)(it >> 1) & 1u;
        ok = __all_sync(0xffffffffu, dsn_wait(bar_tempty + 8 * acc, acc_phase ^ 1u, abort_flag, p.status, 62));
        if (!ok) break;
        tc_fence_after();
        const uint32_t idesc = make_idesc_i8(2 * BM, (t.ncols + 31) & ~31);
        const uint32_t d_tmem = tmem_base + (uint32_t)(acc * g.BN);
        const int tail_ks = ((t.ki & (kBKB - 1)) + 31) >> 5;  // K steps of a partial last chunk (0: none)
        uint32_t accumulate = 0;
        const int whole = t.ki >> 7;                          // chunks of 128 columns
        // The next stage's barrier is looked at before this stage's products are issued (64 rows of 4096 -> 4096, where 32 chunks are issued one
        // after the other: 12.7 -> 11.7 us).  A look, not a wait: try_wait would hold the warp for microseconds at a barrier of no tile.
        uint32_t here = mbar_test_wait(bar_full + 8 * stage, phase);
        for (int kc = 0; kc < whole + (tail_ks ? 1 : 0); ++kc) {
          if (!__all_sync(0xffffffffu, here)) {
            ok = __all_sync(0xffffffffu, dsn_wait(bar_full + 8 * stage, phase, abort_flag, p.status, 63));
            if (!ok) break;
          }
          tc_fence_after();
          const uint32_t this_empty = bar_empty + 8 * stage;
          const uint64_t ca = da, cb = db;
          da += dstep;
          db += dstep;
          if (++stage == stages) { stage = 0; phase ^= 1u; da = da0; db = db0; }
          here = mbar_test_wait(bar_full + 8 * stage, phase);
          if (kc < whole) {
            if (elect_one()) {
              umma_i8_pair(d_tmem, ca, cb, idesc, accumulate);  // +32 bytes per K step
              umma_i8_pair(d_tmem, ca + 2u, cb + 2u, idesc, 1u);
              umma_i8_pair(d_tmem, ca + 4u, cb + 4u, idesc, 1u);
              umma_i8_pair(d_tmem, ca + 6u, cb + 6u, idesc, 1u);
              umma_commit_pair(this_empty);
            }
          } else if (elect_one()) {
            umma_i8_pair(d_tmem, ca, cb, idesc, accumulate);
            if (tail_ks > 1) umma_i8_pair(d_tmem, ca + 2u, cb + 2u, idesc, 1u);
            if (tail_ks > 2) umma_i8_pair(d_tmem, ca + 4u, cb + 4u, idesc, 1u);
            if (tail_ks > 3) umma_i8_pair(d_tmem, ca + 6u, cb + 6u, idesc, 1u);
            umma_commit_pair(this_empty);
          }
          accumulate = 1;
        }
        if (ok && elect_one()) umma_commit_pair(bar_tfull + 8 * acc);
      }
    }
  } else if (warp == 2 + kEpiWarps) {
    // ------------------------------------------------------------------ preparation (both CTAs): four rows and eight columns a lane
    int it = 0;
    for (int tile = pair; tile < total; tile += npairs, ++it) {
      const PairTile t = decode_pair_tile(p, s_prefix, tile, rank, cursor);
      float mul[8], add[8], sx[4];
      int64_t row[4];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = 32 * j + lane;
        mul[j] = add[j] = 0.f;
        if (c < t.ncols) {
          mul[j] = __ldg(P.w_scale + t.n0 + c);
          if (p.bias) add[j] = __ldg(p.bias + t.n0 + c);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int m = 32 * j + lane;
        int pp, r;   // position and row inside the sample
        bool valid;
        if (g.flat) {
          const int gr = t.row0 + m;
          valid = gr < t.rows_end;
          pp = (int)dsn_div((uint32_t)gr, P.by_R);
          r = gr - pp * g.R;
        } else {
          const int bi = g.nb == 1 ? 0 : m / g.bw;
          r = t.x0 + (m - bi * g.bw);
          pp = t.b0 + bi;
          valid = m < g.bw * g.nb && r < g.R && pp < t.p_end;
        }
        sx[j] = 0.f;
        row[j] = -1;
        if (valid) {
          const int smp = (g.y_input_order || P.scale_input_order) ? p.perm[pp] : 0;
          row[j] = (int64_t)(g.y_input_order ? smp : pp) * g.R + r;
          sx[j] = __ldg(P.x_scale + (int64_t)(P.scale_input_order ? smp : pp) * g.R + r);
        }
      }
      if (p.bn_scale) {
        const int64_t at = (int64_t)t.slice * p.bn_ld + t.n0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = 32 * j + lane;
          if (c < t.ncols) {
            const float sc = __ldg(p.bn_scale + at + c);
            mul[j] *= sc;
            add[j] = fmaf(add[j], sc, __ldg(p.bn_shift + at + c));
          }
        }
      }
      const int b = it & 1;
      if (!__all_sync(0xffffffffu, dsn_wait(bar_done + 8 * b, ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag, p.status, 65))) break;
      Prepared& o = prepared[b];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o.mul[32 * j + lane] = mul[j];
        o.add[32 * j + lane] = add[j];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        o.sx[32 * j + lane] = sx[j];
        o.row[32 * j + lane] = row[j];
      }
      if (lane == 0) {
        o.n0 = t.n0;
        o.ncols = t.ncols;
        o.map = t.map;
        o.ko = t.ko;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_ready + 8 * b);
    }
  } else {
    // ------------------------------------------------------------------ epilogue (warps 2..9, both CTAs)
    const int q = warp & 3;
    const int first = (warp - 2) >> 2;
    const int m = q * 32 + lane;
    int it = 0;
    bool ok = true;
    const int es = F32 ? 4 : 2;
    uint8_t* stage_w = out_stage + (warp - 2) * (32 * 128);
    for (int tile = pair; ok && tile < total; tile += npairs, ++it) {
      const int acc = it & 1;
      const uint32_t acc_phase = (uint32_t)(it >> 1) & 1u;
      ok = __all_sync(0xffffffffu, dsn_wait(bar_ready + 8 * acc, acc_phase, abort_flag, p.status, 66));
      if (!ok) break;
      const Prepared* prep = prepared + acc;
      const float sx = prep->sx[m];
      const int64_t out_row = prep->row[m];
      const bool valid = out_row >= 0;
      const int n0 = prep->n0, ncols = prep->ncols;
      char* yrow = valid ? reinterpret_cast<char*>(p.y) + (out_row * p.ldy + n0) * es : nullptr;
      const void* res_row = (RES && valid) ? reinterpret_cast<const char*>(p.residual) + (out_row * p.ldy + n0) * es : nullptr;
      const long long base_row = __shfl_sync(0xffffffffu, (long long)out_row, 0);
      const bool contig = __all_sync(0xffffffffu, valid && out_row == base_row + lane) && prep->ko >= 8;

      ok = __all_sync(0xffffffffu, dsn_wait(bar_tfull + 8 * acc, acc_phase, abort_flag, p.status, 64));
      if (!ok) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * g.BN);
      const CUtensorMap* mY = &p.mapY[prep->map];
      const uint32_t tempty = leader_addr(bar_tempty + 8 * acc);   // the even CTA's issuing warp waits on it
      switch (p.act) {
        case DSN_ACT_NONE: epilogue_i8_tile<F32, DSN_ACT_NONE, RES>(taddr, ncols, n0, first, sx, res_row, stage_w, prep, yrow, lane, contig, mY, (int)base_row, tempty, g.BN); break;
        case DSN_ACT_RELU: epilogue_i8_tile<F32, DSN_ACT_RELU, RES>(taddr, ncols, n0, first, sx, res_row, stage_w, prep, yrow, lane, contig, mY, (int)base_row, tempty, g.BN); break;
        default: epilogue_i8_tile<F32, DSN_ACT_GELU, RES>(taddr, ncols, n0, first, sx, res_row, stage_w, prep, yrow, lane, contig, mY, (int)base_row, tempty, g.BN); break;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_done + 8 * acc);
    }
    if (elect_one()) bulk_wait0();  // the lane that issued this warp's TMA stores
  }

  // ------------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // neither CTA retires while its partner may still read its memory or signal its barriers
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, tmem_cols);
  }
}

}  // namespace

size_t dsn_gemm_i8_smem_bytes(int BN, int stages, int G) {
  return 1024 + kCtrlBytes + (size_t)stages * (kABytes + (size_t)(BN / 2) * kBKB) + kStageOutBytes + 2 * sizeof(Prepared) + sizeof(int32_t) * (3 * (size_t)G + 3);
}

cudaError_t dsn_launch_gemm_i8(const GemmI8Params& p, int f32, int clusters, size_t smem_bytes, cudaStream_t s) {
  static size_t configured[4][DSN_MAX_DEVICES] = {};
  const int form = (f32 ? 2 : 0) + (p.g.residual ? 1 : 0);
  void (*kernel)(GemmI8Params) = form == 3 ? gemm_i8_pair_kernel<true, true>
                                 : form == 2 ? gemm_i8_pair_kernel<true, false>
                                 : form == 1 ? gemm_i8_pair_kernel<false, true> : gemm_i8_pair_kernel<false, false>;
  const cudaError_t e = dsn_ensure_dynamic_smem(kernel, smem_bytes, configured[form]);
  if (e != cudaSuccess) return e;
  return dsn_launch(kernel, dim3(2 * clusters), dim3(kI8Threads), smem_bytes, s, 2, p);
}
