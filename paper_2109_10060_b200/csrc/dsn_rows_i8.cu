// Linear layer on 8-bit codes for a few rows in all (single tokens of a small batch): y = act(sx sw sum x W + ...).
// Bound by the bytes of the weights, which are read once for all rows.  A CTA owns 16 output channels, its eight warps
// split the reduction and meet in shared memory (integers: any order gives the same sum).  The products go through
// the warp-level 8-bit matrix instruction (16 channels x 8 rows x 32 columns): at most 32 rows cannot fill the 128 rows of a
// tensor-memory tile, and this form takes its operands straight from registers.  The order of the columns inside a sum
// is free, so a lane's 16 consecutive bytes serve as its pieces of two instructions, the same way for weights and rows.
// One row of 4096 x 4096 takes 4.8 us in a graph, weights in L2, against 2.6 for its bytes (launch, one round trip to memory and the meeting are the
// rest), 32 rows 6.5 us; from 33 rows on the tensor-memory form is the faster one (64 rows: 11.3 us, with eight tiles of rows here 19.4).  Weights that
// come from memory: one row of 8192 x 8192 16.5 us against 10.2.
// Rows of narrower paths are zero beyond their k_in, so all rows share one reduction over the widest path's columns.
#include "dsn_transformer.cuh"

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
// Steps of 64 columns whose weights a warp has in flight.  One row, 4096 x 4096 from L2: 4.7, 5.3, 5.7 us with 1, 2, 4 (more registers, fewer CTAs an
// SM); 8192 x 8192 from memory: 17.5, 17.3, 26.5 us; 16 rows of 4096 x 8192: 17.0, 16.4, 16.2 us.
constexpr int kAhead = 2;

struct RowInfo {
  int64_t src, dst;   // rows of x and y; dst < 0: the row does not exist
  float sx;
  int ki, ko, slice;
};

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The bytes off .. off + 15 of a row, zero at and beyond `end`.  (Out of line: inlined at each of the loads, the byte-wise end of a row was most
// of the kernel's code.)
__device__ __noinline__ uint4 load_end(const int8_t* row, int off, int end) {
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (off + i < end) w[i >> 2] |= (uint32_t)(uint8_t)row[off + i] << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 load16(const int8_t* row, int off, int end) {
  if (off + 16 <= end) return __ldg(reinterpret_cast<const uint4*>(row + off));
  if (off >= end) return make_uint4(0u, 0u, 0u, 0u);
  return load_end(row, off, end);
}

// NT tiles of eight rows.
template <bool F32, int NT>
__global__ void __launch_bounds__(kThreads) rows_i8_kernel(const __grid_constant__ RowsI8Params p) {
  __shared__ RowInfo info[8 * NT];
  __shared__ int part[kWarps][8 * NT][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, q = lane & 3;
  const int o0 = blockIdx.x * 16;
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  // channels beyond the last read the last one's weights: their sums go nowhere
  const int top = p.max_ko - 1;
  const int8_t* w0 = p.W + (int64_t)(o0 + g < top ? o0 + g : top) * p.ldw + 16 * q;
  const int8_t* w1 = p.W + (int64_t)(o0 + g + 8 < top ? o0 + g + 8 : top) * p.ldw + 16 * q;
  const int whole = p.max_ki >> 6;       // steps that lie inside the widest path
  uint4 a0[kAhead], a1[kAhead];
  auto fetch = [&](int j, int st) {
    if (st < whole) {
      a0[j] = __ldg(reinterpret_cast<const uint4*>(w0 + 64 * st));
      a1[j] = __ldg(reinterpret_cast<const uint4*>(w1 + 64 * st));
    }
  };
#pragma unroll
  for (int j = 0; j < kAhead; ++j) fetch(j, warp + j * kWarps);   // the weights do not wait for the rows' paths
  // this thread's output channel at the end is the same for all of its rows
  const int o = o0 + (threadIdx.x & 15);
  const float sw = o < p.max_ko ? __ldg(p.w_scale + o) : 0.f, bias = (p.bias && o < p.max_ko) ? __ldg(p.bias + o) : 0.f;
  const int rows = p.B * p.R;
  if (warp == 0) {   // one row a lane
    RowInfo ri{0, -1, 0.f, 0x7fffffff, 0, 0};   // a row that does not exist reads the first one's codes: its sums go nowhere
    const int pos = lane < rows ? lane / p.R : p.B, r = lane - pos * p.R;
    const PosInfo at = dsn_locate_lanes(pos, p.B, p.G, p.T, p.offsets, p.perm, p.group_slice);
    if (at.slice >= 0) {
      ri.src = (int64_t)(p.in_input_order ? at.sample : pos) * p.R + r;
      ri.dst = (int64_t)(p.out_input_order ? at.sample : pos) * p.R + r;
      ri.sx = p.x_scale[ri.src];
      ri.ki = p.k_in[at.slice];
      ri.ko = p.k_out[at.slice];
      ri.slice = at.slice;
    }
    if (lane < 8 * NT) info[lane] = ri;
  }
  __syncthreads();
  const int8_t* xr[NT];
  int xe[NT], least = p.max_ki;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    xr[n] = p.x + info[8 * n + g].src * p.ldx;
    xe[n] = info[8 * n + g].ki < p.max_ki ? info[8 * n + g].ki : p.max_ki;
    least = xe[n] < least ? xe[n] : least;
  }
  least = __reduce_min_sync(0xffffffffu, least);   // columns that every row has
  int c[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) c[n][i] = 0;
  for (int base = warp; base < whole; base += kAhead * kWarps) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int st = base + j * kWarps, off = 64 * st + 16 * q;
      if (st < whole) {
        uint4 b[NT];
        if (64 * st + 64 <= least) {
#pragma unroll
          for (int n = 0; n < NT; ++n) b[n] = __ldg(reinterpret_cast<const uint4*>(xr[n] + off));
        } else {
#pragma unroll
          for (int n = 0; n < NT; ++n) b[n] = load16(xr[n], off, xe[n]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_s8(c[n], a0[j].x, a1[j].x, a0[j].y, a1[j].y, b[n].x, b[n].y);
          mma_s8(c[n], a0[j].z, a1[j].z, a0[j].w, a1[j].w, b[n].z, b[n].w);
        }
        fetch(j, st + kAhead * kWarps);   // this slot's next step
      }
    }
  }
  if ((p.max_ki & 63) && warp == (whole & (kWarps - 1))) {   // the step that the widest path ends in
    const int off = 64 * whole + 16 * q;
    const uint4 a = load16(w0 - 16 * q, off, p.max_ki), a8 = load16(w1 - 16 * q, off, p.max_ki);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint4 b = load16(xr[n], off, xe[n]);
      mma_s8(c[n], a.x, a8.x, a.y, a8.y, b.x, b.y);
      mma_s8(c[n], a.z, a8.z, a.w, a8.w, b.z, b.w);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {   // accumulator: channels g and g + 8, rows 2 q and 2 q + 1 of the tile
    part[warp][8 * n + 2 * q][g] = c[n][0];
    part[warp][8 * n + 2 * q + 1][g] = c[n][1];
    part[warp][8 * n + 2 * q][g + 8] = c[n][2];
    part[warp][8 * n + 2 * q + 1][g + 8] = c[n][3];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 16 * 8 * NT; e += kThreads) {
    const int row = e >> 4, ch = e & 15;
    const RowInfo ri = info[row];
    if (ri.dst < 0 || o >= ri.ko) continue;
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) sum += part[i][row][ch];
    float v = fmaf((float)sum * ri.sx, sw, bias);
    if (p.bn_scale) v = fmaf(v, p.bn_scale[(int64_t)ri.slice * p.bn_ld + o], p.bn_shift[(int64_t)ri.slice * p.bn_ld + o]);
    const int64_t at = ri.dst * p.ldy + o;
    if (p.residual) v += F32 ? static_cast<const float*>(p.residual)[at] : __bfloat162float(static_cast<const __nv_bfloat16*>(p.residual)[at]);
    if (p.act == DSN_ACT_RELU) asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(v), "f"(0.f));   // a NaN stays visible
    if (p.act == DSN_ACT_GELU) v = 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
    if (F32) static_cast<float*>(p.y)[at] = v; else static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
  }
}

// Rows of short samples from input order to grouped order, 16 bytes a thread; a piece that runs past its row's k_in takes along
// what lies there (the products' loads stop at k_in), except behind the very last row, where nothing need be allocated.
__global__ void __launch_bounds__(kThreads) gather_i8_kernel(const __grid_constant__ RowsI8Params p, int8_t* dst, int64_t ld, FastDiv by_pieces, FastDiv by_R) {
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const uint64_t e = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
  if (e >= (uint64_t)p.B * p.R * by_pieces.d) return;
  const uint32_t row = e < 0x80000000ull ? dsn_div((uint32_t)e, by_pieces) : (uint32_t)(e / by_pieces.d);
  const int c = 16 * (int)(e - (uint64_t)row * by_pieces.d);
  const int pos = (int)dsn_div(row, by_R), r = (int)(row - (uint32_t)pos * (uint32_t)p.R);
  const PosInfo at = dsn_locate(pos, p.G, p.T, p.offsets, p.perm, p.group_slice);
  if (at.slice < 0 || c >= p.k_in[at.slice]) return;
  const int64_t from = (int64_t)at.sample * p.R + r;
  const int8_t* s = p.x + from * p.ldx;
  const bool tight = from + 1 == (int64_t)p.B * p.R;
  *reinterpret_cast<uint4*>(dst + (int64_t)row * ld + c) = load16(s, c, tight ? p.C_in : (int)ld);
}

template <bool F32>
cudaError_t pick(const RowsI8Params& p, cudaStream_t s) {
  const dim3 grid((p.max_ko + 15) / 16), block(kThreads);
  const int rows = p.B * p.R;
  if (rows <= 8) return dsn_launch(rows_i8_kernel<F32, 1>, grid, block, 0, s, 1, p);
  if (rows <= 16) return dsn_launch(rows_i8_kernel<F32, 2>, grid, block, 0, s, 1, p);
  return dsn_launch(rows_i8_kernel<F32, 4>, grid, block, 0, s, 1, p);
}

}  // namespace

cudaError_t dsn_launch_rows_i8(const RowsI8Params& p, int f32, cudaStream_t s) {
  return f32 ? pick<true>(p, s) : pick<false>(p, s);
}

cudaError_t dsn_launch_gather_i8(const RowsI8Params& p, int8_t* dst, int64_t ld, cudaStream_t s) {
  const uint32_t pieces = (uint32_t)((p.max_ki + 15) / 16);
  const int64_t n = (int64_t)p.B * p.R * pieces;
  return dsn_launch(gather_i8_kernel, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, 1, p, dst, ld, dsn_fast_div(pieces),
                    dsn_fast_div((uint32_t)p.R));
}
