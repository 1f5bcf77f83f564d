// Attention over the 4-bit cache, many rows.
#include "dsn_cache.cuh"

namespace {

// One warp a query vector; 32 keys at a time, a lane a key for the scores, a lane D / 32 elements for the values.
template <int D>
__global__ void __launch_bounds__(128) cache_attention_simple(const __grid_constant__ CacheAttParams p) {
  constexpr int E = D / 32;
  __shared__ float s_q[4][D];
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t per_row = (int64_t)p.max_heads * p.group, items = (int64_t)p.B * p.R * per_row;
  const uint32_t block = dsn_cache_block_bytes(D);
  for (int64_t it = (int64_t)blockIdx.x * 4 + warp; it < items; it += (int64_t)gridDim.x * 4) {
    const int64_t row = it / per_row;
    const int vec = (int)(it - row * per_row), head = vec / p.group, e = vec - head * p.group;
    const int pos = (int)(row / p.R), r = (int)(row - (int64_t)pos * p.R);
    const PosInfo at = dsn_locate_warp(pos, p.G, p.T, p.offsets, p.perm, p.group_slice);
    if (at.slice < 0 || at.sample >= p.B || head >= p.heads[at.slice]) continue;
    const int most = p.max_pages * p.page;
    const int len_in = p.lengths[at.sample], n_in = p.placed ? p.placed[at.sample] : p.R;
    const int L = min(max(len_in, 0), most), n = min(max(n_in, 0), p.R);
    if ((L != len_in || n != n_in) && lane == 0) dsn_set_status(p.status, DSN_ERR_BAD_INDEX, at.sample);
    if (r >= n) continue;
    const int64_t xrow = (int64_t)(p.grouped ? pos : at.sample) * p.R + r;
    const __nv_bfloat16* q = p.qkv + xrow * p.ld_qkv + ((int64_t)head * (p.group + 2) + e) * D;
    __syncwarp();
    for (int j = lane; j < D; j += 32) s_q[warp][j] = __bfloat162float(q[j]);
    __syncwarp();
    const int me = L - n + r;                                   // this query's token
    const int lo = p.window ? max(0, me - p.window + 1) : 0;
    float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
    for (int j = 0; j < E; ++j) o[j] = 0.f;
    for (int k0 = lo & ~15; k0 <= me; k0 += 32) {
      const int key = k0 + lane;
      const int col = key / p.page;
      const int pg = key <= me ? p.table[(int64_t)at.sample * p.max_pages + col] : 0;
      bool seen = key >= lo && key <= me;
      if (seen && (pg < 0 || pg >= p.n_pages)) {
        dsn_set_status(p.status, DSN_ERR_BAD_INDEX, at.sample);
        seen = false;
      }
      const int tok = key - col * p.page;
      const uint8_t* blk = p.pages + (((int64_t)(seen ? pg : 0) * p.H + head) * (p.page / 16) + (seen ? tok / 16 : 0)) * block;
      const int t = tok & 15;
      float sc = -INFINITY;
      if (seen) {
        sc = 0.f;
        for (int g = 0; g < D / 64; ++g) {
          const uint32_t pr = *reinterpret_cast<const uint32_t*>(blk + D / 64 * 512 + (g * 16 + t) * 4);
          float dot = 0.f, sum = 0.f;
          for (int w = 0; w < 8; ++w) {
            const uint32_t c = *reinterpret_cast<const uint32_t*>(blk + (g * 16 + t) * 32 + w * 4);
            for (int j = 0; j < 8; ++j) {
              const float qv = s_q[warp][g * 64 + w * 8 + j];
              dot = fmaf(qv, (float)((int)((c >> (4 * j)) & 15) - 8), dot);
              sum += qv;
            }
          }
          sc += dot * __uint_as_float(pr << 16) + sum * __uint_as_float(pr & 0xffff0000u);
        }
        sc *= p.scale_log2;
      }
      float mx = sc;
      for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
      const float m2 = fmaxf(m, mx);
      const float pr = seen ? exp2f(sc - (m2 == -INFINITY ? 0.f : m2)) : 0.f;
      const float keep = m2 == -INFINITY ? 1.f : exp2f(m - m2);
      m = m2;
      l = l * keep + pr;
#pragma unroll
      for (int j = 0; j < E; ++j) o[j] *= keep;
      for (int i = 0; i < 32; ++i) {
        const float pi = __shfl_sync(0xffffffffu, pr, i);
        const uint64_t bi = __shfl_sync(0xffffffffu, (unsigned long long)reinterpret_cast<uint64_t>(blk), i);
        const int ti = __shfl_sync(0xffffffffu, t, i);
        if (!__shfl_sync(0xffffffffu, (int)seen, i)) continue;
        const uint8_t* v = reinterpret_cast<const uint8_t*>(bi) + block / 2;
        const int d0 = lane * E, g = d0 / 64;
        const uint32_t prm = *reinterpret_cast<const uint32_t*>(v + D / 64 * 512 + (g * 16 + ti) * 4);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const int d = d0 + j - g * 64;
          const int c = (v[(g * 16 + ti) * 32 + d / 2] >> (4 * (d & 1))) & 15;
          const float z = __uint_as_float(prm & 0xffff0000u), s = __uint_as_float(prm << 16);
          o[j] = fmaf(pi, z == z ? fmaf(s, (float)(c - 8), z) : 0.f, o[j]);   // NaN tokens come through the scores
        }
      }
    }
    for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
#pragma unroll
    for (int j = 0; j < E; ++j)
      p.out[xrow * p.ld_out + ((int64_t)head * p.group + e) * D + lane * E + j] = __float2bfloat16_rn(l == 0.f ? 0.f : o[j] / l);
  }
}

}  // namespace

cudaError_t dsn_launch_cache_attention_rows(const CacheAttParams& p, int D, int sm_count, cudaStream_t s) {
  const int64_t ctas = ((int64_t)p.B * p.R * p.max_heads * p.group + 3) / 4, most = (int64_t)sm_count * 16;
  const dim3 grid((unsigned)(ctas < most ? ctas : most));
  return D == 64 ? dsn_launch(cache_attention_simple<64>, grid, dim3(128), 0, s, 1, p) : dsn_launch(cache_attention_simple<128>, grid, dim3(128), 0, s, 1, p);
}
