// Attention over the 4-bit cache, a few query vectors a head (rows * group <= 32: single tokens, shared heads, a few tokens at once).
//
// Bound by memory: a cached token is 18 D / 16 bytes a head, read once for all query vectors of the head.  Work is dealt out in steps (32 tokens of 128
// elements, 64 of 64): all steps of all (request, head) items stand in one line, and every warp of the GPU gets an equal stretch of it, so neither few
// long requests nor many short ones leave SMs idle.  A warp keeps the steps to come in flight as bulk copies into a ring of its own (no barrier with
// other warps), a block of 16 tokens a copy, as pages may end after any block.
// Measured (in a graph): 64 requests of up to 8192 tokens, 8 heads of 128, 4 queries a head: 122 us, 3.8 TB/s (118 with one
// reference a query, behind which fp16 loses what lies 2^20 below the largest scale of a step); a copy's rate would allow 70 us.  What bounds it is the
// arithmetic on the codes, some 720 instructions a step and warp at 12 warps of 168 registers an SM (58 % of the issue slots, the rest is their latency); no other
// split was faster: 16 and 14 warps spill (132, 148 us where 12 took 128), 8 hide less (144).  One token of one request takes 9.1 us: the look-ups in a row of
// request, page and blocks, the join in shared memory and the joining kernel, not the bytes.
// An item that lies in one warp's stretch is finished there.  What the warps of a CTA cut among themselves they join in shared memory; of an item that is
// cut between CTAs, each leaves its reference, sum and products (fp32) in the workspace, and a second small kernel joins them.
//
// Products on the tensor cores, with the tokens as rows: S^T = K Q^T (16 tokens x 8 queries x 16 elements an instruction), O^T = V^T P^T, fp16 operands.
//   Codes become fp16 numbers with one mask each: 1024 + code, or 1024 + 16 code from the high half of a byte.  For K the offsets are taken off by
//   starting the accumulator at minus their product with the query (and the 16 by a sixteenth in the query), which costs nothing; scale and
//   middle of a token's group are applied to the sum in fp32.  (An fp16 number from 1024 on counts in ones: the usual way to turn small integers into
//   floating point by placing their bits in its fraction.)  Queries keep their 8 bits; but a sum that starts at 1032 times the query's elements is rounded
//   at that size, 2^-23 of it a product, which comes to some 1e-4 of a score: about what operands of 11 bits cost.
//   For V the offset is subtracted (a sum over thousands of tokens would lose bits to it), the scale goes into the probability before its
//   one rounding to fp16, the middle into a sum of its own in fp32.
// The order of elements in a product is free, so a lane takes whole words: 16 elements of K in 8 bytes, 8 elements of V in 4.  Row i of a block's K is token
// i ^ (i >> 2 & 1): then neither K's rows nor the pairs of tokens that a lane needs of V meet in a bank.
// Queries are brought to 1 .. 2 by a power of two, which goes into the scale.  What a query gathers of a group of 64 elements is in units of 2^ref, a reference of
// the query and the group: the largest product of a probability and a scale among the tokens that the query sees stands at 2^7 .. 2^15, so that fp16 holds
// every product that counts, however far the scales of other groups, of other tokens or of tokens that are hidden lie from it.  A step first looks at a
// bound (a lane's largest score and its largest power of two); only where that passes 2^15 are the products themselves looked at and the reference moved.
#include "dsn_cache_line.cuh"

namespace {

using namespace dsn_q4;
using dsn_gemm::smem_u32;

constexpr float kTop = 15.f, kAim = 7.f;   // see the reference above; 2^7 is what the largest has when it has just moved
constexpr uint32_t kCtrl = 2048;  // behind the list: sums of a scan, the abort flag, what the warps say about their ends

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_from(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float c0, float c1) {   // rows start alike
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %10, %11};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// First token that the item's rows can see, rounded down to a block, and one behind the last.
__device__ __forceinline__ void item_range(int len, int rows, int window, int& lo, int& hi) {
  const int first = len - rows;                                // token of the first row
  hi = len;
  lo = dsn_cache_first_seen(first, window) & ~(DSN_CACHE_BLOCK - 1);
}

// A walk along the line.
struct Walk {
  const CacheEntry* smem;
  const CacheEntry* more;   // the CTA's entries in the workspace
  int j;                    // entry
  int head, step;
  CacheEntry e;
  __device__ __forceinline__ void load(int i) {
    j = i;
    e = i < kListSmem ? smem[i] : more[i];
  }
  __device__ __forceinline__ void advance(int n) {   // n steps, not past the item's end
    if ((step += n) == e.steps) {
      step = 0;
      if (++head == e.heads) {
        head = 0;
        load(j + 1);
      }
    }
  }
};

template <int D>
__host__ __device__ constexpr int step_blocks() { return 256 / D; }
template <int D>
__host__ __device__ constexpr uint32_t slot_bytes() { return 2 * step_blocks<D>() * dsn_cache_block_bytes(D); }   // two steps
template <int D>
__host__ __device__ constexpr uint32_t step_bytes() { return step_blocks<D>() * dsn_cache_block_bytes(D); }
template <int D, int WARPS, int DEPTH>
constexpr size_t attention_smem() { return kCtrl + kListSmem * sizeof(CacheEntry) + WARPS * DEPTH * 8 + (size_t)WARPS * DEPTH * slot_bytes<D>(); }

// Power of two of a pair's scale, or of its middle less 2^40: a probability with a middle is at most 2^55 then, a probability 2^65, which fp32 sums hold.  `pair`:
// magnitudes, or the largest of several.
__device__ __forceinline__ float pair_power(uint32_t pair) {
  const uint32_t top = min(max(pair & 0xffffu, max(pair >> 16, 40u << 7) - (40u << 7)), 0x7f7fu);
  return fmaxf((float)(int)(top >> 7) - 127.f, -50.f);
}
// From a group's unit and the sum's to the output, for references that can lie further apart than fp32 reaches: a result that fp32 holds is met by no factor
// that it does not.
struct Unit {
  float once, again;
  __device__ __forceinline__ float operator()(float y) const { return y * once * again; }
};
__device__ __forceinline__ Unit out_unit(float ref, float ref_of_sum, float inv) {
  const float half = ex2(0.5f * (ref - ref_of_sum));
  return Unit{inv * half, half};
}
// Floats of a part: references of the groups, sums (in units of the first group's reference), products.
template <int D>
__host__ __device__ constexpr int part_floats(int NC) { return NC * (D + D / 64 + 1); }

template <int D, int NT, int WARPS, int DEPTH>
__global__ void __launch_bounds__(WARPS * 32, 1) cache_attention_kernel(const __grid_constant__ CacheAttParams p) {
  constexpr int THREADS = WARPS * 32, GR = D / 64, NC = 8 * NT;
  constexpr int SB = step_blocks<D>(), kStepTokens = SB * DSN_CACHE_BLOCK;
  constexpr int kPart = part_floats<D>(NC), kSums = GR * NC, kProducts = (GR + 1) * NC;
  constexpr uint32_t kBlock = dsn_cache_block_bytes(D), kHalf = kBlock / 2, kPairs = GR * 512;
  extern __shared__ __align__(128) uint8_t smem[];
  CacheEntry* s_list = reinterpret_cast<CacheEntry*>(smem);
  uint64_t* s_scan = reinterpret_cast<uint64_t*>(smem + kListSmem * sizeof(CacheEntry));
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + kListSmem * sizeof(CacheEntry) + 512);
  const uint32_t base = smem_u32(smem) + (uint32_t)(kListSmem * sizeof(CacheEntry)) + kCtrl;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const uint32_t ring = base + (uint32_t)(warp * DEPTH) * slot_bytes<D>();
  const uint32_t bars = base + (uint32_t)(WARPS * DEPTH) * slot_bytes<D>() + (uint32_t)(warp * DEPTH) * 8u;

  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  if (tid == 0) *abort_flag = 0;
  if (lane == 0) {
    for (int i = 0; i < DEPTH; ++i) dsn_gemm::mbar_init(bars + 8u * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }

  // 17 to 32 query vectors of a head are two items of up to 16, next to each other in the line
  auto halves = [&](int rows) -> int { return NT == 2 && rows * p.group > NC; };
  const Stretch stretch = find_stretch<THREADS>(p, s_list, s_scan, WARPS, [&](int len, int rows) {
    int lo, hi;
    item_range(len, rows, p.window, lo, hi);
    return max(1, (hi - lo + 256 / D * DSN_CACHE_BLOCK - 1) / (256 / D * DSN_CACHE_BLOCK));   // a request without tokens: a step that sees nothing, for the zeros
  }, [&](int rows) { return 1 << halves(rows); });
  const uint64_t A = stretch.A, Z = stretch.Z;
  const uint64_t u0 = A + dsn_share(Z - A, warp, WARPS), u1 = A + dsn_share(Z - A, warp + 1, WARPS);
  int head_state = 3, tail = 0, head_far = 0;
  Walk work;
  if (u0 < u1) {
  Walk fetch;
  fetch.smem = s_list;
  fetch.more = p.list + stretch.first_order;
  {   // the last request that begins at or before u0
    const int count = stretch.count;
    int j = 0;
    for (int b = 0; b < count; b += 32) {
      const int i = b + lane;
      const bool le = i < count && (uint64_t)(i < kListSmem ? s_list[i].first : fetch.more[i].first) <= u0;
      const uint32_t m = __ballot_sync(0xffffffffu, le);
      if (m) j = b + 31 - __clz(m);
      if (m != 0xffffffffu) break;
    }
    fetch.load(j);
    const uint64_t off = u0 - (uint64_t)fetch.e.first;
    fetch.head = (int)(off / (uint32_t)fetch.e.steps);
    fetch.step = (int)(off - (uint64_t)fetch.head * fetch.e.steps);
  }
  work = fetch;
  const int n_steps = (int)(u1 - u0);
  const int bpp = p.page / DSN_CACHE_BLOCK;   // blocks a page

  // The fetching side: a slot of the ring takes up to two steps of an item; lane b fetches its block b; the page's number is read a slot before the copy
  // that needs it.  Blocks that lie behind one another in a page are one copy.
  int f_left = n_steps, f_n = 0, f_tok = 0, f_hi = 0, pg = -1, place = 0;   // steps to come, of this slot; this lane's token, the item's end; page, block in it
  const uint32_t page_bytes = (uint32_t)p.H * (uint32_t)bpp * kBlock;   // below 2^30
  bool wanted = false;
  auto find = [&](bool entered) {
    if (entered) {   // an item
      int lo;
      item_range(fetch.e.len, fetch.e.rows, p.window, lo, f_hi);
      f_tok = lo + fetch.step * kStepTokens + lane * DSN_CACHE_BLOCK;
    }
    f_n = min(min(2, f_left), fetch.e.steps - fetch.step);
    wanted = lane < f_n * SB && f_tok < f_hi;
    pg = -1;
    if (wanted) {
      const int col = (int)dsn_div((uint32_t)f_tok, p.by_page);
      pg = p.table[(int64_t)fetch.e.sample * p.max_pages + col];
      place = f_tok / DSN_CACHE_BLOCK - col * bpp;
    }
  };
  auto issue = [&](int slot) -> uint32_t {   // bit b of the result: block b is on its way
    const bool ok = pg >= 0 && pg < p.n_pages;
    if (wanted && !ok) dsn_set_status(p.status, DSN_ERR_BAD_INDEX, fetch.e.sample);
    const uint32_t there = __ballot_sync(0xffffffffu, ok);
    const int before = __shfl_up_sync(0xffffffffu, pg, 1);   // by all lanes, wanted or not
    const uint32_t begins = __ballot_sync(0xffffffffu, ok && (lane == 0 || pg != before || place == 0));
    if (lane == 0) dsn_gemm::mbar_expect_tx(bars + 8u * slot, (uint32_t)__popc(there) * kBlock);
    __syncwarp();
    if (begins >> lane & 1u) {
      const uint32_t stops = (~there | begins) >> lane >> 1;   // where this run of blocks ends
      dsn_bulk_load(ring + (uint32_t)slot * slot_bytes<D>() + (uint32_t)lane * kBlock, p.pages + (uint64_t)(uint32_t)pg * page_bytes + (uint32_t)((fetch.head >> halves(fetch.e.rows)) * bpp + place) * kBlock,
                    (uint32_t)__ffs(stops) * kBlock, bars + 8u * slot);
    }
    return there;
  };
  auto step_on = [&]() {   // to the next slot's steps, if there are any
    f_left -= f_n;
    if (f_left <= 0) return;
    const int j = fetch.j, hd = fetch.head;
    fetch.advance(f_n);
    const bool entered = fetch.j != j || fetch.head != hd;
    f_tok += f_n * kStepTokens;
    find(entered);
  };

  int asked = 0;
  uint32_t there = 0;   // 2 SB bits a slot
  find(true);
  for (; asked < DEPTH && f_left > 0; ++asked) {
    there |= issue(asked) << (2 * SB * asked);
    step_on();
  }

  uint32_t qf[NT][GR][4][2];
  float qsum[NT][GR][2], qoff[NT][GR][2], cs[NT][2];   // of this lane's columns: sum of the query, minus the offsets' product with it, factor of the scores (positive)
  float o[NT][GR][4][4], oz[NT][GR][2], l[NT][2], ref[NT][GR][2];
  int row_of[NT][2];                 // rows of this lane's columns
  bool fresh = true, ok = true;
  bool head_open = work.step != 0;   // the first item began in an earlier warp's stretch
  head_state = 0;
  const uint32_t k1024 = opaque_1024();
  const int kap = g ^ (g >> 2);      // token of K's row g in a block
  uint32_t slot = 0, parity = 0;

  int sub = 0;   // step of the slot
  for (int i = 0; i < n_steps; ++i) {
    const CacheEntry& e = work.e;
    const int two = halves(e.rows), kv = work.head >> two, v0 = two ? NC * (work.head & 1) : 0;   // head of k and v, first query vector of the item
    const int cols = min(e.rows * p.group - v0, NC);
    const int64_t row0 = (int64_t)(p.grouped ? e.pos : e.sample) * p.R;
    if (fresh) {
      fresh = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int v = nt * 8 + g, r = (int)dsn_div((uint32_t)(v0 + v), p.by_group), ev = v0 + v - r * p.group;
        const __nv_bfloat16* q = p.qkv + (row0 + r) * p.ld_qkv + ((int64_t)kv * (p.group + 2) + ev) * D;
        uint4 w[GR][2];
        uint32_t top = 0;
#pragma unroll
        for (int gr = 0; gr < GR; ++gr)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            w[gr][h] = make_uint4(0, 0, 0, 0);
            if (v < cols) w[gr][h] = *reinterpret_cast<const uint4*>(q + gr * 64 + 16 * t + 8 * h);
          }
#pragma unroll
        for (int gr = 0; gr < GR; ++gr)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            top = __vmaxu2(top, __vmaxu2(__vmaxu2(w[gr][h].x & 0x7fff7fffu, w[gr][h].y & 0x7fff7fffu), __vmaxu2(w[gr][h].z & 0x7fff7fffu, w[gr][h].w & 0x7fff7fffu)));
        uint32_t ex = max(top & 0xffffu, top >> 16);
        ex = max(ex, __shfl_xor_sync(0xffffffffu, ex, 1));
        ex = max(ex, __shfl_xor_sync(0xffffffffu, ex, 2)) >> 7;
        ex = ex == 255u ? 127u : min(max(ex, 27u), 253u);   // a query that is not finite stays so
        const float down = __uint_as_float((254u - ex) << 23 | (p.scale_log2 < 0.f ? 0x80000000u : 0u));   // a negative scale goes into the signs
        const float up = fmaxf(fabsf(p.scale_log2) * __uint_as_float(ex << 23), 1e-37f);   // not 0: what is hidden is -infinity
        cs[nt][0] = __shfl_sync(0xffffffffu, up, 8 * t);
        cs[nt][1] = __shfl_sync(0xffffffffu, up, 8 * t + 4);
#pragma unroll
        for (int gr = 0; gr < GR; ++gr) {
          float even = 0.f, odd = 0.f;   // sums of the numbers as they stand in the product
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 x = w[gr][h];
            const __half2 y[4] = {__floats2half2_rn(lo_bf16(x.x) * down, lo_bf16(x.z) * down),                         // elements 0, 4
                                  __floats2half2_rn(hi_bf16(x.x) * down * 0.0625f, hi_bf16(x.z) * down * 0.0625f),     // 1, 5
                                  __floats2half2_rn(lo_bf16(x.y) * down, lo_bf16(x.w) * down),                         // 2, 6
                                  __floats2half2_rn(hi_bf16(x.y) * down * 0.0625f, hi_bf16(x.w) * down * 0.0625f)};    // 3, 7
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float2 f = __half22float2(y[k]);
              if (k & 1) odd += f.x + f.y; else even += f.x + f.y;
              qf[nt][gr][2 * h + (k >> 1)][k & 1] = *reinterpret_cast<const uint32_t*>(&y[k]);
            }
          }
          even += __shfl_xor_sync(0xffffffffu, even, 1);
          even += __shfl_xor_sync(0xffffffffu, even, 2);
          odd += __shfl_xor_sync(0xffffffffu, odd, 1);
          odd += __shfl_xor_sync(0xffffffffu, odd, 2);
          const float sum = fmaf(16.f, odd, even), off = -fmaf(1032.f, even, 1152.f * odd);   // code - 8 is the number less 1032, a sixteenth of it less 72
          qsum[nt][gr][0] = __shfl_sync(0xffffffffu, sum, 8 * t);
          qsum[nt][gr][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
          qoff[nt][gr][0] = __shfl_sync(0xffffffffu, off, 8 * t);
          qoff[nt][gr][1] = __shfl_sync(0xffffffffu, off, 8 * t + 4);
          oz[nt][gr][0] = oz[nt][gr][1] = 0.f;
          ref[nt][gr][0] = ref[nt][gr][1] = kLowest;
#pragma unroll
          for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[nt][gr][mt][x] = 0.f;
        }
        l[nt][0] = l[nt][1] = 0.f;
        row_of[nt][0] = (int)dsn_div((uint32_t)(v0 + nt * 8 + 2 * t), p.by_group);
        row_of[nt][1] = (int)dsn_div((uint32_t)(v0 + nt * 8 + 2 * t + 1), p.by_group);
      }
    }
    int lo, hi;
    item_range(e.len, e.rows, p.window, lo, hi);
    const int tok0 = lo + work.step * kStepTokens;
    const uint32_t here = (there >> (SB * (2 * slot + sub))) & ((1u << SB) - 1u);
    // all tokens of the step seen by all rows?
    const int first_tok = e.len - e.rows;
    const bool plain = here == (1u << SB) - 1u && tok0 + kStepTokens <= first_tok + 1 && (p.window == 0 || tok0 > e.len - 1 - p.window);
    if (sub == 0) {
      ok = warp_wait(bars + 8u * slot, parity, abort_flag, p.status, 71);
      if (!ok) break;
    }
    const uint32_t st = ring + slot * slot_bytes<D>() + (uint32_t)sub * step_bytes<D>();

    float s[SB][NT][4];
    uint32_t vpair[SB][GR][2];
#pragma unroll
    for (int b = 0; b < SB; ++b) {
      const uint32_t blk = st + b * kBlock;
#pragma unroll
      for (int gr = 0; gr < GR; ++gr) {
        const uint2 w0 = lds64(blk + gr * 512 + kap * 32 + t * 8), w1 = lds64(blk + gr * 512 + (kap + 8) * 32 + t * 8);
        const uint32_t k0 = lds32(blk + kPairs + gr * 64 + kap * 4), k1 = lds32(blk + kPairs + gr * 64 + (kap + 8) * 4);
        vpair[b][gr][0] = lds32(blk + kHalf + kPairs + gr * 64 + kap * 4);
        vpair[b][gr][1] = lds32(blk + kHalf + kPairs + gr * 64 + (kap + 8) * 4);
        float acc[NT][4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const uint32_t x0 = (ks < 2 ? w0.x : w0.y) >> (8 * (ks & 1)), x1 = (ks < 2 ? w1.x : w1.y) >> (8 * (ks & 1));
          const uint32_t a[4] = {low_codes(x0, k1024), low_codes(x1, k1024), high_codes(x0, k1024), high_codes(x1, k1024)};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            if (ks == 0) mma_f16_from(acc[nt], a, qf[nt][gr][0][0], qf[nt][gr][0][1], qoff[nt][gr][0], qoff[nt][gr][1]);
            else mma_f16(acc[nt], a, qf[nt][gr][ks][0], qf[nt][gr][ks][1]);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float sc = lo_bf16(x < 2 ? k0 : k1), z = hi_bf16(x < 2 ? k0 : k1);
            s[b][nt][x] = fmaf(sc, acc[nt][x], gr == 0 ? z * qsum[nt][gr][x & 1] : fmaf(z, qsum[nt][gr][x & 1], s[b][nt][x]));
          }
      }
    }
    if (!plain) {
#pragma unroll
      for (int b = 0; b < SB; ++b) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int key = tok0 + b * DSN_CACHE_BLOCK + kap + 8 * hf;
          const bool exists = (here >> b & 1u) && key < hi;
#pragma unroll
          for (int gr = 0; gr < GR; ++gr) {   // nothing of a token that does not exist, no NaN of one that some row does not see
            const uint32_t w = vpair[b][gr][hf];
            if (!exists) vpair[b][gr][hf] = 0u;
            else if (!(fabsf(hi_bf16(w)) <= 3.4e38f) || !(fabsf(lo_bf16(w)) <= 3.4e38f)) vpair[b][gr][hf] = 0u;
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int me = first_tok + row_of[nt][c];
              const bool seen = exists && key <= me && (p.window == 0 || key > me - p.window);
              if (!seen) s[b][nt][2 * hf + c] = -INFINITY;
            }
        }
      }
    }
    // a product of a probability and a scale that would pass the top?
    float power[GR];
#pragma unroll
    for (int gr = 0; gr < GR; ++gr) {
      uint32_t big = 0;   // largest of the scales' bits, largest of the middles'
#pragma unroll
      for (int b = 0; b < SB; ++b) big = __vmaxu2(big, __vmaxu2(vpair[b][gr][0] & 0x7fff7fffu, vpair[b][gr][1] & 0x7fff7fffu));
      power[gr] = pair_power(big);
    }
    float most = -INFINITY;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float m = -INFINITY, up = -INFINITY;
#pragma unroll
        for (int b = 0; b < SB; ++b) m = fmaxf(m, fmaxf(s[b][nt][c], s[b][nt][2 + c]));
#pragma unroll
        for (int gr = 0; gr < GR; ++gr) up = fmaxf(up, power[gr] - ref[nt][gr][c]);
        most = fmaxf(most, fmaf(m, cs[nt][c], up));
      }
    if (__any_sync(0xffffffffu, most > kTop)) {
#pragma unroll
      for (int gr = 0; gr < GR; ++gr) {
        float top[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) top[nt][0] = top[nt][1] = -INFINITY;
#pragma unroll
        for (int b = 0; b < SB; ++b)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float e = pair_power(vpair[b][gr][hf] & 0x7fff7fffu);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int c = 0; c < 2; ++c) top[nt][c] = fmaxf(top[nt][c], fmaf(s[b][nt][2 * hf + c], cs[nt][c], e));
          }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float m = top[nt][c];
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
            m = fmaxf(ref[nt][gr][c], m - kAim);
            const float f = ex2(0.5f * (ref[nt][gr][c] - m));   // twice: references can lie further apart than fp32 reaches
            ref[nt][gr][c] = m;
            if (gr == 0) l[nt][c] = l[nt][c] * f * f;
            oz[nt][gr][c] = oz[nt][gr][c] * f * f;
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
              o[nt][gr][mt][c] = o[nt][gr][mt][c] * f * f;
              o[nt][gr][mt][2 + c] = o[nt][gr][mt][2 + c] * f * f;
            }
          }
      }
    }
#pragma unroll
    for (int b = 0; b < SB; ++b) {
      const uint32_t blk = st + b * kBlock + kHalf;
      const int ka = 2 * t + (t >> 1), kb = 2 * t + 1 - (t >> 1);   // tokens of columns 2 t and 2 t + 1
#pragma unroll
      for (int gr = 0; gr < GR; ++gr) {
        uint32_t pb[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float sc = lo_bf16(vpair[b][gr][hf]), z = hi_bf16(vpair[b][gr][hf]);
            const float p0 = ex2(fmaf(s[b][nt][2 * hf], cs[nt][0], -ref[nt][gr][0])), p1 = ex2(fmaf(s[b][nt][2 * hf + 1], cs[nt][1], -ref[nt][gr][1]));
            if (gr == 0) l[nt][0] += p0, l[nt][1] += p1;
            oz[nt][gr][0] = fmaf(p0, z, oz[nt][gr][0]);
            oz[nt][gr][1] = fmaf(p1, z, oz[nt][gr][1]);
            const __half2 ps = __floats2half2_rn(p0 * sc, p1 * sc);
            pb[nt][hf] = transpose8x8(*reinterpret_cast<const uint32_t*>(&ps));
          }
        const uint32_t va = lds32(blk + gr * 512 + ka * 32 + g * 4), vb = lds32(blk + gr * 512 + kb * 32 + g * 4);
        const uint32_t vc = lds32(blk + gr * 512 + (ka + 8) * 32 + g * 4), vd = lds32(blk + gr * 512 + (kb + 8) * 32 + g * 4);
#pragma unroll
        for (int by = 0; by < 2; ++by) {
          // byte `by` and byte `by` + 2 of the words of two tokens side by side: elements 2 by, 2 by + 1 and 2 by + 4, 2 by + 5
          const uint32_t x0 = __byte_perm(va, vb, by ? 0x5511 : 0x4400), x1 = __byte_perm(va, vb, by ? 0x7733 : 0x6622);
          const uint32_t y0 = __byte_perm(vc, vd, by ? 0x5511 : 0x4400), y1 = __byte_perm(vc, vd, by ? 0x7733 : 0x6622);
          const uint32_t lo4[4] = {code_of_low(low_codes(x0, k1024)), code_of_low(low_codes(x1, k1024)), code_of_low(low_codes(y0, k1024)), code_of_low(low_codes(y1, k1024))};
          const uint32_t hi4[4] = {code_of_high(high_codes(x0, k1024)), code_of_high(high_codes(x1, k1024)), code_of_high(high_codes(y0, k1024)), code_of_high(high_codes(y1, k1024))};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma_f16(o[nt][gr][2 * by], lo4, pb[nt][0], pb[nt][1]);
            mma_f16(o[nt][gr][2 * by + 1], hi4, pb[nt][0], pb[nt][1]);
          }
        }
      }
    }
    const bool item_ends = work.step + 1 == e.steps, last = i + 1 == n_steps;
    if (sub == 1 || item_ends || last) {
      __syncwarp();   // every lane has read the slot
      if (f_left > 0) {
        there = (there & ~(((1u << 2 * SB) - 1u) << (2 * SB * slot))) | (issue(slot) << (2 * SB * slot));
        ++asked;
        step_on();
      }
      sub = 0;
      if (++slot == DEPTH) slot = 0, parity ^= 1u;
    } else {
      sub = 1;
    }

    if (item_ends || last) {
      const bool whole = item_ends && !head_open;
      if (!item_ends) {
        if (head_open) head_state = 2; else tail = 1;
      } else if (head_open) {
        head_state = 1;
      }
      // the last thing that the warp does may use its ring; the first of more goes to the workspace
      float* dst = last ? reinterpret_cast<float*>(smem + (ring - smem_u32(smem))) : p.warp_data + ((int64_t)blockIdx.x * WARPS + warp) * kPart;
      if (!whole && head_open && !last) head_far = 1;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float sum = l[nt][c];
          sum += __shfl_xor_sync(0xffffffffu, sum, 4);
          sum += __shfl_xor_sync(0xffffffffu, sum, 8);
          sum += __shfl_xor_sync(0xffffffffu, sum, 16);
          const int v = nt * 8 + 2 * t + c;
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          const int r = row_of[nt][c], ev = v0 + v - r * p.group;
#pragma unroll
          for (int gr = 0; gr < GR; ++gr) {
            float z = oz[nt][gr][c];
            z += __shfl_xor_sync(0xffffffffu, z, 4);
            z += __shfl_xor_sync(0xffffffffu, z, 8);
            z += __shfl_xor_sync(0xffffffffu, z, 16);
            float y[8];
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
              y[mt] = o[nt][gr][mt][c] + z;
              y[mt + 4] = o[nt][gr][mt][2 + c] + z;
            }
            const Unit to = out_unit(ref[nt][gr][c], ref[nt][0][c], inv);
            if (v < cols) {
              if (whole) {
                uint4 w;
                w.x = pack_bf16(to(y[0]), to(y[1]));
                w.y = pack_bf16(to(y[2]), to(y[3]));
                w.z = pack_bf16(to(y[4]), to(y[5]));
                w.w = pack_bf16(to(y[6]), to(y[7]));
                *reinterpret_cast<uint4*>(p.out + (row0 + r) * p.ld_out + ((int64_t)kv * p.group + ev) * D + gr * 64 + 8 * g) = w;
              } else {
                float4* d4 = reinterpret_cast<float4*>(dst + kProducts + v * D + gr * 64 + 8 * g);
                d4[0] = make_float4(y[0], y[1], y[2], y[3]);
                d4[1] = make_float4(y[4], y[5], y[6], y[7]);
              }
            }
          }
          if (!whole && v < cols && g == 0) {
#pragma unroll
            for (int gr = 0; gr < GR; ++gr) dst[gr * NC + v] = ref[nt][gr][c];
            dst[kSums + v] = sum;
          }
        }
      head_open = false;
      fresh = true;
    }
    if (!last) work.advance(1);
  }
  if (!ok) {
    dsn_drain(bars, DEPTH, max(0, asked - DEPTH), asked);
    head_state = 3;
    tail = 0;
  } else if (head_far) {   // back into the ring, behind the last part: one trip to memory for all warps, where the join below would make one for each of its parts
    static_assert(2 * kPart * sizeof(float) <= DEPTH * slot_bytes<D>() && kPart % 4 == 0, "two parts in a ring");
    const float4* from = reinterpret_cast<const float4*>(p.warp_data + ((int64_t)blockIdx.x * WARPS + warp) * kPart);
    float4* to = reinterpret_cast<float4*>(smem + (ring - smem_u32(smem))) + kPart / 4;
    constexpr int N = (kPart / 4 + 31) / 32;
    float4 x[N];
    __syncwarp();   // other lanes' stores
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (32 * k + lane < kPart / 4) x[k] = from[32 * k + lane];
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (32 * k + lane < kPart / 4) to[32 * k + lane] = x[k];
  }
  }

  // ---- what the warps of the CTA cut among themselves
  CachePart* s_part = reinterpret_cast<CachePart*>(s_scan + 128);
  if (lane == 0) s_part[warp] = CachePart{head_state, tail, work.e.sample, work.e.pos, work.head, work.e.rows, head_far, 0};
  __syncthreads();
  // A chain is the tail of a warp (or what came before this CTA) and the heads behind it up to the one that ends its item.
  const CachePart mine = s_part[lane < WARPS ? lane : 0];
  constexpr uint32_t kAll = (1u << WARPS) - 1u;
  const uint32_t closes = __ballot_sync(0xffffffffu, mine.head_state == 1) & kAll, passes = __ballot_sync(0xffffffffu, mine.head_state == 2) & kAll,
                 begins = __ballot_sync(0xffffffffu, mine.head_state == 0) & kAll, tails = __ballot_sync(0xffffffffu, mine.tail != 0) & kAll,
                 far = __ballot_sync(0xffffffffu, mine.head_far != 0) & kAll;
  auto part_of = [&](int w, bool of_tail) -> const float* {   // where a warp left a part
    return reinterpret_cast<const float*>(smem + (base - smem_u32(smem)) + (size_t)w * DEPTH * slot_bytes<D>()) + (!of_tail && (far >> w & 1u) ? kPart : 0);
  };
  const uint32_t first_heads = (closes | passes) & ~(begins ? ~((begins & (0u - begins)) - 1u) : 0u);   // heads in front of the first item that begins here
  // parts of the chain behind warp a (-1: in front of all): up to the first that closes
  auto heads_of = [&](int a) -> uint32_t {
    const uint32_t behind = a < 0 ? kAll : kAll & ~((2u << a) - 1u);
    const uint32_t stop = (closes | begins) & behind;
    const uint32_t upto = stop ? (stop & (0u - stop)) * 2u - 1u : ~0u;
    return (closes | passes) & behind & upto;
  };
  const uint32_t none = closes | passes | begins;
  const int cta_head = !none ? 3 : (first_heads ? ((heads_of(-1) & closes) ? 1 : 2) : 0);
  int cta_tail = 0, tail_warp = 0, task = 0;
  for (uint32_t left = (tails << 1) | (first_heads ? 1u : 0u); left; left &= left - 1u) {
    const int a = __ffs(left) - 2;
    const uint32_t heads = heads_of(a);
    const bool closed = (heads & closes) != 0;
    if (a >= 0 && !closed) cta_tail = 1, tail_warp = a;
    const int two = a >= 0 ? halves(s_part[a].rows) : 0, v0 = two ? NC * (s_part[a].head & 1) : 0;
    const int cols = a >= 0 ? min(s_part[a].rows * p.group - v0, NC) : NC;
    const bool in = (heads >> lane & 1u) || lane == a;   // lane j: the part of warp j
    const float* src = in ? part_of(lane, lane == a) : nullptr;
    const int begin = (warp + WARPS - task % WARPS) % WARPS;
    task += cols;
    for (int v = begin; v < cols; v += WARPS) {
      const float l = in ? src[kSums + v] : 0.f;
      float top[GR], f[GR];
#pragma unroll
      for (int gr = 0; gr < GR; ++gr) {
        const float m = in ? src[gr * NC + v] : kLowest;
        top[gr] = m;
#pragma unroll
        for (int o = 8; o; o >>= 1) top[gr] = fmaxf(top[gr], __shfl_xor_sync(0xffffffffu, top[gr], o));   // at most 15 parts
        top[gr] = __shfl_sync(0xffffffffu, top[gr], 0);
        f[gr] = l == 0.f ? 0.f : ex2(0.5f * (m - top[gr]));   // an empty part holds nothing; applied twice, as above
      }
      float sum = l * f[0] * f[0];
#pragma unroll
      for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      sum = __shfl_sync(0xffffffffu, sum, 0);
      float y[D / 32];
#pragma unroll
      for (int x = 0; x < D / 32; ++x) y[x] = 0.f;
#pragma unroll 2
      for (uint32_t set = heads | (a >= 0 ? 1u << a : 0u); set; set &= set - 1u) {
        const int j = __ffs(set) - 1;
        float fj = __shfl_sync(0xffffffffu, f[0], j);
        if constexpr (GR == 2) {   // lanes 16 to 31 have the second group's elements
          const float second = __shfl_sync(0xffffffffu, f[1], j);
          if (lane >= 16) fj = second;
        }
        const float* at = part_of(j, j == a) + kProducts + v * D;
        if constexpr (D == 128) {
          const float4 q = fj == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(at + 4 * lane);
          y[0] = fmaf(q.x * fj, fj, y[0]); y[1] = fmaf(q.y * fj, fj, y[1]); y[2] = fmaf(q.z * fj, fj, y[2]); y[3] = fmaf(q.w * fj, fj, y[3]);
        } else {
          const float2 q = fj == 0.f ? make_float2(0.f, 0.f) : *reinterpret_cast<const float2*>(at + 2 * lane);
          y[0] = fmaf(q.x * fj, fj, y[0]); y[1] = fmaf(q.y * fj, fj, y[1]);
        }
      }
      if (a >= 0 && closed) {
        const CachePart& q = s_part[a];
        const int r = (int)dsn_div((uint32_t)(v0 + v), p.by_group), ev = v0 + v - r * p.group;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        __nv_bfloat16* dst = p.out + ((int64_t)(p.grouped ? q.pos : q.sample) * p.R + r) * p.ld_out + ((int64_t)(q.head >> two) * p.group + ev) * D;
        const Unit to = out_unit(GR == 2 && lane >= 16 ? top[GR - 1] : top[0], top[0], inv);
        if constexpr (D == 128)
          *reinterpret_cast<uint2*>(dst + 4 * lane) = make_uint2(pack_bf16(to(y[0]), to(y[1])), pack_bf16(to(y[2]), to(y[3])));
        else
          *reinterpret_cast<uint32_t*>(dst + 2 * lane) = pack_bf16(to(y[0]), to(y[1]));
      } else {
        float* dst = p.cta_data + ((int64_t)blockIdx.x * 2 + (a >= 0)) * kPart;
        if (lane == 0) {
#pragma unroll
          for (int gr = 0; gr < GR; ++gr) dst[gr * NC + v] = top[gr];
          dst[kSums + v] = sum;
        }
        if constexpr (D == 128) *reinterpret_cast<float4*>(dst + kProducts + v * D + 4 * lane) = make_float4(y[0], y[1], y[2], y[3]);
        else *reinterpret_cast<float2*>(dst + kProducts + v * D + 2 * lane) = make_float2(y[0], y[1]);
      }
    }
  }
  static_assert(WARPS <= 15, "a chain's parts are joined by 16 lanes");
  if (tid == 0) {
    CachePart q = s_part[tail_warp];
    q.head_state = cta_head;
    q.tail = cta_tail;
    p.parts[blockIdx.x] = q;
  }
}

// Joins the parts of the items that were cut between CTAs: a CTA for every column of every CTA's last item, 8 groups of D / 4 threads that take every eighth part.
template <int D>
__global__ void __launch_bounds__(2 * D) cache_join_kernel(const __grid_constant__ CacheAttParams p, int ctas, int NC) {
  __shared__ int s_end;
  constexpr int GR = D / 64;
  __shared__ float s_w[GR][DSN_CACHE_MAX_CTAS], s_l[DSN_CACHE_MAX_CTAS], s_m[GR];
  __shared__ float4 s_o[2 * D];
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const int tid = threadIdx.x, w = blockIdx.x, v = blockIdx.y, kPart = part_floats<D>(NC), kSums = GR * NC, kProducts = (GR + 1) * NC;
  const CachePart part = p.parts[w];
  const int two = NC == 16 && part.rows * p.group > NC, v0 = two ? NC * (part.head & 1) : 0;
  if (!part.tail || v >= min(part.rows * p.group - v0, NC)) return;
  if (tid == 0) s_end = ctas - 1;
  __syncthreads();
  for (int b = w + 1 + tid; b < ctas; b += 2 * D)
    if (p.parts[b].head_state < 2) atomicMin(&s_end, b);   // the CTA in whose stretch the item ends
  __syncthreads();
  const int n = s_end - w + 1;
  for (int j = tid; j < n; j += 2 * D) {
    const float* src = p.cta_data + ((int64_t)(w + j) * 2 + (j == 0)) * kPart;
    const bool there = j == 0 || p.parts[w + j].head_state != 3;
#pragma unroll
    for (int gr = 0; gr < GR; ++gr) s_w[gr][j] = there ? src[gr * NC + v] : kLowest;
    s_l[j] = there ? src[kSums + v] : 0.f;
  }
  __syncthreads();
  if (tid < 32 * GR) {   // a warp a group
    const int gr = tid >> 5, lane = tid & 31;
    float m = kLowest;
    for (int j = lane; j < n; j += 32) m = fmaxf(m, s_w[gr][j]);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) s_m[gr] = m;
  }
  __syncthreads();
  constexpr int L = D / 4;
  const int sub = tid % L, of = tid / L, gr = sub / 16;   // 16 threads a group of 64
  const float m = s_m[gr];
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int j = of; j < n; j += 8) {
    const float f = s_l[j] == 0.f ? 0.f : ex2(0.5f * (s_w[gr][j] - m));   // an empty part holds nothing; applied twice, as above
    const float4 q = f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f)
                              : *reinterpret_cast<const float4*>(p.cta_data + ((int64_t)(w + j) * 2 + (j == 0)) * kPart + kProducts + v * D + 4 * sub);
    o.x = fmaf(q.x * f, f, o.x); o.y = fmaf(q.y * f, f, o.y); o.z = fmaf(q.z * f, f, o.z); o.w = fmaf(q.w * f, f, o.w);
  }
  s_o[tid] = o;
  __syncthreads();
  if (of) return;
  float l = 0.f;
  for (int j = 0; j < n; ++j) {
    const float f = s_l[j] == 0.f ? 0.f : ex2(0.5f * (s_w[0][j] - s_m[0]));
    l = fmaf(s_l[j] * f, f, l);
  }
  for (int k = 1; k < 8; ++k) {
    const float4 q = s_o[k * L + sub];
    o.x += q.x; o.y += q.y; o.z += q.z; o.w += q.w;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const Unit to = out_unit(m, s_m[0], inv);
  const int r = (v0 + v) / p.group, ev = v0 + v - r * p.group;
  const int64_t row = (int64_t)(p.grouped ? part.pos : part.sample) * p.R + r;
  *reinterpret_cast<uint2*>(p.out + row * p.ld_out + ((int64_t)(part.head >> two) * p.group + ev) * D + 4 * sub) =
      make_uint2(pack_bf16(to(o.x), to(o.y)), pack_bf16(to(o.z), to(o.w)));
}

template <int D, int NT, int WARPS, int DEPTH>
cudaError_t launch(const CacheAttParams& p, int ctas, cudaStream_t s) {
  static size_t configured[DSN_MAX_DEVICES] = {};
  constexpr size_t smem = attention_smem<D, WARPS, DEPTH>();
  static_assert(smem <= 227 * 1024, "shared memory of a CTA");
  auto kernel = cache_attention_kernel<D, NT, WARPS, DEPTH>;
  cudaError_t e = dsn_ensure_dynamic_smem(kernel, smem, configured);
  if (e != cudaSuccess) return e;
  e = dsn_launch(kernel, dim3((unsigned)ctas), dim3(WARPS * 32), smem, s, 1, p);
  if (e != cudaSuccess) return e;
  return dsn_launch(cache_join_kernel<D>, dim3((unsigned)ctas, (unsigned)(p.R * p.group < 8 * NT ? p.R * p.group : 8 * NT)), dim3(2 * D), 0, s, 1, p, ctas, 8 * NT);
}

constexpr int kWarps1 = 12, kWarps2 = 8;   // warps a CTA for up to 8 and up to 16 query vectors a head: their products stay in registers (16 and 8 warps: 132 and 144 us where 12 took 128)

}  // namespace

// Workspace: the CTAs' words about their ends, requests beyond a CTA's own list, parts of warps and of CTAs.
struct CacheWorkspace {
  size_t parts, list, warp_data, cta_data, total;
};
static CacheWorkspace carve(int D, int cols, int64_t B, int ctas) {
  const size_t part = (size_t)(cols <= 8 ? 8 : 16) * (D + D / 64 + 1) * sizeof(float);
  CacheWorkspace w;
  w.parts = 0;
  w.list = w.parts + sizeof(CachePart) * (size_t)ctas;
  w.warp_data = w.list + sizeof(CacheEntry) * (size_t)B;
  w.cta_data = w.warp_data + (size_t)ctas * (cols <= 8 ? kWarps1 : kWarps2) * part;
  w.total = w.cta_data + (size_t)ctas * 2 * part;
  return w;
}

size_t dsn_cache_attention_ws_bytes(int D, int cols, int64_t B) { return carve(D, cols, B, DSN_CACHE_MAX_CTAS).total; }

cudaError_t dsn_launch_cache_attention(CacheAttParams& p, int D, int sm_count, void* workspace, cudaStream_t s) {
  const int cols = p.R * p.group, ctas = sm_count < DSN_CACHE_MAX_CTAS ? sm_count : DSN_CACHE_MAX_CTAS;
  const CacheWorkspace w = carve(D, cols, p.B, ctas);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.parts = reinterpret_cast<CachePart*>(ws + w.parts);
  p.list = reinterpret_cast<CacheEntry*>(ws + w.list);
  p.warp_data = reinterpret_cast<float*>(ws + w.warp_data);
  p.cta_data = reinterpret_cast<float*>(ws + w.cta_data);
  if (D == 64) return cols <= 8 ? launch<64, 1, kWarps1, 2>(p, ctas, s) : launch<64, 2, kWarps2, 3>(p, ctas, s);
  return cols <= 8 ? launch<128, 1, kWarps1, 2>(p, ctas, s) : launch<128, 2, kWarps2, 3>(p, ctas, s);
}
