// Attention over the 4-bit cache, many query vectors a head (rows * group > 32: prompts, pieces of prompts), on tcgen05.
//
// One item = (request, head, 256 query vectors in a row: two halves of 128 TMEM lanes), walked along its tokens in tiles of 64; the tiles of all items
// stand in one line, of which every CTA (one an SM) gets an equal stretch.  An item that is cut leaves references, sums and products of its
// rows (fp32) in the workspace, and a second kernel joins them.
// Measured (in a graph): 2 requests of 4096 rows behind nothing, 8 heads of 128, 4 queries a head: 484 us, 570 TFLOP/s of the visible pairs, where products at a
// plain matrix product's rate would take 170.  What bounds it is the chain of a tile in the softmax: some 2,900 cycles for 64 tokens, while the exponentials of its 256
// rows need 1,024 (16 a cycle) and its products as many.  Load from TMEM, maximum, exponentials and store follow one another in a warp, eight warps of 128
// registers are all that fit, and the tensor pipe is busy 35 % of the time (26 % for 2 x 512 rows behind up to 9999 tokens, 70 us).
// Tried: 128 tokens a tile with one S buffer 491 us, two threads a row 709, more registers for the softmax warps 507 to 550 (where this form took 476 to 485), a part of the exponentials as
// polynomials within 3 %.
// Roles (512 threads):
//   warps 0-4    values: K and V tiles of fp16 in shared memory, swizzled as the products read them, four buffers each.  A unit is K or V of a block of 16
//                tokens, two lanes a token.  Every element is made once for 256 rows.
//   warp 5       loader: pages' numbers, the blocks as bulk copies into two slots of a tile, and the tile's powers of two (see below).
//   warps 6-7    issue, one a half: S_h = Q_h K^T and O_h += P_h V.  S has two buffers a half: a half's product of scores runs a tile ahead, so its softmax
//                never waits for it.  (One warp for both spends more time on barriers than the products take.)
//   warps 8-11   softmax of half 0, warps 12-15 of half 1: a thread a row (= TMEM lane), the tile's row of S in registers; maximum, exp2, sum, probabilities over the columns of S, from where the second product takes them.  They also fetch the
//                rows of Q and write those of O.
// Operands are fp16 (11 bits, where bf16's 8 would double the output's error) and keep bf16's range by powers of two: a row of Q has one, which
// goes into the scale of its scores; a tile has one for K, which goes there, too, and one for V, which the probabilities of its tokens
// take up.  Everything of a row is in units of 2^g, g a reference that moves only when a probability with its power of two would
// pass 2^15: then O is read, scaled and written back.  A tile's powers count what some row of the item sees or could see: tokens behind its last row and in front
// of its first row's window are no part of it, those that single rows do not see are.
// The eight elements of a code word come out in the order 0 4 1 5 2 6 3 7 (a mask each pair), so Q's and O's columns are in that order, too.
// TMEM: 512 columns = two regions of 256: two buffers of S_h at 0 and 64, P_h over the first half of each, O_h from 128.  Every wait is bounded.
#include "dsn_cache_line.cuh"

namespace {

using namespace dsn_q4;
using namespace dsn_gemm;

constexpr int kThreadsR = 512, kRows = 256, kTile = 64, kStages = 4;
constexpr int kValueWarps = 5, kLoadWarp = 5, kIssueWarp = 6, kSoftWarp = 8;
constexpr float kTop = 15.f, kAim = 7.f;     // a probability with its power of two is at most 2^15, 2^7 where the reference has just moved
constexpr uint32_t kTileBytes = 128 * 128;   // 128 rows of 64 bf16
constexpr uint32_t kCtrlR = 4096;
constexpr uint32_t kRegion = 256, kOCol = 128;

__device__ __forceinline__ void mma_a_tmem(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void tmem_st_8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void tmem_ld_8(uint32_t taddr, uint32_t (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_st_16(uint32_t taddr, const uint32_t (&v)[32]) {   // the first 16
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_done() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float max3_nan(float a, float b, float c) {   // NaN if any of them is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// V as it lies: rows are tokens, 64 elements in 128 bytes; 128 elements are two such pieces of a stage.
__device__ __forceinline__ uint64_t make_desc_mn(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(kTileBytes / 2 >> 4) << 16;   // from 64 elements to the next 64
  d |= (uint64_t)(1024 >> 4) << 32;         // from 8 tokens to the next 8
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// 256 (or the last) query vectors of a head of a request: their tokens and the tiles that they need.
struct Span {
  int v0, v1;         // vectors
  int me0, me1;       // tokens of the first and the last
  int lo, tiles;      // first token of the first tile, tiles
};
__device__ __forceinline__ Span span_of(int len, int rows, int ct, int group, const FastDiv& by_group, int window) {
  Span s;
  s.v0 = ct * kRows;
  s.v1 = min(rows * group, s.v0 + kRows);
  const int first = len - rows;
  s.me0 = first + (int)dsn_div((uint32_t)s.v0, by_group);
  s.me1 = first + (int)dsn_div((uint32_t)(s.v1 - 1), by_group);
  s.lo = dsn_cache_first_seen(s.me0, window) & ~(DSN_CACHE_BLOCK - 1);
  s.tiles = max(1, (s.me1 + 1 - s.lo + kTile - 1) / kTile);
  return s;
}
__device__ __forceinline__ int head_tiles(int len, int rows, int group, const FastDiv& by_group, int window) {
  const int cts = (rows * group + kRows - 1) / kRows;
  int sum = 0;
  for (int ct = 0; ct < cts; ++ct) sum += span_of(len, rows, ct, group, by_group, window).tiles;
  return sum;
}

// What a CTA does of one item: tiles c0 .. c1 - 1 of the span.
struct Item {
  CacheEntry e;
  Span s;
  int head, c0, c1;
};
struct RowWalk {
  const CacheEntry* smem;
  const CacheEntry* more;
  int j, head, ct, c0;
  int64_t left;         // tiles of the stretch still to come
  CacheEntry e;
  __device__ __forceinline__ void load(int i) {
    j = i;
    e = i < kListSmem ? smem[i] : more[i];
  }
  __device__ __forceinline__ bool next(const CacheAttParams& p, Item& it) {
    if (left <= 0) return false;
    it.e = e;
    it.head = head;
    it.s = span_of(e.len, e.rows, ct, p.group, p.by_group, p.window);
    it.c0 = c0;
    it.c1 = (int)min((int64_t)it.s.tiles, c0 + left);
    left -= it.c1 - it.c0;
    if (left > 0) {
      c0 = 0;
      if (it.s.v1 == e.rows * p.group) {
        ct = 0;
        if (++head == e.heads) {
          head = 0;
          load(j + 1);
        }
      } else {
        ++ct;
      }
    }
    return true;
  }
};
// Tiles of the CTA's part that half h of the item needs: a .. b - 1 (none: a == b).
__device__ __forceinline__ void half_tiles(const Item& it, int h, const FastDiv& by_group, int window, int& a, int& b) {
  const int w0 = it.s.v0 + 128 * h, w1 = min(it.s.v1, w0 + 128);
  a = b = it.c0;
  if (w0 >= w1) return;
  const int first = it.e.len - it.e.rows, m0 = first + (int)dsn_div((uint32_t)w0, by_group), m1 = first + (int)dsn_div((uint32_t)(w1 - 1), by_group);
  if (m1 < 0) return;
  a = max(it.c0, (dsn_cache_first_seen(m0, window) - it.s.lo) / kTile);
  b = min(it.c1, (m1 + 1 - it.s.lo + kTile - 1) / kTile);
  if (b < a) b = a;
}

template <int D>
__global__ void __launch_bounds__(kThreadsR, 1) cache_rows_kernel(const __grid_constant__ CacheAttParams p) {
  constexpr int GR = D / 64;
  constexpr uint32_t kBlock = dsn_cache_block_bytes(D), kOperand = GR * kTileBytes, kStage = kOperand / 2, kSlot = kTile / DSN_CACHE_BLOCK * kBlock;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw);
  // barriers: [2 halves] of q, o_empty and idle, [4 stages] of k and v, [2 slots] of raw, [2 halves][2 buffers] of s, p, o
  const uint32_t q_full = base, o_empty = base + 16, k_full = base + 32, k_empty = base + 64, v_full = base + 96, v_empty = base + 128,
                 raw_full = base + 160, raw_empty = base + 176, raw_ready = base + 304, idle = base + 336, s_full = base + 192, p_full = base + 224, o_full = base + 256;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 288);
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + 292);
  uint32_t* s_raw = reinterpret_cast<uint32_t*>(smem + 296);                       // [2 slots]: bit b: block b is there; tokens in front of every row's window << 4; tokens << 8; exponents that K and V are divided by << 16, << 24
  uint8_t* s_bad = smem + 320;                                                     // [16 tiles]: bit b: block b is of a page outside the cache
  float2* s_fac = reinterpret_cast<float2*>(smem + 384);                           // [16 tiles]: K's power of two; V's, as its exponent
  uint64_t* s_scan = reinterpret_cast<uint64_t*>(smem + 640);
  CacheEntry* s_list = reinterpret_cast<CacheEntry*>(smem + 1024);
  static_assert(1024 + kListSmem * sizeof(CacheEntry) <= kCtrlR, "control block");
  const uint32_t q_at = base + kCtrlR, k_at = q_at + 2 * kOperand, v_at = k_at + kStages * kStage, raw_at = v_at + kStages * kStage;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full + 8 * i, 4);
      mbar_init(o_empty + 8 * i, 4);
      mbar_init(raw_full + 8 * i, 1);
      mbar_init(raw_empty + 8 * i, 8);
      mbar_init(raw_ready + 8 * i, 1);
      mbar_init(idle + 8 * i, 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(k_full + 8 * i, 4);   // units of 16 tokens
      mbar_init(v_full + 8 * i, 4);
      mbar_init(k_empty + 8 * i, 2);   // the halves
      mbar_init(v_empty + 8 * i, 2);
      mbar_init(s_full + 8 * i, 1);
      mbar_init(p_full + 8 * i, 4);
      mbar_init(o_full + 8 * i, 1);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const Stretch stretch = find_stretch<kThreadsR>(p, s_list, s_scan, 1u, [&](int len, int rows) { return head_tiles(len, rows, p.group, p.by_group, p.window); },
                                                     [](int) { return 1; });
  if (warp == kIssueWarp) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  RowWalk walk;
  walk.smem = s_list;
  walk.more = p.list + stretch.first_order;
  walk.left = (int64_t)(stretch.Z - stretch.A);
  if (walk.left > 0) {
    walk.load(0);   // the request that holds tile A is the list's first
    uint64_t off = stretch.A - (uint64_t)walk.e.first;
    walk.head = (int)(off / (uint32_t)walk.e.steps);
    int in_head = (int)(off - (uint64_t)walk.head * walk.e.steps);
    walk.ct = 0;
    while (true) {
      const int n = span_of(walk.e.len, walk.e.rows, walk.ct, p.group, p.by_group, p.window).tiles;
      if (in_head < n) break;
      in_head -= n;
      ++walk.ct;
    }
    walk.c0 = in_head;
  }
  Item it;


  if (warp < kValueWarps) {
    // ------------------------------------------------------------------------------ codes to values
    // Unit u of tile number i: K (0-3) or V (4-7) of block u & 3; warp w takes units w, w + 5, ... of all.
    const uint32_t units = 8u * (uint32_t)(stretch.Z - stretch.A);
    const uint32_t k1024 = opaque_1024();
    const int tok = lane & 15, part = lane >> 4;      // D = 128: a lane takes a group; D = 64: half of it
#pragma unroll 1
    for (uint32_t unit = (uint32_t)warp; unit < units; unit += kValueWarps) {
      const uint32_t i = unit >> 3, s = i % kStages, b = unit & 3u;
      const bool is_v = (unit & 4u) != 0;
      if (!warp_wait(raw_ready + 8 * (i & 1u), (i >> 1) & 1u, abort_flag, p.status, 82)) break;
      const uint32_t info = *reinterpret_cast<const volatile uint32_t*>(s_raw + (i & 1u));
      const uint32_t number = b * 16u + (uint32_t)tok;
      const bool there = (info >> b & 1u) && number < (info >> 8 & 0xffu) && number >= (info >> 4 & 15u);
      const uint32_t slot = raw_at + (i & 1u) * kSlot, src = slot + b * kBlock + (is_v ? kBlock / 2 : 0u);
      uint32_t pair = there ? lds32(src + GR * 512u + (GR == 2 ? (uint32_t)part * 64u : 0u) + (uint32_t)tok * 4u) : 0u;
      // a token that is not finite shows in its scores; rows that do not see it must not meet it in V
      if (is_v && (!(fabsf(lo_bf16(pair)) <= 3.4e38f) || !(fabsf(hi_bf16(pair)) <= 3.4e38f))) pair = 0u;
      const uint32_t e = is_v ? info >> 24 : info >> 16 & 0xffu;
      uint32_t q[GR][4];
#pragma unroll
      for (int x = 0; x < GR; ++x) lds128(src + (GR == 2 ? (uint32_t)(part * 512 + tok * 32 + 16 * x) : (uint32_t)(tok * 32 + 16 * part)), q[x]);
      if (i >= kStages && !warp_wait((is_v ? v_empty : k_empty) + 8 * s, (i / kStages - 1u) & 1u, abort_flag, p.status, 81)) break;
      const float down = __uint_as_float((254u - e) << 23);
      const __half2 s2 = __float2half2_rn(lo_bf16(pair) * down), z2 = __float2half2_rn(hi_bf16(pair) * down);
      const uint32_t dst = (is_v ? v_at : k_at) + s * kStage + (b * 16u + (uint32_t)tok) * 128u + (GR == 2 ? (uint32_t)part * (kTileBytes / 2) : 0u);
#pragma unroll
      for (int x = 0; x < GR; ++x)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t lo = q[x][w], hi = lo >> 8;   // elements (0, 4), (1, 5), (2, 6), (3, 7)
          uint32_t o[4] = {code_of_low(low_codes(lo, k1024)), code_of_high(high_codes(lo, k1024)), code_of_low(low_codes(hi, k1024)),
                           code_of_high(high_codes(hi, k1024))};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __half2 y = __hfma2(*reinterpret_cast<const __half2*>(&o[j]), s2, z2);
            o[j] = *reinterpret_cast<const uint32_t*>(&y);
          }
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (uint32_t)((((GR == 2 ? 4 * x : 4 * part) + w) ^ (tok & 7)) << 4)), "r"(o[0]), "r"(o[1]),
                       "r"(o[2]), "r"(o[3])
                       : "memory");
        }
      fence_async_smem();
      __syncwarp();   // every lane has read its codes and written its elements
      if (lane == 0) {
        mbar_arrive((is_v ? v_full : k_full) + 8 * s);
        mbar_arrive(raw_empty + 8 * (i & 1u));
      }
    }
  } else if (warp == kLoadWarp) {
    // ------------------------------------------------------------------------------ codes from the pages
    const int bpp = p.page / DSN_CACHE_BLOCK;
    bool more = walk.next(p, it);
    int tile = it.c0, pg = -1, place = 0;   // page of this lane's block, the block in it
    bool exists = false;
    auto find = [&]() {
      const int key = it.s.lo + tile * kTile + DSN_CACHE_BLOCK * lane;
      exists = more && lane < kTile / DSN_CACHE_BLOCK && key <= it.s.me1;
      pg = -1;
      if (exists) {
        const int col = (int)dsn_div((uint32_t)key, p.by_page);
        pg = p.table[(int64_t)it.e.sample * p.max_pages + col];
        place = key / DSN_CACHE_BLOCK - col * bpp;
      }
    };
    // exponent of the largest element of the tile's K or V, held where 2^e and 2^-e are normal numbers; V's from 2^-50 up: fp32 holds the probabilities and
    // their sums without the power, too
    auto exponent = [&](uint32_t slot, uint32_t go, uint32_t skip, uint32_t left, bool of_v) -> uint32_t {
      uint32_t e = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int t = lane + 32 * i;
        const bool there = (go >> (t >> 4) & 1u) && t >= (int)skip && t < (int)left;
#pragma unroll
        for (int gr = 0; gr < GR; ++gr) {
          const uint32_t pr = lds32(slot + (uint32_t)(t >> 4) * kBlock + (of_v ? kBlock / 2 : 0u) + GR * 512 + gr * 64 + (t & 15) * 4);
          const float top = fabsf(hi_bf16(pr)) + 8.f * fabsf(lo_bf16(pr));
          if (there && top <= 3.4e38f) e = max(e, __float_as_uint(top) >> 23);
        }
      }
      return min(max(__reduce_max_sync(0xffffffffu, e), of_v ? 77u : 27u), 253u);
    };
    int asked = 0;   // tiles whose copies were issued
    find();
    for (uint32_t i = 0; more; ++i) {
      const uint32_t slot = i & 1u;
      if (i >= 2 && !warp_wait(raw_empty + 8 * slot, ((i >> 1) - 1u) & 1u, abort_flag, p.status, 91)) break;
      const bool ok = pg >= 0 && pg < p.n_pages, lost = exists && !ok;
      if (lost) dsn_set_status(p.status, DSN_ERR_BAD_INDEX, it.e.sample);
      const uint32_t go = __ballot_sync(0xffffffffu, ok), bad = __ballot_sync(0xffffffffu, lost);
      if (lane == 0) {
        mbar_expect_tx(raw_full + 8 * slot, (uint32_t)__popc(go) * kBlock);
      }
      __syncwarp();
      if (ok)
        dsn_bulk_load(raw_at + slot * kSlot + (uint32_t)lane * kBlock, p.pages + (((int64_t)pg * p.H + it.head) * bpp + place) * kBlock, kBlock,
                      raw_full + 8 * slot);
      ++asked;
      const uint32_t left = (uint32_t)min(max(it.s.me1 + 1 - (it.s.lo + tile * kTile), 0), kTile);
      // in front of the window of the item's first row: below 16, as tiles begin at its block
      const uint32_t skip = (uint32_t)max(dsn_cache_first_seen(it.s.me0, p.window) - (it.s.lo + tile * kTile), 0);
      if (++tile == it.c1) {
        more = walk.next(p, it);
        tile = it.c0;
      }
      find();
      // what the tile's K and V are divided by, from their pairs
      if (!warp_wait(raw_full + 8 * slot, (i >> 1) & 1u, abort_flag, p.status, 93)) break;
      const uint32_t ke = exponent(raw_at + slot * kSlot, go, skip, left, false), ve = exponent(raw_at + slot * kSlot, go, skip, left, true);
      if (lane == 0) {
        s_bad[i & 15u] = (uint8_t)bad;
        s_fac[i & 15u] = make_float2(__uint_as_float(ke << 23), (float)((int)ve - 127));
        *reinterpret_cast<volatile uint32_t*>(s_raw + slot) = go | skip << 4 | left << 8 | ke << 16 | ve << 24;
        mbar_arrive(raw_ready + 8 * slot);
      }
      __syncwarp();
    }
    if (*abort_flag) dsn_drain(raw_full, 2, max(0, asked - 2), asked);   // the tile whose wait ran out among them
  } else if (warp < kSoftWarp) {
    // ------------------------------------------------------------------------------ products
    // A warp issues what one half needs.  The scores of tile number m (of those that the half needs) go to buffer m & 1, which the product with the
    // probabilities of number m - 2 has read by then: that one is issued first, so up to two of them wait for their softmax.
    const int h = warp - kIssueWarp;
    const uint32_t f16 = ~((1u << 7) | (1u << 10));                                               // both operands fp16
    const uint32_t idesc_s = make_idesc(128, kTile) & f16, idesc_o = (make_idesc(128, D) & f16) | (1u << 16);   // V: elements first
    const uint32_t region = tmem + h * kRegion;
    const uint64_t dq = make_smem_desc(q_at + h * kOperand);
    uint32_t n = 0, freed = 0;                     // tiles so far; stages of V given back
    uint32_t n_s = 0, n_p = 0, n_q = 0, n_o = 0;   // scores and products issued, Q waited for, items begun
    uint32_t at0 = 0, at1 = 0;                     // tiles of the products that are due, the older first
    bool first0 = false, first1 = false;           // of those: the first of an item
    bool ok = true;
    auto pv = [&]() {   // O_h (+)= P_h V, the oldest that is due
      const uint32_t s = at0 % kStages, buf = n_p & 1u;
      ok = ok && warp_wait(p_full + 16 * h + 8 * buf, (n_p >> 1) & 1u, abort_flag, p.status, 83);
      ok = ok && warp_wait(v_full + 8 * s, (at0 / kStages) & 1u, abort_flag, p.status, 84);
      if (first0 && n_o++ > 0) ok = ok && warp_wait(o_empty + 8 * h, (n_o - 2u) & 1u, abort_flag, p.status, 85);
      if (!ok) return;
      if (elect_one()) {
        tc_fence_after();
        const uint64_t dv = make_desc_mn(v_at + s * kStage);
#pragma unroll
        for (int ks = 0; ks < kTile / 16; ++ks)
          mma_a_tmem(region + kOCol, region + kTile * buf + 8u * ks, dv + 128u * ks, idesc_o, ks > 0 ? 1u : (first0 ? 0u : 1u));
        umma_commit(o_full + 16 * h + 8 * buf);
      }
      __syncwarp();
      ++n_p;
      at0 = at1;
      first0 = first1;
    };
    auto release = [&](uint32_t bar) {
      if (elect_one()) umma_commit(bar);
      __syncwarp();
    };
    while (ok && walk.next(p, it)) {
      int a, b;
      half_tiles(it, h, p.by_group, p.window, a, b);
      for (int j = it.c0; j < it.c1 && ok; ++j, ++n) {
        const uint32_t s = n % kStages;
        const bool needed = j >= a && j < b;
        // a half that rests owes nothing: its softmax must come to the end of its item to fetch the next one's Q, and V's stages must come back
        while (n_s - n_p > (needed ? 1u : 0u) && ok) pv();
        if (needed && j == a) ok = ok && warp_wait(q_full + 8 * h, n_q++ & 1u, abort_flag, p.status, 86);
        ok = ok && warp_wait(k_full + 8 * s, (n / kStages) & 1u, abort_flag, p.status, 87);
        if (!ok) break;
        if (elect_one()) {
          if (needed) {
            tc_fence_after();
            const uint64_t dk = make_smem_desc(k_at + s * kStage);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
              umma_bf16(region + kTile * (n_s & 1u), dq + (uint32_t)(ks >> 2) * (kTileBytes >> 4) + 2u * (ks & 3),
                        dk + (uint32_t)(ks >> 2) * (kTileBytes >> 5) + 2u * (ks & 3), idesc_s, ks > 0 ? 1u : 0u);
            umma_commit(s_full + 16 * h + 8 * (n_s & 1u));
          }
          umma_commit(k_empty + 8 * s);
        }
        __syncwarp();
        if (needed) {
          if (n_s == n_p) at0 = n, first0 = j == a;
          else at1 = n, first1 = j == a;
          ++n_s;
        }
        // V's stages that no product is due with
        const uint32_t due = n_s != n_p ? at0 : n + 1u;
        for (; freed < due && ok; ++freed) {
          ok = warp_wait(v_full + 8 * (freed % kStages), (freed / kStages) & 1u, abort_flag, p.status, 92);
          if (ok) release(v_empty + 8 * (freed % kStages));
        }
      }
    }
    while (n_s != n_p && ok) pv();
    if (!ok) products_end(idle + 8 * h);
  } else if (warp >= kSoftWarp) {
    // ------------------------------------------------------------------------------ softmax, a thread a row
    const int h = (warp - kSoftWarp) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t region = tmem + h * kRegion + ((uint32_t)(quarter * 32) << 16);
    const float c2 = fabsf(p.scale_log2);
    const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;   // a negative scale goes into Q's signs
    uint32_t m = 0, n = 0;   // tiles of the half, of both
    bool ok = true;
    // The warp's rows of Q as fp16, the largest element of each brought to 1 .. 2; returns the power of two that goes into the scores of this lane's row.
    // D / 8 lanes read a row; one in front of the first token sees nothing, whatever it holds.
    auto load_q = [&](const Item& x) -> float {
      constexpr int L = D / 8, PER = 32 / L, NB = 8;   // lanes a row, rows a load, loads at once
      const int v = x.s.v0 + 128 * h + row;
      const int r = (int)dsn_div((uint32_t)v, p.by_group), ev = v - r * p.group;
      const long long mine = v < x.s.v1 && x.e.len - x.e.rows + r >= 0 ? ((long long)(p.grouped ? x.e.pos : x.e.sample) * p.R + r) * p.ld_qkv + ((long long)x.head * (p.group + 2) + ev) * D
                                        : -1;
      const int sub = lane % L, of = lane / L;
      uint32_t my_e = 127u;
#pragma unroll
      for (int b = 0; b < 32; b += NB * PER) {
        uint4 w[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const long long at = __shfl_sync(0xffffffffu, mine, b + i * PER + of);
          w[i] = at >= 0 ? *reinterpret_cast<const uint4*>(p.qkv + at + 8 * sub) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const int rr = b + i * PER + of, row_at = quarter * 32 + rr;
          const uint32_t m2 = __vmaxu2(__vmaxu2(w[i].x & 0x7fff7fffu, w[i].y & 0x7fff7fffu), __vmaxu2(w[i].z & 0x7fff7fffu, w[i].w & 0x7fff7fffu));
          uint32_t e = max(m2 & 0xffffu, m2 >> 16);
#pragma unroll
          for (int o = 1; o < L; o <<= 1) e = max(e, __shfl_xor_sync(0xffffffffu, e, o));
          e >>= 7;
          e = e == 255u ? e : min(max(e, 27u), 253u);
          const uint32_t given = __shfl_sync(0xffffffffu, e, (lane % PER) * L);
          if (lane / PER == b / PER + i) my_e = given;
          const float down = __uint_as_float((254u - e) << 23);
          const uint32_t y0 = w[i].x ^ flip, y1 = w[i].y ^ flip, y2 = w[i].z ^ flip, y3 = w[i].w ^ flip;
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_at + h * kOperand + (uint32_t)row_at * 128u + (uint32_t)(sub >> 3) * kTileBytes +
                                                                        (uint32_t)(((sub & 7) ^ (row_at & 7)) << 4)),
                       "r"(pack_f16(lo_bf16(y0) * down, lo_bf16(y2) * down)), "r"(pack_f16(hi_bf16(y0) * down, hi_bf16(y2) * down)),
                       "r"(pack_f16(lo_bf16(y1) * down, lo_bf16(y3) * down)), "r"(pack_f16(hi_bf16(y1) * down, hi_bf16(y3) * down))
                       : "memory");
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full + 8 * h);
      // NaN for a row that is not finite: an infinity alone could give all tokens scores of minus infinity, as if the row saw none
      return my_e == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(my_e << 23);
    };
    // the lines of this lane's row of Q on their way to the second level of cache
    auto warm_q = [&](const Item& x) {
      const int v = x.s.v0 + 128 * h + row;
      if (v >= x.s.v1) return;
      const int r = (int)dsn_div((uint32_t)v, p.by_group), ev = v - r * p.group;
      const __nv_bfloat16* q = p.qkv + ((int64_t)(p.grouped ? x.e.pos : x.e.sample) * p.R + r) * p.ld_qkv + ((int64_t)x.head * (p.group + 2) + ev) * D;
#pragma unroll
      for (int i = 0; i < D; i += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + i));
    };
    CachePart ends{3, 0, 0, 0, 0, 0, 0, 0};   // what the CTA has to say about the ends of its stretch; rows: the tail's first vector, pad: one behind its last
    bool have = walk.next(p, it);
    int a = 0, b = 0;
    float up = 1.f, up_next = 1.f;
    if (have) {
      half_tiles(it, h, p.by_group, p.window, a, b);
      if (a < b) up = load_q(it);
    }
    while (have && ok) {
      Item nx;
      int na = 0, nb = 0;
      have = walk.next(p, nx);
      if (have) half_tiles(nx, h, p.by_group, p.window, na, nb);
      const int v = it.s.v0 + 128 * h + row;
      const bool live = v < it.s.v1;
      const int me = it.e.len - it.e.rows + (int)dsn_div((uint32_t)v, p.by_group);
      float ref = kLowest, l = 0.f;
      const float cs = c2 * up;
      // tiles that all rows of the warp see whole: plain0 .. plain1 - 1 (rows in a row: the first sees least, the last begins last)
      const int first_me = __reduce_min_sync(0xffffffffu, live ? me : INT32_MAX), last_me = __reduce_max_sync(0xffffffffu, live ? me : INT32_MIN);
      const int plain1 = first_me == INT32_MAX ? INT32_MAX : max(0, first_me + 1 - it.s.lo) / kTile;
      const int plain0 = p.window && last_me != INT32_MIN ? (max(0, last_me - p.window + 1 - it.s.lo) + kTile - 1) / kTile : 0;
      if (na < nb) warm_q(nx);
      if (a == b && na < nb) up_next = load_q(nx);
      for (int j = a; j < b && ok; ++j) {
        const uint32_t buf = m & 1u;
        ok = warp_wait(s_full + 16 * h + 8 * buf, (m >> 1) & 1u, abort_flag, p.status, 88);
        if (!ok) break;
        tc_fence_after();
        if (j + 1 == b && na < nb) up_next = load_q(nx);   // every product with this item's Q has run
        if (first_me == INT32_MAX) {   // rows that do not exist: whatever stands in their lanes stays there
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full + 16 * h + 8 * buf);
          ++m;
          continue;
        }
        const uint32_t at = region + kTile * buf;
        const uint32_t nt = (n + (uint32_t)(j - it.c0)) & 15u;
        const uint32_t bad = *reinterpret_cast<const volatile uint8_t*>(s_bad + nt);
        // scores to units of the exponent (not 0: what is hidden is -infinity), V's power of two
        const float2 fac = s_fac[nt];
        const float t = max3_nan(cs * fac.x, 1e-37f, 1e-37f), sh = fac.y;
        uint32_t x[2][32];
        tmem_ld_32x32(at, x[0]);
        tmem_ld_32x32(at + 32, x[1]);
        tmem_ld_wait();
        if (j < plain0 || j >= plain1 || bad != 0) {   // columns that the row does not see
          const int t0 = it.s.lo + j * kTile, k1 = me + 1 - t0, k0 = p.window ? me - p.window + 1 - t0 : 0;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int e1 = min(max(k1 - 32 * c, 0), 32), e0 = min(max(k0 - 32 * c, 0), 32);
            uint32_t m = (e1 >= 32 ? 0xffffffffu : (1u << e1) - 1u) & (e0 >= 32 ? 0u : 0xffffffffu << e0);
            if (bad >> (2 * c) & 1u) m &= 0xffff0000u;
            if (bad >> (2 * c) & 2u) m &= 0x0000ffffu;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!(m >> i & 1u)) x[c][i] = 0xff800000u;
          }
        }
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 32; i += 4)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            top[k] = max3_nan(top[k], __uint_as_float(x[k >> 1][i + 2 * (k & 1)]), __uint_as_float(x[k >> 1][i + 2 * (k & 1) + 1]));
        const float need = fmaf(max3_nan(max3_nan(top[0], top[1], top[2]), top[3], top[3]), t, sh);
        if (need != need) l = need;   // a token that is not finite: so is the row
        if (__any_sync(0xffffffffu, need > ref + kTop)) {
          const float to = fmaxf(ref, need - kAim), f = ex2(0.5f * (ref - to));   // twice: references can lie further apart than fp32 reaches
          ref = to;
          l = l * f * f;
          if (j > a) {
            ok = warp_wait(o_full + 16 * h + 8 * (buf ^ 1u), ((m - 1u) >> 1) & 1u, abort_flag, p.status, 89);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 8) {
              uint32_t y[8];
              tmem_ld_8(region + kOCol + c, y);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = __float_as_uint(__uint_as_float(y[i]) * f * f);
              tmem_st_8(region + kOCol + c, y);
            }
          }
        }
        const uint64_t t_2 = pack2(t, t), ref_2 = pack2(sh - ref, sh - ref);
        uint64_t sum_a = pack2(0.f, 0.f), sum_b = sum_a;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float t0, t1;
            unpack2(ffma2(pack2(__uint_as_float(x[c][2 * e]), __uint_as_float(x[c][2 * e + 1])), t_2, ref_2), t0, t1);
            const float x0 = ex2(t0), x1 = ex2(t1);
            if (e & 1) sum_b = fadd2(sum_b, pack2(x0, x1)); else sum_a = fadd2(sum_a, pack2(x0, x1));
            x[c][e] = pack_f16(x0, x1);
          }
          tmem_st_16(at + (uint32_t)(16 * c), x[c]);
        }
        float s0, s1;
        unpack2(fadd2(sum_a, sum_b), s0, s1);
        l = fmaf(s0 + s1, __uint_as_float((127u - (uint32_t)(int)sh) << 23), l);   // in units of 2^ref, without V's power
        tmem_st_done();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 16 * h + 8 * buf);
        ++m;
      }
      if (!ok) break;
      const bool ran = a < b;
      if (ran) {
        ok = warp_wait(o_full + 16 * h + 8 * ((m - 1u) & 1u), ((m - 1u) >> 1) & 1u, abort_flag, p.status, 90);
        if (!ok) break;
        tc_fence_after();
      }
      const bool whole = it.c0 == 0 && it.c1 == it.s.tiles;
      const int r = (int)dsn_div((uint32_t)v, p.by_group), ev = v - r * p.group;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      __nv_bfloat16* dst = p.out + ((int64_t)(p.grouped ? it.e.pos : it.e.sample) * p.R + r) * p.ld_out + ((int64_t)it.head * p.group + ev) * D;
      // a part: references, sums, then four elements of every row after the other
      float* part = p.cta_data + ((int64_t)blockIdx.x * 2 + (it.c0 == 0)) * (kRows * (D + 2)) + 128 * h + row;
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        if (ran) {
          tmem_ld_32x32(region + kOCol + c, o);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0u;
        }
        if (c + 32 == D && ran) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(o_empty + 8 * h);
        }
        if (!live) continue;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          float y[8];   // columns 0 4 1 5 2 6 3 7
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(o[8 * x + i]);
          if (whole) {
            uint4 w;
            w.x = pack_bf16(y[0] * inv, y[2] * inv);
            w.y = pack_bf16(y[4] * inv, y[6] * inv);
            w.z = pack_bf16(y[1] * inv, y[3] * inv);
            w.w = pack_bf16(y[5] * inv, y[7] * inv);
            *reinterpret_cast<uint4*>(dst + c + 8 * x) = w;
          } else {
            float* to = part - (128 * h + row) + 2 * kRows + (int64_t)((c + 8 * x) / 4) * (4 * kRows) + 4 * (128 * h + row);
            *reinterpret_cast<float4*>(to) = make_float4(y[0], y[2], y[4], y[6]);
            *reinterpret_cast<float4*>(to + 4 * kRows) = make_float4(y[1], y[3], y[5], y[7]);
          }
        }
      }
      if (!whole && live) {
        part[0] = ref;
        part[kRows] = l;
      }
      if (it.c0 > 0) ends.head_state = it.c1 == it.s.tiles ? 1 : 2;
      else if (ends.head_state == 3) ends.head_state = 0;
      if (it.c0 == 0 && !whole)
        ends = CachePart{ends.head_state, 1, it.e.sample, it.e.pos, it.head, it.s.v0, 0, it.s.v1};
      n += (uint32_t)(it.c1 - it.c0);
      it = nx;
      a = na;
      b = nb;
      up = up_next;
    }
    if (!ok) ends.head_state = 3, ends.tail = 0;
    if (warp == kSoftWarp && lane == 0) p.parts[blockIdx.x] = ends;
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarp) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Joins the parts of the items that were cut: rows of a CTA's last item by threads, D / 8 CTAs for the elements.
template <int D>
__global__ void __launch_bounds__(kRows) cache_rows_join_kernel(const __grid_constant__ CacheAttParams p, int ctas) {
  __shared__ int s_end;
  dsn_grid_dependency_wait();
  dsn_grid_launch_dependents();
  const int w = blockIdx.x, c = 8 * blockIdx.y, i = threadIdx.x;
  const CachePart part = p.parts[w];
  if (!part.tail) return;
  if (i == 0) s_end = ctas - 1;
  __syncthreads();
  for (int b = w + 1 + i; b < ctas; b += kRows)
    if (p.parts[b].head_state < 2) atomicMin(&s_end, b);
  __syncthreads();
  const int v = part.rows + i, end = s_end;
  if (v >= part.pad) return;
  float m = kLowest, l = 0.f, y[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) y[x] = 0.f;
#pragma unroll 4
  for (int j = w; j <= end; ++j) {
    if (j > w && p.parts[j].head_state == 3) continue;
    const float* src = p.cta_data + ((int64_t)j * 2 + (j == w)) * (kRows * (D + 2));
    const float4 q0 = *reinterpret_cast<const float4*>(src + 2 * kRows + (int64_t)(c / 4) * (4 * kRows) + 4 * i);
    const float4 q1 = *reinterpret_cast<const float4*>(src + 2 * kRows + (int64_t)(c / 4 + 1) * (4 * kRows) + 4 * i);
    const float mj = src[i], lj = src[kRows + i], m2 = fmaxf(m, mj), fa = ex2(0.5f * (m - m2)), fb = ex2(0.5f * (mj - m2));   // twice, as above
    m = m2;
    l = l * fa * fa + lj * fb * fb;
    y[0] = y[0] * fa * fa + q0.x * fb * fb; y[1] = y[1] * fa * fa + q0.y * fb * fb; y[2] = y[2] * fa * fa + q0.z * fb * fb; y[3] = y[3] * fa * fa + q0.w * fb * fb;
    y[4] = y[4] * fa * fa + q1.x * fb * fb; y[5] = y[5] * fa * fa + q1.y * fb * fb; y[6] = y[6] * fa * fa + q1.z * fb * fb; y[7] = y[7] * fa * fa + q1.w * fb * fb;
  }
  const int r = v / p.group, ev = v - r * p.group;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint4 o;
  o.x = pack_bf16(y[0] * inv, y[1] * inv);
  o.y = pack_bf16(y[2] * inv, y[3] * inv);
  o.z = pack_bf16(y[4] * inv, y[5] * inv);
  o.w = pack_bf16(y[6] * inv, y[7] * inv);
  *reinterpret_cast<uint4*>(p.out + ((int64_t)(p.grouped ? part.pos : part.sample) * p.R + r) * p.ld_out + ((int64_t)part.head * p.group + ev) * D + c) = o;
}

template <int D>
cudaError_t launch(const CacheAttParams& p, int ctas, cudaStream_t s) {
  static size_t configured[DSN_MAX_DEVICES] = {};
  constexpr size_t smem = 1024 + kCtrlR + 6 * (size_t)(D / 64) * kTileBytes + 2 * (kTile / DSN_CACHE_BLOCK) * dsn_cache_block_bytes(D);
  static_assert(smem <= 227 * 1024, "shared memory of a CTA");
  cudaError_t e = dsn_ensure_dynamic_smem(cache_rows_kernel<D>, smem, configured);
  if (e != cudaSuccess) return e;
  e = dsn_launch(cache_rows_kernel<D>, dim3((unsigned)ctas), dim3(kThreadsR), smem, s, 1, p);
  if (e != cudaSuccess) return e;
  return dsn_launch(cache_rows_join_kernel<D>, dim3((unsigned)ctas, D / 8), dim3(kRows), 0, s, 1, p, ctas);
}

struct RowsWorkspace {
  size_t parts, list, data, total;
};
RowsWorkspace carve(int D, int64_t B, int ctas) {
  RowsWorkspace w;
  w.parts = 0;
  w.list = w.parts + sizeof(CachePart) * (size_t)ctas;
  w.data = w.list + sizeof(CacheEntry) * (size_t)B;
  w.total = w.data + (size_t)ctas * 2 * kRows * (D + 2) * sizeof(float);
  return w;
}

}  // namespace

size_t dsn_cache_rows_ws_bytes(int D, int64_t B) { return carve(D, B, DSN_CACHE_MAX_CTAS).total; }

cudaError_t dsn_launch_cache_attention_rows(CacheAttParams& p, int D, int sm_count, void* workspace, cudaStream_t s) {
  const int ctas = sm_count < DSN_CACHE_MAX_CTAS ? sm_count : DSN_CACHE_MAX_CTAS;
  const RowsWorkspace w = carve(D, p.B, ctas);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.parts = reinterpret_cast<CachePart*>(ws + w.parts);
  p.list = reinterpret_cast<CacheEntry*>(ws + w.list);
  p.cta_data = reinterpret_cast<float*>(ws + w.data);
  return D == 64 ? launch<64>(p, ctas, s) : launch<128>(p, ctas, s);
}
