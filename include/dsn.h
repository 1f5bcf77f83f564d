/*
 * dsn.h -- C ABI of the dynamic-weight-slicing inference library (NVIDIA B200, sm_100a).
 *
 * The library runs the batched inference path of DS-Net++ ("Dynamic Weight Slicing"):
 * a per-sample gate picks one of T paths, samples are grouped by path, every group runs a
 * dense contraction against the leading slice W[:k_out, :k_in] of the statically stored
 * full weight, and results return in input order.
 *
 * Conventions
 *   - Every function returns DSN_OK (0) or a negative dsn_status code.  No exceptions, no abort.
 *   - "device" pointers are CUDA device memory of the context's GPU; "host" pointers are
 *     ordinary host memory.  The caller owns every buffer; the library owns only dsn_ctx.
 *     No entry point allocates memory per call unless its comment says so.
 *   - Calls are asynchronous on `stream` (a cudaStream_t passed as void*; NULL = default stream).
 *     Errors the host can detect are returned at once and nothing is launched.  Conditions only
 *     the device can detect (routing index out of range, a bounded wait that ran out, non-finite
 *     gate scores) are recorded in a device status word read by dsn_get_status().
 *   - Weights are stored [out][in] (linear) or [out][KH][KW][in] (convolution, "OHWI"),
 *     row-major, and are never modified, copied or repacked.  Activations are [B][R][C]
 *     (tokens) or [B][H][W][C] (channels last); R = H*W.
 *   - Paths are numbered 0..T-1 (the paper numbers them 1..|t|, smallest first).
 */
#ifndef DSN_H
#define DSN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct dsn_ctx dsn_ctx;

enum dsn_status {
  DSN_OK = 0,
  DSN_ERR_INVALID_ARG = -1, /* NULL pointer, non-positive size, k > C, T out of range ...   */
  DSN_ERR_ALIGNMENT = -2,   /* a pointer or leading dimension breaks the stated alignment  */
  DSN_ERR_WORKSPACE = -3,   /* workspace missing or smaller than dsn_*_workspace_bytes      */
  DSN_ERR_UNSUPPORTED = -4, /* a combination this build has no kernel for                  */
  DSN_ERR_BAD_INDEX = -5,   /* (device) a routing index outside [0, T)                     */
  DSN_ERR_CUDA = -6,        /* a CUDA runtime / driver call failed                         */
  DSN_ERR_TIMEOUT = -7,     /* (device) a bounded wait inside a kernel ran out             */
  DSN_ERR_NONFINITE = -8,   /* (device) a gate score was NaN or infinite                   */
  DSN_ERR_CACHE_FULL = -9   /* (device) a request's new tokens found no room in the cache  */
};

enum dsn_dtype { DSN_F32 = 0, DSN_BF16 = 1 };
/* DSN_ACT_GELU: x/2 (1 + erf(x / sqrt 2)).  How a kernel evaluates it, and how far from the erf form that is, before the output is rounded:
 *   bf16 layers, and 8-bit layers with bf16 outputs of more than 32 rows (B * R): erf as the hardware tanh of a fitted odd quintic,
 *     within 3e-5 + |x| 2^-12 (1e-3 at |x| = 4: a fraction of a bfloat16 rounding step at x = 4, more than the value itself at x = -4);
 *   8-bit layers with fp32 outputs of more than 32 rows: formula 7.1.26 of Abramowitz and Stegun, within 0.75e-7 |x| besides roundings;
 *   fp32 layers, depthwise layers (unless DSN_DWPW=fused joins them with the next layer: the first form) and 8-bit layers of at most 32 rows: erff.
 * A row of an 8-bit layer can therefore differ by these bounds between a call of 32 rows and one of 33. */
enum dsn_act { DSN_ACT_NONE = 0, DSN_ACT_RELU = 1, DSN_ACT_GELU = 2 };
enum dsn_order { DSN_INPUT_ORDER = 0, DSN_GROUPED = 1 };
enum dsn_tail { DSN_TAIL_UNTOUCHED = 0, DSN_TAIL_ZERO = 1 };
/* Frequencies of rotary positions: one ladder over all pairs of a head, or one ladder for each axis. */
enum dsn_rotary_ladder { DSN_ROTARY_SHARED = 0, DSN_ROTARY_PER_AXIS = 1 };
/* Which elements of a head turn together: (i, i + pairs) or (2 i, 2 i + 1). */
enum dsn_rotary_pairing { DSN_ROTARY_HALVES = 0, DSN_ROTARY_INTERLEAVED = 1 };
enum dsn_layer_kind { DSN_LAYER_LINEAR = 0, DSN_LAYER_CONV = 1, DSN_LAYER_ATTENTION = 2, DSN_LAYER_DEPTHWISE = 3 };

#define DSN_MAX_SLICES 64   /* largest T                                               */
#define DSN_MAX_GROUPS 4096 /* largest G of a caller-built group list                  */
#define DSN_MAX_CHAIN 6     /* layers per dsn_layer_forward call (a ViT block: QKV, attention, proj, fc1, fc2) */

/* Batch grouping (not in the paper, which defines only per-sample behaviour, Eq. (dyn_net):
 * every input runs the path its own gate picks).  Grouped position p holds sample perm[p];
 * group g occupies positions offsets[g] .. offsets[g+1]-1 and uses slice group_slice[g]
 * (slice g when group_slice is NULL).  dsn_route() fills it with G = T; a caller may instead
 * build any list of G <= DSN_MAX_GROUPS groups, several of which may share a slice.
 * All five arrays are device memory. */
typedef struct dsn_routing {
  int32_t B;                  /* samples                                                 */
  int32_t G;                  /* groups                                                  */
  int32_t* counts;            /* [G]                                                     */
  int32_t* offsets;           /* [G+1], exclusive prefix sum of counts                   */
  int32_t* perm;              /* [B]                                                     */
  int32_t* inv_perm;          /* [B], inv_perm[perm[p]] = p                              */
  const int32_t* group_slice; /* [G] or NULL                                             */
} dsn_routing;

/* Gate routing head (Sec. 3.5): X_E = mean over the R positions; scores = W2 ReLU(W1 X_E);
 * index = first position of the maximum score. */
typedef struct dsn_gate_desc {
  int32_t dtype;   /* dtype of x: DSN_BF16 or DSN_F32                                    */
  int32_t B, R;    /* samples, positions per sample                                      */
  int32_t C_full;  /* columns of W1                                                      */
  int32_t c_valid; /* leading channels of x that are read (elastic input), <= C_full     */
  int32_t C_mlp;   /* hidden width                                                       */
  int32_t T;       /* number of paths, 1..DSN_MAX_SLICES                                 */
  int64_t ldx;     /* elements between consecutive positions of x, >= c_valid            */
  const float* W1; /* device [C_mlp][C_full] fp32                                        */
  const float* b1; /* device [C_mlp] or NULL                                             */
  const float* W2; /* device [T][C_mlp] fp32                                             */
  const float* b2; /* device [T] or NULL                                                 */
} dsn_gate_desc;

/* Sliced linear layer (Eq. (weight_slicing); ViT forms in Sec. 3.4):
 * y[i][r][o] = act(bias[o] + sum_{c < k_in[t]} x[i][r][c] * W[o][c]),  o < k_out[t],  t = path of i. */
typedef struct dsn_linear_desc {
  int32_t dtype;        /* DSN_BF16 (x, W, y bf16; fp32 accumulate) or DSN_F32 (all fp32, plain FMA) */
  int32_t R;            /* rows per sample                                               */
  int32_t C_in, C_out;  /* full extents                                                  */
  int64_t ldx, ldw, ldy;/* elements between rows of x, W, y.  bf16: multiples of 8       */
  int32_t T;
  const int32_t* k_in;  /* host [T], 1..C_in                                             */
  const int32_t* k_out; /* host [T], 1..C_out                                            */
  const void* W;        /* device [C_out][ldw]; bf16: 16-byte aligned                    */
  const float* bias;    /* device [C_out] fp32 or NULL                                   */
  const float* bn_scale;/* device [T][C_out] fp32 or NULL: per-path affine a_t of Re-SBN (dsn_resbn_fold) */
  const float* bn_shift;/* device [T][C_out] fp32 (required with bn_scale): b_t          */
  const void* residual; /* device, same dtype, order and leading dimension as y, or NULL: the skip features of a
                           residual block (Sec. 5, DS-ResNet), added before the activation; may not alias y */
  int32_t act;          /* dsn_act; order of operations: contraction, + bias, * a_t + b_t, + residual, activation */
  int32_t in_order;     /* dsn_order of x: INPUT_ORDER [B][R][ldx] by sample, or GROUPED by position */
  int32_t out_order;    /* dsn_order of y                                                */
  int32_t tail;         /* dsn_tail: columns >= k_out[t] left untouched, or zero-filled up to C_out */
} dsn_linear_desc;

/* Slice-able convolution, filter-number / input-channel slicing (Sec. 3.3):
 * y = W[:k_out, :k_in] * x, cross-correlation, zero padding, stride 1, K = 2*pad+1 in {1, 3}. */
typedef struct dsn_conv_desc {
  int32_t dtype;        /* DSN_BF16 only                                                 */
  int32_t H, W_;        /* spatial size (output = input size)                            */
  int32_t K, pad;       /* kernel size 1 (pad 0) or 3 (pad 1)                            */
  int32_t C_in, C_out;
  int64_t ldx, ldy;     /* elements between pixels of x, y; multiples of 8               */
  int32_t T;
  const int32_t* k_in;  /* host [T]                                                      */
  const int32_t* k_out; /* host [T]                                                      */
  const void* W;        /* device [C_out][K][K][C_in] bf16, dense, 16-byte aligned, C_in % 8 == 0 */
  const float* bias;
  const float* bn_scale;/* as in dsn_linear_desc                                         */
  const float* bn_shift;
  const void* residual; /* as in dsn_linear_desc                                         */
  int32_t act;
  int32_t in_order, out_order, tail;
} dsn_conv_desc;

/* Slice-able depthwise convolution (Sec. 3.3: group convolution whose group count follows the elastic
 * input width; kernel-size slicing = the centred k x k part of the K x K filter; the padding follows
 * the kernel size so that every k gives the same output size).  x [B][H][W][ldx], y [B][Ho][Wo][ldy]
 * channels last with Ho = (H-1)/stride + 1; filter [K][K][C] bf16 (channels last), K odd <= 7.
 * A sample of path t uses channels < c[t] and kernel size ksize[t]. */
typedef struct dsn_depthwise_desc {
  int32_t dtype;         /* DSN_BF16                                                     */
  int32_t H, W_;         /* input size                                                   */
  int32_t K;             /* stored kernel size (odd, <= 7)                               */
  int32_t stride;        /* 1 or 2                                                       */
  int32_t C;             /* full channel count                                           */
  int64_t ldx, ldy;      /* elements between pixels of x, y (>= C)                       */
  int32_t T;
  const int32_t* c;      /* host [T] channels of each path, 1..C                         */
  const int32_t* ksize;  /* host [T] kernel size of each path, odd, <= K                 */
  const void* W;         /* device [K][K][C] bf16                                        */
  const float* bias;     /* device [C] or NULL                                           */
  const float* bn_scale; /* device [T][C] or NULL (dsn_resbn_fold)                       */
  const float* bn_shift;
  int32_t act;
  int32_t in_order, out_order;
} dsn_depthwise_desc;

/* Slimmable self-attention core (Sec. 3.4): A_a = Softmax(Q_a K_a^T / sqrt(D_h)) V_a for the h heads of
 * the sample's path, concatenated.  qkv rows are laid out [head][q|k|v][D_h] (the output of the sliced
 * QKV layer with the head-major fused weight), out rows [head][D_h]; heads >= h are neither read nor
 * written.  qkv and out are both in `order` (all rows of a sample are contiguous either way). */
typedef struct dsn_attention_desc {
  int32_t dtype;        /* DSN_BF16                                                      */
  int32_t N;            /* tokens per sample, 1..256                                     */
  int32_t H, D_h;       /* full head count; head dimension (64)                          */
  int64_t ld_qkv;       /* elements between rows of qkv, >= 3*H*D_h, multiple of 8       */
  int64_t ld_out;       /* elements between rows of out, >= H*D_h, multiple of 8         */
  int32_t T;
  const int32_t* heads; /* host [T]: head count of each path, 1..H                       */
  int32_t order;        /* dsn_order of qkv and out                                      */
} dsn_attention_desc;

/* Pre-norm of a transformer block on elastic widths, with the residual's addition before it and 8-bit codes behind it
 * (not in the paper, whose blocks are evaluated in one precision).  A row of a sample of path t has k[t] columns:
 *   h = x + residual                                     (fp32; h = x without a residual)
 *   n = h / sqrt(mean_c h^2 + eps) * weight              (fp32)
 *   s = max_c |n| / 127,   q = round(n / s) to the nearest, ties to even, in -127 .. 127   (an all-zero row: s = 0, q = 0)
 * The code is computed as round(h weight * (127 * (1 / max|h weight|))) in fp32, each operation rounded once: the factor that
 * all columns share drops out, so a code does not depend on the order of the sum of squares.
 * A row that holds a NaN or an infinity comes out as s = NaN, q = 0, y = NaN.  Rows whose squares, or products with the weight, leave the range
 * of fp32 do not: they are scaled by powers of two, which changes neither code nor n. */
typedef struct dsn_norm_desc {
  int32_t dtype;        /* DSN_BF16 or DSN_F32: x, residual, sum, y                      */
  int32_t R;            /* rows per sample                                               */
  int32_t C;            /* full width, 1..32767                                          */
  int64_t ldx, ld_res, ld_sum, ldy; /* elements between rows of x, residual, sum, y: multiples of 16 bytes, >= C */
  int64_t ldq;          /* bytes between rows of q: a multiple of 16, >= C               */
  int32_t T;
  const int32_t* k;     /* host [T], 1..C                                                */
  const float* weight;  /* device [C], 16-byte aligned, or NULL (all ones)               */
  float eps;            /* 1e-20 or more, finite                                         */
  int32_t in_order;     /* dsn_order of x, residual and sum (the stream keeps its order) */
  int32_t out_order;    /* dsn_order of q, q_scale and y: the gather to grouped order is part of the pass */
} dsn_norm_desc;

/* Sliced linear layer on 8-bit integers with a scale for every row of x and for every output channel:
 *   y[i][r][o] = act((sum_{c < k_in[t]} x[i][r][c] W[o][c]) * x_scale[i][r] * w_scale[o] + bias[o] ...),  o < k_out[t],
 * the products summed exactly in 32-bit integers; everything behind the sum as in dsn_linear_desc, in fp32. */
typedef struct dsn_linear_i8_desc {
  int32_t R;
  int32_t C_in, C_out;
  int64_t ldx, ldw;     /* bytes between rows of x, W: multiples of 16, >= C_in          */
  int64_t ldy;          /* elements between rows of y and residual: a multiple of 16 bytes, >= C_out */
  int32_t T;
  const int32_t* k_in;  /* host [T], 1..C_in                                             */
  const int32_t* k_out; /* host [T], 1..C_out                                            */
  const int8_t* W;      /* device [C_out][ldw], 16-byte aligned                          */
  const float* w_scale; /* device [C_out]                                                */
  const float* bias;    /* device [C_out] or NULL                                        */
  const float* bn_scale;/* device [T][C_out] or NULL, as in dsn_linear_desc              */
  const float* bn_shift;
  const void* residual; /* as in dsn_linear_desc: y's type, order and leading dimension  */
  int32_t y_dtype;      /* DSN_BF16 or DSN_F32: y and residual                           */
  int32_t act;          /* dsn_act; which form of GELU runs depends on y_dtype and on the number of rows (see there) */
  int32_t in_order;     /* dsn_order of x and x_scale                                    */
  int32_t out_order;    /* dsn_order of y and residual                                   */
  int32_t tail;
} dsn_linear_i8_desc;

/* Rotary positions with one to three axes (time, height, width of image and video tokens; one axis: text).
 * A row holds H heads of `vectors` vectors of D elements each, of which the first `rotated` turn: vectors = 3, rotated = 2 is
 * the [head][q|k|v][D_h] layout of the sliced attention core, vectors = 1 a plain row of heads.  The first
 * 2 * (pairs[0] + pairs[1] + pairs[2]) elements of a vector turn, in P = pairs[0] + ... pairs; the first pairs[0] of them follow
 * axis 0, the next pairs[1] axis 1, the rest axis 2:
 *   angle(i) = position[axis(i)] * base^(-e),   e = i / P (DSN_ROTARY_SHARED) or j / pairs[axis], j counted inside the axis
 *   (u, v) -> (u cos - v sin, u sin + v cos)
 * Angles are reduced modulo a full turn in 64-bit fixed point, so they stay exact for every 32-bit position.  `inverse` turns
 * back, which is also the gradient with respect to the input.  Heads >= heads[t] of a sample of path t are neither read nor written. */
typedef struct dsn_rotary_desc {
  int32_t dtype;        /* DSN_BF16 or DSN_F32                                           */
  int32_t N;            /* rows (tokens) per sample                                      */
  int32_t H, D;         /* full head count 1..4096, elements per vector 2..256           */
  int32_t vectors, rotated; /* 1..8 vectors per head, of which the first 1..vectors turn */
  int64_t ldx, ldy;     /* elements between rows, >= H * vectors * D                     */
  int32_t T;
  const int32_t* heads; /* host [T]: head count of each path, 1..H                       */
  int32_t order;        /* dsn_order of x and y                                          */
  int32_t n_axes;       /* 1..3                                                          */
  int32_t pairs[3];     /* pairs that follow each axis, >= 1 for the axes used; 2 * their sum <= D */
  int32_t ladder;       /* dsn_rotary_ladder                                             */
  int32_t pairing;      /* dsn_rotary_pairing                                            */
  double base;          /* > 1, finite                                                   */
  int32_t shared_positions; /* 1: positions [n_axes][N], the same for every sample; 0: [n_axes][B * N], in the order of x's rows */
  int32_t inverse;      /* 1: turn by the negative angle                                 */
} dsn_rotary_desc;

/* Cache of keys and values in 4 bits, for transformer blocks that run token by token or piece by piece (not in the paper).
 * A sample of the batch is a request that keeps its cache from call to call; it has to keep its path, or move to one with fewer
 * heads, for as long as it is cached (a head that an earlier token's path did not have holds nothing for that token).
 *
 * Rows of a call lie as everywhere, [B][R][ld]; request i has rows 0 .. placed[i] - 1 of its R, the rest is padding that is neither
 * read nor written.  A row of qkv holds H heads of group + 2 vectors of D_h elements, [head][q x group | k | v][D_h]: group = 1 is the
 * layout of the sliced attention core, larger groups share a head's keys and values among their queries (dsn_rotary_axes turns rows of
 * group <= 6 in a call, wider ones head by head, up to eight vectors a call).  A row of the output holds [head][group][D_h].  Heads >= heads[t] of a request of path t are neither read nor written.
 *
 * Pages: [n_pages][H][page / 16] blocks of 16 tokens.  A block holds the keys, then the values, each as
 *   codes [D_h / 64][16][32 bytes]   64 elements a token, element 2 j in the low half of byte j, 2 j + 1 in the high half
 *   pairs [D_h / 64][16]             scale and middle, bfloat16 each
 * which makes 18 D_h bytes a block (1152 for D_h = 64).  An element is middle + scale * (code - 8).
 * A group of 64 elements x with least and greatest value a, b is rounded as follows, every operation once in fp32:
 *   scale = bf16(b / 15 - a / 15), the quotients as products with the fp32 number nearest 1 / 15;  0 if that is below 2^-126
 *   middle = bf16(2 (a / 2 + 4 scale));  code = round((x - middle) * (1 / scale)) + 8, ties to even, held in 0 .. 15;  8 where scale = 0
 * (b - a and a + 8 scale could leave fp32's range.)  A token whose k or v holds a NaN or an infinity in a head is stored as NaN there:
 * middle NaN, scale 0 in all groups of k and v, and every query of the head that sees it comes out as NaN.
 *
 * Token number n of request i (0 is its first) lies in page table[i][n / page], at place n % page of it. */
typedef struct dsn_cache_desc {
  int32_t dtype;        /* DSN_BF16: qkv, out, values                                    */
  int32_t R;            /* rows per request in this call, 1..2^24                        */
  int32_t H, D_h;       /* full head count 1..4096 (heads of k and v); 64 or 128         */
  int32_t group;        /* query vectors per head, 1..64                                 */
  int32_t page;         /* tokens per page: a multiple of 16, 16..1024                   */
  int32_t n_pages;      /* pages that exist; n_pages * page < 2^31                       */
  int32_t max_pages;    /* columns of the table: the most pages that a request can hold; max_pages * page < 2^30 */
  int64_t ld_qkv;       /* elements between rows of qkv, >= H * (group + 2) * D_h, a multiple of 8 */
  int64_t ld_out;       /* of out, >= H * group * D_h, a multiple of 8                   */
  int64_t ld_values;    /* of values, >= H * 2 * D_h, a multiple of 8                    */
  int32_t T;
  const int32_t* heads; /* host [T]: head count of each path, 1..H                       */
  int32_t order;        /* dsn_order of the rows of qkv, out and values; what dsn_cache holds is always by request */
  float scale;          /* of the scores, finite; 0: 1 / sqrt(D_h)                       */
  int32_t window;       /* a query sees the last `window` tokens up to and with its own; 0: all of them */
} dsn_cache_desc;

/* Where a cache lies; all of it device memory of the caller. */
typedef struct dsn_cache {
  uint8_t* pages;       /* dsn_cache_bytes(), 16-byte aligned                            */
  int32_t* table;       /* [B][max_pages]; entries behind the pages that a request holds mean nothing */
  int32_t* lengths;     /* [B] tokens of each request                                    */
  int32_t* placed;      /* [B] rows of each request in this call                         */
  int32_t* slots;       /* [B][R] where each row's token goes: page * tokens per page + place, -1: nowhere */
  int32_t* pool;        /* [n_pages] ring of the pages that no request holds             */
  int32_t* pool_state;  /* [2] place of the first of them in the ring, how many there are */
} dsn_cache;

/* One dynamic block: optional gate, routing, then up to DSN_MAX_CHAIN layers that all inherit
 * the block's routing (Sec. 5, "inherit the control signal").  Layer j reads layer j-1's output;
 * layer 0 reads x in input order, the last layer writes y in input order; intermediate
 * activations live in the workspace in grouped order. */
typedef struct dsn_layer_desc {
  const dsn_gate_desc* gate;        /* NULL: gate bypassed, idx_in supplies the path of every sample */
  int32_t B;
  int32_t T;
  int32_t n_layers;                 /* 1..DSN_MAX_CHAIN                                  */
  int32_t kind[DSN_MAX_CHAIN];      /* dsn_layer_kind                                    */
  const void* layer[DSN_MAX_CHAIN]; /* dsn_linear_desc*, dsn_conv_desc*, dsn_depthwise_desc* (not as the last element) or
                                       (between two layers) dsn_attention_desc*; order and leading-dimension fields of
                                       chained elements are ignored.  A depthwise element followed by a 1x1 layer whose
                                       k_in equals the depthwise widths (the DS-MBNet separable block, Sec. 3.3) can run
                                       as ONE kernel in which the depthwise result feeds the tensor core from shared
                                       memory and never reaches global memory (DSN_DWPW=fused; bf16, widths and row
                                       pitches multiples of 8); by default the two run one after the other through the
                                       workspace, which is the faster form on this GPU */
} dsn_layer_desc;

/* ---- context ------------------------------------------------------------------------- */
/* Creates a context on CUDA device `device` (allocates a few hundred bytes of device memory
 * for the status word; the only allocation the library ever makes).
 * Environment switches, read here, that select between kernels computing the same results (for
 * comparisons and as fallbacks): DSN_GEMM_MODE=1cta (one CTA per tile instead of CTA pairs),
 * DSN_CHAIN=0 (dsn_layer_forward: one launch per layer even for small batches), DSN_CONV3X3=taps
 * (3x3 layers: one activation load per tap instead of one tile with its halo), DSN_HALO_SCHED=strided
 * (staged 3x3 kernel: tiles dealt out round-robin instead of one time-balanced range per CTA pair), DSN_ATTENTION=items (the
 * attention core with one (sample, head, query half) per CTA pass instead of the warp-specialised form),
 * DSN_DWPW=fused (depthwise + following 1x1 layer as one kernel), DSN_CHAIN_FUSE=1 (chained launch: the last 1x1 layer
 * takes the output of the layer before from tensor memory instead of global memory), DSN_PDL=0 (no programmatic
 * dependent launch).
 * Every later call must be made with `device` as the calling thread's current CUDA device (else
 * DSN_ERR_INVALID_ARG): launches and kernel attributes act on the current device. */
int dsn_create(dsn_ctx** ctx, int device);
int dsn_destroy(dsn_ctx* ctx);
const char* dsn_strerror(int code);
/* Waits for `stream`, returns the first device-detected condition since the last call
 * (code = DSN_OK if none; detail = a count or position) and clears it. */
int dsn_get_status(dsn_ctx* ctx, void* stream, int32_t* code, int32_t* detail);

/* Limit of the bounded waits inside the kernels (every wait on a barrier or counter gives up after this
 * long, records DSN_ERR_TIMEOUT with a position code and lets the kernel return; the context stays usable).
 * microseconds = 0 restores the default of 2 s.  Synchronises `stream`.  (Failure detection; the paper has
 * no counterpart.) */
int dsn_set_wait_limit(dsn_ctx* ctx, uint32_t microseconds, void* stream);
/* Self-test of that mechanism: launches one small kernel that waits, with the library's own wait routine,
 * on a barrier nothing arrives at.  It returns after the wait limit; dsn_get_status() then reports
 * DSN_ERR_TIMEOUT (detail 9001).  Nothing faults and later calls run normally. */
int dsn_selftest_bounded_wait(dsn_ctx* ctx, void* stream);

/* The context keeps the TMA tensor maps it has encoded (keyed by base pointer, extents, strides and box; 512 slots,
 * host memory), so that repeated calls on the same buffers and slices skip the encoding (about a microsecond per
 * map, up to three maps per distinct slice and layer).  A map describes addresses and geometry only, so a hit stays
 * valid for as long as the caller's buffer does.  DSN_MAP_CACHE=0 at dsn_create turns the cache off.
 * Returns the hit and miss counts since the context was created. */
int dsn_map_cache_stats(dsn_ctx* ctx, uint64_t* hits, uint64_t* misses);

/* What a context has launched since it was created (host-side counters; kernels of this library only).  With
 * DSN_LOG=1 in the environment at dsn_create, every sliced-layer and dsn_layer_forward call also writes one line to
 * stderr. */
typedef struct dsn_stats {
  uint64_t calls;                 /* sliced-layer and dsn_layer_forward calls                              */
  uint64_t launches;              /* kernels launched, all families                                        */
  uint64_t launches_gemm_pair;    /* grouped GEMM on CTA pairs                                             */
  uint64_t launches_gemm_halo;    /* 3x3 layers, halo form                                                 */
  uint64_t launches_gemm_chain;   /* a block's layers as one launch                                        */
  uint64_t launches_gemm_one_cta; /* grouped GEMM, one CTA per tile                                        */
  uint64_t launches_linear_f32;
  uint64_t launches_attention;
  uint64_t launches_depthwise;
  uint64_t launches_dwpw;         /* depthwise + pointwise as one kernel                                   */
  uint64_t launches_gate;         /* pooling, hidden layer, scores (3 per gate), attention head            */
  uint64_t launches_route;
  uint64_t launches_copy;         /* gather / scatter, zero fill, channel scaling, Re-SBN folding          */
  uint64_t map_hits, map_misses;  /* tensor-map cache                                                      */
  uint64_t launches_gemm_chain_tmem; /* of launches_gemm_chain: last layer fed from tensor memory          */
  uint64_t launches_norm;         /* residual + norm + 8-bit codes                                         */
  uint64_t launches_gemm_i8;      /* 8-bit linear layers on the tensor cores, CTA pairs                    */
  uint64_t launches_rows_i8;      /* 8-bit linear layers of a few rows                                     */
  uint64_t launches_rotary;
  uint64_t launches_cache_plan;   /* 4-bit cache: pages and slots                                          */
  uint64_t launches_cache_write;  /* 4-bit cache: keys and values rounded into their pages                 */
  uint64_t launches_cache_attention; /* 4-bit cache: attention over the pages, with the joining of its parts */
} dsn_stats;
int dsn_get_stats(dsn_ctx* ctx, dsn_stats* out);

/* Ratio list -> channel counts (host only).  granule g = 0 picks g = min(8, C/32);
 * k = g*floor(r*C/g + 1/2) clamped to [g, C].  The paper lists channel counts, not a rounding
 * rule; this rule reproduces its DS-MBNet list 224..640 step 32 from ratios 0.35..1.0. */
int dsn_widths_from_ratios(int32_t C, const double* ratios, int32_t T, int32_t granule,
                           int32_t* widths_out /* host [T] */);

/* Multiply-adds the sliced layer executes for a routing histogram (Sec. 4.3, MAdds on the fly):
 * sum_t counts[t] * R * k_in[t] * k_out[t] * K*K.  Host arrays. */
int64_t dsn_executed_macs(const int32_t* counts, int32_t T, int32_t R, const int32_t* k_in,
                          const int32_t* k_out, int32_t K);

/* ---- gate (Sec. 3.5) ------------------------------------------------------------------ */
size_t dsn_gate_workspace_bytes(const dsn_gate_desc* g);
/* x: device [B][R][ldx].  idx_out: device [B].  logits_out: device [B][T] fp32 or NULL.
 * workspace: device, 16-byte aligned, >= dsn_gate_workspace_bytes (partial sums of the pooling). */
int dsn_gate(dsn_ctx* ctx, const dsn_gate_desc* g, const void* x, int32_t* idx_out,
             float* logits_out, void* workspace, size_t ws_bytes, void* stream);

/* The same gate for callers that cannot allocate device memory (the paper has no counterpart;
 * this is a deployment convenience).  Typical such callers: a serving loop that must never enter
 * the CUDA allocator once it is running, a plug-in that is handed only its input and output
 * buffers, code running while the process's memory pool is fully handed out.  The pooling scratch
 * lives in a fixed 4 MiB array inside the library image (every GPU that loads the library keeps it
 * until the process exits), so the call takes no workspace and performs no allocation of any kind.
 *   - Limit: B * (splits * c_valid + C_mlp) <= 1,048,576 floats, where splits (1..64) is the
 *     row-band count the gate picks for this GPU; larger problems return DSN_ERR_WORKSPACE and
 *     launch nothing.  The ResNet-50 and ViT workloads fit (128 samples x (4 splits x 1024 + 128) on a
 *     148-SM GPU, 1024 x (1 x 768 + 128)).
 *   - The context's device must be the current device (else DSN_ERR_INVALID_ARG).
 *   - The first call on a device looks up the array's device address (a synchronous runtime
 *     query); make that first call before starting any stream capture.
 *   - All calls on one GPU share the array and it keeps the previous call's contents.  Nothing has
 *     to start at zero (each call overwrites every value it later reads), but two calls that
 *     overlap on the GPU (different streams, or different contexts of one process) race on it:
 *     keep calls to this entry point ordered on one stream per GPU.
 * Arguments and results are those of dsn_gate. */
int dsn_gate_static(dsn_ctx* ctx, const dsn_gate_desc* g, const void* x, int32_t* idx_out,
                    float* logits_out, void* stream);

/* Double-headed gate (Sec. 3.5): the routing head of dsn_gate plus the channel-attention head that
 * shares W1: scale[i][c] = 1 + tanh(b3[c] + sum_j W3[c][j] * ReLU(W1 X_E + b1)[j]), c < c_valid.
 * W3: device [C_full][C_mlp] fp32, b3: device [C_full] or NULL.  scale_out: device [B][c_valid] fp32.
 * idx_out / logits_out as in dsn_gate (both heads always run).  Workspace as for dsn_gate. */
int dsn_gate_attention(dsn_ctx* ctx, const dsn_gate_desc* g, const float* W3, const float* b3, const void* x,
                       int32_t* idx_out, float* logits_out, float* scale_out, void* workspace, size_t ws_bytes,
                       void* stream);

/* Applies the attention head: y[p or i][r][c] = x[i][r][c] * scale[i][c] for c < c_valid (bf16 or fp32
 * activations, fp32 scale).  With r != NULL and to_grouped = 1 the result is written in grouped
 * order (position p holds sample perm[p]), i.e. the scaling is fused with the gather; otherwise y is
 * in input order.  x and y may be the same buffer when the order does not change. */
int dsn_scale_channels(dsn_ctx* ctx, const dsn_routing* r, int32_t to_grouped, int32_t dtype, int32_t B,
                       int32_t R, int32_t c_valid, const void* x, int64_t ldx, const float* scale, void* y,
                       int64_t ldy, void* stream);

/* Split batch norm with re-calibration (Sec. 3.3): gamma[:c] * (X - mu_t) / sigma_t + beta[:c] with
 * per-route statistics.  At inference it is the per-path per-channel affine a_t = gamma / sigma_t,
 * b_t = beta - gamma * mu_t / sigma_t, which the sliced layers apply in their epilogue
 * (bn_scale / bn_shift).  gamma, beta: device [C]; mu, sigma: device [T][C]; outputs device [T][C]. */
int dsn_resbn_fold(dsn_ctx* ctx, int32_t T, int32_t C, const float* gamma, const float* beta, const float* mu,
                   const float* sigma, float* scale_out, float* shift_out, void* stream);

/* ---- routing (stable grouping by path index; one-hot routing of Sec. 3.1) -------------- */
/* idx: device [B], values in [0, T).  Fills out->counts/offsets/perm/inv_perm (device arrays the
 * caller allocated, G = T, B as given); integer-exact and deterministic.  A value outside
 * [0, T) sets DSN_ERR_BAD_INDEX in the status word; that sample joins no group and the unused
 * tail of perm is set to -1. */
int dsn_route(dsn_ctx* ctx, const int32_t* idx, int32_t B, int32_t T, dsn_routing* out, void* stream);

/* ---- gather / scatter between input order and grouped order ---------------------------- */
/* Copies, for every sample, R rows of the leading k[t] columns (t = its path; k host [T]).
 * to_grouped = 1: dst position p <- src sample perm[p]; 0: dst sample perm[p] <- src position p. */
int dsn_permute_rows(dsn_ctx* ctx, const dsn_routing* r, int32_t dtype, int32_t R, int32_t T,
                     const int32_t* k /* host [T] */, const void* src, int64_t ld_src, void* dst,
                     int64_t ld_dst, int32_t to_grouped, void* stream);

/* ---- sliced layers --------------------------------------------------------------------- */
size_t dsn_linear_workspace_bytes(const dsn_linear_desc* d, int32_t B);
size_t dsn_conv_workspace_bytes(const dsn_conv_desc* d, int32_t B);
/* x, y: device, 16-byte aligned, laid out as d->in_order / d->out_order say.  r: routing of the
 * batch (r->B samples).  workspace may be NULL when the size query returns 0. */
int dsn_sliced_linear(dsn_ctx* ctx, const dsn_linear_desc* d, const dsn_routing* r, const void* x,
                      void* y, void* workspace, size_t ws_bytes, void* stream);
int dsn_sliced_conv(dsn_ctx* ctx, const dsn_conv_desc* d, const dsn_routing* r, const void* x,
                    void* y, void* workspace, size_t ws_bytes, void* stream);

int dsn_sliced_depthwise(dsn_ctx* ctx, const dsn_depthwise_desc* d, const dsn_routing* r, const void* x, void* y,
                         void* stream);

/* qkv, out: device bf16, 16-byte aligned.  fp32 scores and softmax, bf16 probabilities for the
 * second contraction, bf16 output. */
int dsn_sliced_attention(dsn_ctx* ctx, const dsn_attention_desc* d, const dsn_routing* r, const void* qkv,
                         void* out, void* stream);

/* ---- transformer blocks in 8 bits -------------------------------------------------------- */
/* x, residual (or NULL), sum (or NULL: h in x's type is not wanted): rows in d->in_order.  q with q_scale (device float, one per
 * row), both or neither; y (or NULL) in x's type: the values that the codes stand for, q * s, where q is given, else n itself.
 * At least one of sum, q, y is given.  sum may be x or residual itself (same leading dimension); q and y overlap nothing else.
 * Columns >= k[t] of every output keep what they held.  All row pointers 16-byte aligned. */
int dsn_rmsnorm_quant(dsn_ctx* ctx, const dsn_norm_desc* d, const dsn_routing* r, const void* x, const void* residual,
                      void* sum, int8_t* q, float* q_scale, void* y, void* stream);

/* x: device int8, 16-byte aligned, rows as d->in_order says; x_scale: device float [B * R] in the same order of rows.
 * workspace: device, 16-byte aligned, of dsn_linear_i8_workspace_bytes (0 for most calls): room for the rows of many short samples that
 * arrive in input order, gathered.  With less, or NULL, the rows are tiled where they lie: the same results, more slowly. */
size_t dsn_linear_i8_workspace_bytes(const dsn_linear_i8_desc* d, int32_t B);
int dsn_sliced_linear_i8(dsn_ctx* ctx, const dsn_linear_i8_desc* d, const dsn_routing* r, const int8_t* x,
                         const float* x_scale, void* y, void* workspace, size_t ws_bytes, void* stream);

/* positions: device int32, any values.  y may be x itself (same leading dimension).  The heads of a sample's path are written whole, the
 * vectors and elements that do not turn as they were. */
int dsn_rotary_axes(dsn_ctx* ctx, const dsn_rotary_desc* d, const dsn_routing* r, const int32_t* positions, const void* x,
                    void* y, void* stream);

/* ---- attention over a 4-bit cache -------------------------------------------------------- */
/* Bytes of dsn_cache.pages (0: the descriptor is not valid). */
size_t dsn_cache_bytes(const dsn_cache_desc* d);
/* An empty cache: lengths 0, every page in the pool.  Uses lengths, pool, pool_state. */
int dsn_cache_reset(dsn_ctx* ctx, const dsn_cache_desc* d, const dsn_cache* c, int32_t B, void* stream);

/* Finds room for the new tokens of every request: new_tokens device [B], 0 .. R to append, -1 to end the request (its pages go back
 * to the pool, from which the next call can take them).  Requests are served in order.  One whose row of the table has no room for its tokens is not
 * served and asks the pool for nothing.  Any other that needs pages gets them if its need and that of all such requests before it, served or not, fits into the
 * pool.  Of a request that is not served nothing is placed, and DSN_ERR_CACHE_FULL is recorded with its number.  A length or new_tokens value out of range counts as a request that changes nothing and records
 * DSN_ERR_BAD_INDEX.  Pages leave the ring from its front and return at its end, in the order of requests: the same call gives the same pages.
 * Reads lengths, table, pool, pool_state; writes the new entries of table, placed (rows placed, 0 for a request that ended), slots, the
 * returned entries of pool, and lengths and pool_state after the call to lengths_out [B] and pool_state_out [2] (NULL, or c's own: in place).
 * Only pages that were taken here may be given back here: none is held by two requests. */
int dsn_cache_plan(dsn_ctx* ctx, const dsn_cache_desc* d, const dsn_cache* c, int32_t B, const int32_t* new_tokens, int32_t* lengths_out,
                   int32_t* pool_state_out, void* stream);

/* Rounds k and v of the rows to 4 bits and writes them to their slots (rows with slot -1 go nowhere; other slots outside the cache record
 * DSN_ERR_BAD_INDEX and go nowhere either; no two rows may have the same slot).  values (or NULL): the values that the codes stand for, rounded
 * to bfloat16, rows [head][k | v][D_h]; they overlap nothing else.  Uses pages and slots. */
int dsn_cache_write_q4(dsn_ctx* ctx, const dsn_cache_desc* d, const dsn_cache* c, const dsn_routing* r, const void* qkv, void* values,
                       void* stream);

/* out = softmax(scale * q k^T) v over the cached tokens that a row's query sees: row j of request i is token n = lengths[i] - placed[i] + j of
 * it (its keys are in the cache already) and sees tokens max(0, n - window + 1) .. n.  Softmax and sums in fp32; the operands of both products are rounded to
 * 11 bits (fp16 behind powers of two: q and k, a probability or its product with v's scale, v).  With R * group <= 32 magnitudes of v from 1e-15 to 1e34 in a
 * cache keep them, whatever other groups of 64 elements, other tokens or tokens that a row does not see hold (above 1e30 weights below 2^-20 of a row's greatest can be lost).  With R * group > 32, 64
 * tokens in a row share a power of k and one of v over all their elements, seen by a row or not (up to 256 query vectors of a head go together: what lies in front
 * of the window of them all does not count).  With w and a the greatest weight of a row and the greatest magnitude of v among 64 tokens in a row, an
 * output is off by up to 2^-20 of the mean of a under the weights and 2^-30 of the largest w a for each token that the row can see, beside those 11 bits; a score by
 * 2^-20 of the one that the greatest magnitude of k among the 64 would give.
 * A row that sees nothing (n < 0) comes out as zeros, any other whose query holds a NaN or an infinity as NaN; a score, times log2(e), has to lie
 * within fp32's range.  Uses pages, table, lengths, and placed (NULL: R rows of every request).  A length or
 * placed value out of range is held at the nearest end of it, tokens of a page outside the cache are left out, and both record DSN_ERR_BAD_INDEX.
 * out overlaps nothing else.  workspace: device, 16-byte aligned, of dsn_cache_attention_q4_workspace_bytes; nothing in it has to start at
 * zero.  It must not be used by two calls at once. */
size_t dsn_cache_attention_q4_workspace_bytes(const dsn_cache_desc* d, int32_t B);
int dsn_cache_attention_q4(dsn_ctx* ctx, const dsn_cache_desc* d, const dsn_cache* c, const dsn_routing* r, const void* qkv, void* out,
                           void* workspace, size_t ws_bytes, void* stream);

/* ---- whole dynamic block (Eq. (dyn_net)) ------------------------------------------------ */
size_t dsn_layer_workspace_bytes(const dsn_layer_desc* L);
/* Gate (or the given indices) -> routing -> the block's layers, all layers under the one decision
 * (Sec. 5).  Batches of at most two samples per SM pair whose samples have 150..256 rows (14x14
 * images, 197 tokens) run their 2-3 sliced layers as ONE launch in which every SM pair walks whole
 * samples through the layers (skip features included); otherwise (and whenever the block holds the attention core
 * or a depthwise element) one launch per layer.  The two forms agree to within one bfloat16 rounding step of an
 * output on a few percent of the elements (the 3x3 layer sums its taps in a different order), not bit for bit.
 * x, y in input order.  idx_in: device [B], required when L->gate is NULL, ignored otherwise.
 * r_out (optional): receives pointers into the workspace holding the block's routing arrays
 * (valid until the workspace is reused).  idx_out (optional): device [B], the gate's choice. */
int dsn_layer_forward(dsn_ctx* ctx, const dsn_layer_desc* L, const void* x, const int32_t* idx_in,
                      void* y, dsn_routing* r_out, int32_t* idx_out, void* workspace, size_t ws_bytes,
                      void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DSN_H */
