/*
 * gl.h - C ABI of the access-pattern evaluator for B200 (sm_100a).
 *
 * The calls follow the operators of "Pure Tensor Program Rewriting via Access
 * Patterns" (Glenside): the access-pattern transformers of Section 4.2 (first
 * table of Section 4) and the operators applied by `compute` (Section 4.3,
 * operator table).  An access pattern is a dense row-major tensor whose
 * dimensions are split into access dimensions S_A (iterated over) and compute
 * dimensions S_C (computed on); its tensor shape is S_A ++ S_C (Section 4.1).
 *
 * Conventions for every call
 *   - Return value: GL_OK or a GL_ERR_* code; gl_strerror() names it.
 *   - All arguments are validated, and every descriptor a call needs is prepared,
 *     before anything is enqueued: a call that returns any error other than a
 *     failed kernel launch has launched nothing and written nothing.  (A launch
 *     that the runtime itself refuses, GL_ERR_CUDA, may follow an earlier launch
 *     of the same call, which has then written the workspace but not `out`.)
 *   - gl_shape_* calls are host-only: they read shapes, never `data`.
 *   - Device calls enqueue kernels on `stream` (a cudaStream_t passed as
 *     void*, NULL = the default stream).  They never synchronise and never
 *     allocate.  `data` pointers are DEVICE pointers owned by the caller, who
 *     also owns outputs and workspaces.  `out->shape`, `out->ndim`,
 *     `out->access_ndim` and `out->dtype` must already equal what the matching
 *     gl_shape_* call returns, otherwise GL_ERR_SHAPE / GL_ERR_DTYPE.
 *   - Inputs are read-only and must not overlap outputs (gl_compute_relu, gl_compute_rotate and
 *     gl_compute_norm_rms may run in place; a gl_cache4 is what gl_cache4_append writes).  Data pointers must be 16-byte aligned (GL_ERR_ALIGN).
 *   - There is no CPU fallback: a combination the kernels do not cover
 *     returns GL_ERR_UNSUPPORTED.
 *   - Calls are re-entrant from several host threads.
 */
#ifndef GL_H_
#define GL_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define GL_API __attribute__((visibility("default")))
#else
#define GL_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

enum {
  GL_OK = 0,
  GL_ERR_NULL = 1,        /* a required pointer is NULL                              */
  GL_ERR_DTYPE = 2,       /* dtype not accepted by this call                         */
  GL_ERR_NDIM = 3,        /* ndim / access_ndim out of range                         */
  GL_ERR_SHAPE = 4,       /* shapes disagree (with each other or with gl_shape_*)    */
  GL_ERR_PERM = 5,        /* not a permutation of 0..ndim-1                          */
  GL_ERR_ALIGN = 6,       /* a data pointer is not 16-byte aligned                   */
  GL_ERR_UNSUPPORTED = 7, /* valid program, but no kernel covers it                  */
  GL_ERR_WORKSPACE = 8,   /* workspace missing or smaller than the _workspace() size */
  GL_ERR_CUDA = 9,        /* the CUDA runtime or driver reported an error            */
  GL_ERR_TIMEOUT = 10     /* a bounded wait inside a kernel gave up                  */
};

enum { GL_BF16 = 1, GL_F32 = 2 };
enum { GL_PAD_ZERO = 0, GL_PAD_NEG_INF = 1 };

#define GL_MAX_DIMS 8

/* Access pattern (Section 4.1): tensor of shape S_A ++ S_C, dense, row-major. */
typedef struct {
  void* data;          /* device pointer (ignored by gl_shape_*)                 */
  int32_t dtype;       /* GL_BF16 or GL_F32                                       */
  int32_t ndim;        /* |S_A| + |S_C|, 0..GL_MAX_DIMS                           */
  int32_t access_ndim; /* |S_A|: `(access T access_ndim)`                         */
  int32_t reserved_;
  int64_t shape[GL_MAX_DIMS];
} gl_ap;

/* Arguments of `windows` (transformer table): one window extent and one
 * stride per COMPUTE dimension of the input.  pad_lo / pad_hi describe a
 * `pad` of that compute dimension applied first (pad is not in the paper;
 * it is the constant border that ML convolutions and pools use): the padded
 * tensor is never written, out-of-range cells read as the fill value. */
typedef struct {
  int32_t n;        /* number of compute dims of the input = ndim - access_ndim */
  int32_t pad_kind; /* GL_PAD_ZERO or GL_PAD_NEG_INF                             */
  int64_t wshape[GL_MAX_DIMS];
  int64_t stride[GL_MAX_DIMS];
  int64_t pad_lo[GL_MAX_DIMS];
  int64_t pad_hi[GL_MAX_DIMS];
} gl_windows;

/* Flags of gl_cartesian_dot */
#define GL_EPILOGUE_RELU 0x2u       /* apply compute relu to every result before it is stored  */
#define GL_OUT_NCHW 0x4u             /* conv2d only: store transpose(squeeze(...)) of Fig. 2a, i.e.
                                        ((N, O, H', W'),()); see gl_shape_cartesian_dot_nchw      */
#define GL_OUT_BF16 0x8u             /* store the results rounded to bf16 (nearest even) instead of fp32: `out`
                                      * must then be GL_BF16.  Sums are still carried in fp32; the rounding is
                                      * the last step, after relu.  Lets the next layer read its operand as is
                                      * and halves the bytes written. */
#define GL_ROTATE_BACK 0x10u         /* gl_compute_rotate only: turn by the negative angles */
#define GL_DOT_GENERAL_KERNEL 0x100u /* skip the tensor-core path: run the general kernel, which
                                        takes any shape and sums each window in index order      */

/* ----------------------------------------------------------------------- */
/* Host-only shape inference.  Each fills out->ndim, access_ndim, shape and  */
/* dtype (copied from the input, GL_F32 for dot products) and leaves         */
/* out->data untouched.                                                      */
/* ----------------------------------------------------------------------- */

/* `access` (transformer table, row 1): move the split to position i. */
GL_API int gl_shape_access(const gl_ap* in, int32_t i, gl_ap* out);

/* `windows` (transformer table): ((a..),(b_0..b_n)) -> ((a.., b'_0..b'_n),(w_0..w_n)),
 * b'_i = ceil((b_i + pad_lo_i + pad_hi_i - (w_i - 1)) / s_i).  A window larger than
 * its padded dimension, or a pad not smaller than the window, is GL_ERR_SHAPE. */
GL_API int gl_shape_windows(const gl_ap* in, const gl_windows* w, gl_ap* out);

/* `flatten` (transformer table): ((prod a),(prod b)); a side without dims stays empty. */
GL_API int gl_shape_flatten(const gl_ap* in, gl_ap* out);

/* `transpose` (transformer table, Section 4.2): output dim j = input dim perm[j];
 * perm covers all ndim dims; the split position is kept. */
GL_API int gl_shape_transpose(const gl_ap* in, const int32_t* perm, gl_ap* out);

/* `pad` (not in the paper): dimension `dim` grows by lo + hi. */
GL_API int gl_shape_pad(const gl_ap* in, int32_t dim, int64_t lo, int64_t hi, gl_ap* out);

/* `slice` (transformer table): dimension `dim` keeps [lo, hi). */
GL_API int gl_shape_slice(const gl_ap* in, int32_t dim, int64_t lo, int64_t hi, gl_ap* out);

/* `concat` (used by the blocking rewrites of Section 5.4, Fig. 7): join a and b along `dim`; all
 * other extents, the split position and the dtype must agree. */
GL_API int gl_shape_concat(const gl_ap* a, const gl_ap* b, int32_t dim, gl_ap* out);

/* `pair` (transformer table): two patterns of one shape -> ((a..),(2, c..)). */
GL_API int gl_shape_pair(const gl_ap* a, const gl_ap* b, gl_ap* out);

/* `squeeze` (transformer table): drop dimension `dim`, which must have extent 1.  Metadata only:
 * the data of the result is the data of the input. */
GL_API int gl_shape_squeeze(const gl_ap* in, int32_t dim, gl_ap* out);

/* `reshape` (transformer table): new shape `shape[0..ndim)` split at `access_ndim`; the element
 * counts of the access side and of the compute side must both be kept.  Metadata only. */
GL_API int gl_shape_reshape(const gl_ap* in, const int64_t* shape, int32_t ndim, int32_t access_ndim, gl_ap* out);

/* compute reduceSum (operator table): ((access dims),()). */
GL_API int gl_shape_reduce_sum(const gl_ap* in, gl_ap* out);

/* compute dotProd (cartProd (windows? a0) a1)  (Section 4.2 cartProd, Section 4.3
 * dotProd, Fig. 2a/2b): with A = windows(a0) (or a0 itself when w is NULL) of shape
 * ((m..),(k..)) and a1 of shape ((o..),(k..)), the result is ((m.., o..),()), GL_F32. */
GL_API int gl_shape_cartesian_dot(const gl_ap* a0, const gl_windows* w_or_null, const gl_ap* a1, gl_ap* out);

/* The whole conv2d of Fig. 2a: transpose (squeeze (compute dotProd (cartProd (windows a0) a1)) 1)
 * (0 3 1 2).  a0 must be ((n..),(C,H,W)) with window (C,Kh,Kw), or ((n..),(H,W,C)) with window
 * (Kh,Kw,C); the result is ((n.., o.., H', W'),()), GL_F32: the window-position dims move behind
 * the filter dims and the size-1 channel position is squeezed away.  This is the shape
 * gl_cartesian_dot expects for `out` when GL_OUT_NCHW is set. */
GL_API int gl_shape_cartesian_dot_nchw(const gl_ap* a0, const gl_windows* w, const gl_ap* a1, gl_ap* out);

/* compute reduceMax (windows? in) (operator table; Fig. 2c): ((access dims of A),()). */
GL_API int gl_shape_reduce_max(const gl_ap* in, const gl_windows* w_or_null, gl_ap* out);

/* ----------------------------------------------------------------------- */
/* Device operations                                                         */
/* ----------------------------------------------------------------------- */

/* Materialised `windows` (transformer table; Section 5.3 calls the result, once
 * flattened, the im2col matrix): out[a.., p.., q..] = in[a.., p_i*s_i + q_i - pad_lo_i],
 * the fill value where that index is outside the input.  GL_F32 or GL_BF16. */
GL_API int gl_access_windows(const gl_ap* in, const gl_windows* w, gl_ap* out, void* stream);

/* `flatten` is metadata on dense data: fills out's shape and sets out->data = in->data. */
GL_API int gl_access_flatten(const gl_ap* in, gl_ap* out);

/* `transpose` with data movement: out[i_0..] = in[j_0..] with j_{perm[d]} = i_d.
 * GL_F32 or GL_BF16, any rank up to GL_MAX_DIMS. */
GL_API int gl_access_transpose(const gl_ap* in, const int32_t* perm, gl_ap* out, void* stream);

/* Materialised `pad` of one dimension with 0 or -inf (not in the paper). */
GL_API int gl_access_pad(const gl_ap* in, int32_t dim, int64_t lo, int64_t hi, int32_t pad_kind,
                  gl_ap* out, void* stream);

/* `slice`, `concat`, `pair` with data movement (transformer table; Fig. 7).  GL_F32 or GL_BF16. */
GL_API int gl_access_slice(const gl_ap* in, int32_t dim, int64_t lo, int64_t hi, gl_ap* out, void* stream);
GL_API int gl_access_concat(const gl_ap* a, const gl_ap* b, int32_t dim, gl_ap* out, void* stream);
GL_API int gl_access_pair(const gl_ap* a, const gl_ap* b, gl_ap* out, void* stream);

/* compute reduceSum (operator table): the sum of every item, GL_F32, added in a fixed order (a
 * strided partial sum per lane of one warp, then a butterfly), so results repeat bit for bit. */
GL_API int gl_compute_reduce_sum(const gl_ap* in, gl_ap* out, void* stream);

/* out = compute dotProd (cartProd (windows? a0) a1), optionally followed by compute
 * relu (Fig. 2a for conv2d with w given, Fig. 2b / Fig. 6 for matrix products with
 * w NULL).  a0 and a1 are GL_BF16, products and sums are carried in fp32, out is
 * GL_F32 (GL_BF16 with GL_OUT_BF16) with the access dims of A followed by those of a1,
 * i.e. row-major [M, O].
 * Two item layouts take the tensor-core path:
 *   - w NULL, a0 ((M),(K)), a1 ((O),(K)) with K a multiple of 8;
 *   - a0 ((N),(C,H,W)) with window (C,Kh,Kw), stride (1,Sh,Sw), or a0 ((N),(H,W,C))
 *     with window (Kh,Kw,C), stride (Sh,Sw,1); a1 ((O),(same item shape as the window)).
 * Everything else runs on a slower general kernel.  The sum over the window is
 * taken in an unspecified order.  `workspace` must hold at least
 * gl_cartesian_dot_workspace() bytes (it may be NULL when that is 0) and must be
 * 1024-byte aligned; its contents are scratch.  Few-channel convolutions (at most
 * 8 / Sw channels, the RGB stem), channels-last items with a channel count that is
 * a multiple of 8, and 1x1 unpadded windows over (C,H,W) items whose rows the TMA
 * unit can address (C a multiple of 8 and at least 64; unit strides with H*W a
 * multiple of 8, or W a multiple of 8 up to 64 with a column stride of 1 or 2) need
 * none: the kernels read both operands where they are.  Encoded tensor maps are kept per argument list, so a repeated call on the
 * same buffers skips the driver's encoding.  The kernels are launched with programmatic
 * stream serialisation: their set-up may run while the preceding kernel of the stream
 * drains, and they wait for its completion before their first access to memory. */
GL_API int gl_cartesian_dot(const gl_ap* a0, const gl_windows* w_or_null, const gl_ap* a1, gl_ap* out,
                     uint32_t flags, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of scratch gl_cartesian_dot needs for these arguments (0 on invalid ones). */
GL_API size_t gl_cartesian_dot_workspace(const gl_ap* a0, const gl_windows* w_or_null, const gl_ap* a1,
                                  uint32_t flags);

/* gl_cartesian_dot for callers that cannot allocate device memory.  (The paper has no
 * counterpart: this is a property of the host program, not of the method.)
 *
 * gl_cartesian_dot wants a caller-owned workspace whenever it has to make channels-last
 * copies of its operands.  Code that runs where no allocator may be called - inside
 * another framework's operator, in a plug-in that is handed nothing but its input and
 * output buffers, in a process whose device memory is entirely owned by a pool - cannot
 * provide one.  This variant takes no workspace: it uses a fixed scratch array of
 * GL_STATIC_SCRATCH_BYTES (32 MiB) that is part of the library image, so every GPU that
 * loads the library holds that much memory until the process exits.  It calls no
 * cudaMalloc, cudaFree or other allocating routine.
 *
 *   - Same arguments, results and error codes as gl_cartesian_dot without the workspace
 *     pair.  If the layout copies of these arguments exceed GL_STATIC_SCRATCH_BYTES
 *     the call returns GL_ERR_WORKSPACE and launches nothing (for scale: the (C,H,W)
 *     activations of a 32x64x56x56 convolution need 12.3 MiB).  A contraction that
 *     gl_cartesian_dot would split, and whose partial planes do not fit beside the
 *     copies, runs unsplit instead.
 *   - The first call on each device looks up the array's device address (that device
 *     must be current); make that first call before any stream capture begins.
 *   - All calls share the one array and it keeps whatever the last call left in it.
 *     Nothing in it has to start at zero: each call overwrites every byte it later
 *     reads.  Two calls whose kernels can overlap on the GPU (different streams, or
 *     different host threads without ordering) race on the array; order them. */
#define GL_STATIC_SCRATCH_BYTES (32u << 20)
GL_API int gl_cartesian_dot_static(const gl_ap* a0, const gl_windows* w_or_null, const gl_ap* a1, gl_ap* out,
                                   uint32_t flags, void* stream);

/* compute reduceMax (windows? in) (operator table, Fig. 2c max pooling): the largest
 * value of every item; with w given the windows are formed on the fly and never
 * stored.  GL_F32 in any form.  GL_BF16 (results of GL_OUT_BF16 convolutions) in two forms:
 * 2D windows over ((..),(H,W)) items, and channels-last items ((N),(H,W,C)) with window
 * (Kh,Kw,1), stride (Sh,Sw,1) and C a multiple of 8; other bf16 forms return
 * GL_ERR_UNSUPPORTED.  The largest of a set of values is one of them, so nothing is rounded.
 * Inputs must be NaN-free. */
GL_API int gl_compute_reduce_max(const gl_ap* in, const gl_windows* w_or_null, gl_ap* out, void* stream);

/* compute relu (not in the paper's operator table): out = in > 0 ? in : +0, item
 * shape kept.  GL_F32.  in->data == out->data is allowed. */
GL_API int gl_compute_relu(const gl_ap* in, gl_ap* out, void* stream);

/* ----------------------------------------------------------------------- */
/* Operands held in 4 bits (MX4; not in the paper)                           */
/* ----------------------------------------------------------------------- */

/* A pattern of shape S_A ++ S_C whose items (the prod(S_C) = K values of one access index) are cut into blocks of 32
 * consecutive values.  A block is 32 E2M1 codes (sign and 0, 0.5, 1, 1.5, 2, 3, 4 or 6) and one E8M0 scale: value =
 * code * 2^(scale - 127), scale 255 = NaN for the whole block.
 *   data:  gl_mx4_data_bytes() bytes; one row per item of ceil(K/32)*16 bytes, two codes a byte, the even index in the
 *          low half; codes past K are zero.
 *   scale: gl_mx4_scale_bytes() bytes; tiles of 128 rows x 4 blocks, 512 bytes each, row tiles outermost; row r and
 *          block b of a tile at byte (r % 32) * 16 + (r / 32) * 4 + b.
 * Both device pointers are 16-byte aligned.  Size limits (else GL_ERR_UNSUPPORTED): fewer than 2^31 - 256 rows, K <= 2^30, and
 * for what a call rounds or widens rows * ceil(K/128)*16 < 2^31; nothing else is assumed of K or of the rows. */
typedef struct {
  void* data;
  void* scale;
  int32_t ndim;
  int32_t access_ndim;
  int64_t shape[GL_MAX_DIMS];
} gl_mx4;

/* Bytes of the two arrays (0 on an invalid shape). */
GL_API size_t gl_mx4_data_bytes(const gl_mx4* a);
GL_API size_t gl_mx4_scale_bytes(const gl_mx4* a);

/* Rounds `in` (GL_F32 or GL_BF16) to `out`, which carries the same shape: scale 2^(floor(log2 max|v|) - 2) of the
 * block, not below 2^-127; values divided by it are rounded to the nearest code, ties to the even mantissa, larger
 * values than 6 to 6.  A block that holds an Inf or a NaN becomes NaN as a whole. */
GL_API int gl_mx4_quantize(const gl_ap* in, gl_mx4* out, void* stream);

/* The values of `in` as `out` (GL_F32 or GL_BF16; both hold every one of them exactly). */
GL_API int gl_mx4_dequantize(const gl_mx4* in, gl_ap* out, void* stream);

/* compute dotProd (cartProd a0 a1) of two MX4 patterns of the same compute shape: ((m..),(k..)), ((o..),(k..)) ->
 * ((m.., o..),()), sums in fp32, on the tensor cores' block-scaled 4-bit products.  flags: GL_EPILOGUE_RELU (NaN stays
 * NaN), GL_OUT_BF16; `out` is GL_F32 or, with GL_OUT_BF16, GL_BF16. */
GL_API int gl_cartesian_dot_mx4(const gl_mx4* a0, const gl_mx4* a1, gl_ap* out, uint32_t flags, void* stream);

/* The same with the left operand given as GL_F32 or GL_BF16 and rounded to MX4 by the call (a dense layer: activations
 * a0, weights a1 laid out once by gl_mx4_quantize).  The result does not depend on how many rows a0 has beyond the
 * order of the sums.  `workspace`: gl_dense_mx4_workspace() bytes, 1024-byte aligned, scratch: calls that can overlap on
 * the GPU need one each. */
GL_API int gl_dense_mx4(const gl_ap* a0, const gl_mx4* a1, gl_ap* out, uint32_t flags, void* workspace,
                        size_t workspace_bytes, void* stream);
GL_API size_t gl_dense_mx4_workspace(const gl_ap* a0, const gl_mx4* a1);

/* Pages of keys and values held in MX4, blocks along the head dimension.  A page holds `page_tokens` consecutive tokens
 * of all kv heads: [kv_heads][page_tokens / 16] groups of 16 tokens, 17 * head_dim bytes each; the order inside a group
 * is the library's own (gl_cache4_read gives values back).  head_dim 64, 128 or 256; page_tokens a multiple of 16. */
typedef struct {
  void* data;           /* gl_cache4_bytes() bytes, 16-byte aligned                                     */
  int64_t pages;
  int32_t kv_heads;
  int32_t head_dim;
  int32_t page_tokens;
  int32_t reserved_;
} gl_cache4;

/* Where the tokens of a batch lie.  Token t of sequence b is token t % page_tokens of page
 * page_table[b * table_width + t / page_tokens].  lengths[b] counts the tokens of sequence b, those of this call
 * included.  Both arrays are in DEVICE memory and cannot be checked by the host: lengths are taken as
 * 0..table_width * page_tokens, a token on a page that does not exist is not stored, reads as zeros and is not seen.
 * The calls read them while they run: like every input they must not change until the call has ended on the GPU. */
typedef struct {
  const int32_t* page_table;
  const int32_t* lengths;
  int32_t batch;
  int32_t table_width;
} gl_pages;

GL_API size_t gl_cache4_bytes(const gl_cache4* cache);

/* Rounds k and v, ((B, T, kv_heads),(head_dim)) GL_BF16, into the cache: token i of sequence b becomes its token
 * lengths[b] - T + i; those before token 0 (left padding of a ragged batch) are skipped.  token_pitch: elements between
 * successive tokens of k and of v, those of a sequence's end and the next one's start too, a multiple of 8 (0: dense), so
 * that both may be parts of one projection.  Pages that two sequences share may be read but not appended to. */
GL_API int gl_cache4_append(const gl_cache4* cache, const gl_ap* k, const gl_ap* v, int64_t token_pitch, const gl_pages* at,
                            void* stream);

/* The values of the last T tokens of every sequence, k and v ((B, T, kv_heads),(head_dim)) dense GL_BF16; zeros where
 * there is no such token. */
GL_API int gl_cache4_read(const gl_cache4* cache, const gl_pages* at, gl_ap* k, gl_ap* v, void* stream);

/* Attention of q, ((B, T, heads),(head_dim)) GL_BF16, over the cache: row (b, i, h) is token lengths[b] - T + i of its
 * sequence, sees the tokens up to and including itself and reads kv head h / (heads / kv_heads):
 *   out[b,i,h] = sum_t p_t V_t,  p = softmax_t(scale * q . K_t);  zeros for a row that sees nothing.
 * scale > 0, 2^127 at most; token_pitch as above; out is dense, GL_F32 or, with GL_OUT_BF16 in flags, GL_BF16.
 * Scores, softmax statistics and sums are fp32.  The weights p are rounded when the result is bf16, to fp16 or, where more
 * than 32 rows share a kv head, to bf16, and their sum is that of the rounded ones; for fp32 results they are carried in two
 * such terms (three of bf16).  fp16 ends at 2^-24: with up to 32 rows per kv head every weight may besides be off by 2^-32 of
 * the row's largest (below 2^-31 of it a weight is nothing), which shows where values of next to no weight are very large.
 * Keys, values and queries may lie anywhere in bf16's range as long as the scores, before and after `scale`, and sum |p V|
 * stay in fp32's; with up to 32 rows, blocks of keys with a scale below 2^-109 count as zeros.  Results repeat bit for bit.
 * `workspace`: gl_attend_cache4_workspace() bytes, 1024-byte aligned, scratch: calls that can overlap on the GPU need one
 * each. */
GL_API int gl_attend_cache4(const gl_ap* q, int64_t token_pitch, const gl_cache4* cache, const gl_pages* at, float scale,
                            gl_ap* out, uint32_t flags, void* workspace, size_t workspace_bytes, void* stream);
GL_API size_t gl_attend_cache4_workspace(const gl_ap* q, const gl_cache4* cache);

/* ----------------------------------------------------------------------- */
/* Operands held in 8 bits (F8; not in the paper)                            */
/* ----------------------------------------------------------------------- */

/* A pattern of shape S_A ++ S_C whose items (the prod(S_C) = K values of one access index) are cut into blocks of 128
 * consecutive values.  A block is 128 E4M3 codes (sign, 4 bits of exponent, 3 of mantissa, magnitudes up to 448) and one E8M0
 * scale: value = code * 2^(scale - 127), scale 255 = NaN for the whole block.
 *   data:  gl_f8_data_bytes() bytes; one row per item of ceil(K/16)*16 bytes, codes past K are zero.
 *   scale: gl_f8_scale_bytes() bytes; tiles of 128 rows x 4 blocks, 512 bytes each, row tiles outermost; row r and
 *          block b of a tile at byte (r % 32) * 16 + (r / 32) * 4 + b.
 * Both device pointers are 16-byte aligned.  Size limits (else GL_ERR_UNSUPPORTED): fewer than 2^31 - 256 rows, K <= 2^28,
 * rows * (ceil(K/128) + 1) < 2^31. */
typedef struct {
  void* data;
  void* scale;
  int32_t ndim;
  int32_t access_ndim;
  int64_t shape[GL_MAX_DIMS];
} gl_f8;

/* Bytes of the two arrays (0 on an invalid shape). */
GL_API size_t gl_f8_data_bytes(const gl_f8* a);
GL_API size_t gl_f8_scale_bytes(const gl_f8* a);

/* Rounds `in` (GL_F32 or GL_BF16) to `out`, which carries the same shape.  The scale of a block is the smallest power of two,
 * 2^-127 at least, that its largest magnitude divided by it does not exceed 448; the quotients are rounded to the nearest code,
 * ties to the even mantissa.  A block that holds an Inf or a NaN becomes NaN as a whole. */
GL_API int gl_f8_quantize(const gl_ap* in, gl_f8* out, void* stream);

/* The values of `in` as `out`.  GL_F32 holds every one exactly, GL_BF16 those of scales from 2^-124 on (smaller ones are rounded);
 * a value that its rounding took to 2^128 is Inf. */
GL_API int gl_f8_dequantize(const gl_f8* in, gl_ap* out, void* stream);

/* compute dotProd (cartProd a0 a1) of two F8 patterns of the same compute shape: ((m..),(k..)), ((o..),(k..)) ->
 * ((m.., o..),()), sums in fp32, on the tensor cores' block-scaled 8-bit products.  These cut every product to 2^-25 of the
 * largest term that it is added to, and every sum of 32 toward zero, so that many small products behind a large one are lost; K
 * beyond 65536 is summed in stretches of that length, which are added with rounding to nearest.  Results lie within
 * min(K, 65536) * 2^-24.8 + K * 2^-40 + 2^-21 times sum |a||b|.  Results repeat bit for bit.  flags: GL_EPILOGUE_RELU (NaN stays
 * NaN), GL_OUT_BF16; `out` is GL_F32 or, with GL_OUT_BF16, GL_BF16. */
GL_API int gl_cartesian_dot_f8(const gl_f8* a0, const gl_f8* a1, gl_ap* out, uint32_t flags, void* stream);

/* The same with the left operand given as GL_F32 or GL_BF16 and rounded to F8 by the call (a dense layer: activations
 * a0, weights a1 laid out once by gl_f8_quantize).  The result does not depend on how many rows a0 has beyond the
 * order of the sums.  `workspace`: gl_dense_f8_workspace() bytes, 1024-byte aligned, scratch: calls that can overlap on
 * the GPU need one each. */
GL_API int gl_dense_f8(const gl_ap* a0, const gl_f8* a1, gl_ap* out, uint32_t flags, void* workspace,
                       size_t workspace_bytes, void* stream);
GL_API size_t gl_dense_f8_workspace(const gl_ap* a0, const gl_f8* a1);

/* ----------------------------------------------------------------------- */
/* Norm and positions (not in the paper)                                     */
/* ----------------------------------------------------------------------- */

/* compute norm_rms: every item h = x + residual divided by its root mean square,
 *   out = h / sqrt(mean(h^2) + eps) * weight,   sum = h rounded to its type.
 * x ((a..),(c..)) with c not empty, GL_F32 or GL_BF16; `residual` (NULL: none) and `sum` (NULL: not wanted; only with a
 * residual) of the same shape and of one type, GL_F32 or GL_BF16, which may differ from x's; `weight` (NULL: ones)
 * ((),(c..)), GL_F32 or GL_BF16; eps >= 0 and finite.  out: the shape of x, GL_F32, GL_BF16 or F8.  The norm is that of the
 * unrounded h, in fp32 throughout (units of eight squares are added in 64 bits where a row is longer than a block holds); squares
 * have to stay in fp32's range.  `sum` may be `residual` itself, or x where the types agree, and `out` may be x or `residual`,
 * unless that is `sum`, where the types agree; any other overlap of a result with
 * an operand or the other result is refused (GL_ERR_UNSUPPORTED).
 * Size limits as for F8.  Results repeat bit for bit; the F8 result is the GL_F32 result rounded as gl_f8_quantize rounds. */
GL_API int gl_compute_norm_rms(const gl_ap* x, const gl_ap* residual, const gl_ap* weight, float eps, gl_ap* sum, gl_ap* out,
                               void* stream);
GL_API int gl_compute_norm_rms_f8(const gl_ap* x, const gl_ap* residual, const gl_ap* weight, float eps, gl_ap* sum, gl_f8* out,
                                  void* stream);

/* Rotary positions.  The first 2 * pairs values of a head form pairs, (i, pairs + i) or, `adjacent`, (2i, 2i + 1); pair i belongs
 * to axis axis[i] and is turned by step[i] * position / 2^64 turns.  gl_rotary_plan fills the struct, which a caller may
 * change afterwards (other splits of the pairs between the axes, other frequencies). */
#define GL_MAX_PAIRS 128
typedef struct {
  int32_t pairs;                  /* 1..GL_MAX_PAIRS                                       */
  int32_t axes;                   /* position axes (time, height, width, ..), 1..pairs     */
  int32_t adjacent;               /* 0 or 1                                                */
  int32_t reserved_;
  uint64_t step[GL_MAX_PAIRS];    /* 2^64 * turns per position, modulo 2^64                */
  uint8_t axis[GL_MAX_PAIRS];
} gl_rotary;

/* Host only.  Pair i turns by freq[i] radians per position, base^(-i / pairs) where freq is NULL (1 <= base <= 1e30); sections[a]
 * consecutive pairs belong to axis a (they add up to `pairs`; NULL with one axis).  A step is off by half a unit and |freq[i]| * 2^-62
 * units at most, by two thirds of a unit where a base gives the frequencies. */
GL_API int gl_rotary_plan(int32_t pairs, double base, const double* freq, const int32_t* sections, int32_t axes,
                          int32_t adjacent, gl_rotary* out);

/* compute rotate of x ((B, T, heads),(head_dim)), GL_F32 or GL_BF16: in every head the pair (u, v) of pair i of token (b, t) becomes
 * (u cos - v sin, u sin + v cos) of its angle at positions[axis[i]][b][t]; values behind the pairs are copied.  `positions`:
 * int32 in DEVICE memory, [axes][B][T], any value.  out: shape and type of x; it may be x itself (same data and
 * pitch), otherwise no token of one shares a value with a token of the other (GL_ERR_UNSUPPORTED; either may lie in the other's
 * gaps).  token_pitch, out_pitch: elements between successive tokens (0: dense), at least heads * head_dim.  GL_ROTATE_BACK in
 * flags turns by the negative angles: the inverse, and the gradient.
 * Angles are step[i] * position, exact but for a last rounding of 2^-24 of themselves, cosines and products fp32.  Limits (else
 * GL_ERR_UNSUPPORTED): B * T <= 2^31, heads * head_dim <= 2^24. */
GL_API int gl_compute_rotate(const gl_ap* x, int64_t token_pitch, const gl_rotary* plan, const int32_t* positions, gl_ap* out,
                             int64_t out_pitch, uint32_t flags, void* stream);

/* Synchronises `stream`, then reports and clears the device status word:
 * GL_ERR_TIMEOUT if a bounded wait inside a kernel gave up since the last poll
 * (that kernel's output is then undefined), GL_ERR_CUDA on a runtime error. */
GL_API int gl_poll_device_status(void* stream);

/* Failure-path self-test that faults nothing: launches one block that waits, for at most
 * `limit_ms` (1..1000), on a barrier nothing ever arrives at, using the same bounded wait as the
 * tensor-core pipeline.  The kernel returns normally; the next gl_poll_device_status() on that
 * stream must report GL_ERR_TIMEOUT (and clear it). */
GL_API int gl_selftest_bounded_wait(uint32_t limit_ms, void* stream);

GL_API const char* gl_strerror(int code);
GL_API int gl_version(void);

#ifdef __cplusplus
}
#endif
#endif /* GL_H_ */
