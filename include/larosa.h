/*
 * liblarosa -- decode-time hot path of LaRoSA (layerwise rotated sparse activation,
 * arXiv 2507.01299) for one AMD MI355X (gfx950).
 *
 * Per token and per projection the method computes  y = S_k(x Q) (W Q)^T  (Sec. 4.3,
 * Eq. 9-10): rotate the block input with the layer's orthogonal matrix Q, keep the k
 * entries of largest magnitude (Eq. 8), and multiply by the folded weight, of which only
 * the k kept input channels are read (Sec. 4.4).
 *
 * Conventions common to every entry point
 *  - Every data pointer is a DEVICE pointer owned by the caller.  The library allocates
 *    nothing, frees nothing, and never synchronises: all work is enqueued on `stream`
 *    (a hipStream_t passed as void*; NULL = the default stream).
 *  - 16-bit tensors are IEEE binary16 (LAROSA_F16) or bfloat16 (LAROSA_BF16), row-major,
 *    with fp32 accumulation inside the kernels and one round-to-nearest-even at each store.
 *  - A folded weight W' is stored input-channel-major: row-major [d_in][d_out], so that
 *    input channel i owns one contiguous run of d_out values (Sec. 4.4, point 1: the
 *    "column-major" layout of the [d_out][d_in] linear-layer weight).
 *  - Data pointers must be 16-byte aligned; d_out and d must be multiples of 8.
 *  - Scratch memory comes from the caller's workspace `ws` (256-byte aligned) of at least
 *    the number of bytes the matching *_workspace_bytes() query returns.  A workspace must
 *    be passed once through larosa_workspace_init() after allocation (it zeroes the
 *    arrival counters at its head; the kernels leave them zero again on exit).
 *    One workspace serves one stream: two calls that use the same workspace must be ordered on
 *    one stream (calls that overlap on one workspace corrupt each other's partial sums and
 *    counters, silently).
 *  - Return value: LAROSA_OK (0) or a negative larosa_status.  Invalid arguments are
 *    rejected before anything is enqueued.  LAROSA_EHIP reports a failed launch
 *    (hipGetLastError() != hipSuccess after enqueueing).  After LAROSA_EHIP -- or after any
 *    launch that was aborted or faulted -- the arrival counters of the workspace may be left
 *    non-zero: pass it through larosa_workspace_init() again before the next call.
 *  - Index values (idx) are not range-checked: an index outside [0, d_in) reads outside Wp.
 */
#ifndef LAROSA_H
#define LAROSA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LAROSA_F16 = 0,
  LAROSA_BF16 = 1,
  LAROSA_F32 = 2              /* logits of larosa_logprobs only */
} larosa_dtype;

typedef enum {
  LAROSA_OK = 0,
  LAROSA_EINVAL = -1,       /* null pointer, size out of range, misalignment, unknown dtype */
  LAROSA_EUNSUPPORTED = -2, /* valid request outside what the kernels cover (e.g. d > 32768 in Top-K) */
  LAROSA_EWORKSPACE = -3,   /* workspace missing, misaligned or too small */
  LAROSA_EHIP = -4          /* the HIP runtime reported an error at launch */
} larosa_status;

/* Static, NUL-terminated description of a status code.  Never NULL. */
const char* larosa_status_string(int status);

/* Library version: major*10000 + minor*100 + patch. */
int larosa_version(void);

/* Bytes of workspace that larosa_rotate / larosa_topk / larosa_sparse_gemv need for B tokens
 * with input width <= d_in_max, output width <= d_out_max and kept count <= K_max.
 * Pure host function (no device access).  Returns 0 for non-positive arguments. */
size_t larosa_workspace_bytes(int B, int d_in_max, int d_out_max, int K_max);

/* Zero the arrival counters at the head of a freshly allocated workspace (device pointer,
 * >= larosa_workspace_bytes(1,8,8,1) bytes).  Enqueued on `stream` as a fill kernel. */
int larosa_workspace_init(void* ws, size_t ws_bytes, void* stream);

/* Rotation (Sec. 4.3: the rotated activation x Q; App. A: h_i = sum_j x_j Q_ji).
 *   h[b,i] = sum_j x[b,j] * Q[j,i]
 * x [B,d], Q [d,d] row-major (row j = input channel j; column i = i-th principal direction),
 * h [B,d].  Also serves the residual adapter x (Q_l^T Q_{l+1}) (Sec. 4.2) and, being a dense
 * mat-vec over an input-channel-major matrix, the dense comparator (larosa_dense_gemv is the
 * same operation with a rectangular matrix). */
int larosa_rotate(const void* x, const void* Q, void* h, int B, int d, larosa_dtype t,
                  void* ws, size_t ws_bytes, void* stream);

/* Dense product over an input-channel-major matrix:  y[b,o] = sum_j x[b,j] * Wp[j,o].
 * x [B,d_in], Wp [d_in,d_out], y [B,d_out].  (Eq. 1 with the stored layout; the K = d_in
 * special case of the sparse projection, used as the dense baseline on the same GPU.) */
int larosa_dense_gemv(const void* Wp, const void* x, void* y, int B, int d_in, int d_out,
                      larosa_dtype t, void* ws, size_t ws_bytes, void* stream);

/* Top-K sparsifier S_k (Sec. 4.3, Eq. 8): for each token b, the K indices of largest |h[b,:]|.
 * Magnitudes are compared on the stored 16-bit values (sign bit cleared, bit pattern as an
 * unsigned integer); ties go to the larger magnitude, then to the lower index; exactly K
 * indices are produced, in ascending order.
 * h [B,d]; idx [B,K] int32 (output); vals [B,K] (output, nullable) receives h[b, idx[b,t]].
 * 1 <= K <= d <= 32768.  ws / ws_bytes are not used (the selection needs no scratch in device
 * memory; the arguments keep the signature uniform) and may be NULL / 0. */
int larosa_topk(const void* h, int B, int d, int K, int32_t* idx, void* vals,
                larosa_dtype t, void* ws, size_t ws_bytes, void* stream);

/* Column-sparse projection (Sec. 4.3, Eq. 10; Sec. 4.4 point 3):
 *   y[b,o] = sum_{t<K} h[b, idx[b,t]] * Wp[idx[b,t], o]
 * Only the rows of Wp named by idx are read.  Wp [d_in,d_out] input-channel-major,
 * h [B,d_in], idx [B,K] int32 with 0 <= idx < d_in (per-token index sets; need not be sorted,
 * must not repeat within a token), y [B,d_out] (output). */
int larosa_sparse_gemv(const void* Wp, const void* h, const int32_t* idx, void* y,
                       int B, int d_in, int d_out, int K, larosa_dtype t,
                       void* ws, size_t ws_bytes, void* stream);

/* larosa_sparse_gemv for callers that cannot allocate device memory or bring a workspace (code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): same arguments
 * without `ws`, same kernels, same result bit for bit.  The arrival counters and partial strips
 * live in a device array of LAROSA_STATIC_SCRATCH_BYTES inside the library (one copy per GPU,
 * held until the process ends); the call allocates and frees nothing.  A request whose scratch
 * need exceeds that size returns LAROSA_EUNSUPPORTED and enqueues nothing (batch 1 always fits
 * for d_out <= 262144; for B > 1 the need is that of larosa_workspace_bytes(B, d_in, d_out, K)).
 * The array's address is looked up on the first call on each device (a host-side query, no
 * stream work).  The counters are zeroed by a fill kernel at the start of every call, so the
 * state a previous call left is irrelevant; every call on one GPU shares the one array, so two
 * calls that overlap on that GPU (different streams) race: order them on one stream. */
#define LAROSA_STATIC_SCRATCH_BYTES (8u << 20)
int larosa_sparse_gemv_static(const void* Wp, const void* h, const int32_t* idx, void* y,
                              int B, int d_in, int d_out, int K, larosa_dtype t, void* stream);

/* One decoder layer (Fig. 2; Sec. 3.1 for h1..h4; Sec. 4.2-4.3).  All pointers device, borrowed
 * for the duration of the call. */
typedef struct {
  int d, d_q, d_kv, d_ff;     /* hidden, q/o width, k/v width, intermediate */
  int head_dim;               /* d_q and d_kv are multiples of it; (d_q/head_dim) % (d_kv/head_dim) == 0 */
  int K1, K2, K3, K4;         /* kept counts for h1 (d), h2 (d_q), h3 (d), h4 (d_ff) */
  const void* Wqkv;           /* [d, d_q+2*d_kv]  q|k|v, folded with Q^T on the input side when h1 is rotated */
  const void* Wo;             /* [d_q, d]         meets the unrotated h2 (Q = I, Sec. 4.3) */
  const void* Wgu;            /* [d, 2*d_ff]      gate|up, folded like Wqkv */
  const void* Wdown;          /* [d_ff, d]        meets the unrotated h4 */
  const void* Q_attn;         /* [d,d] or NULL: NULL = x already arrives in the layer's basis (folded form) */
  const void* Q_mlp;          /* [d,d] or NULL */
  const void* adapter;        /* [d,d] Q_l^T Q_{l+1} applied to the layer output, or NULL */
  const void* rms_attn;       /* [d] pre-norm scale or NULL = 1 */
  const void* rms_mlp;        /* [d] or NULL */
  float rms_eps;              /* < 0 disables both pre-norms */
  int attn_mode;              /* 0: context-length-1 attention (softmax over one key = 1, so each query
                                    head outputs the value head of its group); must be 0.  A caller with an
                                    attention core of its own uses larosa_layer_qkv and
                                    larosa_layer_after_attention instead of larosa_layer_forward, one that
                                    wants the library's uses larosa_layer_forward_kv4. */
  larosa_dtype dtype;
  /* Residual adapters on the two shortcuts (Sec. 4.2; with block-level rotations, Sec. 5.4, there is
   * one per block), each [d,d] or NULL = identity: the stream that skips the attention block is taken
   * through shortcut_attn (Q_attn^T Q_mlp when Wo was folded with Q_mlp on its output side), the one
   * that skips the MLP block through shortcut_mlp (Q_mlp^T Q_next with Wdown folded with Q_next).
   * They depend only on the block's input, so they run beside the block's first projection. */
  const void* shortcut_attn;
  const void* shortcut_mlp;
} larosa_layer;

/* Optional copies of every stage (device pointers, each nullable), for stage-by-stage checks:
 * h1 [B,d]; idx1 [B,K1]; qkv [B,d_q+2d_kv]; h2 [B,d_q]; idx2 [B,K2]; o [B,d]; x1 [B,d];
 * h3 [B,d]; idx3 [B,K3]; gu [B,2d_ff]; h4 [B,d_ff]; idx4 [B,K4]; down [B,d]; x2 [B,d];
 * s1, s2 [B,d]: the shortcut values (written only when the layer has that shortcut adapter). */
typedef struct {
  void *h1, *qkv, *h2, *o, *x1, *h3, *gu, *h4, *down, *x2;
  int32_t *idx1, *idx2, *idx3, *idx4;
  void *s1, *s2;
  /* Optional caller-created hipEvent_t handles (each nullable), recorded on `stream` at the stage
   * boundaries so a caller can time the stages of one call: [0] on entry, [1] after the h1 stage
   * (rotation / pre-norm), [2] after q|k|v, [3] after o, [4] after the h3 stage, [5] after gate|up,
   * [6] after down, [7] after the adapter.  Do not pass events while the stream is being captured. */
  void* stage_events[8];
} larosa_trace;

/* Workspace bytes larosa_layer_forward needs for this layer and B tokens (host only). */
size_t larosa_layer_workspace_bytes(const larosa_layer* L, int B);

/* x [B,d] -> x_out [B,d]:
 *   h1 = R(norm(x) Q_attn); qkv = R(S_K1(h1) Wqkv); h2 = attention core of qkv;
 *   o = R(S_K2(h2) Wo); x1 = R(s1 + o); h3 = R(norm(x1) Q_mlp); gu = R(S_K3(h3) Wgu);
 *   h4 = R(SiLU(gate) * up); down = R(S_K4(h4) Wdown); x2 = R(s2 + down);
 *   x_out = R(x2 adapter) or x2;  s1 = R(x shortcut_attn) or x;  s2 = R(x1 shortcut_mlp) or x1.
 *   R = one rounding to the layer dtype.
 * trace may be NULL.  x_out must not alias x.  Rows: the projections of several rows take a counter of the workspace for each
 * group of 32 rows (an explicit rotation behind a learned pre-norm scale: of 4) and 128 output columns (those of a shortcut adapter
 * beside its projection's included), and there are 4096: with gate|up 28672 wide up to 576 rows.  More are LAROSA_EUNSUPPORTED. */
int larosa_layer_forward(const larosa_layer* L, const void* x, void* x_out, int B,
                         const larosa_trace* trace, void* ws, size_t ws_bytes, void* stream);

/* The same layer split around the caller's own attention core (KV cache, softmax: the method leaves it
 * unchanged and only sparsifies its output h2, Sec. 3.1).  Same workspace size, trace and errors as
 * larosa_layer_forward; each call writes only the trace fields of its own stages.
 *
 * larosa_layer_qkv: x [B,d] -> qkv [B, d_q+2*d_kv] = R(S_K1(h1) Wqkv), and, when the layer has
 * shortcut_attn, s1 [B,d] = R(x shortcut_attn) (required then; ignored and may be NULL otherwise).
 * trace->qkv and trace->s1 are not written (the caller has both).
 *
 * larosa_layer_after_attention: attn [B,d_q] is the attention core's output in the layer dtype and
 * takes the place of h2; residual [B,d] is what the attention block's output is added to: the layer
 * input x, or the s1 written by larosa_layer_qkv when the layer has shortcut_attn.  Runs
 * o = R(S_K2(attn) Wo); x1 = R(residual + o); then the MLP block and the adapter as above.
 * x_out must not alias residual. */
int larosa_layer_qkv(const larosa_layer* L, const void* x, void* qkv, void* s1, int B,
                     const larosa_trace* trace, void* ws, size_t ws_bytes, void* stream);
int larosa_layer_after_attention(const larosa_layer* L, const void* residual, const void* attn, void* x_out,
                                 int B, const larosa_trace* trace, void* ws, size_t ws_bytes, void* stream);

/* ---- Offline part on the GPU (Sec. 4.2: PCA rotation of each layer's input, rotation folded into the
 * neighbouring weights, residual adapter between consecutive layers).  The eigendecomposition itself
 * is left to the caller's solver: these calls produce its input and consume its output.
 * All pointers are device memory; matrices are dense row-major; d, d_in, d_out are multiples of 8;
 * 16-bit tensors are of type t; every call is asynchronous on `stream`.  Rotations are passed in fp32
 * and are NOT rounded to 16 bits before the products: they are split into 16-bit terms in `ws`
 * (borrowed for the duration of the call's kernels, 256-byte aligned).  Errors as for the calls above:
 * LAROSA_EINVAL for null/misaligned pointers or bad sizes, LAROSA_EWORKSPACE for a workspace that is
 * too small, LAROSA_EHIP when a launch fails. */

/* Bytes of workspace the three folding calls below need for d x d rotations of type t (host only). */
size_t larosa_offline_workspace_bytes(int d, larosa_dtype t);

/* Second-moment accumulation (Sec. 4.2): C (+)= X^T X for n_tokens calibration rows X [n_tokens, d]
 * (16-bit, type t), C [d, d] fp32, exactly symmetric.  accumulate = 0 overwrites C, 1 adds to it, so a
 * calibration set can be fed in batches; the caller divides by the token count if it wants the
 * average (the eigenvectors do not depend on it).  fp32 accumulation on the matrix cores. */
int larosa_second_moment(const void* X, int n_tokens, int d, larosa_dtype t, float* C, int accumulate,
                         void* stream);

/* Input-side fold (Sec. 4.2, Eq. 9-10): W_out = Q^T W for W [d, d_out] in the input-channel-major layout
 * the projections read, Q [d, d] fp32 with the principal directions as columns.  W_out [d, d_out] is
 * rounded once to type t.  W_out must not alias W. */
int larosa_fold_input(const float* Q, const void* W, int d, int d_out, larosa_dtype t, void* W_out, void* ws,
                      size_t ws_bytes, void* stream);

/* Output-side fold (Sec. 3.2): W_out = W Q for W [d_in, d]: the projection then emits its output in the
 * basis Q.  W_out [d_in, d], rounded once to type t, must not alias W. */
int larosa_fold_output(const void* W, const float* Q, int d_in, int d, larosa_dtype t, void* W_out, void* ws,
                       size_t ws_bytes, void* stream);

/* Residual adapter (Sec. 4.2): A = Q_l^T Q_next, [d, d], rounded once to type t: the dense mat-vec that
 * takes the residual stream from layer l's basis to the next layer's. */
int larosa_residual_adapter(const float* Q_l, const float* Q_next, int d, larosa_dtype t, void* A_out, void* ws,
                            size_t ws_bytes, void* stream);

/* ---- 4-bit weights (W4A16).  The paper reports that the method keeps its accuracy on round-to-nearest
 * and calibrated 4-bit weights (Sec. 5.4, Table 9) and names a kernel that does both as future work;
 * it fixes no storage format, so the one here is this library's own:
 *   Wq     [d_in, d_out/8] uint32: nibble k (bits 4k..4k+3) of dword m of row j = code q of column 8m+k
 *   scales [d_in, ceil(d_out/128)] 16-bit (type t): weight(j, o) = (q - 8) * scales[j, o/128]
 * i.e. symmetric codes with one scale per input-channel row and per group of 128 output columns, so
 * that a kept row is still one contiguous burst and its scales fold into the row's coefficient. */

/* Round-to-nearest quantisation of W [d_in, d_out] (16-bit, type t): scale = max|w| over the group / 7
 * rounded to type t, q = clip(rint(w / scale), -8, 7) + 8 (q = 8 where the scale is 0).
 * d_out % 8 == 0.  Device pointers, 16-byte aligned; asynchronous on `stream`. */
int larosa_quantize_w4(const void* W, int d_in, int d_out, larosa_dtype t, void* Wq, void* scales, void* stream);

/* Column-sparse projection (Sec. 4.3, Eq. 10) over the 4-bit weight:
 *   y[b,o] = sum_t h[b, idx[b,t]] * (q[idx[b,t], o] - 8) * scales[idx[b,t], o/128],  fp32 accumulate,
 * one rounding to type t.  idx as for larosa_sparse_gemv (ascending, distinct, per token), or NULL
 * with K == d_in for the dense product over all rows.  Workspace as for larosa_sparse_gemv. */
int larosa_sparse_gemv_w4(const void* Wq, const void* scales, const void* h, const int32_t* idx, void* y, int B,
                          int d_in, int d_out, int K, larosa_dtype t, void* ws, size_t ws_bytes, void* stream);

/* ---- Magnitude-threshold sparsifier S_eps (Eq. 4-5), the comparison method of Sec. 4.1 whose kept count
 * depends on the token: idx[b*d .. b*d + count[b]) = ascending channels with |h[b,i]| > eps (compared
 * exactly: 16-bit magnitudes widened to fp32 against the fp32 eps; NaN is dropped).
 * h [B, d] 16-bit, idx [B, d] int32 (capacity d per token), count [B] int32; device pointers;
 * d % 8 == 0, d <= 32768.  Feeding a token's idx and count[b] (read back by the caller) to
 * larosa_sparse_gemv gives the variable-K projection that the fixed-K Top-K path is compared with. */
int larosa_threshold_select(const void* h, int B, int d, float eps, larosa_dtype t, int32_t* idx, int32_t* count,
                            void* stream);

/* ---- Key/value cache in 4 bits and the attention over it: the core that larosa_layer_qkv and
 * larosa_layer_after_attention leave to the caller.  The method does not touch the attention core (Sec. 3.1), so the format is
 * this library's own: pages of page_tokens tokens, shared between sequences and handed out through a page table.
 *
 *   data    n_layers pools one after the other, each n_pages pages of larosa_kv4_page_bytes() bytes.  A page holds, for
 *           each key/value head, page_tokens / 32 blocks of 34 head_dim bytes (32 tokens each):
 *           codes of K (16 head_dim bytes), codes of V (16 head_dim), scales of K (head_dim), scales of V (head_dim).
 *   value   = code * 2^(scale - 127): code = sign (bit 3) and magnitude 0, 1/2, 1, 3/2, 2, 3, 4, 6 (bits 0..2); one scale byte for
 *           32 neighbouring values of a head (value i belongs to group i / 32); a group with scale 255 is NaN.
 *   layout  with D = head_dim, token t of the block, u = t / 16, W = min(16, D / 8), byte b of a lane's D / 8:
 *           at(lane, b) = u 8 D + (b / W) 64 W + lane W + b mod W, even values in the low nibble;
 *           K value i: lane = (i / (D/4)) 16 + t mod 16, b = (i mod D/4) / 2, at at(lane, b);
 *           V value i: lane = (t mod 16 / 4) 16 + i / (D/16), b = (t mod 4) D/32 + (i mod D/16) / 2, at 16 D + at(lane, b);
 *           scale of K, group g: 32 D + u D/2 + 16 g + t mod 16;
 *           scale of V, group g: 33 D + u D/2 + ((t mod 16 / 4) D/32 + g) 4 + t mod 4.
 *   table   [n_slots, max_pages]: page of tokens [p page_tokens, (p + 1) page_tokens) of the sequence in a slot, -1 = none
 *   length  [n_slots]: tokens of the sequence in a slot (0: the slot is free)
 *   refs    [n_pages]: table entries that name the page (0: the page is free)
 * head_dim is 64, 128 or 256; page_tokens 32, 64, 128 or 256; at most 2^18 slots, 2^28 pages and 2^43 bytes of data,
 * which is 16-byte aligned.  A page id outside [0, n_pages) is
 * never followed: tokens on it are not stored and not seen.  Two calls that use one cache are ordered on one stream. */
typedef struct {
  int n_layers, n_pages, page_tokens, n_slots, max_pages;
  int n_kv_heads, head_dim;
  larosa_dtype dtype;         /* of the keys and values that go in and of the queries */
  void* data;
  int32_t *refs, *table, *length;
} larosa_kv4_cache;

/* Which rows of a batch are the newest tokens of which sequence.  Rows starts[s] .. starts[s+1] - 1 (starts NULL: row s alone)
 * are the last tokens of the sequence in slots[s], whose length counts them already (larosa_kv4_grow).  A slot
 * outside [0, n_slots) marks a sequence as padding.  Rows outside [0, n_rows), rows of no sequence and rows past the first
 * max_new of a sequence are neither read nor written. */
typedef struct {
  const int32_t* slots;       /* [n_seq], device; a slot at most once */
  const int32_t* starts;      /* [n_seq + 1], device, or NULL */
  int n_seq, n_rows;
  int max_new;                /* most new tokens of one sequence, up to 2^18; 1 with starts NULL */
} larosa_kv4_batch;

/* Rotary positions.  Frequency j < rot_dim / 2 turns the pair of values (j, j + rot_dim / 2) of a head, or (2 j, 2 j + 1) if
 * interleaved; values from rot_dim on stay.  The angle of frequency j at position p is given by its cosine table[p, j] and its sine
 * table[p, rot_dim / 2 + j] (fp32).  Several axes (time, height, width of a picture's tokens): the first axis_pairs[0] frequencies
 * take their position from positions[0, row], the next axis_pairs[1] from positions[1, row], and so on.  positions NULL (one axis
 * only): a token's place in its sequence.  A position outside [0, n_positions) makes the values it turns NaN. */
typedef struct {
  const float* table;         /* [n_positions, rot_dim], device */
  int n_positions, rot_dim;   /* rot_dim: multiple of 16, at most head_dim */
  int interleaved;
  const int32_t* positions;   /* [n_axes, n_rows], device, or NULL */
  int n_axes;                 /* 1 to 4 */
  int axis_pairs[4];          /* n_axes > 1: frequencies of each axis, together rot_dim / 2 */
} larosa_rotary;

/* Bytes of one page of one layer, and of a whole cache's data (0 for sizes that are not supported). */
size_t larosa_kv4_page_bytes(int page_tokens, int n_kv_heads, int head_dim);
size_t larosa_kv4_data_bytes(const larosa_kv4_cache* C);

/* Make the cache empty: refs and length 0, table -1 (data stays as it is). */
int larosa_kv4_clear(const larosa_kv4_cache* C, void* stream);

/* New tokens of one layer into the cache.  qkv [n_rows, ld_qkv]: q | k | v of each row, n_heads, n_kv_heads and n_kv_heads heads of
 * head_dim values (what larosa_layer_qkv writes).  q and k are turned by `rotary` (NULL: not), in fp32 with every product and sum
 * rounded; k and v are stored in 4 bits: with m the largest magnitude of a group, e = floor(log2 m) - 2, one more if
 * m > 7 2^e, held to [-23, 13] (F16) or [-100, 125] (BF16), the nearest code of value / 2^e, ties to the even code, 6 for more;
 * a group that holds a NaN or infinity becomes NaN.  Tokens without a page, or whose place would be negative, are not stored.
 * out [n_rows, ld_out] (nullable without rotary): q as turned, k and v as the cache now holds them, rounded once to the type; it
 * may be qkv itself (with ld_out == ld_qkv).  ld_qkv, ld_out: multiples of 8.  The pages that are written must belong to one
 * sequence (larosa_kv4_grow sees to it). */
int larosa_kv4_append(const larosa_kv4_cache* C, int layer, const larosa_kv4_batch* batch, const void* qkv, int ld_qkv,
                      int n_heads, const larosa_rotary* rotary, void* out, int ld_out, void* stream);

/* Attention of the batch's rows over the cache of one layer (n_heads a multiple of n_kv_heads, query head h reads
 * key/value head h / (n_heads / n_kv_heads)):
 *   out[row, h, :] = sum_t w_t v_t / sum_t w_t,   w_t = exp(scale (q[row, h, :] . k_t) - max)
 * over the tokens t <= place of the row in its sequence and, with window > 0, t > place - window.  A row that sees no token (an
 * empty sequence, padding of a batch with starts, pages missing) gets zeros, and so does one whose logits are all -infinity.  Sums and the
 * maximum are fp32; the weights w_t are rounded to 16 bits, above and below alike (f16: those below 2^-21 of a row's largest may
 * lose more), the values are exact.  Sums of bf16 values are fp32's too: many of more than 2^110 overflow.
 * q [n_rows, ld_q], out [n_rows, ld_out]: multiples of 8 apart, out rounded once.
 * max_len: about the longest sequence, by which the work is divided over the chip (0: max_pages * page_tokens); longer ones are
 * right too.  Workspace: larosa_kv4_attention_workspace_bytes of the same arguments, initialised by larosa_workspace_init. */
size_t larosa_kv4_attention_workspace_bytes(const larosa_kv4_cache* C, const larosa_kv4_batch* batch, int n_heads, int max_len);
int larosa_kv4_attention(const larosa_kv4_cache* C, int layer, const larosa_kv4_batch* batch, const void* q, int ld_q,
                         int n_heads, float scale, int window, int max_len, void* out, int ld_out, void* ws, size_t ws_bytes,
                         void* stream);

/* ---- Pages of the cache.  The bookkeeping lives on the device and is changed in stream order; nothing returns to the host
 * unless the caller reads it.  Lists hold slots (int32, device).  Free pages are handed out from the lowest id on, in the order of
 * the list, so that equal calls give equal tables.  `status` (one int32, device) receives 0, or says why nothing was changed.
 * Workspace: larosa_kv4_pages_workspace_bytes, initialised by larosa_workspace_init like any other. */
size_t larosa_kv4_pages_workspace_bytes(const larosa_kv4_cache* C);

/* Room for counts[i] more tokens (counts NULL: one) in every listed slot; length grows by as much, and the tokens are then stored by
 * one larosa_kv4_append for each layer.  Where a slot's last page is not full and shared, the slot takes a copy of it (of
 * all layers) first; if all that share it are in the list, the last of them keeps it.  status: 0; the number of pages that
 * are missing; or -1: a slot out of range or listed twice, a negative count, a table row too short.  1 <= n <= n_slots. */
int larosa_kv4_grow(const larosa_kv4_cache* C, const int32_t* slots, const int32_t* counts, int n, int32_t* status, void* ws,
                    size_t ws_bytes, void* stream);

/* The sequence of src[i] becomes that of the free slot dst[i] too; all pages are shared.  status: 0, or -1: a slot out of
 * range, dst[i] not free, listed twice or among src.  A src may be listed several times.  1 <= n <= n_slots. */
int larosa_kv4_fork(const larosa_kv4_cache* C, const int32_t* src, const int32_t* dst, int n, int32_t* status, void* stream);

/* Every listed slot keeps its first keep[i] tokens at most (keep NULL: none, the slot is free again); pages that no table names
 * any more are free.  Slots out of range are passed over, a negative keep counts as 0; of a slot listed several times the smallest
 * keep counts. */
int larosa_kv4_trim(const larosa_kv4_cache* C, const int32_t* slots, const int32_t* keep, int n, void* stream);

/* Pages in use move to the lowest ids: with n of them, those with ids from n on (ascending) into the free ids below n (ascending);
 * tables and refs follow.  live (one int32, device, nullable) receives n: pages from n on are free. */
int larosa_kv4_compact(const larosa_kv4_cache* C, int32_t* live, void* ws, size_t ws_bytes, void* stream);

/* Page src[i] of every layer into page dst[i], for a caller with bookkeeping of its own; pairs with an id out of range are passed
 * over.  No dst twice or among src.  tables and refs are not touched. */
int larosa_kv4_copy_pages(const larosa_kv4_cache* C, const int32_t* src, const int32_t* dst, int n, void* stream);

/* One decoder layer with this cache as its attention core: larosa_layer_qkv, larosa_kv4_append, larosa_kv4_attention and
 * larosa_layer_after_attention over batch->n_rows rows, x [n_rows, d] -> x_out [n_rows, d].  The lengths count the rows'
 * tokens already (larosa_kv4_grow once for all layers).  L's head_dim, d_kv and dtype are the cache's.  trace as in the split calls.
 * Rows of no sequence come out unspecified.  Rows up to what larosa_layer_forward takes: longer prompts go through in pieces, the cache
 * holds what came before.  Workspace: larosa_layer_kv4_workspace_bytes (0 for a call that would be refused), initialised as ever. */
size_t larosa_layer_kv4_workspace_bytes(const larosa_layer* L, const larosa_kv4_cache* C, const larosa_kv4_batch* batch, int max_len);
int larosa_layer_forward_kv4(const larosa_layer* L, const larosa_kv4_cache* C, int layer, const larosa_kv4_batch* batch,
                             const larosa_rotary* rotary, float scale, int window, int max_len, const void* x, void* x_out,
                             const larosa_trace* trace, void* ws, size_t ws_bytes, void* stream);

/* ---- Weights in 8-bit floating point: products of any number of rows (prompts, the output head) and what is read off the head's
 * logits.  The method leaves prompts and the output head dense (Sec. 4.4 is about decoding; perplexity and scored choices are what it is judged
 * by, Tables 1 and 2); the format is this library's own:
 *   codes   e4m3 (sign, 4 bits of exponent, 3 of mantissa; at most 448; 0x7F and 0xFF are NaN)
 *   scales  one byte for each block of 128: 2^(byte - 127), a power of two, which the matrix instructions apply by themselves
 *   weight  of d_out output and d_in input channels: codes [d_out, P], scales [ceil(d_out / 128), S], a block is 128 x 128
 *   rows    codes [n_rows, P], scales [n_rows, S], a block is 128 neighbouring values of a row
 *           P = d_in rounded up to 16 (zeros behind d_in), S = ceil(d_in / 128) rounded up to 4 (127 behind the last block)
 *   value   = code * 2^(byte - 127), with the byte of the value's block
 * A block's scale is the least 2^e >= 2^-64 for which its largest magnitude is at most 448 * 2^e, its codes are nearest to value / 2^e, ties
 * to the even one; a block that holds a NaN or infinity gets scale 1 and NaN codes.  Values below 2^-74 in a block of such values count as 0.
 * Scale bytes that a caller brings lie in 63 .. 247, as these do.
 * d_in is at most 2^20, d_out and ld_y below 2^21, n_rows at most 2^24; codes are 16-byte aligned, scales 4-byte. */

/* W [d_in, d_out] (16-bit, type t, the layout of every weight of this library; d_out a multiple of 8) -> codes, scales.  An output head of any
 * other number of tokens: fill W up with columns of zeros, which change no scale, and use the first n_vocab rows of the codes with all scales. */
int larosa_quantize_w8(const void* W, int d_in, int d_out, larosa_dtype t, void* codes, void* scales, void* stream);

/* x [n_rows, d] (16-bit, type t, rows ld_x apart, a multiple of 8) -> codes, scales.  rms_eps >= 0: behind a norm,
 * x / sqrt(mean(x^2) + rms_eps) * rms (rms [d] or NULL = 1), in fp32 and not rounded before the codes; rms_eps < 0: as they are (rms is
 * not read). */
int larosa_quantize_rows8(const void* x, int ld_x, int n_rows, int d, const void* rms, float rms_eps, larosa_dtype t, void* codes,
                          void* scales, void* stream);

/* y[m, o] = sum_i x[m, i] W[o, i] over the values that rows and weight stand for; y [n_rows, d_out] (type t, rows ld_y apart, a multiple of
 * 8), rounded once.  d_out is a multiple of 8.  Sums are fp32; from 17 rows on the products of eight neighbours are added by the 8-bit matrix
 * instruction, which cuts them 13 bits below the largest one's exponent (about 2^-16 of the result's norm, with a few strong channels 2^-14.5).
 * So a row's last bits depend on how many rows are with it; the same call gives the same bits every time.
 * Workspace: larosa_product8_workspace_bytes, initialised by larosa_workspace_init; one for n_rows rows serves any smaller number of
 * them too, here and in the calls below (the query looks at all of them: once for a workspace, not at every call).  Up to 2^23 tiles of 128 rows x 128 channels. */
size_t larosa_product8_workspace_bytes(int n_rows, int d_in, int d_out);
int larosa_product8(const void* w_codes, const void* w_scales, const void* x_codes, const void* x_scales, void* y, int ld_y,
                    int n_rows, int d_in, int d_out, larosa_dtype t, void* ws, size_t ws_bytes, void* stream);

/* larosa_quantize_rows8 into the workspace and larosa_product8: x, y and rms in type t; y must not overlap x. */
size_t larosa_dense_w8_workspace_bytes(int n_rows, int d_in, int d_out);
int larosa_dense_w8(const void* w_codes, const void* w_scales, const void* x, int ld_x, const void* rms, float rms_eps, void* y,
                    int ld_y, int n_rows, int d_in, int d_out, larosa_dtype t, void* ws, size_t ws_bytes, void* stream);

/* Log probabilities.  For each row of logits [n_rows, n_vocab] (type t, F32 too; rows ld apart, any ld >= n_vocab; aligned to their type), with
 * z = scale * logit (0 < scale <= 2^126: one over a temperature):
 *   logp[r, i]  = z[given[r, i]] - ln sum exp z       given, logp [n_rows, n_given]; a negative id is padding: 0; an id >= n_vocab: NaN
 *   entropy[r]  = - sum p ln p, in nats               [n_rows], nullable
 *   top_id, top_logp [n_rows, n_top]: the n_top largest logits, ties to the lower id, with their log probabilities (top_logp nullable)
 * A logit of -infinity has probability 0; a row of nothing else gets logp -infinity and entropy 0.  A row that holds a NaN or +infinity gets
 * NaN everywhere and top_id -1.  A logit counts as -infinity where its difference to the row's largest leaves fp32.  Sums and statistics
 * are fp32.  n_given >= 0, 0 <= n_top <= min(64, n_vocab); outputs that are not asked for (n_given or n_top 0) may be NULL.
 * Workspace: larosa_logprobs_workspace_bytes (the same for every type), initialised by larosa_workspace_init; at most 2^24 rows of at most 2^28 logits. */
size_t larosa_logprobs_workspace_bytes(int n_rows, int n_vocab, int n_top, larosa_dtype t);
int larosa_logprobs(const void* logits, int ld, int n_rows, int n_vocab, larosa_dtype t, float scale, const int32_t* given,
                    int n_given, float* logp, float* entropy, int n_top, int32_t* top_id, float* top_logp, void* ws,
                    size_t ws_bytes, void* stream);

/* From hidden rows to log probabilities: norm (rms, rms_eps as above), rows to 8 bits, the output head (codes, scales of n_vocab output
 * channels, any number), larosa_logprobs of its fp32 logits.  The logits of a part of the rows at a time lie in the workspace. */
size_t larosa_score_w8_workspace_bytes(int n_rows, int d_in, int n_vocab, int n_top);
int larosa_score_w8(const void* w_codes, const void* w_scales, const void* x, int ld_x, const void* rms, float rms_eps, int n_rows,
                    int d_in, int n_vocab, larosa_dtype t, float scale, const int32_t* given, int n_given, float* logp,
                    float* entropy, int n_top, int32_t* top_id, float* top_logp, void* ws, size_t ws_bytes, void* stream);

/* ---- NOT part of the stable interface: launch tuning for tests and experiments.
 * Process-wide host state read by every call (launch shapes AND workspace sizes depend on it): not
 * thread-safe; change it only while no call of this library is in flight, and before sizing a workspace.
 * Production callers never call it: the defaults are derived from the arguments of each call.
 * key 0 = target number of workgroups of the row-streaming kernels (0 = automatic),
 * key 1 = minimum kept rows per workgroup, key 2 = row-waves per workgroup of the stand-alone
 * row-streaming kernel (0: 8, 1: 16, 2: 4), key 3 = decoder layer with the Top-K fused into the
 * projection kernels (1, default) or as separate kernels (0),
 * key 5 / key 6 = workgroups of a projection / of the shortcut adapter that shares its launch
 * (0 = chosen from the two jobs' sizes, default),
 * key 7 = narrowest output width for which the 4-bit projection uses its 2048-column geometry,
 * key 8 = with key 9 = 0: widest MLP intermediate vector whose Top-K runs inside the down projection's
 * workgroups (wider ones are selected once by the Top-K kernel),
 * key 9 = batch-1 decoder layer: the down projection takes its Top-K threshold from key histograms
 * that the gate|up launch builds (1, default) or selects for itself (0),
 * key 10 = workgroup tile of the offline contractions: 0 = chosen by size (default), 1 = 128 x 128, 2 = 256 x 256,
 * key 11 = workgroup tile (output channels x rows) of the products over 8-bit weights from 17 rows on: 0 = chosen by size (default),
 * 1 = 256 x 256, 2 = 256 x 192, 3 = 128 x 256, 4 = 128 x 128, 5 = 128 x 64 (more than 2^23 of the tile asked for: LAROSA_EUNSUPPORTED).
 * Returns LAROSA_EINVAL for an unknown key or a value out of range. */
int larosa_set_tuning(int key, int value);

/* How larosa_kv4_attention would divide a call (host only): plan[0] = rows of a tile (16 or 32), [1] = tiles of a key/value head's
 * rows, [2] = blocks of 32 tokens that a workgroup takes at most, unless it is a tile's last, [3] = most workgroups of a tile, [4] = floats that
 * each of them leaves where there are several.  Pointers of the cache and the batch's starts are not followed. */
int larosa_kv4_attention_plan(const larosa_kv4_cache* C, const larosa_kv4_batch* batch, int n_heads, int window, int max_len,
                              int* plan);

#ifdef __cplusplus
}
#endif
#endif /* LAROSA_H */
