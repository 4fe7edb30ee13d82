/*
 * dynakv.h - C ABI of the token-adaptive KV-cache compression path for AMD MI355X (gfx950):
 * spectral projection, differentiable truncation gate, ragged store and low-rank
 * reconstruction (Sec. 3 "Dynamic Compressing" of the paper, Eqs. 1-8) and the retain-rate
 * regulariser of the training objective (Sec. 3.3, Eq. 9).  Further below, what reads a KV cache
 * and makes it smaller: attention, eviction, a cache in 4 bits.
 *
 * Notation (the paper's): a token's pre-RoPE key or value state is the row vector x with
 * d = d_kv entries; U [d x d] is the spectral basis, W [d x d] and b [d] the gate layer,
 * tau the threshold.  Keys and values have separate parameters: one call handles one stream.
 *
 * Conventions
 *  - Every pointer is DEVICE memory owned by the caller, except the descriptor (host).  The
 *    library allocates nothing and keeps no state between calls; `ws` is scratch whose
 *    contents are undefined after a call, except the error word read by dynakv_check().
 *  - Matrices are row-major.  x has row stride ldx; every other matrix is dense (row stride d).
 *    Matrix pointers must be 16-byte aligned, `ws` 256-byte aligned.
 *  - `stream` is a hipStream_t passed as void* (NULL = the default stream); calls enqueue work
 *    and return without synchronising.
 *  - Return value: LMHEAD_OK or a negative LMHEAD_E_* code (lmhead.h).  Argument errors are
 *    found on the host before anything is launched and leave all outputs untouched.
 *  - Results are bit-reproducible from run to run: no floating-point atomics are used.  Sums are grouped by the size of
 *    the call: x~ and the gradients of a few tokens (their contraction is shared by sixteen wavefronts) and of many
 *    may round differently, and so may the mask where it decides k.
 *  - A workspace sized for a long stream serves every shorter one.
 *
 * Readings of the paper taken by this library (also listed in the design notes):
 *  - Eq. 6 is evaluated as the reverse cumulative sum m_i = sum_{j >= i} p_j, which is the mask
 *    its text describes (1 before the predicted cut-off, 0 after it).  The formula as printed,
 *    Flip(cumsum(p))_i = sum_{j <= d-1-i} p_j, is selected by DYNAKV_FLAG_LITERAL_FLIP; the two
 *    differ by relabelling the gate's output columns j <-> d-1-j.
 *  - The spectral state x~ is rounded to the storage type before it enters the gate layer and
 *    the cache.  Logits, softmax and the mask are fp32; Eq. 8 compares fp32 values.
 *  - The store keeps x~[0:k] of token i at element offset off[i], a multiple of 8 elements
 *    (16 bytes for bf16); the unused tail of the last 8-element granule is written as 0.
 *  - U^-1 of Eq. 3 is an input (U^T for an orthogonal U); the library inverts nothing.
 */
#ifndef DYNAKV_H_
#define DYNAKV_H_

#include <stddef.h>
#include <stdint.h>

#include "lmhead.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
  DYNAKV_FLAG_LITERAL_FLIP = 1u << 0, /* Eq. 6 as printed instead of the reverse cumulative sum */
  DYNAKV_FLAG_ACCUM_GRAD = 1u << 1    /* dynakv_gate_bwd adds to dU, dW, db instead of overwriting them
                                         (the other calls ignore it) */
};

enum { DYNAKV_GRANULE = 8 }; /* elements; segment offsets in the store are multiples of this */

/* Problem descriptor (host memory). */
typedef struct dynakv_desc {
  int32_t n;        /* tokens in this call (> 0)                                              */
  int32_t d;        /* d_kv: a multiple of 64, at most 8192                                   */
  int32_t dtype;    /* LMHEAD_F32 or LMHEAD_BF16: storage type of x, U, W, U_inv, x~, the      */
                    /* store and x_bar.  n * d * sizeof(type) must not exceed 2^31 - 2^20.     */
  uint32_t flags;   /* DYNAKV_FLAG_*                                                           */
  int64_t ldx;      /* row stride of x in elements (>= d, ldx * sizeof(type) % 16 == 0; rows   */
                    /* of which 64 to 256 do not lie within 2 GiB are copied together first)   */
  int64_t reserved; /* must be 0                                                               */
} dynakv_desc;

/* Scratch bytes needed by any of the calls below for this descriptor; 0 if it is invalid.
 * Host-only. */
LMHEAD_API size_t dynakv_workspace_bytes(const dynakv_desc* desc);

/* LMHEAD_OK or the code the compute entry points would return for this descriptor. Host-only. */
LMHEAD_API int dynakv_validate_desc(const dynakv_desc* desc);

/*
 * The gate (Eqs. 1, 5, 6, 7, 8).  Per token (row) i:
 *     x~   = x U                         rounded to the storage type           (Eq. 1)
 *     p    = Softmax(x~ W + b)           fp32                                   (Eq. 5)
 *     m_j  = sum_{l >= j} p_l            soft mask, non-increasing, m_0 = 1     (Eq. 6)
 *     x^   = x~ * m                      element-wise, storage type             (Eq. 7)
 *     k    = #{ j : m_j > tau }          retained leading components            (Eq. 8)
 *   x     [n x d] row stride ldx  (in)     U, W  [d x d]  (in)     b  float[d]  (in)
 *   xt    [n x d] storage type    (out)    x~
 *   k     int32[n]                (out)    the hard mask of token i is 1 on [0, k[i]) and 0 after.  From 10240 bf16
 *                                          tokens on (d = 512 or 1024) a call without m and xhat adds the mask up in
 *                                          another order than one with them: k may differ where m_j is within rounding of tau
 *   m     float[n x d] or NULL    (out)    soft mask (training)
 *   xhat  [n x d] storage type or NULL (out)  softly gated state (training)
 */
LMHEAD_API int dynakv_gate(const dynakv_desc* desc, const void* x, const void* U, const void* W,
                           const float* b, float tau, void* xt, int32_t* k, float* m, void* xhat,
                           void* ws, size_t ws_bytes, void* stream);

/*
 * The ragged store (the components that Eq. 2 leaves and that are "explicitly persisted").
 *     off[0] = off_base,  off[i+1] = off[i] + roundup(k[i], 8)
 *     packed[off[i] + j] = xt[i][j]  for j < k[i],   0 for k[i] <= j < roundup(k[i], 8)
 *   xt       [n x d] storage type (in)      k  int32[n], each in [0, d]  (in)
 *   off_base first element offset to use: 0 for a new store; to append the tokens of a decoding step
 *            to a cache, pass the cache's current end (its off[n_prev]) with `off` pointing at that
 *            entry of the cache's offset array and `packed` at the cache's base.  A multiple of 8, >= 0.
 *   off      int64[n+1]           (out)
 *   packed   storage type, `capacity` elements counted from `packed` (out); 16-byte aligned
 * A k[i] outside [0, d] is clamped into it, and a token whose segment would end beyond
 * `capacity` is not written; either sets the error word (dynakv_check -> LMHEAD_E_RANGE).
 * off_base + n * d elements always suffice.
 */
LMHEAD_API int dynakv_store(const dynakv_desc* desc, const void* xt, const int32_t* k, int64_t off_base,
                            int64_t* off, void* packed, int64_t capacity, void* ws, size_t ws_bytes,
                            void* stream);

/*
 * Dynamic low-rank reconstruction (Eq. 3): x_bar_i = x^_i[0:k_i] U^-1[0:k_i, :], a product whose
 * contraction length differs from token to token.  Tokens are grouped by length on the device so
 * that each matrix-core tile only runs as many steps as its longest token needs.
 *   packed, off, k   as written by dynakv_store; `packed_elems` = elements readable at `packed`
 *                    (at least off[n], at most 2^31 bytes worth)
 *   U_inv   [d x d] storage type (in)
 *   xbar    [n x d] storage type (out)
 * Offsets or counts that point outside `packed_elems` read as zeros and set the error word.
 */
LMHEAD_API int dynakv_reconstruct(const dynakv_desc* desc, const void* packed, int64_t packed_elems,
                                  const int64_t* off, const int32_t* k, const void* U_inv, void* xbar,
                                  void* ws, size_t ws_bytes, void* stream);

/*
 * Retain rate (Eq. 4) and the regulariser of the training objective (Eq. 9).
 *     R_hard = mean_i k[i] / d                         (k may be NULL: reported as 0)
 *     R_soft = mean_{i,j} m[i][j]                      (m may be NULL: reported as 0)
 *     penalty = alpha * R_soft^2,   g_m[i][j] = d penalty / d m[i][j] = 2 alpha R_soft / (n d)
 *   out   float[3] = { R_hard, R_soft, penalty }   (device)
 *   g_m   float[n x d] or NULL                      (device)
 * The sums are taken in a fixed order (deterministic tree), in fp32 with fp64 block totals.
 */
LMHEAD_API int dynakv_retain(const dynakv_desc* desc, const int32_t* k, const float* m, float alpha,
                             float* out, float* g_m, void* ws, size_t ws_bytes, void* stream);

/*
 * Backward of the training-time gate: the chain rule through Eqs. 1, 5, 6 and 7 (the paper trains U, W
 * and b through this "differentiable gate" with the objective of Eq. 9 and states the forward pass only).
 * Given g_xhat = dL/dx^ and, optionally, a direct gradient on the soft mask (the regulariser's is the
 * constant 2 alpha R / (n d): pass it as g_m_const), per token, with p and m recomputed from x~:
 *     q    = dL/dm      = g_xhat * x~ + g_m + g_m_const
 *     r_j  = dL/dp_j    = sum_{i <= j} q_i             (p_j feeds m_0 .. m_j;
 *                                                       sum_{i <= d-1-j} q_i with DYNAKV_FLAG_LITERAL_FLIP)
 *     g_l  = dL/dlogits = p * (r - sum_j p_j r_j)       fp32, then rounded to the storage type
 *     g_x~ = dL/dx~     = g_xhat * m + g_l W^T          storage type (the rounding of x~ is passed
 *                                                       straight through)
 *     dx = g_x~ U^T,    dU = x^T g_x~,    dW = x~^T g_l,    db = sum over tokens of g_l.
 *   x      [n x d] row stride ldx (in)     U, W [d x d] (in)     b float[d] (in)
 *   xt     [n x d] storage type   (in)     x~ as written by dynakv_gate for the same x, U
 *   g_xhat [n x d] storage type   (in)
 *   g_m    float[n x d] or NULL   (in)     g_m_const: added to every element of dL/dm
 *   dx     [n x d] storage type, dense (out)
 *   dU, dW float[d x d]; db float[d]  (out; added to with DYNAKV_FLAG_ACCUM_GRAD)
 *   ws     dynakv_bwd_workspace_bytes(desc) bytes (larger than the forward's: it holds the logits, the
 *          two token-major gradients and the slices of the contractions of dW and dU)
 * The contractions over the tokens accumulate in fp32, in slices summed in a fixed order.
 */
LMHEAD_API size_t dynakv_bwd_workspace_bytes(const dynakv_desc* desc);
LMHEAD_API int dynakv_gate_bwd(const dynakv_desc* desc, const void* x, const void* U, const void* W,
                               const float* b, const void* xt, const void* g_xhat, const float* g_m,
                               float g_m_const, void* dx, float* dU, float* dW, float* db, void* ws,
                               size_t ws_bytes, void* stream);

/* Synchronises `stream` and returns LMHEAD_E_RANGE if the most recent dynakv_* call that used
 * `ws` met a device-side range fault (see dynakv_store / dynakv_reconstruct), else LMHEAD_OK
 * (every call clears the word when it starts). */
LMHEAD_API int dynakv_check(void* ws, void* stream);

/*
 * ---- What reads a KV cache and makes it smaller: attention with a sliding window and a few first tokens that stay visible,
 * and its backward; eviction of tokens by accumulated attention weight; a cache held in 4 bits and attention over it. ----
 *
 * Notation: B sequences; sequence b has lk = len_k[b] keys, in slots 0 .. lk-1 of Tk, and lq = len_q[b] queries, in slots
 * 0 .. lq-1 of Tq, which are its last tokens: query i stands at key position p = lk - lq + i.  It sees key j if
 *     0 <= j <= p   and   (window == 0  or  j > p - window  or  j < sinks).
 * Query head h reads key head h / (Hq / Hkv).  With s = scale <q_i, k_j> over the keys that i sees,
 *     lse_i = log sum_j exp(s_ij),   P_ij = exp(s_ij - lse_i),   out_i = sum_j P_ij v_j.
 * A query that sees no key (p < 0, or a slot from lq on) gives out = 0 and lse = -inf, and so does one whose logits are all -inf.
 *
 *  - As above, the library allocates nothing and keeps no state between calls, argument errors are found before anything is
 *    launched, and results are bit-reproducible (the grouping of sums depends on the sizes of the call).  Descriptors and plane
 *    lists are host memory.  The workspace's error word is read by lmhead_check(): a length outside [0, T], taken as the nearest
 *    one inside.  A workspace belongs to one call at a time.
 *  - What lies in slots from a sequence's length on is never used, whatever its bits, nor is a key that no query of the call
 *    sees.  An infinity or NaN in a key or value that some queries see can reach out and dq of others that do not, whose rows share a
 *    tile of a matrix product with it (0 times an infinity is NaN): those up to 127 positions from one that sees it.  One in a query
 *    or in its g_out can likewise reach dk and dv of keys that the query does not see: those up to 62 positions from one that it sees.
 *  - Logits, softmax and all sums are fp32.  With bf16 storage P, and in the backward dS, are rounded to bf16 before they
 *    enter a matrix product, as are the outputs.  Sixteen bits of P enter out where a key head has up to 32 rows (queries times
 *    heads) over keys in bf16, and sixteen of dS enter dq, and dk of keys that few queries see.
 *  - Logits of up to 2^30 either way are told apart as fp32 tells them.  lse is fp32 too: P that is recomputed from it (the backward, and
 *    weights of more than 8 rows of a key head) is off by |lse| 2^-24 besides, relative to itself.
 */

/* Where element (sequence b, slot t, head h, c) lies: b * seq + t * slot + h * head + c, in elements.  Each stride is a
 * multiple of 16 bytes, not negative, and such that tensors which are written do not overlap themselves; slot strides are below 16 MiB. */
typedef struct attn_layout {
  int64_t seq, slot, head;
} attn_layout;

/* Problem descriptor (host memory). */
typedef struct attn_desc {
  int32_t B;        /* sequences, at most 65535                                               */
  int32_t Tq, Tk;   /* slots for queries, and for keys, of one sequence                       */
  int32_t Hq, Hkv;  /* heads; Hq is a multiple of Hkv, at most 1024                           */
  int32_t D;        /* width of a head: a multiple of 8, at most 128 (4-bit cache: of 32)     */
  int32_t window;   /* 0: all keys up to the query's own position                             */
  int32_t sinks;    /* >= 0                                                                   */
  int32_t dtype;    /* LMHEAD_F32 or LMHEAD_BF16: q, k, v, out and their gradients            */
  float scale;      /* of the logits: finite, > 0                                             */
  uint32_t flags;   /* must be 0                                                              */
  int32_t reserved; /* must be 0                                                              */
  attn_layout q, k, v, o;  /* o: out and its gradient; gradients of q, k, v lie as those do.  */
                           /* Pointers are 16-byte aligned                                    */
} attn_desc;

/* LMHEAD_OK or the code that the calls below would return for this descriptor.  Host-only. */
LMHEAD_API int attn_validate_desc(const attn_desc* desc);

/* Scratch bytes of attn_fwd, kv4_store and kv4_attn; 0 if the descriptor is invalid.  Up to 8 rows of a key head (queries times the heads that read it)
 * have four bytes for each row and key among them, for the logits that `weight` is added up from, whether a call asks for it or not.  Host-only. */
LMHEAD_API size_t attn_workspace_bytes(const attn_desc* desc);

/*
 * Attention, and the weight that each key gets.
 *   q, k, v         (in)
 *   len_q, len_k    int32[B] or NULL: all slots  (in)
 *   out             (out) 0 in the slots of queries that see no key
 *   lse             float[B][Hq][Tq] or NULL     (out)
 *   weight          float[B][Hkv][Tk] or NULL    (in/out) weight[b][h][j] = decay * weight[b][h][j] + sum of P_ij over the
 *                   queries i and the heads that read h, for j < len_k[b]; the rest is left as it was.  With decay = 0 the old
 *                   value is not read.
 *   decay           finite, >= 0
 * Outputs, and the part of the workspace that is used, share no memory with an input or each other.  Here and below a call is refused
 * (LMHEAD_E_SHAPE) where two of them begin at the same place, or where one without gaps shares memory with another; of two tensors
 * with gaps, such as heads of one buffer side by side, that is the caller's to see to.
 */
LMHEAD_API int attn_fwd(const attn_desc* desc, const void* q, const void* k, const void* v, const int32_t* len_q,
                        const int32_t* len_k, void* out, float* lse, float* weight, float decay, void* ws, size_t ws_bytes,
                        void* stream);

/*
 * Backward, given g_out = dL/dout:
 *     dP_ij = <g_i, v_j>,   delta_i = <g_i, out_i>,   dS_ij = P_ij (dP_ij - delta_i)
 *     dq_i = scale sum_j dS_ij k_j,   dk_j = scale sum_i dS_ij q_i,   dv_j = sum_i P_ij g_i
 * (dk, dv: over the queries of all heads that read the key's head).  P is recomputed from q, k and lse.  With bf16 storage
 * <g_i, out_i> is corrected for the rounding of out, so that sum_j dS_ij = 0 as it is for the exact output.
 *   out, lse        as attn_fwd left them for the same q, k, v and lengths  (in)
 *   dq, dk, dv      (out) every slot is written: 0 where nothing is seen, or seen by nobody.  A slot of the padding is 0 too.
 *   ws              attn_bwd_workspace_bytes(desc) bytes
 */
LMHEAD_API size_t attn_bwd_workspace_bytes(const attn_desc* desc);
LMHEAD_API int attn_bwd(const attn_desc* desc, const void* q, const void* k, const void* v, const int32_t* len_q,
                        const int32_t* len_k, const void* out, const float* lse, const void* g_out, void* dq, void* dk,
                        void* dv, void* ws, size_t ws_bytes, void* stream);

/*
 * A cache in 4 bits.  A row of D values of a token and head is cut into blocks of 32.  A block has the scale 2^e with
 * the smallest e >= -126 for which max |x| <= 6 * 2^e, but at most 2^125, stored as the byte e + 127, and a code of four bits
 * for each value: bit 3 the sign, bits 0-2 the index into { 0, 0.5, 1, 1.5, 2, 3, 4, 6 } of x / 2^e, rounded to nearest, of two
 * as near ones to the even index (so the values are e2m1 numbers, and all are finite in bf16).
 * A block with an infinity or a NaN has the scale byte 255 and codes 0 and stands for 32 NaN.
 *   k_codes, v_codes    uint8[B][Hkv][Tk][D / 2]: value 2c in the lower half of byte c, value 2c + 1 in the upper half
 *   k_scales, v_scales  uint8[B][Hkv][Tk][D / 32]
 * Both are dense; codes are 16-byte aligned, scales 4-byte aligned.  Tk and the descriptor's heads are the cache's.
 *
 * kv4_store puts the last len_q[b] tokens of each sequence into it: row i of k and v (Tq slots, layouts desc->k and desc->v)
 * goes to slot len_k[b] - len_q[b] + i; rows of negative slots are left out.  Other slots are left as they are.
 */
LMHEAD_API int kv4_store(const attn_desc* desc, const void* k, const void* v, const int32_t* len_q, const int32_t* len_k,
                         uint8_t* k_codes, uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, void* ws, size_t ws_bytes,
                         void* stream);

/* attn_fwd over such a cache (desc->k and desc->v are not used, but have to be valid).  Scale bytes that
 * kv4_store does not write (0, 253, 254) are no error and stand for no particular value. */
LMHEAD_API int kv4_attn(const attn_desc* desc, const void* q, const uint8_t* k_codes, const uint8_t* k_scales,
                        const uint8_t* v_codes, const uint8_t* v_scales, const int32_t* len_q, const int32_t* len_k, void* out,
                        float* lse, float* weight, float decay, void* ws, size_t ws_bytes, void* stream);

/* ---- eviction ---- */

typedef struct evict_desc {
  int32_t B, T, Hkv;  /* sequences (at most 65535), slots, key heads (at most 1024)            */
  int32_t keep;       /* tokens that stay, 1 .. T                                              */
  int32_t sinks;      /* the first ones, which stay whatever their weight                      */
  int32_t recent;     /* the last ones, which stay too; sinks + recent <= keep                 */
  int32_t flags, reserved; /* must be 0                                                        */
} evict_desc;

/* One tensor of the cache, of rows of `bytes` bytes: row (b, t, h) begins at data + b * seq + t * slot + h * head.  Everything
 * here is in bytes and a multiple of 4 (of 16: rows are then moved 16 bytes at a time). */
typedef struct cache_plane {
  void* data;
  int64_t seq, slot, head;
  int64_t bytes;      /* 4 .. 4096 */
} cache_plane;

enum { EVICT_PLANES = 4 };

LMHEAD_API int evict_validate_desc(const evict_desc* desc);
LMHEAD_API size_t evict_workspace_bytes(const evict_desc* desc);

/*
 * Tokens leave the cache, per key head.  Of a sequence with n = len[b] > keep tokens each key head keeps the first `sinks`, the last
 * `recent` and, of those between, the keep - sinks - recent with the largest weight; of equal weights the lowest slot stays.  A
 * NaN counts as less than any number.  The kept rows close up to slots 0 .. keep-1 in their order, in all planes and in `weight`,
 * whose slots keep .. n-1 become 0.  A sequence with n <= keep stays as it is.  Rows of slots from keep on are left as they were.
 *   planes   1 .. EVICT_PLANES of them (host memory); they share no memory with each other  (in/out)
 *   weight   float[B][Hkv][T]                                                    (in/out)
 *   len      int32[B] or NULL: T each                                            (in)
 *   len_out  int32[B]                                                            (out) min(n, keep); not `len` itself
 *   kept     int32[B][Hkv][keep]: the old slot of each row, ascending; -1 from n on   (out)
 *   ws       evict_workspace_bytes(desc) bytes
 */
LMHEAD_API int cache_evict(const evict_desc* desc, const cache_plane* planes, int32_t count, float* weight, const int32_t* len,
                           int32_t* len_out, int32_t* kept, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DYNAKV_H_ */
