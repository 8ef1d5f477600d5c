/*
 * tri.h -- C ABI of libtri: the Thinker decoder-layer forward on one MI355X
 * (gfx950), in the two arithmetic-intensity regimes the paper contrasts.
 *
 * The paper's Thinker stage (Section II-A) consumes its token stream in a
 * compute-bound prefill and then decodes autoregressively over a KV cache;
 * Section II-C (Observation 2) attributes prefill to dense GEMM kernels and
 * decode to GEMV-like operators, and Section III-A1 labels each scheduler step
 * prefill, decode or mixed from its per-request scheduled-token counts.  This
 * library computes one decoder layer for such a step:
 *
 *   h   = RMSNorm(x; attn_norm)                      y = x / sqrt(mean(x^2)+eps) * g
 *   q,k,v = h W_qkv^T (+ b_qkv), optionally each q and k head RMS-normalised
 *         (TRI_F_QK_NORM), rotary embedding on q and k at each token's
 *         position (rotate-half pairs (i, i+D/2), angle pos * base^(-2i/D)
 *         formed in double precision; with TRI_F_MROPE frequency i takes the
 *         temporal, height or width id of the token by its section), k and v
 *         appended to the cache
 *   o   = causal grouped-query softmax attention over the cache (query head j
 *         reads KV head floor(j*Hkv/Hq)), scale 1/sqrt(D)
 *   x1  = x + o W_o^T
 *   h2  = RMSNorm(x1; mlp_norm)
 *   out = x1 + SwiGLU(h2)                             dense
 *   out = x1 + sum_j w_j SwiGLU_{e_j}(h2)             MoE, top-k softmax routing
 *
 * The paper gives no layer equations; the structure is the Qwen2-family
 * pre-norm decoder of the model it serves (Section IV-A), and every
 * convention above is a declared reading.
 *
 * Conventions common to all entry points
 *  - Every pointer named "device" is a device (HBM) address; host structs are
 *    read during the call only.  The caller owns every buffer (weights, cache,
 *    activations, outputs, workspace); the library allocates nothing and keeps
 *    no pointer after returning.
 *  - Calls are asynchronous on `stream` (a hipStream_t; NULL = the default
 *    stream) and never synchronise with the host.
 *  - Arguments are validated on the host before any launch; a negative status
 *    means nothing was launched and nothing was written.  TRI_ERR_HIP means a
 *    launch failed: outputs and this call's cache rows are then unspecified.
 *  - Device-side index arrays (cu_q, ctx_len, slot, pos) cannot be checked on
 *    the host.  Kernels never read or write outside the buffers described
 *    here: a token whose slot is >= n_slots or whose cache row is >= max_seq
 *    is skipped (its outputs are unspecified).
 *  - Element type ("storage type" below): bfloat16 (TRI_BF16, the serving
 *    path) or float32 (TRI_F32, the tight-parity mode) for the weights, the
 *    activations, the KV cache and the workspace intermediates, as
 *    tri_layer_config.dtype says; arithmetic accumulates in float32 in both.
 *    TRI_F32 runs the same kernels on fp32 storage: every projection on the
 *    matrix cores over bf16 operand planes of the fp32 values (activations
 *    split hi | lo | hi, weights hi | hi | lo, v = hi + lo with hi = bf16(v),
 *    lo = bf16(v - hi)), which keeps each product to ~2^-16 relative, and
 *    attention on the fp32 matrix instruction; it rebuilds the weight planes
 *    in the workspace on every call and is not meant for speed.  Weights are
 *    row-major [out, in].  All device buffers must be 16-byte aligned.
 */
#ifndef TRI_H
#define TRI_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TRI_OK = 0,
  TRI_ERR_NULL = -1,        /* a required pointer is NULL                         */
  TRI_ERR_SHAPE = -2,       /* inconsistent sizes                                 */
  TRI_ERR_UNSUPPORTED = -3, /* valid but not implemented (dtype, head_dim, flag)  */
  TRI_ERR_RANGE = -4,       /* a size exceeds a buffer (e.g. ctx + q > max_seq)   */
  TRI_ERR_ALIGN = -5,       /* a device pointer is not 16-byte aligned            */
  TRI_ERR_WORKSPACE = -6,   /* workspace smaller than tri_workspace_size()        */
  TRI_ERR_HIP = -7,         /* a HIP launch failed                                */
  TRI_ERR_ALIAS = -8,       /* an output overlaps an input it must not overlap    */
  TRI_ERR_SCRATCH = -9      /* the call needs more than the library's fixed
                               scratch (tri_layer_decode_noalloc)               */
} tri_status;

typedef enum { TRI_BF16 = 0, TRI_F32 = 1 } tri_dtype;

enum {
  TRI_F_QKV_BIAS = 1,   /* add b_qkv after the q/k/v projection                   */
  TRI_F_MOE = 2,        /* mixture-of-experts FFN instead of the dense SwiGLU      */
  TRI_F_MOE_RENORM = 4, /* renormalise the top-k routing weights to sum to 1       */
  TRI_F_QK_NORM = 8,    /* per-head RMSNorm of q and k (gains q_norm, k_norm, eps
                           rms_eps) after the projection, before the rotation: the
                           Qwen3-family variant of the layer                         */
  TRI_F_MROPE = 16,     /* multi-section rotary positions (the multimodal rotary
                           embedding of the Qwen2-VL / Qwen2.5-Omni family): every
                           token has three position ids (temporal, height, width;
                           tri_batch.pos is then [3][n_tokens]) and rotary
                           frequency i < mrope_section[0] takes the temporal id,
                           i < mrope_section[0] + mrope_section[1] the height id,
                           the rest the width id                                     */
  TRI_F_ALL = 31
};

typedef struct {
  int32_t hidden;         /* H; multiple of 64                                      */
  int32_t n_q_heads;      /* Hq                                                     */
  int32_t n_kv_heads;     /* Hkv; Hq % Hkv == 0, Hq / Hkv <= 32                     */
  int32_t head_dim;       /* D in {64, 128}                                         */
  int32_t ffn_dim;        /* dense SwiGLU width F; multiple of 64 (dense only)      */
  int32_t n_experts;      /* E (MoE only), 1..256                                   */
  int32_t top_k;          /* k (MoE only), 1..min(E, 16)                            */
  int32_t expert_ffn_dim; /* per-expert SwiGLU width (MoE only); multiple of 64     */
  float rms_eps;          /* RMSNorm epsilon (>= 0)                                 */
  float rope_base;        /* rotary base (> 0)                                      */
  int32_t dtype;          /* tri_dtype: storage type of every tensor of the call    */
  int32_t flags;          /* TRI_F_* bits                                           */
  int32_t mrope_section[3]; /* TRI_F_MROPE: frequencies per section (temporal,
                             height, width), each >= 0, summing to D/2
                             (TRI_ERR_SHAPE otherwise); ignored without the flag   */
} tri_layer_config;

/* Device pointers to one layer's weights, row-major [out, in], storage type.   */
typedef struct {
  const void* attn_norm; /* [H]                                                    */
  const void* w_qkv;     /* [(Hq + 2 Hkv) D, H]: q heads, then k heads, then v     */
  const void* b_qkv;     /* [(Hq + 2 Hkv) D]; required iff TRI_F_QKV_BIAS          */
  const void* w_o;       /* [H, Hq D]                                              */
  const void* mlp_norm;  /* [H]                                                    */
  const void* w_gate_up; /* dense [2F, H] (gate rows [0,F), up rows [F,2F));
                            MoE   [E, 2Fe, H] (same split per expert)             */
  const void* w_down;    /* dense [H, F]; MoE [E, H, Fe]                           */
  const void* w_router;  /* MoE [E, H]; NULL for a dense layer                     */
  const void* q_norm;    /* [D]; required iff TRI_F_QK_NORM, else ignored          */
  const void* k_norm;    /* [D]; required iff TRI_F_QK_NORM, else ignored          */
} tri_layer_weights;

/* KV cache (device, storage type).  Keys are stored after the rotary embedding.
 * Row r of a slot holds the token at position r of the sequence occupying
 * that slot.  Two layouts:
 *  - contiguous (block_table == NULL): K and V each [n_slots, Hkv, max_seq, D];
 *  - paged, the fixed-size cache blocks of the PagedAttention memory manager
 *    under the serving framework of Section II-A: K and V are pools
 *    [n_blocks, Hkv, block_size, D], and row r of slot s lives in block
 *    block_table[s * (max_seq / block_size) + r / block_size] at row
 *    r % block_size.  block_size is a multiple of 64 that divides max_seq;
 *    block_table is device int32 [n_slots, max_seq / block_size], 4-byte
 *    aligned, and may leave entries that no row of the batch uses unset.
 *    An entry outside [0, n_blocks) is never dereferenced: its rows read as
 *    zero and writes to it are dropped (the sequence's results are then
 *    unspecified).  The layer reads and writes only the blocks the batch's
 *    rows map to.                                                               */
typedef struct {
  void* k;
  void* v;
  int32_t n_slots;              /* sequences (block-table rows when paged)       */
  int32_t max_seq;              /* logical rows per sequence                     */
  const int32_t* block_table;   /* NULL: contiguous                              */
  int32_t block_size;           /* paged: rows per block; else ignored           */
  int32_t n_blocks;             /* paged: blocks in each pool; else ignored      */
} tri_kv_cache;

/* A ragged batch (one scheduler step).  Host scalars size the launches; the
 * arrays are device int32.  Sequence s owns new tokens cu_q[s] .. cu_q[s+1]-1
 * of x; its new token i is written to cache row ctx_len[s] + i of slot
 * slot[s] and attends to rows 0 .. ctx_len[s] + i.  pos[t] is the rotary
 * position of token t (normally ctx_len + i); with TRI_F_MROPE, pos holds
 * three planes, pos[k * n_tokens + t] being id k (temporal, height, width) of
 * token t (for text tokens all three normally equal ctx_len + i).  The caller guarantees
 * ctx_len[s] + q_len[s] <= max_seq for every sequence; a sequence violating it
 * is skipped on the device (no access outside the cache).                     */
typedef struct {
  int32_t n_seqs;      /* >= 0                                                     */
  int32_t n_tokens;    /* T = cu_q[n_seqs]                                         */
  int32_t max_q_len;   /* >= max_s (cu_q[s+1] - cu_q[s])                           */
  int32_t max_ctx_len; /* >= max_s ctx_len[s]; < max_seq (TRI_ERR_RANGE otherwise) */
  const int32_t* cu_q;    /* [n_seqs + 1], cu_q[0] = 0, non-decreasing             */
  const int32_t* ctx_len; /* [n_seqs]                                              */
  const int32_t* slot;    /* [n_seqs], distinct                                    */
  const int32_t* pos;     /* [n_tokens], or [3][n_tokens] with TRI_F_MROPE         */
} tri_batch;

/* Byte offsets of the layer's intermediates inside the workspace (for
 * inspection after a call; contents are valid once the stream has finished).
 * Element type of h .. act: the storage type.                                 */
typedef struct {
  size_t h;      /* [T, H]   RMSNorm(x)                                             */
  size_t q;      /* [T, Hq, D] rotated queries                                      */
  size_t attn;   /* [T, Hq D] attention output                                      */
  size_t x1;     /* [T, H]   x + attn W_o^T                                         */
  size_t h2;     /* [T, H]   RMSNorm(x1)                                            */
  size_t act;    /* dense: [T, F] SwiGLU activation silu(g)*u;
                    MoE: [T*top_k, Fe], rows in routed order                       */
  size_t perm;   /* MoE: [T*top_k] int32 routed order -> pair id t*top_k + j
                    (pairs grouped by expert, ascending pair id within an expert)   */
  size_t y;      /* MoE: [T*top_k, H] fp32 expert outputs, rows in routed order     */
  size_t total;  /* == tri_workspace_size()                                         */
} tri_workspace_map;

/* Workspace bytes needed by tri_layer_prefill / tri_layer_decode for a batch
 * with these host scalars (device arrays are not read).  For a fixed config the
 * size never decreases as n_tokens, n_seqs, max_q_len or max_ctx_len grows, so a
 * workspace sized for the largest batch serves every smaller one.              */
tri_status tri_workspace_size(const tri_layer_config* cfg, const tri_batch* batch,
                              size_t* bytes);

/* The workspace layout used for this config and batch.                        */
tri_status tri_workspace_layout(const tri_layer_config* cfg, const tri_batch* batch,
                                tri_workspace_map* map);

/* One decoder layer over a ragged batch (prefill, chunked prefill with a
 * cached prefix, decode, or any mix: the mixed step of Section III-A1).
 *  x_in      device [T, H] storage type, token activations in batch order
 *  x_out     device [T, H] storage type, layer output; must not overlap x_in
 *  route_idx device [T, top_k] int32 or NULL (MoE: chosen experts, descending
 *            logit, ties to the lower expert index)
 *  route_w   device [T, top_k] float or NULL (MoE: routing weights)
 *  workspace device, >= tri_workspace_size() bytes, 256-byte aligned
 * Cache rows ctx_len[s] .. ctx_len[s] + q_len - 1 of every sequence are
 * written; no other cache row is touched.                                      */
tri_status tri_layer_prefill(const tri_layer_config* cfg, const tri_layer_weights* w,
                             const tri_kv_cache* cache, const tri_batch* batch,
                             const void* x_in, void* x_out, int32_t* route_idx,
                             float* route_w, void* workspace, size_t workspace_bytes,
                             void* stream);

/* The decode step (every sequence has exactly one new token: n_tokens ==
 * n_seqs, max_q_len == 1), on the memory-bound path: skinny projections that
 * stream each weight once and split-KV attention.  Same arguments and
 * results as tri_layer_prefill.                                                */
tri_status tri_layer_decode(const tri_layer_config* cfg, const tri_layer_weights* w,
                            const tri_kv_cache* cache, const tri_batch* batch,
                            const void* x_in, void* x_out, int32_t* route_idx,
                            float* route_w, void* workspace, size_t workspace_bytes,
                            void* stream);

/* The decode step of tri_layer_decode without a workspace argument, for
 * callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation).  The scratch lives
 * in a fixed device array of TRI_NOALLOC_SCRATCH_BYTES inside the library,
 * one per GPU, held until the process ends; the call itself allocates
 * nothing (no hipMalloc, no allocating library routine, no profiling events).
 * Same arguments and results as tri_layer_decode, minus the workspace.
 * Errors: those of tri_layer_decode; TRI_ERR_SCRATCH, before any launch, when
 * tri_workspace_size() of the batch exceeds TRI_NOALLOC_SCRATCH_BYTES (64 MiB:
 * the 7B-class decode at batch 64 and KV 4096 needs 34 MiB, the 128-expert
 * MoE decode at batch 128 and KV 2048 60 MiB); TRI_ERR_HIP if the scratch's
 * device address cannot be obtained.  Calls on one GPU share its scratch:
 * calls that overlap in time on one GPU (several streams or host threads)
 * race and must be serialised by the caller.                                */
#define TRI_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
tri_status tri_layer_decode_noalloc(const tri_layer_config* cfg, const tri_layer_weights* w,
                                    const tri_kv_cache* cache, const tri_batch* batch,
                                    const void* x_in, void* x_out, int32_t* route_idx,
                                    float* route_w, void* stream);

/* KV-cache append (the cache write of Section II-A's decode loop, done inside
 * the layer calls as well): for every new token t of sequence s,
 *   k[slot[s]][h][ctx_len[s] + i][:] = k_new[t][h][:]   (same for v).
 *  k_new, v_new  device [T, Hkv, D], storage type.                              */
tri_status tri_kvcache_append(const tri_layer_config* cfg, const tri_kv_cache* cache,
                              const tri_batch* batch, const void* k_new, const void* v_new,
                              void* stream);

/* ---- operators of a long context: rotary positions of other models' kinds, a
 * key/value cache of one byte per value, attention over it and its eviction.
 * They take the pieces that the layer calls fuse (the serving loop around the
 * Thinker, Section II-A, calls them between its own projections); conventions
 * and errors as above.  At most 65535 sequences and heads a call
 * (TRI_ERR_RANGE): they are extents of the launch grid.                       */

/* Rotary positions.  Of every head's head_dim values the first rotary_dim are
 * rotated in pairs, the rest copied:
 *   (a, b) -> m (a cos t - b sin t, b cos t + a sin t),  t = pos * f_i
 * for pair i < rotary_dim / 2, in double precision up to the reduced angle.
 * Pairs: TRI_ROPE_HALF (i, i + rotary_dim/2), TRI_ROPE_INTERLEAVED (2i, 2i+1).
 * Frequencies, w_i = base^(-2i / rotary_dim):
 *  TRI_ROPE_PLAIN   f = w
 *  TRI_ROPE_LINEAR  f = w / factor (positions interpolated)
 *  TRI_ROPE_BASE    base scaled: f = (base factor^(r/(r-2)))^(-2i/r), r = rotary_dim
 *                   (as PLAIN for r = 2)
 *  TRI_ROPE_TURNS   by the turns n = original_len w / (2 pi) that a pair makes over
 *                   the context it was trained on: t = clamp((n - low) / (high -
 *                   low), 0, 1), f = w (t + (1 - t) / factor)
 *  TRI_ROPE_INDEX   the same blend, linear in the index between the pairs that
 *                   make `high` and `low` turns: at(n) = r ln(original_len / (2 pi
 *                   n)) / (2 ln base), lo = max(floor(at(high)), 0), hi =
 *                   min(ceil(at(low)), r - 1), u = clamp((i - lo) / max(hi - lo,
 *                   0.001), 0, 1), f = w (1 - u) + (w / factor) u
 * magnitude m scales cos and sin (1 for none).                                 */
typedef enum { TRI_ROPE_HALF = 0, TRI_ROPE_INTERLEAVED = 1 } tri_rope_layout;
typedef enum {
  TRI_ROPE_PLAIN = 0,
  TRI_ROPE_LINEAR = 1,
  TRI_ROPE_BASE = 2,
  TRI_ROPE_TURNS = 3,
  TRI_ROPE_INDEX = 4
} tri_rope_scaling;
typedef struct {
  int32_t head_dim;     /* 2 .. 256, even                                         */
  int32_t rotary_dim;   /* 2 .. head_dim, even                                    */
  int32_t layout;       /* tri_rope_layout                                        */
  int32_t scaling;      /* tri_rope_scaling                                       */
  int32_t original_len; /* TURNS, INDEX: the trained context (> 0)                */
  float base;           /* > 0; INDEX: > 1                                        */
  float factor;         /* > 0 (every kind but PLAIN)                             */
  float low, high;      /* TURNS, INDEX: 0 < low < high                           */
  float magnitude;      /* finite                                                 */
} tri_rope_config;

/* The configuration as the kernels take it, formed once and kept by the caller: every
 * pair's turns per position, f_i / (2 pi).  Host only.  Errors: TRI_ERR_NULL,
 * TRI_ERR_UNSUPPORTED (head_dim, layout, scaling), TRI_ERR_SHAPE (rotary_dim),
 * TRI_ERR_RANGE (the numbers).                                                    */
#define TRI_ROPE_MAX_PAIRS 128
typedef struct {
  int32_t head_dim, rotary_dim, layout;
  float magnitude;
  double turns[TRI_ROPE_MAX_PAIRS];
} tri_rope_table;
tri_status tri_rope_table_make(const tri_rope_config* cfg, tri_rope_table* table);

/* y = x rotated.  x and y: device [n_tokens][n_heads][head_dim] of dtype (bf16 or
 * float32), tokens x_stride and y_stride elements apart (>= n_heads * head_dim:
 * the q and k heads of fused projection rows are one call); aligned to an
 * element, fastest where addresses and strides are multiples of 16 bytes and
 * rotary_dim of 32 bytes.  y may be x itself (same stride); any other overlap is
 * TRI_ERR_ALIAS.  pos: device int32 [n_tokens], any sign.                       */
tri_status tri_rope(const tri_rope_table* table, const void* x, int64_t x_stride, void* y,
                    int64_t y_stride, const int32_t* pos, int32_t n_tokens, int32_t n_heads,
                    int32_t dtype, void* stream);

/* 8-bit KV cache (device).  Rows, slots and pages as in tri_kv_cache; the panel P
 * of a row is its slot (contiguous) or its page, of R = max_seq or block_size
 * rows.  A value is code * scale with one scale per head and scale_rows
 * consecutive rows of a panel (a scale block):
 *  TRI_KV8_INT8  code an 8-bit integer in [-127, 127]
 *  TRI_KV8_E4M3  code an 8-bit float of 4 exponent and 3 mantissa bits, at most 448
 * A scale is a power of two, 2^-100 or more, so that codes move to a larger one by a
 * shift.  A scale of NaN marks a block into which a value that is not finite was
 * appended: every value of it is NaN, and so are the output and the weights of a token
 * that sees one of the block's rows, for the head's queries.  max_seq <= 2^23
 * (TRI_ERR_RANGE).  n_tokens may exceed cu_q[n_seqs]: tokens behind the last sequence
 * are neither read nor written by the calls below that take a batch (but the layer's).
 * A page that two sequences of a batch hold is read by both; no row of it may be
 * appended or moved to, and `mass` must be NULL for the attention (its sums would race).
 * The library reads n_q_heads, n_kv_heads, head_dim (64 or 128) and dtype
 * (TRI_BF16) of the tri_layer_config.                                           */
typedef enum { TRI_KV8_INT8 = 0, TRI_KV8_E4M3 = 1 } tri_kv8_format;
typedef struct {
  void* k;                      /* codes [P, Hkv, R, D], one byte each, 16-byte
                                   aligned                                        */
  void* v;
  float* k_scale;               /* [P, Hkv, ceil(R / scale_rows)]                 */
  float* v_scale;
  float* mass;                  /* [P, Hkv, R] accumulated attention weight of each
                                   row, or NULL                                   */
  int32_t* stamp;               /* [P, Hkv, R] position of the token in each row, or
                                   NULL                                           */
  int32_t n_slots;
  int32_t max_seq;
  const int32_t* block_table;   /* as in tri_kv_cache                             */
  int32_t block_size;
  int32_t n_blocks;
  int32_t format;               /* tri_kv8_format                                 */
  int32_t scale_rows;           /* 32, 64 or 128; paged: divides block_size       */
} tri_kv8_cache;

/* Append to an 8-bit cache: rows ctx_len[s] + i of slot[s] take the batch's new keys
 * and values (rotated already).  Per head and scale block touched the scale becomes
 * the least power of two s >= 2^-100 with max |x| <= 127 s (448 s) over the new rows,
 * or the block's own scale where rows before ctx_len are held in it and that is
 * larger; where it grew, the held codes are rounded once more (to nearest even, as
 * the new ones).  The roundings of a value that was appended early add up to less
 * than one step of the final scale.  Writes mass 0 and stamp pos[t] where the cache
 * has them (pos[t] is needed then only; with more planes, the first).
 *  k_new, v_new  device bf16 [T][Hkv][D], tokens `stride` elements apart (a multiple
 *                of 8, >= Hkv D), 16-byte aligned
 * A sequence with a slot out of range or rows past max_seq is skipped.           */
tri_status tri_kv8_append(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                          const tri_batch* batch, const void* k_new, const void* v_new,
                          int64_t stride, void* stream);

/* Causal grouped-query attention over an 8-bit cache: token i of sequence s attends
 * to rows 0 .. ctx_len[s] + i of its slot, which hold the batch's own rows already
 * (tri_kv8_append first).  Any mix of chunks and single tokens.
 *  q    device bf16 [T][Hq][D], tokens q_stride elements apart (a multiple of 8,
 *       Hq D .. 2^22), 16-byte aligned;  Hq / Hkv <= 32, T Hq < 2^31 - 2^23
 *  out  device bf16 [T][Hq][D]; must not overlap q
 * Where the cache has `mass`, mass[row] += the row's attention weights summed over
 * the KV head's query heads and the new tokens of the sequence (in one fixed order:
 * the same inputs give the same sums).  Codes are exact in the products; scores,
 * running maximum, sums and outputs are float32.  For the product with the values a
 * weight times its value's scale is rounded to 11 bits, or, where it is below 2^-14 of
 * the token's largest such product, to a multiple of at most 2^-24 of that: a channel
 * that only rows of far smaller value scales fill has as many bits fewer.  A weight
 * counts in its output's denominator down to 2^(d - 126) of the largest, where the value
 * scales of the rows that the token sees differ by up to 2^d (zeros have the scale
 * 2^-100: d < 102, so 2^-24, while no value beside them passes 2^8).  Tokens of a skipped
 * sequence (as in the append) are left as they were.
 * workspace: device, 256-byte aligned, of tri_kv8_attention_workspace_size bytes
 * (the cache's and the batch's host fields are read; it never shrinks as n_tokens, n_seqs,
 * max_ctx_len or max_q_len grows).                                               */
tri_status tri_kv8_attention_workspace_size(const tri_layer_config* cfg,
                                            const tri_kv8_cache* cache, const tri_batch* batch,
                                            size_t* bytes);
tri_status tri_kv8_attention(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                             const tri_batch* batch, const void* q, int64_t q_stride, void* out,
                             void* workspace, size_t workspace_bytes, void* stream);

/* The decoder layer over an 8-bit cache: tri_layer_prefill and tri_layer_decode with the
 * cache written by tri_kv8_append and attended to by tri_kv8_attention (mass included)
 * in place of the bf16 cache; every other stage is the same.  cfg->dtype is TRI_BF16.
 * The per-stage timers count the append as kv_append and all kernels of the attention,
 * weight sums included, as attn_decode (tri_layer_decode_kv8) or attn_prefill;
 * tri_layer_work describes the layer on the bf16 cache, with its bytes, alone.
 * The attention sees the step's own rows as the cache holds them.  workspace: of
 * tri_workspace_size_kv8 bytes (which never decrease, as those of tri_workspace_size). */
tri_status tri_workspace_size_kv8(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                                  const tri_batch* batch, size_t* bytes);
tri_status tri_layer_prefill_kv8(const tri_layer_config* cfg, const tri_layer_weights* w,
                                 const tri_kv8_cache* cache, const tri_batch* batch,
                                 const void* x_in, void* x_out, int32_t* route_idx,
                                 float* route_w, void* workspace, size_t workspace_bytes,
                                 void* stream);
tri_status tri_layer_decode_kv8(const tri_layer_config* cfg, const tri_layer_weights* w,
                                const tri_kv8_cache* cache, const tri_batch* batch,
                                const void* x_in, void* x_out, int32_t* route_idx,
                                float* route_w, void* workspace, size_t workspace_bytes,
                                void* stream);

/* Eviction, first half: which rows stay.  Of the n = ctx_len[s] + q_len rows of a
 * sequence's slot, every KV head keeps `budget` (all where n <= budget): rows with
 * stamp < n_first or stamp > newest - n_recent (newest: the largest stamp of the
 * head's rows; row numbers stand in for stamps where the cache has none) before all
 * others, those by descending mass, NaN last, ties to the lower row.  cache->mass is
 * required.  A kept row below budget stays where it is; kept rows at or past budget
 * take, in order, the places of evicted ones below it:
 *  plan     device int32 [n_seqs][Hkv][budget]: row r is to hold what is in row
 *           plan[r] (r itself where nothing changes, -1 past the rows held)
 *  new_len  device int32 [n_seqs]: min(n, budget); or NULL
 * budget: a multiple of scale_rows, <= max_seq; n_first, n_recent >= 0 with n_first +
 * n_recent <= budget.  The rows kept are no longer in order of position: the stamps
 * tell it, and keys are cached rotated, so attention does not mind.  A skipped
 * sequence (also one whose lengths exceed the batch's host fields) gets -1 throughout
 * and new_len 0.
 * workspace: device, 256-byte aligned, of tri_kv8_select_workspace_size bytes (0, and NULL
 * will do, unless max_ctx_len + max_q_len exceeds 16384 rows).                     */
tri_status tri_kv8_select_workspace_size(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                                         const tri_batch* batch, int32_t budget, size_t* bytes);
tri_status tri_kv8_select(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                          const tri_batch* batch, int32_t budget, int32_t n_first,
                          int32_t n_recent, int32_t* plan, int32_t* new_len, void* workspace,
                          size_t workspace_bytes, void* stream);

/* Eviction, second half: row r of every KV head takes what is in row plan[r] (codes,
 * mass, stamp), r < budget.  A scale block into which rows move takes the largest of
 * its rows' scales; codes are shifted to it.  Rows at or past budget are left as they
 * were, and a later append starts at new_len.  `batch` gives n_seqs and slots (as in
 * the select).  An entry below 0 or at or past max_seq is left out: its row keeps what it
 * holds, and counts among the block's rows where others move into it.  An entry r' != r
 * must be >= budget.  A page shared between sequences must not be moved into.     */
tri_status tri_kv8_move(const tri_layer_config* cfg, const tri_kv8_cache* cache,
                        const tri_batch* batch, const int32_t* plan, int32_t budget,
                        void* stream);

/* Plain projection C = A B^T on the layer's GEMM kernels: the matrix
 * multiply of the Thinker's projections (Section II-A) and the synthetic
 * kernel of the paper's roofline benchmark over arithmetic intensity
 * (Section II-C, frequency-locked roofline benchmarking).
 *  A [M, K], B [N, K] (the nn.Linear weight layout), C [M, N]: bf16,
 *    row-major, device memory, 16-byte aligned; fp32 accumulation, C rounded
 *    to nearest even.  M, N, K >= 1, K a multiple of 64, N a multiple of 4,
 *    A and B each under 2 GiB; C overlaps neither operand.
 *  workspace: device scratch of tri_linear_workspace_size bytes (split
 *    partials; 256-byte aligned), or NULL when that size is 0.
 *  stream: hipStream_t (NULL = default stream).
 * Errors (before any launch): TRI_ERR_NULL, TRI_ERR_SHAPE, TRI_ERR_RANGE,
 * TRI_ERR_ALIGN, TRI_ERR_WORKSPACE, TRI_ERR_ALIAS; TRI_ERR_HIP if a launch
 * fails. */
tri_status tri_linear_workspace_size(int32_t M, int32_t N, int32_t K, size_t* bytes);
tri_status tri_linear(const void* A, const void* B, void* C, int32_t M, int32_t N, int32_t K,
                      void* workspace, size_t workspace_bytes, void* stream);

/* MoE routing alone (test hook for bit-exact routing): logits = h2 W_r^T in
 * float32 (one fixed summation order per logit), softmax over all experts,
 * top_k by logit (descending, ties to the lower index), weights p[idx]
 * (renormalised if TRI_F_MOE_RENORM).  Inside the layer the router reads h2
 * in the storage type (bf16 widened exactly to float32, or float32).
 *  h2        device [n_tokens, H] float32
 *  w_router  device [E, H] storage type
 *  idx, w    device [n_tokens, top_k] int32 / float32                          */
tri_status tri_moe_route(const tri_layer_config* cfg, const float* h2, const void* w_router,
                         int32_t n_tokens, int32_t* idx, float* w, void* stream);

/* Per-stage timing for benchmarks.  While enabled, the layer entry points
 * record a HIP event pair on the caller's stream around every stage (the
 * stage names are listed in tri_profile.name).  tri_profile_enable(1) resets
 * the counters; tri_profile_read waits for the recorded events and returns
 * launches and total milliseconds per stage.  Not thread-safe with
 * concurrent layer calls from several host threads.                          */
#define TRI_MAX_STAGES 16
typedef struct {
  int32_t n_stages;
  const char* name[TRI_MAX_STAGES];
  int32_t launches[TRI_MAX_STAGES];
  double total_ms[TRI_MAX_STAGES];
} tri_profile;

tri_status tri_profile_enable(int32_t on);
tri_status tri_profile_read(tri_profile* out);

/* Algorithmic work of one layer call, stage by stage: the per-kernel
 * arithmetic intensity from which Section III-C forms the time-weighted
 * intensity of a phase (Eq. 5).  Index i and name[i] are the stage of
 * tri_profile with the same index.  The counts follow the operations'
 * definitions, not the kernels' internals:
 *  flops  2 per multiply-add of every matrix product (the projections, the
 *         two attention products over the causally visible keys, the router,
 *         the experts); a stage without a product counts its multiply-adds
 *         (RMSNorm 4 per element, split merge 2 per partial element, MoE
 *         combine 2 per routed element).  Rotary, softmax and SwiGLU
 *         transcendentals are not counted.
 *  bytes  compulsory HBM traffic in the storage type: every input a stage
 *         reads and every output it writes, once (weights, activations, the
 *         K/V rows attended, once per KV head, cache rows written, the
 *         split-KV partials passed from attn_decode to attn_combine).
 *         On-chip re-reads are not counted.  (The model follows the bf16
 *         launch sequence; the fp32 mode's operand planes are not counted.)
 * Arguments (host memory):
 *  decode         1 for tri_layer_decode's launch sequence, 0 for
 *                 tri_layer_prefill's
 *  q_len, ctx_len [n_seqs] new tokens and cached prefix of each sequence
 *  expert_rows    MoE: [n_experts] routed rows per expert (summing to
 *                 n_tokens * top_k), or NULL, in which case min(E, T * top_k)
 *                 experts are taken as touched
 *  out            every stage filled; runs[i] = 1 iff the call launches stage i
 * Errors: TRI_ERR_NULL; the config's status; TRI_ERR_SHAPE for a negative
 * length, a decode sequence with q_len != 1 or expert_rows of the wrong sum.  */
typedef struct {
  int32_t n_stages;
  const char* name[TRI_MAX_STAGES];
  int32_t runs[TRI_MAX_STAGES];
  double flops[TRI_MAX_STAGES];
  double bytes[TRI_MAX_STAGES];
} tri_work;

tri_status tri_layer_work(const tri_layer_config* cfg, int32_t decode, int32_t n_seqs,
                          const int32_t* q_len, const int32_t* ctx_len,
                          const int32_t* expert_rows, tri_work* out);

/* Time-weighted arithmetic intensity of a phase (Section III-C, Eq. 5):
 *   ai = sum_i d_i (flops_i / bytes_i) / sum_i d_i
 * over the stages i with work->runs[i] set, d_i = prof->total_ms[i]; stages
 * with d_i = 0, or with no work (flops and bytes both 0), drop out.  The work of several calls may be summed stage by
 * stage first; a stage then stands for all its launches.  Host only.
 * Errors: TRI_ERR_NULL; TRI_ERR_SHAPE if the stage counts differ or no stage
 * has time; TRI_ERR_RANGE for a negative time or a timed stage with no bytes. */
tri_status tri_phase_intensity(const tri_work* work, const tri_profile* prof, double* ai);

/* Static description of a status code.                                         */
const char* tri_status_string(tri_status s);

/* Library version: major * 10000 + minor * 100 + patch.                         */
int32_t tri_version(void);

#ifdef __cplusplus
}
#endif
#endif /* TRI_H */
