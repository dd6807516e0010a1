/*
 * qmla — low-bit MLA decode attention on one GB300 (sm_103a).
 *
 * C ABI of the library libqmla.so. It implements the decode hot path of
 * QuantMLA (arXiv 2609.36760): Multi-head Latent Attention read directly from a
 * jointly low-bit paged cache, with unpacking and dequantisation fused into the
 * attention (Sec. 3.3; App. C.5).
 *
 *   qmla_quant_append   quantise + pack new tokens into the paged cache
 *                       (App. C.4 quantiser; App. C.5 "cache update": content- and
 *                       RoPE-cache quantisation, integer packing, slot-mapped
 *                       page insertion)
 *   qmla_mla_decode     split-KV decode attention over the packed cache, plus the
 *                       split-result combination (Eq. mla_compact; App. C.5
 *                       "global attention normalization")
 *   *_protected         the same with sink4/local128 BF16 protection (App. C.5)
 *   *_c4r4              the same over the paper's own 20,480-byte INT4 page
 *   qmla_mla_decode_multi  several query tokens per sequence under the causal mask
 *   qmla_mla_decode_ex  every decode variant from one descriptor, with optional
 *                       per-call events around the main kernel
 *   qmla_rope_append    the cache writer for rows as the projections leave them: the
 *                       latent normalised and the RoPE key rotated on the way
 *   qmla_rope_query     rotates the RoPE part of queries
 *   qmla_cache_read     cached tokens back as bf16 rows
 *   qmla_mla_prefill    attention of ragged prompts over expanded keys and values
 *   qmla_mla_decode_tree  decode attention of a tree of drafted tokens
 *   qmla_tree_verify    verification of such a tree against the target's probabilities
 *   qmla_cache_keep     the accepted tokens' cache rows moved together, the new lengths
 *
 * Conventions for every call
 * --------------------------
 * - Pointers named *_dev are device pointers owned by the caller; the library
 *   never allocates, frees or keeps them. Host pointers are marked _host.
 * - Every call that launches work is asynchronous on `stream` (a cudaStream_t;
 *   NULL = legacy default stream) and returns a status code immediately.
 *   Arguments are validated on the host before anything is launched; an invalid
 *   argument launches nothing.
 * - Problems only visible on the device (a bad block id, a position beyond the
 *   block table, a pipeline wait that ran out) are OR-ed into the caller's
 *   32-bit error word `dev_err_dev` (QMLA_DEVERR_*), unless it is NULL. The offending
 *   access is skipped; no call traps or aborts. Read the word with qmla_read_dev_err.
 * - bf16 / fp16 tensors are passed as uint16_t bit patterns.
 * - Plain launches on one stream keep stream order, whatever memory they share. Kernels
 *   that a caller launches with programmatic stream serialisation have to know two things.
 *   The cache writers let their dependents start at once (griddepcontrol
 *   .launch_dependents), so such a kernel right behind a writer runs beside it: it must
 *   execute griddepcontrol.wait, even if it uses nothing of the cache, for a decode
 *   behind it waits for that kernel alone. And a decode's first kernel is such a launch
 *   itself: it reads q_latent, q_pe, block_table and seq_lens (and of a tree parents and
 *   tree_lens) before it waits, so a kernel right before the decode must not let its
 *   dependents start before it has written those. (Everything else a decode reads, and all that it writes but bits of the
 *   error word, comes after the wait.)
 *
 * Cache format (this library's own 64-token block, little-endian)
 * ----------------------------------------------------------------
 * Each token is quantised in 9 groups of 64 coordinates: groups 0..7 are the
 * content latent c_KV channels [64g, 64g+64) at c_bits (4 or 2), group 8 is the
 * decoupled RoPE key k_pe (d_r = 64) at 4 bits. Per group, per token
 * (App. C.4, with the fp16 staging fixed by this library):
 *     d = RN_f32(x_max - x_min);  s = RN_f16(RN_f32(max(d, 1e-8) / m)), m = 2^b - 1
 *     (s = 2^-24 if that underflows to 0, 65504 if it overflows)
 *     z = clip(rne(-x_min / s), 0, m);  q = clip(rne(x / s + z), 0, m)
 * Codes are packed low bits first: INT4 byte j = q[2j] | q[2j+1] << 4, INT2
 * byte j = q[4j] | q[4j+1] << 2 | q[4j+2] << 4 | q[4j+3] << 6.
 * A block of 64 token slots, cb = 64 * c_bits / 8:
 *     [0, 8*64*cb)                 content codes   [group 8][slot 64][cb bytes]
 *     [8*64*cb, +2048)             RoPE-key codes  [slot 64][32 bytes]
 *     [8*64*cb + 2048, +2304)      scale/zero      [group 9][slot 64][fp16 s, fp16 z]
 * INT4 content: 20736 bytes per block; INT2 content: 12544 bytes per block.
 * Token at position p of sequence b lives in block block_table[b*max_blocks + p/64],
 * slot p % 64.
 *
 * The BF16 comparison cache (qmla_bf16_append / qmla_mla_decode_bf16cache)
 * stores each token as 576 bf16 (latent then k_pe): blocks of 64 x 1152 bytes,
 * the paper's BF16 page (App. C.5, storage layout).
 */
#ifndef QMLA_H_
#define QMLA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* qmla_stream_t; /* same type as cudaStream_t */

/* Status codes returned by every call. */
enum qmla_status {
  QMLA_OK = 0,
  QMLA_ERR_INVALID_ARG = 1,          /* null pointer, bad size, bad bit width, misalignment */
  QMLA_ERR_UNSUPPORTED = 2,          /* no sm_103a device, or a shape outside the supported range */
  QMLA_ERR_WORKSPACE_TOO_SMALL = 3,  /* decode workspace smaller than qmla_decode_workspace_bytes */
  QMLA_ERR_CUDA = 4                  /* a CUDA runtime call failed; see qmla_last_cuda_error */
};

/* Bits of the device error word. */
enum qmla_device_error {
  QMLA_DEVERR_BAD_BLOCK = 1u,     /* a block-table entry outside [0, num_blocks) was needed */
  QMLA_DEVERR_BAD_POSITION = 2u,  /* a position or sequence length < 0 or beyond max_blocks*64 */
  QMLA_DEVERR_BAD_SEQ = 4u,       /* an append sequence id outside [0, num_seqs) */
  QMLA_DEVERR_TIMEOUT = 8u,       /* an on-chip pipeline wait ran out; that kernel left early */
  QMLA_DEVERR_BAD_OFFSETS = 16u,  /* a prompt's offsets decrease or leave the rows given; it was left out */
  QMLA_DEVERR_BAD_TREE = 32u,     /* a tree's node count, parent, token or path is not one (see the call) */
  QMLA_DEVERR_BAD_PROBS = 64u     /* probabilities to draw a token from have no positive, finite sum */
};

/* Cache kinds besides the content bit widths 4 and 2: the paper's page, the BF16 cache. */
#define QMLA_CACHE_C4R4 5
#define QMLA_CACHE_BF16 16

/* Most query tokens per sequence qmla_mla_decode_multi accepts. */
#define QMLA_MAX_Q_TOKENS 8

/* Most nodes of a tree of drafted tokens (qmla_mla_decode_tree and the calls beside it). */
#define QMLA_MAX_TREE_NODES 64

/* Types of probabilities (qmla_tree_verify). */
#define QMLA_PROBS_F32 0
#define QMLA_PROBS_BF16 1

/* Bytes of one 64-token block for content bit width c_bits (4 -> 20736,
 * 2 -> 12544); 0 if c_bits is not supported. */
size_t qmla_block_bytes(int c_bits);

/* Bytes of one 64-token BF16 comparison block (73728). */
size_t qmla_bf16_block_bytes(void);

/*
 * Quantise n new tokens and insert them into the packed cache
 * (App. C.4 quantiser; App. C.5 fused writer without the BF16 protection
 * buffers).
 *
 *   pool_dev        [num_blocks * qmla_block_bytes(c_bits)] bytes, 32-byte aligned
 *                   (every call that takes a pool requires this: the decode
 *                   reads a token's 32-byte code row in one request);
 *                   only the slots of the given tokens are written
 *   c_bits          content bit width, 4 or 2 (the RoPE key is always 4-bit)
 *   latent_dev      [n, 512] bf16, row-major, 4-byte aligned: content latent c_KV
 *   k_pe_dev        [n, 64]  bf16, row-major, 4-byte aligned: decoupled RoPE key
 *   seq_ids_dev     [n] int32 sequence of each token, or NULL meaning token i
 *                   belongs to sequence i
 *   positions_dev   [n] int32 zero-based position of each token in its sequence
 *   block_table_dev [num_seqs, max_blocks] int32 physical block ids
 *   dev_err_dev     device error word (see above)
 * Two tokens with the same (sequence, position) in one call race; the result
 * is one of them. n == 0 is a no-op.
 */
int qmla_quant_append(void* pool_dev, int c_bits, int num_blocks, const uint16_t* latent_dev,
                      const uint16_t* k_pe_dev, const int32_t* seq_ids_dev,
                      const int32_t* positions_dev, int n, const int32_t* block_table_dev,
                      int num_seqs, int max_blocks, uint32_t* dev_err_dev, qmla_stream_t stream);

/* Same insertion into the BF16 comparison cache (blocks of qmla_bf16_block_bytes()):
 * the 576 bf16 values of each token are copied unchanged. */
int qmla_bf16_append(void* pool_dev, int num_blocks, const uint16_t* latent_dev,
                     const uint16_t* k_pe_dev, const int32_t* seq_ids_dev,
                     const int32_t* positions_dev, int n, const int32_t* block_table_dev,
                     int num_seqs, int max_blocks, uint32_t* dev_err_dev, qmla_stream_t stream);

/*
 * Sink4/local128 BF16 protection (App. C.5, "BF16 protection and cache
 * lifecycle"). For a request of L cached tokens the protected positions are
 *     P_L = {0, ..., min(4, L) - 1}  U  {max(0, L - 128), ..., L - 1};
 * attention reads their pre-quantisation bf16 content and RoPE-key values and
 * reads every other position from the packed cache, all under one softmax. A
 * packed copy is written for every token, protected or not, so a token leaving
 * the recent window switches to its packed copy with no further work.
 *
 * Protection buffer (caller-owned, one per request): [num_seqs][132][576] bf16,
 * qmla_protect_bytes_per_seq() = 132 * 576 * 2 = 152064 bytes per request (the
 * paper's figure), 16-byte aligned. A row holds a token's 512 latent values
 * then its 64 RoPE-key values; rows 0..3 hold sink positions 0..3, row
 * 4 + (p mod 128) holds recent position p. The buffer needs no initialisation:
 * a row is only read once the writer has filled it.
 */
size_t qmla_protect_bytes_per_seq(void);

/* qmla_quant_append plus the protection rows: token i (request s = seq_ids[i],
 * position p) is also copied into row p when p < 4 and into row 4 + (p mod 128)
 * when p >= seq_lens_dev[s] - 128, where seq_lens_dev [num_seqs] int32 holds the
 * requests' lengths after this call. So one call may carry a whole prefill:
 * positions older than the recent window never reach the ring, and no two
 * positions of one call share a row. latent_dev, k_pe_dev and prot_dev must be
 * 16-byte aligned; the other arguments and errors are those of qmla_quant_append. */
int qmla_quant_append_protected(void* pool_dev, int c_bits, int num_blocks, const uint16_t* latent_dev,
                                const uint16_t* k_pe_dev, const int32_t* seq_ids_dev,
                                const int32_t* positions_dev, int n, const int32_t* block_table_dev,
                                int num_seqs, int max_blocks, const int32_t* seq_lens_dev, void* prot_dev,
                                uint32_t* dev_err_dev, qmla_stream_t stream);

/* Workspace bytes qmla_mla_decode needs for this batch and head count on the
 * current device (split plan + split partials). For qmla_mla_decode_multi pass
 * heads = q_tokens x heads (up to 128 x QMLA_MAX_Q_TOKENS); 0 for bad arguments. */
size_t qmla_decode_workspace_bytes(int batch, int heads);

/*
 * Decode attention of one query token per sequence over the packed cache
 * (Eq. mla_compact with the dequantised cache s (q - z), App. C.4):
 *     S[b,h,t] = softmax_scale * (q_latent[b,h,:] . C_hat[b,t,:] + q_pe[b,h,:] . K_hat[b,t,:])
 *     out[b,h,:] = sum_t softmax_t(S[b,h,:]) C_hat[b,t,:]      (t < seq_lens[b])
 *     lse[b,h]   = log sum_t exp(S[b,h,t])
 * The caller applies the value/output up-projection. Sequences are split
 * across the GPU's SMs and the split results merged with the App. C.5 rule.
 *
 *   pool_dev        packed cache written by qmla_quant_append with the same c_bits,
 *                   32-byte aligned
 *   q_latent_dev    [batch, heads, 512] bf16 absorbed content query, 16-byte aligned
 *   q_pe_dev        [batch, heads, 64]  bf16 RoPE query, 16-byte aligned
 *   heads           1..128
 *   block_table_dev [batch, max_blocks] int32
 *   seq_lens_dev    [batch] int32 tokens to attend to (including any just appended)
 *   softmax_scale   tau, e.g. 1/sqrt(192)
 *   out_dev         [batch, heads, 512] float32
 *   lse_dev         [batch, heads] float32 natural-log LSE, or NULL
 *   workspace_dev   >= qmla_decode_workspace_bytes(batch, heads) bytes, 256-byte aligned;
 *                   contents need no initialisation and are scratch after the call
 * A sequence with seq_lens == 0 gets out = 0 and lse = -inf.
 *
 * With 65..128 query rows per sequence (193..256, ...: an even number of 64-row groups)
 * longer contexts run on pairs of CTAs and shorter ones on single CTAs. The lengths are on
 * the device, so the choice goes by the longest sequence that block_table has room for,
 * max_blocks x 64: with a table much wider than its sequences a short decode takes up to
 * 14% longer than with one cut to what they need (INT2, 16 x 2,000 tokens, 128 heads, a
 * table for 128K: 43.6 against 38.1 us). Cut the table, or pass max_len to
 * qmla_mla_decode_ex. Results agree to fp32 rounding (2-norm 2e-5) either way, a raised
 * softmax reference apart (2^-11).
 */
int qmla_mla_decode(const void* pool_dev, int c_bits, int num_blocks, const uint16_t* q_latent_dev,
                    const uint16_t* q_pe_dev, int batch, int heads, const int32_t* block_table_dev,
                    int max_blocks, const int32_t* seq_lens_dev, float softmax_scale,
                    float* out_dev, float* lse_dev, void* workspace_dev, size_t workspace_bytes,
                    uint32_t* dev_err_dev, qmla_stream_t stream);

/* qmla_mla_decode under sink4/local128 protection: for request b with
 * L = seq_lens_dev[b], positions in P_L read row p (p < 4) or row 4 + (p mod 128)
 * of prot_dev[b] (rounded to fp16 like the BF16 cache path), every other
 * position the packed cache; one global softmax over all L positions. The
 * buffer must hold every protected position (qmla_quant_append_protected with
 * the same lengths leaves it so). prot_dev 16-byte aligned, non-null; outputs,
 * workspace and errors as qmla_mla_decode. */
int qmla_mla_decode_protected(const void* pool_dev, int c_bits, int num_blocks, const uint16_t* q_latent_dev,
                              const uint16_t* q_pe_dev, int batch, int heads, const int32_t* block_table_dev,
                              int max_blocks, const int32_t* seq_lens_dev, const void* prot_dev,
                              float softmax_scale, float* out_dev, float* lse_dev, void* workspace_dev,
                              size_t workspace_bytes, uint32_t* dev_err_dev, qmla_stream_t stream);

/* Decode with q_tokens query tokens per sequence (multi-token prediction,
 * speculative verification): Eq. mla_compact with its additive causal mask.
 * For sequence b with L = seq_lens_dev[b] cached tokens (the q_tokens new ones
 * included, written by the append beforehand), query token t sits at position
 * L - q_tokens + t and attends to positions [0, L - q_tokens + t]:
 *     S[b,t,h,p] = softmax_scale * (q_latent[b,t,h,:] . C_hat[b,p,:] + q_pe[b,t,h,:] . K_hat[b,p,:]),
 *                  p <= L - q_tokens + t
 *     out[b,t,h,:] = sum_p softmax_p(S[b,t,h,:]) C_hat[b,p,:];  lse[b,t,h] = log sum_p exp(S[b,t,h,p])
 * A query token with no admissible position (L - q_tokens + t < 0) gets out = 0,
 * lse = -inf. One pass over each sequence's cache serves all its query tokens:
 * the kernel treats the q_tokens x heads (token, head) pairs as heads.
 *
 *   q_latent_dev    [batch, q_tokens, heads, 512] bf16, 16-byte aligned
 *   q_pe_dev        [batch, q_tokens, heads, 64]  bf16, 16-byte aligned
 *   q_tokens        1 .. QMLA_MAX_Q_TOKENS; heads 1..128 per token
 *   prot_dev        NULL, or the sink4/local128 protection buffer (as
 *                   qmla_mla_decode_protected; P_L from the full length L)
 *   out_dev         [batch, q_tokens, heads, 512] float32
 *   lse_dev         [batch, q_tokens, heads] float32, or NULL
 *   workspace_dev   >= qmla_decode_workspace_bytes(batch, q_tokens * heads)
 * Other arguments, ownership and errors as qmla_mla_decode; q_tokens = 1 is
 * qmla_mla_decode. */
int qmla_mla_decode_multi(const void* pool_dev, int c_bits, int num_blocks, const uint16_t* q_latent_dev,
                          const uint16_t* q_pe_dev, int batch, int q_tokens, int heads,
                          const int32_t* block_table_dev, int max_blocks, const int32_t* seq_lens_dev,
                          const void* prot_dev, float softmax_scale, float* out_dev, float* lse_dev,
                          void* workspace_dev, size_t workspace_bytes, uint32_t* dev_err_dev,
                          qmla_stream_t stream);

/* The same decode over the BF16 comparison cache (same kernel, no dequantisation;
 * the paper's BF16 baseline, App. F.1). */
int qmla_mla_decode_bf16cache(const void* pool_dev, int num_blocks, const uint16_t* q_latent_dev,
                              const uint16_t* q_pe_dev, int batch, int heads,
                              const int32_t* block_table_dev, int max_blocks,
                              const int32_t* seq_lens_dev, float softmax_scale, float* out_dev,
                              float* lse_dev, void* workspace_dev, size_t workspace_bytes,
                              uint32_t* dev_err_dev, qmla_stream_t stream);

/*
 * The paper's own INT4 page ("C4R4": 4-bit content, 4-bit RoPE key; App. C.5,
 * storage layout; App. C.4, scale precisions). Same codes, groups and packing as
 * the c_bits = 4 block above; the metadata differ: per token and group a bf16
 * scale for content groups, an fp32 scale for the RoPE group, and a uint8 zero
 * point. Staging (App. C.4 with m = 15; d = RN_f32(x_max - x_min)):
 *     content  s = RN_bf16(RN_f32(max(d, 1e-8) / 15))
 *     RoPE     s = RN_f32(max(d, 1e-8) / 15)
 *     z = clip(rne(RN_f32(-x_min / s)), 0, 15);  q = clip(rne(RN_f32(RN_f32(x / s) + z)), 0, 15)
 * (for content groups the fp32 quotients give the exact-arithmetic codes, since
 * a bf16 x over a bf16 s is never within fp32 rounding of a half-integer).
 * A page of 64 token slots, 20480 bytes (320 per token):
 *     [0, 16384)       content codes   [group 8][slot 64][32 bytes]
 *     [16384, 18432)   RoPE-key codes  [slot 64][32 bytes]
 *     [18432, 19456)   content scales  [group 8][slot 64] bf16
 *     [19456, 19712)   RoPE scales     [slot 64] fp32
 *     [19712, 20288)   zero points     [group 9][slot 64] uint8 (group 8: RoPE key)
 *     [20288, 20480)   padding, never written or read
 * The decode's fp16 tile value of a code is RN_f16(s (q - z)) for content and
 * RN_f16(RN_f32(s (q - z))) for the RoPE key.
 */
size_t qmla_c4r4_page_bytes(void);

/* qmla_quant_append into pages of the paper's format (qmla_c4r4_page_bytes()
 * bytes each). prot_dev is optional: NULL writes the packed pages only; non-NULL
 * also writes the sink4/local128 protection rows as qmla_quant_append_protected
 * does, and then seq_lens_dev (lengths after this call) must be non-NULL and
 * latent_dev, k_pe_dev, prot_dev 16-byte aligned. Errors as qmla_quant_append. */
int qmla_quant_append_c4r4(void* pool_dev, int num_blocks, const uint16_t* latent_dev, const uint16_t* k_pe_dev,
                           const int32_t* seq_ids_dev, const int32_t* positions_dev, int n,
                           const int32_t* block_table_dev, int num_seqs, int max_blocks,
                           const int32_t* seq_lens_dev, void* prot_dev, uint32_t* dev_err_dev,
                           qmla_stream_t stream);

/* qmla_mla_decode over pages of the paper's format. prot_dev NULL attends over
 * the packed pages only; non-NULL (16-byte aligned) applies sink4/local128
 * protection as qmla_mla_decode_protected does. Outputs, workspace
 * (qmla_decode_workspace_bytes) and errors as qmla_mla_decode. */
int qmla_mla_decode_c4r4(const void* pool_dev, int num_blocks, const uint16_t* q_latent_dev,
                         const uint16_t* q_pe_dev, int batch, int heads, const int32_t* block_table_dev,
                         int max_blocks, const int32_t* seq_lens_dev, const void* prot_dev, float softmax_scale,
                         float* out_dev, float* lse_dev, void* workspace_dev, size_t workspace_bytes,
                         uint32_t* dev_err_dev, qmla_stream_t stream);

/*
 * Every decode variant above from one descriptor (Eq. mla_compact; App. C.5):
 * qmla_mla_decode, _protected, _c4r4, _multi and _bf16cache are this call with
 * some fields fixed. Fields:
 *   cache_kind      4 or 2 (this library's block at that content width),
 *                   QMLA_CACHE_C4R4 (the paper's page) or QMLA_CACHE_BF16
 *   pool, num_blocks, q_latent, q_pe, block_table, max_blocks, seq_lens,
 *   softmax_scale, out, lse, workspace, workspace_bytes, dev_err
 *                   as in qmla_mla_decode (q_latent / q_pe / out / lse shaped
 *                   [batch, q_tokens, heads, ...] when q_tokens > 1)
 *   batch, q_tokens, heads
 *                   q_tokens 1..QMLA_MAX_Q_TOKENS query tokens per sequence,
 *                   heads 1..128 per token (as qmla_mla_decode_multi)
 *   prot            sink4/local128 protection buffer or NULL (not with BF16)
 *   max_len         a bound of seq_lens known on the host, or 0 (max_blocks x 64
 *                   then). It only chooses between the library's two main kernels
 *                   (see qmla_mla_decode): a wrong value costs time, never results.
 *                   (It lies where the structure had padding.)
 *   ev_before_main, ev_after_main
 *                   optional cudaEvent_t (NULL = none): recorded on `stream`
 *                   immediately before and after the main decode kernel of
 *                   this call only, so that a caller can time that kernel
 *                   with cudaEventElapsedTime. With either set, the call's
 *                   launches wait for one another in full instead of
 *                   overlapping their start-up, so that the events bracket
 *                   the main kernel alone. The library keeps no reference to
 *                   them after the call returns.
 * Returns QMLA_ERR_INVALID_ARG for a NULL descriptor or a bad field, else as
 * qmla_mla_decode. The descriptor is read during the call only.
 */
typedef struct qmla_decode_desc {
  const void* pool;
  int cache_kind;
  int num_blocks;
  const uint16_t* q_latent;
  const uint16_t* q_pe;
  int batch;
  int q_tokens;
  int heads;
  const int32_t* block_table;
  int max_blocks;
  int max_len;
  const int32_t* seq_lens;
  const void* prot;
  float softmax_scale;
  float* out;
  float* lse;
  void* workspace;
  size_t workspace_bytes;
  uint32_t* dev_err;
  void* ev_before_main;
  void* ev_after_main;
} qmla_decode_desc;
int qmla_mla_decode_ex(const qmla_decode_desc* desc, qmla_stream_t stream);

/*
 * The cache writer for rows as a layer's down-projection leaves them: the latent is
 * normalised and the RoPE key rotated on the way into any of the four caches, in one
 * pass (App. C.5's fused writer takes them normalised and rotated; the offline
 * transformations are folded into the weights, so with a content rotation the norm's
 * weight is the content scale S_C). Token i, with latent x, RoPE key k and position p:
 *     x'_c = RN_bf16(RN_f32(w_c x_c / sqrt(mean_c(x_c^2) + eps)))          (norm != 0)
 *     k'   = RN_bf16(RN_f32(k turned by the angles of position p))
 * and (x', k') is then stored exactly as qmla_quant_append (_protected, _c4r4) or
 * qmla_bf16_append store a row. The sums and products carry their rounding errors
 * along, so that the stored bytes do not depend on the order of a sum; that holds for every
 * finite row, the smallest and the largest too, with |w_c| below 2^64 (results below 2^-80
 * may be off by one step of bf16, or 2^-104). A NaN makes its row's latent NaN; in a row with
 * an infinity the finite values become 0 and the infinite ones NaN; a row of zeros is NaN with
 * eps = 0, as the formula has it.
 *
 *   pool, num_blocks, seq_ids, positions, n, block_table, num_seqs, max_blocks, dev_err
 *                   as in qmla_quant_append; cache_kind 4, 2, QMLA_CACHE_C4R4 or
 *                   QMLA_CACHE_BF16
 *   latent, latent_stride
 *                   [n] rows of 512 bf16, latent_stride elements apart (even, >= 512; not used when n == 1)
 *   k_pe, k_pe_stride
 *                   [n] rows of 64 bf16, k_pe_stride elements apart (even, >= 64; not used when n == 1).
 *                   Both 4-byte aligned; 16-byte aligned rows (and strides that are multiples of
 *                   8) are read in wider pieces: 32,797 INT4 tokens 23 against 39 us
 *                   (So the two may be the columns of one [n, 576] projection output.)
 *   norm, norm_weight, norm_eps
 *                   norm 0: the latent is stored as it is. Otherwise w is norm_weight
 *                   [512] bf16 (16-byte aligned) or, NULL, all ones, and eps is 0 .. 1e30
 *   cos_sin, rope_len
 *                   [rope_len][64] fp32, 16-byte aligned: the cosines of a position's 32
 *                   angles, then the sines. A position at or beyond rope_len is a bad position
 *   interleaved     0: channel i turns with channel i + 32 (a, b -> a c - b s, a s + b c);
 *                   1: channel 2 i turns with channel 2 i + 1
 *   seq_lens, prot  the sink4/local128 protection buffer and the lengths after this call,
 *                   as in qmla_quant_append_protected, or NULL (not with QMLA_CACHE_BF16).
 *                   The protection rows hold the normalised and rotated values
 * A token with a bad sequence, position or block is not written (dev_err says so). Two
 * tokens of one call at the same place race, group by group.
 * The descriptor is read during the call only. n == 0 is a no-op.
 */
typedef struct qmla_append_desc {
  void* pool;
  int cache_kind;
  int num_blocks;
  const uint16_t* latent;
  long long latent_stride;
  const uint16_t* k_pe;
  long long k_pe_stride;
  int norm;
  float norm_eps;
  const uint16_t* norm_weight;
  const float* cos_sin;
  int rope_len;
  int interleaved;
  const int32_t* seq_ids;
  const int32_t* positions;
  int n;
  int num_seqs;
  const int32_t* block_table;
  int max_blocks;
  const int32_t* seq_lens;
  void* prot;
  uint32_t* dev_err;
} qmla_append_desc;
int qmla_rope_append(const qmla_append_desc* desc, qmla_stream_t stream);

/* qmla_rope_append with the keys turned by the angles of rope_positions[i] ([n] int32)
 * instead of those of the cache position positions[i]: the nodes of a tree of drafts lie side
 * by side in the cache, but siblings have the same position in the text. A rope position
 * below 0 or at or beyond rope_len is a bad position. NULL: as qmla_rope_append. */
int qmla_rope_append_at(const qmla_append_desc* desc, const int32_t* rope_positions_dev, qmla_stream_t stream);

/*
 * Turns the RoPE part of queries by the angles of their positions, with the
 * convention and table of qmla_rope_append, in fp32 (a product and an FMA), rounded to
 * bf16:
 *   q_pe_dev        [n, heads, 64] bf16, rows q_token_stride and q_head_stride elements
 *                   apart (multiples of 8, not negative, below 2^38; not used where that axis
 *                   has one element), 16-byte aligned. (So it may be the last 64 columns of a
 *                   [n, heads, 192] projection output.)
 *   heads           1 .. 2^24, n x heads at most 2^36
 *   positions_dev   [n] int32
 *   out_dev         [n, heads, 64] bf16 with strides of its own, 16-byte aligned. It may
 *                   be q_pe_dev with the same strides (in place) or share no memory with it;
 *                   its rows must not overlap one another
 * The heads of a token whose position is negative or at or beyond rope_len are left
 * unwritten (QMLA_DEVERR_BAD_POSITION). n == 0 is a no-op.
 */
int qmla_rope_query(const uint16_t* q_pe_dev, long long q_token_stride, long long q_head_stride,
                    const int32_t* positions_dev, int n, int heads, const float* cos_sin_dev, int rope_len,
                    int interleaved, uint16_t* out_dev, long long out_token_stride, long long out_head_stride,
                    uint32_t* dev_err_dev, qmla_stream_t stream);

/*
 * Reads cached tokens back as bf16 rows (512 latent values, then the RoPE key's 64),
 * for whatever needs the values themselves: the up-projection of a chunked prompt's
 * context (qmla_mla_prefill), a cache handed to another replica.
 *   rows[i] = RN_bf16(RN_f32(s (q - z))) of the token at positions[i] of sequence
 *   seq_ids[i] (NULL: sequence i); the BF16 cache's rows and protected positions
 *   (prot non-NULL; P_L from seq_lens, as in qmla_mla_decode_protected) unchanged.
 *   rows, row_stride   [n] rows of 576 bf16, row_stride elements apart (a multiple of 8,
 *                   >= 576; not used when n == 1), 16-byte aligned
 * Other fields as in qmla_append_desc. A token with a bad sequence, position (with prot
 * also one at or beyond its sequence's length) or block leaves its row unwritten
 * (dev_err says so). n == 0 is a no-op.
 */
typedef struct qmla_read_desc {
  const void* pool;
  int cache_kind;
  int num_blocks;
  const int32_t* seq_ids;
  const int32_t* positions;
  int n;
  int num_seqs;
  const int32_t* block_table;
  int max_blocks;
  const int32_t* seq_lens;
  const void* prot;
  uint16_t* rows;
  long long row_stride;
  uint32_t* dev_err;
} qmla_read_desc;
int qmla_cache_read(const qmla_read_desc* desc, qmla_stream_t stream);

/*
 * The expanded form of the attention, for prompts: every head has its own 128
 * content channels of key and value (the up-projected latent), and all heads share
 * the token's RoPE key. Sequence b holds the queries cu_q[b] .. cu_q[b + 1] - 1 and
 * the keys cu_kv[b] .. cu_kv[b + 1] - 1, Lq and Lk of them; query i of it sees key j when
 *     causal != 0:  j <= i + Lk - Lq   (the queries are the last Lq of Lk tokens)
 *     causal == 0:  always
 *     S[i,h,j]   = softmax_scale * (q[i,h,:128] . k[j,h,:] + q[i,h,128:] . k_pe[j,:])
 *     out[i,h,:] = RN_bf16(sum_j softmax_j(S[i,h,:]) v[j,h,:]);  lse[i,h] = log sum_j exp(S[i,h,j])
 * over the keys it sees; a query that sees none gets out = 0 and lse = -inf. Scores,
 * softmax statistics and sums are fp32; the weights reach the tensor cores as bf16.
 *
 *   q, q_token_stride, q_head_stride   [n_q, heads, 192] bf16, RoPE part rotated
 *   k, v and their strides             [n_kv, heads, 128] bf16 each (so the two may be
 *                   the halves of one [n_kv, heads, 256] projection output)
 *   k_pe, k_pe_stride                  [n_kv, 64] bf16, rotated
 *                   All four 16-byte aligned; strides in elements, positive multiples of 8
 *                   below 2^38 (ignored where that axis has one element)
 *   n_q, n_kv, heads, batch            rows given (at most 2^26), heads 1..1024, sequences
 *                   1..65536. n_kv may be 0 (k, v, k_pe and their strides are not used then);
 *                   n_q == 0 is a no-op
 *   cu_q, cu_kv     [batch + 1] int32 offsets, not decreasing. A sequence whose offsets
 *                   decrease, are negative or lie beyond n_q / n_kv is left out, and so is
 *                   one whose queries begin before the end of an earlier sequence that has
 *                   none of these faults (QMLA_DEVERR_BAD_OFFSETS); the others are computed
 *   softmax_scale   above 0, at most 1e30
 *   out             [n_q, heads, 128] bf16, contiguous, 32-byte aligned; shares no memory
 *                   with the inputs
 *   lse             [n_q, heads] float32, contiguous, or NULL
 *                   Rows that belong to no sequence are left as they were
 *   workspace       >= qmla_prefill_workspace_bytes(batch, n_q) bytes, 256-byte aligned,
 *                   scratch as for qmla_mla_decode. Calls that overlap need one each
 * Keys and values of other sequences never reach a result, whatever they hold. Within
 * a sequence a value that is not finite may reach queries before it (weight 0 x inf).
 */
typedef struct qmla_prefill_desc {
  const uint16_t* q;
  long long q_token_stride, q_head_stride;
  const uint16_t* k;
  long long k_token_stride, k_head_stride;
  const uint16_t* v;
  long long v_token_stride, v_head_stride;
  const uint16_t* k_pe;
  long long k_pe_stride;
  int n_q, n_kv, heads, batch;
  const int32_t* cu_q;
  const int32_t* cu_kv;
  int causal;
  float softmax_scale;
  uint16_t* out;
  float* lse;
  void* workspace;
  size_t workspace_bytes;
  uint32_t* dev_err;
} qmla_prefill_desc;
int qmla_mla_prefill(const qmla_prefill_desc* desc, qmla_stream_t stream);

/* Workspace bytes qmla_mla_prefill needs; 0 for bad arguments. Room for 320 partial results of
 * long contexts (42.6 MB) whatever the call, and 64 bytes per 256 rows and per sequence. */
size_t qmla_prefill_workspace_bytes(int batch, int n_q);

/*
 * A step of speculative decoding with a tree of drafted tokens. Node 0 of a sequence's tree
 * is its last committed token, the others are drafts; parents[b, t] is the node that node t
 * continues: an earlier one, or -1. The nodes lie in the cache in their order, behind the
 * context: with n nodes and L = seq_lens[b] tokens (the nodes included), node t is position
 * ctx + t, ctx = L - n. (It is written there, and rotated by the angles of the position
 * that it would have in the text, ctx + its depth.) A step is
 *   qmla_rope_append_at    the nodes' rows into the cache
 *   qmla_mla_decode_tree   their attention, in every layer
 *   qmla_tree_verify       which of them the target accepts, and the token after them
 *   qmla_cache_keep        their rows moved together behind the context, in every layer.
 *
 * qmla_mla_decode_tree: node t attends to the ctx positions of the context, to the nodes
 * above it and to itself, A(t) = {t} U A(parents[t]):
 *     S[b,t,h,p] = softmax_scale * (q_latent[b,t,h,:] . C_hat[b,p,:] + q_pe[b,t,h,:] . K_hat[b,p,:]),
 *                  p < ctx or p - ctx in A(t)
 *     out[b,t,h,:] = RN_bf16(sum_p softmax_p(S[b,t,h,:]) C_hat[b,p,:]);  lse[b,t,h] = log sum_p exp(S[b,t,h,p])
 *   pool, cache_kind, num_blocks, block_table, max_blocks, softmax_scale, dev_err
 *                   as in qmla_mla_decode_ex, any of the four cache kinds
 *   max_len         a bound of seq_lens, or 0 (max_blocks x 64 then). Longer sequences are bad ones.
 *                   (The launches and each sequence's room in the workspace go by it: pass one with
 *                   a table wider than its sequences)
 *   q_latent, q_pe  [batch, nodes, heads, 512] and [batch, nodes, heads, 64] bf16, 16-byte aligned
 *   nodes, heads    1 .. QMLA_MAX_TREE_NODES, 1 .. 128
 *   parents         [batch, nodes] int32
 *   seq_lens        [batch] int32, the nodes included
 *   tree_lens       [batch] int32: nodes of each sequence (its first ones; 0: no tree), or
 *                   NULL: all of them
 *   prot, draft_rows  sink4/local128 protection, both or neither (not with QMLA_CACHE_BF16):
 *                   the protection buffer holds the rows of the context, P_L for L = ctx, and
 *                   draft_rows [batch][64][576] bf16, 16-byte aligned, the nodes' own rows
 *                   (row t of sequence b: node t's latent, then its RoPE key), which are read
 *                   in the place of their packed copies. (The drafts are not in the ring:
 *                   they would take the places of context that is protected once they are
 *                   refused. The layout is a BF16 cache's with one block a sequence, so that
 *                   qmla_rope_append_at writes these rows too.)
 *   out             [batch, nodes, heads, 512] bf16, 32-byte aligned
 *   lse             [batch, nodes, heads] float32, or NULL
 *   workspace       >= qmla_tree_workspace_bytes(batch, nodes, heads, 0) bytes, 256-byte
 *                   aligned, scratch as for qmla_mla_decode. With the bytes for the call's
 *                   max_len (or max_blocks x 64) tokens the context is dequantised once for all
 *                   rows of a sequence, in the workspace; where they are fewer, for as many
 *                   sequences at a time as they hold, in as many launches one after the other.
 *                   (Not with up to 64 rows, nodes x heads, over more than 40,960 tokens, batch x
 *                   bound, unless lse of a quantised cache is asked for.) lse is then of the scores
 *                   of s (q - z) itself instead of its fp16 value (which leaves lse 2e-6 to 4e-5 of
 *                   itself off, the more the fewer keys have the weight) and sums the weights before
 *                   their rounding to fp16 (which leaves 4e-6)
 * A node behind the last of its sequence gets out = 0 and lse = -inf. So do a node whose
 * parent is not an earlier node or -1 and the nodes below it (QMLA_DEVERR_BAD_TREE), and
 * every node of a sequence whose count is below 0, above `nodes` or above its length (the
 * same) or whose length is bad (QMLA_DEVERR_BAD_POSITION). Queries, cached values and weights are
 * fp16 in the tensor core: BF16 values below 2^-14 lose bits, those beyond 65,504 are infinite. A
 * value that is not finite in a cache row reaches the nodes that see it, and no others; one in a query
 * leaves that row, and no other, without a result of meaning.
 */
typedef struct qmla_tree_desc {
  const void* pool;
  int cache_kind;
  int num_blocks;
  const uint16_t* q_latent;
  const uint16_t* q_pe;
  int batch, nodes, heads;
  int max_len;
  const int32_t* parents;
  const int32_t* tree_lens;
  const int32_t* block_table;
  int max_blocks;
  float softmax_scale;
  const int32_t* seq_lens;
  const void* prot;
  const uint16_t* draft_rows;
  uint16_t* out;
  float* lse;
  void* workspace;
  size_t workspace_bytes;
  uint32_t* dev_err;
} qmla_tree_desc;
int qmla_mla_decode_tree(const qmla_tree_desc* desc, qmla_stream_t stream);

/* Workspace bytes of qmla_mla_decode_tree on the current device for sequences up to max_tokens
 * (2,304 bytes a token of each; without lse, or over a BF16 cache, half of them are used), or,
 * with max_tokens 0, the least that it needs; 0 for bad arguments. */
size_t qmla_tree_workspace_bytes(int batch, int nodes, int heads, int max_tokens);

/*
 * Walks each tree from node 0 and keeps the drafts that the target accepts, so that the
 * tokens kept and the one drawn after them are distributed as the target's own. At node c,
 * with the target's probabilities p = target[b, c, :] of what follows it and the draft's
 * q = draft[b, c, :], from which the tokens of c's children were drawn independently, the
 * children x = tokens[b, t] are looked at in the order of their nodes:
 *     r(v) = max(p(v) - a q(v), 0), R = 1 and a = 0 at first
 *     the child is accepted if u_t q(x) R < r(x), u_t = uniforms[b, t]: the walk goes on at it;
 *     if not, a grows by R and R becomes sum_v r(v) of the new a.
 * (r / R is what is left of p after the refusals: max(r / R - q, 0) is r's next value over R.)
 * With draft NULL the children's tokens were chosen without randomness: the child is accepted
 * if u_t R < p(x); if not, R loses p(x), and p(x) becomes 0. Where no child is accepted the
 * walk ends, and the next token is the first v with
 *     sum_{w <= v} r(w) > u_0 sum_w r(w)
 * (r = p where nothing was refused), the last v with r(v) > 0 where rounding leaves none.
 * Sums and terms carry their rounding errors along: about 2^-46 of a sum is left, whatever
 * the vocabulary. Only a decision whose two sides are that near each other depends on the order
 * of a sum, which goes by vocab, batch and the rows' alignment; one call repeats itself exactly.
 *
 *   target, target_seq_stride, target_row_stride
 *                   [batch, nodes, vocab] probabilities of type probs (QMLA_PROBS_*), rows
 *                   and sequences that many elements apart (not negative, below 2^40; not used
 *                   where that axis has one element). Rows are not normalised; a target's value
 *                   below 0 counts as 0; the draft's are not below 0, and one that is not finite
 *                   leaves nothing of its token after a refusal. 16-byte aligned rows whose vocab
 *                   and strides are multiples of 16 bytes are read in wider pieces
 *   draft, ...      the same for the draft, or NULL. Rows of nodes without children are not read
 *   batch, nodes, vocab   1 .. 65535, 1 .. QMLA_MAX_TREE_NODES, 1 .. 2^24
 *   tokens, parents [batch, nodes] int32; tree_lens [batch] int32 or NULL, as above
 *   uniforms        [batch, nodes] float32 in [0, 1) (others count as the nearest, NaN as 0).
 *                   The number of node 0, which is not drawn, is the one for the next token
 *   path            [batch, nodes] int32 out: the kept nodes, 0 first, then -1
 *   kept            [batch] int32 out: how many they are
 *   next_token      [batch] int32 out
 * A sequence without a tree gets kept = 0, next_token = -1 and no path, and so does one whose
 * count is bad (QMLA_DEVERR_BAD_TREE). A node is passed over whose token is not in the
 * vocabulary or whose parent is not an earlier node or -1 (the same); but node 0 is kept
 * whatever they are, and a parent of it other than -1 reported. Where the sum of r is not positive
 * and finite, next_token is -1 (QMLA_DEVERR_BAD_PROBS). Outputs share no memory with the inputs
 * or one another.
 */
typedef struct qmla_verify_desc {
  const void* target;
  long long target_seq_stride, target_row_stride;
  const void* draft;
  long long draft_seq_stride, draft_row_stride;
  int probs;
  int batch, nodes, vocab;
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* tree_lens;
  const float* uniforms;
  int32_t* path;
  int32_t* kept;
  int32_t* next_token;
  uint32_t* dev_err;
} qmla_verify_desc;
int qmla_tree_verify(const qmla_verify_desc* desc, qmla_stream_t stream);

/*
 * Keeps the nodes path[b, 0 .. kept[b] - 1] of each sequence's tree in its cache and drops
 * the others: the row at position ctx + path[b, i] moves to ctx + i, in place and unchanged,
 * and new_lens[b] = ctx + kept[b] (ctx = seq_lens[b] - n, n = tree_lens[b] or `nodes`). One
 * call per layer's cache.
 *   pool, cache_kind, num_blocks, block_table, max_blocks, dev_err   as in qmla_append_desc
 *   batch, nodes    sequences, 1 .. QMLA_MAX_TREE_NODES
 *   path, kept      as qmla_tree_verify leaves them; path increases
 *   prot, draft_rows  as in qmla_mla_decode_tree, both or neither: the kept nodes' rows are
 *                   also copied from draft_rows into the protection buffer, which then holds
 *                   P_L for L = new_lens[b]
 *   seq_lens, new_lens   [batch] int32; they may be the same array (not with a second call of
 *                   the step to follow)
 * A sequence whose count, kept or path is bad (kept > n, a path that does not increase or
 * leaves 0 .. n - 1: QMLA_DEVERR_BAD_TREE; or a bad length: QMLA_DEVERR_BAD_POSITION) is left
 * as it is, with new_lens[b] = seq_lens[b]. A row from or to a bad block is not moved.
 * Sequences that share blocks must not share those of their nodes.
 */
typedef struct qmla_keep_desc {
  void* pool;
  int cache_kind;
  int num_blocks;
  int batch, nodes;
  const int32_t* block_table;
  int max_blocks;
  const int32_t* seq_lens;
  const int32_t* tree_lens;
  const int32_t* path;
  const int32_t* kept;
  void* prot;
  const uint16_t* draft_rows;
  int32_t* new_lens;
  uint32_t* dev_err;
} qmla_keep_desc;
int qmla_cache_keep(const qmla_keep_desc* desc, qmla_stream_t stream);

/* Bytes of the fixed device scratch array qmla_mla_decode_static uses
 * (32 MiB). */
size_t qmla_static_scratch_bytes(void);

/*
 * qmla_mla_decode without a workspace argument, for callers that cannot
 * allocate device memory where they call it (for example code running inside
 * an allocator-free region of a serving loop, or a host library that is
 * handed finished buffers and must not call cudaMalloc, whose implicit
 * synchronisation and memory growth it does not control). The paper has no
 * counterpart; this is a deployment convenience.
 *
 * Inputs, outputs and results are exactly those of qmla_mla_decode. The
 * scratch the decode needs lives in one file-scope device array of
 * qmla_static_scratch_bytes() bytes that every GPU loading this library holds
 * until the process exits. Nothing is allocated or freed by this call.
 * - The first call on a device looks up that array's device address
 *   (cudaGetSymbolAddress) with the device current; make that first call
 *   before capturing any stream.
 * - Accepts batch x heads whose workspace fits the array:
 *   qmla_decode_workspace_bytes(batch, heads) <= qmla_static_scratch_bytes().
 *   Larger ones return QMLA_ERR_WORKSPACE_TOO_SMALL before any launch. The
 *   workspace grows with the SM count; on a 152-SM GB300 32 sequences at 128
 *   heads fit, 64 sequences at 128 heads do not.
 * - Every call shares the array, which keeps the last call's contents;
 *   nothing in it needs to start at zero (each call rewrites or clears
 *   everything it reads). Calls whose work overlaps on the GPU (different
 *   streams, or different host threads on one device) race on it: serialise
 *   them.
 * - The looked-up address is kept for the life of the process: after a
 *   cudaDeviceReset of a device this entry point has run on, the address is
 *   stale, so do not call it on that device again in the same process.
 * - It is qmla_mla_decode_ex with the array as the workspace: argument checks
 *   and errors are those of qmla_mla_decode.
 */
int qmla_mla_decode_static(const void* pool_dev, int c_bits, int num_blocks, const uint16_t* q_latent_dev,
                           const uint16_t* q_pe_dev, int batch, int heads, const int32_t* block_table_dev,
                           int max_blocks, const int32_t* seq_lens_dev, float softmax_scale, float* out_dev,
                           float* lse_dev, uint32_t* dev_err_dev, qmla_stream_t stream);

/*
 * Test hook (no counterpart in the paper): the fp16 tile the decode kernel builds
 * from the cache for tile j (positions 128 j .. 128 j + 127) of sequence b, made
 * by the decode's own row loaders into its swizzled shared-memory chunks and
 * written out row-major in channel order.
 *   cache_kind   4 or 2: this library's block with that content width;
 *                QMLA_CACHE_C4R4: the paper's page; QMLA_CACHE_BF16: the BF16 cache
 *   prot_dev     NULL, or the sink4/local128 protection buffer (packed kinds):
 *                rows in P_L come from it as in qmla_mla_decode_protected
 *   tile_dev     [128][576] fp16 (uint16 bits), 16-byte aligned; row r holds the
 *                512 latent then 64 RoPE-key values of position 128 j + r, zero for
 *                rows at or past seq_lens_dev[b]
 * Table, lengths and errors as qmla_mla_decode; 0 <= b < batch, 0 <= j. One CTA
 * of 128 threads; not a fast path.
 */
int qmla_debug_tile(const void* pool_dev, int cache_kind, int num_blocks, const int32_t* block_table_dev,
                    int max_blocks, const int32_t* seq_lens_dev, int batch, int b, int j, const void* prot_dev,
                    uint16_t* tile_dev, uint32_t* dev_err_dev, qmla_stream_t stream);

/* Test hook (no counterpart in the paper): one warp waits, through the decode
 * kernel's bounded wait, for a barrier phase that nothing completes. After
 * limit_us microseconds (1 .. 1000000) the wait gives up and ORs
 * QMLA_DEVERR_TIMEOUT | QMLA_DEVERR_SITE_SOFTMAX into *dev_err_dev, and the
 * kernel returns; the context stays usable. The decode's own waits give up after
 * 2 s the same way (one site bit per wait, bits 8 and up). */
#define QMLA_DEVERR_SITE_SOFTMAX (0x100u << 5)
int qmla_debug_wait_timeout(uint32_t limit_us, uint32_t* dev_err_dev, qmla_stream_t stream);

/* Test hook: the main kernel that qmla_mla_decode_ex runs for this descriptor on a GPU
 * of `sms` SMs: 0 single CTAs (decode_main), 1 CTA pairs (decode_pair), -1 for a bad
 * descriptor. Looks at cache_kind, batch, q_tokens, heads, max_blocks, max_len and whether
 * prot is set; nothing is dereferenced and no device is needed. */
int qmla_debug_decode_route(const qmla_decode_desc* desc, int sms);

/* Copies the device error word to *host_out after synchronising `stream`. */
int qmla_read_dev_err(const uint32_t* dev_err_dev, uint32_t* host_out, qmla_stream_t stream);

/* The cudaError_t of the last failed CUDA call in this thread (0 if none). */
int qmla_last_cuda_error(void);

/* Static text for a status code. */
const char* qmla_status_string(int status);

/* Number of SMs of the current device (the decode grid size), or -1. */
int qmla_num_sms(void);

#ifdef __cplusplus
}
#endif

#endif /* QMLA_H_ */
