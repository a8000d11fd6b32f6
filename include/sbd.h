/*
 * sbd.h -- C ABI of the Set Block Decoding (SBD) block step on GB300 (sm_103a).
 *
 * One SBD forward over a block of k positions (arXiv 2509.04185, Sec. 2.3,
 * Eq. 5 and Algorithm 3) is served by three calls, issued in this order on
 * one CUDA stream:
 *
 *   sbd_block_attention      block queries attend to the exact KV cache and,
 *                            bidirectionally, to each other (Eq. 5; Fig. 3);
 *   sbd_head_entropy_sample  LM head over the masked positions, reduced in
 *                            the same kernel to a softmax entropy and a
 *                            Gumbel-max token per position (Eqs. 6-7);
 *   sbd_eb_select            entropy-bounded unmasking (Eq. 3).
 *
 * Conventions shared by every call
 *   - Every tensor argument is a caller-owned DEVICE pointer to contiguous
 *     row-major memory, aligned to 16 bytes.  Shapes are given in the call's
 *     descriptor; the library never keeps a pointer after the call returns.
 *   - `stream` is a cudaStream_t (NULL = the legacy default stream).  Work is
 *     enqueued asynchronously; the calls never synchronise the device.
 *   - The library allocates no device memory.  Calls that need scratch take
 *     a caller-owned `workspace` of at least the size returned by the
 *     matching *_workspace_size() query; the scratch content between calls
 *     is irrelevant (nothing needs zeroing).
 *   - Argument errors are detected on the host before anything is enqueued
 *     and returned as a status; sbd_last_error() then gives a one-line
 *     explanation (per calling thread).  Launch failures return
 *     SBD_ERR_CUDA.  No C++ exception crosses this interface.
 *   - Device-side faults that the host cannot see before launch (a cache
 *     length outside [0, max_cache_len], a wait that timed out) are recorded
 *     in a device error word read by sbd_device_error().
 *   - Calls are thread-safe; concurrent calls may share nothing but
 *     read-only inputs (each needs its own outputs and workspace).
 */
#ifndef SBD_H
#define SBD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SBD_OK = 0,
  SBD_ERR_INVALID_ARG = 1, /* null pointer, bad size, misalignment, bad gamma/tau */
  SBD_ERR_UNSUPPORTED = 2, /* valid but outside what the kernels implement */
  SBD_ERR_WORKSPACE = 3,   /* workspace missing or smaller than required */
  SBD_ERR_CUDA = 4         /* a CUDA runtime/driver call or a launch failed */
} sbd_status;

typedef enum { SBD_DTYPE_F32 = 0, SBD_DTYPE_BF16 = 1 } sbd_dtype;

/* ------------------------------------------------------------------------
 * Block attention (Eq. 5 with the inference mask of Fig. 3 and of the
 * FlexAttention appendix listing): every block query row i of sequence b
 * sees the cached keys 0 .. cache_len[b]-1 and all k block keys.
 *
 *   q        [B, k, Hq, D]          block queries (already position-encoded)
 *   k_cache  [B, Lmax, Hkv, D]      exact KV cache of x_<t; slots at or past
 *   v_cache  [B, Lmax, Hkv, D]      cache_len[b] are never used (may hold NaN)
 *   cache_len[B] int32 (device)     0 <= cache_len[b] <= Lmax
 *   k_blk    [B, k, Hkv, D]         keys/values of the k block positions
 *   v_blk    [B, k, Hkv, D]         (recomputed every forward, not cached)
 *   out      [B, k, Hq, D]          attention output, same dtype as q
 *
 * Query head h reads KV head h / (Hq / Hkv).  s = scale * q.k with
 * scale = desc->scale, or 1/sqrt(D) when desc->scale == 0.  All inputs share
 * desc->dtype; accumulation is fp32.
 * Supported: 1 <= k <= 32, D in {64, 128}, Hq % Hkv == 0,
 * (Hq/Hkv) * k <= 128.  desc->num_splits = 0 picks the KV split count.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t batch;          /* B   */
  int32_t block_k;        /* k   */
  int32_t n_q_heads;      /* Hq  */
  int32_t n_kv_heads;     /* Hkv */
  int32_t head_dim;       /* D   */
  int32_t max_cache_len;  /* Lmax (row count of k_cache / v_cache) */
  int32_t dtype;          /* sbd_dtype */
  float scale;            /* 0 -> 1/sqrt(D) */
  int32_t num_splits;     /* 0 -> automatic; else KV splits per (b, kv head) */
} sbd_attn_desc;

size_t sbd_block_attention_workspace_size(const sbd_attn_desc* desc);

sbd_status sbd_block_attention(const sbd_attn_desc* desc, const void* q,
                               const void* k_cache, const void* v_cache,
                               const int32_t* cache_len, const void* k_blk,
                               const void* v_blk, void* out, void* workspace,
                               size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Block attention of the first iteration of a block after the previous one
 * (Algorithm 3, "first iteration and t >= k"; the inference mask of the
 * FlexAttention appendix listing with its causal point at the new block).
 * The forward carries the n_causal tokens of the previous block, which the
 * cache does not hold yet, as the leading block rows:
 *   block row i <  n_causal  sees the cached keys and block keys j <= i;
 *   block row i >= n_causal  sees the cached keys and all block keys;
 * and the keys/values of rows i < n_causal are written into the caches at
 * positions cache_len[b] + i.  cache_len itself is not changed: the caller
 * advances it by n_causal once the call has completed.  Arguments, layouts,
 * workspace and errors are those of sbd_block_attention, except that
 * k_cache / v_cache are written (only at the n_causal new positions), and
 * 0 <= n_causal <= block_k (else SBD_ERR_INVALID_ARG).  A sequence with
 * cache_len[b] + n_causal > max_cache_len gets no append and sets
 * SBD_DEVERR_CACHE_LEN.  n_causal = 0 is sbd_block_attention.
 * ---------------------------------------------------------------------- */
sbd_status sbd_block_attention_causal_prefix(const sbd_attn_desc* desc, int32_t n_causal,
                                             const void* q, void* k_cache, void* v_cache,
                                             const int32_t* cache_len, const void* k_blk,
                                             const void* v_blk, void* out, void* workspace,
                                             size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * LM head + entropy + Gumbel-max sample (Eqs. 6-7; Algorithm 3 "compute
 * probabilities"), over the MASKED block positions only.  For masked
 * position (b, i) with hidden row h = hidden[b, i, :]:
 *   z_v      = sum_c h_c * w[v, c]                (fp32 accumulate)
 *   entropy  = -sum_v p_v log p_v, p = softmax(z)  (nats)
 *   token    = argmax_v (z_v + tau * gumbel[b, i, v]), lowest v on ties
 * Logits are never written to memory.  Unmasked positions get
 * entropy = +inf and token = -1.
 *
 *   hidden [B, k, H], w [V, H] (nn.Linear layout), same dtype
 *   masked [B, k] uint8 (nonzero = masked)
 *   gumbel [B, k, V] fp32, indexed by block position; may be NULL iff
 *          tau == 0 (greedy); rows of unmasked positions are not read
 *   entropy [B, k] fp32 out, token [B, k] int32 out
 * Supported: B * k <= 512, H % 64 == 0 for bf16 (H % 4 == 0 for fp32),
 * tau >= 0 and finite.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t batch;    /* B */
  int32_t block_k;  /* k */
  int32_t hidden;   /* H */
  int32_t vocab;    /* V */
  int32_t dtype;    /* sbd_dtype of hidden and w */
} sbd_head_desc;

size_t sbd_head_entropy_sample_workspace_size(const sbd_head_desc* desc);

sbd_status sbd_head_entropy_sample(const sbd_head_desc* desc, const void* hidden,
                                   const void* w, const uint8_t* masked,
                                   const float* gumbel, float tau, float* entropy,
                                   int32_t* token, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * sbd_head_entropy_sample plus the confidence of every masked position, for
 * the confidence-ordered selection rules of the Appendix "Sampling
 * algorithm" (Factor decoding; EB-Sampler with the confidence proxy):
 *   confidence = max_v p_v,  p = softmax(z) at temperature 1,
 * computed from the same merged statistics as the entropy (1 / sum_v
 * exp(z_v - max z)).  Unmasked positions get confidence = 0.
 *   confidence [B, k] fp32 out; every other argument, the workspace (size
 *   from sbd_head_entropy_sample_workspace_size) and the errors are those of
 *   sbd_head_entropy_sample.
 * ---------------------------------------------------------------------- */
sbd_status sbd_head_entropy_confidence_sample(const sbd_head_desc* desc, const void* hidden,
                                              const void* w, const uint8_t* masked,
                                              const float* gumbel, float tau, float* entropy,
                                              float* confidence, int32_t* token,
                                              void* workspace, size_t workspace_bytes,
                                              void* stream);

/* ------------------------------------------------------------------------
 * sbd_head_entropy_sample with counter-based Gumbel noise generated inside
 * the kernel instead of read from a [B, k, V] buffer (the buffer read is
 * 4 R V bytes per call).  The noise of block position n = b * k + i and
 * vocabulary id v is
 *   x = word (v mod 4) of Philox4x32-10(counter = (v div 4, n, offset_lo,
 *       offset_hi), key = (seed_lo, seed_hi))
 *       (Salmon, Moraes, Dror, Shaw, SC 2011; 10 rounds),
 *   u = ((x >> 9) + 1/2) * 2^-23   (exact in fp32, strictly inside (0, 1)),
 *   g = -ln(-ln u)                 (fp32, full-precision logarithms),
 * and token = argmax_v (z_v + tau * g).  A new offset (or seed) per step
 * gives fresh noise.  Every other argument, the workspace and the errors are
 * those of sbd_head_entropy_sample; tau = 0 is greedy.
 * ---------------------------------------------------------------------- */
sbd_status sbd_head_entropy_sample_philox(const sbd_head_desc* desc, const void* hidden,
                                          const void* w, const uint8_t* masked, uint64_t seed,
                                          uint64_t offset, float tau, float* entropy,
                                          int32_t* token, void* workspace,
                                          size_t workspace_bytes, void* stream);

/* The same noise written out: out[r, v] = g(row_ids[r], v) for 0 <= v < vocab.
 *   row_ids [n_rows] int32 (device): block positions n = b * k + i
 *   out [n_rows, vocab] fp32 (device)
 * Supported: n_rows <= 65535. */
sbd_status sbd_gumbel_philox(int32_t n_rows, const int32_t* row_ids, int32_t vocab,
                             uint64_t seed, uint64_t offset, float* out, void* stream);

/* ------------------------------------------------------------------------
 * A plain linear layer on the LM-head kernel: y = x W^T, the GEMMs of a
 * transformer layer at decode shapes (few rows, weights streamed once).
 * Used to time full forwards of a model around the block step (the
 * paper's timing section models the linear layers as GEMMs); it is not
 * part of the block step itself.
 *
 *   x [rows, in_features]           bf16, row-major (device)
 *   w [out_features, in_features]   bf16, row-major, nn.Linear layout (device)
 *   y [rows, out_features]          bf16, row-major (device, written)
 *   workspace                       sbd_linear_workspace_size(desc) bytes
 *                                   (device, 16-byte aligned; may be NULL
 *                                   when the size is 0)
 *
 * y is the fp32 sum over in_features of the bf16 products, rounded to
 * bf16 (round to nearest even).  When a layer has too few output tiles to
 * fill the GPU, the in_features are cut into ranges whose fp32 partials are
 * summed in range order: up to 160 rows inside a thread-block cluster where
 * one of that size fits, else through the workspace by a second kernel (the
 * split is chosen per call from the shape).  Above 160 rows the product runs on
 * pairs of SMs (2-SM tensor-core MMAs).  All pointers 16-byte aligned,
 * caller-owned.  Asynchronous on `stream`.
 * Supported: dtype bf16, 0 <= rows <= 512, in_features a positive multiple
 * of 64, out_features >= 1; SBD_ERR_UNSUPPORTED otherwise; a workspace
 * smaller than needed gives SBD_ERR_WORKSPACE.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t rows, in_features, out_features;
  sbd_dtype dtype;
} sbd_linear_desc;

/* Bytes for the largest split the call may choose: a function of the
 * shape only, the same on every device (0 when no split is possible); 0
 * for an invalid descriptor. */
size_t sbd_linear_workspace_size(const sbd_linear_desc* desc);
sbd_status sbd_linear(const sbd_linear_desc* desc, const void* x, const void* w, void* y,
                      void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * No-allocation variant of sbd_head_entropy_sample.  The paper has no
 * counterpart: this entry point exists for callers that cannot allocate
 * device memory -- a host framework that owns the whole device memory pool,
 * a latency-critical loop that cannot afford the device synchronisation of
 * cudaMalloc/cudaFree, or a plug-in with no allocator to borrow a workspace
 * from.  Same arguments, semantics and results as sbd_head_entropy_sample,
 * minus the workspace: the scratch is a fixed array inside the library, of
 * SBD_HEAD_NOALLOC_MAX_SCRATCH bytes, which every GPU that loads the library
 * holds until the process exits.
 *   - Shapes whose scratch (sbd_head_entropy_sample_workspace_size) exceeds
 *     that size are rejected with SBD_ERR_UNSUPPORTED before any launch.
 *   - The first call on a device looks up the array's device address
 *     (cudaGetSymbolAddress, with that device current); make that first
 *     call before any stream capture on that device.
 *   - All calls on a device share the one array, which keeps the last
 *     call's contents (nothing in it needs to start at zero).  Calls whose
 *     kernels overlap on the GPU -- on different streams, or from several
 *     host threads -- race on it: serialise them (one stream, or events).
 *   - Allocates nothing: no cudaMalloc/cudaFree or allocating library call.
 * ---------------------------------------------------------------------- */
#define SBD_HEAD_NOALLOC_MAX_SCRATCH (8u << 20) /* 8 MiB */

sbd_status sbd_head_entropy_sample_noalloc(const sbd_head_desc* desc, const void* hidden,
                                           const void* w, const uint8_t* masked,
                                           const float* gumbel, float tau, float* entropy,
                                           int32_t* token, void* stream);

/* ------------------------------------------------------------------------
 * Entropy-bounded select, entropy proxy (Eq. 3; Algorithm 3 "unmask").  Per
 * sequence b: sort the masked positions by (entropy, position) ascending,
 * i_1, i_2, ...; accept the first s >= 1 positions, s the largest value with
 *   H_{i_1} + ... + H_{i_{s-1}} <= gamma     (fp32 prefix sums)
 * capped at the number of masked positions; for each accepted i write
 * block_tokens[b, i] = token[b, i] and masked[b, i] = 0, and set
 * n_unmasked[b] = s (0 when nothing is masked).  Entropies of masked
 * positions must be >= 0 (as produced by sbd_head_entropy_sample); a NaN
 * sorts last.  Entropies/tokens of unmasked positions are not read.
 *
 *   entropy [B, k] fp32, token [B, k] int32   inputs
 *   masked [B, k] uint8, block_tokens [B, k] int32 (-1 = mask)   in/out
 *   n_unmasked [B] int32 out (may be NULL)
 * Supported: 1 <= k <= 32, gamma >= 0 and finite.
 * ---------------------------------------------------------------------- */
sbd_status sbd_eb_select(int32_t batch, int32_t block_k, const float* entropy,
                         const int32_t* token, float gamma, uint8_t* masked,
                         int32_t* block_tokens, int32_t* n_unmasked, void* stream);

/* ------------------------------------------------------------------------
 * One unmasking step under a selectable rule (Algorithm 3 "unmask"; the
 * rules of Eq. 3 and of the Appendix "Sampling algorithm").  Per sequence b
 * the masked positions are ordered by the rule's key (ties to the lower
 * position), the first s accepted, their tokens committed and their flags
 * cleared, exactly as in sbd_eb_select:
 *   SBD_SELECT_EB_ENTROPY          entropy ascending; s of Eq. 3 with
 *                                  threshold = gamma.  Identical to
 *                                  sbd_eb_select (confidence not read).
 *   SBD_SELECT_EB_CONFIDENCE       confidence descending; s >= 1 the largest
 *                                  count with  sum_{j<=s} H_{i_j} -
 *                                  max_{j'<=s} H_{i_j'} <= gamma  (the
 *                                  general EB bound), capped at |M|.
 *   SBD_SELECT_FACTOR              confidence descending, c^1 >= c^2 >= ...;
 *                                  s the largest n in 1..|M| with
 *                                  (n + 1) c^n < f  (threshold = f), s = 1
 *                                  when no n qualifies.
 *   SBD_SELECT_FACTOR_COMPLEMENT   as FACTOR with (n + 1)(1 - c^n) < f.
 * Sums, maxima and products in fp32.  A NaN key sorts last.
 *
 *   entropy [B, k] fp32, confidence [B, k] fp32 (may be NULL for
 *   SBD_SELECT_EB_ENTROPY), token [B, k] int32   inputs
 *   masked [B, k] uint8, block_tokens [B, k] int32 (-1 = mask)   in/out
 *   n_unmasked [B] int32 out (may be NULL)
 * Supported: 1 <= k <= 32; threshold finite and >= 0.  An unknown rule is
 * SBD_ERR_INVALID_ARG.
 * ---------------------------------------------------------------------- */
typedef enum {
  SBD_SELECT_EB_ENTROPY = 0,
  SBD_SELECT_EB_CONFIDENCE = 1,
  SBD_SELECT_FACTOR = 2,
  SBD_SELECT_FACTOR_COMPLEMENT = 3
} sbd_select_rule;

sbd_status sbd_select(int32_t rule, int32_t batch, int32_t block_k, const float* entropy,
                      const float* confidence, const int32_t* token, float threshold,
                      uint8_t* masked, int32_t* block_tokens, int32_t* n_unmasked,
                      void* stream);

/* ------------------------------------------------------------------------
 * A paged KV cache in 8 bits, for serving batches of uneven requests.
 *
 *   k_cache, v_cache [n_pages, Hkv, P, D]  e4m3 codes (4 exponent bits of bias 7,
 *                                          3 mantissa bits, largest 448, no infinity)
 *   k_scale, v_scale [n_pages, Hkv]        fp32; a value is its page's scale * code
 *   block_table      [B, max_pages] int32  page of a request's tokens p P .. p P + P - 1
 *                                          in column p; -1 where it holds none
 * A token's slot is page * P + its place in the page.  P in {16, 32, 64, 128},
 * D in {64, 128}, n_pages * P < 2^31, n_pages * Hkv < 2^31.
 *
 * One turn of a serving loop: sbd_block_tables gives the requests the pages of
 * the lengths they are to have, sbd_cache_append_q8 fills the new slots, and
 * sbd_block_attention_q8 reads the cache.
 * ---------------------------------------------------------------------- */

/* ------------------------------------------------------------------------
 * Block tables and slot maps from request lengths.  A request grows from
 * cache_len[b] to target_len[b] tokens, or shrinks (0: it ends), holding
 * ceil(length / P) pages before and after.
 *
 *   cache_len, target_len [B] int32       0 .. max_pages * P
 *   block_table [B, max_pages] int32      as it is; not changed
 *   free_pages [n_pages] int32, n_free [1] int32
 *                                         the free pages: a stack of n_free entries;
 *                                         released pages are written above them
 *   block_table_out [B, max_pages] int32  as it is after; -1 past a request's pages
 *   len_out [B] int32                     target_len[b], or cache_len[b] where refused
 *   new_start [B + 1] int32               tokens gained before request b (last: in all)
 *   slot_map [max_new] int32              slots of the new tokens, in request order from
 *                                         new_start[b]; -1 for a refused request's and
 *                                         past the last one
 *   n_free_out [1] int32                  free pages after
 *
 * Released pages (request by request, in a request's order) go on the stack
 * first, the first one topmost; then pages are granted from the top.  Shrinking
 * what a call granted therefore restores the stack.  A request is refused as a
 * whole when the pages of all requests up to and with it exceed the free ones,
 * or its tokens end past max_new; it keeps what it has.  Nothing of block_table
 * is overwritten, so a step in flight may still read it; block_table_out must
 * be other memory.  A length out of range is clamped, its request left as it is,
 * and SBD_DEVERR_CACHE_LEN set.  An n_free out of range is clamped, and a page id
 * out of range, kept, granted or released, becomes -1 in block_table_out or on
 * the stack (it counts as a page there) and the slots of its tokens -1; both set
 * SBD_DEVERR_PAGE.  No workspace.
 * Supported: 1 <= B <= 4096, B * max_pages < 2^31, max_new >= 0.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t batch;      /* B */
  int32_t page_size;  /* P */
  int32_t max_pages;  /* columns of a block table */
  int32_t n_pages;    /* pages of the cache, entries of free_pages */
  int32_t max_new;    /* entries of slot_map */
} sbd_tables_desc;

sbd_status sbd_block_tables(const sbd_tables_desc* desc, const int32_t* cache_len,
                            const int32_t* target_len, const int32_t* block_table,
                            int32_t* free_pages, const int32_t* n_free,
                            int32_t* block_table_out, int32_t* len_out, int32_t* new_start,
                            int32_t* slot_map, int32_t* n_free_out, void* stream);

/* ------------------------------------------------------------------------
 * New keys and values into their slots, in 8 bits.
 *
 *   k_new, v_new [T, Hkv, D]   desc->dtype; token t lies (t / group) * group_stride +
 *                              (t % group) * token_stride elements behind the first
 *                              (heads contiguous), so that they may be slices of a
 *                              fused projection or the leading rows of a block
 *   slot_map [T] int32         slot of every token; negative: not stored
 *   k_cache, v_cache, k_scale, v_scale   written (see above)
 *
 * A run of tokens with consecutive slots of one page is a segment.  For every
 * segment and head, with a = max |x| over its finite elements, s_new is the
 * smallest power of two with a <= 448 s_new (2^-126 at least).  A segment that
 * begins its page (place 0) sets the page's scale to s_new, whatever it was;
 * another one to max(old, s_new), and where that is larger than the old one
 * the codes in the places before it become e4m3(code * old / new).  New codes
 * are e4m3(x / scale), to nearest even; infinities become +-448, NaN stays.
 * A page may receive one segment a call, and its earlier places must hold
 * tokens.  A slot past the cache is not stored and sets SBD_DEVERR_PAGE.
 * Supported: strides that are multiples of 16 bytes; group >= 1.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t tokens;     /* T */
  int32_t group;      /* tokens of a group; T where there is one stride only */
  int32_t n_kv_heads; /* Hkv */
  int32_t head_dim;   /* D */
  int32_t page_size;  /* P */
  int32_t n_pages;
  int32_t dtype;      /* sbd_dtype of k_new and v_new */
  int64_t k_group_stride, k_token_stride; /* elements */
  int64_t v_group_stride, v_token_stride;
} sbd_append_q8_desc;

sbd_status sbd_cache_append_q8(const sbd_append_q8_desc* desc, const void* k_new,
                               const void* v_new, const int32_t* slot_map, void* k_cache,
                               void* v_cache, float* k_scale, float* v_scale, void* stream);

/* ------------------------------------------------------------------------
 * Block attention over the paged 8-bit cache: sbd_block_attention with
 * k_cache and v_cache as above.  Every block row sees the cached keys
 * 0 .. cache_len[b]-1; row i >= n_causal sees all k block keys, row
 * i < n_causal (the first iteration of a block, with the previous block's
 * tokens as its leading rows) the block keys j <= i.  The cache is only read:
 * a previous block enters it with sbd_cache_append_q8.
 *
 *   q [B, k, Hq, D], k_blk, v_blk [B, k, Hkv, D], out [B, k, Hq, D]  desc->dtype
 *   cache_len [B] int32, 0 .. max_pages * P; what the cache holds past it (and
 *   pages it does not reach) is never used and may be NaN
 *
 * Products accumulate in fp32, scales, maxima and sums are fp32.  With bf16
 * activations the tensor cores read the codes; a row of q and of k_blk enters as
 * x = s (hi + lo), two e4m3 codes an element (8 bits of the row's largest; what is
 * not finite becomes NaN), a probability as 8 bits (11 above 32 packed rows k G)
 * relative to its own 256 (128) keys' largest.  Scales are positive.  A value scale
 * enters as fp16, relative to the largest among the same 256 (128) keys: exact for
 * powers of two (the append's) down to 2^-14 of it, below that bits are lost; one
 * that is no power of two costs two roundings of 2^-11.  Key scales stay fp32.
 * With fp32 activations everything is fp32.
 *
 * No workspace: its size is 0 and the arguments are not looked at.
 * A length out of range is clamped and sets SBD_DEVERR_CACHE_LEN; a page id out
 * of range sets SBD_DEVERR_PAGE and its keys and values count as zeros.
 * Supported: 1 <= k <= 32, D in {64, 128}, Hq % Hkv == 0, max_pages * P + k <
 * 2^31; scale 0 is 1/sqrt(D); num_splits 0 picks the key ranges.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t batch, block_k, n_q_heads, n_kv_heads, head_dim;
  int32_t page_size, max_pages, n_pages;
  int32_t dtype;      /* sbd_dtype of q, k_blk, v_blk and out */
  int32_t n_causal;   /* leading causal block rows, 0 .. k */
  float scale;
  int32_t num_splits;
} sbd_attn_q8_desc;

size_t sbd_block_attention_q8_workspace_size(const sbd_attn_q8_desc* desc);
sbd_status sbd_block_attention_q8(const sbd_attn_q8_desc* desc, const void* q,
                                  const void* k_cache, const void* v_cache,
                                  const float* k_scale, const float* v_scale,
                                  const int32_t* block_table, const int32_t* cache_len,
                                  const void* k_blk, const void* v_blk, void* out,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * A turn of drafted decoding over the paged 8-bit cache.
 *
 * Drafted tokens (from the k marginals of a block forward, or from another
 * model) are checked against the model's own next-token distribution in one
 * forward.  A request's rows form a tree of n nodes: node 0 is the last token
 * that was kept, not in the cache yet, and node i > 0 a drafted token that
 * follows node parent[b, i] < i.  A node with a negative parent begins a tree of
 * its own: padding, which no walk from node 0 reaches.  A chain is parent = i - 1.
 *
 *   sbd_qk_norm_rope           the nodes' fused projection becomes normed and
 *                              rotated queries and keys, and values
 *   sbd_tree_attention_q8      a node sees the cache, itself and its ancestors
 *   sbd_verify_tree            which nodes are accepted, and the token after them
 *   sbd_block_tables           pages for the accepted nodes: target_len =
 *                              cache_len + count
 *   sbd_cache_append_path_q8   their keys and values enter the cache
 *
 * A parent that is not below its node, a drafted token outside [0, vocab) or a
 * path entry outside [0, n) sets SBD_DEVERR_TREE; the node then begins a tree of
 * its own, the token is passed over, the entry is not stored.
 * ---------------------------------------------------------------------- */

/* ------------------------------------------------------------------------
 * Queries and keys normed by head and rotated by position, values copied:
 *   y = w * x / sqrt(mean_d x_d^2 + eps)      (w NULL: y = x)
 *   pair j < R / 2 of y turns by the angle a = positions[t] * inv_freq[j]:
 *     (y1 cos a - y2 sin a, y2 cos a + y1 sin a)
 * where pair j is (j, j + R / 2), or (2 j, 2 j + 1) where desc->interleaved; what
 * lies past the first R = rotary_dim dimensions is not turned.  One rounding at the
 * end; squares may leave fp32's range.  Angles are within 2^-26 of a turn, and 2^-52 of their whole turns where those are
 * more than 2^26 (the product is kept in fixed point, whole turns dropped).
 *
 *   q [T, Hq, D], k, v [T, Hkv, D]   desc->dtype; token t lies (t / group) *
 *                                    group_stride + (t % group) * token_stride
 *                                    elements behind the first (heads contiguous)
 *   positions [T] int32              NULL iff rotary_dim == 0
 *   inv_freq [R / 2] fp32            finite; NULL iff rotary_dim == 0
 *   q_weight, k_weight [D]           desc->dtype; NULL: not normed
 *   q_out [T, Hq, D], k_out, v_out [T, Hkv, D]   contiguous, other memory than the
 *                                    inputs; v and v_out may be NULL (both)
 * Supported: D in {64, 128}, R a multiple of 16, 0 <= R <= D, eps >= 0 and
 * finite, strides that are multiples of 16 bytes, group >= 1.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t tokens;       /* T */
  int32_t group;        /* tokens of a group; T where there is one stride only */
  int32_t n_q_heads;    /* Hq */
  int32_t n_kv_heads;   /* Hkv */
  int32_t head_dim;     /* D */
  int32_t rotary_dim;   /* R */
  int32_t interleaved;  /* pairs are neighbours */
  int32_t dtype;        /* sbd_dtype */
  float eps;
  int64_t q_group_stride, q_token_stride; /* elements */
  int64_t k_group_stride, k_token_stride;
  int64_t v_group_stride, v_token_stride;
} sbd_norm_rope_desc;

sbd_status sbd_qk_norm_rope(const sbd_norm_rope_desc* desc, const void* q, const void* k,
                            const void* v, const int32_t* positions, const float* inv_freq,
                            const void* q_weight, const void* k_weight, void* q_out, void* k_out,
                            void* v_out, void* stream);

/* ------------------------------------------------------------------------
 * sbd_block_attention_q8 for a tree: block row i sees the cached keys and, of
 * the block keys, its own and its ancestors'.  desc->block_k is the number of
 * nodes, 1 .. 64, and desc->n_causal must be 0.
 *   parent [B, n] int32 (device)
 * Everything else, the workspace (none) and the errors are those of
 * sbd_block_attention_q8.
 * ---------------------------------------------------------------------- */
size_t sbd_tree_attention_q8_workspace_size(const sbd_attn_q8_desc* desc);
sbd_status sbd_tree_attention_q8(const sbd_attn_q8_desc* desc, const void* q, const void* k_cache,
                                 const void* v_cache, const float* k_scale, const float* v_scale,
                                 const int32_t* block_table, const int32_t* cache_len,
                                 const void* k_blk, const void* v_blk, const int32_t* parent,
                                 void* out, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Verification of drafted tokens, from given random numbers.  Per request, with
 * p_i = softmax(target_logits[b, i] / tau) and q_i = softmax(draft_logits[b, i] / tau):
 *
 *   node = 0; r = p_0
 *   for every child c of node, in index order, with its token x = token[b, c]:
 *     accept c iff uniform[b, c] * q_node(x) < r(x):  node = c, r = p_c, go on there;
 *     else r = max(r - q_node, 0), normalised (r stays where nothing is left)
 *   where no child is accepted, or there is none: the last token is
 *     argmax_v (ln r(v) + gumbel[b, v]), lowest v on ties
 *
 * The tokens that come out are distributed as p if a node's children were drawn from
 * q_node one by one, uniform is uniform on [0, 1) and gumbel is standard Gumbel noise
 * (sbd_gumbel_philox).  draft_logits NULL: a drafted token was not drawn but given, q is
 * 1 there and 0 elsewhere.  tau = 0: p is 1 at the largest logit (lowest index of equal
 * ones; NaN is below all); draft_logits, uniform and gumbel are not read.  In a
 * softmax only distances from the row's largest logit count, of any size; NaN counts as -inf.
 * What is masked with -inf or a type's lowest value never comes out beside an ordinary logit;
 * in a row of nothing but -inf all count alike, and logits of +inf share all.
 *
 *   target_logits, draft_logits [B, n, V]   desc->dtype; draft row i: what i's children
 *                                           were drawn from (read where it has some)
 *   parent, token [B, n] int32              token[b, 0] is not read
 *   uniform [B, n] fp32, gumbel [B, V] fp32 NULL iff tau == 0
 *   path [B, n] int32 out      accepted nodes from node 0 on, then -1
 *   out_tokens [B, n] int32 out  the tokens of path[1], ..., then the last token, then -1
 *   logprob [B, n] fp32 out    ln p of each of them (at temperature 1 where tau = 0), then 0
 *   count [B] int32 out        nodes on the path = tokens that come out, 1 .. n
 *
 * Exponentials and sums in fp32: what is below 2^-126 of a row may count nothing.
 * No workspace: its size is 0.  Rows that the walk does not come to change nothing.
 * Supported: 1 <= n <= 64, 1 <= V <= 2^24, B <= 65535, tau = 0 or 2^-20 <= tau <= 2^20.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t batch;   /* B */
  int32_t nodes;   /* n */
  int32_t vocab;   /* V */
  int32_t dtype;   /* sbd_dtype of the logits */
} sbd_verify_desc;

size_t sbd_verify_tree_workspace_size(const sbd_verify_desc* desc);
sbd_status sbd_verify_tree(const sbd_verify_desc* desc, const void* target_logits,
                           const void* draft_logits, const int32_t* parent, const int32_t* token,
                           const float* uniform, const float* gumbel, float tau, int32_t* path,
                           int32_t* out_tokens, float* logprob, int32_t* count, void* workspace,
                           size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * The keys and values of accepted nodes into their slots: sbd_cache_append_q8 for
 * nodes that do not lie one behind the other.  Request b gains new_start[b + 1] -
 * new_start[b] tokens (n at most), its j-th in slot slot_map[new_start[b] + j] with the
 * keys and values of node path[b, j].
 *
 *   k_new, v_new [B, n, Hkv, D]   desc->dtype; node i of request b lies b *
 *                                 batch_stride + i * node_stride elements behind the
 *                                 first (heads contiguous)
 *   path [B, n] int32, new_start [B + 1] int32, slot_map [max_new] int32
 *                                 as sbd_verify_tree and sbd_block_tables give them
 *
 * Segments, scales, codes and errors are those of sbd_cache_append_q8; a slot that is
 * negative or past max_new is not stored.  Where that, or an entry that is not stored, cuts a
 * run in two, the second segment enters as by a call after the first's.  Requests do not
 * share the pages they append to.
 * Supported: 1 <= n <= 64, B <= 65535, strides that are multiples of 16 bytes.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t batch, nodes;   /* B, n */
  int32_t n_kv_heads, head_dim, page_size, n_pages;
  int32_t max_new;        /* entries of slot_map */
  int32_t dtype;          /* sbd_dtype of k_new and v_new */
  int64_t k_batch_stride, k_node_stride; /* elements */
  int64_t v_batch_stride, v_node_stride;
} sbd_append_path_desc;

sbd_status sbd_cache_append_path_q8(const sbd_append_path_desc* desc, const void* k_new,
                                    const void* v_new, const int32_t* path,
                                    const int32_t* new_start, const int32_t* slot_map,
                                    void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                                    void* stream);

/* Status name ("SBD_OK", ...). Never NULL. */
const char* sbd_status_string(sbd_status status);

/* Detail of the last failing call on this thread ("" if none). */
const char* sbd_last_error(void);

/* Reads and clears the device error word of the current device
 * (synchronises the device).  *code = 0 when no kernel recorded a fault;
 * otherwise a bit set of SBD_DEVERR_* values. */
sbd_status sbd_device_error(int32_t* code);

#define SBD_DEVERR_CACHE_LEN 1   /* a cache_len entry was outside [0, Lmax] */
#define SBD_DEVERR_TIMEOUT 2     /* a bounded wait inside a kernel gave up  */
#define SBD_DEVERR_ROWS 4        /* more masked rows than the head supports */
#define SBD_DEVERR_PAGE 8        /* a page id, slot or free-page count was out of range */
#define SBD_DEVERR_TREE 16       /* a node's parent, drafted token or path entry was out of range */

/* Library version, major * 10000 + minor * 100 + patch. */
int32_t sbd_version(void);

#ifdef __cplusplus
}
#endif

#endif /* SBD_H */
