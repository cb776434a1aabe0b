/*
 * jetlong.h -- C ABI of libjetlong.so: fused causal bifocal-RoPE attention
 * (Jet-Long, arXiv 2607.07740) for AMD Instinct MI355X (gfx950).
 *
 * The method (Sec. 3, Eq. (1)): a query at position q attends to a key at
 * position k <= q with the score
 *     <R(q) x_q, R(k) x_k>            if q - k <= w_local   (local view)
 *     <R(f(q)) x_q, R(f(k)) x_k>      if q - k >  w_local   (remote view)
 * where R(p) is the RoPE rotation to position p, f(x) = floor(x / G) (Eq. (3))
 * and G = max(1, ceil(L / w_pretrained)) (Eq. (2)) for the current length L.
 * The remote rotation is applied on the fly to raw (pre-RoPE) Q/K as the
 * correction rotation of Sec. 3.2 (Eqs. (5)-(6)); no rotated copy of K is ever
 * written.  Local and remote partial softmax states are merged by the
 * max-shifted, linear-space rule of Sec. 3.3, Eq. (7).
 *
 * Conventions shared by every entry point:
 *  - Tensors are DEVICE pointers to contiguous row-major storage; "bf16" is
 *    IEEE bfloat16 stored as 16-bit words.  Every tensor pointer must be
 *    16-byte aligned.  The caller owns all tensors and workspaces.
 *  - RoPE uses the rotate-half pairing (element i with i + head_dim/2) and
 *    frequencies omega_i = rope_theta^(-2i/head_dim); positions are 0-based;
 *    the softmax scale is 1/sqrt(head_dim).
 *  - Grouped-query attention: query head h reads kv head h / (Hq / Hkv).
 *  - head_dim must be 128 (other values return JL_ERR_UNSUPPORTED).
 *  - Calls are asynchronous on `stream` (a hipStream_t; NULL = the null
 *    stream).  Arguments are validated on the host before anything is
 *    launched; on any error nothing is written and nothing is launched.
 *  - Where a call allocates or waits.  The library keeps per-device caches
 *    that a call may have to build or grow; only then does it allocate and
 *    wait, and a later call with the same shape does neither (nor one with a
 *    smaller shape, but for the prefill scratch: a call that cuts its blocks
 *    needs some where a larger call that fills the CUs needs none):
 *      - the RoPE cos/sin table (per device and rope_theta, grown by
 *        doubling to cover the call's positions): every prefill, decode and
 *        block score entry point; growing allocates and waits for `stream`;
 *      - the prefill scratch (per device and stream): the _varlen forms with
 *        more than 64 sequences, or the frequency map past the window, and of
 *        jl_bifocal_prefill, jl_rope_attention, their _map and _chunk forms
 *        the calls whose query blocks leave CUs idle (see there); growing
 *        waits for `stream`, frees the old buffer and allocates.  Under
 *        stream capture it does not grow: a call that would cut its blocks
 *        runs them whole, a packed call that needs more returns JL_ERR_HIP.
 *        A buffer that a captured call uses is kept until
 *        jl_release_caches;
 *      - the frequency-map table (one per device): jl_bifocal_prefill_map
 *        with JL_REMOTE_FREQ; a new (rope_theta, L, w_pretrained) waits for
 *        the whole device, then rebuilds the table in place, or in a buffer
 *        of at least twice the capacity when L does not fit.
 *    The literal, decode and _varlen_paged entry points use the caller's
 *    workspace and allocate nothing else.  jl_release_caches frees every cache.
 *  - Thread safety: calls may come from several host threads; the library's
 *    shared state (the caches above and the debug settings below) is guarded
 *    by mutexes.  Calls that share output buffers must be ordered by the
 *    caller.
 *  - Status codes are returned; no exception crosses the ABI and nothing
 *    aborts.  jl_last_error() gives a human-readable detail for the calling
 *    thread's most recent failure.
 */
#ifndef JETLONG_H
#define JETLONG_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  JL_OK = 0,
  JL_ERR_INVALID_ARG = 1, /* bad shape, pointer, alignment or window value      */
  JL_ERR_UNSUPPORTED = 2, /* valid but not built (head_dim != 128, GQA group)   */
  JL_ERR_WORKSPACE = 3,   /* workspace missing or smaller than required         */
  JL_ERR_HIP = 4          /* HIP runtime error (launch, allocation, no device)  */
};

/* Name of a status code ("JL_OK", ...); never NULL. */
const char* jl_status_string(int status);

/* Detail message of the calling thread's last failed call ("" if none). */
const char* jl_last_error(void);

/* ABI version: major * 10000 + minor * 100 + patch. */
int jl_version(void);

/*
 * Group size of Sec. 3.1, Eq. (2), computed on the host:
 * G = max(1, ceil(L / w_pretrained)).  Returns -1 if L < 1 or w_pretrained < 1.
 */
int64_t jl_group_size(int64_t L, int64_t w_pretrained);

/*
 * Bifocal prefill (Sec. 3, Eq. (1); merge of Sec. 3.3, Eq. (7)).
 *   q   bf16 [B, L, Hq, head_dim]   raw (pre-RoPE) queries, position = row index
 *   k   bf16 [B, L, Hkv, head_dim]  raw (pre-RoPE) keys
 *   v   bf16 [B, L, Hkv, head_dim]
 *   o   bf16 [B, L, Hq, head_dim]   output (written)
 *   lse fp32 [B, Hq, L] or NULL     natural-log softmax normaliser per row
 * One G for the whole call, from this call's L (all B sequences share L).
 * w_pretrained >= 1, w_local >= 0; keys with q - k <= w_local use the base
 * rotation, older keys the remote one.  When G == 1 the output equals
 * jl_rope_attention bit for bit (the method reduces to the base model).
 * Requires Hq % Hkv == 0, 256 % (Hq / Hkv) == 0 and B * Hkv <= 65535.
 * K is read raw: the keys of each 64-key tile are loaded into registers and
 * rotated to the view of the visit (R(k) x_k on the band, R(f(k)) x_k beyond
 * it, Sec. 3.2); the rotated tile is kept only in on-chip memory and no
 * rotated key is written anywhere.
 * A call with fewer query blocks than CUs (a block is 256 / (Hq / Hkv) query
 * positions of one sequence and kv head), or whose blocks make up a few whole
 * waves of the CUs and a small rest, cuts the idle CUs' share of its blocks
 * into parts of the key range and merges their fp32 states (133 KB per part, at
 * most 16 parts a block, in the prefill scratch); others need no scratch.  So the
 * bits of such a call depend on the count of CUs and on the size of the batch, by
 * the order of the fp32 sums over the parts.
 * q, k, v are only read.
 */
int jl_bifocal_prefill(const void* q, const void* k, const void* v, void* o, float* lse, int B,
                       int Hq, int Hkv, int L, int head_dim, double rope_theta, int w_pretrained,
                       int w_local, void* stream);

/* Remote-view maps for jl_bifocal_prefill_map. */
enum {
  JL_REMOTE_ALIAS = 0, /* Eq. (3): remote positions f(x) = floor(x / G), base frequencies */
  JL_REMOTE_FREQ = 1   /* Sec. 4.5 / Table 6 ablation: positions kept, frequencies rescaled */
};

/*
 * jl_bifocal_prefill with a choice of remote view (Sec. 4.5, Table 6, the
 * ablation that replaces position aliasing by frequency interpolation).
 *   remote_map = JL_REMOTE_ALIAS  identical to jl_bifocal_prefill;
 *   remote_map = JL_REMOTE_FREQ   the remote view keeps each query and key at
 *     its own position and rotates it with rescaled frequencies omega'_i: with
 *     s = max(1, L / w_pretrained) and r_i = w_pretrained * omega_i / (2 pi) the
 *     number of turns pair i completes over the pretraining window,
 *     gamma_i = clamp((r_i - 1) / 31, 0, 1) and
 *     omega'_i = (1 - gamma_i) omega_i / s + gamma_i omega_i (YaRN's per-pair
 *     ramp, alpha = 1, beta = 32; no attention temperature).  The local window,
 *     the masks and the Eq. (7) merge are unchanged.
 * When L <= w_pretrained (s = 1, G = 1) both maps run the vanilla kernel.
 * The frequency map keeps one library-owned table of cos/sin(p * omega'_i),
 * L x 512 bytes per device, for the last (rope_theta, L, w_pretrained) used;
 * a new configuration waits for the whole device and rebuilds that table in
 * place (in a new buffer of at least twice the capacity when L does not fit,
 * the old one freed), then waits for the stream.  jl_release_caches frees it.
 * Other arguments, scratch and errors as in jl_bifocal_prefill; remote_map
 * outside {0, 1} -> JL_ERR_INVALID_ARG.
 */
int jl_bifocal_prefill_map(const void* q, const void* k, const void* v, void* o, float* lse,
                           int B, int Hq, int Hkv, int L, int head_dim, double rope_theta,
                           int w_pretrained, int w_local, int remote_map, void* stream);

/*
 * Continued (chunked) prefill over an existing raw cache (Sec. 3.2: the cache
 * keeps keys at base coordinates and is never rewritten when G changes).
 *   q       bf16 [B, n_queries, Hq, head_dim]  raw queries at positions
 *                                              q_start .. q_start + n_queries - 1
 *   k_cache bf16 [B, max_len, Hkv, head_dim]   raw keys; rows [0, q_start + n_queries)
 *   v_cache bf16 [B, max_len, Hkv, head_dim]   must hold the chunk's own keys too
 *   o       bf16 [B, n_queries, Hq, head_dim]  output (written)
 *   lse     fp32 [B, Hq, n_queries] or NULL
 * The call's sequence length is L = q_start + n_queries: G = max(1,
 * ceil(L / w_pretrained)) for every query of the chunk, as in a prefill of
 * length L, so the output equals rows q_start .. L - 1 of
 * jl_bifocal_prefill over the first L cache rows: bit for bit where neither
 * call cuts its blocks (see there), and up to the order of the fp32 sums over
 * the parts otherwise.  The caches are only read:
 * keys are rotated on chip per visit, as in jl_bifocal_prefill.  Requires 0 <= q_start, n_queries >= 1,
 * q_start + n_queries <= max_len; other requirements and errors as in
 * jl_bifocal_prefill.
 */
int jl_bifocal_prefill_chunk(const void* q, const void* k_cache, const void* v_cache, void* o,
                             float* lse, int B, int Hq, int Hkv, int q_start, int n_queries,
                             int max_len, int head_dim, double rope_theta, int w_pretrained,
                             int w_local, void* stream);

/* The vanilla counterpart of jl_bifocal_prefill_chunk (base rotation only). */
int jl_rope_attention_chunk(const void* q, const void* k_cache, const void* v_cache, void* o,
                            float* lse, int B, int Hq, int Hkv, int q_start, int n_queries,
                            int max_len, int head_dim, double rope_theta, void* stream);

/*
 * jl_bifocal_prefill_chunk over paged caches (Sec. 3.2: the raw cache is
 * read, never rewritten, whatever G the chunk's length gives).
 *   k_pages, v_pages bf16 [n_pages, page_size, Hkv, head_dim] device pools
 *   block_table int32 [B, max_pages] (device): key x of sequence b is row
 *               x % page_size of page block_table[b][x / page_size]
 * The pages of keys [0, q_start + n_queries) must be written (the chunk's own
 * keys included); entries outside [0, n_pages) are clamped into the pool
 * (garbage in, no fault).  The output equals jl_bifocal_prefill_chunk's on a
 * dense cache holding the same rows, bit for bit.  page_size must be a power
 * of two, max_pages, n_pages >= 1, and q_start + n_queries <=
 * max_pages * page_size (else JL_ERR_INVALID_ARG); page_size < 64 (a page
 * must hold whole 64-key tiles) or more than 4096 pages per sequence (the
 * attention kernel keeps the list in LDS) -> JL_ERR_UNSUPPORTED.  q, o, lse,
 * scratch and the other arguments and errors as in jl_bifocal_prefill_chunk.
 */
int jl_bifocal_prefill_chunk_paged(const void* q, const void* k_pages, const void* v_pages,
                                   const int32_t* block_table, int max_pages, int page_size,
                                   int n_pages, void* o, float* lse, int B, int Hq, int Hkv,
                                   int q_start, int n_queries, int head_dim, double rope_theta,
                                   int w_pretrained, int w_local, void* stream);

/* The vanilla counterpart of jl_bifocal_prefill_chunk_paged. */
int jl_rope_attention_chunk_paged(const void* q, const void* k_pages, const void* v_pages,
                                  const int32_t* block_table, int max_pages, int page_size,
                                  int n_pages, void* o, float* lse, int B, int Hq, int Hkv,
                                  int q_start, int n_queries, int head_dim, double rope_theta,
                                  void* stream);

/*
 * Packed (variable-length) bifocal prefill: B independent sequences of
 * different lengths in one call, each computed exactly as jl_bifocal_prefill
 * would compute it alone (where that call cuts no block) -- its own L,
 * G = max(1, ceil(L / w_pretrained)) (Eq. (2)), positions 0 .. L - 1, Eq. (3)
 * remote positions and the Eq. (7) bifocal result (a sequence with G = 1 gets
 * the base model, as there).
 *   q, o: bf16 [total_tokens, Hq, head_dim]; k, v: bf16 [total_tokens, Hkv,
 *     head_dim] (raw, before RoPE); sequence s holds rows
 *     cu_seqlens[s] .. cu_seqlens[s + 1] - 1.
 *   lse: NULL or fp32 [Hq, total_tokens], natural-log row sums.
 *   cu_seqlens: DEVICE int32 [B + 1], non-decreasing from 0 to total_tokens
 *     (read by the kernels only; the call does not synchronise).
 *   max_seqlen: an upper bound of the sequence lengths; sets the RoPE table
 *     size.  Longer sequences are cut to their first max_seqlen rows.
 * Malformed cu_seqlens cannot cause an access outside the tensors: bounds are
 * clamped into [0, total_tokens] (a decreasing step gives an empty sequence)
 * and a sequence whose work would not fit the lists sized for well-formed
 * input is skipped; output rows of skipped, cut or uncovered positions are
 * left as they were.  Scratch (the library's, per stream): none up to 64
 * sequences, beyond that a work list of 16 bytes per query block.  Other
 * requirements and errors as in jl_bifocal_prefill; only the Eq. (3) map.
 */
int jl_bifocal_prefill_varlen(const void* q, const void* k, const void* v, void* o, float* lse,
                              const int32_t* cu_seqlens, int B, int total_tokens, int max_seqlen,
                              int Hq, int Hkv, int head_dim, double rope_theta, int w_pretrained,
                              int w_local, void* stream);

/*
 * jl_bifocal_prefill_varlen with a choice of remote map (Sec. 4.5, Tab. 6),
 * as jl_bifocal_prefill_map offers it for one sequence.  JL_REMOTE_ALIAS is
 * jl_bifocal_prefill_varlen bit for bit; JL_REMOTE_FREQ gives every sequence
 * the frequency map of its own length: factor s = max(1, L / w_pretrained),
 * positions unchanged, each sequence equal bit for bit to jl_bifocal_prefill_map
 * on that sequence alone (where that call cuts no block, see
 * jl_bifocal_prefill).  The per-sequence tables (768 bytes per token) are
 * built on the device into the library scratch.  Other arguments and errors
 * as in jl_bifocal_prefill_varlen; remote_map outside {0, 1} ->
 * JL_ERR_INVALID_ARG.
 */
int jl_bifocal_prefill_varlen_map(const void* q, const void* k, const void* v, void* o,
                                  float* lse, const int32_t* cu_seqlens, int B, int total_tokens,
                                  int max_seqlen, int Hq, int Hkv, int head_dim, double rope_theta,
                                  int w_pretrained, int w_local, int remote_map, void* stream);

/* The vanilla counterpart of jl_bifocal_prefill_varlen (base rotation only). */
int jl_rope_attention_varlen(const void* q, const void* k, const void* v, void* o, float* lse,
                             const int32_t* cu_seqlens, int B, int total_tokens, int max_seqlen,
                             int Hq, int Hkv, int head_dim, double rope_theta, void* stream);

/*
 * Vanilla causal RoPE attention with the same tiling and RoPE of raw Q/K at
 * base positions: the base model of Sec. 3 and the denominator of the
 * overhead measurements.  Arguments and scratch as in jl_bifocal_prefill.
 */
int jl_rope_attention(const void* q, const void* k, const void* v, void* o, float* lse, int B,
                      int Hq, int Hkv, int L, int head_dim, double rope_theta, void* stream);

/*
 * Bytes of device workspace jl_bifocal_prefill_literal needs for this shape:
 * 3 * B * L * Hq * head_dim * 4 (the window outputs) + the window LSEs
 * (3 * B * Hq * L * 4, rounded up to 256) + B * Hkv * ceil(L / 64) * 16 KB +
 * 256 + 4 * B * Hkv * L (a region that is not used and stays part of the size).
 * Returns 0 for invalid arguments.
 */
size_t jl_prefill_literal_workspace_bytes(int B, int Hq, int Hkv, int L, int head_dim);

/*
 * Bifocal prefill with Eq. (7) of Sec. 3.3 taken literally: the three
 * attention calls A (band q - k <= w_local, base rotation), B (all causal
 * keys, remote rotation) and C (band, remote rotation) run as three calls
 * of the attention kernel (each as the fused call runs: a fast pass, then the
 * checked pass of the blocks that need it), each writing its normalised output
 * O_X and its natural-log LSE_X, and a fourth kernel merges them per row with
 *   M = max(LSE_A, LSE_B, LSE_C), W_X = exp(LSE_X - M),
 *   O = (W_A O_A + (W_B O_B - W_C O_C)) / (W_A + (W_B - W_C)),
 *   lse = M + ln(W_A + (W_B - W_C)),
 * in fp32.  This is the unfused variant the fused kernel of
 * jl_bifocal_prefill replaces; the two agree up to rounding, except where the
 * band dominates window B so strongly that the subtraction cancels (the
 * literal form loses precision there; the fused form does not subtract).
 * Arguments as in jl_bifocal_prefill, plus
 *   workspace, workspace_bytes: device memory of at least
 *     jl_prefill_literal_workspace_bytes(B, Hq, Hkv, L, head_dim) bytes,
 *     256-byte aligned, owned by the caller; contents on entry do not matter.
 *     On return (after the stream completes) it holds, for X = A, B, C
 *     (x = 0, 1, 2), O_X as fp32 [B, L, Hq, head_dim] at float offset
 *     x * B * L * Hq * head_dim, and LSE_X as fp32 [B, Hq, L] at float offset
 *     3 * B * L * Hq * head_dim + x * B * Hq * L.
 * When G == 1 the call runs the vanilla kernel, as jl_bifocal_prefill does, but
 * never cuts its blocks: the same bits where that call cuts none, and equal up to
 * the order of the fp32 sums over the parts otherwise.  The window outputs and
 * LSEs are left unwritten.  Either way no library
 * scratch is used (only the RoPE table cache, as for every entry point).
 */
int jl_bifocal_prefill_literal(const void* q, const void* k, const void* v, void* o, float* lse,
                               int B, int Hq, int Hkv, int L, int head_dim, double rope_theta,
                               int w_pretrained, int w_local, void* workspace,
                               size_t workspace_bytes, void* stream);

/*
 * Bytes of device workspace the decode entry points use for this shape
 * (split-K partial softmax states).  Returns 0 for invalid arguments.
 * A smaller workspace is accepted down to B * Hq * n * 528 bytes with n =
 * min(128, ceil(max_len / 16)) up to B = 64 and n = min(ceil(256 / (B *
 * ceil(Hkv / 4))), 128, ceil(max_len / 16)) beyond: the call then runs fewer
 * workgroups, or the batch in parts one after another, and its results equal
 * those with the full workspace up to the splits of the softmax sums.
 */
size_t jl_decode_workspace_bytes(int B, int Hq, int Hkv, int max_len, int head_dim);

/*
 * Bifocal single-query decode on a raw KV cache (Sec. 3.2, Eqs. (4)-(6)).
 *   q        bf16 [B, Hq, head_dim]           raw new queries; the query of
 *                                              sequence b sits at position
 *                                              kv_lens[b] - 1
 *   k_cache  bf16 [B, max_len, Hkv, head_dim] raw (pre-RoPE) keys, the new
 *                                              token already appended
 *   v_cache  bf16 [B, max_len, Hkv, head_dim]
 *   kv_lens  int32 [B] DEVICE array, 1 <= kv_lens[b] <= max_len; positions
 *            at or past kv_lens[b] are never read.  The host cannot check
 *            it: a value below 1 is read as 1 and one past max_len as
 *            max_len, so a bad length gives wrong values, never an
 *            out-of-bounds read
 *   o        bf16 [B, Hq, head_dim] output (written)
 *   workspace, workspace_bytes: device scratch of
 *            jl_decode_workspace_bytes(B, Hq, Hkv, max_len, head_dim) bytes
 *            (or somewhat less, see there), 16-byte aligned; its contents on
 *            entry do not matter.
 * G is taken per sequence from L = kv_lens[b] on the device, so one cache
 * serves every length and G change without being rewritten.
 * Requires Hq % Hkv == 0 and Hq / Hkv <= 8; max_len > 8388608 (2^23)
 * returns JL_ERR_UNSUPPORTED.
 */
int jl_bifocal_decode(const void* q, const void* k_cache, const void* v_cache,
                      const int32_t* kv_lens, int max_len, void* o, int B, int Hq, int Hkv,
                      int head_dim, double rope_theta, int w_pretrained, int w_local,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * jl_bifocal_decode for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc).  Same arguments and results, bit for bit, without the
 * workspace: the split states and the fp32 cos/sin table live in one fixed
 * device array that the library holds on each device it runs on until the
 * process ends (93 MiB: the table of positions [0, 131072) and 29 MiB of
 * states).  No call allocates or frees device memory.
 *   max_len > 131072, or more than 24 MiB of states, counted as the smallest
 *   workspace is (see jl_decode_workspace_bytes) -> JL_ERR_UNSUPPORTED, checked on the host before any device work.
 * The first call on a device for a given rope_theta builds the table and
 * waits for it on `stream` (make that call outside graph capture); later
 * calls with that theta launch the two decode kernels only.  Every call on a
 * device shares that device's array, so calls that overlap on one device
 * (other streams, other threads) race; serialise them.  Other requirements
 * and errors as in jl_bifocal_decode.
 */
int jl_bifocal_decode_noalloc(const void* q, const void* k_cache, const void* v_cache,
                              const int32_t* kv_lens, int max_len, void* o, int B, int Hq,
                              int Hkv, int head_dim, double rope_theta, int w_pretrained,
                              int w_local, void* stream);

/* Vanilla RoPE decode with the same kernels (base rotation for every key). */
int jl_rope_attention_decode(const void* q, const void* k_cache, const void* v_cache,
                             const int32_t* kv_lens, int max_len, void* o, int B, int Hq,
                             int Hkv, int head_dim, double rope_theta, void* workspace,
                             size_t workspace_bytes, void* stream);

/*
 * Bytes of workspace jl_bifocal_decode_map needs: jl_decode_workspace_bytes,
 * for either remote map.  Returns 0 for invalid arguments.
 */
size_t jl_decode_map_workspace_bytes(int B, int Hq, int Hkv, int max_len, int head_dim,
                                     int remote_map);

/*
 * jl_bifocal_decode with a choice of remote map (the Sec. 4.5 / Tab. 6
 * ablation, as jl_bifocal_prefill_map does for prefill).
 *   remote_map  JL_REMOTE_ALIAS: identical to jl_bifocal_decode.
 *               JL_REMOTE_FREQ: remote pairs (q - k > w_local) keep their
 *               positions and rotate by omega'_i = (1 - gamma_i) omega_i / s +
 *               gamma_i omega_i (YaRN's ramp, alpha = 1, beta = 32, no
 *               temperature), with s = max(1, kv_lens[b] / w_pretrained) per
 *               sequence, so a ragged batch mixes factors the way it mixes G.
 *               Each workgroup forms the cos/sin rows it needs from its
 *               sequence's length (which lives on the device).
 *   workspace   at least jl_decode_map_workspace_bytes(..., remote_map) bytes,
 *               16-byte aligned, contents on entry irrelevant.
 * Other arguments, requirements and errors as in jl_bifocal_decode.
 */
int jl_bifocal_decode_map(const void* q, const void* k_cache, const void* v_cache,
                          const int32_t* kv_lens, int max_len, void* o, int B, int Hq, int Hkv,
                          int head_dim, double rope_theta, int w_pretrained, int w_local,
                          int remote_map, void* workspace, size_t workspace_bytes, void* stream);

/*
 * jl_bifocal_decode on a paged cache: keys and values live in pools of
 * fixed-size pages and each sequence lists its pages in a block table.
 *   k_pages, v_pages bf16 [n_pages, page_size, Hkv, head_dim] raw pools
 *   block_table      int32 [B, max_pages] DEVICE array: key k of sequence b
 *                    is row k % page_size of page block_table[b][k / page_size]
 *   kv_lens          int32 [B] DEVICE array, 1 <= kv_lens[b] <= max_pages * page_size
 *                    (clamped into that range as in jl_bifocal_decode)
 * page_size is a power of two, at least 16 (a 16-key step of the kernel never
 * straddles two pages).  Page indices outside [0, n_pages) are clamped into
 * the pool, so a bad table gives wrong values, never an out-of-bounds read.
 * Workspace as for jl_bifocal_decode with max_len = max_pages * page_size.
 * Other arguments, requirements and errors as in jl_bifocal_decode.
 */
int jl_bifocal_decode_paged(const void* q, const void* k_pages, const void* v_pages,
                            const int32_t* block_table, int max_pages, int page_size, int n_pages,
                            const int32_t* kv_lens, void* o, int B, int Hq, int Hkv,
                            int head_dim, double rope_theta, int w_pretrained, int w_local,
                            void* workspace, size_t workspace_bytes, void* stream);

/*
 * jl_bifocal_decode_paged with a choice of remote map, as jl_bifocal_decode_map
 * offers it for dense caches: remote_map JL_REMOTE_ALIAS is
 * jl_bifocal_decode_paged bit for bit, JL_REMOTE_FREQ the Sec. 4.5 frequency
 * map with each sequence's factor from its own kv_len.  The workspace must
 * hold jl_decode_map_workspace_bytes(B, Hq, Hkv, max_pages * page_size,
 * head_dim, remote_map) bytes.  Other arguments and errors as in
 * jl_bifocal_decode_paged; remote_map outside {0, 1} -> JL_ERR_INVALID_ARG.
 */
int jl_bifocal_decode_paged_map(const void* q, const void* k_pages, const void* v_pages,
                                const int32_t* block_table, int max_pages, int page_size,
                                int n_pages, const int32_t* kv_lens, void* o, int B, int Hq,
                                int Hkv, int head_dim, double rope_theta, int w_pretrained,
                                int w_local, int remote_map, void* workspace,
                                size_t workspace_bytes, void* stream);

/* The vanilla counterpart of jl_bifocal_decode_paged. */
int jl_rope_attention_decode_paged(const void* q, const void* k_pages, const void* v_pages,
                                   const int32_t* block_table, int max_pages, int page_size,
                                   int n_pages, const int32_t* kv_lens, void* o, int B, int Hq,
                                   int Hkv, int head_dim, double rope_theta, void* workspace,
                                   size_t workspace_bytes, void* stream);

/*
 * ---- 8-bit cache -----------------------------------------------------------
 * Keys (raw, before RoPE) and values held as OCP e4m3 in blocks of 64 tokens
 * of one kv head, with one fp32 power-of-two scale per block for K and one for
 * V: a value is its scale times its e4m3 number.  256 bytes per token and kv
 * head instead of 512.  Pools, all on one device and owned by the caller:
 *   k, v             uint8 [n_pages, Hkv, page_size, head_dim]: per (page, head)
 *                    page_size / 64 images of 8192 bytes.  Inside an image
 *     K  key 32 a + 16 t + r,         channel 64 p + 32 u + 8 g + j  at [a 2][t 2][u 2][g 4][r 16][j 8][p 2]
 *     V  key 32 a + 16 t + 4 g + i,   channel 32 c + 16 e + m        at [a 2][c 4][g 4][m 16][e 2][t 2][i 4]
 *   k_scale, v_scale fp32 [n_pages, Hkv, page_size / 64]
 *   k_mean           bf16 [n_pages, Hkv, page_size / 64, head_dim]: the mean of
 *                    the block's dequantised keys
 * page_size is a multiple of 64.  Zero-filled pools are an empty cache.
 * Paged: block_table int32 [B, max_pages] on the device, token x of sequence b
 * in row x % page_size of page block_table[b][x / page_size].  Dense:
 * block_table NULL, sequence b is page b, B <= n_pages, max_pages is not read.
 * A sequence holds at most 8388608 (2^23) positions and the pools fewer than
 * 2^31 blocks (JL_ERR_UNSUPPORTED beyond).  Tables, lengths and lists are device
 * arrays that the host cannot check: reads clamp page indices into the pool and
 * lengths into [0, capacity], so bad ones give wrong values and never an access
 * outside the pools; writes to a page outside the pool are dropped.
 */
typedef struct jl_cache8 {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  void* k_mean;
  int n_pages, page_size, Hkv, head_dim;
} jl_cache8;

/*
 * Appends rows to an 8-bit cache: n tokens of prefill, or one of decode.
 *   k, v    bf16 [B, n, Hkv, head_dim] raw keys and values
 *   starts  int32 [B] DEVICE array: position of each sequence's first new row,
 *           i.e. its length before the call
 *   n_new   int32 [B] DEVICE array or NULL: rows of sequence b that are appended
 *           (its first ones; clamped into [0, n]); NULL: all n
 * Rows at positions outside [0, capacity) are dropped.  For each block that
 * takes new rows
 *   scale = 2^e with the smallest e in [-117, 119] such that the largest
 *           magnitude of the new rows is at most 448 * 2^e (NaN is passed over,
 *           an infinity counts as the largest finite value), or the scale it
 *           had where that is larger and the block holds rows before the first
 *           new one;
 *   rows before the first new one are kept, rounded again where the scale grew;
 *   new rows are x / scale rounded to nearest even e4m3, saturated at 448 (NaN
 *           stays NaN);
 *   rows behind the last new one become zero; the block's mean is taken anew.
 * Every other block is left as it was.  New rows of two sequences, or of two
 * blocks of one, that meet in the same block of the pools (a page that is named
 * twice) race.  Nothing is allocated and nothing waited for.
 */
int jl_cache8_append(const jl_cache8* cache, const int32_t* block_table, int max_pages,
                     const void* k, const void* v, const int32_t* starts, const int32_t* n_new,
                     int B, int n, void* stream);

/*
 * Rows start .. start + n - 1 of every sequence back as bf16 [B, n, Hkv,
 * head_dim] (written), exactly: a bf16 holds every value of the cache.  With
 * them the prefill entry points continue a prompt (jl_bifocal_prefill_chunk with
 * q_start behind the rows).  start + n must not exceed the capacity; rows that
 * were never appended come as the pools hold them.  Nothing is allocated.
 */
int jl_cache8_read(const jl_cache8* cache, const int32_t* block_table, int max_pages, void* k,
                   void* v, int B, int start, int n, void* stream);

/*
 * Bytes of workspace the 8-bit decode entry points need; 0 for invalid arguments.
 * It does not depend on the batch or the lengths.  Its first 4096 bytes (arrival
 * counters) must be zero when it is first used; every call leaves them zero, so
 * one fill serves all later calls, of any shape that fits.  Calls that share a
 * workspace must be ordered by the caller.
 */
size_t jl_decode8_workspace_bytes(int Hq, int Hkv, int head_dim);

/*
 * jl_bifocal_decode over an 8-bit cache.
 *   q        bf16 [B, Hq, head_dim]  raw queries, sequence b's at kv_lens[b] - 1
 *   kv_lens  int32 [B] DEVICE array, the new token already appended; what the
 *            cache holds at or past kv_lens[b] does not matter.  A sequence of
 *            length 0 gets zeros.
 *   o        bf16 [B, Hq, head_dim]  output (written)
 *   workspace, workspace_bytes: jl_decode8_workspace_bytes(Hq, Hkv, head_dim)
 *            bytes, 16-byte aligned, see there
 * Requires Hq % Hkv == 0 and Hq / Hkv <= 8.  Only the cos/sin table may be
 * allocated or grown (to the cache's capacity).  Rounded to fp16 (11 bits; an
 * e4m3 number is exact in it) are
 *   - the query, rotated in fp32, after a power of two has brought its row near
 *     the top of fp16's range: values below 2^-27 of the row's largest may
 *     hold fewer bits, those below 2^-38 become zero;
 *   - a key's rotation inside its block: the (cos, sin) of its offset, one
 *     product and the sum;
 *   - the softmax weights, against the largest of their block of 64 keys and
 *     view: weights below 2^-29 of it hold fewer bits, those below 2^-40 become
 *     zero (2^-14 and 2^-25 where that block's largest score exceeds 2^22 in
 *     units of log2).  The denominator sums the rounded weights.
 * Everything else is kept in fp32; the same call gives the same bits.
 */
int jl_bifocal_decode8(const jl_cache8* cache, const int32_t* block_table, int max_pages,
                       const void* q, const int32_t* kv_lens, void* o, int B, int Hq,
                       double rope_theta, int w_pretrained, int w_local, void* workspace,
                       size_t workspace_bytes, void* stream);

/* The vanilla counterpart of jl_bifocal_decode8 (base rotation for every key). */
int jl_rope_attention_decode8(const jl_cache8* cache, const int32_t* block_table, int max_pages,
                              const void* q, const int32_t* kv_lens, void* o, int B, int Hq,
                              double rope_theta, void* workspace, size_t workspace_bytes,
                              void* stream);

/*
 * jl_bifocal_decode8 over listed blocks only: the softmax runs over the keys
 * below kv_lens[b] of the blocks that blocks[b][h] names.
 *   blocks   int32 [B, Hkv, n_select] DEVICE array of block indices (token / 64),
 *            in any order, one list per kv head.  Entries outside the sequence
 *            (-1 among them) are passed over; one listed twice counts twice.
 * A list without a key gives zeros.  The view of a key, G and the query's
 * position follow from kv_lens[b] as in jl_bifocal_decode8: the full list gives
 * its result up to the order of the sums.
 */
int jl_bifocal_decode8_blocks(const jl_cache8* cache, const int32_t* block_table, int max_pages,
                              const void* q, const int32_t* kv_lens, const int32_t* blocks,
                              int n_select, void* o, int B, int Hq, double rope_theta,
                              int w_pretrained, int w_local, void* workspace,
                              size_t workspace_bytes, void* stream);

/* The vanilla counterpart of jl_bifocal_decode8_blocks. */
int jl_rope_attention_decode8_blocks(const jl_cache8* cache, const int32_t* block_table,
                                     int max_pages, const void* q, const int32_t* kv_lens,
                                     const int32_t* blocks, int n_select, void* o, int B, int Hq,
                                     double rope_theta, void* workspace, size_t workspace_bytes,
                                     void* stream);

/*
 * A cheap score of every block for the query of each sequence:
 *   scores fp32 [B, Hkv, n_blocks] (written), n_blocks = capacity / 64:
 *   max over the query heads of kv head h of
 *     <R(f(q)) x_q, R(f(64 j + 31)) k_mean_j> / sqrt(head_dim)
 * i.e. what the block's mean key would score in the remote view at its middle
 * position; -inf for blocks at or past kv_lens[b].  Arguments as in
 * jl_bifocal_decode8.  A NaN in a query or mean gives NaN.
 */
int jl_bifocal_block_scores8(const jl_cache8* cache, const int32_t* block_table, int max_pages,
                             const void* q, const int32_t* kv_lens, float* scores, int B, int Hq,
                             double rope_theta, int w_pretrained, void* stream);

/* The same with base rotations, for the vanilla decode. */
int jl_rope_block_scores8(const jl_cache8* cache, const int32_t* block_table, int max_pages,
                          const void* q, const int32_t* kv_lens, float* scores, int B, int Hq,
                          double rope_theta, void* stream);

/*
 * The blocks that a query attends to: always the first n_first of its sequence
 * and those that hold a key of the local band (kv_lens[b] - 1 - k <= w_local), then
 * the others by falling score, n_select in all.  Equal scores go to the lower
 * index; NaN counts as larger than any number.
 *   scores  fp32 [B, Hkv, n_blocks]
 *   blocks  int32 [B, Hkv, n_select] output (written): ascending, -1 behind the
 *           last where the sequence has fewer blocks
 * n_select must hold the blocks that are always chosen: at least
 * min(n_blocks, (w_local + 127) / 64 + n_first).  n_blocks <= 131072.
 * The band follows from kv_lens[b] as it is: unlike in the calls on a cache a
 * length past 64 n_blocks is not clamped to it, so that the band may lie partly
 * or wholly behind the last block.
 */
int jl_select_blocks(const float* scores, const int32_t* kv_lens, int32_t* blocks, int B, int Hkv,
                     int n_blocks, int n_select, int w_local, int n_first, void* stream);

/*
 * ---- pages of a batch ------------------------------------------------------
 * The tables of B sequences over one pool of n_pages pages, as the paged entry
 * points read them (table as block_table, lens as kv_lens), and how often each
 * page is named.  All three are device arrays of the caller's:
 *   table  int32 [B, max_pages]: the pages of sequence b are the first
 *          ceil(lens[b] / page_size) entries of its row, the others are -1
 *   lens   int32 [B]: tokens of each sequence, 0 for an empty row
 *   refs   int32 [n_pages], 16-byte aligned: entries of the table that name the
 *          page; a page is free where it is not positive
 * -1 everywhere, zeros and zeros are an empty table.  Pages hold any number of
 * tokens; the bf16 entry points take powers of two, the 8-bit ones multiples of 64.
 * The calls below keep these rules; results follow from the arguments alone, and
 * no call waits for the device or allocates.  The caller may lower lens (rows that
 * are taken back, as rejected drafts are): the pages behind the new end stay the
 * sequence's, counted in refs and copied by forks, until jl_pages_reserve frees
 * them.  Nothing else of the three is the caller's to change, but for restoring
 * all of them to an earlier state.  Entries outside the pool are never
 * followed.  B > 2048 or n_pages > 2^30 -> JL_ERR_UNSUPPORTED.  Calls on one table
 * must be ordered by the caller.
 */
typedef struct jl_pages {
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  int B, max_pages, n_pages, page_size;
} jl_pages;

/*
 * Forks, frees and reorders sequences, all rows at once: row b becomes what row
 * parent[b] was before the call, sharing its pages (the partly filled last one
 * too), and an empty row where parent[b] is outside [0, B).  parent[b] = b leaves
 * row b as it is.  Pages that no row names any more are free.
 *   parent  int32 [B] DEVICE array
 */
int jl_pages_fork(const jl_pages* pages, const int32_t* parent, void* stream);

/*
 * Makes room for n_new[b] rows behind every sequence (none where n_new[b] <= 0): the
 * pages they need are taken from the free ones, in ascending order, sequence after
 * sequence.  A sequence whose rows begin in a partly filled page that other sequences
 * name too gets a page of its own in its place, to which the old one is to be copied
 * (a sequence's last page that all name who write there stays with the last of them).
 * All or nothing: if the pages do not suffice, or a sequence would pass max_pages, the
 * table, lens and refs stay as they were.  Before all this and in any case, entries behind
 * the first ceil(lens[b] / page_size) of every row, up to the first that names no page, become
 * -1 and refs follow: the pages of rows that were taken back are free again.
 *   n_new    int32 [B] DEVICE array
 *   starts   int32 [B] (written): lens before the call, as the append calls take them
 *   granted  int32 [B] (written): max(n_new, 0), or 0 for all if the pages do not
 *            suffice; lens grows by it.  The append calls take it as n_new.
 *   moves    int32 [B, 2] (written): page to copy from, page to copy to, in order of the
 *            sequences; -1 behind the last.  jl_copy_pages has to run before rows are
 *            appended.
 *   info     int32 [4] (written): moves, pages taken, pages missing, sequences that would
 *            pass max_pages
 */
int jl_pages_reserve(const jl_pages* pages, const int32_t* n_new, int32_t* starts,
                     int32_t* granted, int32_t* moves, int32_t* info, void* stream);

/*
 * Makes the pages in use the first ones of the pool: with n of them, the i-th that is
 * numbered n or more gets the number of the i-th free page below n.  Table and refs are
 * rewritten; jl_copy_pages then moves the contents.
 *   moves  int32 [n_pages / 2, 2] (written): from, to, ascending; -1 behind the last
 *   to     int32 [n_pages]: workspace
 *   info   int32 [4] (written): moves, pages in use, 0, 0
 */
int jl_pages_compact(const jl_pages* pages, int32_t* moves, int32_t* to, int32_t* info,
                     void* stream);

/* A pool of pages: page p is the page_bytes bytes (a multiple of 4) at ptr (4-byte
 * aligned) + p * page_bytes. */
typedef struct jl_page_pool {
  void* ptr;
  size_t page_bytes;
} jl_page_pool;

/*
 * Copies pages inside each of n_pools pools (K and V of every layer, the five arrays of an
 * 8-bit cache) as moves says: the first n_moves[0] pairs (from, to) of it, at most max_moves;
 * pairs that name a page outside [0, n_pages) are passed over.  No page may be named as a
 * target twice or as a source and a target; the lists of jl_pages_reserve and
 * jl_pages_compact name none so.
 *   pools    host array, not read after the call returns
 *   moves    int32 [max_moves, 2], n_moves int32 [1]: DEVICE arrays (n_moves: info)
 */
int jl_copy_pages(const jl_page_pool* pools, int n_pools, int n_pages, const int32_t* moves,
                  const int32_t* n_moves, int max_moves, void* stream);

/*
 * Appends rows to a bf16 cache, paged or dense.
 *   k_cache, v_cache  bf16 [n_pages, page_size, Hkv, head_dim] (written)
 *   block_table  int32 [B, max_pages] DEVICE array; NULL: a dense cache, sequence b is
 *                page b (page_size = its capacity, B <= n_pages, max_pages is not read)
 *   k, v     bf16 [B, n, Hkv, head_dim], or with cu_seqlens packed [n, Hkv, head_dim]
 *   starts   int32 [B] DEVICE array: position of each sequence's first new row
 *   n_new    int32 [B] DEVICE array or NULL: only the first n_new[b] rows of sequence b
 *   cu_seqlens  int32 [B + 1] DEVICE array, non-decreasing, or NULL: sequence b's rows are
 *            cu_seqlens[b] .. cu_seqlens[b + 1] - 1 of the packed ones
 * Rows at positions outside [0, capacity), for a page outside the pool or of no sequence are
 * dropped.  Two rows for one place of the pools race.  Nothing is allocated.
 */
int jl_cache_append(void* k_cache, void* v_cache, int n_pages, int page_size,
                    const int32_t* block_table, int max_pages, const void* k, const void* v,
                    const int32_t* starts, const int32_t* n_new, const int32_t* cu_seqlens, int B,
                    int n, int Hkv, int head_dim, void* stream);

/*
 * ---- decode over shared prefixes -------------------------------------------
 * jl_bifocal_decode_paged for batches in which groups of sequences begin with the same
 * tokens on the same pages (forks of a prompt, chats behind one system prompt): the keys
 * and values of a prefix are read once for all the sequences of its group.  What a step's
 * calls have in common is planned once, from the lengths, and serves every layer.
 *
 *   kv_lens       int32 [B] DEVICE array, the new token appended; clamped into
 *                 [0, max_pages * page_size].  A sequence of length 0 gets zeros.
 *   members       int32 [B] DEVICE array or NULL (0 .. B - 1): the sequences, group after
 *                 group, each at most once; others than 0 .. B - 1 are passed over
 *   group_starts  int32 [n_groups + 1] DEVICE array, non-decreasing in [0, B]: group i is
 *                 members[group_starts[i]] .. members[group_starts[i + 1] - 1].  A group may
 *                 be one sequence.  Sequences of no group are left out: their rows of the
 *                 output stay as they were.
 *   shared        int32 [n_groups] DEVICE array: tokens that the group's sequences have in
 *                 common.  Of these whole pages below the shortest length count, and they
 *                 are read from the pages of any of the group's sequences.
 *   plan          jl_shared_plan_bytes(B, n_groups, Hq, Hkv) bytes on the device, 16-byte
 *                 aligned (written).  It holds for decode calls of the same B, n_groups, Hq,
 *                 Hkv, max_pages, page_size and views; a decode call whose plan was made for
 *                 other sizes leaves its output as it was.
 * page_size is a power of two, at least 16.  Hq / Hkv > 8, B or n_groups > 2048, or more than
 * 8388608 (2^23) positions a sequence -> JL_ERR_UNSUPPORTED.  Nothing is allocated.
 */
size_t jl_shared_plan_bytes(int B, int n_groups, int Hq, int Hkv);

int jl_bifocal_shared_plan(const int32_t* kv_lens, const int32_t* members,
                           const int32_t* group_starts, const int32_t* shared, int B, int n_groups,
                           int Hq, int Hkv, int head_dim, int max_pages, int page_size,
                           int w_pretrained, int w_local, void* plan, size_t plan_bytes,
                           void* stream);

/* The plan of the vanilla decode (base rotations). */
int jl_rope_shared_plan(const int32_t* kv_lens, const int32_t* members,
                        const int32_t* group_starts, const int32_t* shared, int B, int n_groups,
                        int Hq, int Hkv, int head_dim, int max_pages, int page_size, void* plan,
                        size_t plan_bytes, void* stream);

/* Bytes of workspace the shared decode needs; 0 for invalid arguments. */
size_t jl_decode_shared_workspace_bytes(int B, int Hq, int Hkv, int head_dim);

/*
 * The decode: the result of jl_bifocal_decode_paged, up to rounding and the order of the
 * sums, for every sequence of the plan.
 *   q          bf16 [B, Hq, head_dim]  raw queries, sequence b's at kv_lens[b] - 1
 *   k_pages, v_pages, block_table, page_size, n_pages: as in jl_bifocal_decode_paged; page
 *              indices are clamped into the pool, which holds fewer than 2^31 tokens
 *   plan       of jl_bifocal_shared_plan with the same sizes and windows
 *   o          bf16 [B, Hq, head_dim]  output (written)
 *   workspace  jl_decode_shared_workspace_bytes(B, Hq, Hkv, head_dim) bytes, 16-byte
 *              aligned; contents on entry do not matter
 * Rounded are the rotated queries, the keys' cos and sin and the rotated keys, to fp16, and the
 * softmax weights, to bf16, whose rounded values the denominator sums; everything else is fp32.
 * Beside a key, or a rotated and scaled query, whose largest channel lies outside [2^-8, 2^15) the
 * first three are rounded to bf16, for all that the same workgroup holds, in twice the time.  The
 * same plan and inputs give the same bits.  Only the cos/sin table may be allocated or grown.
 */
int jl_bifocal_decode_shared(const void* q, const void* k_pages, const void* v_pages,
                             const int32_t* block_table, int max_pages, int page_size, int n_pages,
                             const void* plan, size_t plan_bytes, void* o, int B, int n_groups,
                             int Hq, int Hkv, int head_dim, double rope_theta, int w_pretrained,
                             int w_local, void* workspace, size_t workspace_bytes, void* stream);

/* The vanilla counterpart, with a plan of jl_rope_shared_plan. */
int jl_rope_attention_decode_shared(const void* q, const void* k_pages, const void* v_pages,
                                    const int32_t* block_table, int max_pages, int page_size,
                                    int n_pages, const void* plan, size_t plan_bytes, void* o,
                                    int B, int n_groups, int Hq, int Hkv, int head_dim,
                                    double rope_theta, void* workspace, size_t workspace_bytes,
                                    void* stream);

/*
 * Packed chunks behind paged caches of different lengths: the next turns of several
 * sequences, drafts to be verified, or single tokens among them, in one call.
 *   q, o         bf16 [total_tokens, Hq, head_dim]: sequence b's rows are cu_seqlens[b] ..
 *                cu_seqlens[b + 1] - 1, n of them, at its positions kv_lens[b] - n ..
 *                kv_lens[b] - 1
 *   lse          NULL or fp32 [Hq, total_tokens], natural-log row sums
 *   kv_lens      int32 [B] DEVICE array: keys of each sequence, the chunk's own (written
 *                before the call) among them; clamped into [0, max_pages * page_size]
 *   cu_seqlens   int32 [B + 1] DEVICE array, non-decreasing from 0 to total_tokens; other
 *                bounds are clamped, a decreasing one gives an empty sequence
 *   k_pages, v_pages, block_table, page_size, n_pages: as in jl_bifocal_decode_shared
 * Every sequence has its own G = max(1, ceil(kv_lens[b] / w_pretrained)), as a chunk of
 * jl_bifocal_prefill_chunk_paged that ends there: the same result up to rounding and the
 * order of the sums.  Rows of no sequence, or before position 0 (more rows than keys), are
 * left as they were.  Hq / Hkv at most 256; B > 2048, or about a million rows (total_tokens *
 * Hq / Hkv) in one call -> JL_ERR_UNSUPPORTED.  The same call gives the same bits.
 *
 * Sequences of more than 128 rows (tokens * Hq / Hkv) run as blocks of the prefill kernel where
 * Hq / Hkv divides 256, page_size is 64 or more, max_pages 4096 or less, and (total_tokens - B) *
 * Hq / Hkv 1024 or more; without one of these in the kernel of the short ones, which takes a third
 * longer.  Roundings as in jl_bifocal_decode_shared, but that a part of a block is done again in
 * bf16 by another rule: where eight channels of a key from a multiple of eight on and their
 * partners, or every other eight channels of a rotated and scaled query, are not all zero and
 * the largest of them is outside [2^-12, 2^15).
 *   workspace    jl_varlen_paged_workspace_bytes(...) bytes, 16-byte aligned; contents on entry do
 *                not matter.  The sum of 1056 bytes for every token and query head, 35 MB for the
 *                workgroups, 140 MB where there are blocks, and lists: 310 MB for 8192 tokens of 32
 *                heads without blocks, 449 MB with them.
 * Only the cos/sin table may be allocated or grown.
 */
/* 0 for arguments that the calls refuse. */
size_t jl_varlen_paged_workspace_bytes(int B, int total_tokens, int Hq, int Hkv, int head_dim,
                                       int max_pages, int page_size);

int jl_bifocal_prefill_varlen_paged(const void* q, const void* k_pages, const void* v_pages,
                                    const int32_t* block_table, int max_pages, int page_size,
                                    int n_pages, const int32_t* cu_seqlens,
                                    const int32_t* kv_lens, void* o, float* lse, int B,
                                    int total_tokens, int Hq, int Hkv, int head_dim,
                                    double rope_theta, int w_pretrained, int w_local,
                                    void* workspace, size_t workspace_bytes, void* stream);

/* The vanilla counterpart of jl_bifocal_prefill_varlen_paged. */
int jl_rope_attention_varlen_paged(const void* q, const void* k_pages, const void* v_pages,
                                   const int32_t* block_table, int max_pages, int page_size,
                                   int n_pages, const int32_t* cu_seqlens, const int32_t* kv_lens,
                                   void* o, float* lse, int B, int total_tokens, int Hq, int Hkv,
                                   int head_dim, double rope_theta, void* workspace,
                                   size_t workspace_bytes, void* stream);

/*
 * Debug view of the schedule as the device computes it (Eqs. (2), (3), (5)),
 * for bit-exact tests.  All pointers are device pointers.
 *   lengths    int32 [n_lengths]              sequence lengths L (>= 1)
 *   positions  int32 [n_positions]            positions x (>= 0)
 *   group_out  int32 [n_lengths]              G(L)
 *   remote_out int32 [n_lengths, n_positions] f(x) = floor(x / G(L))
 *   offset_out int32 [n_lengths, n_positions] Delta(x) = f(x) - x
 */
int jl_debug_schedule(const int32_t* lengths, int n_lengths, const int32_t* positions,
                      int n_positions, int w_pretrained, int32_t* group_out, int32_t* remote_out,
                      int32_t* offset_out, void* stream);

/* Tile classes written by jl_debug_prefill_tiles. */
enum { JL_TILE_SKIP = 0, JL_TILE_LOCAL = 1, JL_TILE_REMOTE = 2, JL_TILE_MIXED = 3 };

/*
 * Debug view of the prefill kernel's tile classification (Eq. (1)'s window
 * boundary at tile granularity), computed on the device with the kernel's own
 * block sizes.  Writes int8 classes_out[n_qblocks, n_ktiles] (device) and the
 * block geometry to the host ints *block_q, *block_k, *n_qblocks, *n_ktiles.
 * classes_len is the capacity of classes_out in elements.
 */
int jl_debug_prefill_tiles(int L, int Hq, int Hkv, int w_local, int8_t* classes_out,
                           int64_t classes_len, int* block_q, int* block_k, int* n_qblocks,
                           int* n_ktiles, void* stream);

/*
 * Debug knob for tests, process-wide: the prefill kernels move a row's softmax
 * reference (and rescale the running output) when a key tile's largest score
 * in that row exceeds the reference by more than log2_bound (scores in log2
 * units), or lies more than log2_bound below it before anything was
 * accumulated; the default is 64, far from anything ordinary data reaches.
 * The fused and vanilla calls first run a pass without that check, which only
 * notes whether a tile's probability sum exceeded 2^log2_bound or a row's
 * total fell below 2^-log2_bound; such blocks are then run again, by the same
 * workgroup, with the check.
 * A small bound (e.g. 3) sends almost every block through the rerun and the
 * rescale path, which tests use to check both.  Values outside [1, 100] leave
 * the setting unchanged.  Returns the previous value.  Not for use while
 * prefill calls are in flight.
 */
double jl_debug_prefill_rescale_log2(double log2_bound);

/*
 * Timing hook for benchmarks, process-wide.  which = 0: every later prefill
 * call that runs the fused or vanilla attention kernel (every prefill entry
 * point but the literal one's three window passes) records the HIP event
 * `start` on its stream right before that kernel and `stop` right after it,
 * so hipEventElapsedTime(start, stop) is the attention alone (a packed call's
 * planning kernels stay outside).  which = 1: the
 * same around the split kernel of every decode call that takes a workspace
 * (all but jl_bifocal_decode_noalloc; the reduce stays outside, but the 8-bit
 * decode's one kernel merges too).
 * start, stop: hipEvent_t created and owned by the caller; NULL, NULL clears
 * the hook.  JL_ERR_INVALID_ARG for another `which` or when only one event is
 * NULL.  The events must outlive every call that records them.
 */
int jl_debug_kernel_events(int which, void* start, void* stop);

/* Frees the library-owned cos/sin tables and prefill scratch buffers on every
 * device (they are rebuilt on demand); waits for the streams that own scratch.
 * Must not race with running calls. */
void jl_release_caches(void);

#ifdef __cplusplus
}
#endif

#endif /* JETLONG_H */
