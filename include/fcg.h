/*
 * fcg.h - function-level KV cache grafting on one MI355X (gfx950).
 *
 * C ABI of libfcg.so.  The library holds a segment library of function-level
 * KV states (the two-tier code cache of Sec. 4.1, Eq. 2: every function entry
 * keeps the KV states of its interface and of its implementation), stitches
 * retrieved segments into a composite cache at new positions (cache-stitching,
 * Sec. 4.2, Eq. 4: the interface KV states are concatenated and injected as
 * context), prefills patch tokens over that cache and decodes (cache-patching,
 * Sec. 4.2, Eq. 6: the prefix KV states are reused and only the new span is
 * computed).  Text, tokenizer and model weights are outside this library; its
 * inputs are token-level K/V/Q tensors.
 *
 * Conventions
 *  - Every entry point returns an fcg_status; nothing aborts or throws across
 *    the ABI.  fcg_last_error() gives a thread-local message for the last
 *    failing call on the calling thread.
 *  - A call that returns an error changes no state (an EHIP failure of the
 *    runtime after a call's checks aside).
 *  - "device" pointers are HIP device memory on the current device; "host"
 *    pointers are ordinary host memory, read (or written) before the call
 *    returns.  The caller keeps ownership of everything it passes.
 *  - stream is a hipStream_t (NULL = the default stream).  Calls validate on
 *    the host, enqueue their kernels on the stream and return; results are
 *    ready when the stream reaches that point.  A handle (fcg_lib, fcg_cache)
 *    must not be used by two threads or two streams at the same time.
 *  - Device faults of earlier work surface as FCG_EHIP from a later call.
 *  - Storage dtype: FCG_F32 = IEEE binary32, FCG_BF16 = bfloat16 (raw 16-bit
 *    patterns).  Every narrowing rounds to nearest, ties to even.
 *
 * Tensor layouts (elements of the storage dtype, row-major, innermost last)
 *  - Segment input to fcg_lib_add_segment:   k, v  [L][len][Hkv][D]
 *  - Library slab of one layer:              [Hkv][capacity][D]
 *  - Contiguous cache, one layer:            [n_seqs][Hkv][max_tokens][D]
 *  - Paged cache, one layer:                 [n_pages][Hkv][page_size][D]
 *  - Fresh tokens of fcg_patch_prefill:      q [n][Hq][D], k, v [n][Hkv][D]
 *  - Decode tokens of fcg_decode:            q [n][Hq][D], k, v [n][Hkv][D]
 *  - Attention outputs:                      out [n][Hq][D]
 */
#ifndef FCG_H
#define FCG_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  FCG_OK = 0,
  FCG_EINVAL = 1,   /* malformed argument: null pointer, bad count, unsupported shape, mismatch */
  FCG_ERANGE = 2,   /* index out of range: layer, sequence, segment, position, span end */
  FCG_EOVERLAP = 3, /* a target position is given twice or is already written */
  FCG_EHOLE = 4,    /* attention would read a position that is not written */
  FCG_ENOMEM = 5,   /* device memory, library capacity, host tier or page pool exhausted */
  FCG_ESTATE = 6,   /* operation not valid in the current state (e.g. decode on an empty sequence) */
  FCG_EHIP = 7      /* the HIP runtime reported an error */
} fcg_status;

typedef enum { FCG_F32 = 0, FCG_BF16 = 1 } fcg_dtype;

/* Shape of the attention layers whose KV states are grafted.  Keys carry the
 * rotary position encoding in rotate-half layout: dimension i and i + D/2 turn
 * together by p * theta^(-2i/D) at position p (rope_style 0, the only one). */
typedef struct {
  int32_t n_layers;   /* L >= 1 */
  int32_t n_q_heads;  /* Hq, with Hq / Hkv one of 1, 2, 4, 8, 16 */
  int32_t n_kv_heads; /* Hkv >= 1 */
  int32_t head_dim;   /* D: 64 or 128 */
  double rope_theta;  /* theta > 1 */
  int32_t dtype;      /* fcg_dtype of every K, V, Q and output tensor */
  int32_t rope_style; /* 0 = rotate-half */
} fcg_model_desc;

typedef struct fcg_lib fcg_lib;
typedef struct fcg_cache fcg_cache;
typedef struct fcg_locality fcg_locality;

/* ---------------------------------------------------------------- library */

/* flags of fcg_lib_create and fcg_cache_create */
#define FCG_LAYOUT_ONLY 1u /* no device memory: only the index / layout is kept (planning and tests) */
/* fcg_cache_create, paged caches only: a logical page that one grafted
 * segment covers entirely reads its values from the library in place instead
 * of a copy (values are position-independent; keys are still turned and
 * copied).  The cache binds to the library of its first graft; the library
 * must outlive the cache. */
#define FCG_ALIAS_V 2u

/* Create an empty segment library (the KV side of the two-tier code cache,
 * Sec. 4.1, Eq. 2) holding up to capacity_tokens tokens in up to max_segments
 * segments.  Allocates L * Hkv * capacity_tokens * D elements for K and as
 * many for V (none with FCG_LAYOUT_ONLY: then only the segment index exists,
 * segments are added with k == v == NULL, and grafts into layout-only caches
 * are planned but move nothing).  FCG_ENOMEM if the device cannot hold them. */
fcg_status fcg_lib_create(const fcg_model_desc* desc, int64_t capacity_tokens,
                          int32_t max_segments, uint32_t flags, fcg_lib** out);

/* Append one segment of len tokens whose keys were encoded at source positions
 * src_pos0 .. src_pos0 + len - 1.  k, v: device [L][len][Hkv][D], copied into
 * the slabs on stream.  k == v == NULL reserves the space only (the caller
 * fills it through fcg_lib_device_ptrs).  *seg_id receives the new id
 * (ids are 0, 1, 2, ... in order of addition).  FCG_ENOMEM when capacity or
 * max_segments is exhausted. */
fcg_status fcg_lib_add_segment(fcg_lib* lib, int32_t len, int32_t src_pos0, const void* k,
                               const void* v, void* stream, int32_t* seg_id);

/* The update step of the cache management (Alg. 1; Sec. 4.1: low-scored
 * entries go to DRAM, high-scored ones stay on the GPU): with loc tracking one
 * function per library segment (function id = segment id), decide which
 * segments stay in device memory and move the others: segments read in place
 * by an FCG_ALIAS_V cache stay; then, in descending locality score (Eq. 3),
 * a segment stays while its bytes (len x K+V of all layers) fit in
 * budget_bytes; with ppl_threshold > 0 (the hyperparameter table's
 * perplexity-based eviction threshold, 15.0) segments whose perplexity is
 * below it are placed only after all others.  budget_bytes < 0 takes the
 * table's GPU memory threshold: 0.85 of the device memory less a 2 GB reserve
 * less what the rest of the process holds (at most the slabs).  Offloads are
 * issued first, then reloads, all on stream (a side stream is fine: grafts
 * wait for reloads, and reused ranges wait for earlier grafts).
 * *n_offloaded / *n_reloaded (host, may be NULL) receive the moves.
 * Errors: EINVAL (null arguments, loc's size differs from the segment count,
 * negative threshold), ESTATE (an offload without a host tier), ENOMEM (host
 * tier full, or no device range for a reload: the state stays consistent, the
 * moves made so far remain). */
fcg_status fcg_lib_update_residency(fcg_lib* lib, const fcg_locality* loc, int64_t budget_bytes,
                                    double ppl_threshold, void* stream, int32_t* n_offloaded,
                                    int32_t* n_reloaded);

/* Where segment seg_id sits: tokens tok_off .. tok_off + len - 1 of every
 * [Hkv][capacity][D] slab (tok_off = -1 while offloaded); keys encoded from
 * src_pos0.  Any output may be NULL. */
fcg_status fcg_lib_segment_info(const fcg_lib* lib, int32_t seg_id, int64_t* tok_off,
                                int32_t* len, int32_t* src_pos0);

/* Host tier of the library (the DRAM side of the code cache: low-scored
 * entries are offloaded and reloaded when needed; Sec. 4.1, App. C.5).
 * fcg_lib_host_reserve allocates pinned host slabs of host_tokens tokens
 * (layout as the device slabs); each segment gets a host copy on its first
 * offload, kept until the library is destroyed (segments never change).
 * Errors: EINVAL (host_tokens < 1), ESTATE (reserved already), ENOMEM, EHIP. */
fcg_status fcg_lib_host_reserve(fcg_lib* lib, int64_t host_tokens);

/* Move segment seg_id out of device memory: copy it to its host slot on
 * stream (first offload only) and free its device range for later segments
 * and reloads (first fit; a reused range is written only after the copy has
 * read it).  fcg_graft of an offloaded segment fails with ESTATE.  Async:
 * calls on one library are ordered by the caller (one stream, or events).
 * Errors: ERANGE (seg_id), ESTATE (not in device memory, no host tier, or an
 * FCG_ALIAS_V cache reads its values in place: reset those sequences first),
 * ENOMEM (host tier full), EHIP. */
fcg_status fcg_lib_offload(fcg_lib* lib, int32_t seg_id, void* stream);

/* Bring an offloaded segment back into device memory on stream, at the first
 * free device range that fits (fcg_lib_segment_info gives the new offset).
 * Errors: ERANGE, ESTATE (already in device memory), ENOMEM (no range fits), EHIP. */
fcg_status fcg_lib_reload(fcg_lib* lib, int32_t seg_id, void* stream);

/* *in_device = 1 iff seg_id is in device memory; *on_host = 1 iff it has a host
 * copy (either may be NULL).  Errors: EINVAL, ERANGE. */
fcg_status fcg_lib_segment_state(const fcg_lib* lib, int32_t seg_id, int32_t* in_device, int32_t* on_host);

/* Device base pointers of layer's K and V slab ([Hkv][capacity][D]). */
fcg_status fcg_lib_device_ptrs(const fcg_lib* lib, int32_t layer, void** k, void** v);

fcg_status fcg_lib_destroy(fcg_lib* lib);

/* ------------------------------------------------------------------ cache */

/* Create a composite cache for n_seqs sequences of up to max_tokens positions.
 * page_size == 0: contiguous, one [Hkv][max_tokens][D] region per sequence and
 * layer (n_pages ignored).  page_size == 16: a pool of n_pages pages per
 * layer, one page table per sequence shared by all layers; logical page
 * p / 16 of a sequence is mapped on first write to the lowest-numbered free
 * page, new pages of one call in ascending (sequence, logical page) order.
 * With FCG_LAYOUT_ONLY no device memory is allocated and graft, prefill
 * and decode only validate and record the layout (planning and tests);
 * FCG_ALIAS_V maps value pages onto the library (see the flag).
 * Errors: EINVAL (bad descriptor, n_seqs or max_tokens < 1, max_tokens *
 * head_dim >= 2^31, page_size not 0 or 16, unknown flags, FCG_ALIAS_V on a
 * contiguous cache), ENOMEM, EHIP. */
fcg_status fcg_cache_create(const fcg_model_desc* desc, int32_t n_seqs, int32_t max_tokens,
                            int32_t page_size, int32_t n_pages, uint32_t flags, fcg_cache** out);

/* Forget everything written in seq (all layers) and return its pages. */
fcg_status fcg_cache_reset(fcg_cache* cache, int32_t seq);

/* Cache-patching (Sec. 4.2, Eq. 6; the patch step of Alg. 1): keep only the
 * prefix [0, pos) of seq in every layer, so that the span after it can be
 * regenerated over the reused prefix states (fcg_patch_prefill of new tokens
 * at positions pos.., then fcg_decode).  The stale states past pos are never
 * read.  Pages holding no kept position return to the pool.  Host metadata
 * only, except with FCG_ALIAS_V when the cut splits a page whose values are
 * read from the library: its kept rows are copied into the cache's own page
 * on stream (new tokens will follow them).  pos = 0 empties the sequence;
 * pos = max_tokens keeps everything.  Errors: EINVAL (null cache), ERANGE
 * (seq outside [0, n_seqs), pos outside [0, max_tokens]), EHIP. */
fcg_status fcg_cache_truncate(fcg_cache* cache, int32_t seq, int32_t pos, void* stream);

/* Host copy of the layout of seq: page_table [ceil(max_tokens / page_size)]
 * physical page or -1 (paged caches only; may be NULL), *seq_len = 1 + the
 * highest written position of layer (0 if none; may be NULL), written
 * [max_tokens] bytes 1/0 per position of layer (may be NULL). */
fcg_status fcg_cache_export_layout(const fcg_cache* cache, int32_t seq, int32_t layer,
                                   int32_t* page_table, int32_t* seq_len, uint8_t* written);

/* FCG_ALIAS_V caches: v_alias [ceil(max_tokens / 16)] receives, per logical
 * page of seq, the library token (index into the [Hkv][capacity][D] slabs)
 * whose value row holds the page's first position, or -1 where the page holds
 * its own values.  -1 everywhere for other caches.  Errors: EINVAL (null
 * argument), ERANGE (seq). */
fcg_status fcg_cache_export_v_alias(const fcg_cache* cache, int32_t seq, int32_t* v_alias);

/* Device base pointers of layer's K and V region (layouts in the file header). */
fcg_status fcg_cache_device_ptrs(const fcg_cache* cache, int32_t layer, void** k, void** v);

fcg_status fcg_cache_destroy(fcg_cache* cache);

/* --------------------------------------------------------------- hot path */

/* Cache-stitching (Sec. 4.2, Eq. 4; App. B.1, module-level cache reuse):
 * for every item i, graft library segment seg[i] into sequence seq[i] at
 * positions dst[i] .. dst[i] + len - 1, in all layers, keeping its token
 * order.  Keys are turned by delta = dst[i] - src_pos0 (the rotary encoding of
 * a key at position p becomes that of p + delta) and rounded to the storage
 * dtype; values are copied bit for bit.  One launch covers every item and
 * layer.  seq, seg, dst: host arrays of n_items.
 * Errors: ERANGE (seq, seg, span outside [0, max_tokens)), EOVERLAP (spans
 * meet each other or written positions of any layer), ENOMEM (pages), EINVAL
 * (lib and cache shapes differ, null arrays, a layout-only library with a
 * cache that has device memory, an FCG_ALIAS_V cache bound to another
 * library), ESTATE (after all of the above pass: a segment is offloaded). */
fcg_status fcg_graft(fcg_cache* cache, const fcg_lib* lib, int32_t n_items, const int32_t* seq,
                     const int32_t* seg, const int32_t* dst, void* stream);

/* Patch prefill at one layer (Sec. 4.2, Eq. 6; App. B.1, cache-patching):
 * token t (host seq[t], pos[t]) gets its query and key encoded at pos[t]
 * (rounded to storage), its key and value stored at pos[t], and
 * out[t] = softmax(q k^T / sqrt(D)) v over every position <= pos[t] of its
 * sequence, query head h reading kv head h / (Hq / Hkv).  Tokens may belong to
 * several sequences and come in any order.  q, k, v, out: device, starting at
 * any element (here and in the decode calls; multiples of 16 bytes take the
 * faster loads).
 * Errors: ERANGE, EOVERLAP (position given twice or already written in this
 * layer), EHOLE (a position below a query's is unwritten after the call),
 * ENOMEM (pages). */
fcg_status fcg_patch_prefill(fcg_cache* cache, int32_t layer, int32_t n_tok, const int32_t* seq,
                             const int32_t* pos, const void* q, const void* k, const void* v,
                             void* out, void* stream);

/* One decode step at one layer for n_seqs distinct sequences (host seqs):
 * each appends its token at its current length in that layer and attends
 * over every position up to it, as in fcg_patch_prefill.  positions_out
 * (host, may be NULL) receives the positions used.
 * Errors: EINVAL (duplicate sequence), ERANGE (sequence full), ESTATE
 * (nothing written in this layer), EHOLE, ENOMEM. */
fcg_status fcg_decode(fcg_cache* cache, int32_t layer, int32_t n_seqs, const int32_t* seqs,
                      const void* q, const void* k, const void* v, void* out,
                      int32_t* positions_out, void* stream);

/* fcg_decode for callers that cannot allocate device memory: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, semantics, results and errors as fcg_decode; it calls no
 * hipMalloc / hipFree and uploads nothing.  Its split partials and arrival
 * counters live in a static device array of the library (8.5 MiB per GPU,
 * held until the process ends), not in memory of the cache; the cache itself
 * must exist already (fcg_cache_create allocates).  Every call on one GPU
 * shares that array: calls that overlap on one GPU (several streams or host
 * threads) race.  The first call on a device also launches a small kernel that
 * zeroes the counters.  Kernel timing (fcg_cache_timing) does not cover it.
 * Extra errors: EINVAL (more than 64 kv heads), ENOMEM (the step needs more
 * than 8 MiB of split partials: many long sequences at once; use fcg_decode). */
fcg_status fcg_decode_noalloc(fcg_cache* cache, int32_t layer, int32_t n_seqs, const int32_t* seqs,
                              const void* q, const void* k, const void* v, void* out,
                              int32_t* positions_out, void* stream);

/* ------------------------- rotary forms, appending, attention over a shared prefix */

/* The cache's own rotary form (rotate-half over the whole head, theta of the
 * descriptor) is what fcg_graft, fcg_patch_prefill and fcg_decode use.  For
 * models of another form, a rotary handle describes it, and the calls of this
 * section take the handle: fcg_rope_apply encodes the keys of a library
 * segment, fcg_graft_rope grafts them, fcg_append places fresh tokens and
 * encodes their queries, fcg_prefix_attend attends.
 *
 * Tensors of this section are given with strides, so that slices of a fused
 * projection need no copy.  Strides count elements of the storage dtype; the
 * head_dim elements of a row are adjacent.  A row may start at any element. */
typedef struct {
  void* data;    /* device; null = not given, where that is allowed */
  int64_t layer; /* from a layer's tensor to the next (calls of several layers) */
  int64_t token; /* from a token to the next; >= 0 */
  int64_t head;  /* from a head to the next; >= 0 */
} fcg_tensor;

typedef struct fcg_rope fcg_rope;

/* layout: which dimensions turn together, for pair i < rotary_dim / 2 */
#define FCG_ROPE_HALF 0  /* i and i + rotary_dim / 2 */
#define FCG_ROPE_PAIRS 1 /* 2i and 2i + 1 (interleaved) */
/* scaling of the frequencies w_i = theta^(-2i / rotary_dim) for long contexts */
#define FCG_ROPE_PLAIN 0  /* none */
#define FCG_ROPE_LINEAR 1 /* w_i / factor (positions interpolated) */
#define FCG_ROPE_NTK 2    /* theta * factor^(R / (R - 2)) in place of theta, R = rotary_dim (>= 4 by its rule) */
#define FCG_ROPE_PARTS 3  /* by parts: with r = orig_tokens * w_i / (2 pi) turns over the trained length and
                             c = (r - low_turns) / (high_turns - low_turns) clamped to [0, 1]:
                             w_i ((1 - c) / factor + c).  Models that ramp over the pair's index between
                             rounded bounds instead: their frequencies through FCG_ROPE_GIVEN */
#define FCG_ROPE_GIVEN 4  /* freqs[i] */

typedef struct {
  int32_t rotary_dim;   /* R: a multiple of 16; dimensions >= R of a head pass unturned */
  int32_t layout;       /* FCG_ROPE_HALF or FCG_ROPE_PAIRS */
  int32_t scaling;      /* FCG_ROPE_PLAIN .. FCG_ROPE_GIVEN; the fields below that a kind does not name are ignored */
  double theta;         /* > 1 (not FCG_ROPE_GIVEN) */
  double factor;        /* >= 1 (LINEAR, NTK, PARTS) */
  double orig_tokens;   /* > 0 (PARTS) */
  double low_turns;     /* 0 <= low_turns < high_turns (PARTS) */
  double high_turns;
  double attn_factor;   /* m > 0, a normal fp32 number: the rotated dimensions of encoded queries and keys are
                           multiplied by it */
  const double* freqs;  /* host [R / 2], finite (and 2^31 times as much), in radians per position (GIVEN), read by the call */
} fcg_rope_desc;

/* Create a rotary handle: host memory only, usable on every device and from
 * several threads and streams at once.
 * Errors: EINVAL (null argument, rotary_dim not a multiple of 16 in [16, 128],
 * a field out of its range), ENOMEM. */
fcg_status fcg_rope_create(const fcg_rope_desc* desc, fcg_rope** out);
/* freqs [R / 2] (host) receives the frequencies after scaling.  Errors: EINVAL. */
fcg_status fcg_rope_frequencies(const fcg_rope* rope, double* freqs);
fcg_status fcg_rope_destroy(fcg_rope* rope);

/* Encode n_tok tokens of n_layers layers at their positions: with p = pos[t]
 * (device int32 [n_tok], any value, shared by the layers) and m the attention
 * factor, the pair (a, b) of every head becomes
 *   (m (a cos(p w_i) - b sin(p w_i)), m (b cos(p w_i) + a sin(p w_i))),
 * the angle taken in 64 bits (within 2^-51 |p w_i| radians: it holds little past
 * |p w_i| of 2^45), its cos and sin (within 2^-22) and the turn in 32, rounded once
 * to dtype; dimensions past rotary_dim are copied.  FCG_ROPE_BACKWARD: the gradient of that map (the
 * angle negated, the factor kept), from the gradient of its result to that of
 * its input.  q [n_layers][n_tok][n_q_heads][head_dim] and k alike, each with
 * an output of its own shape; either may be left out (null pointer or zero
 * heads).  An output may be its input (the same data and strides), and must not
 * overlap it otherwise; rows of an output must not overlap each other, rows of
 * an input may (stride 0).  Nothing is allocated or uploaded: the call can be
 * captured into a graph, whose replays read pos, q and k anew.
 * Errors: EINVAL (null rope, pos or tensor, dtype, head_dim not 64 or 128 or
 * below rotary_dim, negative counts, flags or strides, more than 2^30 tokens,
 * 4096 heads or 65535 layers, overlapping output rows), EHIP.  Runs on the
 * current device, as the pointers do. */
#define FCG_ROPE_BACKWARD 1u
fcg_status fcg_rope_apply(const fcg_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_tok,
                          const int32_t* pos, int32_t n_q_heads, const fcg_tensor* q, const fcg_tensor* q_out,
                          int32_t n_k_heads, const fcg_tensor* k, const fcg_tensor* k_out, uint32_t flags,
                          void* stream);

/* Cache-stitching as fcg_graft, for segments whose keys carry the rotary form
 * of `rope`: keys turn by the angles of delta = dst[i] - src_pos0 (without the
 * attention factor, which the encoded keys hold already), cos and sin as in
 * fcg_rope_apply (fcg_graft's are 64-bit ones rounded to fp32, so a handle of the
 * cache's own form may leave other last bits), dimensions past rotary_dim and
 * values are copied bit for bit.  Errors as fcg_graft, and
 * EINVAL (null rope, rotary_dim above the head). */
fcg_status fcg_graft_rope(fcg_cache* cache, const fcg_lib* lib, const fcg_rope* rope, int32_t n_items,
                          const int32_t* seq, const int32_t* seg, const int32_t* dst, void* stream);

/* Append without attending: token t (host seq[t], pos[t]) has its key encoded
 * at pos[t] and rounded to storage, and key and value stored at pos[t], in the
 * layers layer .. layer + n_layers - 1; with q, its query is encoded as
 * well and written to q_out.  rope null: the cache's own rotary form, the same
 * bits fcg_patch_prefill stores.  k, v [n_layers][n_tok][Hkv][D], q and q_out
 * [n_layers][n_tok][Hq][D]; q_out may be q (the same data and strides), and
 * must not overlap q otherwise, nor its own rows.  k and v both null reserve
 * the positions only (pages mapped, positions written, their rows' content
 * whatever the memory holds; q must be null then).  Tokens come in any
 * order, and positions may leave holes, which fcg_patch_prefill and fcg_decode
 * refuse to attend over and fcg_prefix_attend fills from its prefix.
 * FCG_REPLACE: positions already written are written over (a retried span, a
 * rejected draft) instead of refused.
 * A call can be captured into a graph if it maps no page and the tokens form at
 * most 64 runs (consecutive positions of one sequence at consecutive indices)
 * on at most 384 pages; replays write the same places.  A reservation that maps no
 * page launches nothing.
 * Errors: EINVAL (null arrays or tensors, negative counts or strides, flags,
 * rotary_dim above the head, overlapping rows of q_out), ERANGE (layers,
 * sequence, position), EOVERLAP (a position given twice; one written in one of
 * the layers, without FCG_REPLACE), ESTATE (with FCG_REPLACE: a position whose
 * value is read from the library, FCG_ALIAS_V; a capture that would need an
 * upload), ENOMEM (pages), EHIP. */
#define FCG_REPLACE 1u
fcg_status fcg_append(fcg_cache* cache, int32_t layer, int32_t n_layers, int32_t n_tok, const int32_t* seq,
                      const int32_t* pos, const fcg_rope* rope, const fcg_tensor* q, const fcg_tensor* q_out,
                      const fcg_tensor* k, const fcg_tensor* v, uint32_t flags, void* stream);

/* Attention of a batch over one shared prefix, read once for all of it.  The
 * prefix is positions [0, prefix_len) of sequence prefix_seq; token t (host
 * seq[t], pos[t]) attends to it and to positions prefix_len .. pos[t] of its own
 * sequence at one layer:
 *   out[t] = softmax(q k^T / sqrt(D)) v,  lse[t] = ln sum exp(q k^T / sqrt(D))
 * over these keys, query head h reading kv head h / (Hq / Hkv).  q is encoded
 * already (fcg_append's q_out, fcg_rope_apply); nothing is written to the
 * cache.  Positions of seq[t] below prefix_len, if any are written, are not
 * read.  pos[t] = prefix_len - 1 attends to the prefix only; with prefix_len = 0
 * as well there is no key, out[t] is 0 and lse[t] -inf.  prefix_len = 0 is
 * attention over each token's own sequence (prefix_seq is then ignored).
 * Tokens come in any order, several of a sequence, the same position twice.
 * q, out [n_tok][Hq][D] with strides (layer strides ignored); lse fp32
 * [n_tok][Hq], contiguous, may be null.  out may be q (the same data and
 * strides).
 * The split partials sit in a workspace of the cache, enlarged when a call
 * needs more.  A call can be captured into a graph if it, or one whose partials
 * take as much, ran before, and it has at most 128 tokens, of at most 64 sequences, none with
 * 96 (fp32: 48) query rows a kv head or more; a workspace that a capture used is
 * kept until the cache is destroyed, and the calls and graphs of one cache share
 * it, so they must not overlap.
 * Errors: EINVAL (null arrays or tensors, negative counts or strides, more than
 * 2^24 - 1 tokens or 2^30 query rows, overlapping rows of out), ERANGE (layer, sequences, prefix_len outside [0,
 * max_tokens], pos[t] outside [prefix_len - 1, max_tokens)), EHOLE (an attended
 * position is not written), ESTATE (a capture that would need an upload or a
 * larger workspace), ENOMEM, EHIP. */
fcg_status fcg_prefix_attend(fcg_cache* cache, int32_t layer, int32_t prefix_seq, int32_t prefix_len, int32_t n_tok,
                             const int32_t* seq, const int32_t* pos, const fcg_tensor* q, const fcg_tensor* out,
                             float* lse, void* stream);

/* ------------------------------------------- norms of queries and keys */

/* Models that normalise queries and keys head by head before they turn them.
 * A row x of head_dim elements becomes
 *   n = (offset + weight) x / sqrt(mean(x^2) + eps),
 * the mean over the head, in fp32.  weight: device, storage dtype, head_dim
 * adjacent elements that may start anywhere, `head` elements from a head's to
 * the next head's and `layer` from a layer's to the next (0: shared); null: all
 * ones, offset ignored.  offset is 1 for models that store the distance from 1. */
typedef struct {
  const void* weight;
  int64_t layer; /* >= 0; layers count from the call's first one */
  int64_t head;  /* >= 0 */
  double eps;    /* > 0, a normal fp32 number */
  double offset; /* finite in fp32 */
} fcg_norm;

/* fcg_rope_apply of normalised rows in one pass: norm, turn and attention
 * factor in fp32, rounded once to dtype.  Arguments, in-place outputs and
 * capture as there; q_norm or k_norm null: those rows are turned only.  A row
 * of which an element is not finite, or whose squares add up past the fp32
 * range, gives what that arithmetic gives (NaN; zeros).
 * Errors: as fcg_rope_apply, and EINVAL (a norm's strides, eps or offset). */
fcg_status fcg_norm_rope_apply(const fcg_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_tok,
                               const int32_t* pos, int32_t n_q_heads, const fcg_norm* q_norm, const fcg_tensor* q,
                               const fcg_tensor* q_out, int32_t n_k_heads, const fcg_norm* k_norm,
                               const fcg_tensor* k, const fcg_tensor* k_out, void* stream);

/* One side, queries or keys, of fcg_norm_rope_backward. */
typedef struct {
  int32_t heads;
  const fcg_norm* norm; /* null: rows that are turned only */
  fcg_tensor x;         /* the forward pass's input (not read with norm null) */
  fcg_tensor grad;      /* the gradient of its result */
  fcg_tensor dx;        /* receives the gradient of its input; may be x or grad in place */
  float* dweight;       /* receives the gradient of the weights, device fp32, contiguous: [n_layers][heads][head_dim],
                           or [n_layers][head_dim] where the norm's head stride is 0 or there is one head (weights shared
                           by layers: their sum over layers is the caller's); null: not wanted */
} fcg_norm_side;

/* Device bytes that fcg_norm_rope_backward needs with weight gradients for such
 * sides (heads of 0: none).  Errors: EINVAL (counts, head_dim, null output). */
fcg_status fcg_norm_rope_workspace(int32_t head_dim, int32_t n_layers, int32_t n_tok, int32_t n_q_heads,
                                   int32_t n_k_heads, int64_t* bytes);

/* The gradient of fcg_norm_rope_apply: with dn the gradient turned back (and
 * times the attention factor), s = 1 / sqrt(mean(x^2) + eps) and w the weights
 * with their offset,
 *   dweight = sum over rows of dn x s,  dx = s (dn w - x s mean(dn w x s)),
 * in fp32; dx rounded once to dtype, dweight fp32, added up in a fixed order
 * (the same call gives the same bits).  q, k: host; either may be null.
 * workspace: device, 16-byte aligned, fcg_norm_rope_workspace bytes, of any
 * content, for this call alone until it is done; null where no dweight is
 * wanted.  Nothing is allocated or uploaded: the call can be captured.
 * Errors: as fcg_norm_rope_apply, and EINVAL (a dweight without weights, a
 * workspace that is too small or not aligned). */
fcg_status fcg_norm_rope_backward(const fcg_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_layers,
                                  int32_t n_tok, const int32_t* pos, const fcg_norm_side* q, const fcg_norm_side* k,
                                  void* workspace, int64_t workspace_bytes, void* stream);

/* fcg_append of normalised queries and keys (values as they are).  q_norm and
 * k_norm may be null: those rows are turned only.  The same bits for a query or
 * key as fcg_norm_rope_apply with the same rope gives.
 * Errors: as fcg_append, and EINVAL (a norm's strides, eps or offset; a norm
 * without the rows it is for). */
fcg_status fcg_append_norm(fcg_cache* cache, int32_t layer, int32_t n_layers, int32_t n_tok, const int32_t* seq,
                           const int32_t* pos, const fcg_rope* rope, const fcg_norm* q_norm, const fcg_norm* k_norm,
                           const fcg_tensor* q, const fcg_tensor* q_out, const fcg_tensor* k, const fcg_tensor* v,
                           uint32_t flags, void* stream);

/* ------------------------------------ what a cache keeps of its positions */

/* The attention weight that the tokens of a call put on each position they
 * attend to: for the tokens, keys and q of an fcg_prefix_attend at one layer and
 * the lse it returned (device fp32 [n_tok][Hq], contiguous),
 *   weights[s][h][j] = sum of exp(q k_j / sqrt(D) - lse[t])
 * over the tokens t that attend to position j of sequence s and over the query
 * heads of kv head h, in fp32, added up in a fixed order (the same call gives
 * the same bits).  weights: device fp32 [n_seqs][Hkv][max_tokens], one layer's,
 * contiguous: prefix positions in row prefix_seq, own positions in each token's
 * row; elements of positions that no token of the call attends to stay as they
 * are.  FCG_ADD: the sums are added to what the elements hold (a decode loop
 * that keeps score; clear them first).
 * Split partials sit in the workspace of fcg_prefix_attend, with its rules for
 * captures and overlapping calls; a call can be captured if it has at most 128
 * tokens of at most 64 sequences (and attends to less than 8 million positions).
 * Errors: as fcg_prefix_attend (of q, lse and weights none may be null). */
#define FCG_ADD 1u
fcg_status fcg_attend_weights(fcg_cache* cache, int32_t layer, int32_t prefix_seq, int32_t prefix_len, int32_t n_tok,
                              const int32_t* seq, const int32_t* pos, const fcg_tensor* q, const float* lse,
                              float* weights, uint32_t flags, void* stream);

/* Squeeze sequences to the positions of most weight.  Item i keeps, of the n
 * positions of sequence src[i], min(keep[i], n): in each layer and kv head by
 * itself the first n_first ones, the last n_recent ones (where keep[i] is
 * smaller, first ones go before last ones), and of the others those of the
 * largest weight, the lower position where weights are equal (NaN counts as
 * less than any number).  In order of position they become positions 0, 1, ..
 * of sequence dst[i] in all layers: keys turned to their new position (by the
 * distance moved, without the attention factor; unmoved keys and all values are
 * copied bit for bit) in the form of `rope`, null the cache's own.
 *   dst[i] = src[i]: in place; what is behind is forgotten and its pages return.
 *   dst[i] another sequence: emptied first; src[i] stays as it is, and may be
 *   the source of several items.
 * A prefix that sequences share (fcg_prefix_attend): squeeze it into another
 * sequence, over which others start.  Those that have positions behind it attend to
 * it as it was; after an eviction in place they cannot (EHOLE), nor are they whole
 * sequences that could be squeezed themselves.
 * weights: device fp32 [n_layers][n_seqs][Hkv][max_tokens], contiguous
 * (fcg_attend_weights of each layer): read in row src[i]; row dst[i] receives
 * the kept positions' weights in their new order and zeros after them, to
 * max_tokens.  kept: device int32 [n_layers][n_items][Hkv][largest keep[i]],
 * contiguous, may be null: receives the former positions; elements past an
 * item's stay as they are.
 * The kept positions (where kept is null) and a table of turns sit in the
 * workspace of fcg_prefix_attend, with its rules for captures and overlapping calls;
 * a call that maps no page can be captured, and replays move from the same
 * positions to the same ones.
 * Errors: EINVAL (null arrays, negative counts, rotary_dim above the head, a dst
 * given twice or also the src of another item, more than 32767 kv heads or 2^20
 * over all layers), ERANGE (sequences, keep outside [0, max_tokens]), ESTATE
 * (layers of a src that differ in length; in place with values read from the
 * library, FCG_ALIAS_V; a capture that would map pages or needs a larger
 * workspace), EHOLE (an unwritten position below the length), ENOMEM (pages),
 * ENOMEM of host memory and EHIP (other dst may be left empty; a sequence in
 * place is squeezed or has the rows and the length that it had, but its weights
 * may be rewritten then). */
fcg_status fcg_evict(fcg_cache* cache, int32_t n_items, const int32_t* src, const int32_t* dst, const int32_t* keep,
                     int32_t n_first, int32_t n_recent, const fcg_rope* rope, float* weights, int32_t* kept,
                     void* stream);

/* -------------------------------------------------- log probabilities */

/* Of each row of logits [n_rows][vocab] (device, dtype, rows row_stride >= 0
 * elements apart, starting anywhere), in fp32 and one pass over it, any of
 *   lse[r]     = ln sum_j exp(x_j),
 *   logprob[r] = x_t - lse with t = targets[r] (device int32 [n_rows]; a t outside
 *                [0, vocab) is no target: 0),
 *   entropy[r] = - sum_j p_j ln p_j, p_j = exp(x_j - lse),
 *   top_id, top_logprob [n_rows][n_top]: the n_top <= 64 most likely tokens, the most likely
 *                first, the lower id where logits are equal (NaN counts as less than any
 *                number), and their x - lse.
 * Outputs are device, fp32 (ids int32), contiguous; null: not wanted (top_id only
 * with n_top = 0).  Logits of -inf are tokens ruled out; a row of nothing else has
 * lse -inf, log probabilities -inf and entropy 0; a row with a NaN has NaN for all three.
 * workspace: device, 16-byte aligned, fcg_token_logprobs_workspace bytes (0 for
 * many rows), of any content, for this call alone until it is done.  Nothing is allocated or
 * uploaded: the call can be captured.  Runs on the current device.
 * Errors: EINVAL (dtype, negative counts or stride, vocab outside [1, 2^30], n_top
 * outside [0, min(64, vocab)], null logits, logprob without targets, alternatives without
 * top_id, a workspace that is too small or not aligned), EHIP. */
fcg_status fcg_token_logprobs_workspace(int32_t n_rows, int32_t vocab, int32_t n_top, int64_t* bytes);
fcg_status fcg_token_logprobs(int32_t dtype, int32_t n_rows, int32_t vocab, const void* logits, int64_t row_stride,
                              const int32_t* targets, float* logprob, float* entropy, float* lse, int32_t n_top,
                              int32_t* top_id, float* top_logprob, void* workspace, int64_t workspace_bytes,
                              void* stream);

/* The gradient of the logits from those of logprob, entropy and lse (device fp32
 * [n_rows], each may be null: zero):
 *   dx_j = p_j (g_lse - g_logprob - g_entropy (ln p_j + entropy)) + g_logprob [j = t],
 * in fp32, rounded once to dtype; 0 where x_j is -inf (but at the target), and no
 * g_logprob in rows without a target.  lse and, with g_entropy, entropy: what
 * fcg_token_logprobs gave.  dlogits [n_rows][vocab], rows d_stride apart; may be the
 * logits in place (the same stride), and must not overlap them otherwise.  Can be captured.
 * Errors: EINVAL (dtype, negative counts or stride, vocab, null tensors, a gradient
 * without targets or entropy, overlapping rows of dlogits), EHIP. */
fcg_status fcg_token_logprobs_backward(int32_t dtype, int32_t n_rows, int32_t vocab, const void* logits,
                                       int64_t row_stride, const int32_t* targets, const float* lse,
                                       const float* entropy, const float* g_logprob, const float* g_entropy,
                                       const float* g_lse, void* dlogits, int64_t d_stride, void* stream);

/* ------------------------------------------------- code-cache management */

/* Locality score of the cache entries (Sec. 4.1, Eq. 3; App. B.1, Eq. 8-10;
 * the update step of Alg. 1), host only:
 *   l(f) = (1 - l_curr(f)) (alpha l_freq(f) + beta sum_j l_asso(j | f)
 *          + gamma l_sema(f)) + l_curr(f),
 *   l_freq(f) = count(f) / max_j count(j),
 *   l_asso(j | f) = cooccur(f, j) / count(f),
 *   l_sema(f) = PPL(f) / max_j PPL(j).
 * Functions are ids 0 .. n_funcs - 1 (a caller's map to library segments).
 * Statistics cover the last `window` recorded execution traces (one per task;
 * the paper uses 20); cooccur(f, j) counts calls of j that immediately follow
 * a call of f in one trace; l_curr(f) = 1 iff f occurs in the latest trace;
 * a component with a zero denominator is 0.  Weights: >= 0, summing to 1 (the
 * paper uses 0.4, 0.3, 0.3).
 * Errors: EINVAL (n_funcs or window < 1, bad weights, null output), ENOMEM. */
fcg_status fcg_locality_create(int32_t n_funcs, int32_t window, double alpha, double beta, double gamma,
                               fcg_locality** out);
/* Record one task's execution trace: func_ids[n] (host) in call order.
 * Errors: EINVAL (null handle, n < 0, null ids), ERANGE (an id). */
fcg_status fcg_locality_record(fcg_locality* loc, int32_t n, const int32_t* func_ids);
/* Perplexity of function func's implementation (>= 0; 0 until set).
 * Errors: EINVAL (null handle, negative or NaN ppl), ERANGE (func). */
fcg_status fcg_locality_set_ppl(fcg_locality* loc, int32_t func, double ppl);
/* The same for n functions at once, measured: logprob (device fp32) holds the log
 * probabilities of n_tok[i] >= 1 tokens of funcs[i] (host arrays), function after
 * function, as fcg_token_logprobs gives them (every token with a target); PPL = exp(-their mean),
 * summed in 64 bits.  Waits for the stream.  On an error no perplexity changes.
 * Errors: EINVAL (null arguments, a negative count, a function without tokens, a perplexity
 * that is not finite), ERANGE (a function), ESTATE (the stream is being captured), ENOMEM,
 * EHIP. */
fcg_status fcg_locality_measure_ppl(fcg_locality* loc, int32_t n, const int32_t* funcs, const int32_t* n_tok,
                                    const float* logprob, void* stream);
/* scores[n_funcs] (host) receives l(f), each in [0, 1].  Errors: EINVAL. */
fcg_status fcg_locality_scores(const fcg_locality* loc, double* scores);
/* Which entries stay in device memory under a budget: in descending score
 * (ties: ascending id), an entry is kept when its cost[f] (host, >= 0, e.g.
 * bytes or tokens) still fits in what the kept ones leave of budget.
 * resident[n_funcs] (host) receives 1 / 0.  Errors: EINVAL (null arguments,
 * negative budget or cost). */
fcg_status fcg_locality_residency(const fcg_locality* loc, int64_t budget, const int64_t* cost, uint8_t* resident);
fcg_status fcg_locality_destroy(fcg_locality* loc);

/* ------------------------------------------------------------- diagnostics */

/* Kernel timing (measurement, not part of the method).  While enabled, every
 * call on this cache records HIP events on its stream around its kernels:
 *   FCG_TIME_GRAFT        the graft kernel of fcg_graft and fcg_graft_rope
 *   FCG_TIME_PREFILL_ATTN the attention kernel of fcg_patch_prefill
 *   FCG_TIME_PREFILL      all kernels of fcg_patch_prefill (append, attention, merge)
 *   FCG_TIME_DECODE       all kernels of fcg_decode (one per group of 64 sequences)
 *   FCG_TIME_DECODE_ATTN  the attention kernels of fcg_decode (the same kernels: the
 *                         split merge runs inside them)
 * Plan uploads, host work, fcg_append and fcg_prefix_attend are outside the
 * intervals.  fcg_cache_timing_read
 * waits for the recorded events, returns the number of intervals and their
 * summed duration in milliseconds for one kind (ERANGE for another value),
 * and forgets them.  enable = 0 stops recording (recorded intervals stay
 * readable). */
#define FCG_TIME_GRAFT 0
#define FCG_TIME_PREFILL_ATTN 1
#define FCG_TIME_PREFILL 2
#define FCG_TIME_DECODE 3
#define FCG_TIME_DECODE_ATTN 4
fcg_status fcg_cache_timing(fcg_cache* cache, int32_t enable);
fcg_status fcg_cache_timing_read(fcg_cache* cache, int32_t kind, int32_t* count, double* total_ms);

/* Name of a status code; the message of the calling thread's last failed
 * call (kept until its next failure; empty before any).  Both strings are
 * owned by the library. */
const char* fcg_status_string(fcg_status s);
const char* fcg_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FCG_H */
