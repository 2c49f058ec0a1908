/*
 * blindsight.h — C ABI of the MI355X sparse prefill-attention library.
 *
 * The library computes causal prefill attention over an interleaved text/image prompt in
 * which every query head carries one of four offline-assigned sparsity classes and the mask
 * follows from the prompt's image-span table alone (paper Sec. 3.2, Sec. 5, App. "BlindSight
 * Attention Kernel").  Two steps:
 *
 *   bs_build_tilemap   host, integer only: span table + class vector -> for every class and
 *                      every query tile the list of key tiles to run, each FULL (no masking
 *                      needed) or PARTIAL (element predicate needed); all other tiles are
 *                      skipped.  This replaces the paper kernel's per-tile metadata
 *                      (sink_end[M], first_image[M], the all/any(istext) tests of Alg. 3).
 *   bs_attn_prefill    device: one flash-style pass over the listed tiles (Alg. 3-7 folded
 *                      into one loop with a single running softmax per row).
 *
 * All functions return BS_OK (0) or a negative BS_E* code; nothing throws or aborts across
 * this boundary.  No function synchronises the device except where stated.
 */
#ifndef BLINDSIGHT_H
#define BLINDSIGHT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BS_OK            0
#define BS_EINVAL       (-1)  /* null pointer, negative size, malformed span table, bad class   */
#define BS_EUNSUPPORTED (-2)  /* tile size / head_dim / dtype the kernels do not implement      */
#define BS_ENOMEM       (-3)  /* host or device allocation failed                              */
#define BS_EHIP         (-4)  /* a HIP runtime call failed (no device, launch error, ...)      */

/* Head classes (paper Sec. 3.2; "headtype" in Alg. 3).  Bit 0 = sink keys visible,
 * bit 1 = own-image keys visible. */
typedef enum {
    BS_DENSE      = 0,  /* every earlier key                                        */
    BS_SINK       = 1,  /* text keys + sink keys                                    */
    BS_INTRA      = 2,  /* text keys + keys of the query's own image                */
    BS_INTRA_SINK = 3   /* union of the two                                         */
} bs_head_class;

/* Element types of q/k/v/out. */
#define BS_BF16 0
#define BS_F32  1

/* One image: tokens [start, end) of the prompt; its first `sink` tokens are sink keys
 * (paper Sec. 6.1 "Sparse Mask Generation": sinks sit at the start of an image).
 * Tokens outside every span are text (imgid = 0 in the paper's notation). */
typedef struct { int32_t start, end, sink; } bs_span;

typedef struct bs_tilemap bs_tilemap;   /* opaque; owns its host arrays and device buffers */

/*
 * Build the tile map of one prompt.
 *   spans        host pointer, n_spans rows sorted by start, non-overlapping, inside
 *                [0, seq_len), 0 <= sink <= end - start (may be NULL when n_spans == 0)
 *   seq_len      L > 0
 *   head_class   host pointer, n_q_heads values in 0..3
 *   sink_len     positions [0, sink_len) are sink keys too (0 <= sink_len <= L)
 *   block_m/n    query / key tile edge (the paper's block_m, block_n).  The builder accepts
 *                any positive sizes; the attention kernels need 128 x 64.
 *   out          receives the new map; untouched on failure.  Free with bs_tilemap_destroy.
 * Tile (m, n) covers queries [m*block_m, +block_m) x keys [n*block_n, +block_n); positions
 * >= L count as masked.  SKIP = no allowed pair, FULL = every pair allowed, else PARTIAL.
 * A pair (i, j) is allowed iff j <= i and ( query i is text, or class is Dense, or key j is
 * text, or (class has the sink bit and j is a sink key), or (class has the intra bit and
 * i, j belong to the same image) ).
 * Host only: needs no GPU.  Errors: BS_EINVAL, BS_ENOMEM.
 */
int bs_build_tilemap(const bs_span *spans, int32_t n_spans, int32_t seq_len,
                     const uint8_t *head_class, int32_t n_q_heads, int32_t sink_len,
                     int32_t block_m, int32_t block_n, bs_tilemap **out);

/*
 * Same, with options (flags = 0 is bs_build_tilemap):
 *   BS_MAP_REGROUP_ROWS   the query rows are taken in another order than their positions: all
 *       image rows first, then all text rows, each group in position order and padded to whole
 *       query tiles.  Why: a text query attends to every earlier token (Sec. 3.2), so a query
 *       tile that holds a single text row has to walk every causal key tile for every head
 *       class; with the text rows in tiles of their own, the image rows of the sparse classes
 *       keep their skipped tiles (the Q-side counterpart of the paper kernel's packing of
 *       sink keys, App. kernel "Notation").  Only the grouping of rows into work items changes:
 *       q, k, v, out keep their layout and the result is the same function of the inputs.
 *       n_q_tiles becomes ceil(image rows / block_m) + ceil(text rows / block_m); query tile m
 *       covers the rows bs_tilemap_row_order reports.  No effect on a prompt without text or
 *       without image tokens.
 * Errors: BS_EINVAL (also for unknown flag bits), BS_ENOMEM.
 */
#define BS_MAP_REGROUP_ROWS 1u
/*   BS_MAP_PACK_KEYS (implies BS_MAP_REGROUP_ROWS)   the map also gets compact key tiles: the free
 *       keys of the prompt -- text keys and sink keys, which are what an image query of a sparse
 *       class may see outside its own image -- gathered in position order into tiles of their
 *       own, after the prompt's key tiles (n_k_tiles counts both).  The paper's kernel permutes
 *       K / V so that text and sink keys are contiguous (App. kernel, "Attention Sink Subroutine",
 *       Alg. 6); here they are a second copy, written by the bf16 pre-pass, because text queries
 *       and Dense heads keep walking the prompt order.  An image-only query tile of a sparse
 *       class then walks the compact tiles up to its causal bound (Sink: every slot; Intra-Image:
 *       the text slots; Intra-Image+Sink: the slots outside its own image) plus, for the classes
 *       with the intra bit, the prompt tiles of its own image, in which only own-image keys count.
 *       Every allowed pair is still counted exactly once.  bs_tilemap_key_order reports the key
 *       of every tile slot.
 *       No effect on a prompt without images, without free keys, or made of free keys only. */
#define BS_MAP_PACK_KEYS 2u
/*   BS_MAP_BIDIR_IMAGES   model variant in which the tokens of one image attend to each other in
 *       both directions (Gemma 3; paper Sec. 2: the dense mask is the model's default mask; Sec. 6.1
 *       states that this model does not attend causally inside an image).  The causal condition j <= i of the pair
 *       rule above becomes "j <= i, or i and j belong to the same image", for every class: a sparse
 *       mask is its class pattern inside the model's dense mask.  An image query then sees exactly
 *       what the last query of its image sees under the causal rule, which is how the map and the
 *       kernels treat it.  Text queries are unchanged.  Combines with the other flags. */
#define BS_MAP_BIDIR_IMAGES 4u
int bs_build_tilemap_ex(const bs_span *spans, int32_t n_spans, int32_t seq_len,
                        const uint8_t *head_class, int32_t n_q_heads, int32_t sink_len,
                        int32_t block_m, int32_t block_n, uint32_t flags, bs_tilemap **out);

/*
 * Same, for models whose image sinks are not a prefix of the image: sink_offsets (host, n_sink_offsets
 * values >= 0, may be NULL when the count is 0) lists offsets inside an image; the token at
 * start + offset of EVERY image is a sink key as well (offsets at or past an image's length are ignored
 * for that image), in addition to the spans' `sink` prefixes and the sink_len prefix of the prompt.
 * Paper Sec. 6.1 and App. "Attention Sink Positions in Gemma 3": that model tokenises every image to
 * the same length and its sinks sit at fixed locations inside every image (the paper keeps the 10 % most
 * frequent locations found on its characterisation set; the list itself is the caller's input).
 * window > 0 makes the map one of a sliding-window layer: the layer's dense mask keeps, for every query
 * (text queries too) and every class, only the keys with i - j < window (paper App. kernel, "Dense
 * Attention Subroutine": text queries follow the model's own dense mask, which is causal or a sliding
 * window depending on the model; the sparse masks live inside the dense mask).  0 = no window; a window of seq_len or
 * more is no window.  With a window BS_MAP_PACK_KEYS acts as BS_MAP_REGROUP_ROWS in everything that the map
 * reports (the kernels then have compact tiles of their own, bs_tilemap_walked).  Together with BS_MAP_BIDIR_IMAGES the keys of
 * the query's own image stay visible at any distance, also for images longer than the window: an image
 * query then sees its class pattern inside [min(window start, image start), image end).
 * Errors: as bs_build_tilemap_ex; BS_EINVAL for a negative offset, count or window.
 */
int bs_build_tilemap_model(const bs_span *spans, int32_t n_spans, int32_t seq_len,
                           const uint8_t *head_class, int32_t n_q_heads, int32_t sink_len,
                           int32_t block_m, int32_t block_n, uint32_t flags,
                           const int32_t *sink_offsets, int32_t n_sink_offsets, int32_t window,
                           bs_tilemap **out);

/*
 * Same, for a chunk of queries at the end of the prompt: the query rows are the positions q_begin .. seq_len - 1
 * only (0 <= q_begin < seq_len), attending to all seq_len keys under the same masks.  This is how the masks of
 * Sec. 3.2 carry over to chunked prefill and to decoding with the KV cache kept whole (the paper prunes no
 * KV entries, Sec. 6.1: its masks only drop attention pairs): the chunk's rows are rows of the same L x L mask.
 * With such a map, q and out of bs_attn_prefill hold seq_len - q_begin rows per head ([n_q_heads][seq_len -
 * q_begin][head_dim], row r = position q_begin + r); k and v hold all seq_len positions.  n_q_tiles counts the
 * tiles of those rows, bs_tilemap_row_order reports positions, allowed_pairs / empty_rows count those rows.
 * q_begin = 0 is bs_build_tilemap_model.  Errors: as bs_build_tilemap_model; BS_EINVAL for q_begin outside
 * [0, seq_len).
 */
int bs_build_tilemap_suffix(const bs_span *spans, int32_t n_spans, int32_t seq_len,
                            const uint8_t *head_class, int32_t n_q_heads, int32_t sink_len,
                            int32_t block_m, int32_t block_n, uint32_t flags,
                            const int32_t *sink_offsets, int32_t n_sink_offsets, int32_t window,
                            int32_t q_begin, bs_tilemap **out);

/* End of a map's life (the paper builds its mask metadata once per prompt, Sec. 5 "no runtime overhead";
 * so does a caller here, and destroys the map when the prompt's prefill is over).
 * Frees the host arrays; device buffers (if any) go back to a per-process cache of the library
 * and are handed to a later map only after the work queued with this map has finished (the
 * next owner's stream waits for an event recorded after this map's last call).  So a map may be
 * destroyed as soon as its last bs_attn_prefill has returned, without waiting for the stream,
 * and destroying it does not synchronise the device.  The cache keeps at most a few dozen
 * blocks until the process ends.  NULL is allowed. */
void bs_tilemap_destroy(bs_tilemap *tm);

/* Geometry of the map, in the paper's symbols (App. kernel, "Notation"): seq_len = L, n_q_tiles = M =
 * number of block_m-row query tiles, n_k_tiles = N = number of block_n-key tiles (compact tiles included).
 * Any output pointer may be NULL. */
int bs_tilemap_dims(const bs_tilemap *tm, int32_t *seq_len, int32_t *n_q_tiles,
                    int32_t *n_k_tiles, int32_t *n_q_heads);

/* rows[n_q_tiles * block_m] (host): the position of every row of every query tile, -1 where a
 * tile has no row (the last tile of the prompt, or of a group of regrouped rows). */
int bs_tilemap_row_order(const bs_tilemap *tm, int32_t *rows);

/* What the map options did (any pointer may be NULL): regrouped = the row order differs from the
 * position order; packed = compact key tiles exist; intra_compact = Intra-Image heads take their
 * text keys from the compact tiles (they keep the prompt's tiles when those hold the text keys in
 * fewer tiles, e.g. a few long images with little text between them). */
int bs_tilemap_layout(const bs_tilemap *tm, int32_t *regrouped, int32_t *packed, int32_t *intra_compact);

/* keys[n_k_tiles * block_n] (host, may be NULL): the position of the key in every slot of every
 * key tile, -1 where a tile has no key; n_prompt_tiles (may be NULL): how many of the tiles are
 * the prompt in position order (all of them unless the map was built with BS_MAP_PACK_KEYS). */
int bs_tilemap_key_order(const bs_tilemap *tm, int32_t *keys, int32_t *n_prompt_tiles);

/* The per-tile decision of the paper's kernel (App. kernel, Overview: fully masked tiles are skipped, tiles at
 * a mask boundary are masked element-wise) made explicit for the bit-exact check against the element-wise mask
 * of Sec. 3.2.  Expand the range lists of class `cls` for query tiles [q_tile_begin, +q_tile_count) into
 * states[q_tile_count][n_k_tiles] (host, row-major): 0 skip, 1 partial, 2 full. */
int bs_tilemap_tile_states(const bs_tilemap *tm, int32_t cls, int32_t q_tile_begin,
                           int32_t q_tile_count, uint8_t *states);

/* The same decision as the kernels walk it, for one query tile: they may take keys from compact tiles of their own
 * behind the map's n_k_tiles (the text keys once more, without the sinks, for Intra-Image heads; with a window free keys and
 * text keys), where that means fewer tiles.  *n_tiles = how many key tiles they know; states[*n_tiles] as above; keys[*n_tiles * block_n] the position of the
 * key in every slot, -1 where there is none; *compact = the tile's image rows take the keys outside their own image from
 * compact tiles, and only their own image's (classes with the intra bit) from the prompt's tiles.  Every allowed pair is
 * in exactly one tile.  Any output pointer may be NULL.  Host only, for tests and accounting. */
int bs_tilemap_walked(const bs_tilemap *tm, int32_t cls, int32_t q_tile, int32_t *n_tiles, uint8_t *states,
                      int32_t *keys, int32_t *compact);

/* Per-class accounting behind the FLOP figures (the paper counts attention FLOPs per unmasked pair, App.
 * "FLOPs Reduction"; Sec. 3.2 defines which pairs a class keeps).  Any output pointer may be NULL:
 *   visited = full + partial tiles over all query tiles; allowed_pairs = number of allowed
 *   (i, j) pairs, from span geometry (the bench's "4 d FLOP per unmasked pair" counts these);
 *   empty_rows = query rows whose allowed set is empty (their output is zero);
 *   n_ranges = entries in the class's range list. */
int bs_tilemap_stats(const bs_tilemap *tm, int32_t cls, int64_t *visited, int64_t *full,
                     int64_t *partial, int64_t *allowed_pairs, int64_t *empty_rows,
                     int64_t *n_ranges);

/*
 * Plan (and check) the work units the bf16 kernel uses for `gqa_group` query heads per KV head:
 * pairs of (head, query tile) items that read the same KV head and walk one merged key-tile
 * list, so a workgroup streams every K / V tile once for two items.  Returns BS_OK only if
 * every (head, query tile) appears in exactly one unit and each unit's merged list reproduces
 * both items' tile states as the kernel walks them (bs_tilemap_walked).  Outputs (may be NULL): number of units, key tiles summed over the
 * units' merged lists, and steps on which one of a unit's items has nothing to do.
 * Host only.  bs_attn_prefill plans by itself; this entry point is for tests and accounting.
 */
int bs_tilemap_pair_plan(bs_tilemap *tm, int32_t gqa_group, int64_t *n_units, int64_t *unit_tiles,
                         int64_t *skip_steps);

/*
 * Plan (and check) how those units are cut into equal shares for `n_wgs` workgroups (one per compute unit in
 * bs_attn_prefill), where a launch has too few units for the queues to balance it; gqa_group 0: the units of the fp32
 * kernel, one (head, query tile) item each.  Returns BS_OK only if every unit has a part, the parts of a unit walk each
 * of its key tiles once, each part is in one share or one queue, and the list of cut items names every part's slot.
 * Outputs (may be NULL): parts (0: the units stay in the queues), units that were cut, parts left to the queues.
 * Host only, for tests and accounting.
 */
int bs_tilemap_share_plan(bs_tilemap *tm, int32_t gqa_group, int32_t n_wgs, int64_t *n_parts, int64_t *n_cut_units,
                          int64_t *n_queued);

/*
 * Bind a built map to another class vector (paper Sec. 4: every layer of a model has its own offline-assigned
 * head classes, while the mask metadata depends on the prompt alone, Sec. 5): the four per-class tile lists,
 * token codes, row and key order -- everything bs_build_tilemap derived from the span table -- are kept,
 * on the host and on the device; only the work list / work units are planned again by the next
 * bs_attn_prefill (or bs_tilemap_prepare).  So a model builds ONE map per prompt and rebinds it per layer.
 *   head_class   host, n_q_heads values in 0..3 (n_q_heads may differ from the count the map was built with)
 * Host only, O(n_q_heads); binding the vector the map already has is free.  Stream order makes it safe to
 * rebind while kernels of the previous binding are still queued on the stream of the next call.
 * Errors: BS_EINVAL, BS_ENOMEM.
 */
int bs_tilemap_rebind(bs_tilemap *tm, const uint8_t *head_class, int32_t n_q_heads);

/*
 * Do, ahead of time, everything bs_attn_prefill would do on the first call with this map and these
 * arguments except the kernels: upload the prompt part (once per map), plan and upload the work list
 * (BS_F32, for either head dimension, with the workspace of the call) or the work units for `gqa_group`
 * (BS_BF16) of the current class vector, raise the kernels' dynamic-LDS limits and look up the address
 * of the static scratch on the current device.  Enqueues copies on `stream`, does not wait.  May allocate
 * (block cache / hipMalloc, pinned staging).  After it, an fp32 call and, with the same map, class vector and
 * gqa_group, bs_attn_prefill_static allocate nothing.
 * Errors: BS_EINVAL, BS_EUNSUPPORTED, BS_ENOMEM, BS_EHIP.
 */
int bs_tilemap_prepare(bs_tilemap *tm, int32_t dtype, int32_t gqa_group, void *stream);

/* Copy the map to the current HIP device and wait until the copy is done (default stream,
 * then hipStreamSynchronize on it).  Optional: bs_attn_prefill uploads on first use, on its own
 * stream and without waiting.  Not thread-safe against concurrent calls on the same map.
 * Errors: BS_EHIP, BS_ENOMEM. */
int bs_tilemap_upload(bs_tilemap *tm);

/*
 * Sparse causal prefill attention (paper Sec. 3.1 for the definition, App. kernel Alg. 3-7
 * for the tiled form):  for query head h with class head_class[h] and KV head h / gqa_group,
 *   out[h, i, :] = sum_j softmax_j( scale * <q[h,i], k[h/G,j]> over allowed j ) * v[h/G, j, :]
 * and zeros for a row with no allowed key.
 *   q, out   device pointers, [n_q_heads][L][head_dim], contiguous
 *   k, v     device pointers, [n_q_heads / gqa_group][L][head_dim], contiguous
 *   tm       map built for this prompt with block 128 x 64 and the same n_q_heads
 *   dtype    BS_BF16 (bf16 MFMA, fp32 accumulate, P rounded to bf16 before P.V) or
 *            BS_F32 (fp32 MFMA throughout)
 *   head_dim 64 or 128
 *   scale    finite and > 0 (1/sqrt(d_k) in the paper)
 *   stream   hipStream_t (NULL = default stream).  The call only enqueues work; the caller
 *            owns q/k/v/out and keeps them alive until the stream has drained.
 * bf16 path: a pre-pass first packs the keys and values of compact tiles, and all of V (transposed) where its tiles are
 * walked often, into per-key-tile blocks in a workspace the map owns (n_kv_heads * (2 n_tiles - seq_len / 64) * head_dim * 128 bytes, n_tiles from
 * bs_tilemap_walked: the size of V, whether or not all of it is packed, and twice as much more as there are compact tiles; and the partial results of work units that are
 * cut; taken from the library's block cache or hipMalloc on first use).  Calls with a few rows that see the
 * whole cache read K and V where they are; they and the fp32 path use the workspace for partial results.
 * Calls that share a map share that workspace: the library orders a call after
 * the map's previous call when the stream changes, but two threads must not call with one map
 * at the same time.
 * Values of k and v have to be finite: one that is not makes the rows that see its key not finite, and may reach
 * rows that do not see the key but stand in one work unit with rows that do (calls with a few rows excepted).
 * The first call on a map uploads it: the arrays are staged through pinned host buffers and
 * copied on `stream`; the host does not wait for the device (it may wait for an upload queued
 * eight uploads earlier, whose staging buffer it reuses).
 * Errors: BS_EINVAL (null pointers, head counts that do not match), BS_EUNSUPPORTED,
 * BS_EHIP, BS_ENOMEM.  Nothing is launched on error.
 */
int bs_attn_prefill(const void *q, const void *k, const void *v, void *out, bs_tilemap *tm,
                    int32_t dtype, int32_t n_q_heads, int32_t gqa_group, int32_t head_dim,
                    float scale, void *stream);

/*
 * Same call, for profiling harnesses: if non-NULL, ev_main_start / ev_main_stop (hipEvent_t,
 * created by the caller with timing enabled) are recorded on `stream` immediately before and
 * after the attention kernel itself, i.e. excluding the bf16 path's K / V^T tile-pack pre-pass
 *.  hipEventElapsedTime between them is that kernel's duration.
 */
int bs_attn_prefill_ex(const void *q, const void *k, const void *v, void *out, bs_tilemap *tm,
                       int32_t dtype, int32_t n_q_heads, int32_t gqa_group, int32_t head_dim,
                       float scale, void *stream, void *ev_main_start, void *ev_main_stop);

/*
 * bs_attn_prefill (bf16) for callers that cannot allocate: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same kernels and same result as bs_attn_prefill with BS_BF16;
 * the packed K / V^T tiles of the pre-pass go to a static device array of BS_STATIC_SCRATCH_MIB MiB
 * inside the library (one copy per GPU, held until the process ends) instead of a workspace owned by the
 * map.  Calls no hipMalloc / hipFree, creates no events, uploads nothing.
 *   tm       must have been prepared: bs_tilemap_prepare(tm, BS_BF16, gqa_group, stream) after the build and
 *            after every bs_tilemap_rebind; BS_EINVAL otherwise (bs_last_error says so)
 *   limit    n_kv_heads * n_k_tiles * head_dim * 256 bytes (K plus V^T, as if both were packed) must fit the scratch:
 *            BS_EUNSUPPORTED otherwise, nothing launched (96 MiB hold 4 KV heads x 768 key tiles of d = 128:
 *            a 40K-token prompt with its compact tiles).  Partial results of work units that are cut (few rows
 *            behind many keys) go behind the packed tiles or, if there is no room, to a workspace that
 *            bs_tilemap_prepare takes
 * Every call on a GPU uses that GPU's one array: calls that overlap in time on one GPU (two streams, two
 * threads) race on it; calls queued on one stream are safe.  The pre-pass rewrites every tile slot it
 * uses, so nothing needs clearing between calls.
 * Other arguments and errors as bs_attn_prefill.
 */
#define BS_STATIC_SCRATCH_MIB 96
int bs_attn_prefill_static(const void *q, const void *k, const void *v, void *out, bs_tilemap *tm,
                           int32_t n_q_heads, int32_t gqa_group, int32_t head_dim, float scale, void *stream);

/* Size of that array in bytes. */
int64_t bs_static_scratch_bytes(void);

/*
 * Offline characterisation, prompt level (paper Sec. 4.1, Alg. 1), for all query heads of one layer:
 * the attention output under the dense causal mask is the reference; for the masks Sink,
 * Intra-Image, Intra-Image+Sink, in this order,
 *     NMSE = || Attn_mask - Attn_ref ||^2 / || Attn_ref ||^2      (over the head's [L, head_dim] output)
 * and the head takes the first mask with NMSE < alpha (strictly), Dense if none passes.
 *   q, k, v      device pointers, layouts as for bs_attn_prefill; spans / seq_len / sink_len as for
 *                bs_build_tilemap (host)
 *   alpha        the layer's threshold alpha_layer (the paper recommends 0.1 for Qwen-type models)
 *   map_flags    options for the tile map the call builds (BS_MAP_*); sink_offsets /
 *                n_sink_offsets / window as for bs_build_tilemap_model
 *   head_type    host, n_q_heads values out (bs_head_class)
 *   nmse         host, [3][n_q_heads] out, row m = mask m + 1; may be NULL.  All three masks are
 *                evaluated for every head (Alg. 1 stops at the first that passes, which only saves
 *                work: the head types are the same).  A reference of norm zero gives 0 if the masked
 *                output is zero as well, +inf otherwise.
 * The four outputs come from bs_attn_prefill in `dtype` (bf16: the outputs are rounded to bf16 before
 * they are compared, which puts a floor of about 1e-5 under the NMSE), the squared errors are
 * accumulated in fp64 and the decision is taken in fp64.
 * Builds ONE tile map of the prompt and binds it to the four class vectors in turn (bs_tilemap_rebind).  Takes
 * two output-sized device buffers from the library's block cache for the duration of the call (hipMalloc only
 * while the cache is cold; the blocks stay cached afterwards) and returns after `stream` has drained (this
 * is an offline routine).
 * Errors: as bs_build_tilemap_ex and bs_attn_prefill; nothing is written to head_type / nmse on error.
 */
int bs_characterize_prompt(const void *q, const void *k, const void *v, const bs_span *spans,
                           int32_t n_spans, int32_t seq_len, int32_t sink_len, int32_t dtype,
                           int32_t n_q_heads, int32_t gqa_group, int32_t head_dim, float scale,
                           double alpha, uint32_t map_flags, const int32_t *sink_offsets,
                           int32_t n_sink_offsets, int32_t window, uint8_t *head_type, double *nmse,
                           void *stream);

/*
 * The error measure of Alg. 1 on its own: for each of n_heads contiguous blocks of elems_per_head
 * elements, sums[2*h] = sum (attn_mask - attn_ref)^2 and sums[2*h+1] = sum attn_ref^2.
 *   attn_mask, attn_ref   device pointers, 16-byte aligned, dtype BS_BF16 or BS_F32
 *   sums                  device pointer, 2 * n_heads doubles (cleared by the call)
 * Enqueues on `stream` and does not wait.  The sums are accumulated in fp64; the order of the
 * additions across workgroups is not fixed (fp64 atomics), so the last bits may differ between runs.
 * Errors: BS_EINVAL; BS_EUNSUPPORTED (dtype, misaligned pointers, or several heads whose size in
 * bytes is not a multiple of 16); BS_EHIP.
 */
int bs_head_sq_error(const void *attn_mask, const void *attn_ref, int32_t dtype, int32_t n_heads,
                     int64_t elems_per_head, double *sums, void *stream);

/*
 * Offline characterisation, data-set level (paper Sec. 4.2, Alg. 2), for one head: fraction[c] is the
 * share of characterised prompts on which Alg. 1 chose class c (host, 4 values).  Returns Dense if
 * fraction[Dense] > gamma_d, else Sink if fraction[Sink] > gamma_s, else Intra-Image if
 * fraction[Intra-Image] > gamma_i, else Intra-Image+Sink (paper defaults gamma_d = 0.25, gamma_s = 0.6;
 * it names no value for gamma_i).  Host only.  Returns the class (0..3) or BS_EINVAL.
 */
int bs_aggregate_head_type(const double *fraction, double gamma_d, double gamma_s, double gamma_i);

/*
 * Alg. 2 for all heads of a layer, from the prompt-level results: head_types (host) is
 * [n_prompts][n_q_heads], one row per characterised prompt as bs_characterize_prompt returned it.
 * Counts, per head, the share of prompts that chose each class (the head_type_fraction of Alg. 2;
 * written to fraction[n_q_heads][4] if non-NULL) and applies bs_aggregate_head_type to it:
 * head_class[n_q_heads] (host) is the class vector to pass to bs_build_tilemap for this layer.
 * Host only.  Errors: BS_EINVAL (null pointers, non-positive counts, a type above 3).
 */
int bs_aggregate_layer(const uint8_t *head_types, int32_t n_prompts, int32_t n_q_heads, double gamma_d,
                       double gamma_s, double gamma_i, uint8_t *head_class, double *fraction);

/*
 * The layer threshold of Alg. 1 under the paper's linear schedule (App. "Impact of Linear alpha_layer
 * for Gemma 3"): alpha_first + (alpha_last - alpha_first) * layer_idx / num_layers, which keeps the
 * first layers denser.  The paper uses 0.005 .. 0.195 for Gemma 3 (12B), 0.001 .. 0.099 for Gemma 3 (4B)
 * and a fixed 0.1 (alpha_first = alpha_last) for the Qwen-type models.  Host only.  NaN for
 * num_layers <= 0 or layer_idx outside [0, num_layers].
 */
double bs_alpha_layer(double alpha_first, double alpha_last, int32_t layer_idx, int32_t num_layers);

/* ---------------------------------------------------------------------------------------------------------------
 * Around the KV cache: rotary positions, a cache in pages, attention of one new token per sequence over it, and eviction
 * from it.  With bs_attn_prefill before them these are a model's attention from the prompt to the last token of the answer.
 * A generated token is text, and text tokens see every earlier token under every head class (paper Sec. 3.2), so the
 * classes play no part here.  (The paper keeps the whole cache; bs_cache_evict is for those who cannot.)
 *
 * These calls keep nothing: no state of the library, no allocation, no wait.  They enqueue kernels on `stream` (NULL = default
 * stream) and can be captured into a HIP graph; what changes from token to token (lengths, slots, positions, page
 * tables) lies on the device.  Workspaces are the caller's: a call owns its workspace until its kernels are done, so calls that may
 * overlap, and graphs that may be replayed at the same time, need one each.  All pointers are device pointers of the
 * current HIP device unless they say host, and `stream` is one of its streams.  Threads may call at the same time.
 * Errors of all of them: BS_EINVAL (null pointers, sizes or strides that cannot be, a workspace that is too small),
 * BS_EUNSUPPORTED (dtype, head_dim, page size, alignment or a size beyond 32 bits that the kernels do not implement), BS_EHIP.  Nothing is
 * launched on error.
 */

/* Some heads of some tokens: element c of head h of token t at data[h * head_stride + t * token_stride + c], strides in
 * elements, >= 0.  [n_heads][n_tokens][head_dim] and [n_tokens][n_heads][head_dim] are both of this kind. */
typedef struct { void *data; int64_t head_stride, token_stride; int32_t n_heads; } bs_heads;

#define BS_ROPE_HALF        0   /* channel i turns with channel i + rotary_dim / 2        */
#define BS_ROPE_INTERLEAVED 1   /* channel 2 i turns with channel 2 i + 1                 */

#define BS_ROPE_PLAIN  0   /* f_i = base^(-2 i / rotary_dim), in radians per position                                        */
#define BS_ROPE_LINEAR 1   /* f_i / factor                                                                                   */
#define BS_ROPE_BASE   2   /* f_i of the base times factor^(rotary_dim / (rotary_dim - 2)): the slowest pair turns 1 / factor as fast */
#define BS_ROPE_PARTS  3   /* f_i (g + (1 - g) / factor), g = (n_i - slow) / (fast - slow) held within [0, 1], n_i the turns that pair i
                              makes over original_len positions: fast pairs stay as they are, slow ones are interpolated       */

#define BS_ROPE_MAX_PAIRS 128
#define BS_ROPE_MAX_AXES  4

/* Rotary positions: pair i of a head is turned by the angle position[axis[i]] * freq[i] and multiplied by `magnitude`; channels
 * from rotary_dim on are left as they are.  Plain data on the host, copied by every call: bs_rope_init fills it in, and a
 * caller may change freq, axis or magnitude afterwards. */
typedef struct {
    int32_t rotary_dim;                  /* even, 2 .. 2 * BS_ROPE_MAX_PAIRS                  */
    int32_t layout;                      /* BS_ROPE_HALF or BS_ROPE_INTERLEAVED               */
    int32_t n_axes;                      /* axes of a position, 1 .. BS_ROPE_MAX_AXES         */
    float magnitude;
    double freq[BS_ROPE_MAX_PAIRS];
    uint8_t axis[BS_ROPE_MAX_PAIRS];     /* which axis of the position turns a pair           */
} bs_rope;

/*
 * Fill in *rope (host only).  original_len, fast and slow are looked at for BS_ROPE_PARTS only, factor for all but
 * BS_ROPE_PLAIN.  sections (host, n_axes values >= 0 that add up to rotary_dim / 2; NULL for one axis): the first
 * sections[0] pairs follow axis 0, the next ones axis 1, and so on (multimodal models: time, height, width).
 * Errors: BS_EINVAL; *rope is untouched then.
 */
int bs_rope_init(bs_rope *rope, int32_t rotary_dim, int32_t layout, double base, int32_t scaling, double factor,
                 int32_t original_len, double fast, double slow, double magnitude, const int32_t *sections, int32_t n_axes);

#define BS_ROPE_INVERSE 1u   /* turn backwards: the gradient of the rotation (same magnitude) */

/*
 * Apply rotary positions to n_tensors (1 or 2: q and k of a layer) sets of heads of the same tokens.
 *   x, y       host, [n_tensors]; y[i] as many heads as x[i].  y may be x itself (same data and strides), else they do
 *              not overlap; rows of y lie apart (BS_EINVAL), those of x may be the same one (stride 0)
 *   head_dim   even, rotary_dim <= head_dim <= 2 * BS_ROPE_MAX_PAIRS
 *   positions  device, row a = axis a, axis_stride elements apart: positions[a * axis_stride + t], any 32-bit value
 *   flags      0 or BS_ROPE_INVERSE
 * The angle is formed and reduced in 64 bits, off by at most 3 |angle| 2^-53: less than the fp32 sine's 2^-24 up to 10^8 radians, 7e-7
 * at 2^31.  The product is fp32, rounded
 * once.  Any alignment and stride; 16-byte loads are used where pointers, strides and sizes allow them.  n_tokens may be 0, and pointers to
 * data, positions and lists of tokens null then (as of bs_cache_append).
 * BS_EUNSUPPORTED for more than 2^31 - 1 pieces, n_tokens times those of a row: head_dim / 2 channels in loads of up to 16 bytes.
 */
int bs_rope_apply(const bs_rope *rope, const bs_heads *x, const bs_heads *y, int32_t n_tensors, int32_t dtype, int32_t n_tokens,
                  int32_t head_dim, const int32_t *positions, int64_t axis_stride, uint32_t flags, void *stream);

/* A KV cache in pages.  Slot j of sequence s and KV head h lies in page p = page_table[s * max_pages + j / page_size] at
 * k[p * page_stride + h * head_stride + (j % page_size) * slot_stride], head_dim contiguous elements, and likewise in v; strides in
 * elements; where the cache is written, its rows lie apart, the axes nested in any order (BS_EINVAL), so that [page][head][slot][d] and
 * [page][slot][head][d] both fit, and k and v do not overlap.  A page number outside [0, n_pages) means that these
 * slots have no page: they are not written, and nobody sees them.  k and v 16-byte aligned, strides multiples of 16 bytes;
 * head_dim a multiple of 8 up to 256 (bs_attn_decode: 64 or 128), page_size a multiple of 16. */
typedef struct {
    void *k, *v;
    const int32_t *page_table;                       /* device [n_seqs][max_pages]                     */
    int64_t page_stride, head_stride, slot_stride;
    int32_t dtype;                                   /* BS_BF16 or BS_F32                              */
    int32_t n_kv_heads, head_dim, page_size, n_pages;
    int32_t n_seqs, max_pages;
} bs_cache;

/* What is known of every slot besides K and V, per sequence and KV head; row s * n_kv_heads + h, row_stride >= max_pages *
 * page_size elements apart.  weights: the attention that the slot has received; order: the running number of its token in the
 * sequence (once slots were evicted, slots no longer lie in that order). */
typedef struct { float *weights; int32_t *order; int64_t row_stride; } bs_slots;

/*
 * Write new tokens into the cache: K rotated if `rope` is not NULL, V as it is; and rotate q of the same step along.
 *   k, v         n_kv_heads heads of n_tokens tokens in the cache's dtype; any strides
 *   token_seq    device [n_tokens]: the sequence of each token; NULL: token t belongs to sequence t
 *   token_slot   device [n_tokens]: the slot it goes to.  A token whose sequence or slot is out of range (a padded batch: -1), or
 *                whose slot has no page, is not written.  No two tokens may name one slot.
 *   rope, positions, axis_stride   as for bs_rope_apply; NULL: K and q are not rotated
 *   q, q_out     as x and y of bs_rope_apply; both NULL: no q.  With q, rope may not be NULL.
 *   slots        NULL, or what is set for every slot written (either pointer may be NULL): weights 0, order token_order[t] (device
 *                [n_tokens]; NULL: the slot's number)
 * The lengths of the sequences are the caller's to count.
 */
int bs_cache_append(const bs_cache *cache, const bs_heads *k, const bs_heads *v, int32_t n_tokens, const int32_t *token_seq,
                    const int32_t *token_slot, const bs_rope *rope, const int32_t *positions, int64_t axis_stride, const bs_heads *q,
                    const bs_heads *q_out, const bs_slots *slots, const int32_t *token_order, void *stream);

/* Root-mean-square norm of every head's d channels: x -> x (mean x^2 + eps)^-1/2 (weight + offset).  Squares and sums are fp32, so channels
 * beyond 10^18 overflow. */
typedef struct {
    const void *weight[2];   /* device, [head_dim] each: of the first and the second tensor of a call (bs_cache_append_norm: of q, of k); NULL: ones, without the offset */
    int32_t weight_dtype;    /* BS_BF16 or BS_F32, both alike; any alignment of their elements */
    float eps;               /* > 0 (at least the smallest normal fp32 number) */
    float offset;            /* 0, or 1 where a model keeps its weights less one */
} bs_norm;

/*
 * Norm of every head and the rotary positions behind it in one pass: bs_rope_apply of the normed rows, which are not rounded in between.
 * Arguments as those of bs_rope_apply; rope NULL: no rotation (positions are not looked at then).  y may be x.  BS_EUNSUPPORTED as there, with the pieces of a row
 * rounded up to a power of two, at most 64.
 */
int bs_norm_rope(const bs_norm *norm, const bs_rope *rope, const bs_heads *x, const bs_heads *y, int32_t n_tensors, int32_t dtype, int32_t n_tokens,
                 int32_t head_dim, const int32_t *positions, int64_t axis_stride, void *stream);

/*
 * Its gradient: from x and dy (the gradient of y) dx, and dweight [n_tensors][head_dim] in fp32, the sum over all heads and tokens (NULL: not wanted; it is
 * written, not added to; of no tokens it is zero).  Nothing is kept from the way there.
 *   dx           as many heads as x; may be x or dy (same data and strides), else it does not overlap them; rows of dx lie apart, those of x and dy may be
 *                the same one (stride 0)
 *   workspace    at least bs_norm_rope_grad_workspace bytes, 16-byte aligned; not looked at if dweight is NULL
 * Any number of tokens.  Same inputs, same bits.
 */
int bs_norm_rope_grad(const bs_norm *norm, const bs_rope *rope, const bs_heads *x, const bs_heads *dy, const bs_heads *dx, float *dweight, int32_t n_tensors,
                      int32_t dtype, int32_t n_tokens, int32_t head_dim, const int32_t *positions, int64_t axis_stride, void *workspace, int64_t workspace_bytes,
                      void *stream);

/* Bytes of workspace of bs_norm_rope_grad (at most 4 MB); a negative error code for arguments that the call would refuse. */
int64_t bs_norm_rope_grad_workspace(int32_t n_tensors, int32_t dtype, int32_t n_tokens, int32_t head_dim);

/*
 * bs_cache_append with norms: K goes into the cache normed with norm->weight[1] and rotated if `rope` is not NULL, V as it is; q of the same step is normed with
 * norm->weight[0] and rotated likewise.  All else as of bs_cache_append, but q may come without a rope.
 */
int bs_cache_append_norm(const bs_cache *cache, const bs_heads *k, const bs_heads *v, int32_t n_tokens, const int32_t *token_seq, const int32_t *token_slot,
                         const bs_norm *norm, const bs_rope *rope, const int32_t *positions, int64_t axis_stride, const bs_heads *q, const bs_heads *q_out,
                         const bs_slots *slots, const int32_t *token_order, void *stream);

/*
 * Attention of one new token per sequence over the cache, its own slot included:
 *   out[s, h, :] = sum_j softmax_j( scale * <q[s, h], K[s, h / G, j]> ) * V[s, h / G, j, :],  G = n_q_heads / n_kv_heads,
 * over the slots j < lens[s], with window > 0 only those with lens[s] - j <= window; zeros where there is none.
 *   q, out       n_q_heads heads of n_seqs tokens (token s = sequence s) in the cache's dtype, 16-byte aligned, strides
 *                multiples of 16 bytes; n_q_heads a multiple of n_kv_heads; out does not overlap q
 *   lens         device [n_seqs]; held within [0, max_pages * page_size]
 *   slots, slots_out   NULL, or (both) weights_out[j] = weights[j] + the sum over the group's G heads of the probability of slot j,
 *                for j < lens[s]; other entries are not touched.  slots_out may be slots, else they do not overlap.  order is
 *                not looked at.  Not together with a window (BS_EUNSUPPORTED), which bounds a layer's cache without weights.
 *   workspace    at least bs_attn_decode_workspace bytes, 16-byte aligned
 * Slots that are not seen may hold anything, infinities and NaN too; a seen one with such a value can make the rows that see it
 * not finite.  Probabilities (bf16: as three bf16 numbers each), scores, sums and weights are fp32; the result is rounded once.
 * Same inputs, same bits: nothing depends on the order in which workgroups finish.
 */
int bs_attn_decode(const bs_cache *cache, const bs_heads *q, const bs_heads *out, const int32_t *lens, int32_t window, float scale,
                   const bs_slots *slots, const bs_slots *slots_out, void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of workspace of bs_attn_decode for this cache and head count, with weights or without; a negative error code for
 * arguments that the call would refuse.  Depends on the sizes in *cache, not on lengths; on the current device's number of compute units.  With
 * weights the scores of every slot that the page table has room for: 4 n_seqs n_q_heads max_pages page_size bytes and some (48 sequences, 40 heads, a table of
 * 131072 slots: 1.0 GB; of 16384: 0.13), else a few MB at most. */
int64_t bs_attn_decode_workspace(const bs_cache *cache, int32_t n_q_heads, int32_t with_weights);

#define BS_TREE_MAX_TOKENS 256

/*
 * Attention of a few drafted tokens per sequence over the cache, their own slots included.  The drafted tokens of a sequence may be a tree, several guesses at
 * what comes next: each sees the sequence and those of the drafted tokens that its mask names.
 *   out[t, h, :] = sum_j softmax_j( f(scale * <q[t, h], K[s, h / G, j]>) ) * V[s, h / G, j, :],  G = n_q_heads / n_kv_heads,  f(x) = x, or with cap > 0 cap tanh(x / cap)
 *   q, out       n_q_heads heads of n_tokens tokens in the cache's dtype, 16-byte aligned, strides multiples of 16 bytes; n_q_heads a multiple of n_kv_heads; out
 *                does not overlap q
 *   first        device [n_seqs + 1], ascending: tokens first[s] .. first[s + 1] - 1 are sequence s's; a sequence may have none.  Tokens that no sequence has, and those of a sequence behind its
 *                max_tokens-th, are left as they were.  (Values are held within [0, n_tokens].)
 *   lens         device [n_seqs]: slots in use before the drafted tokens; held within [0, max_pages * page_size].  Drafted token i of sequence s is in slot lens[s] + i, and
 *                a token sees all slots below lens[s].
 *   max_tokens   most drafted tokens of a sequence, 1 .. BS_TREE_MAX_TOKENS
 *   mask         device [n_tokens][mask_words]: bit a % 64 of word a / 64 of token t is set if it sees drafted token a of its sequence (itself is one of them).
 *                mask_words >= max_tokens / 64, rounded up; bits of tokens that the sequence does not have mean nothing.  NULL (mask_words 0): a chain, each token sees itself
 *                and the drafted ones before it.  A row that sees nothing is zero.
 *   window       > 0: of the slots that a token sees by the above, only the last `window`
 *   cap          >= 0; 0: none
 *   workspace    at least bs_attn_tree_workspace bytes, 16-byte aligned
 * n_tokens may be 0, and pointers to q, out and the mask null then (as of bs_cache_append).
 * Slots that no token sees may hold anything, infinities and NaN too, and a slot that only some see leaves the others as they are; one with such a value
 * can make the rows that see it not finite.  Probabilities (bf16: as three bf16 numbers each), scores and sums are fp32; the result is rounded once.  Same inputs,
 * same bits.
 */
int bs_attn_tree(const bs_cache *cache, const bs_heads *q, const bs_heads *out, int32_t n_tokens, const int32_t *first, const int32_t *lens, int32_t max_tokens,
                 const uint64_t *mask, int32_t mask_words, int32_t window, float scale, float cap, void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of workspace of bs_attn_tree for these sizes; a negative error code for arguments that the call would refuse.  Sizes decide, not lengths; at most 70 MB. */
int64_t bs_attn_tree_workspace(const bs_cache *cache, int32_t n_q_heads, int32_t n_tokens, int32_t max_tokens);

/*
 * Keep the drafted tokens that were accepted: slot lens[s] + i takes what slot lens[s] + path[s][i] held when the call began, K, V, weight and order, for
 * i < n_path[s], and lens_out[s] = lens[s] + n_path[s].  Other slots stay as they are, those of rejected tokens among them; they are free again.
 *   lens, lens_out   device [n_seqs], held within [0, max_pages * page_size]; may be the same, else lens_out overlaps nothing that is read
 *   path         device [n_seqs][max_path]: numbers of drafted tokens, in any order, one more than once too; where one is outside [0, BS_TREE_MAX_TOKENS), or either slot has
 *                no page, that slot stays as it is
 *   n_path       device [n_seqs], held within [0, max_path]
 *   max_path     0 .. BS_TREE_MAX_TOKENS
 *   slots        NULL, or weights and order (either pointer may be NULL) that move along
 * Pages that are moved into must not be shared with other sequences.
 */
int bs_cache_accept(const bs_cache *cache, const int32_t *lens, int32_t *lens_out, const int32_t *path, const int32_t *n_path, int32_t max_path,
                    const bs_slots *slots, void *stream);

/*
 * Cut the cache back to `keep` slots per sequence and KV head, where it holds more.  Kept are the slots whose order is below
 * keep_first or above (the largest order of the row) - keep_last, and of the others those with the largest weights; of equal
 * weights the lower slot; a NaN counts as the smallest.  keep >= 1, keep_first + keep_last <= keep.  (Where orders repeat, so
 * that the first two are more than `keep`: the lowest of these slots.)
 * Kept slots at or behind `keep` move into the evicted slots before it, the first into the first, and so on, K, V, weight and order
 * alike; all other slots stay where they are.  (So as few as can be move: a row cut back from 4160 slots to 4096 moves at most 64.  Keys
 * carry their positions, attention does not mind the order.)
 * A sequence that is cut back (lens[s] > keep) needs a page for every slot below lens[s]; others may lack some.  (Page numbers are on the device, so
 * this cannot be refused.  A slot without a page is ranked like any other, and only its weight and order move: a token that moves into it is
 * lost, and a hole that it moves into shows the evicted token's K and V under its name.  So a sequence whose first pages were given back, behind
 * a window, is not one to cut back.  Nothing outside the cache is touched in any case.)
 *   lens, lens_out     device [n_seqs]: slots in use (held within [0, max_pages * page_size]), and min(lens, keep); may be the same
 *   slots, slots_out   weights and order before and after; entries from lens_out on are not touched; may be the same, else they do not
 *                      overlap
 *   workspace          at least bs_cache_evict_workspace bytes, 16-byte aligned
 * Pages that are moved into must not be shared with other sequences.
 */
int bs_cache_evict(const bs_cache *cache, const int32_t *lens, int32_t *lens_out, int32_t keep, int32_t keep_first, int32_t keep_last,
                   const bs_slots *slots, const bs_slots *slots_out, void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of workspace of bs_cache_evict for this cache; a negative error code for arguments that the call would refuse.  Sizes decide, not lengths, and so they
 * do how the call works: 64 sequences of 8 heads cut from 4160 slots to 4096 take 28 us where the page table has room for 4160 or 8192 slots, 36 with 32768, 64
 * with 131072.  A caller whose sequences are short passes a cache whose table is cut to that (rows of max_pages
 * entries). */
int64_t bs_cache_evict_workspace(const bs_cache *cache, int32_t keep);

/* Static description of an error code (error behaviour of this boundary; no passage of the paper). */
const char *bs_strerror(int code);

/* Detail of the most recent BS_EHIP / BS_ENOMEM failure on the calling thread (the HIP call
 * that failed and its error string); "" if none.  The pointer stays valid for the thread's life. */
const char *bs_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* BLINDSIGHT_H */
