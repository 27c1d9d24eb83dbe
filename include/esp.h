/*
 * esp.h -- C ABI of libesp: one GPU's share of elastic-sequence-parallel (ESP)
 * attention on AMD MI355X (gfx950), after LoongServe (arXiv 2404.09526).
 *
 * The library computes, with hand-written HIP kernels only (there is no CPU or
 * library fallback):
 *   esp_partial_attn_prefill  a causal query chunk against ONE local KV shard
 *   esp_partial_attn_decode   one query token per request against the KV rows
 *                             this instance holds in its token-granular pool
 *   esp_merge_partials        log-sum-exp combination of partial results
 *   esp_kv_append             scatter of K/V rows into scheduler-chosen slots
 *   esp_partial_attn_decode_shared  decode of requests that share a long prefix
 *   esp_qk_norm_rope_append   norm and rotation of new queries and keys on their
 *                             way to attention and into the pool
 *   esp_extend_block_table, esp_build_slots  pages and slot lists from lengths
 *   esp_kv_append_q4, esp_kv_gather_q4, esp_partial_attn_decode_q4  the pool in 4 bits
 *   esp_accumulate_attn_weights, esp_evict_slots  a pool of fewer tokens: attention
 *                             weights summed per slot, the slots that stay chosen by them
 * and, on the host, the scheduler's two numeric helpers for the prefill phase:
 *   esp_plan_prefill_batches  batching plan (dynamic program over requests and instances)
 *   esp_fit_prefill_model     least-squares fit of the iteration-time model
 *
 * Conventions common to all calls
 *   - Every data pointer is DEVICE memory owned by the caller unless a
 *     parameter says "host".  The library never allocates, frees or keeps
 *     device memory.  Its only state between calls is process-wide and small:
 *     a launch counter that tags the prefill workspace (see there) and the
 *     debugging switches at the end of this file.
 *   - bf16 tensors are passed as `const void*` (16-bit patterns); layouts are
 *     token-major and dense: Q/O [T, Hq, D], K/V [T, Hkv, D], pools
 *     [S, Hkv, D] (one for K, one for V), LSE [T, Hq] float.
 *   - Query head h reads KV head h / (Hq / Hkv).  D must be 128.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *     Work is enqueued asynchronously; the library never synchronises.
 *   - Results are deterministic: the same inputs give the same bits, in any
 *     workspace of at least the size that the matching *_bytes() reports (a
 *     smaller one that is accepted, see the prefill and decode calls, cuts the
 *     work into fewer parts, and fp32 sums are then added in another order).
 *   - Return value: ESP_OK or a negative esp_status; nothing is enqueued when
 *     an error is returned, except for ESP_ERR_HIP where the launch itself
 *     failed.  esp_last_error() gives a thread-local message.
 *   - The CONTENT of device index arrays (positions, offsets, slots) is
 *     trusted, as it comes from the scheduler (scaling plan, Sec. 3 and 4.1):
 *     out-of-range or duplicate slots are undefined behaviour.  With
 *     ESP_DEBUG_VALIDATE=1 in the environment the calls check them first, on
 *     the host (the stream is waited for and the arrays are copied back; a
 *     debugging aid): prefix offsets must run from 0 to the row count without
 *     decreasing, with no piece above the stated maximum; decode slots must lie
 *     in [0, num_slots); append slots must be below num_slots and, where not
 *     negative, distinct.  A violation returns ESP_ERR_INVALID_ARG.
 *   - A row with no visible key yields O = 0 and LSE = -inf, never NaN.  A row
 *     that sees a key with a NaN score yields NaN in both.
 *   - LSE is the natural logarithm of the sum of exp(softmax_scale * q.k)
 *     over the visible keys.
 */
#ifndef ESP_H_
#define ESP_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t esp_status;
#define ESP_OK                0
#define ESP_ERR_INVALID_ARG  (-1) /* null pointer, negative size, Hq % Hkv != 0, P out of range */
#define ESP_ERR_UNSUPPORTED  (-2) /* D != 128                                                   */
#define ESP_ERR_WORKSPACE    (-3) /* workspace missing or too small for the call               */
#define ESP_ERR_HIP          (-4) /* a HIP launch failed; see esp_last_error()                 */

#define ESP_MAX_PARTIALS 16

/*
 * Prefill partial attention (Sec. 2.3, Fig. 1: instance i attends its local
 * queries q_i to a key-value segment kv_j; kernel remarks in Sec. 6).
 *
 * For every local query row t and head h: softmax attention over the rows of
 * ONE KV shard that belong to the same request, restricted (causal != 0) to
 * rows with kv_pos <= q_pos[t] on GLOBAL token positions, so that contiguous,
 * striped or arbitrary sequence-parallel layouts use the same call.  Emits the
 * un-merged output O (bf16, normalised within the shard) and LSE (float).
 *
 *   q [Tq,Hq,D], k/v [Tkv,Hkv,D] bf16; q_pos [Tq], kv_pos [Tkv] int32.
 *   cu_q, cu_kv: int32 [batch+1] prefix offsets of the requests packed in q and
 *     in the shard (request r owns rows cu[r]..cu[r+1]); both NULL with
 *     batch = 1 means one request spanning everything.
 *   max_q, max_kv: upper bounds on a request's row counts (host-known).  Results
 *     do not depend on them but for the order of fp32 sums; whether and how the
 *     keys of a batch are cut into parts follows the longest request, max_kv, so
 *     a bound that is far from it costs time.
 *   O [Tq,Hq,D] bf16, LSE [Tq,Hq] float: written for every row.
 *   workspace: at least esp_prefill_workspace_bytes(...) bytes, 256-byte
 *     aligned; contents need not be preserved between calls.  It holds, for calls
 *     with few query rows against many keys, the partial results of the parts the
 *     keys are cut into (a smaller block, down to 256 bytes, is accepted: such a
 *     call then runs in as many parts as fit, or uncut, and slower; the size does not grow with Tq and Tkv
 *     throughout, so a block for several calls takes the largest of theirs; for a
 *     batch it covers requests of unequal length too, up to 64 MB of parts), and
 *     work counters that are never cleared: every launch tags them with a number of
 *     its own (a per-process random 32-bit start, then +1 per call), so memory
 *     that has never been written is mistaken for the current launch's counters
 *     with probability 2^-32 per fresh workspace (query tiles would then be
 *     skipped).  A caller that wants certainty zeroes a new workspace once:
 *     the tag is never 0.  Calls that may run at the same time need a
 *     workspace each.
 * Positions may be in any order; ascending order inside a request lets whole
 * tiles be skipped or left unmasked.
 */
esp_status esp_partial_attn_prefill(
    const void* q, const void* k, const void* v,
    const int32_t* q_pos, const int32_t* kv_pos,
    const int32_t* cu_q, const int32_t* cu_kv, int32_t batch,
    int32_t Tq, int32_t Tkv, int32_t max_q, int32_t max_kv,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale, int32_t causal,
    void* O, float* LSE,
    void* workspace, size_t workspace_bytes, void* stream);

size_t esp_prefill_workspace_bytes(int32_t Tq, int32_t Tkv, int32_t batch,
                                   int32_t Hq, int32_t Hkv, int32_t D);

/*
 * The same call with O [Tq,Hq,D] written as float: for partials that stay on this
 * GPU until they are combined (the rounds of sequence-parallel prefill, Sec. 2.3:
 * one call per key-value segment that passes by, one combination at the end), so
 * that the combined result is rounded to bf16 once, by esp_merge_partials_f32,
 * and not once per partial and again after the combination.  Everything else,
 * the workspace included, as in esp_partial_attn_prefill.
 */
esp_status esp_partial_attn_prefill_f32(
    const void* q, const void* k, const void* v,
    const int32_t* q_pos, const int32_t* kv_pos,
    const int32_t* cu_q, const int32_t* cu_kv, int32_t batch,
    int32_t Tq, int32_t Tkv, int32_t max_q, int32_t max_kv,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale, int32_t causal,
    float* O, float* LSE,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Decode partial attention (Sec. 4.2, Fig. 8: every instance of the group runs
 * the local attention of the batch's query tokens against the key-value rows it
 * holds; token-granular pool of Sec. 6).
 *
 * Request b attends its single query token to the pool rows
 * slot_idx[seq_offsets[b] .. seq_offsets[b+1]) (no mask: all resident tokens
 * precede the query).  A request with no resident row gives O = 0, LSE = -inf.
 *
 *   q [B,Hq,D] bf16; k_pool/v_pool [num_slots,Hkv,D] bf16;
 *   slot_idx int32 [total_tokens]; seq_offsets int32 [B+1], seq_offsets[0] = 0,
 *   seq_offsets[B] = total_tokens; max_len >= every request's length.
 *   O [B,Hq,D] bf16, LSE [B,Hq] float.
 *   workspace: at least esp_decode_workspace_bytes(...) bytes, 256-byte aligned.
 *     A smaller one is accepted down to room for ranges of 512 tokens or a
 *     1024th of total_tokens, whichever is more (eight steps of the kernel on
 *     the layouts read in whole rows, see below); the call then runs on fewer
 *     ranges than it would like, and may be slower.
 * Every Hq that is a multiple of Hkv is accepted (MHA, GQA, MQA).  With 4, 8, 16 or
 * a multiple of 32 KV heads and 1 or 2 query heads per KV head a pool row is read
 * in whole-row bursts and multiplied on the vector ALU; every other layout is read
 * one KV head (256 bytes of a row) at a time and multiplied on the matrix cores,
 * the query heads of a KV head as the columns of a tile.
 */
esp_status esp_partial_attn_decode(
    const void* q, const void* k_pool, const void* v_pool, int64_t num_slots,
    const int32_t* slot_idx, const int32_t* seq_offsets, int32_t B,
    int32_t total_tokens, int32_t max_len,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale,
    void* O, float* LSE,
    void* workspace, size_t workspace_bytes, void* stream);

size_t esp_decode_workspace_bytes(int32_t B, int32_t total_tokens, int32_t max_len,
                                  int32_t Hq, int32_t Hkv, int32_t D);

/*
 * esp_partial_attn_decode for callers that cannot allocate or hand over a
 * workspace: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc.  Same arguments, results and kernels, minus the workspace:
 * the split-K partials go to a block of ESP_DECODE_STATIC_SCRATCH_BYTES of
 * device memory built into the library (each GPU the library runs on holds it
 * until the process ends).  The call allocates and frees nothing.  A call whose
 * esp_decode_workspace_bytes(...) exceeds the block returns ESP_ERR_WORKSPACE.
 * All calls on one GPU share the block: calls that may overlap in time on one
 * GPU (two streams, two threads) race and must use esp_partial_attn_decode
 * with a workspace each.  Nothing in the block has to be cleared between calls.
 */
#define ESP_DECODE_STATIC_SCRATCH_BYTES (32u << 20)
esp_status esp_partial_attn_decode_static(
    const void* q, const void* k_pool, const void* v_pool, int64_t num_slots,
    const int32_t* slot_idx, const int32_t* seq_offsets, int32_t B,
    int32_t total_tokens, int32_t max_len,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale,
    void* O, float* LSE, void* stream);

/*
 * The master's step of a multi-master decode (Sec. 4.2): its local partial
 * attention over the token pool, combined in the same pass with the partial
 * results its peers sent back for the same queries (the combination stated
 * below for esp_merge_partials, with the local result as one more partial).
 * The local result is never rounded to bf16 on its own and no separate merge
 * launch follows.  Arguments as esp_partial_attn_decode, plus
 *   peer_O   : HOST array of n_peers DEVICE pointers, each bf16 [B, Hq, D];
 *   peer_LSE : HOST array of n_peers DEVICE pointers, each fp32 [B, Hq];
 *   n_peers  : 0 .. ESP_MAX_PARTIALS - 1 (0: plain esp_partial_attn_decode).
 * The pointer arrays are read during the call only.  O / LSE receive the
 * FINAL result and must not overlap a peer's arrays (ESP_ERR_INVALID_ARG).
 * The peers' arrays need 4-byte alignment (ESP_ERR_INVALID_ARG), O no more.
 * A master that holds no token of a request (seq_offsets[b+1] ==
 * seq_offsets[b]) passes its peers' combination through.  Errors as
 * esp_partial_attn_decode.
 */
esp_status esp_partial_attn_decode_merge(
    const void* q, const void* k_pool, const void* v_pool, int64_t num_slots,
    const int32_t* slot_idx, const int32_t* seq_offsets, int32_t B,
    int32_t total_tokens, int32_t max_len,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale,
    const void* const* peer_O, const float* const* peer_LSE, int32_t n_peers,
    void* O, float* LSE,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Combination of partial results ("generate the final output", Sec. 2.3;
 * results "sent back to the master", Sec. 4.2).  For each (token, head):
 *   m = max_p LSE_p,  w_p = exp(LSE_p - m),
 *   O = sum_p w_p O_p / sum_p w_p,   LSE = m + ln sum_p w_p.
 * Partials with LSE = -inf weigh 0; all -inf gives O = 0, LSE = -inf.  A NaN
 * LSE_p makes the pair's O and LSE NaN.
 *
 *   O_parts, LSE_parts: HOST arrays of P device pointers (1 <= P <=
 *     ESP_MAX_PARTIALS) to bf16 [T,Hq,D] and float [T,Hq]; read before return.
 *   O [T,Hq,D] bf16; LSE_out [T,Hq] float or NULL.  O may alias O_parts[i].
 */
esp_status esp_merge_partials(
    const void* const* O_parts, const float* const* LSE_parts, int32_t P,
    int32_t T, int32_t Hq, int32_t D,
    void* O, float* LSE_out, void* stream);

/*
 * The same combination of float partials (O_parts[p]: float [T,Hq,D], as
 * esp_partial_attn_prefill_f32 writes them); O is still bf16 and must not alias
 * a partial.
 */
esp_status esp_merge_partials_f32(
    const float* const* O_parts, const float* const* LSE_parts, int32_t P,
    int32_t T, int32_t Hq, int32_t D,
    void* O, float* LSE_out, void* stream);

/*
 * KV append / selective retention (Sec. 4.1, Fig. 7: instances of the new
 * group save selected key-value rows into their pool at the places the scaling
 * plan names; Sec. 4.2: a master saves the new token's K/V into its pool).
 *   k_pool[slot_idx[t]] = k[t], v_pool[slot_idx[t]] = v[t] for slot_idx[t] >= 0;
 *   rows with a negative slot are not kept.  A pure copy of 16-bit patterns.
 *
 *   k, v [T,Hkv,D] bf16; slot_idx int32 [T]; pools [num_slots,Hkv,D] bf16.
 */
esp_status esp_kv_append(
    const void* k, const void* v, const int32_t* slot_idx, int32_t T,
    void* k_pool, void* v_pool, int64_t num_slots, int32_t Hkv, int32_t D,
    void* stream);

/*
 * Prefill partial attention that keeps rows of the shard on the way (proactive
 * scale-down, Sec. 4.1, Fig. 7: while the key-value segments circulate during
 * prefill, every instance of the new, smaller group saves the rows the scaling
 * plan assigns to it into its pool, so that no migration is needed afterwards;
 * overhead claim of Sec. 7.4, Fig. 14).  The attention part is
 * esp_partial_attn_prefill (out_f32 != 0: esp_partial_attn_prefill_f32, O then
 * points to float); in the same pass
 *   k_pool[retain_slot[t]] = k[t], v_pool[retain_slot[t]] = v[t]
 * for every shard row t with retain_slot[t] >= 0, as esp_kv_append would do, but
 * from the tiles that pass through on-chip memory anyway: the rows are read from
 * device memory once.  Rows of requests that have no query row in this call, and
 * rows no query can see, are kept all the same.  With Tq = 0 the call is a plain
 * esp_kv_append.
 *
 *   retain_slot int32 [Tkv] (device); pools [num_slots,Hkv,D] bf16; slots that are
 *   not negative must be distinct and below num_slots (checked only under
 *   esp_debug_set_validate).  Everything else as in esp_partial_attn_prefill.
 */
esp_status esp_partial_attn_prefill_retain(
    const void* q, const void* k, const void* v,
    const int32_t* q_pos, const int32_t* kv_pos,
    const int32_t* cu_q, const int32_t* cu_kv, int32_t batch,
    int32_t Tq, int32_t Tkv, int32_t max_q, int32_t max_kv,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale, int32_t causal,
    const int32_t* retain_slot, void* k_pool, void* v_pool, int64_t num_slots,
    int32_t out_f32, void* O, float* LSE,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Dense view of pool-resident rows: the inverse of esp_kv_append.  The key-value
 * rows a request keeps on this instance live in the token-granular pool at the
 * slots the scheduler chose (Sec. 4.1, Fig. 7; Sec. 6 "unified distributed
 * key-value cache pool"); a later prefill pass over them (the next chunk of a
 * long prompt, a follow-up turn) needs them as one shard.
 *   k[t] = k_pool[slot_idx[t]], v[t] = v_pool[slot_idx[t]]; a slot that is negative
 *   or not below num_slots gives a row of zeros.  A pure copy of 16-bit patterns.
 *
 *   pools [num_slots,Hkv,D] bf16; slot_idx int32 [T]; k, v [T,Hkv,D] bf16 (written).
 */
esp_status esp_kv_gather(
    const void* k_pool, const void* v_pool, const int32_t* slot_idx, int32_t T,
    int64_t num_slots, int32_t Hkv, int32_t D, void* k, void* v, void* stream);

/*
 * esp_partial_attn_prefill over a shard that lives in the pool: row i of the
 * shard is pool row slot_idx[i] (kv_pos[i] is its global position; cu_kv counts
 * shard rows, i.e. entries of slot_idx).  Same results as esp_kv_gather followed
 * by esp_partial_attn_prefill, which is how it is carried out: the gathered rows
 * are staged in the workspace (2 * Tkv * Hkv * D * 2 bytes ahead of the dense
 * call's own block).  All other arguments as in esp_partial_attn_prefill.
 */
esp_status esp_partial_attn_prefill_pool(
    const void* q, const void* k_pool, const void* v_pool, int64_t num_slots,
    const int32_t* slot_idx, const int32_t* q_pos, const int32_t* kv_pos,
    const int32_t* cu_q, const int32_t* cu_kv, int32_t batch,
    int32_t Tq, int32_t Tkv, int32_t max_q, int32_t max_kv,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale, int32_t causal,
    void* O, float* LSE,
    void* workspace, size_t workspace_bytes, void* stream);

size_t esp_prefill_pool_workspace_bytes(int32_t Tq, int32_t Tkv, int32_t batch,
                                        int32_t Hq, int32_t Hkv, int32_t D);

/*
 * The same without staging: the kernel's tile transfers take every row from
 * its pool slot (the slots of a tile travel to on-chip memory one step ahead
 * of the tile, each lane forms the address of the row its 16 bytes belong
 * to), so nothing is copied first and the workspace is the dense call's,
 * esp_prefill_workspace_bytes(...).  Sec. 4.1 / 4.2: key-value rows that an
 * instance kept stay at the slots they were placed in.  Arguments as
 * esp_partial_attn_prefill_pool, plus out_f32 (0: O is bf16; else fp32, as in
 * esp_partial_attn_prefill_f32).  Every slot_idx[i] must lie in
 * [0, num_slots): the kernel trusts it (checked on the host only while
 * esp_debug_set_validate is on).  Results equal those of the staged call up to
 * the order of fp32 additions (the same bound against the exact result holds).
 */
esp_status esp_partial_attn_prefill_pool_direct(
    const void* q, const void* k_pool, const void* v_pool, int64_t num_slots,
    const int32_t* slot_idx, const int32_t* q_pos, const int32_t* kv_pos,
    const int32_t* cu_q, const int32_t* cu_kv, int32_t batch,
    int32_t Tq, int32_t Tkv, int32_t max_q, int32_t max_kv,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale, int32_t causal,
    int32_t out_f32, void* O, float* LSE,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Decode partial attention behind shared prefixes: requests that begin with the
 * same tokens (a system prompt, a document that many questions are asked about)
 * name the same pool rows for them, and those are read once for all of the
 * requests and not once for each.  Requests come in groups of consecutive ones;
 * request b of group g attends its single query token to the rows
 *   prefix_slots[prefix_offsets[g] .. prefix_offsets[g+1])   and
 *   slot_idx[seq_offsets[b] .. seq_offsets[b+1])
 * (no mask).  The result is that of esp_partial_attn_decode on the two lists put
 * together, up to the order of fp32 additions and the rounding of the weights to bf16 (which that
 * call does too, but for 1 or 2 query heads to each of 4, 8, 16 or a multiple of 32 KV heads: there
 * this one's error against 64 bits is 1.2 .. 1.4 times as large, the rounding of O included).  It pays
 * from two requests a group on behind prefixes of some 2000 tokens; where next to nothing is shared, groups of one or prefixes of a
 * few dozen tokens, that call on joined lists takes up to a fifth less time.  Either list may be
 * empty; a request that has neither gives O = 0, LSE = -inf.  An infinity in V shows as itself
 * in the elements of O that see it (with prefix_total = 0 the call is esp_partial_attn_decode, which
 * may show NaN there).
 *
 *   group_offsets int32 [n_groups+1]: requests of group g, from 0 to B;
 *   prefix_offsets int32 [n_groups+1], from 0 to prefix_total; prefix_slots int32 [prefix_total].
 *   max_prefix, max_group: upper bounds of a prefix's tokens and of a group's
 *     requests (host-known; at most prefix_total and B).  A request past max_group of its group is left
 *     without the prefix, a prefix longer than max_prefix is read as far as that.
 *   Everything else as in esp_partial_attn_decode (max_len: of the requests' own
 *   lists).  B = 0 writes nothing.  n_groups = 0 needs prefix_total = 0: the group arrays may
 *   then be NULL.
 *   q, the pools and O lie on 16 bytes (ESP_ERR_INVALID_ARG).
 *   workspace: at least esp_decode_shared_workspace_bytes(...) bytes, 256-byte
 *   aligned; contents need not be preserved.  0 from there: the call would be refused.
 *   That rises with every size but the heads (a block for the largest step is large
 *   enough for all smaller ones), and beyond 128 MiB for the prefixes and as much for the own tokens only as
 *   ranges of 4096 keys of the one and 512 of the other need: a row of 520 Hq bytes for each range of each request.
 * With esp_debug_set_validate the two lists and three offset arrays are checked as
 * in esp_partial_attn_decode.
 */
esp_status esp_partial_attn_decode_shared(
    const void* q, const void* k_pool, const void* v_pool, int64_t num_slots,
    const int32_t* prefix_slots, const int32_t* prefix_offsets, const int32_t* group_offsets,
    int32_t n_groups, int32_t prefix_total, int32_t max_prefix, int32_t max_group,
    const int32_t* slot_idx, const int32_t* seq_offsets, int32_t B,
    int32_t total_tokens, int32_t max_len,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale,
    void* O, float* LSE,
    void* workspace, size_t workspace_bytes, void* stream);

size_t esp_decode_shared_workspace_bytes(int32_t B, int32_t n_groups, int32_t prefix_total, int32_t max_prefix,
                                         int32_t max_group, int32_t total_tokens, int32_t max_len,
                                         int32_t Hq, int32_t Hkv, int32_t D);

/*
 * What new queries and keys go through between their projection and attention,
 * in one pass over them: the norm of every head (where there are weights)
 *   y = x / sqrt(mean(x^2) + eps) * weight          (over the head's 128 elements)
 * the rotation of its first `rot` elements by the token's position
 *   (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t_i = q_pos * inv_freq[i],
 * pair i being elements i and i + rot / 2, or with interleaved != 0 elements 2i and
 * 2i + 1, and the append: K (rotated) and V go to their pool slots as in
 * esp_kv_append.  All arithmetic is fp32, the angle fp64 (a position of 2^20 leaves an
 * fp32 angle a tenth of a radian off); each result is rounded to bf16 once.
 *
 *   q [T,Hq,D], k, v [T,Hkv,D] bf16, a token's heads dense, consecutive tokens
 *     q_stride, k_stride, v_stride elements apart (multiples of 8, at least a
 *     token's heads): q, k and v may be parts of one projection's rows.
 *   q_pos int32 [T]; inv_freq float [rot / 2].  rot = 0: no rotation, both may be NULL.  rot is
 *     even and at most D, without interleaved a multiple of 16.
 *   q_weight, k_weight bf16 [D] or NULL (that norm is left out); eps >= 0.
 *   q_out bf16 [T,Hq,D], tokens q_out_stride elements apart; may be q itself (with q_stride).
 *   k_out, v_out bf16 [T,Hkv,D] dense, or NULL: the rows for a prefill call.  May be k and v themselves where those are dense.
 *   slot_idx int32 [T], k_pool, v_pool [num_slots,Hkv,D]: all NULL, or rows with a
 *     slot in [0, num_slots) are written there (slots must be distinct).
 * Outputs overlap their input only where they are it, and nothing else (q_out next to q, or over q with other strides, is
 * told apart and refused where rows meet: ESP_ERR_INVALID_ARG; so are k_out with k and v_out with v).  Bulk pointers and
 * weights lie on 16 bytes (ESP_ERR_INVALID_ARG).
 */
esp_status esp_qk_norm_rope_append(
    const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
    const int32_t* q_pos, const float* inv_freq, int32_t rot, int32_t interleaved,
    const void* q_weight, const void* k_weight, float eps,
    int32_t T, int32_t Hq, int32_t Hkv, int32_t D,
    void* q_out, int64_t q_out_stride, void* k_out, void* v_out,
    const int32_t* slot_idx, void* k_pool, void* v_pool, int64_t num_slots, void* stream);

/*
 * Block tables and slot lists from request lengths, on the GPU: what a serving step
 * otherwise builds on the host and copies over.  A block table int32 [rows, width] names
 * the pages of each request in order, page p holding the pool slots p * page ..
 * p * page + page - 1 (page = 1: a pool of single tokens); -1: no page.  Request b of
 * a call is row req_row[b] (NULL: row b).  A row outside the table has no tokens' pages.
 *
 * esp_extend_block_table gives the requests the pages that their tokens
 * old_lens[b] .. new_lens[b] - 1 need, ceil(new / page) - ceil(old / page) each (none
 * where that is negative; none past the table's width), in order of the requests
 * from free_pages [n_free] on; an entry for which that holds no page any more gets -1.  Entries
 * of tokens that the requests hold stay as they are.  pages_taken int32 [B+1]: request b got free_pages[
 * pages_taken[b] .. pages_taken[b+1]); pages_taken[B] > n_free says that they
 * did not suffice.  The next call's list begins pages_taken[B] further on, which the host knows from the lengths or
 * reads back: free_pages and n_free are arguments, a captured call takes the same ones each time.  The rows of a call must be distinct.
 *
 * esp_build_slots lists the slots of tokens first_token[b] (NULL: 0) .. lens[b] - 1 of the
 * requests, one request after another, in the form that decode, append, gather and
 * prefill over the pool take.  keep_last > 0: of those only the last keep_last before lens[b], and of the first
 * keep_first of the request (a sliding window behind a few first tokens).  A token
 * without a page has slot -1 (append: not kept; gather: zeros; attention over such a list is undefined).
 *   seq_offsets int32 [B+1]; slot_idx int32 [capacity]; token_pos int32 [capacity] or NULL: pos_first +
 *   pos_stride * (the token's number in its request): global positions of striped shards.
 *   A list longer than `capacity` is cut there, its offsets too (they never exceed
 *   capacity); entries past seq_offsets[B] stay as they were.
 * Lengths below 0 count as 0.  B = 0 writes the single offset 0.
 */
esp_status esp_extend_block_table(
    const int32_t* free_pages, int32_t n_free, const int32_t* req_row,
    const int32_t* old_lens, const int32_t* new_lens, int32_t B, int32_t page,
    int32_t* block_table, int32_t rows, int32_t width, int32_t* pages_taken, void* stream);

esp_status esp_build_slots(
    const int32_t* block_table, int32_t rows, int32_t width, int32_t page, const int32_t* req_row,
    const int32_t* first_token, const int32_t* lens, int32_t B,
    int32_t keep_first, int32_t keep_last, int32_t pos_first, int32_t pos_stride,
    int32_t capacity, int32_t* seq_offsets, int32_t* slot_idx, int32_t* token_pos, void* stream);

/*
 * The pool in 4 bits: the same slots, each head of a slot ESP_Q4_HEAD_BYTES = 68 bytes
 * and not 256, for contexts that the pool in bf16 has no room for, and for decode, whose
 * time is the pool's bytes.  Byte i < 64 of a head holds element 2i in its low and
 * 2i + 1 in its high half, as E2M1 codes (bit 3 the sign; 0, 0.5, 1, 1.5, 2, 3, 4, 6); byte
 * 64 + j is the scale of elements 32j .. 32j + 31, E8M0: s stands for 2^(s - 127), 255 for
 * NaN (of all 32).  (OCP Microscaling formats, MXFP4.)
 * A block is written with the power of two with which no element is off by more than
 * half a step: of its largest magnitude a, 2^(floor(log2 a) - 2), and twice that from a =
 * 1.75 * 2^floor(log2 a) on; at least 2^-125 and at most 2^125 (magnitudes above 6 * 2^125 become
 * that).  Elements go to the nearest code, of two as
 * near to the even one.  A block that holds an infinity or a NaN becomes NaN.
 *
 *   k_pool, v_pool: num_slots slots of [Hkv, 68] bytes, consecutive slots slot_bytes
 *     apart (the same in both; a multiple of 4, at least Hkv * 68), on 4 bytes.  They may
 *     be parts of one block: K and V of a slot next to each other (slot_bytes = Hkv * 136, v_pool
 *     = k_pool + Hkv * 68) are read in one burst.
 *
 * esp_kv_append_q4 writes rows t with a slot in [0, num_slots) there (slots must be distinct); all
 * others are not kept.  k, v bf16 [T,Hkv,D], a token's heads dense, consecutive tokens k_stride and
 * v_stride elements apart (multiples of 8, at least Hkv * D).  Pointers of k and v lie on 16 bytes.
 * esp_kv_gather_q4 gives the values of listed slots as bf16 [T,Hkv,D] (exactly: the values of 4
 * bits are bf16 numbers; with scales of 2^126 and 2^127 the largest would be infinite), for a prefill pass over them; a slot outside the pool gives a row of
 * zeros.  k, v lie on 16 bytes.
 * esp_partial_attn_decode_q4 is esp_partial_attn_decode over such a pool, for any Hq that is a
 * multiple of Hkv.  An infinite value (of those scales) makes the elements of O that it enters infinite.  Weights times
 * values are summed in fp32 before the division, as in all decode calls: over thousands of rows of values next to the largest that sum may pass its range.
 * softmax_scale * log2(e) is a finite number in this call and the next two (ESP_ERR_INVALID_ARG).  q lies on 16 bytes, O on 4.  workspace: at least
 * esp_decode_q4_workspace_bytes(...) bytes (ESP_ERR_WORKSPACE otherwise), 256-byte aligned; it rises with every size,
 * contents need not be preserved.  Calls that may run at the same time need a workspace each.
 * esp_qk_norm_rope_append and esp_partial_attn_decode_shared take the pool in bf16 alone: rows that the first leaves dense go into this one by
 * esp_kv_append_q4, and requests that share a prefix have its slots in their own lists.
 */
#define ESP_Q4_HEAD_BYTES 68
esp_status esp_kv_append_q4(
    const void* k, const void* v, int64_t k_stride, int64_t v_stride, const int32_t* slot_idx, int32_t T,
    void* k_pool, void* v_pool, int64_t slot_bytes, int64_t num_slots, int32_t Hkv, int32_t D, void* stream);

esp_status esp_kv_gather_q4(
    const void* k_pool, const void* v_pool, int64_t slot_bytes, const int32_t* slot_idx, int32_t T,
    int64_t num_slots, int32_t Hkv, int32_t D, void* k, void* v, void* stream);

esp_status esp_partial_attn_decode_q4(
    const void* q, const void* k_pool, const void* v_pool, int64_t slot_bytes, int64_t num_slots,
    const int32_t* slot_idx, const int32_t* seq_offsets, int32_t B,
    int32_t total_tokens, int32_t max_len,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale,
    void* O, float* LSE,
    void* workspace, size_t workspace_bytes, void* stream);

size_t esp_decode_q4_workspace_bytes(int32_t B, int32_t total_tokens, int32_t max_len,
                                     int32_t Hq, int32_t Hkv, int32_t D);

/*
 * Eviction by accumulated attention weight: contexts that the pool has no room for keep the
 * tokens that queries look at.  After a step's attention esp_accumulate_attn_weights adds up,
 * per pool slot, the weights that the step's queries gave it; now and then esp_evict_slots
 * chooses from the sums which entries of the requests' lists stay.
 *
 * esp_accumulate_attn_weights.  Request b has the slots slot_idx[seq_offsets[b] ..
 * seq_offsets[b+1]) and the queries q_offsets[b] .. q_offsets[b+1] - 1 (q_offsets NULL: query b).
 * For each of its entries i,
 *   weight_sum[slot_idx[i]] = decay * weight_sum[slot_idx[i]]
 *     + sum over its queries t and heads h of exp(softmax_scale * q[t,h] . k[slot_idx[i], h/G] - LSE[t,h])
 * with G = Hq / Hkv, in fp32.  With positions, query t leaves out keys of kv_pos[i] > q_pos[t].
 * The LSE is that of the whole attention: a master's merged one where keys are spread over instances.
 * A query with LSE = -inf saw nothing and gives nothing, whatever q holds there; a NaN among the others' q, K or LSE
 * shows in the sums that it enters.  The last `fresh` entries of each list are new tokens: their sums begin at 0, whatever
 * their slots held.  So do all with decay = 0 (nothing is read then).
 *   q bf16 [Tq,Hq,D], LSE float [Tq,Hq]; k_pool bf16 [num_slots,Hkv,D], or (_q4) in 4 bits, slots
 *   slot_bytes apart; q_pos int32 [Tq], kv_pos int32 [total_tokens], both or neither; max_q >= every
 *   request's queries (one that has more: the first max_q), max_len >= every request's entries.
 *   weight_sum float [num_slots].  Slots lie in the pool, none twice in one call (a prefix that requests share
 *   is a list of its own, with the queries of all of them).  q and the pool lie on 16 bytes (in 4 bits: on 4).
 *
 * esp_evict_slots.  Of request b's n entries m = min(n, max(budget, keep_first + keep_last)) stay
 * (budgets int32 [B], device: budgets[b] for budget): the first keep_first, the last
 * keep_last, and of the others those with the largest weight_sum of their slot, of equal ones the
 * first.  NaN is above all, a slot outside the pool below all.  Both lists keep the entries' order:
 *   kept_offsets, freed_offsets int32 [B+1]; kept_slots int32 [kept_capacity], kept_pos the same of
 *   token_pos int32 [total_tokens] (NULL: not asked for), freed_slots int32 [freed_capacity].
 *   A list longer than its capacity is cut there, its offsets too; entries past the last stay as they
 *   were.  kept_slots and kept_offsets are a list that the other calls take, without room between the requests: to go on
 *   with it, it becomes the rows of a block table with pages of one token, which esp_extend_block_table (freed_slots are its free
 *   pages) and esp_build_slots take; larger pages have no holes.  Outputs must not overlap the inputs (ESP_ERR_INVALID_ARG).  B = 0 writes the offsets 0.
 *   workspace: at least esp_evict_workspace_bytes(...) bytes (ESP_ERR_WORKSPACE otherwise), 256-byte
 *   aligned; contents need not be preserved; it rises with every size.
 */
esp_status esp_accumulate_attn_weights(
    const void* q, const float* LSE, const void* k_pool, int64_t num_slots,
    const int32_t* slot_idx, const int32_t* seq_offsets, int32_t B, int32_t total_tokens, int32_t max_len,
    const int32_t* q_offsets, int32_t Tq, int32_t max_q, const int32_t* q_pos, const int32_t* kv_pos,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale, float decay, int32_t fresh,
    float* weight_sum, void* stream);

esp_status esp_accumulate_attn_weights_q4(
    const void* q, const float* LSE, const void* k_pool, int64_t slot_bytes, int64_t num_slots,
    const int32_t* slot_idx, const int32_t* seq_offsets, int32_t B, int32_t total_tokens, int32_t max_len,
    const int32_t* q_offsets, int32_t Tq, int32_t max_q, const int32_t* q_pos, const int32_t* kv_pos,
    int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale, float decay, int32_t fresh,
    float* weight_sum, void* stream);

esp_status esp_evict_slots(
    const float* weight_sum, int64_t num_slots, const int32_t* slot_idx, const int32_t* token_pos,
    const int32_t* seq_offsets, int32_t B, int32_t total_tokens, int32_t max_len,
    const int32_t* budgets, int32_t budget, int32_t keep_first, int32_t keep_last,
    int32_t kept_capacity, int32_t* kept_offsets, int32_t* kept_slots, int32_t* kept_pos,
    int32_t freed_capacity, int32_t* freed_offsets, int32_t* freed_slots,
    void* workspace, size_t workspace_bytes, void* stream);

size_t esp_evict_workspace_bytes(int32_t B, int32_t total_tokens, int32_t max_len);

/*
 * Measurement aids (no part of the method): what this GPU sustains on the two
 * resources that bound the path, for the benchmark's "achievable" figures.
 *   esp_probe_mfma_bf16: every wavefront (8 per CU, all CUs) runs `iters` rounds of
 *     four independent 32x32x16 bf16 MFMAs on register operands taken from
 *     `operands` (device, 16-byte aligned, operand_bytes a multiple of 16; the
 *     values decide how much the multipliers switch, hence the clock under the
 *     power limit).  *flops (host, nullable) receives the FLOPs of the launch.
 *   esp_probe_stream_read: reads `bytes` (a multiple of 16) of device memory once.
 *   sink: 4 bytes of device memory (written only in a case that does not occur).
 */
esp_status esp_probe_mfma_bf16(const void* operands, int64_t operand_bytes, int32_t iters,
                               void* sink, int64_t* flops, void* stream);
esp_status esp_probe_stream_read(const void* src, int64_t bytes, void* sink, void* stream);

/*
 * Prefill batching plan (Sec. 5.3 "Batching", the dynamic program over sorted requests and sorted elastic
 * instances) -- host code, no GPU work; every pointer is HOST memory.
 *
 * Requests are given longest first (req_len[0] >= req_len[1] >= ... >= 1 tokens), instances in the scheduler's
 * order with their unused key-value slots.  A plan cuts the requests and a prefix of the instances into the same
 * number of consecutive non-empty pieces; batch b = requests [req_cuts[b-1], req_cuts[b]) on instances
 * [inst_cuts[b-1], inst_cuts[b]) (cuts start at 0), and must fit: its tokens <= the unused slots of its instances.
 * A batch costs sum over its requests of T / len, with T the iteration-time model below at the coefficients of
 * its degree of parallelism d = its number of instances: coefs[3*(d-1) .. 3*(d-1)+2] = alpha, beta, gamma.
 * The plan of least total cost is returned: *n_batches pieces, their end cuts in req_cuts / inst_cuts (room for
 * min(n_req, n_inst) entries each), the cost in *cost.  If nothing fits, *n_batches = 0 and *cost = +inf.
 * split_req / split_ins: NULL, or [(n_req+1) x (n_inst+1)] tables that receive, for the first i requests on the
 * first k instances, where the last batch starts (the two monotone tables of the section; -1 = no plan).
 */
esp_status esp_plan_prefill_batches(
    const int64_t* req_len, int32_t n_req, const int64_t* free_slots, int32_t n_inst,
    const double* coefs, int32_t* req_cuts, int32_t* inst_cuts, int32_t* n_batches, double* cost,
    int32_t* split_req, int32_t* split_ins);

/*
 * The same plan searched with the monotone split points of Eq. 6 (Sec. 5.3): the search for the last batch of
 * (first i requests, first k instances) starts at split_req[i][k-1] and split_ins[i-1][k] instead of at 0.  The
 * section states the monotonicity as a property; under the cost read here (see esp_plan_prefill_batches) it holds
 * in about three random instances in four, so this is a heuristic: the result is a valid plan (a cell with nothing
 * feasible inside the bounds is searched in full) whose cost is never below the exhaustive search's, equal to it
 * where the property holds, and up to a few times higher where it does not.  The exhaustive search stays the
 * default; the section itself calls it fast enough.  Same arguments and outputs.
 */
esp_status esp_plan_prefill_batches_monotone(
    const int64_t* req_len, int32_t n_req, const int64_t* free_slots, int32_t n_inst,
    const double* coefs, int32_t* req_cuts, int32_t* inst_cuts, int32_t* n_batches, double* cost,
    int32_t* split_req, int32_t* split_ins);

/*
 * Iteration-time model of the prefill phase (Sec. 5.5 "Optimizations", analytical model based on SIB, Eq. 7):
 *   T(R) = alpha + beta * sum_{r in R} len_r + gamma * sum_{r in R} len_r^2,
 * fitted by least squares to n >= 3 profiled batches (HOST arrays: per batch the two sums and the measured
 * time).  weights: NULL, or n non-negative factors; sample i's equation is multiplied by weights[i] before the
 * fit (1 / seconds[i] minimises the relative instead of the absolute residual).  coef receives alpha, beta,
 * gamma; a column without information (all zero) gets coefficient 0.
 */
esp_status esp_fit_prefill_model(
    const double* sum_len, const double* sum_len_sq, const double* seconds, const double* weights, int32_t n,
    double* coef);

/*
 * Debugging switches (the first two process-wide; each returns the previous setting).
 *   esp_debug_set_validate: the host-side check of device index arrays described at
 *     the top (default: ESP_DEBUG_VALIDATE in the environment, read once at load time).
 *   esp_debug_set_prefill_sync_ticks: the longest time, in ticks of the 100 MHz wall
 *     clock, that prefill workgroups sharing a key-value head wait for each other at
 *     the start of a round (default 15000, or ESP_PREFILL_SYNC_TICKS read once at load
 *     time; 0 makes every such wait give up at once; negative restores the default).
 *     It changes timing only, never results.
 *   esp_debug_set_prefill_plan: there are two prefill kernels, one for calls with few
 *     query rows, and a call's keys may be cut into parts.  By default (0) both follow
 *     from an estimate of the call's time; n > 0 makes every prefill call of the CALLING
 *     THREAD run on the main kernel in n parts, n < 0 on the other one in -n, at most
 *     ESP_MAX_PARTIALS (in one where the workspace does not hold them; anything beyond
 *     restores the default).  The workspace sizes asked for on this thread follow.
 *     For tests that are about one of the kernels.
 *   esp_debug_set_decode_plan: 1 makes every decode call of the CALLING THREAD work in
 *     ranges of the token list and combine them in a second launch, 2 in one launch, a
 *     workgroup to a request and key-value head; by default (0, and anything else) that
 *     too follows from an estimate.  Decode behind shared prefixes goes by it as well; 4 and 8 are
 *     1, and there also say of how many wavefronts its workgroups are.  For tests.
 * and, changing nothing,
 *   esp_debug_prefill_plan_for: what a call of these sizes, with or without a causal
 *     mask, that keeps rows in the pool or not, with such a workspace would run on now,
 *     in the same form (0: the sizes are not valid).  Host code.
 *   esp_debug_prefill_plan: the same of a causal call that keeps no rows.
 *   esp_debug_decode_plan: 1 or 2, what a decode call of these sizes would do now (0:
 *     the sizes are not valid).  Host code.
 *   esp_debug_decode_shared_plan: the same of a call behind shared prefixes: 2, or 4 or 8, in
 *     ranges by workgroups of so many wavefronts; without a prefix what esp_debug_decode_plan says.
 */
int32_t esp_debug_set_validate(int32_t on);
int32_t esp_debug_set_prefill_sync_ticks(int32_t ticks);
int32_t esp_debug_set_prefill_plan(int32_t plan);
int32_t esp_debug_set_decode_plan(int32_t plan);
int32_t esp_debug_decode_plan(int32_t B, int32_t total_tokens, int32_t max_len, int32_t Hq, int32_t Hkv);
int32_t esp_debug_decode_shared_plan(int32_t B, int32_t n_groups, int32_t prefix_total, int32_t max_prefix, int32_t max_group,
                                     int32_t total_tokens, int32_t max_len, int32_t Hq, int32_t Hkv);
int32_t esp_debug_prefill_plan(int32_t Tq, int32_t Tkv, int32_t batch, int32_t max_q, int32_t max_kv,
                               int32_t Hq, int32_t Hkv, size_t workspace_bytes);
int32_t esp_debug_prefill_plan_for(int32_t Tq, int32_t Tkv, int32_t batch, int32_t max_q, int32_t max_kv,
                                   int32_t Hq, int32_t Hkv, size_t workspace_bytes, int32_t causal, int32_t kept);

/* Message of the last error on the calling thread (static storage, never NULL). */
const char* esp_last_error(void);

/* Library version string, e.g. "esp 0.1 gfx950". */
const char* esp_version(void);

#ifdef __cplusplus
}
#endif
#endif /* ESP_H_ */
