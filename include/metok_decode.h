/*
 * metok_decode.h -- C ABI of the decoding-time operators beside stage 3 (AMD MI355X, gfx950).
 *
 * Stage 3 of METok (arXiv 2506.02850, Sec. 3.3) leaves a compacted KV cache (Eq. 3); while the answer is written, every new token
 * attends to it and adds a row.  Two operators belong to that loop:
 *   - the attention of one new token per video over a dense or paged cache, which appends the token's own row and, if asked,
 *     adds up how much attention every cached row draws (the decoding-time counterpart of the stage-2 score, Sec. 3.2.2);
 *   - eviction: once a cache has grown beyond a budget, the rows that drew the least attention leave it.
 * The conventions of metok.h hold (caller-owned buffers, no synchronisation, deterministic results, capture into HIP graphs after
 * one ordinary call, error codes, 16-byte alignment, finite inputs).  Two additions:
 *   - Lengths live on the device, so that a captured decoding step can be replayed while the caches grow.  A length below 0 counts
 *     as 0 and one above the capacity as the capacity.
 *   - A workspace may be shared by calls that follow each other (on one stream, or in graphs that are replayed one after the
 *     other); calls that may overlap in time need workspaces of their own.
 */
#ifndef METOK_DECODE_H
#define METOK_DECODE_H

#include "metok.h"

#ifdef __cplusplus
extern "C" {
#endif

#define METOK_MAX_DECODE_BATCH 4096   /* B limit of the calls below */

/* ---------------------------------------------------------------------------------------------
 * Attention of one new token per video over the KV cache.
 *
 *   q            device, [B, Hq, dh] of `dtype`: the new token's queries.  Query head h reads kv head h / (Hq / Hkv).
 *   k_cache, v_cache  device, one layer's cache [B, Hkv, S_cap, dh] of `dtype` (the layout of metok_kv_compact).
 *   len          device, [B] int32: rows every video's cache holds before this call.  Not modified: a caller that appends
 *                adds 1 to all lengths once all layers of the step are done.
 *   k_new, v_new device, [B, Hkv, dh] of `dtype`, or both NULL: the new token's own row.  It is written at row len[b] of the
 *                cache and attended to.  A video whose cache is full (or whose page for that row is not a page of the pool)
 *                attends to it all the same, but it is not stored.
 *   scale        in [1e-30, 1e30): s_j = scale * (q . k_j); usually 1 / sqrt(dh).  q . k_j and 1.45 s_j have to be finite in fp32.
 *   logit_cap    0: none.  c and scale / c in [1e-30, 1e30): s_j becomes c * tanh(s_j / c).
 *   out          device out, [B, Hq, dh] of `dtype`: sum_j p_j v_j with p = softmax(s) over the video's rows, accumulated in
 *                fp32 and rounded once (with bf16 caches p enters the products as the sum of two bf16 numbers).  A video without rows
 *                gets zeros.
 *   lse          device out, [B, Hq] float, or NULL: log sum_j exp(s_j) (-inf without rows), what two such results are joined by.
 *   weight       device in/out, [B, weight_stride] float, or NULL: weight[b][j] grows by the mean of p_j over the Hq heads for
 *                every row j that was there before; that of the new row is set, not added to, where the capacity has a place for it (stored
 *                or not).  Entries behind the last row are left as they were.  weight_stride >= the capacity.
 *   Limits: dh in {32, 64, 128, 256} for bf16, {32, 64, 128} for f32; Hq a multiple of Hkv; 1 <= B <= METOK_MAX_DECODE_BATCH;
 *   Hq <= 1024; capacity below 2^31 - 64; B * Hkv * ceil(Hq / Hkv / 16) * (capacity / 16 + 4) below 2^31.
 *   out, lse, weight, the workspace and the caches must not overlap each other or anything else the call reads or writes; but K and V may
 *   be the same cache where no row is appended.
 *   The work is split by the capacity, not by the lengths, which are on the device: with short requests in paged caches a page_table no wider
 *   than they need is faster (capacities up to 1023 rows in bf16, 511 for heads of 256 and in fp32, take one launch without weights
 *   and with at most 16 query heads to a kv head).
 *   A video that is not there (padding of a batch) has a length of 0 and, where a row is appended, no pages in its table.
 *   workspace    metok_decode_attention_workspace_bytes(), S_cap being the capacity (pages_per_seq * page_size of a paged cache) and
 *                with_weight whether `weight` is given.  Its contents on entry do not matter.
 * ------------------------------------------------------------------------------------------- */
METOK_API size_t metok_decode_attention_workspace_bytes(int B, int Hq, int Hkv, int64_t S_cap, int dh, int dtype, int with_weight);

METOK_API int metok_decode_attention(const void* q, int B, int Hq, int Hkv, int dh, int dtype,
                           void* k_cache, void* v_cache, int64_t S_cap, const int32_t* len,
                           const void* k_new, const void* v_new, double scale, double logit_cap,
                           void* out, float* lse, float* weight, int64_t weight_stride,
                           void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same over a paged cache: k_pool, v_pool [n_pages_pool, Hkv, page_size, dh]; row j of video b is slot j % page_size of page
 * page_table[b][j / page_size] (page_table device, [B, pages_per_seq] int32, as in metok_kv_compact_paged; after
 * metok_kv_relink_paged the layer's own [B, pages_per_seq] part of page_table_out).  Entries outside [0, n_pages_pool) are never
 * dereferenced: the rows behind them take no part.  Pages may be shared between videos as long as none of the appended rows
 * lies in a shared page.  n_pages_pool * Hkv * page_size must be below 2^31.
 */
METOK_API int metok_decode_attention_paged(const void* q, int B, int Hq, int Hkv, int dh, int dtype,
                           void* k_pool, void* v_pool, int64_t n_pages_pool, int page_size,
                           const int32_t* page_table, int pages_per_seq, const int32_t* len,
                           const void* k_new, const void* v_new, double scale, double logit_cap,
                           void* out, float* lse, float* weight, int64_t weight_stride,
                           void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Eviction by accumulated attention weight: every (layer, video) whose cache holds more rows than the layer's budget keeps its
 * first n_first rows, its last n_last rows and, of those between, the rows with the largest weight (the lower index first among
 * equals) until the budget is full.  Rows keep their order (as in stage 3), so a row's rank tells its age.
 *
 *   k_layers, v_layers, L, B, Hkv, S_cap, dh, dtype  the caches, as in metok_kv_compact.
 *   weight       host array of L device pointers, weight[l] [B, weight_stride] float (see `weight` above; weight_stride >= the
 *                capacity); weight[l] == NULL leaves layer l alone.  Weights are compared as numbers; NaNs come at the ends by sign.
 *   weight_out   host array of L device pointers like `weight`: weight_out[l][b][i] = weight of the row that is now row i, for
 *                i < new_len[l][b]; the rest is left as it was.  May be the same buffers as `weight` (or the same array), but not
 *                overlap them otherwise.
 *   len          device, [L, B] int32: rows held now.
 *   budget       host, [L] int32, 1 <= budget[l] <= capacity (ignored where weight[l] is NULL); n_first, n_last >= 0 and
 *                n_first + n_last <= budget[l].
 *   idx          host array of L device pointers, idx[l] [B, budget[l]] int32 out (ignored where weight[l] is NULL): the kept rows, ascending -- the
 *                index lists of metok_kv_compact, _paged and metok_kv_relink_paged with n_keep[l] = budget[l].  A video within the budget has
 *                the list 0, 1, 2, ...: nothing of it moves.
 *   new_len      device out, [L, B] int32: min(len, budget[l]) (len where weight[l] is NULL); may be `len` itself.
 *   Apart from the two cases named (weight_out[l] as weight[l], new_len as len) no output may overlap anything else that the call
 *   reads or writes; of idx, weight, weight_out, len and new_len that is checked.
 * metok_kv_evict and metok_kv_evict_paged select and move the rows of the caches (row i <- row idx[l][b][i]; rows from
 * new_len on are left as they were); metok_kv_evict_select only selects, for callers that relink pages or move the rows themselves.
 *   Paged: one table for all layers (caches relinked by metok_kv_relink_paged, with a table per layer: one call with L = 1 for each, or
 *   metok_kv_evict_select and metok_kv_relink_paged).  Rows are moved in place, so pages that videos share may only hold rows that no
 *   video moves: among their first n_first ones.
 *   workspace    metok_kv_evict_workspace_bytes() for the first two, none for the selection; as in metok_kv_compact its first word
 *                is 0 after the call unless a bounded wait expired.  Rows were left where they were then, while idx, weight_out and
 *                new_len are written: the caches are to be given up.
 * ------------------------------------------------------------------------------------------- */
METOK_API size_t metok_kv_evict_workspace_bytes(int L, int B, int Hkv, int64_t S_cap, int dh, int dtype);

METOK_API int metok_kv_evict(void* const* k_layers, void* const* v_layers, int L, int B, int Hkv, int64_t S_cap, int dh, int dtype,
                           const float* const* weight, float* const* weight_out, int64_t weight_stride,
                           const int32_t* len, const int32_t* budget, int n_first, int n_last,
                           int32_t* const* idx, int32_t* new_len,
                           void* workspace, size_t workspace_bytes, void* stream);

METOK_API int metok_kv_evict_paged(void* const* k_pools, void* const* v_pools, int L, int B, int Hkv,
                           int64_t n_pages_pool, int page_size, int dh, int dtype,
                           const int32_t* page_table, int pages_per_seq,
                           const float* const* weight, float* const* weight_out, int64_t weight_stride,
                           const int32_t* len, const int32_t* budget, int n_first, int n_last,
                           int32_t* const* idx, int32_t* new_len,
                           void* workspace, size_t workspace_bytes, void* stream);

METOK_API int metok_kv_evict_select(const float* const* weight, float* const* weight_out, int64_t weight_stride,
                           int L, int B, int64_t S_cap, const int32_t* len, const int32_t* budget, int n_first, int n_last,
                           int32_t* const* idx, int32_t* new_len, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* METOK_DECODE_H */
