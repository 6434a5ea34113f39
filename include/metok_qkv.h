/*
 * metok_qkv.h -- C ABI of the operators around the queries, keys and values of new tokens (AMD MI355X, gfx950).
 *
 * What a layer does with the products of a token before and while it attends to the caches that METok (arXiv 2506.02850) keeps small:
 *   - queries and keys are normed for each head and rotated by the token's position, which for the tokens of a video has several axes (time, height,
 *     width; after stages 1 and 2 the tokens that are left keep the positions that they had), and keys and values join the cache;
 *   - the rows that stage 3 (Sec. 3.3) keeps can be held in 4 bits, a quarter of the bytes that every new token has to read;
 *   - the attention of one new token over such a cache, the counterpart of metok_decode_attention.
 * The conventions of metok.h hold, and those that metok_decode.h adds: lengths, counts and starts are on the device and clamped to what the
 * caches hold (below 0: 0), and a workspace may be shared by calls that follow each other.
 */
#ifndef METOK_QKV_H
#define METOK_QKV_H

#include "metok_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { METOK_PAIRS_HALVES = 0, METOK_PAIRS_ADJACENT = 1 };   /* which elements of a head are rotated together, see below */
#define METOK_MAX_POSITION_AXES 4

/* ---------------------------------------------------------------------------------------------
 * Norm, rotation and storage of new tokens' queries, keys and values, in one pass.
 *
 *   q, k, v      device, of `dtype`: the rows of B * n tokens, token t = b * n + i; head h of a token's queries is q + t * q_stride + h * dh
 *                (k and v alike, Hkv heads).  The strides are in elements, multiples of 16 bytes, and at least the heads' elements; the three may
 *                be parts of one buffer, as one product leaves them.
 *   count        device, [B] int32, or NULL (= n): video b has its first count[b] tokens; of the others nothing is written, and nothing but their positions may be read.
 *   q_weight, k_weight  device, [dh] of `dtype`, or both NULL (no norm): x_e becomes x_e / sqrt(mean over the head's dh elements of x^2 + eps) *
 *                weight_e.  eps in [0, 1]; a head whose mean square and eps add up to less than 2^-126 becomes zeros.
 *   pos          device, [n_axes, B, n] int32 (1 <= n_axes <= METOK_MAX_POSITION_AXES): the tokens' positions.
 *   inv_freq     device, [rot / 2] float, finite: pair p is rotated by the angle pos[pair_axis[p]] * inv_freq[p] radians.  The product is not rounded to
 *                fp32, so that far positions keep their angles.
 *   pair_axis    host, [rot / 2] uint8 below n_axes (copied during the call), or NULL: all 0.
 *   rot          elements of a head that are rotated: a multiple of 16 and at most dh; the rest is normed, but not rotated (without a norm: copied, whatever it is).
 *   pairs        METOK_PAIRS_HALVES: pair p is the elements p and p + rot / 2; METOK_PAIRS_ADJACENT: 2 p and 2 p + 1.  (x, y) becomes
 *                (x cos - y sin, y cos + x sin).
 *   q_out        device out, [B, Hq, n, dh] of `dtype`, head by head as metok_prefill_prune (q_text) and, with n = 1, the attention calls take it.
 *   k_cache, v_cache  device in/out, [B, Hkv, S_cap, dh] of `dtype`: token i of video b becomes row start[b] + i, its keys normed and
 *                rotated, its values as they are; rows that are not below S_cap are not stored.
 *   start        device, [B] int32, or NULL (= 0).
 *   Norms and rotations are computed in fp32 and rounded once.
 *   Limits: dh in {32, 64, 128, 256} for bf16, {32, 64, 128} for f32; 1 <= B <= METOK_MAX_DECODE_BATCH; 1 <= n and B * n <= 2^26; Hq + 2 Hkv <= 4096; Hq need
 *   not be a multiple of Hkv; S_cap below 2^31 - 64; a head's sum of squares finite in fp32.  q_out and the caches must not overlap each other or anything that the call reads.
 * ------------------------------------------------------------------------------------------- */
METOK_API int metok_rotate_qk(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                           int B, int64_t n, int Hq, int Hkv, int dh, int dtype, const int32_t* count,
                           const void* q_weight, const void* k_weight, double eps,
                           const int32_t* pos, int n_axes, const float* inv_freq, const uint8_t* pair_axis, int rot, int pairs,
                           void* q_out, void* k_cache, void* v_cache, int64_t S_cap, const int32_t* start, void* stream);

/* The same into a paged cache (pools and page_table as in metok_decode_attention_paged): rows whose page is not one of the pool are not stored. */
METOK_API int metok_rotate_qk_paged(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                           int B, int64_t n, int Hq, int Hkv, int dh, int dtype, const int32_t* count,
                           const void* q_weight, const void* k_weight, double eps,
                           const int32_t* pos, int n_axes, const float* inv_freq, const uint8_t* pair_axis, int rot, int pairs,
                           void* q_out, void* k_pool, void* v_pool, int64_t n_pages_pool, int page_size,
                           const int32_t* page_table, int pages_per_seq, const int32_t* start, void* stream);

/* ---------------------------------------------------------------------------------------------
 * A KV cache in 4 bits.
 *
 * 32 neighbouring elements of a row (32 g .. 32 g + 31) share a scale s = 2^e, the smallest power of two with max |x| <= 7 s, -100 <= e <= 100; an element
 * stands for sign * c * s with c the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (the codes 0 .. 7, the sign being bit 3) to |x| / s, ties to the even code.
 * No element is further from its value than s, half of the widest step, as long as max |x| <= 7 * 2^100; larger elements become 6 * 2^100.  Elements are
 * numbers: an infinity becomes 6 * 2^100 (and its group's scale 2^100), and what a NaN becomes is one of the 16 codes.  Rows that came out of such a cache go back
 * into one as the same values.
 *
 * Rows lie in blocks of 16, of 17 * dh / 2 bytes each: K and V are [B, Hkv, S_cap / 16, 17 * dh / 2] bytes each, pools [n_pages, Hkv, page_size / 16, 17 * dh / 2]:
 * S_cap and page_size are multiples of 16, whatever lengths the videos have.  A block is laid out as the lanes of the attention load it.  With w =
 * min(dh, 128), piece p = 0 .. dh / w - 1 of a row being its elements p w .. p w + w - 1, and row 4 c + i of the block:
 *   K, code of element x of the piece       byte p * 8 w + (4 c + i) * w / 2 + x / 2
 *   V, code of element x = u * w / 16 + z   byte p * 8 w + c * 2 w + u * w / 8 + i * w / 32 + z / 2        (z < w / 16)
 *   the even element's code in the byte's low half;
 *   scale of group g < w / 32 of the piece  byte 8 * dh + p * w / 2 + c * w / 8 + g * 4 + i, holding e + 127
 * A cache that is read has to be written by these calls (or hold scale bytes between 27 and 227); rows that no call wrote may hold anything as long as they are behind the
 * videos' lengths.  dh is 32, 64, 128 or 256.
 * ------------------------------------------------------------------------------------------- */
/* Bytes of K (or of V): B * Hkv * S_cap * dh * 17 / 32; n_pages, Hkv, page_size for a pool.  0 for arguments that the calls refuse. */
METOK_API size_t metok_kv4_cache_bytes(int64_t B, int Hkv, int64_t S_cap, int dh);

/*
 * Rows of `dtype` into a 4-bit cache: row start[b] + i of video b receives source row idx[b][i], for i < min(count[b], n), every kv head of K and V.
 *   k, v         device, [B, Hkv, S_src, dh] of `dtype` (a layer's cache, or the rows of a chunk).
 *   idx          device, [B, n] int32, or NULL (= 0, 1, 2, ...; n <= S_src then): the lists of metok_kv_compact, whose compaction this does out of place; in any order,
 *                and an index may come more than once.  Entries outside [0, S_src) are skipped: nothing is stored for them.
 *   count, start device, [B] int32, or NULL (= n, 0).  Rows that are not below S_cap are not stored; all others of the cache stay as they were.
 *   k_cache, v_cache  device in/out, the 4-bit cache.  They must not overlap each other or anything that the call reads.
 *   Limits: 1 <= B <= METOK_MAX_DECODE_BATCH; Hkv <= 1024; 1 <= n; n <= 2^29; S_src and S_cap below 2^31 - 64; dh as above (f32: up to 256, too).
 */
METOK_API int metok_kv4_pack(const void* k, const void* v, int B, int Hkv, int64_t S_src, int dh, int dtype,
                           const int32_t* idx, int64_t n, const int32_t* count,
                           void* k_cache, void* v_cache, int64_t S_cap, const int32_t* start, void* stream);

/* The same into a paged 4-bit cache (page_size a multiple of 16; rows whose page is not one of the pool are not stored; the pages of rows that are stored must be
 * pairwise distinct). */
METOK_API int metok_kv4_pack_paged(const void* k, const void* v, int B, int Hkv, int64_t S_src, int dh, int dtype,
                           const int32_t* idx, int64_t n, const int32_t* count,
                           void* k_pool, void* v_pool, int64_t n_pages_pool, int page_size, const int32_t* page_table, int pages_per_seq,
                           const int32_t* start, void* stream);

/*
 * Rows of a 4-bit cache as the values they stand for (exact in both types): row i of the outputs, i < n, receives row first[b] + i, or row idx[b][i], of video b, where
 * that is below len[b] (and in a page of the pool); other rows of the outputs stay as they were.  What the attention of a prompt's next chunk reads, or a cache
 * that is to be compacted (and packed again: the codes stay what they were).
 *   len          device, [B] int32.
 *   first        device, [B] int32, or NULL (= 0);  idx  device, [B, n] int32, or NULL; not both.  Indices below 0 count as rows that are not there.
 *   k_out, v_out device out, [B, Hkv, S_out, dh] of `dtype`, n <= S_out.  They must not overlap each other or anything that the call reads.
 */
METOK_API int metok_kv4_unpack(const void* k_cache, const void* v_cache, int B, int Hkv, int64_t S_cap, int dh, const int32_t* len,
                           const int32_t* first, const int32_t* idx, int64_t n,
                           void* k_out, void* v_out, int64_t S_out, int dtype, void* stream);

METOK_API int metok_kv4_unpack_paged(const void* k_pool, const void* v_pool, int B, int Hkv, int64_t n_pages_pool, int page_size, int dh,
                           const int32_t* page_table, int pages_per_seq, const int32_t* len,
                           const int32_t* first, const int32_t* idx, int64_t n,
                           void* k_out, void* v_out, int64_t S_out, int dtype, void* stream);

/*
 * Attention of one new token per video over a 4-bit cache: the arguments, results and limits of metok_decode_attention, with these differences.
 *   k_cache, v_cache  the 4-bit cache, S_cap a multiple of 16.
 *   k_new, v_new  rows of `dtype`, which the call puts into 4 bits: what is stored at row len[b] is also what is attended to.
 *   Results are those of the values that the cache stands for (products of `dtype` queries with them, accumulated in fp32; in fp32 with all bits of the queries
 *   and probabilities).  Finite in fp32 have to be: 2^103 * dh * max |q_e| (a value reaches 6 * 2^100) and 1.45 s_j; and 2^8 times the sum of the magnitudes of an
 *   element of V over a video's rows, since a probability may be relative to a maximum that is 2^8 times smaller than the last one (up to 170000 rows of 6 * 2^100).
 *   Limit: B * Hkv * ceil(Hq / Hkv / 16) * (S_cap / 16 + 4) below 2^31.
 *   workspace    metok_kv4_attention_workspace_bytes().
 */
METOK_API size_t metok_kv4_attention_workspace_bytes(int B, int Hq, int Hkv, int64_t S_cap, int dh, int dtype, int with_weight);

METOK_API int metok_kv4_attention(const void* q, int B, int Hq, int Hkv, int dh, int dtype,
                           void* k_cache, void* v_cache, int64_t S_cap, const int32_t* len,
                           const void* k_new, const void* v_new, double scale, double logit_cap,
                           void* out, float* lse, float* weight, int64_t weight_stride,
                           void* workspace, size_t workspace_bytes, void* stream);

/* The same over a paged 4-bit cache: page_size a multiple of 16. */
METOK_API int metok_kv4_attention_paged(const void* q, int B, int Hq, int Hkv, int dh, int dtype,
                           void* k_pool, void* v_pool, int64_t n_pages_pool, int page_size,
                           const int32_t* page_table, int pages_per_seq, const int32_t* len,
                           const void* k_new, const void* v_new, double scale, double logit_cap,
                           void* out, float* lse, float* weight, int64_t weight_stride,
                           void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* METOK_QKV_H */
