/*
 * sol_cache.h -- C ABI of the serving operators of the MI355X (gfx950) attention
 * library: norm and rotation of queries and keys, page tables, a key/value cache
 * held in 4 bits, and attention over it.  One step of autoregressive generation
 * (token- or frame-causal) is, for a ragged batch of requests,
 *
 *   sol_cache_tables    lengths -> pages, slots and positions of the new tokens
 *   sol_qk_norm_rope    queries and keys of the new tokens
 *   sol_cache_append    keys and values of the new tokens into their slots
 *   sol_cache_forward   attention of the new tokens over the whole cache
 *
 * sol_qk_norm_rope also prepares queries and keys for the forward calls of
 * sol_attn.h.  Return codes, element types and sol_attn_last_error() are those of
 * sol_attn.h.  Every entry point checks its arguments on the host and returns
 * before any GPU call when they are invalid.  All pointers are device memory of
 * the current device.  Calls are asynchronous on `stream` (a hipStream_t of the
 * current device, or NULL), allocate nothing, keep nothing between calls and may
 * be captured into a graph.  What device memory says (lengths, slots, table
 * entries, positions) is never trusted with an address: each call states what it
 * does with values out of range.
 *
 * Sizes (B, N, T, S, heads, ...) are positive; a launch takes at most 65,535 heads, 2^27
 * tokens in sol_qk_norm_rope, 2^28 tokens times heads in append and read, and in forward
 * 2^24 tokens times query heads and 2^18 requests times key/value heads.
 *
 * Strides are in elements; the d channels of a head are contiguous.  Rows that
 * are written must not overlap.  Tensors whose start and strides are multiples of
 * 16 bytes are read and written faster.
 *
 * The cache.  A page is SOL_CACHE_PAGE = 64 tokens of one key/value head; slot
 * s of a store of P pages is token s % 64 of page s / 64.  A store is
 * [P][heads][68 d] bytes and starts on 16 bytes; d is 64 or 128.  Keys and values
 * are held in 4 bits: e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6, bit 3 the sign) and
 * a scale 2^(byte - 127) for 32 channels of a token.  The 68 d bytes of a page and head:
 *   keys    [64 tokens][d/2]      byte b: channel 2b in the low half, 2b + 1 in the high one
 *   scales  [2][32][d/64][2]      group 2c + a of token 32w + t at [a][t'][c][w], where t' is t
 *                                 with its bits 2 and 3 exchanged
 *   values  [8][32][8][d/64]      bytes of (o, i, j): channels d/32 i ... of token 8o + j
 *   scales  [8][d/32][8]          group g of token 8o + j at [o][g][j]
 * Nothing else is in a store: a page may be copied or moved as bytes.
 */
#ifndef SOL_CACHE_H
#define SOL_CACHE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { SOL_CACHE_PAGE = 64 };

/* Layout of the rotated pairs: channels (i, i + rot/2), or (2i, 2i + 1). */
enum { SOL_ROPE_HALVES = 0, SOL_ROPE_PAIRS = 1 };

/*
 * RMS norm of each head of queries and keys, and the rotation by position, in one pass:
 *   y_c = x_c / sqrt(mean_c x_c^2 + eps) * w_c,
 *   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin)   for the rot/2 pairs (a, b).
 *
 * q: [B, Hq, N, d] with strides (q_strides[0..2]) of batch, head and token; k likewise
 *   with Hk heads.  k may be NULL (Hk is then 0), and so may q.
 * q_out, k_out: likewise; they must not overlap the inputs.
 * q_weight, k_weight: [d] of the element type `weight_dtype`, or NULL for ones.
 * cos, sin: [P, rot/2] f32 tables, one row for a position; NULL when rot is 0.
 * positions: [B, N] i32 rows of the tables, or NULL: token n takes row n.  A token whose
 *   position is not in [0, P) is left out: its output rows stay as they were.  With
 *   rot = 0 a token is left out where its position is below 0.
 * rot: channels that are rotated, a multiple of 8 from 0 to d; the others are only normed.
 * eps: > 0 and finite.  The arithmetic is f32, rounded once; values whose squares sum
 *   past the f32 range come out as 0.
 */
int sol_qk_norm_rope(const void* q, const void* k, void* q_out, void* k_out,
                     const long long* q_strides, const long long* k_strides,
                     const long long* q_out_strides, const long long* k_out_strides,
                     const void* q_weight, const void* k_weight, const float* cos, const float* sin,
                     const int32_t* positions, int B, int Hq, int Hk, int N, int d, int P, int rot,
                     int pairs, float eps, int dtype, int weight_dtype, void* stream);

/*
 * Pages, slots and positions of one step of S requests, from their lengths.
 *
 * lens: [S] tokens held by each request; add: [S] tokens to add (> 0) or, below 0, to take
 *   back from the end (all of them, where it says more than there are: the request ends).
 * table: [S, max_pages] i32, updated: entry p of request s is the page of its tokens 64p ... .
 *   New pages are written behind those in use; every other entry stays as it was, those of
 *   pages that a request gives back too.
 * ring: [P] i32, updated: the free pages, state[1] of them from ring[state[0]] on, around the
 *   end.  New pages come from its front, in the order of the requests; pages given back go
 *   to its end (a table entry that is not in [0, P) is not given back), so a page is
 *   used again as late as can be.  A page that several requests share is given back once for each: the caller
 *   takes it out of their tables (entry -1) before.
 * A request that would pass max_pages pages is refused; so is one for whose new pages the
 *   free ones do not suffice after those that the requests before it asked for.  A refused
 *   request keeps its length.
 * lens_out [S], state_out [2]: the values after the step; not the arrays lens and state, so a
 *   step that is repeated gives the same pages again.
 * row_start: [S + 1]: the new tokens of request s are rows row_start[s] ... row_start[s + 1] - 1,
 *   max(add, 0) of them, refused or not.
 * slots, positions: [rows] i32: slot and position of every row; -1 in the rows of a refused
 *   request and in those behind the last request.
 * Lengths are taken as clamped to [0, 64 max_pages], state to a ring of P.  S <= 4096.
 */
int sol_cache_tables(const int32_t* lens, const int32_t* add, int32_t* table, int32_t* ring,
                     const int32_t* state, int32_t* lens_out, int32_t* state_out, int32_t* row_start,
                     int32_t* slots, int32_t* positions, int S, int max_pages, int P, int rows,
                     void* stream);

/*
 * Writes keys and values into their slots, in 4 bits.
 *
 * k, v: [heads, T, d] with strides of head and token.  slots: [T] i32; a token whose slot is
 *   not in [0, 64 P) is left out.  Slots of one call must differ from each other.
 * The scale of 32 channels whose largest magnitude is m is 2^e, e = floor(log2 m) - 2, and one
 *   more where m > 7 * 2^e (the choice with the least squared error for normal values);
 *   e is kept in [-100, 125] for keys and in [-23, 13] for values, so that values are exact in
 *   f16 (magnitudes up to 49152, as the range contract of the bf16 forward asks; larger
 *   ones are held as 49152).  Codes are rounded to nearest, ties to the even code, 6 the largest.
 *   Normal keys and values are off by 11 % (root mean square), attention's outputs over them by 16 % where logits have a standard
 *   deviation of 1, by 25 % where it is 2.
 * A token with an infinity or NaN in the key or the value of a head is held there as NaN: every
 *   row that sees it is NaN, and no other row is.
 */
int sol_cache_append(const void* k, const void* v, const long long* k_strides, const long long* v_strides,
                     void* store, const int32_t* slots, int T, int heads, int d, int P, int dtype,
                     void* stream);

/*
 * Reads keys and values of slots back, as the values that the codes stand for (exact in bf16 and f32).
 * k_out, v_out: [heads, T, d] with strides of head and token, either may be NULL.  Slots that are not
 * in [0, 64 P) give zeros; tokens held as NaN give NaN.
 */
int sol_cache_read(const void* store, const int32_t* slots, void* k_out, void* v_out,
                   const long long* k_strides, const long long* v_strides, int T, int heads, int d, int P,
                   int dtype, void* stream);

/*
 * Attention of the new tokens of S requests over the cache:
 *   out = sum_j softmax_j(q . k_j / sqrt(d)) v_j
 * over the tokens j of the row's request with j < min((p / G + 1) G, len), p the row's
 * position: G = causal_granule = 1 is token-causal attention, G = the tokens of a frame
 * frame-causal, G >= len no mask.  Query heads h read key/value head h / (Hq / Hk).
 *
 * q: [Hq, T, d] with strides of head and token; out likewise, not overlapping q.
 * store [P, Hk, 68 d], table [S, max_pages], lens [S], row_start [S + 1], positions [T]: as above;
 *   lens counts the new tokens too (they are appended before).  Rows of positions below 0, and rows
 *   that see no token, give zeros.  Rows outside row_start[0] ... row_start[S] - 1 stay as they were.
 *   Pages of the table that are not in [0, P) take no part, as if their tokens were not there.
 *   Lengths are taken as clamped to [0, 64 max_pages], row_start to [0, T].
 * max_rows: at least the rows of the request that has most; rows past it may be left out.
 * workspace: device scratch of at least sol_cache_workspace_bytes(...) bytes that starts on 16 bytes; calls that
 *   may run at the same time need different ones, and a captured graph keeps using the one
 *   it was captured with.  It may be NULL where 0 bytes are needed.
 * Logits, maxima and sums are f32.  q log2(e) / sqrt(d) is split into 6-bit floats for each channel: three (bf16), whose
 *   sum is off by at most 2^-13.9 of the largest magnitude of its 32 channels, or six (f32, 2^-25.9).  Probabilities are
 *   f32 for f32 rows.  For bf16 rows they are rounded to f16, none to finer steps than 2^-31 of the row's largest, and their
 *   sum is taken before: a row of which one token has nearly all the weight shows what tokens of less than 2^-31 of that give
 *   to at most 2^-32 sum |v|.
 * Results do not depend on the order in which the GPU runs the work.
 */
int sol_cache_forward(const void* q, const long long* q_strides, void* out, const long long* out_strides,
                      const void* store, const int32_t* table, const int32_t* lens,
                      const int32_t* row_start, const int32_t* positions, int S, int T, int max_rows,
                      int Hq, int Hk, int d, int P, int max_pages, int causal_granule, int dtype,
                      void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of a store, and scratch bytes of sol_cache_forward; SIZE_MAX if the arguments are invalid. */
size_t sol_cache_bytes(int P, int heads, int d);
size_t sol_cache_workspace_bytes(int S, int T, int max_rows, int Hq, int Hk, int d, int max_pages);

#ifdef __cplusplus
}
#endif

#endif /* SOL_CACHE_H */
