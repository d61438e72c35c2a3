/*
 * Operators on caller buffers for a verification pass over a batch of sequences that begin alike (one system prompt, one
 * document): rotary tables, rotation with the writes of a paged cache, attention over the shared prefix and every
 * sequence's own positions, and the verification of the drafted tokens against given random numbers.  They stand beside
 * spec_ops.h for programs that run layers of their own; the engine of spec.h keeps caches, attention and accept phase of
 * its own and uses none of them.
 *
 * Same conventions as spec_ops.h: 0 or a negative SPEC_E* code, the text of a failure from spec_last_error(NULL); "device"
 * pointers belong to the current device; work is enqueued on `stream` (a hipStream_t, NULL: the null stream), nothing
 * synchronises or allocates, and every call may be captured into a graph (kernel launches only).  The library keeps no
 * state between calls: calls on different streams may overlap as long as their outputs and workspaces differ.  Inputs,
 * outputs and workspaces must not overlap unless stated otherwise.  Workspaces need no preparation, are overwritten, and
 * calls that may overlap (captured graphs replayed on two streams included) need workspaces of their own.
 *
 * Pages.  A cache is a pool of n_pages pages, keys and values apart, each device [n_pages][n_kv][page_tokens][hd],
 * 16-byte aligned; page_tokens is a power of two from 8 to 2^20.  A slot is page * page_tokens + place in the page, below 2^31.
 */
#ifndef SPEC_BATCH_H
#define SPEC_BATCH_H

#include <stdint.h>

#include "spec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Frequencies of a rotation of `rot` elements, f_j radians a position for pair j < rot / 2, in 64 bits.  With
 * t_j = theta^(-2j / rot):
 *   SPEC_ROPE_PLAIN   f_j = t_j
 *   SPEC_ROPE_LINEAR  f_j = t_j / factor (position interpolation)
 *   SPEC_ROPE_BASE    f_j = (theta * factor^(rot / max(rot - 2, 1)))^(-2j / rot) (another base: the slowest pair is
 *                     interpolated, the fastest stays)
 *   SPEC_ROPE_BANDS   f_j = t_j * (s + (1 - s) / factor), s = clamp((n_j - low) / (high - low), 0, 1), n_j = context * t_j / 2 pi
 *                     the turns of pair j over the original context: fast pairs stay, slow ones are interpolated
 *   SPEC_ROPE_RAMP    f_j = t_j * (1 - g + g / factor), g = clamp((j - a) / max(b - a, 0.001), 0, 1), where a = max(floor(d(high)), 0),
 *                     b = min(ceil(d(low)), rot - 1), d(n) = rot ln(context / (2 pi n)) / (2 ln theta) the pair that turns n
 *                     times over the original context (the ramp by parts of "YaRN", Peng et al. 2023); both tables
 *                     are multiplied by `magnitude`, 0 standing for 0.1 ln(factor) + 1
 * theta > 0 (RAMP: > 1), factor > 0, BANDS and RAMP: 0 <= low < high (RAMP: 0 < low), context > 0; magnitude is read by RAMP
 * alone, finite and >= 0.  Members a scaling does not name are ignored. */
enum { SPEC_ROPE_PLAIN = 0, SPEC_ROPE_LINEAR = 1, SPEC_ROPE_BASE = 2, SPEC_ROPE_BANDS = 3, SPEC_ROPE_RAMP = 4 };

typedef struct {
    double  theta;      /* base */
    int32_t scaling;    /* SPEC_ROPE_* */
    double  factor;     /* how many times longer the context has become */
    double  low, high;  /* turns over the original context below / above which a pair is interpolated / kept */
    double  context;    /* original context, in positions */
    double  magnitude;
} spec_rope;

/* rope_cos[p][j] = cos(p * f_j), rope_sin[p][j] = sin(p * f_j) for p < n_pos, j < rot / 2 (times the magnitude with
 * SPEC_ROPE_RAMP); f_j as arithmetic in 64 bits gives it, angles in 64 bits, results rounded once: off by half a step of fp32 and by
 * 7e-15 + 1e-15 * p * f_j (times the magnitude).  Tables: device fp32 [n_pos][rot / 2], as spec_k_rope_cache and spec_k_qk_norm_rope read them.  rope: host, read by the call.  rot even, 2 to
 * 512; 1 <= n_pos <= 2^28. */
int spec_k_rope_tables(const spec_rope *rope, int32_t rot, int32_t n_pos, float *rope_cos, float *rope_sin, void *stream);

/* Rotate the heads of R rows by their positions, queries to rows, keys and values to pages of a cache.  Of every query
 * and key head the first `rot` elements turn, the others stay; with c = rope_cos[pos[r]][j], s = rope_sin[pos[r]][j], in fp32,
 *     interleaved == 0:  (h[j], h[j + rot/2]) <- (h[j] c - h[j + rot/2] s, h[j + rot/2] c + h[j] s)
 *     interleaved != 0:  (h[2j], h[2j + 1])   <- (h[2j] c - h[2j + 1] s, h[2j + 1] c + h[2j] s)
 * q, k, v: device, dtype SPEC_F32 or SPEC_BF16, head i of row r at element r * ld + i * hd (the parts of a fused QKV row, or
 * arrays of their own), ld* >= heads * hd.  q_out: device, out_dtype, stride ldqo; may be q itself (same pointer, type and
 * stride).  k_pages, v_pages: pages of out_dtype, see above; row r goes to slot[r].  pos, slot: device int32 [R].  A row whose
 * position lies outside 0 .. n_pos - 1 is padding: nothing of it is written.  A row whose slot lies outside the pool writes its
 * queries alone.  Rows with the same slot leave there elements of either.  2 <= hd <= 512, rot even, 2 <= rot <= hd; nq, nkv >= 0,
 * not both 0 (nq == 0: q and q_out are ignored; nkv == 0: k, v, slot and the pages are); R * (nq + 2 nkv) < 2^31. */
int spec_k_rope_cache(const void *q, int64_t ldq, int32_t nq, const void *k, int64_t ldk, const void *v, int64_t ldv, int32_t nkv,
                      int32_t dtype, int32_t hd, int32_t R, const float *rope_cos, const float *rope_sin, int32_t n_pos, int32_t rot,
                      int32_t interleaved, const int32_t *pos, const int32_t *slot, void *q_out, int64_t ldqo, void *k_pages,
                      void *v_pages, int32_t n_pages, int32_t page_tokens, int32_t out_dtype, void *stream);

/* Attention of R query rows, packed one sequence after the other, over a prefix that all sequences share and over their
 * own positions.  Sequence b has rows row_start[b] .. row_start[b + 1] - 1, n of them, and own_len[b] own positions, of which the
 * rows are the last n: its row i sees the prefix and own positions 0 .. own_len[b] - n + i.
 *     o = sum_j softmax_j(scale * q . k_j) v_j  over the positions seen;  a row that sees none gets zeros.
 * q, out: device, dtype, head i of row r at element r * ld + i * hd; query head i reads cache head i / (nq / nkv).  Queries, pages and
 * results have one type: SPEC_F32 (fp32 throughout) or SPEC_BF16 (scores, weights' sums and results are held in fp32; in front of the
 * values' product a weight is rounded to two bf16 terms, off by 2^-16 of itself, or to one, off by 2^-8, in heads of up to 128 elements
 * where more than 32 columns go through the same positions: rows times nq / nkv, of a sequence on average, or of all of them
 * for a prefix that no sequence goes through by itself.  Results are then off by 0.0023 of their norm instead of 0.0017).
 * row_start: device int32 [n_seq + 1]; own_len: device int32 [n_seq]; table: device int32 [n_seq][table_pages], the page of own
 * positions p * page_tokens ..; prefix_table: device int32 [ceil(prefix_len / page_tokens)], the pages of the prefix (NULL where
 * prefix_len is 0).  The own positions begin with a page of their own, wherever the prefix ends.  Rows in front of row_start[0]
 * and from row_start[n_seq] on are left as they were.  Bounds in device memory are never trusted: rows are those within 0 .. R,
 * own_len counts at most table_pages * page_tokens, and positions on pages outside the pool are not seen.  What lies in the pages
 * behind a sequence's end, or at positions that a row does not see, does not reach that row, NaN and infinities included.  A row
 * that sees a value that is one has NaN or an infinity in its channel.  A key's count by their scores: a row with a score that is NaN or
 * plus infinity has NaN in its whole head, and a position whose score is minus infinity has weight 0 (a row whose scores are
 * all of that kind gets zeros, as if it saw none).
 * 8 <= hd <= 256, hd % 8 == 0; nq a multiple of nkv, at most 65536; 1 <= n_seq <= 4096; scale > 0; prefix_len and table_pages * page_tokens below
 * 2^30 (table_pages may be 0: prefix alone); R * nq <= 2^30.  q . k has to stay within fp32's range,
 * and so have values times 2^9 and the number of positions seen.  workspace: device scratch, 16-byte aligned, of at least
 * spec_k_attn_shared_workspace() bytes for these sizes (0: NULL will do).  The same call gives the same bits every time. */
int spec_k_attn_shared(const void *q, int64_t ldq, int32_t nq, int32_t nkv, int32_t hd, int32_t dtype, int32_t R,
                       const int32_t *row_start, int32_t n_seq, const void *k_pages, const void *v_pages, int32_t n_pages,
                       int32_t page_tokens, const int32_t *prefix_table, int32_t prefix_len, const int32_t *table,
                       int32_t table_pages, const int32_t *own_len, float scale, void *out, int64_t ldo, void *workspace,
                       int64_t workspace_bytes, void *stream);

/* Bytes of workspace spec_k_attn_shared must be given (a function of these sizes alone; own_capacity = table_pages *
 * page_tokens); SPEC_EINVAL for sizes it refuses. */
int64_t spec_k_attn_shared_workspace(int32_t R, int32_t n_seq, int32_t nq, int32_t nkv, int32_t hd, int32_t dtype, int32_t prefix_len,
                                     int32_t own_capacity);

/* Verification of drafted tokens, a batch at once, from probabilities (after whatever temperature, filters and penalties
 * the program applies) and uniform random numbers that the caller gives.  Sequence b has k = draft_start[b + 1] - draft_start[b] >= 0
 * drafts, with i = draft_start[b] + n the n-th: drafted[i], u_accept[i], q row i, and k + 1 rows of p from draft_start[b] + b on.
 * The rule is that of spec_accept():
 *     n_accepted[b] = A: the leading drafts with u_accept * q(x) < p(x) (in 64 bits, exact);
 *     next_token[b]: from norm(max(0, p - q)) of row A where A < k, else from p's last row: the lowest j whose
 *                    w_0 + .. + w_j exceeds u_next[b] * (w_0 + .. + w_{vocab-1}), sums in 64 bits.
 * Where max(0, p - q) is zero throughout, the draw is from p.  Where no j exceeds (u_next of 1, or a sum that rounding made
 * equal) it is the last j with a weight above zero, 0 if there is none.  q NULL: drafts without probabilities (looked up, not drawn): q(x) is 1 for
 * the drafted token and 0 for every other.  Weights need not sum to 1; negative ones and NaN count as 0, a comparison with NaN
 * rejects.  A draft outside the vocabulary is rejected (with q NULL the draw is then from p).
 * p: device [n_drafts + n_seq][vocab], q: device [n_drafts][vocab], dtype SPEC_F32 or SPEC_BF16, row strides ldp, ldq >= vocab,
 * aligned to their type; draft_start: device int32 [n_seq + 1]; drafted: device int32, u_accept: device fp32 [n_drafts] (may be NULL
 * where n_drafts is 0); u_next: device fp32, n_accepted, next_token: device int32 [n_seq].  A sequence whose draft_start does not lie
 * within 0 .. n_drafts, rising, gets -1 for both.  1 <= vocab <= 2^24, 0 <= n_seq <= 65535.  workspace: device scratch, 16-byte aligned, of at
 * least spec_k_verify_workspace() bytes. */
int spec_k_verify(const void *p, int64_t ldp, const void *q, int64_t ldq, int32_t dtype, int32_t vocab, const int32_t *draft_start,
                  int32_t n_seq, int32_t n_drafts, const int32_t *drafted, const float *u_accept, const float *u_next,
                  int32_t *n_accepted, int32_t *next_token, void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of workspace spec_k_verify must be given; SPEC_EINVAL for sizes it refuses. */
int64_t spec_k_verify_workspace(int32_t n_seq, int32_t vocab);

#ifdef __cplusplus
}
#endif
#endif
