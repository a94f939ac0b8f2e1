/*
 * kv_cache.h -- C ABI of the MI355X (gfx950) paged cache of keys and values in 8 bits: writing it, attention over it,
 * reading it back.
 *
 * The cache is made of pages.  A page holds `page` consecutive tokens of one sequence, for each kv head their keys and
 * values as e4m3 codes (OCP) with one exponent for the keys and one for the values: a code c stands for c * 2^e.
 *     k      e4m3  [pages, Hkv, page, D]
 *     v      e4m3  [pages, Hkv, D, page]     (transposed: the product with the probabilities sums over tokens)
 *     k_exp  uint8 [pages, Hkv]   e + 127    v_exp  uint8 [pages, Hkv]   e + 127
 * Scales are powers of two: a decoded value is exact in bf16 (e4m3 has four significant bits), and a page whose scale has to
 * grow keeps its codes' values except where they become subnormal.  The bytes of k_exp and v_exp are 27 ... 247 (e from
 * -100 to 120) wherever kv_fp8_write has written; values of a page below 2^-110 become zero.
 *
 * A page table, int32 [B, width], says where the sequences lie: position j of sequence b is token j % page of page
 * table[b * table_pitch + j / page].  An entry outside 0 ... pages - 1 is a missing page: writes to its positions are dropped,
 * attention does not see them, reading gives zeros.  Sequences may share pages (a common beginning) that no call writes.
 *
 * What the page size costs: larger pages need fewer exponents and table entries, smaller ones make a single token's write cheaper,
 * since every column's code of V lies in another line and a scale that grows has the page rounded again.  One token of 64 sequences
 * and 8 heads of 128, pages of 16 / 32 / 64 / 128: 7.0 / 8.4 / 8.7 / 9.4 us, and 7.4 / 9.8 / 12.0 / 15.8 where every scale
 * grows (between two events).
 *
 * All pointers except the strides and the KvFp8Cache itself are DEVICE pointers into caller-owned memory.  The library
 * neither allocates nor frees nor synchronises: every call enqueues its kernels on `stream` (a hipStream_t as void*, NULL =
 * the default stream) and returns.  Thread-safe, no global state.  Every argument check precedes the first HIP call; what
 * the tables and lengths on the device hold is checked by the kernels, as described at each call.  Return codes are those
 * of attn.h.
 *
 * Supported caches: D in {64, 128}; page in {16, 32, 64, 128}; pages, Hkv >= 1, pages * Hkv < 2^31; width >= 1 and
 * width * page < 2^30; k and v 16-byte aligned; fewer than 2^23 workgroups in a call (attention: B * Hkv * blocks of 16 or 128 rows *
 * splits; writing: B * Hkv * pages that S tokens can lie in; reading: B * Hkv * S / 64).  Each *_strides points to 3 HOST integers {batch, head, row} in ELEMENTS, as
 * in attn_fwd_strided: multiples of 8, none negative, row stride >= D and < 2^28.
 */
#ifndef KV_CACHE_MI355X_H
#define KV_CACHE_MI355X_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct KvFp8Cache {
    void *k, *v;
    unsigned char *k_exp, *v_exp;
    int pages, Hkv, page, D;
} KvFp8Cache;

/*
 * Append: token t of sequence b, 0 <= t < count[b] (all S where count is NULL), goes to position start[b] + t.
 *     k, v   bf16 [B, Hkv, S, D]         start, count  int32 [B]
 * start is the number of tokens that the sequence holds before the call; what lay behind them is overwritten.
 * The exponent of a page that gets tokens, for keys and values alike:
 *     need = the least e >= -100 with  max |x| <= 448 * 2^e  over the finite ones of the page's new values
 *     e'   = need where the page held no token before, i.e. start[b] is not behind its first position; else max(e, need)
 * New codes are x * 2^-e' rounded to the nearest e4m3 (ties to even); NaN and infinities, which e4m3 does not have, become
 * the NaN code 0x7f.  Where e' > e the codes of the page's earlier tokens are rounded again to c * 2^(e - e').  All other
 * positions, those behind the last new token among them, keep their codes.
 * count outside 0 ... S is taken as the nearer end, positions outside the table are dropped.  A page that a call writes
 * stands once in the table: written as two pages, of one sequence or of two, it is left in no defined state.
 * Errors: NULL_PTR, BAD_SHAPE, UNSUPPORTED (D, page), MISALIGNED, LAUNCH.
 */
int kv_fp8_write(const KvFp8Cache *cache, const void *k, const void *v,
                 const long long *k_strides, const long long *v_strides,
                 const int *table, long long table_pitch, int width, const int *start, const int *count,
                 int B, int S, void *stream);

/*
 * Read back: k, v bf16 [B, Hkv, S, D], row s of sequence b = position first + s where that is less than lens[b] and its page
 * is there, else zeros.  Every value is exact (2^128, to which numbers next to bf16's largest can round, is infinite there).
 * lens int32 [B]; first >= 0; S >= 1.
 * Errors: as kv_fp8_write.
 */
int kv_fp8_read(const KvFp8Cache *cache, const int *table, long long table_pitch, int width, const int *lens,
                void *k, void *v, const long long *k_strides, const long long *v_strides,
                int B, int S, int first, void *stream);

/*
 * Attention over the cache: the definition of attn.h with sequence b's keys and values at the lens[b] first positions, for
 * q_lens[b] query rows (all Sq where q_lens is NULL), which are its last tokens: row i stands at position
 * p_i = lens[b] - q_lens[b] + i and sees
 *     J(i) = { j in [0, lens[b]), page there :  (!causal or j <= p_i)  and  (window == 0 or j > p_i - window or j < sinks) }
 * i.e. with a window its last `window` positions and the `sinks` first tokens of the sequence.
 *     s_ij = scale * q_i . k_j    lse_i = ln sum_{j in J(i)} exp(s_ij)    o_i = sum_{j in J(i)} exp(s_ij - lse_i) v_j
 *     q, o  bf16 [B, Hq, Sq, D]  (strided)     lse  fp32 [B, Hq, Sq] contiguous, may be NULL      lens, q_lens  int32 [B]
 * Scores, the running maximum and sum and the output are fp32; the probabilities are rounded to bf16 as the second operand
 * of the matrix instruction, o once when it is stored.  A row that sees no key, and rows i >= q_lens[b], get o = 0 and
 * lse = -inf.  NaN and infinities (codes of 256 and more at the exponent 120) in the cache reach the rows that see them and no
 * others, whatever lies behind the mask, behind the last token, or on pages that no sequence holds, codes and exponents.  An infinity
 * in the values makes its column of those rows infinite, or NaN where it meets the other sign or its probability is 0 in fp32.  (O is summed before it is divided, with
 * weights of up to 2^10: sums of values beyond 2^118 / keys can leave fp32.)
 * max_len: no sequence is longer, which the library counts on when it divides the work (0: width * page); lens is taken
 * as at most max_len (and as at most width * page), q_lens as 0 ... Sq.  lens may be less than q_lens: the rows at negative
 * positions see no key under a causal mask.
 *
 * Few query rows and long caches spread over the chip only with memory for fp32 parts: DEVICE memory, 16-byte aligned, its
 * contents irrelevant before and after; calls that overlap need one each.  attn_kv_fp8_workspace_bytes says how much the
 * library's own cut takes (0: none helps; host arithmetic only).  splits: workgroups along the keys of a kv head, 0 = the
 * library's choice, at most 256; splits > 1 needs 4 * B * Hq * Sq * splits * (D + 2) bytes.  With a NULL or too small
 * workspace, or splits = 1, the keys are not cut: the same result up to the order of fp32 sums.  Parts are added in a
 * fixed order: results do not vary from run to run.
 * wg_rows, for tuning and for tests that run every shape both ways: query rows (heads of one kv head side by side) per
 * workgroup, 16, 128, or 0 = the library's choice.
 * Supported: Hq a multiple of Hkv, Hq / Hkv * Sq < 2^28, B * Hq * Sq < 2^31 (cut: 2^24); 0 < scale <= 1e38; window, sinks >= 0.
 * Errors: NULL_PTR, BAD_SHAPE, UNSUPPORTED (D, page, splits, wg_rows), MISALIGNED (q, o, workspace 16 bytes; lse, lens, table 4),
 * BAD_SCALE, LAUNCH.
 */
size_t attn_kv_fp8_workspace_bytes(int B, int Hq, int Hkv, int Sq, int max_len, int D, int window, int sinks);

int attn_kv_fp8(const void *q, const KvFp8Cache *cache, const int *table, long long table_pitch, int width,
                const int *lens, const int *q_lens, void *o, float *lse, int B, int Hq, int Sq,
                const long long *q_strides, const long long *o_strides,
                int causal, int window, int sinks, float scale, int max_len,
                void *workspace, size_t workspace_bytes, int splits, int wg_rows, void *stream);

#ifdef __cplusplus
}
#endif
#endif
