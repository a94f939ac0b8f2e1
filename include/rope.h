/*
 * rope.h -- C ABI of the MI355X (gfx950) rotary position embedding.
 *
 * Operation: the first R columns of a head's row are R/2 pairs, and pair f of the token at position p is turned by the
 * angle p * inv_freq[f]:
 *
 *     c = mscale * cos(p * inv_freq[f])      s = mscale * sin(p * inv_freq[f])
 *     y0 = x0 * c - x1 * s                   y1 = x0 * s + x1 * c
 *
 *     interleaved == 0 :  x0, x1 are columns f and f + R/2           (halves)
 *     interleaved != 0 :  x0, x1 are columns 2 f and 2 f + 1         (neighbours)
 *
 * Columns R ... D-1 are copied.  inverse != 0 turns by the opposite angle (s changes its sign): the transposed rotation,
 * which is the gradient of the operation with respect to x (times mscale, as the operation itself).
 * The angle is formed and reduced to a part of a turn in 64 bits, so that at frequencies of up to one radian per position it
 * is off by less than 2^-20 at any position; sine, cosine and the products are fp32, every result is rounded once to bf16 (nearest even).
 *
 * DEVICE pointers, caller-owned:
 *     q, q_out   bf16 [B, Hq, S, D]      k, k_out  bf16 [B, Hk, S, D], both NULL (and Hk 0): only q
 *     positions  int32 [B, S], entry (b, s) at positions[b * positions_pitch + s] (pitch 0: the same for every sequence);
 *                any value, negative ones too
 *     inv_freq   fp64 [R/2], radians per position: rope_frequencies gives the usual ones
 * Each *_strides points to 3 HOST integers {batch, head, row} in ELEMENTS, as in attn.h: multiples of 8, none negative, the
 * row stride >= D, every stride < 2^40; the D elements of a row are contiguous and 16-byte aligned.  An output may be its
 * input (same pointer and strides); otherwise outputs overlap neither the inputs nor each other nor themselves.
 *
 * Supported: D a multiple of 8, at most 1024; R even, 2 <= R <= D; B, Hq, S >= 1, Hk >= 0, B * S * D < 2^31, Hq + Hk <= 65535;
 * mscale finite.  `stream` is a hipStream_t passed as void* (NULL = the default stream); the call enqueues one kernel there
 * and returns, allocates nothing and holds no state.  Every check precedes the first HIP call.  Return codes are those of
 * attn.h: NULL_PTR, BAD_SHAPE, UNSUPPORTED (D or R), MISALIGNED (rows not 16-byte aligned, positions 4, inv_freq 8),
 * BAD_SCALE (mscale), LAUNCH.
 */
#ifndef ROPE_MI355X_H
#define ROPE_MI355X_H

#ifdef __cplusplus
extern "C" {
#endif

int rope_bf16(const void *q, void *q_out, const void *k, void *k_out,
              int B, int Hq, int Hk, int S, int D, int R,
              const long long *q_strides, const long long *q_out_strides,
              const long long *k_strides, const long long *k_out_strides,
              const int *positions, long long positions_pitch, const double *inv_freq,
              int interleaved, int inverse, float mscale, void *stream);

/*
 * The frequencies of R/2 pairs, inv_freq[f] = base^(-2 f / R), into HOST memory.  For a context `factor` times as long as the
 * `original_len` positions a model was trained on, the pairs that turn often enough there keep their frequency and the slow
 * ones are slowed down by the factor, with a ramp between:
 *     turns = original_len * inv_freq / (2 pi)       keep = clamp((turns - slow) / (fast - slow), 0, 1)
 *     inv_freq' = inv_freq * (keep + (1 - keep) / factor)
 * original_len 0: every frequency is divided by the factor.  Host arithmetic in 64 bits.  BAD_SHAPE: R odd or < 2,
 * original_len negative; BAD_SCALE: base <= 1, factor < 1, slow < 0 or fast <= slow (checked where original_len > 0), or
 * one of them not finite; NULL_PTR.
 */
int rope_frequencies(int R, double base, double factor, int original_len, double slow, double fast, double *inv_freq);

#ifdef __cplusplus
}
#endif
#endif
