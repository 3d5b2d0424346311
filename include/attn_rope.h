/*
 * attn_rope.h -- C ABI of libmi355attn.so: rotary positions for MI355X (gfx950).
 *
 * Every head of q and k is turned by the positions of its token before attention.  A token has a
 * position on each of n_axes axes (one for text; time, height and width for images and video); the
 * R = 2 * (sections[0] + ... + sections[n_axes-1]) leading elements of a head form R/2 pairs, the
 * first sections[0] pairs follow axis 0, the next sections[1] axis 1, and so on.  For pair i on axis a:
 *
 *     t  = pos[a][b][s] * freq[i]
 *     y1 = x1 cos(t) - x2 sin(t)      (x1, x2) = (x[i], x[i + R/2])     interleaved == 0
 *     y2 = x1 sin(t) + x2 cos(t)               = (x[2i], x[2i + 1])     interleaved != 0
 *
 * The elements from R on are copied.  The angle is formed and reduced to one turn in 64 bits (a far
 * position leaves no correct digit of a 32-bit angle), its sine and cosine and the products are 32-bit,
 * and each output is rounded once.  The turn is orthogonal: the gradient with respect to x is the
 * gradient with respect to y turned the other way (inverse != 0).
 */
#ifndef MI355_ATTN_ROPE_H
#define MI355_ATTN_ROPE_H

#ifdef __cplusplus
extern "C" {
#endif

/*
 * attn_rope -- enqueue the turn of q and k on `stream` and return (asynchronous).
 *
 *   q, q_out   device pointers, bf16, heads q[b][h][s] of D elements, b < B, h < H_q, s < S
 *   k, k_out   the same with H_kv heads; H_kv = 0: q only (k and k_out are ignored)
 *   strides    host array of 12: elements from one b, h and s to the next, of q, q_out, k and k_out in
 *              this order; the D elements of a head are contiguous.  Multiples of 8, not negative
 *   pos        device pointer, int32, contiguous [n_axes][B][S]                       (read only)
 *   freq       device pointer, fp64, R/2 radians per unit of position                 (read only)
 *   sections   host array of n_axes counts >= 0
 *   n_axes     1 .. 4
 *   B, H_q, S  >= 1; H_kv >= 0; D 64, 128 or 256; R a multiple of 16, 16 <= R <= D
 *   inverse    0: as above; non-zero: with -t
 *
 * q_out may be q and k_out may be k (same strides); otherwise outputs overlap neither inputs nor each
 * other.  No output row may be stored twice (a stride of 0 is for inputs).
 *
 * Ownership, errors and streams are those of attn_fwd (attn_fwd.h): arguments are validated on the host
 * before any HIP call; ATTN_ERR_SHAPE stands for sizes, sections, strides and R alike, and for a call
 * that would take 2^32 threads (one head of 2^30 tokens at R = 64), ATTN_ERR_ALIGN for tensors that are not 16-byte
 * aligned (pos 4, freq 8).  Bitwise reproducible.
 */
int attn_rope(const void *q, void *q_out, const void *k, void *k_out, const long long *strides,
              const int *pos, const double *freq, const int *sections, int n_axes,
              int B, int H_q, int H_kv, int S, int D, int interleaved, int inverse, void *stream);

/* attn_rope on IEEE fp16 tensors; everything else as attn_rope. */
int attn_rope_f16(const void *q, void *q_out, const void *k, void *k_out, const long long *strides,
                  const int *pos, const double *freq, const int *sections, int n_axes,
                  int B, int H_q, int H_kv, int S, int D, int interleaved, int inverse, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MI355_ATTN_ROPE_H */
