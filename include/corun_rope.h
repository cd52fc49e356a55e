/*
 * Rotary positions, for NVIDIA B200 (sm_100a): the first rot_dim values of a head as rot_dim / 2 pairs (x1, x2),
 *     y1 = m (x1 cos a - x2 sin a),   y2 = m (x2 cos a + x1 sin a),   a = position * f_i   (pair i),
 * the other values as they are (csrc/rope.cu).  The engine's own decoders rotate whole heads in pairs (i, i + rot_dim / 2)
 * at f_i = theta^(-2i / rot_dim); here pairs may also be neighbours, a part of the head may be rotated, and the
 * frequencies may be stretched for contexts longer than the trained one.  Angles are formed and reduced in 64 bits
 * (a position of a million is half a radian off in 32), the products in 32.
 * Data pointers are DEVICE pointers; calls are asynchronous on the given stream.  Status codes are those of corun.h.
 */
#ifndef CORUN_ROPE_H
#define CORUN_ROPE_H

#include <stdint.h>

#include "corun.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of the tensors of this header and of corun_kv8.h. */
typedef enum { CORUN_F32 = 0, CORUN_BF16 = 1, CORUN_F16 = 2 } corun_dtype;

/* Where the values of token t, head h begin: p + t * token_stride + h * head_stride, in values of the tensor's type;
 * a head's values are contiguous. */
typedef struct {
  void *p;
  int64_t token_stride, head_stride;
} corun_heads;

typedef enum {
  CORUN_ROPE_PLAIN = 0,  /* f_i = theta^(-2i / rot_dim)                                                          */
  CORUN_ROPE_LINEAR = 1, /* f_i / factor                                                                         */
  CORUN_ROPE_BASE = 2,   /* theta * factor^(rot_dim / (rot_dim - 2)) instead of theta (known as NTK-aware)        */
  CORUN_ROPE_PARTS = 3,  /* known as YaRN; low and high are its beta_slow and beta_fast.  With d(n) = rot_dim ln(original_context / (2 pi n)) / (2 ln theta), the pair that turns n
                            times in the trained context: r = clamp((i - first) / (last - first), 0, 1) from first =
                            max(floor d(high), 0) to last = min(ceil d(low), rot_dim - 1), f_i (1 - r + r / factor);
                            magnitude 0.1 ln(factor) + 1                                                         */
  CORUN_ROPE_BANDS = 4   /* by wavelength; low and high are called low_freq_factor and high_freq_factor in configurations that
                            use it.  s = clamp((original_context f_i / (2 pi) - low) / (high - low), 0, 1),
                            f_i (s + (1 - s) / factor)                                                           */
} corun_rope_scaling;

typedef struct {
  int32_t rot_dim;          /* even, 2..256                                                    */
  int32_t interleaved;      /* 0: pairs (i, i + rot_dim / 2); 1: pairs (2i, 2i + 1)            */
  int32_t scaling;          /* corun_rope_scaling                                              */
  int32_t original_context; /* PARTS, BANDS: the trained context, > 0                          */
  double theta;             /* > 0 (PARTS: > 1)                                                */
  double factor;            /* >= 1 (PLAIN: not read)                                          */
  double low, high;         /* PARTS, BANDS: 0 < low < high                                    */
  double magnitude;         /* m; 0 = the scaling's own (1 but for PARTS)                      */
} corun_rope_config;

typedef struct corun_rope corun_rope; /* host memory only: usable on every device, by several threads at once */

/* Errors: EINVAL, ENOMEM. */
int corun_rope_create(const corun_rope_config *config, corun_rope **out);
/* Launches already made (and captured) keep their own copy of the table.  NULL is allowed. */
void corun_rope_destroy(corun_rope *r);

/*
 * y[t, h, :] = rotated x[t, h, :] for T tokens of `heads` heads of head_dim values at positions[t] (int32 [T], may be
 * negative).  x and y have the same type; y may be x itself, otherwise the two do not overlap.  T 0 does nothing.
 * rot_dim <= head_dim <= 1024.  16 bytes at a time where every head starts on 16 bytes and a pair's halves lie in whole
 * groups of 16, value by value otherwise; the results are the same.  Errors: EINVAL, ECUDA.
 */
int corun_rope_apply(const corun_rope *r, const corun_heads *x, const corun_heads *y, int32_t dtype, const int32_t *positions,
                     int64_t T, int32_t heads, int32_t head_dim, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif
