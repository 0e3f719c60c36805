/*
 * clq_rope.h - rotary positions over several axes (time, height, width) in
 * libclq, for one GB300 (sm_103a): what stands between the QKV product of a
 * block of an image or video transformer and its attention.
 *
 * Conventions are clq.h's (status codes, device pointers owned by the caller,
 * no allocation, no synchronization, asynchronous on `stream`, arguments
 * checked on the host before anything is launched); `out` shares no memory with positions or turns.
 *
 * A head of D values has P pairs, 2 P <= D; its other D - 2 P values stay as
 * they are.  Pair p of a token belongs to an axis a(p), the first sections[0]
 * pairs to axis 0, the next sections[1] to axis 1, and so on, and is turned by
 * the angle pos[a(p)] f_p:
 *     (x, y) -> (x cos - y sin, y cos + x sin),
 * or back (by the negative angle) if `inverse`, which is the gradient as well.
 * ANGLES.  f_p is given as a fraction of a turn in 64 bits, turns[p] =
 * round(f_p / (2 pi) 2^64) mod 2^64: its product with a whole position, mod
 * 2^64, is the position's own fraction of a turn, so that far positions lose
 * nothing.  A result is within 2^-20 (|x| + |y|) of the exact one, and rounded once.
 */
#ifndef CLQ_ROPE_H
#define CLQ_ROPE_H

#include "clq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t clq_rope_pairs;
#define CLQ_ROPE_INTERLEAVED 0 /* pair p: values 2 p and 2 p + 1 of a head */
#define CLQ_ROPE_HALVES 1      /* pair p: values p and P + p               */

/*
 * x, out: device, `dtype` (fp16 / bf16); token t, head h, value d at
 * t token_stride + h head_stride + d (elements, not negative); out's
 * heads are apart, all of a token inside its stride or all of a head number inside theirs; out may
 * be x itself with the same strides, and does not meet it otherwise (refused; where x has other strides
 * than out, and not 0 instead, ranges of addresses that meet are).  T < 2^30 tokens of H
 * <= 65535 heads of D <= 4096 values.  positions: device int32, that of axis a of
 * token t at t ld_positions + a, any sign.  axes: 1 to 4; host_sections: host int32
 * [axes], pairs of each axis (0 or more), 1 <= P = their sum <= D / 2.  turns: device
 * uint64 [P].  Any alignment of the values; with strides and addresses that are
 * multiples of 16 bytes they travel 16 at a time.
 */
clq_status clq_rope(const void* x, clq_dtype dtype, int32_t T, int32_t H, int32_t D,
                 int64_t token_stride, int64_t head_stride, const int32_t* positions,
                 int32_t ld_positions, int32_t axes, const int32_t* host_sections,
                 const uint64_t* turns, clq_rope_pairs pairs, int32_t inverse, void* out,
                 int64_t out_token_stride, int64_t out_head_stride, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CLQ_ROPE_H */
