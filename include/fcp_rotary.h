/*
 * fcp_rotary.h -- C ABI: rotary positions with several axes, in front of the block attention of fcp.h.
 *
 * A token of text has one position, one of an image or a video has several (time, height, width).  Every pair of a head's dimensions
 * belongs to one axis and turns by that position times the pair's frequency:
 *   (x, y) -> (x cos t - y sin t, x sin t + y cos t),   t = pos[row][axis[p]] * freq[p]
 * so that q . k depends on differences of positions alone.  A turn keeps lengths, so the gradient of a rotated tensor is turned back
 * (`inverse`) to give that of the tensor itself.  Conventions (errors, streams, pointers) as in fcp.h.
 */
#ifndef FCP_ROTARY_H_
#define FCP_ROTARY_H_

#include <stdint.h>

#include "fcp.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FCP_ROTARY_MAX_AXES = 8, FCP_ROTARY_MAX_PARTS = 4, FCP_ROTARY_MAX_DIM = 256 };

/*
 * fcp_rotary_turns -- frequencies as the kernel wants them, once per model (host).
 *
 * freq: host, [n], radians per position, |freq| <= 1e6 (FCP_ERR_INVALID_ARG otherwise).  turn: host, [n]: the fraction of a turn per
 * position, in units of 2^-64, off by at most 1 + |freq| / 4 of them.  A position times it, modulo 2^64, is the angle modulo one
 * turn, off by |pos| (1 + |freq| / 4) 2^-64 turns: with |freq| up to 1 at most 2^-32 of a turn, with the largest 2^-15, at positions of 2^31.
 */
int fcp_rotary_turns(const double* freq, int32_t n, uint64_t* turn);

/* Which dimensions turn, and how fast.  head_dim: a multiple of 16 up to 256.  n_pairs: a multiple of 8 up to head_dim / 2; dimensions
 * from 2 n_pairs on are copied.  Pair p is dimensions (p, p + n_pairs), or (2p, 2p + 1) with interleaved.
 * axis: host, [n_pairs], each in [0, n_axes).  turn: host, [n_pairs], from fcp_rotary_turns. */
typedef struct {
  int32_t head_dim, n_pairs, n_axes, interleaved;
  const int32_t* axis;
  const uint64_t* turn;
} fcp_rotary;

/* One tensor to turn: n_rows tokens of n_heads heads.  Row r is at src + r * src_row_stride elements (its heads follow each other), and
 * goes to dst + r * dst_row_stride: a slice of a fused projection, or the packed buffers of fcp.h (stride n_heads * head_dim).
 * src_f32, dst_f32: fp32 instead of bf16 (gradients as the backward wrote them; rounded once, to nearest even).
 * src, dst: device, rows aligned to 16 bytes.  They may be one tensor (same pointer, stride and type); otherwise they must not overlap,
 * nor may the dst of one part overlap another part of the call.
 * pos: device, int32 [n_rows, n_axes], any values. */
typedef struct {
  const void* src;
  void* dst;
  const int32_t* pos;
  int64_t src_row_stride, dst_row_stride;
  int32_t n_rows, n_heads, src_f32, dst_f32;
} fcp_rotary_part;

/*
 * fcp_rotary_apply -- turn up to FCP_ROTARY_MAX_PARTS tensors in one launch (Q and K, or dQ and dK with inverse = 1).
 *
 * Angles are those of `turn` at every position; sine and cosine are good to 2e-7.  Arithmetic is fp32.  The call keeps nothing and
 * allocates nothing; it may be captured into a graph (the frequencies then are those of the capture).
 * Errors: FCP_ERR_INVALID_ARG (NULL, counts, an axis out of range, a stride below a row, one tensor with two strides or types),
 * FCP_ERR_UNSUPPORTED (dimensions or alignments other than above; more than 2^24 - 1 groups of four rows, which is 67 million rows in one part).
 */
int fcp_rotary_apply(const fcp_rotary* r, const fcp_rotary_part* parts, int32_t n_parts, int32_t inverse, void* stream);

/*
 * fcp_row_positions -- position in its sequence of every row of a problem's buffers (host, integer only).
 *
 * q_rows, kv_rows: host, caller-allocated, one int32 per row of the Q and of the K / V buffer.  A row of a plain block is at the block's
 * position (scores->q_pos / kv_pos where FCP_FLAG_SCORES gives them, else the tokens of its sequence in the kv_blocks before it)
 * plus its place in the block; a row of a packed block is at its place in its member.
 * Errors: as fcp_workspace_bytes; FCP_ERR_INVALID_ARG if a query block is none of the kv_blocks and no positions are given.
 */
int fcp_row_positions(const fcp_problem* p, int32_t* q_rows, int32_t* kv_rows);

#ifdef __cplusplus
}
#endif
#endif /* FCP_ROTARY_H_ */
