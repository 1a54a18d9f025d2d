// Internal declarations of the calls around the attention: norms between blocks, packed attention, gradient clipping.
#ifndef LF_BLOCKS_H
#define LF_BLOCKS_H

#include "lf_common.h"

// ---- norms between blocks ----

// A workgroup has one row at a time: `threads` of it hold `nc` chunks of 8 channels each.
struct lf_norm_lay {
  int nc, threads;
};
#define LF_NORM_MAX_CHANNELS 16384
inline lf_norm_lay lf_lay_norm(int channels, int nc) {
  const int chunks = channels / 8;
  return {nc, ((chunks + nc - 1) / nc + 63) / 64 * 64};
}
// Rows that a workgroup of the forward kernel takes one after the other.
int lf_norm_fwd_rows(const lf_norm_shape* s, lf_norm_lay* lay);
// Rows of a slot of the backward kernel, slots, and the floats of workspace: three sums a slot and channel, two a group and channel.
struct lf_norm_slots {
  lf_norm_lay lay;
  bool waves;          // a row for each of four wavefronts; `lay` is that of one
  int rows;
  int per_group;       // slots of a group (group_len > 0)
  int64_t slots, floats;
};
lf_norm_slots lf_norm_bwd_slots(const lf_norm_shape* s);

struct lf_norm_call {
  const lf_norm_shape* s;            // backward: with the groups that have tokens
  int32_t groups;                    // backward: rows of the tables' gradients
  const void *X, *B;
  const float *gate, *post_weight, *weight, *scale, *shift;
  const int32_t* starts;
  void *Xout, *Y;                    // forward; backward: Xout is read
  const void *dY, *dXout;            // backward
  void *dX, *dB;
  float *dgate, *dpost_weight, *dweight, *dscale, *dshift;
  float* workspace;
};
int lf_launch_gate_norm(const lf_norm_call* c, void* stream);
int lf_launch_gate_norm_bwd(const lf_norm_call* c, void* stream);

// ---- gradient clipping ----

// Elements of a workgroup's share of a tensor: the fewest that leave about 1000 shares or less, since each one has the parts of the norm to add (18 tensors of 0.8 million
// float32: 6.4 us, shares of 4096 7.3), and at the most 65 536 (340 million float32: 236 us; 32 768 244, 4096 377).
inline int64_t lf_grad_chunk(int64_t numel) {
  int64_t c = 16384;
  while (c < 65536 && numel / c > 1024) c *= 2;
  return c;
}
inline int64_t lf_grad_most_chunks(int32_t count, int64_t numel) { return numel / lf_grad_chunk(numel) + count; }
int lf_launch_grad_clip(const lf_grad_tensor* t, int32_t count, int64_t numel, float max_norm, float eps, float* norm, double* part,
                        void* stream);

// ---- packed attention ----

#define LF_PACKED_MAX_PARTS 64
// Which kernels a call takes and how its work is laid over workgroups.
struct lf_packed_plan {
  bool few;            // tiles of 16 or 32 rows, the heads that share a head side by side among them
  int tile;            // rows of a tile (few: of row and head)
  int64_t slots;       // tiles at the most, over all sequences
  int parts;           // workgroups that share a tile's tokens, at the most
  int part_tokens;     // and the fewest tokens that one of them takes
  int64_t state_bytes; // float32 state of the parts
};
lf_packed_plan lf_plan_packed(const lf_packed_shape* s);

struct lf_packed_call {
  const lf_packed_shape* s;
  lf_packed_plan plan;
  const void *Q, *K, *V, *dO;
  void *O, *dQ, *dK, *dV;
  float* lse2;
  const int32_t *q_start, *kv_start;
  float scale;
  void* workspace;
};
int lf_launch_packed_attn(const lf_packed_call* c, void* stream);
int lf_launch_packed_rows(const lf_packed_call* c, void* stream);
int lf_launch_packed_bwd(const lf_packed_call* c, void* stream);

#endif
