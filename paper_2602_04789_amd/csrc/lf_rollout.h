// Internal declarations of the three-axis producer and of the 4-bit cache.
#ifndef LF_ROLLOUT_H
#define LF_ROLLOUT_H

#include "lf_common.h"

// How a call of the three-axis producer is laid over threads: heads of a thread, heads side by side, tokens of a workgroup, threads.
struct lf_axes_lay {
  int ni, hpt, tt, threads;
};
#define LF_AXES_MAX_BLOCKS 512       // workgroups of the backward kernel
#define LF_AXES_MAX_CHANNELS 16384   // heads * head_dim: what 512 threads of four heads each hold
inline lf_axes_lay lf_lay_axes(int H, int d, int want_ni, int want_threads) {
  const int ch = d / 8;
  lf_axes_lay l;
  l.ni = want_ni;
  while (l.ni > 1 && l.ni > H) l.ni /= 2;
  while ((H + l.ni - 1) / l.ni * ch > 512) l.ni *= 2;
  l.hpt = (H + l.ni - 1) / l.ni;
  l.tt = want_threads / (l.hpt * ch);
  if (l.tt < 1) l.tt = 1;
  l.threads = (l.tt * l.hpt * ch + 63) / 64 * 64;
  return l;
}
// More heads to a thread share its angles, fewer shorten its chain.  Forward, us, one / two / four heads (workgroups of 256 / 256 / 512): 1 token of
// 12 x 128: 2.13 / 2.38 / 3.05; 300: 2.96 / 3.07 / 4.2; 600: 3.25 / 3.38 / 4.3; 1 200: 3.71 / 3.75 / 4.43; 2 400: 5.06 / 4.56 / 4.8; 4 680: 8.3 / 7.36 / 7.4;
// 9 000 of 12 x 64 by halves: 9.75 / 8.44 / 7.7; 32 760 of 40 x 128: four to a thread in workgroups of 512 122, of 256 145.
inline lf_axes_lay lf_lay_axes_fwd(int H, int d, int L) {
  const int64_t n = (int64_t)H * d * L;
  return n <= 1 << 20 ? lf_lay_axes(H, d, 1, 256) : n <= 1 << 22 ? lf_lay_axes(H, d, 2, 256) : lf_lay_axes(H, d, 4, 512);
}
// Forward and backward, two heads to a thread / four: 4 680 tokens of 12 x 128: 22.8 / 21.8, 32 760 of 40 x 128: 326 / 340, of 12 x 64: 52 / 58;
// one head, in workgroups of 256: 1 333 of 5 x 64: 11.3 / 10.5, 4 680 of 12 x 128: 22.8 / 29.4.  (126 registers, four to a thread take 230.)
inline lf_axes_lay lf_lay_axes_bwd(int H, int d) { return lf_lay_axes(H, d, 2, 512); }
// Workgroups of the backward kernel; each leaves a row of the norm weight's gradient.
inline int lf_axes_bwd_blocks(int H, int d, int L) {
  const lf_axes_lay l = lf_lay_axes_bwd(H, d);
  const int groups = (L - 1) / l.tt + 1;
  return groups < LF_AXES_MAX_BLOCKS ? groups : LF_AXES_MAX_BLOCKS;
}

// Where the parts of a 4-bit cache begin (bytes): codes of K and V [H][capacity][d/2], their scales [H][capacity][d/32].
struct lf_kvq_parts {
  int64_t codes[2], scales[2], bytes;
};
inline lf_kvq_parts lf_kvq_layout(const lf_kvq_shape& s) {
  auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
  const int64_t rows = (int64_t)s.heads * s.capacity;
  const int64_t codes = up(rows * (s.head_dim / 2)), scales = up(rows * (s.head_dim / 32));
  lf_kvq_parts p;
  p.codes[0] = 0;
  p.codes[1] = codes;
  p.scales[0] = 2 * codes;
  p.scales[1] = 2 * codes + scales;
  p.bytes = 2 * (codes + scales);
  return p;
}

// One call of the attention over the cache, for both entry points.
struct lf_kvq_call {
  const void *Q, *K, *V;       // K, V: rows in bfloat16 behind the cached ones, or null
  void* O;
  const uint8_t* cache;
  lf_kvq_shape cs;
  int H, d, q_len;
  int64_t q_stride_tok, q_stride_head, k_stride_tok, k_stride_head, v_stride_tok, v_stride_head, o_stride_tok, o_stride_head;
  float scale;
  const int32_t* indices;      // null: every token is seen by every row
  int list_len;
  int n, nb, n_q, n_k;         // frames and their blocks (lists)
  int cached, extra;           // tokens in the cache and behind it
  int rows;                    // query rows of a block, at most 64
  int parts;                   // workgroups that share a query block's list
  void* workspace;
};
// 16 query rows each that a wavefront holds.
inline int lf_kvq_tiles(int rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }
#define LF_KVQ_MAX_PARTS 64     // a lane of the joining wavefront each
// Into how many workgroups of four wavefronts the list of a query block is divided: until every compute unit has two, as long as each
// wavefront has a KV block.
inline int lf_kvq_parts_of(int64_t blocks, int64_t entries) {
  int64_t p = blocks > 0 ? 512 / blocks : 1;
  if (p > entries / 4) p = entries / 4;
  return (int)(p < 1 ? 1 : p > LF_KVQ_MAX_PARTS ? LF_KVQ_MAX_PARTS : p);
}
// Whether a call with lists first writes the cache's rows in bfloat16 and runs the bfloat16 kernels on them.  That costs its time for every
// token of the cache (1.4 us a million values), the kernel that converts what it reads pays for every tile of 64 x 64 (2.0 ns more at d = 128, 1.2 at
// d = 64).
inline bool lf_kvq_expands(int d, int64_t blocks, int64_t entries, int64_t H, int64_t kv_len) {
  return blocks * entries * (d == 128 ? 1470 : 860) > H * kv_len * d + 700000;
}
// Float32 state of the parts: O [H n_q][parts][16 tiles][d], then (reference, sum) [H n_q][parts][16 tiles][2].
inline int64_t lf_kvq_state_bytes(int64_t blocks, int parts, int rows, int d) {
  return parts == 1 ? 0 : blocks * parts * 16 * lf_kvq_tiles(rows) * (d + 2) * 4;
}

int lf_launch_rope_axes(const void* X, const float* g, const int32_t* pos, const double* freq, const lf_axes_shape* p, void* Y,
                        void* stream);
int lf_launch_rope_axes_bwd(const void* X, const float* g, const int32_t* pos, const double* freq, const lf_axes_shape* p,
                            const void* dY, void* dX, float* dg, float* part, void* stream);
int lf_launch_kvq_append(const void* K, const void* V, const lf_kvq_shape* s, const lf_kvq_rows* r, uint8_t* cache, void* stream);
int lf_launch_kvq_read(const uint8_t* cache, const lf_kvq_shape* s, const lf_kvq_rows* r, void* K, void* V, void* stream);
int lf_launch_kvq_expand(const lf_kvq_call* c, uint16_t* K, uint16_t* V, void* stream);
int lf_launch_kvq_attn(const lf_kvq_call* c, void* stream);

#endif
