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
// Tiles of 16 query rows of a block; a wavefront holds one or two of them, so two wavefronts share a block of four.
inline int lf_kvq_tiles(int rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }
#define LF_KVQ_MAX_PARTS 64     // a lane of the joining wavefront each
// Into how many workgroups of four wavefronts the list of a query block is divided: until every compute unit has two, as long as each
// wavefront has a KV block.  Lists that give the wavefronts of one workgroup (with more than 32 rows two share a block) four blocks at the
// most stay whole: joining the parts costs more than it brings.  us, divided / whole: 12 heads of 128, one row, 501 tokens 8.9 / 7.2, 701 7.6 / 7.3,
// 1 001 (17 blocks) 8.9 / 9.7, 1 401 9.0 / 11.1; 40 heads of 64, 701 6.5 / 5.8; 8 query blocks of 64 rows, lists of 12 9.2 / 10.4.
inline int lf_kvq_parts_of(int64_t blocks, int64_t entries, int rows) {
  if (entries <= (rows > 32 ? 8 : 16)) return 1;
  int64_t p = 512 / blocks;
  if (p > entries / 4) p = entries / 4;
  return (int)(p < 1 ? 1 : p > LF_KVQ_MAX_PARTS ? LF_KVQ_MAX_PARTS : p);
}
// Whether a call with lists first writes the cache's rows in bfloat16 and runs the bfloat16 kernels on them.  That costs time for every value
// of the cache, whatever the lists keep, and these kernels do not divide a list among workgroups; the kernel that converts what it reads pays for that at
// every tile, once for every query block.  Up to 256 query blocks both sides' times (us) are put together from what they are made of,
// beyond, tiles are weighed against values.  8 340 random calls (1 to 40 heads, frames of 8 to 1 600 tokens, lists of 1 to 3 000 blocks), both ways each:
// this choice costs 0.9 % on the mean over the faster one (0.6 at the worst call), the bfloat16 kernels always 33 % (6.1), the converting one always 12 % (1.7).
inline bool lf_kvq_expands(int d, int64_t blocks, int64_t entries, int rows, int64_t H, int64_t kv_len) {
  const int64_t values = H * kv_len * d;
  const bool wide = d == 128;
  if (blocks > 256) return blocks * entries * (wide ? 1400 : 750) > values;
  const int parts = lf_kvq_parts_of(blocks, entries, rows), at_once = parts * (rows > 32 ? 2 : 4);
  const double tiles = (double)((entries + at_once - 1) / at_once);
  double convert = (wide ? 4.7 : 4.2) + tiles * (blocks * parts <= 256 ? (wide ? 1.8 : 1.2) : (wide ? 2.8 : 1.8));
  if (parts > 1) convert += (wide ? 3.9 : 3.2) + blocks * rows * (wide ? 0.0024 : 0.0014);
  const double expand = (wide ? 9.1 : 8.7) + values * 1.35e-6 +
                        entries * (blocks <= 128 ? (wide ? 0.267 : 0.146) : (wide ? 0.505 : 0.334));
  return expand < convert;
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
