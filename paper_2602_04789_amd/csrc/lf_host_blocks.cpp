// Host side of the calls around the attention: validation, sizes and how a call is laid over workgroups.  No GPU code here.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>

#include "lf_blocks.h"

namespace {

bool misaligned(const void* p, size_t a) { return ((uintptr_t)p % a) != 0; }
constexpr int64_t kMostThreads = (int64_t)1 << 32;      // a grid has fewer

// ---- norms between blocks ----

int check_norm(const lf_norm_shape* s) {
  if (s->tokens < 1 || s->tokens > 1 << 30 || s->channels < 8 || s->channels > LF_NORM_MAX_CHANNELS || s->channels % 8) return LF_ERR_SHAPE;
  if (s->groups < 1 || s->groups > 1 << 24 || s->group_len < 0) return LF_ERR_SHAPE;
  if (s->group_len > 0 && (int64_t)s->group_len * s->groups < s->tokens) return LF_ERR_SHAPE;
  if (s->kind != LF_NORM_LAYER && s->kind != LF_NORM_RMS) return LF_ERR_SHAPE;
  if (!(s->eps >= 0.0f) || isinf(s->eps) || isnan(s->residual_scale) || isinf(s->residual_scale)) return LF_ERR_SHAPE;
  if (s->stream_dtype != LF_BF16 && s->stream_dtype != LF_F32) return LF_ERR_DTYPE;
  return LF_OK;
}
// Row strides of tensors that the call has.
int check_rows(const lf_norm_shape* s, int64_t stride) {
  if (stride < s->channels || stride > (int64_t)1 << 40) return LF_ERR_SHAPE;
  return stride % 8 ? LF_ERR_ALIGN : LF_OK;
}
int check_table(const lf_norm_shape* s, const void* p, int64_t stride) {
  if (!p || s->groups == 1) return LF_OK;
  if (stride < s->channels || stride > (int64_t)1 << 40) return LF_ERR_SHAPE;
  return stride % 4 ? LF_ERR_ALIGN : LF_OK;
}
int first_error(const int* rc, int n) {
  for (int i = 0; i < n; ++i)
    if (rc[i] == LF_ERR_SHAPE) return rc[i];
  for (int i = 0; i < n; ++i)
    if (rc[i] != LF_OK) return rc[i];
  return LF_OK;
}
// The shape with no more of group_len and of groups than the tokens fill: a slot's rows follow from it (4680 rows of 1536 in one group, backward: 27 us, and with a
// group_len of 2^20 taken as it is, so that two of 256 slots have all the rows, 1955).
lf_norm_shape filled(const lf_norm_shape* s) {
  lf_norm_shape f = *s;
  if (f.group_len > 0) {
    f.group_len = std::min(f.group_len, f.tokens);
    f.groups = (f.tokens - 1) / f.group_len + 1;
  }
  return f;
}
int check_slots(const lf_norm_shape* s) {
  const lf_norm_shape f = filled(s);
  const lf_norm_slots n = lf_norm_bwd_slots(&f);
  return n.slots * (n.waves ? 256 : n.lay.threads) < kMostThreads && n.floats <= (int64_t)1 << 38 ? LF_OK : LF_ERR_SHAPE;
}

// ---- packed attention ----

bool heads_overlap(int heads, int64_t stride_head, int tokens, int64_t stride_tok, int d) {
  if (heads < 2 || tokens < 1) return false;
  if (stride_head < d) return true;
  if (tokens < 2 || (stride_head - d) / stride_tok >= tokens - 1 || (stride_tok - d) / stride_head >= heads - 1) return false;
  for (int h = 1; h < heads; ++h) {
    const __int128 off = (__int128)h * stride_head, t = off / stride_tok, past = off - t * stride_tok;
    if (t < tokens && past < d) return true;
    if (t + 1 < tokens && stride_tok - past < d) return true;
  }
  return false;
}
constexpr int64_t kMaxStride = 1 << 20;      // of a token: 64 of them within 32-bit offsets
constexpr int64_t kMaxHeadStride = (int64_t)1 << 44;

int check_stride(int64_t tok, int64_t head, int d) {
  if (tok < d || tok > kMaxStride || head < 0 || head > kMaxHeadStride) return LF_ERR_SHAPE;
  return tok % 8 || head % 8 ? LF_ERR_ALIGN : LF_OK;
}
// Sizes alone.
int check_sizes(const lf_packed_shape* s) {
  if (s->head_dim != 64 && s->head_dim != 128) return LF_ERR_SHAPE;
  if (s->kv_heads < 1 || s->kv_heads > 4096 || s->heads < s->kv_heads || s->heads % s->kv_heads || s->heads / s->kv_heads > 256) return LF_ERR_SHAPE;
  if (s->seqs < 1 || s->seqs > 1 << 20 || s->q_len < 0 || s->q_len > 1 << 30 || s->kv_len < 0 || s->kv_len > 1 << 30) return LF_ERR_SHAPE;
  if (s->causal < 0 || s->causal > 1 << 30) return LF_ERR_SHAPE;
  const int64_t group = s->heads / s->kv_heads;
  if (s->q_len * group > (int64_t)1 << 34) return LF_ERR_SHAPE;
  const lf_packed_plan p = lf_plan_packed(s);
  const int64_t heads = p.few ? s->kv_heads : s->heads;
  int64_t blocks = p.slots * heads * p.parts;
  if (p.parts > 1 && p.slots * heads * (p.tile / 4) > blocks) blocks = p.slots * heads * (p.tile / 4);
  const int64_t dq = ((int64_t)s->q_len / 128 + s->seqs) * s->heads, dkv = ((int64_t)s->kv_len / 64 + s->seqs) * s->kv_heads;
  if (dq > blocks) blocks = dq;
  if (dkv > blocks) blocks = dkv;
  return blocks * 256 < kMostThreads ? LF_OK : LF_ERR_SHAPE;
}
int check_packed(const lf_packed_shape* s) {
  const int rc = check_sizes(s);
  if (rc != LF_OK) return rc;
  if (s->dtype != LF_BF16) return LF_ERR_DTYPE;
  const int all[4] = {check_stride(s->q_stride_tok, s->q_stride_head, s->head_dim), check_stride(s->k_stride_tok, s->k_stride_head, s->head_dim),
                      check_stride(s->v_stride_tok, s->v_stride_head, s->head_dim), check_stride(s->o_stride_tok, s->o_stride_head, s->head_dim)};
  return first_error(all, 4);
}
// The gradients divide the log-sum-exp by it, and logits are taken to lie above -1e30.
bool scale_ok(float s) { return s == 0.0f || (s >= 1e-30f && s <= 1e20f); }
float scale_or_default(float s, int d) { return s > 0.0f ? s : 1.0f / sqrtf((float)d); }

// ---- gradient clipping ----

struct Range {
  uintptr_t from, to;
  bool written;
};
// Whether a tensor that is written shares memory with another one (the same gradient listed twice would be scaled twice, or not).
int written_once(const lf_grad_tensor* t, int32_t count, bool norm_alone) {
  Range few[64], *all = 2 * (int64_t)count <= 64 ? few : (Range*)malloc(2 * (size_t)count * sizeof(Range));
  if (!all) return LF_ERR_WORKSPACE;
  int32_t n = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (t[i].numel == 0) continue;
    const uintptr_t data = (uintptr_t)t[i].data, out = (uintptr_t)t[i].out;
    const bool apart = out && out != data;
    all[n++] = {data, data + (uintptr_t)t[i].numel * (t[i].dtype == LF_F32 ? 4 : 2), !apart && !norm_alone};
    if (apart) all[n++] = {out, out + (uintptr_t)t[i].numel * (t[i].out_dtype == LF_F32 ? 4 : 2), true};
  }
  std::sort(all, all + n, [](const Range& a, const Range& b) { return a.from < b.from; });
  uintptr_t any = 0, written = 0;          // ends of what stands before
  bool once = true;
  for (int32_t i = 0; i < n && once; ++i) {
    once = all[i].from >= (all[i].written ? any : written);
    any = std::max(any, all[i].to);
    if (all[i].written) written = std::max(written, all[i].to);
  }
  if (all != few) free(all);
  return once ? LF_OK : LF_ERR_SHAPE;
}

}  // namespace

// One chunk to a thread as far as 256 threads go (4680 rows, us, with one and with three: of 1536 14.3 and 15.9, of 2048 16.4 and 22.8), then three, which
// four wavefronts hold up to 6144 channels, then two of sixteen.
int lf_norm_fwd_rows(const lf_norm_shape* s, lf_norm_lay* lay) {
  const int chunks = s->channels / 8;
  *lay = lf_lay_norm(s->channels, chunks <= 256 ? 1 : chunks <= 768 ? 3 : 2);
  const int64_t blocks = 256 * 64 / (lay->threads / 64);
  return (int)((s->tokens - 1) / blocks + 1);
}

lf_norm_slots lf_norm_bwd_slots(const lf_norm_shape* s) {
  const int chunks = s->channels / 8;
  lf_norm_slots n;
  n.waves = chunks <= 192;
  n.lay = lf_lay_norm(s->channels, n.waves ? (chunks + 63) / 64 : chunks <= 768 ? 3 : 2);
  // As many slots as the chip has room for at once: with two or three chunks to a thread a SIMD holds one wavefront (4680 rows of 1536: 40 us, two slots
  // of a wavefront each 50); with one it holds more, and two keep the sums of the slots few (8000 rows of 512, both launches, with one, two and three: 26.9,
  // 27.4 and 30.1 us; 32 760 rows 71.8, 65.6 and 65.9).  Wavefronts with rows of their own up to 1536 channels (4680 rows: a row for all four 45 us).
  const int waves = n.lay.threads / 64;
  const int64_t at_once = 256 * (n.waves ? (n.lay.nc == 1 ? 2 : 1) : n.lay.nc == 3 ? 4 / waves : 1);
  if (s->group_len > 0) {
    const int64_t each = at_once / s->groups > 1 ? at_once / s->groups : 1;      // slots of a group
    n.rows = (int)((s->group_len - 1) / each + 1);
    if (n.waves && n.rows < 4) n.rows = 4;
    if (n.rows > s->group_len) n.rows = s->group_len;
    n.per_group = (s->group_len - 1) / n.rows + 1;
    n.slots = (int64_t)n.per_group * s->groups;
  } else {
    n.per_group = 0;
    n.rows = (int)((s->tokens - 1) / (at_once > 2 * s->groups ? at_once - s->groups : at_once / 2) + 1);
    if (n.waves && n.rows < 4) n.rows = 4;
    n.slots = (int64_t)s->tokens / n.rows + s->groups;
  }
  n.floats = (n.slots * 3 + (int64_t)s->groups * 2) * s->channels;
  return n;
}

extern "C" int lf_gate_norm(const void* X, const void* B, const float* gate, const float* post_weight, const float* weight, const float* scale,
                            const float* shift, const int32_t* starts, const lf_norm_shape* s, void* Xout, void* Y, void* stream) {
  if (!s || !X || !Y || (B && !Xout) || (!B && (gate || post_weight))) return LF_ERR_NULL;
  int rc = check_norm(s);
  if (rc != LF_OK) return rc;
  if (s->group_len == 0 && !starts) return LF_ERR_NULL;
  const int all[7] = {check_rows(s, s->x_stride), B ? check_rows(s, s->xo_stride) : LF_OK, B ? check_rows(s, s->b_stride) : LF_OK, check_rows(s, s->y_stride),
                      check_table(s, gate, s->gate_stride), check_table(s, scale, s->scale_stride), check_table(s, shift, s->shift_stride)};
  if ((rc = first_error(all, 7)) != LF_OK) return rc;
  const void* wide[9] = {X, B, gate, post_weight, weight, scale, shift, Xout, Y};
  for (const void* p : wide)
    if (misaligned(p, 16)) return LF_ERR_ALIGN;
  if (misaligned(starts, 4)) return LF_ERR_ALIGN;
  lf_norm_call c;
  memset(&c, 0, sizeof c);
  c.s = s;
  c.X = X; c.B = B; c.gate = gate; c.post_weight = post_weight; c.weight = weight; c.scale = scale; c.shift = shift;
  c.starts = starts; c.Xout = Xout; c.Y = Y;
  return lf_launch_gate_norm(&c, stream);
}

extern "C" size_t lf_gate_norm_bwd_workspace_bytes(const lf_norm_shape* s) {
  if (!s || check_norm(s) != LF_OK || check_slots(s) != LF_OK) return 0;
  const lf_norm_shape f = filled(s);
  return (size_t)lf_norm_bwd_slots(&f).floats * sizeof(float);
}

extern "C" int lf_gate_norm_bwd(const void* Xout, const void* B, const float* gate, const float* post_weight, const float* weight, const float* scale,
                                const int32_t* starts, const lf_norm_shape* s, const void* dY, const void* dXout, void* dX, void* dB, float* dgate,
                                float* dpost_weight, float* dweight, float* dscale, float* dshift, void* workspace, size_t workspace_bytes, void* stream) {
  if (!s || !Xout || !dX || (!B) != (!dB) || (!B && (gate || post_weight || dgate || dpost_weight))) return LF_ERR_NULL;
  if ((dpost_weight && !post_weight) || (dweight && !weight)) return LF_ERR_NULL;
  int rc = check_norm(s);
  if (rc != LF_OK) return rc;
  if ((rc = check_slots(s)) != LF_OK) return rc;
  if (s->group_len == 0 && !starts) return LF_ERR_NULL;
  const int all[5] = {check_rows(s, s->xo_stride), B ? check_rows(s, s->b_stride) : LF_OK, dY ? check_rows(s, s->y_stride) : LF_OK,
                      check_table(s, gate, s->gate_stride), check_table(s, scale, s->scale_stride)};
  if ((rc = first_error(all, 5)) != LF_OK) return rc;
  if (!workspace || workspace_bytes < lf_gate_norm_bwd_workspace_bytes(s)) return LF_ERR_WORKSPACE;
  const void* wide[15] = {Xout, B, gate, post_weight, weight, scale, dY, dXout, dX, dB, dgate, dpost_weight, dweight, dscale, dshift};
  for (const void* p : wide)
    if (misaligned(p, 16)) return LF_ERR_ALIGN;
  if (misaligned(starts, 4) || misaligned(workspace, 256)) return LF_ERR_ALIGN;
  lf_norm_call c;
  memset(&c, 0, sizeof c);
  const lf_norm_shape f = filled(s);
  c.s = &f;
  c.groups = s->groups;
  c.Xout = const_cast<void*>(Xout); c.B = B; c.gate = gate; c.post_weight = post_weight; c.weight = weight; c.scale = scale;
  c.starts = starts; c.dY = dY; c.dXout = dXout; c.dX = dX; c.dB = dB;
  c.dgate = dgate; c.dpost_weight = dpost_weight; c.dweight = dweight; c.dscale = dscale; c.dshift = dshift;
  c.workspace = (float*)workspace;
  return lf_launch_gate_norm_bwd(&c, stream);
}

// Tiles of 16 or 32 rows where sequences have 32 rows of a head or fewer in the mean (us, with them and with tiles of 128: 16 sequences of 7500
// tokens, 40 heads on 8 of 128, 32 rows each 225 and 254, 48 rows 308 and 294; 8 heads of 64, 600 tokens, 32 rows 21 and 31, 48 rows 33 and 32).  16
// rows and heads as 16: 110 us, as 32 113 (64 sequences of 4000 tokens, 8 heads to one); 24 of them as 32 122, as twice 16 185.
// The tokens of a tile are divided among workgroups as long as the chip holds them all at once.  Of few rows a compute unit holds one: 256 for one
// sequence (a row of 12 heads over 32 760 tokens 37 us, with 384 39, with 512 40), and half as many again for several, of which some are shorter than
// they are taken to be (16 rows over 120 003 tokens, 40 heads on 8: sequences of uneven lengths 95 us, with 256 115, with 512 104, with 768 102; of equal ones 95, 91,
// 97 and 103).  Of 128 rows it holds two (12 heads, 1536 rows over 8192 tokens: 101 us, with one 207, with three 112).
// None has fewer than 512 tokens (12 heads, 512 rows over 2048 tokens: 24.0 us, with 256 27.6; 24 rows over 12 000 tokens 21.2 and 25.1), the few rows of one sequence
// 256 (40 heads on 8, 4096 tokens: 10.1 us, with 512 11.5, with 1024 13.8).  512 tokens stay together, and sequences of 256 in the mean.
lf_packed_plan lf_plan_packed(const lf_packed_shape* s) {
  lf_packed_plan p;
  const int64_t group = s->heads / s->kv_heads, rows = (int64_t)s->q_len * group;
  p.few = s->q_len <= (int64_t)32 * s->seqs;
  int64_t tiles, want;
  if (p.few) {
    p.tile = rows <= (int64_t)16 * s->seqs ? 16 : 32;
    p.slots = rows / p.tile + s->seqs;
    const int64_t full = (rows + p.tile - 1) / p.tile, some = s->q_len < s->seqs ? s->q_len : s->seqs;
    tiles = (full > some ? full : some) * s->kv_heads;
    want = s->seqs == 1 ? 256 : 384;
  } else {
    p.tile = 128;
    p.slots = (int64_t)s->q_len / p.tile + s->seqs;
    tiles = ((int64_t)s->q_len + p.tile - 1) / p.tile * s->heads;
    want = tiles <= 256 ? 512 : 1;
  }
  if (tiles < 1) tiles = 1;
  const int64_t mean = (int64_t)s->kv_len / s->seqs, least = p.few && s->seqs == 1 ? 256 : 512, per = want > tiles ? want / tiles : 1;
  int64_t each = want > 1 ? ((mean + per - 1) / per + 63) / 64 * 64 : (int64_t)1 << 30;
  if (each < least) each = least;
  if (each > 1 << 30) each = 1 << 30;
  // the longest sequence is taken to be four times the mean one
  const int64_t longest = s->kv_len < 4 * mean ? s->kv_len : 4 * mean;
  int64_t parts = (longest + each - 1) / each;
  if ((s->seqs == 1 ? longest : 2 * mean) <= 512 || s->q_len == 0) parts = 1;
  if (parts < 1) parts = 1;
  if (parts > LF_PACKED_MAX_PARTS) parts = LF_PACKED_MAX_PARTS;
  p.parts = (int)parts;
  p.part_tokens = (int)each;
  const int64_t states = p.slots * (p.few ? s->kv_heads : s->heads) * p.parts * p.tile;
  p.state_bytes = p.parts == 1 ? 0 : states * (s->head_dim + 2) * 4;
  return p;
}

extern "C" size_t lf_packed_attn_workspace_bytes(const lf_packed_shape* s) {
  if (!s || check_sizes(s) != LF_OK) return 0;
  return (size_t)lf_plan_packed(s).state_bytes;
}

extern "C" int lf_packed_attn(const void* Q, const void* K, const void* V, const lf_packed_shape* s, const int32_t* q_start, const int32_t* kv_start,
                              float softmax_scale, void* O, float* lse2, void* workspace, size_t workspace_bytes, void* stream) {
  if (!s || !q_start || !kv_start) return LF_ERR_NULL;
  const int rc = check_packed(s);
  if (rc != LF_OK) return rc;
  if ((s->q_len > 0 && (!Q || !O)) || (s->kv_len > 0 && (!K || !V))) return LF_ERR_NULL;
  if (!scale_ok(softmax_scale) || heads_overlap(s->heads, s->o_stride_head, s->q_len, s->o_stride_tok, s->head_dim)) return LF_ERR_SHAPE;
  const size_t need = lf_packed_attn_workspace_bytes(s);
  if (need > 0 && (!workspace || workspace_bytes < need)) return LF_ERR_WORKSPACE;
  if (misaligned(Q, 16) || misaligned(K, 16) || misaligned(V, 16) || misaligned(O, 16) || misaligned(lse2, 4) || misaligned(q_start, 4) ||
      misaligned(kv_start, 4) || (need > 0 && misaligned(workspace, 256)))
    return LF_ERR_ALIGN;
  if (s->q_len == 0) return LF_OK;
  lf_packed_call c;
  memset(&c, 0, sizeof c);
  c.s = s;
  c.plan = lf_plan_packed(s);
  c.Q = Q; c.K = K; c.V = V; c.O = O; c.lse2 = lse2;
  c.q_start = q_start; c.kv_start = kv_start;
  c.scale = scale_or_default(softmax_scale, s->head_dim);
  c.workspace = workspace;
  return lf_launch_packed_attn(&c, stream);
}

extern "C" size_t lf_packed_attn_bwd_workspace_bytes(const lf_packed_shape* s) {
  if (!s || check_sizes(s) != LF_OK) return 0;
  return (size_t)s->heads * s->q_len * 2 * sizeof(float);
}

extern "C" int lf_packed_attn_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* lse2, const lf_packed_shape* s,
                                  const int32_t* q_start, const int32_t* kv_start, float softmax_scale, void* dQ, void* dK, void* dV, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  if (!s || !q_start || !kv_start) return LF_ERR_NULL;
  const int rc = check_packed(s);
  if (rc != LF_OK) return rc;
  if ((s->q_len > 0 && (!Q || !O || !dO || !lse2 || !dQ)) || (s->kv_len > 0 && (!K || !V || !dK || !dV))) return LF_ERR_NULL;
  if (!scale_ok(softmax_scale) || heads_overlap(s->heads, s->q_stride_head, s->q_len, s->q_stride_tok, s->head_dim) ||
      heads_overlap(s->kv_heads, s->k_stride_head, s->kv_len, s->k_stride_tok, s->head_dim) ||
      heads_overlap(s->kv_heads, s->v_stride_head, s->kv_len, s->v_stride_tok, s->head_dim))
    return LF_ERR_SHAPE;
  const size_t need = lf_packed_attn_bwd_workspace_bytes(s);
  if (need > 0 && (!workspace || workspace_bytes < need)) return LF_ERR_WORKSPACE;
  const void* wide[8] = {Q, K, V, O, dO, dQ, dK, dV};
  for (const void* p : wide)
    if (misaligned(p, 16)) return LF_ERR_ALIGN;
  if (misaligned(lse2, 4) || misaligned(q_start, 4) || misaligned(kv_start, 4) || (need > 0 && misaligned(workspace, 256))) return LF_ERR_ALIGN;
  lf_packed_call c;
  memset(&c, 0, sizeof c);
  c.s = s;
  c.plan = lf_plan_packed(s);
  c.Q = Q; c.K = K; c.V = V; c.O = const_cast<void*>(O); c.dO = dO; c.lse2 = const_cast<float*>(lse2);
  c.dQ = dQ; c.dK = dK; c.dV = dV;
  c.q_start = q_start; c.kv_start = kv_start;
  c.scale = scale_or_default(softmax_scale, s->head_dim);
  c.workspace = workspace;
  return lf_launch_packed_bwd(&c, stream);
}

// ---- gradient clipping ----

extern "C" size_t lf_grad_workspace_bytes(int32_t count, int64_t numel) {
  if (count < 0 || count > 1 << 20 || numel < 0 || numel > (int64_t)1 << 40) return 0;
  return (size_t)(lf_grad_most_chunks(count, numel) + 1) * sizeof(double);
}

extern "C" int lf_grad_clip(const lf_grad_tensor* t, int32_t count, float max_norm, float eps, float* norm, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if ((count > 0 && !t) || !norm) return LF_ERR_NULL;
  if (count < 0 || count > 1 << 20 || !(max_norm >= 0.0f) || !(eps >= 0.0f) || isinf(eps)) return LF_ERR_SHAPE;
  int64_t numel = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (t[i].numel < 0 || t[i].numel > (int64_t)1 << 40) return LF_ERR_SHAPE;
    numel += t[i].numel;
    if (numel > (int64_t)1 << 40) return LF_ERR_SHAPE;
  }
  for (int32_t i = 0; i < count; ++i) {
    if (t[i].numel == 0) continue;
    if (!t[i].data) return LF_ERR_NULL;
    if ((t[i].dtype != LF_BF16 && t[i].dtype != LF_F32) || (t[i].out && t[i].out_dtype != LF_BF16 && t[i].out_dtype != LF_F32)) return LF_ERR_DTYPE;
    if (t[i].out == t[i].data && t[i].out_dtype != t[i].dtype) return LF_ERR_DTYPE;
    if (misaligned(t[i].data, t[i].dtype == LF_F32 ? 4 : 2) || (t[i].out && misaligned(t[i].out, t[i].out_dtype == LF_F32 ? 4 : 2))) return LF_ERR_ALIGN;
  }
  const int rc = written_once(t, count, isinf(max_norm));
  if (rc != LF_OK) return rc;
  if (!workspace || workspace_bytes < lf_grad_workspace_bytes(count, numel)) return LF_ERR_WORKSPACE;
  if (misaligned(norm, 4) || misaligned(workspace, 256)) return LF_ERR_ALIGN;
  return lf_launch_grad_clip(t, count, numel, max_norm, eps, norm, (double*)workspace, stream);
}
