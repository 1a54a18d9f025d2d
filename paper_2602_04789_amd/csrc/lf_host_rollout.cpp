// Host side of the three-axis producer and of the 4-bit cache: validation and sizes.  No GPU code here.
#include <math.h>
#include <string.h>

#include "lf_rollout.h"

namespace {

bool misaligned(const void* p, size_t a) { return ((uintptr_t)p % a) != 0; }

// A token stride of a row tensor: rows must not overlap, every row 16-byte aligned.
int check_strides(const int64_t* tok_head, int n, int64_t width) {
  for (int i = 0; i < n; ++i) {
    if (tok_head[2 * i] < width || tok_head[2 * i + 1] < 0) return LF_ERR_SHAPE;
    if (tok_head[2 * i] % 8 || tok_head[2 * i + 1] % 8) return LF_ERR_ALIGN;
  }
  return LF_OK;
}

// Whether rows of two heads share an element, in a tensor that is written: head h's token t takes [h stride_head + t stride_tok, .. + d).  One
// head's tokens lie apart (stride_tok >= d).  Layouts with one axis inside a step of the other are seen at once.
bool heads_overlap(int heads, int64_t stride_head, int tokens, int64_t stride_tok, int d) {
  if (heads < 2) return false;
  if (stride_head < d) return true;
  if (tokens < 2 || (stride_head - d) / stride_tok >= tokens - 1 || (stride_tok - d) / stride_head >= heads - 1) return false;
  for (int h = 1; h < heads; ++h) {             // heads h apart, and the tokens on both sides of where the later one begins
    const __int128 off = (__int128)h * stride_head, t = off / stride_tok, past = off - t * stride_tok;
    if (t < tokens && past < d) return true;
    if (t + 1 < tokens && stride_tok - past < d) return true;
  }
  return false;
}

bool scale_ok(float s) { return s >= 0.0f && !isinf(s); }
float scale_or_default(float s, int d) { return s > 0.0f ? s : 1.0f / sqrtf((float)d); }

int check_axes(const lf_axes_shape* p) {
  if (p->head_dim != 64 && p->head_dim != 128) return LF_ERR_SHAPE;
  if (p->heads < 1 || p->heads > LF_AXES_MAX_CHANNELS / p->head_dim) return LF_ERR_SHAPE;
  if (p->tokens < 1 || p->tokens > 1 << 30) return LF_ERR_SHAPE;
  if ((p->across_heads != 0 && p->across_heads != 1) || (p->pairing != 0 && p->pairing != 1)) return LF_ERR_SHAPE;
  int64_t pairs = 0;
  for (int i = 0; i < 3; ++i) {
    if (p->pairs[i] < 0) return LF_ERR_SHAPE;
    pairs += p->pairs[i];
  }
  if (pairs != p->head_dim / 2) return LF_ERR_SHAPE;
  if (!(p->eps >= 0.0f) || isinf(p->eps)) return LF_ERR_SHAPE;
  if (p->x_stride_tok < (int64_t)p->heads * p->head_dim || p->y_stride_tok < p->head_dim || p->y_stride_head < 0) return LF_ERR_SHAPE;
  if (p->x_stride_tok % 8 || p->y_stride_tok % 8 || p->y_stride_head % 8) return LF_ERR_ALIGN;
  const lf_axes_lay l = lf_lay_axes_fwd(p->heads, p->head_dim, p->tokens);       // a grid has less than 2^32 threads
  return ((int64_t)(p->tokens - 1) / l.tt + 1) * l.threads < (int64_t)1 << 32 ? LF_OK : LF_ERR_SHAPE;
}

bool axes_misaligned(const void* X, const float* g, const int32_t* pos, const double* freq) {
  return misaligned(X, 16) || misaligned(g, 16) || misaligned(pos, 4) || misaligned(freq, 8);
}

constexpr int kMaxCapacity = 1 << 24;   // tokens: codes of a head within 32-bit offsets
constexpr int kMaxHeads = 32767;        // the store's grid has a row for K and one for V of every head
constexpr int64_t kMaxBlocks = 1 << 22; // (head, query block) pairs of a launch

int check_cache(const lf_kvq_shape* s) {
  if (s->head_dim != 64 && s->head_dim != 128) return LF_ERR_SHAPE;
  if (s->heads < 1 || s->heads > kMaxHeads || s->capacity < 1 || s->capacity > kMaxCapacity) return LF_ERR_SHAPE;
  return LF_OK;
}

int check_rows(const lf_kvq_shape* s, const lf_kvq_rows* r) {
  if (r->first < 0 || r->tokens < 0 || (int64_t)r->first + r->tokens > s->capacity) return LF_ERR_SHAPE;
  const int64_t st[4] = {r->k_stride_tok, r->k_stride_head, r->v_stride_tok, r->v_stride_head};
  return check_strides(st, 2, s->head_dim);
}

// What the two attention calls share.
int check_call(const void* Q, const void* cache, size_t cache_bytes, const lf_kvq_shape* cs, const void* K, const void* V, float scale,
               const void* O, int heads, int d, int64_t cached) {
  int rc = check_cache(cs);
  if (rc != LF_OK) return rc;
  if (cs->heads != heads || cs->head_dim != d || cached > cs->capacity) return LF_ERR_SHAPE;
  if (!scale_ok(scale)) return LF_ERR_SHAPE;
  if (!cache || cache_bytes < (size_t)lf_kvq_layout(*cs).bytes) return LF_ERR_WORKSPACE;
  if (misaligned(Q, 16) || misaligned(K, 16) || misaligned(V, 16) || misaligned(O, 16) || misaligned(cache, 256)) return LF_ERR_ALIGN;
  return LF_OK;
}

int check_token(const lf_token_shape* s) {
  if (s->head_dim != 64 && s->head_dim != 128) return LF_ERR_SHAPE;
  if (s->heads < 1 || s->heads > kMaxHeads || s->q_len < 1 || s->q_len > 64) return LF_ERR_SHAPE;
  if (s->cached_len < 0 || s->cached_len > kMaxCapacity || s->extra_len < 0 || s->extra_len > kMaxCapacity) return LF_ERR_SHAPE;
  const int64_t st[8] = {s->q_stride_tok, s->q_stride_head, s->o_stride_tok, s->o_stride_head,
                         s->k_stride_tok, s->k_stride_head, s->v_stride_tok, s->v_stride_head};
  return check_strides(st, s->extra_len > 0 ? 4 : 2, s->head_dim);
}

int token_parts(const lf_token_shape* s) {
  return lf_kvq_parts_of(s->heads, ((int64_t)s->cached_len + 63) / 64 + ((int64_t)s->extra_len + 63) / 64, s->q_len);
}

// The call's sizes, its strides apart: those of K and V are asked for only where there are K and V.
int check_lists(const lf_shape* s, int32_t list_len, lf_dims* dm) {
  if (!s) return LF_ERR_NULL;
  lf_shape plain = *s;
  plain.k_stride_tok = plain.v_stride_tok = s->head_dim;
  plain.k_stride_head = plain.v_stride_head = 0;
  const int rc = lf_derive(&plain, nullptr, dm);
  if (rc != LF_OK) return rc;
  if ((int64_t)dm->H * dm->n_q > kMaxBlocks) return LF_ERR_SHAPE;
  return list_len < 1 || list_len > 1 << 30 ? LF_ERR_BUDGET : LF_OK;      // (a walk along a list steps past its end)
}

// K or V of all tokens in bfloat16, padded to 256 bytes.
size_t expanded_bytes(const lf_dims& dm) { return ((size_t)dm.H * dm.F * dm.n * dm.d * 2 + 255) / 256 * 256; }

int list_rows(const lf_dims& dm) { return dm.n < 64 ? dm.n : 64; }

}  // namespace

extern "C" int lf_qk_norm_rope_axes(const void* X, const float* g, const int32_t* pos, const double* freq, const lf_axes_shape* p,
                                    void* Y, void* stream) {
  if (!X || !g || !pos || !freq || !p || !Y) return LF_ERR_NULL;
  const int rc = check_axes(p);
  if (rc != LF_OK) return rc;
  if (heads_overlap(p->heads, p->y_stride_head, p->tokens, p->y_stride_tok, p->head_dim)) return LF_ERR_SHAPE;
  if (axes_misaligned(X, g, pos, freq) || misaligned(Y, 16)) return LF_ERR_ALIGN;
  return lf_launch_rope_axes(X, g, pos, freq, p, Y, stream);
}

extern "C" size_t lf_qk_norm_rope_axes_bwd_workspace_bytes(const lf_axes_shape* p) {
  if (!p || check_axes(p) != LF_OK) return 0;
  return (size_t)lf_axes_bwd_blocks(p->heads, p->head_dim, p->tokens) * p->heads * p->head_dim * sizeof(float);
}

extern "C" int lf_qk_norm_rope_axes_bwd(const void* X, const float* g, const int32_t* pos, const double* freq, const lf_axes_shape* p,
                                        const void* dY, void* dX, float* dg, void* workspace, size_t workspace_bytes, void* stream) {
  if (!X || !g || !pos || !freq || !p || !dY || !dX || !dg) return LF_ERR_NULL;
  const int rc = check_axes(p);
  if (rc != LF_OK) return rc;
  if (!workspace || workspace_bytes < lf_qk_norm_rope_axes_bwd_workspace_bytes(p)) return LF_ERR_WORKSPACE;
  if (axes_misaligned(X, g, pos, freq) || misaligned(dY, 16) || misaligned(dX, 16) || misaligned(dg, 4) || misaligned(workspace, 256))
    return LF_ERR_ALIGN;
  return lf_launch_rope_axes_bwd(X, g, pos, freq, p, dY, dX, dg, (float*)workspace, stream);
}

extern "C" size_t lf_kvq_bytes(const lf_kvq_shape* s) {
  if (!s || check_cache(s) != LF_OK) return 0;
  return (size_t)lf_kvq_layout(*s).bytes;
}

extern "C" int lf_kvq_append(const void* K, const void* V, const lf_kvq_shape* s, const lf_kvq_rows* r, void* cache, size_t cache_bytes,
                             void* stream) {
  if (!s || !r || (r->tokens != 0 && (!K || !V))) return LF_ERR_NULL;
  int rc = check_cache(s);
  if (rc != LF_OK) return rc;
  if ((rc = check_rows(s, r)) != LF_OK) return rc;
  if (!cache || cache_bytes < lf_kvq_bytes(s)) return LF_ERR_WORKSPACE;
  if (misaligned(K, 16) || misaligned(V, 16) || misaligned(cache, 256)) return LF_ERR_ALIGN;
  return r->tokens == 0 ? LF_OK : lf_launch_kvq_append(K, V, s, r, (uint8_t*)cache, stream);
}

extern "C" int lf_kvq_read(const void* cache, size_t cache_bytes, const lf_kvq_shape* s, const lf_kvq_rows* r, void* K, void* V,
                           void* stream) {
  if (!s || !r || (r->tokens != 0 && (!K || !V))) return LF_ERR_NULL;
  int rc = check_cache(s);
  if (rc != LF_OK) return rc;
  if ((rc = check_rows(s, r)) != LF_OK) return rc;
  if (heads_overlap(s->heads, r->k_stride_head, r->tokens, r->k_stride_tok, s->head_dim) ||
      heads_overlap(s->heads, r->v_stride_head, r->tokens, r->v_stride_tok, s->head_dim))
    return LF_ERR_SHAPE;
  if (!cache || cache_bytes < lf_kvq_bytes(s)) return LF_ERR_WORKSPACE;
  if (misaligned(K, 16) || misaligned(V, 16) || misaligned(cache, 256)) return LF_ERR_ALIGN;
  return r->tokens == 0 ? LF_OK : lf_launch_kvq_read((const uint8_t*)cache, s, r, K, V, stream);
}

extern "C" size_t lf_sparse_attn_kvq_workspace_bytes(const lf_shape* s, int32_t list_len) {
  lf_dims dm;
  if (check_lists(s, list_len, &dm) != LF_OK) return 0;
  const int64_t blocks = (int64_t)dm.H * dm.n_q;
  if (lf_kvq_expands(dm.d, blocks, list_len, list_rows(dm), dm.H, s->kv_len)) return 2 * expanded_bytes(dm);
  return (size_t)lf_kvq_state_bytes(blocks, lf_kvq_parts_of(blocks, list_len, list_rows(dm)), list_rows(dm), dm.d);
}

extern "C" int lf_sparse_attn_kvq(const void* Q, const void* cache, size_t cache_bytes, const lf_kvq_shape* cs, const void* K,
                                  const void* V, const lf_shape* s, const int32_t* indices, int32_t list_len, float softmax_scale,
                                  void* O, void* workspace, size_t workspace_bytes, void* stream) {
  if (!Q || !cs || !s || !indices || !O || (!K) != (!V)) return LF_ERR_NULL;
  lf_dims dm;
  int rc = check_lists(s, list_len, &dm);
  if (rc != LF_OK) return rc;
  if (heads_overlap(s->heads, s->o_stride_head, s->q_len, s->o_stride_tok, s->head_dim)) return LF_ERR_SHAPE;
  if (K) {
    const int64_t st[4] = {s->k_stride_tok, s->k_stride_head, s->v_stride_tok, s->v_stride_head};
    if ((rc = check_strides(st, 2, s->head_dim)) != LF_OK) return rc;
  }
  const int cached = K ? s->kv_len - s->q_len : s->kv_len;
  if ((rc = check_call(Q, cache, cache_bytes, cs, K, V, softmax_scale, O, s->heads, s->head_dim, cached)) != LF_OK) return rc;
  if (misaligned(indices, 4)) return LF_ERR_ALIGN;
  const size_t need = lf_sparse_attn_kvq_workspace_bytes(s, list_len);
  if (need > 0 && (!workspace || workspace_bytes < need)) return LF_ERR_WORKSPACE;
  if (need > 0 && misaligned(workspace, 256)) return LF_ERR_ALIGN;
  lf_kvq_call c;
  memset(&c, 0, sizeof c);
  c.Q = Q; c.K = K; c.V = V; c.O = O;
  c.cache = (const uint8_t*)cache;
  c.cs = *cs;
  c.H = dm.H; c.d = dm.d; c.q_len = s->q_len;
  c.q_stride_tok = s->q_stride_tok; c.q_stride_head = s->q_stride_head;
  c.k_stride_tok = s->k_stride_tok; c.k_stride_head = s->k_stride_head;
  c.v_stride_tok = s->v_stride_tok; c.v_stride_head = s->v_stride_head;
  c.o_stride_tok = s->o_stride_tok; c.o_stride_head = s->o_stride_head;
  c.scale = scale_or_default(softmax_scale, dm.d);
  c.indices = indices;
  c.list_len = list_len;
  c.n = dm.n; c.nb = dm.nb; c.n_q = dm.n_q; c.n_k = dm.n_k;
  c.cached = cached;
  c.extra = s->kv_len - cached;
  c.rows = list_rows(dm);
  const int64_t blocks = (int64_t)dm.H * dm.n_q;
  if (lf_kvq_expands(dm.d, blocks, list_len, list_rows(dm), dm.H, s->kv_len)) {
    uint16_t *Kw = (uint16_t*)workspace, *Vw = (uint16_t*)((char*)workspace + expanded_bytes(dm));
    if ((rc = lf_launch_kvq_expand(&c, Kw, Vw, stream)) != LF_OK) return rc;
    lf_shape t = *s;
    t.k_stride_tok = t.v_stride_tok = dm.d;
    t.k_stride_head = t.v_stride_head = (int64_t)s->kv_len * dm.d;
    return lf_launch_attn(Q, Kw, Vw, &t, &dm, indices, list_len, list_len, c.scale, O, nullptr, nullptr, nullptr, stream);
  }
  c.parts = lf_kvq_parts_of(blocks, list_len, c.rows);
  c.workspace = workspace;
  return lf_launch_kvq_attn(&c, stream);
}

extern "C" size_t lf_token_attn_kvq_workspace_bytes(const lf_token_shape* s) {
  if (!s || check_token(s) != LF_OK) return 0;
  return (size_t)lf_kvq_state_bytes(s->heads, token_parts(s), s->q_len, s->head_dim);
}

extern "C" int lf_token_attn_kvq(const void* Q, const void* cache, size_t cache_bytes, const lf_kvq_shape* cs, const void* K,
                                 const void* V, const lf_token_shape* s, float softmax_scale, void* O, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  if (!Q || !cs || !s || !O) return LF_ERR_NULL;
  int rc = check_token(s);
  if (rc != LF_OK) return rc;
  if (s->extra_len == 0) K = V = nullptr;
  else if (!K || !V) return LF_ERR_NULL;
  if (heads_overlap(s->heads, s->o_stride_head, s->q_len, s->o_stride_tok, s->head_dim)) return LF_ERR_SHAPE;
  if ((rc = check_call(Q, cache, cache_bytes, cs, K, V, softmax_scale, O, s->heads, s->head_dim, s->cached_len)) != LF_OK) return rc;
  const size_t need = lf_token_attn_kvq_workspace_bytes(s);
  if (need > 0 && (!workspace || workspace_bytes < need)) return LF_ERR_WORKSPACE;
  if (need > 0 && misaligned(workspace, 256)) return LF_ERR_ALIGN;
  lf_kvq_call c;
  memset(&c, 0, sizeof c);
  c.Q = Q; c.K = K; c.V = V; c.O = O;
  c.cache = (const uint8_t*)cache;
  c.cs = *cs;
  c.H = s->heads; c.d = s->head_dim; c.q_len = s->q_len;
  c.q_stride_tok = s->q_stride_tok; c.q_stride_head = s->q_stride_head;
  c.k_stride_tok = s->k_stride_tok; c.k_stride_head = s->k_stride_head;
  c.v_stride_tok = s->v_stride_tok; c.v_stride_head = s->v_stride_head;
  c.o_stride_tok = s->o_stride_tok; c.o_stride_head = s->o_stride_head;
  c.scale = scale_or_default(softmax_scale, s->head_dim);
  c.n = c.nb = c.n_q = c.n_k = 1;
  c.cached = s->cached_len;
  c.extra = s->extra_len;
  c.rows = s->q_len;
  c.parts = token_parts(s);
  c.workspace = workspace;
  return lf_launch_kvq_attn(&c, stream);
}
