// Host-only driver for the sanitizer build of the rollout's host side: every entry point on sizes drawn from small ones, the limits and the
// ends of their types, the kernel launchers replaced by ones that check what reaches them.  Pointers are never dereferenced here.
#include <stdio.h>
#include <string.h>

#include "lf_rollout.h"

static int g_fail = 0, g_launches = 0;
#define EXPECT(cond) do { if (!(cond)) { printf("FAILED line %d: %s\n", __LINE__, #cond); ++g_fail; } } while (0)

int lf_launch_select(const void*, const void*, const lf_shape*, const lf_budget*, const lf_dims*, int32_t*, void*, void*) { return LF_OK; }
int lf_launch_kcache_update(const void*, const lf_shape*, const lf_dims*, int, int, int, void*, void*) { return LF_OK; }
int lf_launch_select_cached(const void*, const void*, void*, int, const lf_shape*, const lf_budget*, const lf_dims*, int32_t*, void*, void*) { return LF_OK; }
int lf_launch_attn_bwd(const void*, const void*, const void*, const void*, const void*, const float*, const lf_shape*, const lf_dims*, const int32_t*,
                       int32_t, float, void*, void*, void*, float*, int32_t*, int32_t*, int32_t*, void*) { return LF_OK; }
int lf_launch_attn_dense(const void*, const void*, const void*, const lf_shape*, const lf_dims*, int, int, float, float*, float*, void*) { return LF_OK; }
int lf_launch_qk_norm_rope(const void*, const float*, const float*, const float*, const lf_producer_shape*, void*, void*) { return LF_OK; }
int lf_static_scratch(void** p) { *p = (void*)0x20000; return LF_OK; }

static size_t g_need = 0;      // the workspace that the caller has
int lf_launch_attn(const void*, const void* K, const void* V, const lf_shape* s, const lf_dims* dm, const int32_t*, int32_t list_len, int32_t, float scale,
                   void*, const float*, const float*, float*, void*) {
  ++g_launches;
  EXPECT(list_len >= 1 && scale > 0.0f && s->k_stride_tok == dm->d && s->k_stride_head == (int64_t)s->kv_len * dm->d);
  EXPECT((size_t)((const char*)V - (const char*)K) >= (size_t)dm->H * s->kv_len * dm->d * 2 && ((uintptr_t)V & 255) == 0);
  EXPECT((size_t)((const char*)V - (const char*)K) * 2 <= g_need);
  return LF_OK;
}
static void check_lay(const lf_axes_lay& l, const lf_axes_shape* p) {
  const int ch = p->head_dim / 8;
  EXPECT(l.ni == 1 || l.ni == 2 || l.ni == 4);
  EXPECT(l.hpt * l.ni >= p->heads && l.tt >= 1 && l.tt * l.hpt * ch <= l.threads && l.threads <= 512 && l.threads % 64 == 0);
}
int lf_launch_rope_axes(const void*, const float*, const int32_t*, const double*, const lf_axes_shape* p, void*, void*) {
  ++g_launches;
  check_lay(lf_lay_axes_fwd(p->heads, p->head_dim, p->tokens), p);
  return LF_OK;
}
int lf_launch_rope_axes_bwd(const void*, const float*, const int32_t*, const double*, const lf_axes_shape* p, const void*, void*, float*, float*, void*) {
  ++g_launches;
  const lf_axes_lay l = lf_lay_axes_bwd(p->heads, p->head_dim);
  check_lay(l, p);
  EXPECT((int64_t)l.ni * l.tt * l.hpt * p->head_dim * 4 <= 65536);     // LDS
  const int blocks = lf_axes_bwd_blocks(p->heads, p->head_dim, p->tokens);
  EXPECT(blocks >= 1 && blocks <= LF_AXES_MAX_BLOCKS && (size_t)blocks * p->heads * p->head_dim * 4 <= g_need);
  return LF_OK;
}
int lf_launch_kvq_append(const void*, const void*, const lf_kvq_shape* s, const lf_kvq_rows* r, uint8_t*, void*) {
  ++g_launches;
  EXPECT(r->tokens > 0 && (int64_t)r->first + r->tokens <= s->capacity);
  return LF_OK;
}
int lf_launch_kvq_read(const uint8_t* c, const lf_kvq_shape* s, const lf_kvq_rows* r, void*, void*, void*) {
  return lf_launch_kvq_append(nullptr, nullptr, s, r, const_cast<uint8_t*>(c), nullptr);
}
int lf_launch_kvq_expand(const lf_kvq_call* c, uint16_t*, uint16_t*, void*) {
  EXPECT(c->cached >= 0 && c->cached <= c->cs.capacity && c->extra >= 0 && (c->extra == 0) == (c->K == nullptr));
  return LF_OK;
}
int lf_launch_kvq_attn(const lf_kvq_call* c, void*) {
  ++g_launches;
  const int64_t blocks = (int64_t)c->H * c->n_q;
  EXPECT(c->cached >= 0 && c->cached <= c->cs.capacity && c->extra >= 0 && c->rows >= 1 && c->rows <= 64 && c->scale > 0.0f);
  EXPECT(c->extra == 0 || (c->K && c->V));
  EXPECT(c->parts >= 1 && c->parts <= LF_KVQ_MAX_PARTS && blocks * c->parts * 256 < (int64_t)1 << 32);
  EXPECT((size_t)lf_kvq_state_bytes(blocks, c->parts, c->rows, c->d) <= g_need);
  return LF_OK;
}

static uint64_t g_state = 1;
static uint32_t rnd() { g_state = g_state * 6364136223846793005ull + 1442695040888963407ull; return (uint32_t)(g_state >> 33); }
static int pick(const int* v, int n) { return v[rnd() % n]; }
#define PICK(...) ([] { static const int v[] = {__VA_ARGS__}; return pick(v, (int)(sizeof(v) / sizeof(v[0]))); }())
static int64_t stride() {
  static const int64_t v[] = {64, 128, 128, 128, 5120, 8, 0, -8, 132, INT64_MAX, INT64_MAX / 8 * 8, INT64_MIN, (int64_t)1 << 40};
  return v[rnd() % (sizeof(v) / sizeof(v[0]))];
}

int main() {
  void* const P = (void*)0x10000;
  float* const F = (float*)P;
  const float scales[] = {0.0f, 0.125f, -1.0f, 1e-40f, __builtin_inff(), __builtin_nanf("")};
  int ok = 0;
  for (int i = 0; i < 400000; ++i) {
    const int before = g_launches;
    int rc = 0;
    g_need = 0;
    switch (rnd() % 4) {
      case 0: {
        lf_axes_shape p;
        memset(&p, 0, sizeof p);
        p.heads = PICK(1, 2, 12, 40, 128, 256, 257, 0, -1, INT32_MAX); p.head_dim = PICK(64, 128, 96);
        p.tokens = PICK(1, 7, 4680, 1 << 30, 0, -5, INT32_MAX); p.across_heads = rnd() % 2; p.pairing = PICK(0, 1, 1, 2);
        p.pairs[0] = p.head_dim / 2 - 20; p.pairs[1] = PICK(10, 10, 10, INT32_MAX); p.pairs[2] = 10;
        p.eps = 1e-6f;
        p.x_stride_tok = rnd() % 4 ? (int64_t)p.heads * p.head_dim : stride();
        p.y_stride_tok = rnd() % 4 ? p.head_dim : stride();
        p.y_stride_head = rnd() % 4 ? (int64_t)p.head_dim * 4680 : stride();
        g_need = lf_qk_norm_rope_axes_bwd_workspace_bytes(&p);
        rc = lf_qk_norm_rope_axes(P, F, (int32_t*)P, (double*)P, &p, P, nullptr);
        EXPECT((rc == LF_OK) == (g_launches == before + 1));
        const int again = g_launches;
        const int rb = lf_qk_norm_rope_axes_bwd(P, F, (int32_t*)P, (double*)P, &p, P, P, F, P, g_need, nullptr);
        EXPECT((rb == LF_OK) == (g_launches == again + 1) && (rc != LF_OK || rb == LF_OK) && (rb == LF_OK) == (g_need > 0));
        if (rb == LF_OK) EXPECT(lf_qk_norm_rope_axes_bwd(P, F, (int32_t*)P, (double*)P, &p, P, P, F, P, g_need - 1, nullptr) == LF_ERR_WORKSPACE);
        break;
      }
      case 1: {
        lf_kvq_shape s = {PICK(1, 3, 40, 32767, 32768, 0, -1), PICK(64, 128, 32), PICK(1, 77, 32760, 1 << 24, (1 << 24) + 1, 0, INT32_MAX), 0};
        lf_kvq_rows r = {PICK(0, 0, 5, -1, INT32_MAX), PICK(0, 1, 77, -1, INT32_MAX), 128, 128 * 80, 128, 128 * 80};
        if (rnd() % 3 == 0) r.k_stride_tok = stride();
        if (rnd() % 3 == 0) r.v_stride_head = stride();
        const size_t n = lf_kvq_bytes(&s);
        rc = lf_kvq_append(P, P, &s, &r, P, n, nullptr);
        EXPECT((rc == LF_OK && r.tokens > 0) == (g_launches == before + 1));
        const int again = g_launches, rr = lf_kvq_read(P, n, &s, &r, P, P, nullptr);
        EXPECT((rr == LF_OK && r.tokens > 0) == (g_launches == again + 1));
        break;
      }
      case 2: {
        lf_shape s;
        memset(&s, 0, sizeof s);
        s.heads = PICK(1, 2, 12, 40, 32767, 32768, 0); s.head_dim = PICK(64, 128); s.frame_len = PICK(1, 20, 64, 97, 1560, 0, INT32_MAX);
        s.block = 64; s.dtype = LF_BF16;
        const int64_t q = (int64_t)s.frame_len * PICK(1, 2, 3, 70), kv = q * PICK(1, 2, 7, 400);
        s.q_len = q > INT32_MAX ? INT32_MAX : (int)q; s.kv_len = kv > INT32_MAX ? INT32_MAX : (int)kv;
        s.q_stride_tok = s.k_stride_tok = s.v_stride_tok = s.o_stride_tok = s.head_dim;
        s.q_stride_head = s.k_stride_head = s.v_stride_head = s.o_stride_head = (int64_t)s.head_dim * 8;
        if (rnd() % 4 == 0) s.k_stride_tok = stride();
        if (rnd() % 4 == 0) s.q_stride_tok = stride();
        if (rnd() % 4 == 0) s.o_stride_head = stride();
        lf_kvq_shape cs = {s.heads, s.head_dim, rnd() % 2 ? 1 << 24 : s.kv_len, 0};
        const int list_len = PICK(1, 5, 40, 3000, INT32_MAX, 0, -1), own = rnd() % 2;
        g_need = lf_sparse_attn_kvq_workspace_bytes(&s, list_len);
        rc = lf_sparse_attn_kvq(P, P, lf_kvq_bytes(&cs), &cs, own ? P : nullptr, own ? P : nullptr, &s, (int32_t*)P, list_len, scales[rnd() % 6], P, P,
                                g_need, nullptr);
        EXPECT((rc == LF_OK) == (g_launches == before + 1));
        if (rc == LF_OK && g_need > 0)
          EXPECT(lf_sparse_attn_kvq(P, P, lf_kvq_bytes(&cs), &cs, own ? P : nullptr, own ? P : nullptr, &s, (int32_t*)P, list_len, 0.0f, P, P, g_need - 1,
                                    nullptr) == LF_ERR_WORKSPACE);
        break;
      }
      default: {
        lf_token_shape s;
        memset(&s, 0, sizeof s);
        s.heads = PICK(1, 2, 12, 40, 32767, 32768, 0); s.head_dim = PICK(64, 128); s.q_len = PICK(1, 16, 17, 33, 64, 65, 0);
        s.cached_len = PICK(0, 1, 77, 32760, 1 << 24, -1, INT32_MAX); s.extra_len = PICK(0, 1, 64, 1 << 24, -1, INT32_MAX);
        s.q_stride_tok = s.k_stride_tok = s.v_stride_tok = s.o_stride_tok = s.head_dim;
        s.q_stride_head = s.k_stride_head = s.v_stride_head = s.o_stride_head = (int64_t)s.head_dim * 64;
        if (rnd() % 4 == 0) s.k_stride_head = stride();
        if (rnd() % 4 == 0) s.o_stride_tok = stride();
        lf_kvq_shape cs = {s.heads, s.head_dim, rnd() % 2 ? 1 << 24 : 32760, 0};
        g_need = lf_token_attn_kvq_workspace_bytes(&s);
        rc = lf_token_attn_kvq(P, P, lf_kvq_bytes(&cs), &cs, P, P, &s, scales[rnd() % 6], P, P, g_need, nullptr);
        EXPECT((rc == LF_OK) == (g_launches == before + 1));
        break;
      }
    }
    ok += rc == LF_OK;
    if (g_fail > 20) break;
  }
  EXPECT(ok > 20000);
  printf("%d calls let through\n%s\n", ok, g_fail ? "SOME FAILED" : "ALL OK");
  return g_fail != 0;
}
