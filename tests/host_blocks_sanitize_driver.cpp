// Host-only driver for the sanitizer build of the host side of the calls around the attention: every entry point on sizes drawn from small ones, the limits and the
// ends of their types, the kernel launchers replaced by ones that check what reaches them.  Pointers are never dereferenced here.
#include <stdio.h>
#include <string.h>

#include "lf_blocks.h"

static int g_fail = 0, g_launches = 0;
static size_t g_need = 0;      // the workspace that the caller has
#define EXPECT(cond) do { if (!(cond)) { printf("FAILED line %d: %s\n", __LINE__, #cond); ++g_fail; } } while (0)
static const int64_t kThreads = (int64_t)1 << 32;

static void check_lay(const lf_norm_lay& l, int channels, int most) {
  EXPECT(l.nc >= 1 && l.nc <= 3 && l.threads % 64 == 0 && l.threads >= 64 && l.threads <= most && l.threads * l.nc * 8 >= channels);
}
int lf_launch_gate_norm(const lf_norm_call* c, void*) {
  ++g_launches;
  lf_norm_lay l;
  const int rows = lf_norm_fwd_rows(c->s, &l);
  check_lay(l, c->s->channels, l.nc == 2 ? 1024 : 256);
  EXPECT(rows >= 1 && ((int64_t)(c->s->tokens - 1) / rows + 1) * l.threads < kThreads);
  return LF_OK;
}
int lf_launch_gate_norm_bwd(const lf_norm_call* c, void*) {
  ++g_launches;
  const lf_norm_slots n = lf_norm_bwd_slots(c->s);
  check_lay(n.lay, c->s->channels, n.waves ? 64 : n.lay.nc == 2 ? 1024 : 256);
  EXPECT(n.waves || n.lay.nc >= 2);
  EXPECT(n.rows >= 1 && n.slots >= 1 && n.slots * (n.waves ? 256 : n.lay.threads) < kThreads && (size_t)n.floats * 4 <= g_need);
  EXPECT((n.slots * 3 + 2 * (int64_t)c->s->groups) * c->s->channels <= n.floats);
  if (c->s->group_len > 0) EXPECT((int64_t)n.per_group * n.rows >= c->s->group_len && n.slots == (int64_t)n.per_group * c->s->groups);
  else EXPECT(n.slots >= (int64_t)c->s->tokens / n.rows + c->s->groups);
  return LF_OK;
}
static void check_plan(const lf_packed_call* c) {
  const lf_packed_shape* s = c->s;
  const lf_packed_plan& p = c->plan;
  const int64_t heads = p.few ? s->kv_heads : s->heads, group = s->heads / s->kv_heads;
  EXPECT(p.tile == (p.few ? p.tile : 128) && (p.tile == 16 || p.tile == 32 || p.tile == 128));
  EXPECT(p.slots >= (int64_t)s->q_len * (p.few ? group : 1) / p.tile + s->seqs && p.slots <= INT32_MAX);
  EXPECT(p.parts >= 1 && p.parts <= LF_PACKED_MAX_PARTS && p.part_tokens >= 64 && p.part_tokens % 64 == 0);
  EXPECT(p.slots * heads * p.parts * 256 < kThreads && p.slots * heads * (p.tile / 4) * (p.parts > 1 ? 256 : 0) < kThreads);
  EXPECT(c->scale > 0.0f);
}
int lf_launch_packed_attn(const lf_packed_call* c, void*) {
  ++g_launches;
  check_plan(c);
  const int64_t states = c->plan.slots * (c->plan.few ? c->s->kv_heads : c->s->heads) * c->plan.parts * c->plan.tile;
  EXPECT(c->plan.parts == 1 || (size_t)states * (c->s->head_dim + 2) * 4 <= g_need);
  EXPECT(c->s->q_len > 0);
  return LF_OK;
}
int lf_launch_packed_bwd(const lf_packed_call* c, void*) {
  ++g_launches;
  const lf_packed_shape* s = c->s;
  EXPECT((size_t)s->heads * s->q_len * 8 <= g_need);
  EXPECT(((int64_t)s->q_len / 128 + s->seqs) * s->heads * 256 < kThreads && ((int64_t)s->kv_len / 64 + s->seqs) * s->kv_heads * 1024 < 4 * kThreads);
  EXPECT(((int64_t)s->q_len / 32 + 1) * (s->heads / s->kv_heads) <= INT32_MAX);      // steps of a workgroup
  return LF_OK;
}
int lf_launch_grad_clip(const lf_grad_tensor* t, int32_t count, int64_t numel, float, float, float*, double*, void*) {
  ++g_launches;
  const int64_t chunk = lf_grad_chunk(numel);
  int64_t chunks = 0;
  for (int i = 0; i < count; ++i) chunks += (t[i].numel + chunk - 1) / chunk;
  EXPECT(chunk >= 4096 && chunk % 8 == 0 && (size_t)(chunks + 1) * 8 <= g_need);
  return LF_OK;
}

static uint64_t g_state = 1;
static uint32_t rnd() { g_state = g_state * 6364136223846793005ull + 1442695040888963407ull; return (uint32_t)(g_state >> 33); }
static int pick(const int* v, int n) { return v[rnd() % n]; }
#define PICK(...) ([] { static const int v[] = {__VA_ARGS__}; return pick(v, (int)(sizeof(v) / sizeof(v[0]))); }())
static int64_t stride() {
  static const int64_t v[] = {64, 128, 128, 5120, 8, 0, -8, 132, INT64_MAX, INT64_MAX / 8 * 8, INT64_MIN, (int64_t)1 << 40, (int64_t)1 << 44};
  return v[rnd() % (sizeof(v) / sizeof(v[0]))];
}

int main() {
  void* const P = (void*)0x10000;
  float* const F = (float*)P;
  int32_t* const I = (int32_t*)P;
  const float scales[] = {0.0f, 0.125f, -1.0f, 1e-40f, __builtin_inff(), __builtin_nanf("")};
  int ok = 0;
  for (int i = 0; i < 400000; ++i) {
    const int before = g_launches;
    int rc = 0;
    switch (rnd() % 4) {
      case 0: {
        lf_norm_shape s;
        memset(&s, 0, sizeof s);
        s.tokens = PICK(1, 7, 4680, 32760, 1 << 30, 0, INT32_MAX); s.channels = PICK(8, 320, 1536, 1544, 5120, 6144, 6152, 8192, 16384, 16392, 12, 0, INT32_MAX);
        s.groups = PICK(1, 3, 21, 1000, 1 << 24, 0, INT32_MAX); s.group_len = PICK(0, 0, 1, 1560, 4680, 1 << 30, -1, INT32_MAX);
        s.stream_dtype = PICK(0, 0, 1, 2); s.kind = PICK(0, 1, 1, 2); s.eps = 1e-6f; s.residual_scale = 1.0f;
        s.x_stride = s.xo_stride = s.b_stride = s.y_stride = s.gate_stride = s.scale_stride = s.shift_stride = s.channels;
        if (rnd() % 6 == 0) s.xo_stride = stride();
        if (rnd() % 6 == 0) s.scale_stride = stride();
        g_need = lf_gate_norm_bwd_workspace_bytes(&s);
        rc = lf_gate_norm(P, P, F, F, F, F, F, I, &s, P, P, nullptr);
        EXPECT((rc == LF_OK) == (g_launches == before + 1));
        const int again = g_launches;
        const int rb = lf_gate_norm_bwd(P, P, F, F, F, F, I, &s, P, P, P, P, F, F, F, F, F, P, g_need, nullptr);
        EXPECT((rb == LF_OK) == (g_launches == again + 1) && (rb != LF_OK || (rc == LF_OK && g_need > 0)));
        if (rb == LF_OK) EXPECT(lf_gate_norm_bwd(P, P, F, F, F, F, I, &s, P, P, P, P, F, F, F, F, F, P, g_need - 1, nullptr) == LF_ERR_WORKSPACE);
        break;
      }
      case 1:
      case 2: {
        lf_packed_shape s;
        memset(&s, 0, sizeof s);
        s.kv_heads = PICK(1, 2, 8, 12, 4096, 4097, 0, -1, INT32_MAX);
        const int64_t h = (int64_t)s.kv_heads * PICK(1, 1, 3, 5, 256, 257, 0);
        s.heads = h > INT32_MAX ? INT32_MAX : (int)h;
        s.head_dim = PICK(64, 128, 128, 96); s.seqs = PICK(1, 1, 9, 300, 1 << 20, 0, INT32_MAX);
        s.q_len = PICK(0, 1, 16, 300, 4680, 32760, 1 << 30, -1, INT32_MAX); s.kv_len = PICK(0, 1, 77, 32760, 130000, 1 << 30, -1, INT32_MAX);
        s.causal = PICK(0, 1, 4680, 1 << 30, -1, INT32_MAX); s.dtype = PICK(0, 0, 0, 1);
        s.q_stride_tok = s.k_stride_tok = s.v_stride_tok = s.o_stride_tok = s.head_dim;
        s.q_stride_head = s.k_stride_head = s.v_stride_head = s.o_stride_head = (int64_t)s.head_dim << 30;
        if (rnd() % 6 == 0) s.k_stride_tok = stride();
        if (rnd() % 6 == 0) s.o_stride_head = stride();
        if (rnd() % 6 == 0) s.q_stride_head = stride();
        const float scale = scales[rnd() % 6];
        g_need = lf_packed_attn_workspace_bytes(&s);
        rc = lf_packed_attn(P, P, P, &s, I, I, scale, P, F, P, g_need, nullptr);
        EXPECT((rc == LF_OK && s.q_len > 0) == (g_launches == before + 1));
        if (rc == LF_OK && g_need > 0) EXPECT(lf_packed_attn(P, P, P, &s, I, I, 0.0f, P, F, P, g_need - 1, nullptr) == LF_ERR_WORKSPACE);
        const int again = g_launches;
        g_need = lf_packed_attn_bwd_workspace_bytes(&s);
        const int rb = lf_packed_attn_bwd(P, P, P, P, P, F, &s, I, I, scale, P, P, P, P, g_need, nullptr);
        EXPECT((rb == LF_OK) == (g_launches == again + 1));
        break;
      }
      default: {
        lf_grad_tensor t[90];
        const int count = PICK(0, 1, 4, 4, 90);
        int64_t numel = 0;
        const bool apart = rnd() % 4 != 0;        // or all at one place
        for (int k = 0; k < 90; ++k) {
          const int64_t at = apart ? (int64_t)((31 * k) % 90) << 46 : 0;
          t[k] = {(char*)P + at, rnd() % 2 ? (char*)P + at + (apart ? (int64_t)1 << 45 : 0x10000) : nullptr, PICK(0, 1, 7, 4096, 100000, INT32_MAX, -1), PICK(0, 1, 1, 2), PICK(0, 1)};
          if (rnd() % 16 == 0) t[k].numel = stride();
          if (k >= 4 && rnd() % 8) t[k].numel = k, t[k].dtype = 0, t[k].out_dtype = 1;
          if (k < count && t[k].numel > 0 && t[k].numel < (int64_t)1 << 41) numel += t[k].numel;
        }
        g_need = lf_grad_workspace_bytes(count, numel);
        rc = lf_grad_clip(t, count, scales[rnd() % 6], 1e-6f, F, P, g_need, nullptr);
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
