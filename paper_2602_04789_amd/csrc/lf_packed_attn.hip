// Attention over packed sequences, and the joining of divided rows.
//
//   O_x = sum_y softmax_y(q_x . k_y scale) v_y,   y over the first tokens of x's sequence: all of them, or those up to its own or its chunk's end
//
// A workgroup of four wavefronts has 128 rows of one head, 32 of a wavefront, and walks the tokens that its last row sees in tiles of 64 that the
// wavefronts share through LDS (two stages; the next tile is on its way while one is worked on).  The products are computed transposed,
// S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16_bf16: a lane holds one row's scores of half the tokens, P stays in its registers as
// the second product's operand, and V is read through the transposing LDS read.  The online softmax has a reference that moves only when a row's sum
// is about to leave the range (see lf_attn.hip), so no maximum is taken on the way.  Only tiles that a wavefront's first row does not see whole are masked, and
// those that its last row does not see are left out.
//
// Heads of the last rows, which see most, go first; neighbouring workgroups take heads in turn, so that those that share a head of K and V run at
// one time on the XCDs that have it.
//
// Seven prompts, 16 384 tokens, 40 heads on 8 of 128: 580 us (1033 TFLOP/s of what the rows see; 1.40 PFLOP/s is what a large product reaches; 601 us with the products and
// the exponentials of a tile one after the other).  Seven chunks of 4680 tokens, 12 heads: 3.28 ms (1150 TFLOP/s).  4680 rows of 12 heads over 512 tokens: 23.1 us
// (637 TFLOP/s); over none it takes 9.6, over 64 11.6, and every further 64 take 1.5 to 2.2 (1.3 at the rate of a large product).
#include "lf_packed.h"

namespace {

constexpr int kRows = 128;        // of a workgroup
constexpr int kTok = 64;          // tokens of a tile

template <int CH> __device__ __forceinline__ int v_swz(int row, int ch) {
  return CH == 16 ? ch ^ ((row & 3) << 2) : ch ^ (((row >> 1) & 1) << 2);
}

typedef __attribute__((address_space(3))) const u32x4* LdsRow;
typedef __attribute__((address_space(3))) bf16x4* LdsQuad;

template <int D>
__global__ __launch_bounds__(256, 2) void lf_packed_attn_kernel(PackedArgs a) {
  constexpr int CH = D / 8, KS = D / 16, MB = D / 32;
  constexpr int TILE = kTok * CH;           // 16-byte chunks of K or V of a tile
  constexpr int LPW = TILE / 64 / 4;        // load instructions of a wavefront for K or V of a tile
  constexpr int RPI = 64 / CH;              // rows of a load instruction
  __shared__ __attribute__((aligned(64 * TILE))) u32x4 stage[2][2 * TILE];      // K | V: the stages differ in one bit of an address

  int x = blockIdx.x;
  const int hk = x % a.Hk;
  x /= a.Hk;
  const int h = hk * a.G + x % a.G;
  x /= a.G;
  const int part = x / a.slots, place = a.slots - 1 - x % a.slots;        // (parts that a short sequence leaves empty come last)
  int tile;
  const int b = find_tile(a.q_start, a.seqs, a.q_len, 1, kRows, place, tile);
  const Span s = span_of(a, b);
  const int i0 = tile * kRows;
  if (tile < 0 || i0 >= s.nq) return;
  const int rows = min(kRows, s.nq - i0);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ln = lane & 31, kg = lane >> 5;
  const int row = 32 * wave + ln;
  // tokens that this lane's row, the wavefront's first and last and the workgroup's last row see
  const int lim = row_limit(s, a.unit, min(i0 + row, s.nq - 1));
  const bool active = 32 * wave < rows;
  const int lim_first = row_limit(s, a.unit, i0 + 32 * wave);
  const int lim_last = active ? row_limit(s, a.unit, i0 + min(32 * wave + 31, rows - 1)) : 0;
  const int seen = row_limit(s, a.unit, i0 + rows - 1);
  int t0 = 0, t1 = seen;
  if (a.parts > 1) {
    const int len = part_len(a, seen);
    t0 = (int)min((int64_t)part * len, (int64_t)seen);
    t1 = (int)min((int64_t)t0 + len, (int64_t)seen);
    if (t0 >= t1) return;                 // the joining launch leaves it out too
  }

  Frag qf[KS];
  {
    const uint16_t* qp = a.Q + (int64_t)h * a.q_head + (int64_t)(s.q0 + i0 + row) * a.q_tok;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      qf[k].u = u32x4{0, 0, 0, 0};
      if (row < rows) qf[k].u = *reinterpret_cast<const u32x4*>(qp + 16 * k + 8 * kg);
    }
  }
  const uint16_t* Kh = a.K + (int64_t)hk * a.k_head;
  const uint16_t* Vh = a.V + (int64_t)hk * a.v_head;
  const uint32_t k_row = (uint32_t)(a.k_tok * 2), v_row = (uint32_t)(a.v_tok * 2);
  uint32_t koff[LPW], voff[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int r = RPI * (LPW * wave + i) + lane / CH, p = lane % CH;
    koff[i] = (uint32_t)r * k_row + (uint32_t)row_swz<CH>(r, p) * 16u - 1024u * (i & 3);
    voff[i] = (uint32_t)r * v_row + (uint32_t)v_swz<CH>(r, p) * 16u - 1024u * (i & 3);
  }
  auto request = [&](int t, u32x4* to) __attribute__((always_inline)) {
    const int n = min(kTok, t1 - t);
    fetch<LPW>(rows_rsrc(Kh, (int64_t)s.k0 + t, n, k_row), lds_addr(to + LPW * 64 * wave), koff);
    fetch<LPW>(rows_rsrc(Vh, (int64_t)s.k0 + t, n, v_row), lds_addr(to + TILE + LPW * 64 * wave), voff);
  };
  // addresses in the present stage
  const uint32_t base = __builtin_amdgcn_readfirstlane(lds_addr(&stage[0][0]));
  uint32_t kaddr[KS], vaddr[MB];
#pragma unroll
  for (int k = 0; k < KS; ++k) kaddr[k] = base + 16u * (ln * CH + row_swz<CH>(ln, 2 * k + kg));
  {
    const int i16 = lane & 15, tr_row = 4 * kg + (i16 >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int col = 32 * mb + tr_col;
      vaddr[mb] = base + 16u * TILE + 2u * ((tr_row * CH + v_swz<CH>(tr_row, col >> 3)) * 8 + (col & 7));
    }
  }
  auto other_stage = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < KS; ++k) kaddr[k] ^= 32u * TILE;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) vaddr[mb] ^= 32u * TILE;
  };

  f32x16 oacc[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) oacc[mb] = zero16();
  constexpr float kSumMax = 1.0e30f;
  float m_run = -1.0e30f, l_run = 0.0f;
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};

  // One tile of tokens [t, t + 64) of the sequence, in halves: S of the first, S of the second beside the exponentials of the first, O of the first beside those
  // of the second, O of the second.  A slot holds one product, the LDS reads of a fragment of the next block and a share of the exponentials, which go
  // through their stages (scale, exp2, pack and sum) a beat each; sched_barrier keeps the slots as written.
  auto work = [&](int t) __attribute__((always_inline)) {
    static_assert(KS == 2 * MB, "a half tile has as many products of S as of O");
    constexpr int kBeats = 16 / KS;           // of a slot
    Frag k0[KS], k1[KS];
    bf16x8 v0[KS], v1[KS], p0[2], p1[2];
    f32x16 s0 = zero16(), s1 = zero16();
    auto v_frag = [&](int hf, int n) __attribute__((always_inline)) {
      const int u = 2 * hf + n / MB, mb = n % MB;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsQuad)(uintptr_t)(vaddr[mb] + 16u * CH * (16 * u)));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsQuad)(uintptr_t)(vaddr[mb] + 16u * CH * (16 * u + 8)));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto mask = [&](int hf, f32x16& sc) __attribute__((always_inline)) {      // accumulator i: token 8 (i / 4) + 4 kg + i mod 4 of the half tile
      if (t + 32 * hf + 32 > lim_first) {
        const int past = lim - t - 32 * hf - 4 * kg;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i >> 2) + (i & 3) >= past) sc[i] = -INFINITY;
      }
    };
    float x[2], y[2], l_new;
    auto beat = [&](int n, const f32x16& sc, bf16x8 (&p)[2]) __attribute__((always_inline)) {      // 18 of them
      if (n >= 2 && (n & 1)) {
        const int v = n - 2;
        const bf16x2 pr = {(__bf16)y[0], (__bf16)y[1]};
        p[v >> 3][(v & 7) - 1] = pr[0];
        p[v >> 3][v & 7] = pr[1];
        l_new = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l_new, false);
      }
      if (n >= 1 && n < 17) y[(n - 1) & 1] = __builtin_amdgcn_exp2f(x[(n - 1) & 1]);
      if (n < 16) x[n & 1] = fmaf(sc[n], a.c, -m_run);
    };
    // behind the exponentials of a half: the reference moves where the row's sum is about to leave the range
    auto check = [&](const f32x16& sc, bf16x8 (&p)[2]) __attribute__((always_inline)) {
      if (__ballot(l_new > kSumMax) != 0ull) {
        float top = fmaxf(sc[0], sc[1]);
#pragma unroll
        for (int i = 2; i < 16; i += 2) top = fmaxf(top, fmaxf(sc[i], sc[i + 1]));
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * a.c;
        const float m_new = fmaxf(m_run, top), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i) oacc[mb][i] *= alpha;
        l_new = l_run * alpha;
#pragma unroll
        for (int n = 0; n < 18; ++n) beat(n, sc, p);
      }
      l_run = l_new;
    };
#pragma unroll
    for (int n = 0; n < KS; ++n) k0[n].u = *(LdsRow)(uintptr_t)kaddr[n];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < KS; ++n) {
      s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0[n].v, qf[n].v, s0, 0, 0, 0);
      k1[n].u = *(LdsRow)(uintptr_t)(kaddr[n] + 512u * CH);
      __builtin_amdgcn_sched_barrier(0);
    }
    mask(0, s0);
    l_new = l_run;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < KS; ++n) {
      s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1[n].v, qf[n].v, s1, 0, 0, 0);
      v0[n] = v_frag(0, n);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kBeats; ++i)
        if (n > 0) beat(kBeats * (n - 1) + i, s0, p0);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 16 - kBeats; i < 18; ++i) beat(i, s0, p0);
    check(s0, p0);
    mask(1, s1);
    l_new = l_run;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < KS; ++n) {
      oacc[n % MB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v0[n], p0[n / MB], oacc[n % MB], 0, 0, 0);
      v1[n] = v_frag(1, n);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kBeats; ++i) beat(kBeats * n + i, s1, p1);
      __builtin_amdgcn_sched_barrier(0);
    }
    beat(16, s1, p1);
    beat(17, s1, p1);
    check(s1, p1);
#pragma unroll
    for (int n = 0; n < KS; ++n) oacc[n % MB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1[n], p1[n / MB], oacc[n % MB], 0, 0, 0);
  };
  if (t0 < t1) request(t0, stage[0]);
  int cur = 0;
  for (int t = t0; t < t1; t += kTok, cur ^= 1) {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));     // this wavefront's share of the tile
    lds_barrier();                                // everyone's, and nobody reads the other stage any more
    if (t + kTok < t1) request(t + kTok, stage[cur ^ 1]);
    if (t < lim_last) work(t);
    other_stage();
  }

  const float l = l_run + __shfl_xor(l_run, 32);
  if (row >= rows) return;
  if (a.parts > 1) {
    const int64_t at = (((int64_t)place * a.H + h) * a.parts + part) * kRows + row;
    if (kg == 0) a.state_ml[at] = make_float2(m_run, l);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = oacc[mb][4 * g + e];
        *reinterpret_cast<f32x4*>(a.state_o + at * D + 32 * mb + 8 * g + 4 * kg) = o;
      }
    return;
  }
  const int64_t token = (int64_t)s.q0 + i0 + row;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  if (a.lse2 && kg == 0) a.lse2[(int64_t)h * a.q_len + token] = l > 0.0f ? m_run + __builtin_log2f(l) : INFINITY;
  uint16_t* op = a.O + (int64_t)h * a.o_head + token * a.o_tok;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 o4;
#pragma unroll
      for (int e = 0; e < 4; ++e) o4[e] = (__bf16)(oacc[mb][4 * g + e] * inv);
      *reinterpret_cast<bf16x4*>(op + 32 * mb + 8 * g + 4 * kg) = o4;
    }
}

// Joins the parts of a row: a wavefront each, lane p holding part p's weight.  FEW: the row is a row and head of a tile of the few-row kernel.
template <int D>
__global__ __launch_bounds__(256) void lf_packed_join_kernel(PackedArgs a, int tile_rows, int few) {
  constexpr int W = D / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = tile_rows / 4;           // workgroups of a tile: four rows each
  const int64_t x = blockIdx.x;
  const int r = 4 * (int)(x % groups) + wave, heads = few ? a.Hk : a.H;
  const int64_t t = x / groups;
  const int hh = (int)(t % heads), place = (int)(t / heads), mul = few ? a.G : 1;
  int tile;
  const int b = find_tile(a.q_start, a.seqs, a.q_len, mul, tile_rows, place, tile);
  const Span s = span_of(a, b);
  const int64_t i0 = (int64_t)tile * tile_rows, all = (int64_t)s.nq * mul;
  if (tile < 0 || i0 + r >= all) return;
  const int i = (int)((i0 + r) / mul), h = few ? hh * a.G + (int)((i0 + r) % mul) : hh;
  const int seen = row_limit(s, a.unit, (int)((min(i0 + tile_rows, all) - 1) / mul));
  const int len = part_len(a, seen), parts = (seen + len - 1) / len;
  const int64_t first = t * a.parts * tile_rows + r;
  float2 ml = make_float2(-INFINITY, 0.0f);
  if (lane < parts) ml = a.state_ml[first + (int64_t)lane * tile_rows];
  float M = ml.x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
  const float w = ml.y > 0.0f ? __builtin_amdgcn_exp2f(ml.x - M) : 0.0f;
  float L = w * ml.y;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) L += __shfl_xor(L, off);
  float o[W];
#pragma unroll
  for (int e = 0; e < W; ++e) o[e] = 0.0f;
  auto add = [&](int p0, auto many) __attribute__((always_inline)) {         // that many parts, their loads all at once
    constexpr int N = decltype(many)::value;
    float v[N][W];
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < W; ++e) v[k][e] = a.state_o[(first + (int64_t)min(p0 + k, parts - 1) * tile_rows) * D + W * lane + e];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float wk = __shfl(w, p0 + k);
#pragma unroll
      for (int e = 0; e < W; ++e) o[e] = fmaf(wk, p0 + k < parts ? v[k][e] : 0.0f, o[e]);
    }
  };
  if (parts > 0 && parts <= 4) add(0, std::integral_constant<int, 4>{});
  else
    for (int p0 = 0; p0 < parts; p0 += 16) add(p0, std::integral_constant<int, 16>{});
  const float inv = L > 0.0f ? 1.0f / L : 0.0f;
  const int64_t token = (int64_t)s.q0 + i;
  if (a.lse2 && lane == 0) a.lse2[(int64_t)h * a.q_len + token] = L > 0.0f ? M + __builtin_log2f(L) : INFINITY;
  __bf16* to = reinterpret_cast<__bf16*>(a.O + (int64_t)h * a.o_head + token * a.o_tok) + W * lane;
#pragma unroll
  for (int e = 0; e < W; ++e) to[e] = (__bf16)(o[e] * inv);
}

}  // namespace

PackedArgs lf_packed_args(const lf_packed_call* c) {
  const lf_packed_shape* s = c->s;
  PackedArgs a = {};
  a.Q = (const uint16_t*)c->Q; a.K = (const uint16_t*)c->K; a.V = (const uint16_t*)c->V; a.dO = (const uint16_t*)c->dO;
  a.O = (uint16_t*)c->O; a.dQ = (uint16_t*)c->dQ; a.dK = (uint16_t*)c->dK; a.dV = (uint16_t*)c->dV;
  a.lse2 = c->lse2;
  a.q_start = c->q_start; a.kv_start = c->kv_start;
  a.q_tok = s->q_stride_tok; a.q_head = s->q_stride_head; a.k_tok = s->k_stride_tok; a.k_head = s->k_stride_head;
  a.v_tok = s->v_stride_tok; a.v_head = s->v_stride_head; a.o_tok = s->o_stride_tok; a.o_head = s->o_stride_head;
  a.H = s->heads; a.Hk = s->kv_heads; a.G = s->heads / s->kv_heads;
  a.seqs = s->seqs; a.q_len = s->q_len; a.kv_len = s->kv_len; a.unit = s->causal;
  a.slots = (int)c->plan.slots; a.parts = c->plan.parts; a.part_tokens = c->plan.part_tokens;
  a.scale = c->scale;
  a.c = c->scale * 1.44269504088896340736f;
  const int64_t states = c->plan.slots * (c->plan.few ? a.Hk : a.H) * c->plan.parts * c->plan.tile;
  a.state_o = (float*)c->workspace;
  a.state_ml = (float2*)((float*)c->workspace + states * s->head_dim);
  return a;
}

int lf_launch_packed_join(const PackedArgs& a, int d, int tile_rows, bool few, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.slots * (few ? a.Hk : a.H) * (tile_rows / 4)));
  const hipError_t rc = d == 128 ? lf_launch(lf_packed_join_kernel<128>, grid, dim3(256), 0, st, a, tile_rows, (int)few)
                                 : lf_launch(lf_packed_join_kernel<64>, grid, dim3(256), 0, st, a, tile_rows, (int)few);
  return rc == hipSuccess ? LF_OK : LF_ERR_HIP;
}

int lf_launch_packed_attn(const lf_packed_call* c, void* stream) {
  if (c->plan.few) return lf_launch_packed_rows(c, stream);
  const PackedArgs a = lf_packed_args(c);
  const int d = c->s->head_dim;
  hipStream_t st = (hipStream_t)stream;
  // 64 rows of a wavefront where rows see 8192 tokens or more in the mean, unless each sees another one more (us, 32 and 64 rows: 12 heads, 4096 rows of 4096 tokens 110 and
  // 112; 4680 rows of 8192 tokens 223 and 216, of 16 384 tokens 435 and 422; 40 heads of 18 720 tokens 1677 and 1613; by chunks of 4680, 12 heads of 32 760 tokens 3277
  // and 3257, with the gradients, which the chip's power slows, 14 570 and 14 250; causal, 40 heads of 8192 tokens 620 and 650, of 16 384 tokens 2449 and 2460).
  const int64_t seen = c->s->kv_len / (a.unit ? 2 : 1);
  if (d == 128 && a.parts == 1 && a.unit != 1 && c->s->q_len >= 512 * (int64_t)c->s->seqs && seen >= 8192 * (int64_t)c->s->seqs) return lf_launch_packed_attn_wide(a, st);
  const dim3 grid((unsigned)((int64_t)a.slots * a.H * a.parts));
  const hipError_t rc = d == 128 ? lf_launch(lf_packed_attn_kernel<128>, grid, dim3(256), 0, st, a)
                                 : lf_launch(lf_packed_attn_kernel<64>, grid, dim3(256), 0, st, a);
  if (rc != hipSuccess) return LF_ERR_HIP;
  return a.parts > 1 ? lf_launch_packed_join(a, d, kRows, false, st) : LF_OK;
}
