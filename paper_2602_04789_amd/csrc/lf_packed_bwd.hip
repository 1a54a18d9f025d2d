// Backward pass of the packed attention.  With P = exp2(s c - lse2), delta_x = dO_x . O_x, dP = dO V^T, dS = P (dP - delta):
//   dV_y = sum_x P dO_x      dQ_x = scale sum_y dS k_y      dK_y = scale sum_x dS q_x     (dK and dV over the heads that share the head, too)
//
// No atomics, every launch owns its outputs: one owns rows and walks the tokens they see (dQ; it leaves delta for the other), one owns tokens and walks the
// rows that see them, head by head (dK, dV).  Both recompute the scores.  As in the forward kernel the score-like products take their A operand from tiles in
// LDS and their B operand from the owner's rows in registers; P and dS are then the B operand of the accumulating products, whose A operand
// is the same tile through the transposing read.  Matrix work bounds both: seven products for the five that the mathematics counts.
#include "lf_packed.h"

namespace {

constexpr int kTile = 32;         // streamed rows of a step

// Two probabilities on their way to another wavefront, in 32 bits.  0 <= P <= 1 has neither a sign nor the upper bit of the exponent; 16 bits hold the other seven of
// that and nine of the fraction, so P is off by half a step, 2^-10 of the value, down to 2^-126.  (In binary16 what lies below 2^-14 has fewer bits and what lies below 2^-25
// none: beside a token whose logits are 16 above theirs the others' dK was off by 2.8e-2 in the median, so by 2.6e-3.  In bfloat16 dK of 1333 tokens is off by 2.9e-3, so by 2.4e-3.)
__device__ __forceinline__ uint32_t hand_over(float p0, float p1) {
  const uint32_t lo = (__float_as_uint(p0) << 2) + 0x8000u, hi = (__float_as_uint(p1) << 2) + 0x8000u;
  return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
}
__device__ __forceinline__ float taken_over(uint32_t pair, int which) {
  if (which) return __uint_as_float(pair >> 16 << 14);
  uint32_t w;          // (pair & 0xffff) << 14, in one instruction
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:WORD_0" : "=v"(w) : "v"(14), "v"(pair));
  return __uint_as_float(w);
}

// One swizzle for tiles that are read both ways (rows, and transposed: half a wavefront takes four chunks of each of four rows); the transposing
// read of rows 8 .. 15 of 16 sees chunk bit 1 flipped.
template <int CH> __device__ __forceinline__ int both_swz(int row, int ch) {
  return ch ^ (((CH == 16 ? row & 3 : (row >> 1) & 1) << 2) | ((row >> 2) & 3));
}
constexpr int kTrHiFlip = 16;     // of an element's place

// Rows that see this many tokens or fewer get delta = sum_y P dP (the same number) instead of dO . O: O was rounded to bfloat16, and where few
// tokens share a row's probability, one of them nearly all of it, what that leaves in dP - delta is more than the roundings of P and dS (12
// sequences of one to four tokens: dQ off by 4.8e-3 in the 2-norm).
constexpr int kShort = 256;

// dQ, and -delta and -lse2 / c of every row for the launch behind it: four wavefronts of 32 rows each share tiles of 32 tokens of K and V.
// Seven chunks of 4680 tokens, 12 heads of 128: 4.57 ms (1236 TFLOP/s of its three products); the matrix pipes are busy 70 % of the cycles, at 1.7 GHz: the chip's
// power bounds it.  (Three stages, two tiles ahead: 4.96 ms; 64 rows of a wavefront: 5.15 ms.)  1333 tokens in 9 sequences, 6 heads of 64: 13.6 us.
template <int D>
__global__ __launch_bounds__(256, 2) void lf_packed_dq_kernel(PackedArgs a) {
  constexpr int kRows = 128;
  constexpr int CH = D / 8, KS = D / 16, MB = D / 32;
  constexpr int T32 = kTile * CH;
  constexpr int LPW = T32 / 64 / 4;
  constexpr int RPI = 64 / CH;
  __shared__ u32x4 stage[2][2 * T32];      // K | V

  int x = blockIdx.x;
  const int hk = x % a.Hk;
  x /= a.Hk;
  const int h = hk * a.G + x % a.G, place = a.slots - 1 - x / a.G;
  int tile;
  const int b = find_tile(a.q_start, a.seqs, a.q_len, 1, kRows, place, tile);
  const Span s = span_of(a, b);
  const int i0 = tile * kRows;
  if (tile < 0 || i0 >= s.nq) return;
  const int rows = min(kRows, s.nq - i0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ln = lane & 31, kg = lane >> 5;
  const int row = 32 * wave + ln;
  const bool ok = row < rows;
  const int64_t token = (int64_t)s.q0 + i0 + row;
  // A row that sees a single token has no gradient of its scores: P = 1 whatever they are.
  int lim = row_limit(s, a.unit, min(i0 + row, s.nq - 1));
  if (lim == 1) lim = 0;
  const bool active = 32 * wave < rows;
  const int lim_first = s.nk == 1 || row_limit(s, a.unit, i0 + 32 * wave) <= 1 ? 0 : row_limit(s, a.unit, i0 + 32 * wave);
  const int lim_last = active ? row_limit(s, a.unit, i0 + min(32 * wave + 31, rows - 1)) : 0;
  const int seen = row_limit(s, a.unit, i0 + rows - 1);

  Frag qf[KS], gf[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    qf[k].u = gf[k].u = u32x4{0, 0, 0, 0};
    if (ok) {
      qf[k].u = *reinterpret_cast<const u32x4*>(a.Q + (int64_t)h * a.q_head + token * a.q_tok + 16 * k + 8 * kg);
      gf[k].u = *reinterpret_cast<const u32x4*>(a.dO + (int64_t)h * a.o_head + token * a.o_tok + 16 * k + 8 * kg);
    }
  }
  float lse = INFINITY, delta = 0.0f;
  if (ok) {
    lse = a.lse2[(int64_t)h * a.q_len + token];
  }
  const uint16_t* Kh = a.K + (int64_t)hk * a.k_head;
  const uint16_t* Vh = a.V + (int64_t)hk * a.v_head;
  const uint32_t k_row = (uint32_t)(a.k_tok * 2), v_row = (uint32_t)(a.v_tok * 2);
  uint32_t koff[LPW], voff[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int r = RPI * (LPW * wave + i) + lane / CH, p = lane % CH;
    koff[i] = (uint32_t)r * k_row + (uint32_t)both_swz<CH>(r, p) * 16u - 1024u * (i & 3);
    voff[i] = (uint32_t)r * v_row + (uint32_t)row_swz<CH>(r, p) * 16u - 1024u * (i & 3);
  }
  auto request = [&](int t, u32x4* to) __attribute__((always_inline)) {
    const int n = min(kTile, seen - t);
    fetch<LPW>(rows_rsrc(Kh, (int64_t)s.k0 + t, n, k_row), lds_addr(to + LPW * 64 * wave), koff);
    fetch<LPW>(rows_rsrc(Vh, (int64_t)s.k0 + t, n, v_row), lds_addr(to + T32 + LPW * 64 * wave), voff);
  };
  int kaddr[KS], vaddr[KS], tbase[MB];
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    kaddr[k] = ln * CH + both_swz<CH>(ln, 2 * k + kg);
    vaddr[k] = ln * CH + row_swz<CH>(ln, 2 * k + kg);
  }
  {
    const int i16 = lane & 15, tr_row = 4 * kg + (i16 >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int col = 32 * mb + tr_col;
      tbase[mb] = (tr_row * CH + both_swz<CH>(tr_row, col >> 3)) * 8 + (col & 7);
    }
  }
  f32x16 nd16 = zero16();
  auto scores = [&](int t, const u32x4* at, f32x16& sc, f32x16& dp) __attribute__((always_inline)) {
    Frag kf[KS], vf[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      kf[k].u = at[kaddr[k]];
      vf[k].u = at[T32 + vaddr[k]];
    }
    sc = zero16();
    dp = nd16;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k].v, qf[k].v, sc, 0, 0, 0);
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k].v, gf[k].v, dp, 0, 0, 0);
    }
    if (t + kTile > lim_first) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (t + 8 * (i >> 2) + 4 * kg + (i & 3) >= lim) sc[i] = -INFINITY;
    }
  };
  // every tile of tokens that the workgroup's rows see, in turn
  auto walk = [&](auto work) __attribute__((always_inline)) {
    if (seen > 0) request(0, stage[0]);
    int cur = 0;
    for (int t = 0; t < seen; t += kTile, cur ^= 1) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      lds_barrier();
      if (t + kTile < seen) request(t + kTile, stage[cur ^ 1]);
      if (t < lim_last) work(t, stage[cur]);
    }
  };
  if (seen <= kShort) {
    walk([&](int t, const u32x4* at) __attribute__((always_inline)) {
      f32x16 sc, dp;
      scores(t, at, sc, dp);
#pragma unroll
      for (int i = 0; i < 16; ++i) delta = fmaf(__builtin_amdgcn_exp2f(fmaf(sc[i], a.c, -lse)), dp[i], delta);
    });
    lds_barrier();                  // the second walk begins in the first stage
  } else if (ok) {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const u32x4 o = *reinterpret_cast<const u32x4*>(a.O + (int64_t)h * a.o_head + token * a.o_tok + 16 * k + 8 * kg);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        delta = fmaf(__uint_as_float(o[e] << 16), __uint_as_float(gf[k].u[e] << 16), delta);
        delta = fmaf(__uint_as_float(o[e] & 0xffff0000u), __uint_as_float(gf[k].u[e] & 0xffff0000u), delta);
      }
    }
  }
  delta += __shfl_xor(delta, 32);
  if (ok && kg == 0) {
    a.ndelta[(int64_t)h * a.q_len + token] = -delta;
    a.nlse[(int64_t)h * a.q_len + token] = -lse / a.c;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) nd16[i] = -delta;
  f32x16 acc[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) acc[mb] = zero16();
  walk([&](int t, const u32x4* at) __attribute__((always_inline)) {
    f32x16 sc, dp;
    scores(t, at, sc, dp);
    bf16x8 ds[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) ds[i >> 3][i & 7] = (__bf16)(__builtin_amdgcn_exp2f(fmaf(sc[i], a.c, -lse)) * dp[i]);
    const uint16_t* k16 = reinterpret_cast<const uint16_t*>(at);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(bf16x4, k16 + tbase[mb] + 16 * u * CH * 8));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(bf16x4, k16 + (tbase[mb] ^ kTrHiFlip) + (16 * u + 8) * CH * 8));
        acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), ds[u], acc[mb], 0, 0, 0);
      }
  });
  if (!ok) return;
  uint16_t* op = a.dQ + (int64_t)h * a.q_head + token * a.q_tok;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 o4;
#pragma unroll
      for (int e = 0; e < 4; ++e) o4[e] = (__bf16)(acc[mb][4 * g + e] * a.scale);
      *reinterpret_cast<bf16x4*>(op + 32 * mb + 8 * g + 4 * kg) = o4;
    }
}

// dK and dV of 64 tokens: wavefront (rh, role) has 32 of them.  Role 0 computes S = Q K^T, P and dV^T += dO^T P, role 1 dP = dO V^T, dS and
// dK^T += Q^T dS a step later, with the P that its partner has left in LDS (see hand_over); so one barrier a step is enough.  A tile is
// requested two steps ahead; its Q lives for two steps (four stages), its dO for one (three).  SPLIT > 1: the workgroup holds SPLIT such groups with stages of their own, each takes a share of the steps (all the same number; those past
// the end are empty), and their sums are added through LDS in order: for calls with too few tokens to fill the chip.
// 1333 tokens in 9 sequences, 6 heads on 2 of 64: 19 us, 32 with tiles one step ahead and an LDS layout for the transposed reads alone: latency, a step after another.
template <int D, int SPLIT>
__global__ __launch_bounds__(256 * SPLIT, SPLIT == 1 ? 2 : 1) void lf_packed_dkv_kernel(PackedArgs a) {
  constexpr int kTokens = 64;
  constexpr int CH = D / 8, KS = D / 16, MB = D / 32;
  constexpr int T32 = kTile * CH;
  constexpr int LPW = T32 / 64 / 4;
  constexpr int RPI = 64 / CH;
  __shared__ u32x4 buf_all[SPLIT][7][T32];       // Q [step mod 4], dO [step mod 3]
  __shared__ f32x4 st_all[SPLIT][3][4][16];      // [step mod 3] -lse2 / c (role 0) or -delta of the 32 rows, for each wavefront; the upper half takes what the other lanes load
  __shared__ u32x4 ph_all[SPLIT][2][2][2][64];   // P: [step parity][rh][k-step][lane]
  const int group = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
  u32x4 (*const qbuf)[T32] = buf_all[group];
  u32x4 (*const obuf)[T32] = qbuf + 4;
  f32x4 (*const st)[4][16] = st_all[group];
  u32x4 (*const ph)[2][2][64] = ph_all[group];

  int x = blockIdx.x;
  const int hk = x % a.Hk, place = x / a.Hk;
  int tile;
  const int b = find_tile(a.kv_start, a.seqs, a.kv_len, 1, kTokens, place, tile);
  const Span s = span_of(a, b);
  const int j0 = tile * kTokens;
  if (tile < 0 || j0 >= s.nk) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) & 3);
  const int ln = lane & 31, kg = lane >> 5, rh = wave & 1;
  const bool is_ds = (wave >= 2) != ((group & 1) != 0);      // every SIMD has as many wavefronts of either role
  const int j = j0 + 32 * rh + ln;
  const bool ok = j < s.nk;
  const int64_t token = (int64_t)s.k0 + j;
  // the first rows that see this lane's token, the wavefront's last one and the workgroup's first one
  const int from = first_row(s, a.unit, j), from_last = first_row(s, a.unit, min(j0 + 32 * rh + 31, s.nk - 1));
  const int i_first = first_row(s, a.unit, j0) / kTile * kTile;
  const int tiles = i_first < s.nq ? (s.nq - i_first + kTile - 1) / kTile : 0;
  const int steps_all = tiles * a.G, steps = (steps_all + SPLIT - 1) / SPLIT, step0 = group * steps;    // this group's: [step0, step0 + steps), of all heads

  Frag of[KS];
  {
    const uint16_t* p = is_ds ? a.V + (int64_t)hk * a.v_head + token * a.v_tok : a.K + (int64_t)hk * a.k_head + token * a.k_tok;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      of[k].u = u32x4{0, 0, 0, 0};
      if (ok) of[k].u = *reinterpret_cast<const u32x4*>(p + 16 * k + 8 * kg);
    }
  }
  const uint32_t q_row = (uint32_t)(a.q_tok * 2), o_row = (uint32_t)(a.o_tok * 2);
  uint32_t qoff[LPW], ooff[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int r = RPI * (LPW * wave + i) + lane / CH, p = lane % CH;
    qoff[i] = (uint32_t)r * q_row + (uint32_t)both_swz<CH>(r, p) * 16u - 1024u * (i & 3);
    ooff[i] = (uint32_t)r * o_row + (uint32_t)both_swz<CH>(r, p) * 16u - 1024u * (i & 3);
  }
  const uint32_t st_off = (uint32_t)lane * 4u;
  const float* stat = is_ds ? a.ndelta : a.nlse;
  // where the next request goes: rows [ri, ri + 32) of the sequence, head rg of the group
  int ri = tiles > 0 ? i_first + step0 % tiles * kTile : 0, rg = tiles > 0 ? step0 / tiles : 0;
  const int wi0 = ri;
  int q_to = 0, o_to = 0;
  auto request = [&]() __attribute__((always_inline)) {
    const int h = hk * a.G + min(rg, a.G - 1), n = rg < a.G ? min(kTile, s.nq - ri) : 0;
    const int64_t first = (int64_t)s.q0 + ri;
    fetch<LPW>(rows_rsrc(a.Q + (int64_t)h * a.q_head, first, n, q_row), lds_addr(qbuf[q_to] + LPW * 64 * wave), qoff);
    fetch<LPW>(rows_rsrc(a.dO + (int64_t)h * a.o_head, first, n, o_row), lds_addr(obuf[o_to] + LPW * 64 * wave), ooff);
    const int32x4 rs = aged(rows_rsrc(reinterpret_cast<const uint16_t*>(stat + (int64_t)h * a.q_len), first, n, 4u));
    const uint32_t at = __builtin_amdgcn_readfirstlane(lds_addr(st[o_to][wave]));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(at), "v"(st_off), "s"(rs) : "memory", "m0");
    ri += kTile;
    if (ri >= s.nq) {
      ri = i_first;
      ++rg;
    }
    q_to = (q_to + 1) & 3;
    o_to = o_to == 2 ? 0 : o_to + 1;
  };
  int raddr[KS], tbase[MB];
#pragma unroll
  for (int k = 0; k < KS; ++k) raddr[k] = ln * CH + both_swz<CH>(ln, 2 * k + kg);
  {
    const int i16 = lane & 15, tr_row = 4 * kg + (i16 >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int col = 32 * mb + tr_col;
      tbase[mb] = (tr_row * CH + both_swz<CH>(tr_row, col >> 3)) * 8 + (col & 7);
    }
  }
  f32x16 acc[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) acc[mb] = zero16();

  auto tfrag = [&](const u32x4* at, int u, int mb) __attribute__((always_inline)) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(at);
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(bf16x4, p + tbase[mb] + 16 * u * CH * 8));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(bf16x4, p + (tbase[mb] ^ kTrHiFlip) + (16 * u + 8) * CH * 8));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto rows_of = [&](const u32x4* at, Frag (&f)[KS]) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < KS; ++k) f[k].u = at[raddr[k]];
  };
  auto product = [&](const Frag (&f)[KS], f32x16 c) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < KS; ++k) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[k].v, of[k].v, c, 0, 0, 0);
    return c;
  };
  auto first_half = [&](const u32x4* at, bf16x8 (&tf)[MB]) __attribute__((always_inline)) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) tf[mb] = tfrag(at, 0, mb);
  };
  auto accumulate = [&](const u32x4* at, const bf16x8 (&tf)[MB], const bf16x8 (&y)[2]) __attribute__((always_inline)) {
    bf16x8 t2[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) t2[mb] = tfrag(at, 1, mb);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tf[mb], y[0], acc[mb], 0, 0, 0);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t2[mb], y[1], acc[mb], 0, 0, 0);
  };
  auto stats16 = [&](int at) __attribute__((always_inline)) {
    f32x16 v;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 y = st[at][wave][2 * g + kg];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * g + e] = y[e];
    }
    return v;
  };
  // role 0, step t: rows [i, i + 32), in stages qa and at
  auto p_step = [&](int t, int qa, int at, int i) __attribute__((always_inline)) {
    const bool none = SPLIT > 1 && step0 + t >= steps_all;
    Frag f[KS];
    rows_of(qbuf[qa], f);
    f32x16 sc = stats16(at);
    __builtin_amdgcn_sched_barrier(0);
    sc = product(f, sc);
    bf16x8 tf[MB];
    first_half(obuf[at], tf);
    __builtin_amdgcn_sched_barrier(0);
    if (i < from_last || i + kTile > s.nq || none) {        // (rows behind the last one were loaded as zeros, their statistics too)
      const int lo = none ? kTile : from - i - 4 * kg, past = s.nq - i - 4 * kg;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int r = 8 * (e >> 2) + (e & 3);
        if (r < lo || r >= past) sc[e] = -INFINITY;
      }
    }
    bf16x8 pf[2];
    u32x4 ps[2];
    float p[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(sc[e] * a.c), 0.0f, 1.0f);      // (lse2 is of rounded terms: P may come out as 1 + 2^-8)
      pf[e >> 3][e & 7] = (__bf16)p[e];
      if (e & 1) ps[e >> 3][(e & 7) >> 1] = hand_over(p[e - 1], p[e]);
    }
    ph[t & 1][rh][0][lane] = ps[0];
    ph[t & 1][rh][1][lane] = ps[1];
    accumulate(obuf[at], tf, pf);
  };
  // the one row that sees a single token (all rows of a sequence of one token do): see the dQ kernel
  const int lone = a.unit == 1 ? s.nq - s.nk : -1;
  // role 1, step t + 1: dS and dK of step t's rows [i, i + 32)
  auto ds_step = [&](int t, int i, f32x16 dp) __attribute__((always_inline)) {
    const u32x4 ps[2] = {ph[t & 1][rh][0][lane], ph[t & 1][rh][1][lane]};
    bf16x8 tf[MB];
    first_half(qbuf[t & 3], tf);
    __builtin_amdgcn_sched_barrier(0);
    if (s.nk == 1) dp = zero16();
    if (lone >= i && lone < i + kTile) {
      const int r = lone - i - 4 * kg;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (8 * (e >> 2) + (e & 3) == r) dp[e] = 0.0f;
    }
    bf16x8 ds[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) ds[e >> 3][e & 7] = (__bf16)(taken_over(ps[e >> 3][(e & 7) >> 1], e & 1) * dp[e]);
    accumulate(qbuf[t & 3], tf, ds);
  };
  int wi = wi0;               // rows of the present step
  if (steps > 0) {
    constexpr int kLoads = 2 * LPW + 1;       // of a request
    // everyone's share of what was requested two steps ago has landed, and nobody reads what the next request replaces
    auto meet = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(kLoads));
      lds_barrier();
      request();              // (past the last step: zeros, or rows of the next group)
    };
    request();
    request();
    meet();
    // the roles meet at the same barriers
    int cur = 0;
    auto next = [&]() __attribute__((always_inline)) {
      wi += kTile;
      if (wi >= s.nq) wi = i_first;
      cur = cur == 2 ? 0 : cur + 1;
      meet();
    };
    if (!is_ds) {
      p_step(0, 0, 0, wi);
      for (int t = 1; t < steps; ++t) {
        next();
        p_step(t, t & 3, cur, wi);
        __builtin_amdgcn_sched_barrier(0);
      }
      lds_barrier();
    } else {
      Frag f[KS];
      f32x16 dp_prev = stats16(0);
      rows_of(obuf[0], f);
      dp_prev = product(f, dp_prev);
      for (int t = 1; t < steps; ++t) {
        const int wp = wi;
        next();
        rows_of(obuf[cur], f);
        f32x16 dp = stats16(cur);
        __builtin_amdgcn_sched_barrier(0);
        dp = product(f, dp);
        ds_step(t - 1, wp, dp_prev);
        dp_prev = dp;
        __builtin_amdgcn_sched_barrier(0);
      }
      lds_barrier();
      ds_step(steps - 1, wi, dp_prev);
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  }
  if constexpr (SPLIT > 1) {
    // the other groups leave their sums where the tiles were (none is on its way any more), the first adds them to its own
    constexpr int N = MB * 4 * 64;
    static_assert((SPLIT - 1) * 4 * N <= SPLIT * 7 * T32, "the sums fit the stages");
    f32x4* const sums = reinterpret_cast<f32x4*>(&buf_all[0][0][0]);
    f32x4* const mine = sums + ((group - 1) * 4 + 2 * is_ds + rh) * N;
    __syncthreads();
    if (group > 0) {
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int g = 0; g < 4; ++g) mine[(4 * mb + g) * 64 + lane] = f32x4{acc[mb][4 * g], acc[mb][4 * g + 1], acc[mb][4 * g + 2], acc[mb][4 * g + 3]};
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int o = 1; o < SPLIT; ++o) {
      const f32x4* theirs = sums + ((o - 1) * 4 + 2 * is_ds + rh) * N;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 y = theirs[(4 * mb + g) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[mb][4 * g + e] += y[e];
        }
    }
  }
  if (!ok) return;
  uint16_t* op = is_ds ? a.dK + (int64_t)hk * a.k_head + token * a.k_tok : a.dV + (int64_t)hk * a.v_head + token * a.v_tok;
  const float factor = is_ds ? a.scale : 1.0f;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 o4;
#pragma unroll
      for (int e = 0; e < 4; ++e) o4[e] = (__bf16)(acc[mb][4 * g + e] * factor);
      *reinterpret_cast<bf16x4*>(op + 32 * mb + 8 * g + 4 * kg) = o4;
    }
}

template <int D> int launch(const PackedArgs& a, hipStream_t st) {
  if (a.q_len > 0) {
    PackedArgs q = a;
    q.slots = a.q_len / 128 + a.seqs;
    const dim3 grid((unsigned)((int64_t)q.slots * a.H));
    if (lf_launch(lf_packed_dq_kernel<D>, grid, dim3(256), 0, st, q) != hipSuccess) return LF_ERR_HIP;
  }
  if (a.kv_len == 0) return LF_OK;
  // 256 tokens of a workgroup with 112 of them or more; where rows see the tokens ahead of them only, so that the first workgroups work longest, 352
  // (both gradients, us, with them and with the better of the two below: 12 heads of 2048 tokens 161 and 136, 2731 230 and 255; causal, 32 heads on 4 of
  // 16 384 tokens 9195 and 8191, 24 000 15 871 and 16 815; by chunks of 512, 12 heads of 4096 304 and 252, 8192 697 and 746).  Those are single sequences.  Short ones
  // leave wavefronts of 64 tokens without any, which the rule does not look at (12 heads, 100 sequences of 300 tokens 464 and 407, 500 of 64 357 and 262).
  if (D == 128 && (int64_t)a.kv_len * a.Hk >= 256 * (a.unit ? 352 : 112)) return lf_launch_packed_dkv_wide(a, st);
  constexpr int kSplit = D == 128 ? 2 : 4;       // groups that a compute unit's LDS has room for
  const int64_t blocks = (int64_t)(a.kv_len / 64 + a.seqs) * a.Hk;
  // several groups to a workgroup while a compute unit has two of them or fewer (divided and not: 32 heads on 4 of 128, 8192 tokens, causal 2174 and
  // 2513, 12 000 tokens 4710 and 4384; 8 heads of 64, 2048 tokens, causal 67 and 81; 256 sequences of 200 tokens, 8 heads on 2 of 64, 239 and 197; but 12 heads of 128, 2048
  // tokens, 144 and 136).  Few tokens under many rows leave compute units without work either way (12 heads, 32 760 rows over 512 tokens 725 and 926).
  const bool split = (int64_t)(a.kv_len / 64 + a.seqs - 1) * a.Hk <= 2 * 256;
  const hipError_t rc = split ? lf_launch(lf_packed_dkv_kernel<D, kSplit>, dim3((unsigned)blocks), dim3(256 * kSplit), 0, st, a)
                              : lf_launch(lf_packed_dkv_kernel<D, 1>, dim3((unsigned)blocks), dim3(256), 0, st, a);
  return rc == hipSuccess ? LF_OK : LF_ERR_HIP;
}

}  // namespace

int lf_launch_packed_bwd(const lf_packed_call* c, void* stream) {
  PackedArgs a = lf_packed_args(c);
  a.ndelta = (float*)c->workspace;
  a.nlse = a.ndelta + (int64_t)a.H * a.q_len;
  a.parts = 1;
  return c->s->head_dim == 128 ? launch<128>(a, (hipStream_t)stream) : launch<64>(a, (hipStream_t)stream);
}
