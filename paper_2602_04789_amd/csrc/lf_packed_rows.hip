// Attention over packed sequences for calls of few rows: single tokens over a long cache, or a few of them.
//
// The rows of a tile are the rows of a sequence with the G heads that share a head of K and V side by side (row i, head g: place i G + g), so that
// K and V are read once for all of them; 16 or 32 such rows are a tile.  HBM bounds the call: 2 d bytes of K and of V a token.  The tokens of a tile
// are divided among workgroups (part_tokens of them at least) and inside one among its four wavefronts, tile of 64 by tile of 64, each with an
// online softmax and with rows of K and V of its own in LDS, so no barrier stands in the loop: what a wavefront has used up it requests again at
// once (K of the next tile while P and the second product are computed, V of it before the next scores), 32 KB of a wavefront at d = 128.
//
// Products transposed, S^T = K Q^T and O^T = V^T P^T, with v_mfma_f32_16x16x32_bf16: the first one leaves a lane the scores of the tokens 4 kg + {0..3}
// of each 16, which are its operand of the second.  P goes into the products in two bfloat16 parts (16 bits) with 16 rows, where bytes are the
// bound, and in one with 32.  The states of the wavefronts are joined through LDS, those of the parts by a launch of their own.
//
// 16 single rows over 120 003 tokens, 40 heads on 8 of 128: 90 us (492 MB, 5.5 TB/s) and 5 for the join.  One row of 12 heads over 77 tokens: 5.4 us.
#include "lf_packed.h"

namespace {

constexpr int kWaves = 4;
constexpr int kTok = 64;
constexpr float kMostSum = 16384.0f;   // a larger sum of a tile's P moves the reference

// V's rows for the transposing read: 16 lanes take 32 bytes (two chunks) of each of four rows, 32 lanes of eight.
template <int CH> __device__ __forceinline__ int pair_swz(int row, int ch) {
  return ch ^ (CH == 16 ? (row & 7) << 1 : (row >> 1 & 3) << 1);
}

template <int D, int NQ>
__global__ __launch_bounds__(64 * kWaves, 1) void lf_packed_rows_kernel(PackedArgs a) {
  constexpr int R = 16 * NQ;
  constexpr int KS = D / 32, MB = D / 16, CH = D / 8;
  constexpr int TILE = kTok * CH;         // 16-byte chunks of K or V of a tile
  constexpr int LD = TILE / 64;           // load instructions for them
  constexpr int RPI = 64 / CH;
  constexpr bool TWO = NQ == 1;
  __shared__ u32x4 kv[kWaves][2 * TILE];
  __shared__ float2 ml[kWaves][R];

  int x = blockIdx.x;
  const int hk = x % a.Hk;
  x /= a.Hk;
  const int place = x % a.slots, part = x / a.slots;      // (parts that a short sequence leaves empty come last)
  int tile;
  const int b = find_tile(a.q_start, a.seqs, a.q_len, a.G, R, place, tile);
  const Span s = span_of(a, b);
  const int64_t i0 = (int64_t)tile * R, all = (int64_t)s.nq * a.G;       // rows and heads
  if (tile < 0 || i0 >= all) return;
  const int rows = (int)min((int64_t)R, all - i0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, kg = lane >> 4;
  const int lim_first = row_limit(s, a.unit, (int)(i0 / a.G)), seen = row_limit(s, a.unit, (int)((i0 + rows - 1) / a.G));
  int t0 = 0, t1 = seen;
  if (a.parts > 1) {
    const int len = part_len(a, seen);
    t0 = (int)min((int64_t)part * len, (int64_t)seen);
    t1 = (int)min((int64_t)t0 + len, (int64_t)seen);
    if (t0 >= t1) return;
  }

  // A lane takes chunk 4 u + kg of a row in step u: 64 bytes of a row side by side.
  Frag qf[NQ][KS];
  int lim[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int64_t at = i0 + min(16 * q + col, rows - 1);
    const int i = (int)(at / a.G), h = hk * a.G + (int)(at % a.G);
    lim[q] = row_limit(s, a.unit, i);
    const uint16_t* p = a.Q + (int64_t)h * a.q_head + (int64_t)(s.q0 + i) * a.q_tok + 8 * kg;
#pragma unroll
    for (int u = 0; u < KS; ++u) qf[q][u].u = *reinterpret_cast<const u32x4*>(p + 32 * u);
  }
  const uint16_t* Kh = a.K + (int64_t)hk * a.k_head;
  const uint16_t* Vh = a.V + (int64_t)hk * a.v_head;
  const uint32_t k_row = (uint32_t)(a.k_tok * 2), v_row = (uint32_t)(a.v_tok * 2);
  u32x4* const kt = kv[wave];
  u32x4* const vt = kt + TILE;
  // offsets of the first four loads (4 RPI rows); the others follow by whole steps of them
  uint32_t koff[4], voff[4];
  static_assert(LD % 4 == 0 && (4 * RPI) % 16 == 0, "the swizzles repeat after 16 rows");
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = RPI * i + lane / CH, p = lane % CH;
    koff[i] = (uint32_t)r * k_row + (uint32_t)row_swz<CH>(r, p) * 16u - 1024u * i;
    voff[i] = (uint32_t)r * v_row + (uint32_t)pair_swz<CH>(r, p) * 16u - 1024u * i;
  }
  auto request = [&](const uint16_t* base, int t, uint32_t row_bytes, const uint32_t (&off)[4], const u32x4* to) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < LD / 4; ++g)
      fetch<4>(rows_rsrc(base, (int64_t)s.k0 + t + 4 * RPI * g, min(4 * RPI, t1 - t - 4 * RPI * g), row_bytes), lds_addr(to + 256 * g), off);
  };
  auto own_lds = []() __attribute__((always_inline)) {    // what this wavefront has read from its rows is in registers
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_s_waitcnt(0xc07f);
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  };
  auto landed = [](auto n) __attribute__((always_inline)) {   // all but the n youngest loads
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(decltype(n)::value));
    asm volatile("" ::: "memory");
  };

  f32x4 oacc[NQ][MB];
  float m_run[NQ], l_run[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    m_run[q] = -1.0e30f;
    l_run[q] = 0.0f;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) oacc[q][mb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;

  const int first = t0 + kTok * wave;
  if (first < t1) {
    request(Kh, first, k_row, koff, kt);
    request(Vh, first, v_row, voff, vt);
  }
  for (int t = first; t < t1; t += kTok * kWaves) {
    const bool more = t + kTok * kWaves < t1;
    landed(std::integral_constant<int, LD>{});      // K of this tile (V's loads are the youngest)
    f32x4 sacc[NQ][4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      Frag kf[KS];
      const int r = 16 * g + col;
#pragma unroll
      for (int u = 0; u < KS; ++u) kf[u].u = kt[r * CH + row_swz<CH>(r, 4 * u + kg)];
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        sacc[q][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < KS; ++u) sacc[q][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u].v, qf[q][u].v, sacc[q][g], 0, 0, 0);
      }
    }
    own_lds();
    if (more) request(Kh, t + kTok * kWaves, k_row, koff, kt);
    if (t + kTok > lim_first) {
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (t + 16 * (i >> 2) + 4 * kg + (i & 3) >= lim[q]) sacc[q][i >> 2][i & 3] = -INFINITY;
    }
    float p[NQ][16];
    bf16x8 pf[NQ][2], rest[2];
    f32x4 sum[NQ];
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[q][i] = __builtin_amdgcn_exp2f(fmaf(sacc[q][i >> 2][i & 3], a.c, -m_run[q]));
#pragma unroll
        for (int i = 0; i < 16; ++i) pf[q][i >> 3][i & 7] = (__bf16)p[q][i];
        sum[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) sum[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[q][hf], sum[q], 0, 0, 0);
      }
    };
    weights();
    bool past = false;
#pragma unroll
    for (int q = 0; q < NQ; ++q) past = past || sum[q][0] > kMostSum;
    if (__ballot(past) != 0ull) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        float top = sacc[q][0][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, sacc[q][i >> 2][i & 3]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32)) * a.c;
        const float m_new = fmaxf(m_run[q], top), alpha = __builtin_amdgcn_exp2f(m_run[q] - m_new);
        m_run[q] = m_new;
        l_run[q] *= alpha;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 4; ++i) oacc[q][mb][i] *= alpha;
      }
      weights();
    }
    if constexpr (TWO) {      // what P's rounding left off
#pragma unroll
      for (int i = 0; i < 16; ++i) rest[i >> 3][i & 7] = (__bf16)(p[0][i] - (float)pf[0][i >> 3][i & 7]);
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) sum[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, rest[hf], sum[0], 0, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) l_run[q] += sum[q][0];
    if (more) landed(std::integral_constant<int, LD>{});      // V of this tile (K's next loads are the youngest)
    else landed(std::integral_constant<int, 0>{});
    const uint16_t* v16 = reinterpret_cast<const uint16_t*>(vt);
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      bf16x8 vf[MB];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        const int r = 4 * kg + (col >> 2), c = 16 * mb + 4 * (col & 3);
        const int off = (r * CH + pair_swz<CH>(r, c >> 3)) * 8 + (c & 7) + 32 * hf * CH * 8;     // (16 rows on the swizzle is the same)
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(bf16x4, v16 + off));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(bf16x4, v16 + off + 16 * CH * 8));
        vf[mb] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int q = 0; q < NQ; ++q) oacc[q][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[mb], pf[q][hf], oacc[q][mb], 0, 0, 0);
      if constexpr (TWO) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) oacc[0][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[mb], rest[hf], oacc[0][mb], 0, 0, 0);
      }
    }
    own_lds();
    if (more) request(Vh, t + kTok * kWaves, v_row, voff, vt);
  }

  // The states of the wavefronts become one: wavefront w adds and writes a quarter of the channels.
#pragma unroll
  for (int q = 0; q < NQ; ++q)
    if (kg == 0) ml[wave][16 * q + col] = make_float2(m_run[q], l_run[q]);
  __syncthreads();        // (every wavefront has used its rows up: their place takes the sums)
  f32x4* const buf = reinterpret_cast<f32x4*>(&kv[0][0]);
  static_assert(sizeof(kv) >= (size_t)NQ * MB * kWaves * 64 * 16, "sums of all wavefronts");
  float M[NQ], L[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    M[q] = -INFINITY;
    L[q] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M[q] = fmaxf(M[q], ml[w][16 * q + col].x);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 y = ml[w][16 * q + col];
      L[q] += y.y * __builtin_amdgcn_exp2f(y.x - M[q]);
    }
    const float f = __builtin_amdgcn_exp2f(m_run[q] - M[q]);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      f32x4 o = oacc[q][mb];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= f;
      buf[((q * MB + mb) * kWaves + wave) * 64 + lane] = o;
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int r = 16 * q + col;
    const int64_t at = i0 + min(r, rows - 1);
    const int64_t token = (int64_t)s.q0 + at / a.G;
    const int h = hk * a.G + (int)(at % a.G);
    const int64_t state = (((int64_t)place * a.Hk + hk) * a.parts + part) * R + r;
    const float inv = L[q] > 0.0f ? 1.0f / L[q] : 0.0f;
    if (r < rows && wave == 0 && kg == 0) {
      if (a.parts > 1) a.state_ml[state] = make_float2(M[q], L[q]);
      else if (a.lse2) a.lse2[(int64_t)h * a.q_len + token] = L[q] > 0.0f ? M[q] + __builtin_log2f(L[q]) : INFINITY;
    }
#pragma unroll
    for (int k = 0; k < MB / kWaves; ++k) {
      const int mb = k * kWaves + wave;
      f32x4 o = buf[(q * MB + mb) * kWaves * 64 + lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        const f32x4 y = buf[((q * MB + mb) * kWaves + w) * 64 + lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += y[i];
      }
      if (r >= rows) continue;
      if (a.parts > 1) {
        *reinterpret_cast<f32x4*>(a.state_o + state * D + 16 * mb + 4 * kg) = o;
      } else {
        bf16x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (__bf16)(o[i] * inv);
        *reinterpret_cast<bf16x4*>(a.O + (int64_t)h * a.o_head + token * a.o_tok + 16 * mb + 4 * kg) = y;
      }
    }
  }
}

}  // namespace

int lf_launch_packed_rows(const lf_packed_call* c, void* stream) {
  const PackedArgs a = lf_packed_args(c);
  const int d = c->s->head_dim, tile = c->plan.tile;
  hipStream_t st = (hipStream_t)stream;
  auto kernel = d == 128 ? (tile == 16 ? lf_packed_rows_kernel<128, 1> : lf_packed_rows_kernel<128, 2>)
                         : (tile == 16 ? lf_packed_rows_kernel<64, 1> : lf_packed_rows_kernel<64, 2>);
  const dim3 grid((unsigned)((int64_t)a.slots * a.Hk * a.parts));
  if (lf_launch(kernel, grid, dim3(64 * kWaves), 0, st, a) != hipSuccess) return LF_ERR_HIP;
  return a.parts > 1 ? lf_launch_packed_join(a, d, tile, true, st) : LF_OK;
}
