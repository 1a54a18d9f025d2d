// dK and dV of the packed attention at head dimension 128, for calls with enough tokens: one wavefront per SIMD, 64 tokens of a wavefront.
//
//   P = exp2(c (S - lse2 / c)),  S = Q K^T      dP = dO V^T      dV^T += dO^T P      dS = P (dP - delta)      dK^T += Q^T dS
//
// A workgroup has 256 tokens of a head of K and V and walks the rows that see them, head by head, in tiles of 32 that its four wavefronts share (three
// stages in LDS).  A wavefront keeps its 64 rows of V in registers (64), its sums of dK and dV in the accumulation half of the register
// file (256), and S and dP of a tile (64); its rows of K wait in LDS.  Every fragment of Q and dO that it reads from LDS feeds two products, one for each half of its tokens, and P never
// leaves its registers, so dS is rounded once.  With 32 tokens a wavefront and two wavefronts a SIMD, each with one role, LDS reads were the
// bound (as many bytes as a compute unit's LDS delivers while the products run).
//
// A step on a tile is 64 slots of one matrix instruction each (32 cycles), in four phases of 16: S, dP, dV, dK.  The exponentials stand beside
// dP and the first half of dV, dS beside dV, the LDS reads of a fragment some slots ahead of its product; sched_barrier keeps them there.  S and dP start from
// -lse2 / c and -delta, so no subtraction is left.  The products into the accumulation registers are inline assembly (left to itself the compiler copies the
// sums around the loop); two wait states stand ahead of each, since the compiler does not count those behind the vector instruction that packed its operand.
//
// Seven chunks of 4680 tokens, 12 heads: 5.92 ms (1274 TFLOP/s of its four products; with 32 tokens of a wavefront 12.0 ms).  The matrix pipes are busy 63 % of
// the cycles; the rest is issue of the vector instructions, and the chip's power holds the clock at 1.9 GHz.
#include "lf_packed.h"

namespace {

constexpr int D = 128, CH = D / 8, KS = D / 16, MB = D / 32;
constexpr int kTile = 32, kTokens = 256;
constexpr int T32 = kTile * CH;           // 16-byte chunks of a tile of Q or dO
constexpr uint32_t kBytes = T32 * 16;

struct Stages {
  u32x4 q[3][T32], o[3][T32];
  u32x4 k[4][2 * T32];                    // K of each wavefront's 64 tokens
  f32x4 nl[3][16], nd[3][16];             // -lse2 / c and -delta of the 32 rows; the upper halves take what the other lanes load
};

// A tile is read both ways: rows, and transposed (half a wavefront takes four chunks of each of four rows).
__device__ __forceinline__ int both_swz(int row, int ch) { return ch ^ (((row & 3) << 2) | ((row >> 2) & 3)); }

typedef __attribute__((address_space(3))) const u32x4* LdsRow;
typedef __attribute__((address_space(3))) const f32x4* LdsStat;

__global__ __launch_bounds__(256, 1) void lf_packed_dkv_wide_kernel(PackedArgs a) {
  __shared__ Stages st;
  int x = blockIdx.x;
  const int hk = x % a.Hk, place = x / a.Hk;
  int tile;
  const int b = find_tile(a.kv_start, a.seqs, a.kv_len, 1, kTokens, place, tile);
  const Span s = span_of(a, b);
  const int j0 = tile * kTokens;
  if (tile < 0 || j0 >= s.nk) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ln = lane & 31, kg = lane >> 5;
  const int jw = j0 + 64 * wave;
  // the first rows that see this lane's tokens and the wavefront's last one
  int from[2];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) from[hh] = first_row(s, a.unit, jw + 32 * hh + ln);
  const int from_last = first_row(s, a.unit, min(jw + 63, s.nk - 1));
  const int i_first = first_row(s, a.unit, j0) / kTile * kTile;
  const int tiles = i_first < s.nq ? (s.nq - i_first + kTile - 1) / kTile : 0, steps = tiles * a.G;
  // the one row that sees a single token has no gradient of its scores (all rows of a sequence of one token: nk = 1)
  const int lone = a.unit == 1 ? s.nq - s.nk : -1;

  bf16x8 vf[2][KS];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    const int j = jw + 32 * hh + ln;
    const int64_t token = (int64_t)s.k0 + j;
    const uint16_t* vp = a.V + (int64_t)hk * a.v_head + token * a.v_tok + 8 * kg;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      u32x4 v = {0, 0, 0, 0};
      if (j < s.nk) v = *reinterpret_cast<const u32x4*>(vp + 16 * k);
      vf[hh][k] = __builtin_bit_cast(bf16x8, v);
    }
  }
  const uint32_t q_row = (uint32_t)(a.q_tok * 2), o_row = (uint32_t)(a.o_tok * 2);
  uint32_t qoff[2], ooff[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 4 * (2 * wave + i) + lane / CH, p = lane % CH;
    qoff[i] = (uint32_t)r * q_row + (uint32_t)both_swz(r, p) * 16u - 1024u * i;
    ooff[i] = (uint32_t)r * o_row + (uint32_t)both_swz(r, p) * 16u - 1024u * i;
  }
  const uint32_t base = __builtin_amdgcn_readfirstlane(lds_addr(&st));
  const uint32_t st_off = (uint32_t)lane * 4u;
  int ri = i_first, rg = 0;               // where the next request goes: rows [ri, ri + 32) of the sequence, head rg of the group
  auto request = [&](int to) __attribute__((always_inline)) {
    const int h = hk * a.G + rg, n = min(kTile, s.nq - ri);
    const int64_t first = (int64_t)s.q0 + ri;
    fetch<2>(rows_rsrc(a.Q + (int64_t)h * a.q_head, first, n, q_row), lds_addr(st.q[to]) + 2048u * wave, qoff);
    fetch<2>(rows_rsrc(a.dO + (int64_t)h * a.o_head, first, n, o_row), lds_addr(st.o[to]) + 2048u * wave, ooff);
    if (wave < 2) {
      const float* stat = wave == 0 ? a.nlse : a.ndelta;
      const int32x4 rs = aged(rows_rsrc(reinterpret_cast<const uint16_t*>(stat + (int64_t)h * a.q_len), first, n, 4u));
      const uint32_t at = __builtin_amdgcn_readfirstlane(lds_addr(wave == 0 ? st.nl[to] : st.nd[to]));
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(at), "v"(st_off), "s"(rs) : "memory", "m0");
    }
    ri += kTile;
    if (ri >= s.nq) {
      ri = i_first;
      ++rg;
    }
  };
  // Addresses of this lane's fragments in stage 0 of Q: rows, and transposed (rows 8 .. 15 of 16 see chunk bit 1 flipped).
  uint32_t raddr[KS], taddr[2][MB], saddr = base + (uint32_t)offsetof(Stages, nl) + 16u * kg;
#pragma unroll
  for (int k = 0; k < KS; ++k) raddr[k] = base + 16u * (ln * CH + both_swz(ln, 2 * k + kg));
  {
    const int i16 = lane & 15, tr_row = 4 * kg + (i16 >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int col = 32 * mb + tr_col, at = (tr_row * CH + both_swz(tr_row, col >> 3)) * 8 + (col & 7);
      taddr[0][mb] = base + 2u * at;
      taddr[1][mb] = base + 2u * (at ^ 16) + 8u * CH * 16u;
    }
  }
  constexpr uint32_t kO = offsetof(Stages, o), kNd = offsetof(Stages, nd) - offsetof(Stages, nl);
  auto row_frag = [&](uint32_t at, int k) __attribute__((always_inline)) { return __builtin_bit_cast(bf16x8, *(LdsRow)(uintptr_t)(raddr[k] + at)); };
  auto tread = [&](uint32_t at, int u, int mb, int hf) __attribute__((always_inline)) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(uintptr_t)(taddr[hf][mb] + at + 16u * u * CH * 16u));
  };
  auto join = [](const bf16x4& lo, const bf16x4& hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); };
  auto stat4 = [&](f32x16& v, uint32_t at, int g) __attribute__((always_inline)) {
    const f32x4 y = *(LdsStat)(uintptr_t)(saddr + at + 32u * g);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * g + e] = y[e];
  };

  f32x16 dk[2][MB], dv[2][MB];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) dk[hh][mb] = dv[hh][mb] = zero16();
  auto accumulate = [](f32x16& c, const bf16x8& y, const u32x4& z) __attribute__((always_inline)) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(y), "v"(z));
  };

  const uint32_t k_at = (uint32_t)offsetof(Stages, k) + 2u * kBytes * wave;      // from stage 0 of Q
  if (steps > 0) {
    {
      const uint32_t k_row = (uint32_t)(a.k_tok * 2);
      uint32_t koff[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int r = 4 * n + lane / CH, p = lane % CH;
        koff[n] = (uint32_t)r * k_row + (uint32_t)both_swz(r, p) * 16u - 1024u * n;
      }
#pragma unroll
      for (int n = 0; n < 4; ++n)
        fetch<4>(rows_rsrc(a.K + (int64_t)hk * a.k_head, (int64_t)s.k0 + jw + 16 * n, min(16, s.nk - jw - 16 * n), k_row), base + k_at + 4096u * n, koff);
    }
    request(0);
    if (steps > 1) request(1);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    bf16x8 qr[KS], orow[KS], kf[2][KS];
    bf16x4 tlo[2 * MB], thi[2 * MB], ulo[2 * MB], uhi[2 * MB];      // transposed fragments of dO and Q: [k-step MB + channels]
    f32x16 nl, nd, S[2], dP[2];
    u32x4 pk[2][2], ds[2][2];
#pragma unroll
    for (int g = 0; g < 4; ++g) stat4(nl, 0, g);
#pragma unroll
    for (int k = 0; k < 4; ++k) qr[k] = row_frag(0, k);
#pragma unroll
    for (int n = 0; n < 4; ++n) kf[n & 1][n >> 1] = row_frag(k_at + kBytes * (n & 1), n >> 1);
    int i = i_first;              // rows of the present tile
    int cur = 0;                  // its stage
    for (int t = 0; t < steps; ++t) {
      const int nxt = cur == 2 ? 0 : cur + 1, third = nxt == 2 ? 0 : nxt + 1;
      const uint32_t at = cur * kBytes, at_next = nxt * kBytes, st_at = cur * 256u, st_next = nxt * 256u;
      __builtin_amdgcn_sched_barrier(0);
      // S
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        const int k = n >> 1, hh = n & 1;
        S[hh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qr[k], kf[hh][k], k == 0 ? nl : S[hh], 0, 0, 0);
        if (n + 4 < 16) kf[hh][k + 2] = row_frag(k_at + kBytes * hh, k + 2);
        if (n < 8 && !(n & 1)) qr[4 + k] = row_frag(at, 4 + k);
        if (n >= 8 && !(n & 1)) orow[k - 4] = row_frag(kO + at, k - 4);
        if (n >= 8 && (n & 1)) stat4(nd, kNd + st_at, k - 4);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (i < from_last || i + kTile > s.nq) {      // (rows behind the last one were loaded as zeros, their statistics too)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = i + 8 * (e >> 2) + 4 * kg + (e & 3);
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
            if (r < from[hh] || r >= s.nq) S[hh][e] = -INFINITY;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      // Value v of 32 (values 0 .. 7 of both halves, then 8 .. 15) is scaled at beat v, exp2 at the next and packed (odd v) at the one behind, dS a slot
      // ahead of where it is packed: no instruction waits for the one before it.
      float y[4];
      auto stay = [](auto& w) __attribute__((always_inline)) { asm volatile("" : "+v"(w)); };      // in its slot
      auto half_of = [](int v) { return (v >> 3) & 1; };
      auto at_of = [](int v) { return 8 * (v >> 4) + (v & 7); };
      auto beat = [&](int n) __attribute__((always_inline)) {
        if (n >= 2 && n < 34 && (n & 1)) {
          const int v = n - 2, hh = half_of(v);
          const bf16x2 p = {(__bf16)S[hh][at_of(v) - 1], (__bf16)S[hh][at_of(v)]};
          uint32_t w = __builtin_bit_cast(uint32_t, p);
          stay(w);
          pk[hh][v >> 4][(v & 7) >> 1] = w;
        }
        if (n >= 1 && n < 33) {
          float w = __builtin_amdgcn_exp2f(y[(n - 1) & 3]);
          stay(w);
          S[half_of(n - 1)][at_of(n - 1)] = w;
        }
        if (n < 32) {
          y[n & 3] = S[half_of(n)][at_of(n)] * a.c;
          stay(y[n & 3]);
        }
      };
      auto grad = [&](int v) __attribute__((always_inline)) {
        float w = dP[half_of(v)][at_of(v)] * S[half_of(v)][at_of(v)];
        stay(w);
        dP[half_of(v)][at_of(v)] = w;
      };
      auto pack = [&](int v) __attribute__((always_inline)) {        // v odd
        const int hh = half_of(v);
        const bf16x2 p = {(__bf16)dP[hh][at_of(v) - 1], (__bf16)dP[hh][at_of(v)]};
        uint32_t w = __builtin_bit_cast(uint32_t, p);
        stay(w);
        ds[hh][v >> 4][(v & 7) >> 1] = w;
      };
      // dP, with 24 of the 32 exponentials
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        const int k = n >> 1, hh = n & 1;
        dP[hh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(orow[k], vf[hh][k], k == 0 ? nd : dP[hh], 0, 0, 0);
        if (n < 8 && !(n & 1)) orow[4 + k] = row_frag(kO + at, 4 + k);
        if (n >= 8) {
          const int mb = (n - 8) >> 1;
          if (n & 1) thi[mb] = tread(kO + at, 0, mb, 1);
          else tlo[mb] = tread(kO + at, 0, mb, 0);
        }
#pragma unroll
        for (int v = n * 3 / 2; v < (n + 1) * 3 / 2; ++v) beat(v);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (s.nk == 1 || (lone >= i && lone < i + kTile)) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (s.nk == 1 || i + 8 * (e >> 2) + 4 * kg + (e & 3) == lone) dP[0][e] = dP[1][e] = 0.0f;
        __builtin_amdgcn_sched_barrier(0);
      }
      // dV, with the others and dS
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        const int u = n >> 3, mb = (n >> 1) & 3, hh = n & 1;
        accumulate(dv[hh][mb], join(tlo[u * MB + mb], thi[u * MB + mb]), pk[hh][u]);
        if (n < 8) {
          if (n & 1) thi[MB + mb] = tread(kO + at, 1, mb, 1);
          else tlo[MB + mb] = tread(kO + at, 1, mb, 0);
          beat(24 + n);
          if (n == 7) {
            beat(32);
            beat(33);
          }
        } else {
          if (n & 1) uhi[mb] = tread(at, 0, mb, 1);
          else ulo[mb] = tread(at, 0, mb, 0);
        }
        if (n > 0) pack(2 * n - 1);
        grad(2 * n);
        grad(2 * n + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      // the next tile has landed for everyone, and nobody reads the tile before this one any more
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (t + 2 < steps) request(third);
      __builtin_amdgcn_sched_barrier(0);
      // dK, with the first reads of the next tile
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        const int u = n >> 3, mb = (n >> 1) & 3, hh = n & 1;
        accumulate(dk[hh][mb], join(ulo[u * MB + mb], uhi[u * MB + mb]), ds[hh][u]);
        if (n == 0) pack(31);
        if (n < 8) {
          if (n & 1) uhi[MB + mb] = tread(at, 1, mb, 1);
          else ulo[MB + mb] = tread(at, 1, mb, 0);
        } else {
          if (n & 1) qr[(n - 8) >> 1] = row_frag(at_next, (n - 8) >> 1);
          else stat4(nl, st_next, (n - 8) >> 1);
          if (n >= 12) kf[n & 1][(n - 12) >> 1] = row_frag(k_at + kBytes * (n & 1), (n - 12) >> 1);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      i += kTile;
      if (i >= s.nq) i = i_first;
      cur = nxt;
    }
  }
  // the last products have been written
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    asm volatile("s_nop 15\n\ts_nop 7" : "+a"(dk[hh][0]), "+a"(dk[hh][1]), "+a"(dk[hh][2]), "+a"(dk[hh][3]));
    asm volatile("s_nop 0" : "+a"(dv[hh][0]), "+a"(dv[hh][1]), "+a"(dv[hh][2]), "+a"(dv[hh][3]));
  }
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    const int j = jw + 32 * hh + ln;
    const int64_t token = (int64_t)s.k0 + j;
    if (j >= s.nk) continue;
    uint16_t* kp = a.dK + (int64_t)hk * a.k_head + token * a.k_tok + 4 * kg;
    uint16_t* vp = a.dV + (int64_t)hk * a.v_head + token * a.v_tok + 4 * kg;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 y, z;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = (__bf16)(dk[hh][mb][4 * g + e] * a.scale);
          z[e] = (__bf16)dv[hh][mb][4 * g + e];
        }
        *reinterpret_cast<bf16x4*>(kp + 32 * mb + 8 * g) = y;
        *reinterpret_cast<bf16x4*>(vp + 32 * mb + 8 * g) = z;
      }
  }
}

}  // namespace

int lf_launch_packed_dkv_wide(const PackedArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)(a.kv_len / kTokens + a.seqs) * a.Hk));
  return lf_launch(lf_packed_dkv_wide_kernel, grid, dim3(256), 0, st, a) == hipSuccess ? LF_OK : LF_ERR_HIP;
}
