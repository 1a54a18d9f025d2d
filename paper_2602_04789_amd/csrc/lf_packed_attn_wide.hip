// Attention over packed sequences at head dimension 128, for calls of many rows that see many tokens: one wavefront per SIMD, 64 rows of a wavefront.
//
// As lf_packed_attn.hip, with 256 rows of a workgroup: a fragment of K or V that a wavefront reads from LDS feeds two products, one for each half of its
// rows, so LDS delivers half as much for a product.  The rows of Q and the sums of O are in the accumulation half of the register file.
//
// A step works on a tile of 32 tokens in 32 slots of one matrix instruction each: S of tile t + 1, and then O += V^T P of tile t - 1, with the
// exponentials of tile t beside both, one to a slot and in stages of a slot each; sched_barrier keeps the slots as written.  Steps go
// in pairs, whose scores and probabilities change places; a wavefront's last pair may end on a tile that its rows do not see.  K and V have four
// stages each, and a tile is requested two steps ahead of its use; the workgroup meets once a step, between the two halves.  The stages that a pair uses
// change with bit 14 of the LDS addresses.
// The products into the accumulation registers are inline assembly, two wait states ahead of each (see lf_packed_dkv_wide.hip).
//
// 4680 rows of 12 heads over 16 384 tokens: 422 us (1117 TFLOP/s; 435 with 32 rows of a wavefront); seven chunks of 4680 tokens 3.26 ms (3.28).
// The matrix pipes are busy 59 % of the cycles, the rest is issue of the exponentials, and the chip's power holds the clock at 1.8 to 2.0 GHz.
#include "lf_packed.h"

namespace {

constexpr int D = 128, CH = D / 8, KS = D / 16, MB = D / 32;
constexpr int kTile = 32, kRows = 256;
constexpr int T32 = kTile * CH;
constexpr uint32_t kBytes = T32 * 16;           // 8 KB
constexpr uint32_t kPair = 2 * kBytes;          // a pair of stages: one bit of an address
static_assert(kPair == 1u << 14, "pairs of stages change with one bit");

struct Stages {
  u32x4 k[4][T32], v[4][T32];
};
__device__ __forceinline__ int v_swz(int row, int ch) { return ch ^ ((row & 3) << 2); }
typedef __attribute__((address_space(3))) const u32x4* LdsRow;

__global__ __launch_bounds__(256, 1) void lf_packed_attn_wide_kernel(PackedArgs a) {
  __shared__ __attribute__((aligned(32768))) Stages st;
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
  int lim[2];
  bf16x8 qf[2][KS];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    const int row = 64 * wave + 32 * hh + ln;
    lim[hh] = row_limit(s, a.unit, min(i0 + row, s.nq - 1));
    const uint16_t* qp = a.Q + (int64_t)h * a.q_head + ((int64_t)s.q0 + i0 + row) * a.q_tok + 8 * kg;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      u32x4 u = {0, 0, 0, 0};
      if (row < rows) u = *reinterpret_cast<const u32x4*>(qp + 16 * k);
      qf[hh][k] = __builtin_bit_cast(bf16x8, u);
    }
  }
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int k = 0; k < KS; ++k) asm volatile("" : "+a"(qf[hh][k]));
  const int lim_first = row_limit(s, a.unit, min(i0 + 64 * wave, s.nq - 1));
  const int seen = row_limit(s, a.unit, i0 + rows - 1);
  const int lim_last = 64 * wave < rows ? row_limit(s, a.unit, i0 + min(64 * wave + 63, rows - 1)) : 0;
  // steps of the workgroup and of the wavefront, in pairs
  const int nt = (seen + 2 * kTile - 1) / (2 * kTile) * 2, nw = (lim_last + 2 * kTile - 1) / (2 * kTile) * 2;

  const uint16_t* Kh = a.K + (int64_t)hk * a.k_head;
  const uint16_t* Vh = a.V + (int64_t)hk * a.v_head;
  const uint32_t k_row = (uint32_t)(a.k_tok * 2), v_row = (uint32_t)(a.v_tok * 2);
  uint32_t koff[2], voff[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 4 * (2 * wave + i) + lane / CH, p = lane % CH;
    koff[i] = (uint32_t)r * k_row + (uint32_t)row_swz<CH>(r, p) * 16u - 1024u * i;
    voff[i] = (uint32_t)r * v_row + (uint32_t)v_swz(r, p) * 16u - 1024u * i;
  }
  const uint32_t base = __builtin_amdgcn_readfirstlane(lds_addr(&st));
  // tile t of K or V into its stage; a tile that is not there is zeros
  auto request = [&](const uint16_t* of, int t, uint32_t row_bytes, uint32_t region, const uint32_t (&off)[2]) __attribute__((always_inline)) {
    const int n = t < 0 ? 0 : min(kTile, seen - t * kTile);
    fetch<2>(rows_rsrc(of, (int64_t)s.k0 + max(t, 0) * kTile, n, row_bytes), base + region + (uint32_t)(t & 3) * kBytes + 2048u * wave, off);
  };
  constexpr uint32_t kV = offsetof(Stages, v);
  auto requests = [&](int t) __attribute__((always_inline)) {
    request(Kh, t + 4, k_row, 0, koff);
    request(Vh, t + 2, v_row, kV, voff);
  };
  uint32_t raddr[KS], taddr[MB];
#pragma unroll
  for (int k = 0; k < KS; ++k) raddr[k] = base + 16u * (ln * CH + row_swz<CH>(ln, 2 * k + kg));
  {
    const int i16 = lane & 15, tr_row = 4 * kg + (i16 >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int col = 32 * mb + tr_col;
      taddr[mb] = base + kV + 2u * ((tr_row * CH + v_swz(tr_row, col >> 3)) * 8 + (col & 7));
    }
  }
  auto row_frag = [&](uint32_t at, int k) __attribute__((always_inline)) { return __builtin_bit_cast(bf16x8, *(LdsRow)(uintptr_t)(raddr[k] + at)); };
  auto tread = [&](uint32_t at, int u, int mb, int hf) __attribute__((always_inline)) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(uintptr_t)(taddr[mb] + at + (16u * u + 8u * hf) * CH * 16u));
  };
  auto join = [](const bf16x4& lo, const bf16x4& hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); };

  f32x16 o[2][MB];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[hh][mb] = zero16();
  auto accumulate = [](f32x16& c, const bf16x8& y, const u32x4& z) __attribute__((always_inline)) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(y), "v"(z));
  };
  // waits for the products on their way into O, and behind a change of O ahead of the next ones
  auto settle = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) asm volatile("s_nop 15\n\ts_nop 3" : "+a"(o[hh][0]), "+a"(o[hh][1]), "+a"(o[hh][2]), "+a"(o[hh][3]));
  };
  constexpr float kSumMax = 1.0e30f;
  float m_run[2] = {-1.0e30f, -1.0e30f};
  f32x4 l_run[2];            // a lane's four results are all the sum of its own values
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) l_run[hh] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  const s16x4 ones = {0x3f80, 0x3f80, 0x3f80, 0x3f80};
  bf16x8 kr[KS];
  bf16x4 tlo[2 * MB], thi[2 * MB];
  f32x16 S[2][2];
  u32x4 P[2][2][2];           // [step mod 2][half][k-step]
  if (nt > 0) {
    requests(-4);
    requests(-3);
    requests(-2);
    requests(-1);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(8));       // K of tiles 0 and 1; V of "tile -1" is zeros
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int u = 0; u < 2; ++u) P[1][hh][u] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const bf16x8 f = row_frag(0, k);
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) S[0][hh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[hh][k], k == 0 ? zero16() : S[0][hh], 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) kr[k] = row_frag(kBytes, k);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) taddr[mb] ^= kPair;      // the pair before the first
    // everyone's share of what was requested two steps ago has landed, and nobody reads what the next requests replace
    auto meet = [&](int t) __attribute__((always_inline)) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(4));
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      requests(t);
    };
    auto products = [&](uint32_t at, const u32x4 (&p)[2][2], auto beside) __attribute__((always_inline)) {
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        const int u = n >> 3, mb = (n >> 1) & 3, hh = n & 1;
        accumulate(o[hh][mb], join(tlo[u * MB + mb], thi[u * MB + mb]), p[hh][u]);
        if (n < 8) {
          if (n & 1) thi[MB + mb] = tread(at, 1, mb, 1);
          else tlo[MB + mb] = tread(at, 1, mb, 0);
        }
        beside(n);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto step = [&](int t, auto odd) __attribute__((always_inline)) {
      constexpr int c = decltype(odd)::value;             // S[c], P[c]: this tile's; the others the next tile's S and the last one's P
      constexpr uint32_t k_at = c ? 0u : kBytes, k_next = c ? kBytes : 0u, v_at = c ? 0u : kBytes;
      f32x16 (&sc)[2] = S[c];
      f32x16 (&sn)[2] = S[1 - c];
      u32x4 (&pc)[2][2] = P[c];
      __builtin_amdgcn_sched_barrier(0);
      if ((t + 1) * kTile > lim_first) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (t * kTile + 8 * (e >> 2) + 4 * kg + (e & 3) >= lim[hh]) sc[hh][e] = -INFINITY;
        __builtin_amdgcn_sched_barrier(0);
      }
      const float l_old[2] = {l_run[0][0], l_run[1][0]};
      // Value v of 32 (values 0 .. 7 of both halves, then 8 .. 15) is scaled at beat v, exp2 at the next, packed (odd v) at the one behind and, four at a time,
      // added to the row's sum at the last: no instruction waits for the one before it. 
      float x[4], y[4];
      auto stay = [](auto& w) __attribute__((always_inline)) { asm volatile("" : "+v"(w)); };      // in its slot
      auto half_of = [](int v) { return (v >> 3) & 1; };
      auto scale_of = [&](int v) __attribute__((always_inline)) {
        x[v & 3] = fmaf(sc[half_of(v)][8 * (v >> 4) + (v & 7)], a.c, -m_run[half_of(v)]);
        stay(x[v & 3]);
      };
      auto exp_of = [&](int v) __attribute__((always_inline)) {
        y[v & 3] = __builtin_amdgcn_exp2f(x[v & 3]);
        stay(y[v & 3]);
      };
      auto pack_of = [&](int v) __attribute__((always_inline)) {
        const bf16x2 p = {(__bf16)y[(v - 1) & 3], (__bf16)y[v & 3]};
        uint32_t q = __builtin_bit_cast(uint32_t, p);
        stay(q);
        pc[half_of(v)][v >> 4][(v & 7) >> 1] = q;
      };
      auto sum_of = [&](int v) __attribute__((always_inline)) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const int hh = half_of(v), u = v >> 4;
        const u32x2 four = {pc[hh][u][((v & 7) >> 1) - 1], pc[hh][u][(v & 7) >> 1]};
        l_run[hh] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones, __builtin_bit_cast(s16x4, four), l_run[hh], 0, 0, 0);
      };
      auto beat = [&](int n) __attribute__((always_inline)) {
        if (n >= 2 && n < 34 && (n & 1)) pack_of(n - 2);
        if (n >= 1 && n < 33) exp_of(n - 1);
        if (n < 32) scale_of(n);
        if (n >= 6 && ((n - 3) & 3) == 3) sum_of(n - 3);
      };
      auto prob = [&](int n) __attribute__((always_inline)) {       // slot n
        if (n < 3) {
          beat(2 * n);
          beat(2 * n + 1);
        } else {
          beat(n + 3);
        }
      };
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        const int k = n >> 1, hh = n & 1;
        sn[hh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kr[k], qf[hh][k], k == 0 ? zero16() : sn[hh], 0, 0, 0);
        if (n < 8 && !(n & 1)) kr[4 + k] = row_frag(k_at, 4 + k);
        if (n >= 8) {
          const int mb = (n - 8) >> 1;
          if (n & 1) thi[mb] = tread(v_at, 0, mb, 1);
          else tlo[mb] = tread(v_at, 0, mb, 0);
        }
        prob(n);
        __builtin_amdgcn_sched_barrier(0);
      }
      meet(t);
      if constexpr (c == 0) {
#pragma unroll
        for (int k = 0; k < KS; ++k) raddr[k] ^= kPair;
      }
      __builtin_amdgcn_sched_barrier(0);
      products(v_at, P[1 - c], [&](int n) __attribute__((always_inline)) {
        if (n >= 8 && !(n & 1)) kr[(n - 8) >> 1] = row_frag(k_next, (n - 8) >> 1);
        prob(16 + n);
      });
      if constexpr (c == 0) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) taddr[mb] ^= kPair;
      }
      if (__ballot(fmaxf(l_run[0][0], l_run[1][0]) > kSumMax) != 0ull) {
        settle();
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          float top = sc[hh][0];
#pragma unroll
          for (int e = 1; e < 16; ++e) top = fmaxf(top, sc[hh][e]);
          const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
          top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * a.c;
          const float m_new = fmaxf(m_run[hh], top), alpha = __builtin_amdgcn_exp2f(m_run[hh] - m_new);
          m_run[hh] = m_new;
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[hh][mb][e] *= alpha;
          const float l = l_old[hh] * alpha;
          l_run[hh] = f32x4{l, l, l, l};
        }
        settle();
#pragma unroll
        for (int n = 0; n < 35; ++n) beat(n);
      }
    };
    int t = 0;
    for (; t < nw; t += 2) {
      step(t, std::integral_constant<int, 0>{});
      step(t + 1, std::integral_constant<int, 1>{});
    }
    if (nw > 0) {             // the last tile's products: its V is in the pair's second stage
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(4));
      asm volatile("" ::: "memory");
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        tlo[mb] = tread(kBytes, 0, mb, 0);
        thi[mb] = tread(kBytes, 0, mb, 1);
      }
      products(kBytes, P[1], [](int) {});
    }
    for (; t < nt; ++t) meet(t);            // tiles that this wavefront's rows do not see
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    settle();
  }
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    float l = l_run[hh][0];
    l += __shfl_xor(l, 32);
    const int row = 64 * wave + 32 * hh + ln;
    if (row >= rows) continue;
    const int64_t token = (int64_t)s.q0 + i0 + row;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    if (a.lse2 && kg == 0) a.lse2[(int64_t)h * a.q_len + token] = l > 0.0f ? m_run[hh] + __builtin_log2f(l) : INFINITY;
    uint16_t* op = a.O + (int64_t)h * a.o_head + token * a.o_tok + 4 * kg;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[hh][mb][4 * g + e] * inv);
        *reinterpret_cast<bf16x4*>(op + 32 * mb + 8 * g) = y;
      }
  }
}

}  // namespace

int lf_launch_packed_attn_wide(PackedArgs a, hipStream_t st) {
  a.slots = a.q_len / kRows + a.seqs;
  const dim3 grid((unsigned)((int64_t)a.slots * a.H));
  return lf_launch(lf_packed_attn_wide_kernel, grid, dim3(256), 0, st, a) == hipSuccess ? LF_OK : LF_ERR_HIP;
}
