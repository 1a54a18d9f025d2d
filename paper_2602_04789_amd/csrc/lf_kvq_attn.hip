// Attention of blocks of up to 64 query rows over a cache held in 4 bits (and rows in bfloat16 behind it).
//
//   O_x = sum_y softmax_y(q_x . k_y scale) v_y,   y over the tokens of the listed blocks, or over all tokens
//
// Few query rows share the cache's bytes, so HBM bounds the call (one row over 131 076 tokens of 12 x 128: 42 us, 5.1 TB/s of codes and scales),
// or the work on a tile where many rows share them (64 rows of 40 x 64 over 32 824 tokens: 43 us, 0.5 PFLOP/s, 2.3 times what the bytes take): two
// wavefronts that share the rows each convert and stage all of it.  A wavefront has up
// to 32 rows of the block (33 to 64 rows: two wavefronts share them; all in one, with tiles half as long, took 55 us there) and tiles of 64 tokens of
// its own: the tiles of a list are dealt out over the four wavefronts of `parts` workgroups, with an online softmax each and nothing shared until
// the end, so no barrier stands in the loop.
//
// The products are computed transposed, S^T = K Q^T and O^T = V^T P^T, with v_mfma_f32_16x16x32_bf16.  Their sums run over
// channels and tokens in any order that both operands agree on.  For S^T a lane takes D/4 neighbouring channels of one token: at d = 128 a
// whole scaled group, 16 bytes and one scale, straight from memory into the operand, through the conversions that apply the
// scale.  For O^T a lane takes the tokens whose scores the first product left it (4 kg + {0..3} of each 16 tokens of the tile),
// so P stays in its registers; V goes through LDS as bfloat16 rows, half a tile at a time, and comes back by the transposing read.  The bytes of
// the next tile are requested as soon as those of the present one are converted.
//
// Softmax is float32 in the exp2 domain, P = exp2(s c - m), against a reference m per row that moves only when a tile's sum of P is large:
// without that no lane asks another and no maximum of scores is taken.  P is rounded to bfloat16 for the product (as the output is); the
// row's sum is the product of the same P with ones, in float32.  Up to 16 rows P goes into both products in two bfloat16 parts, 16 bits: bytes
// bound these calls, so it costs little (one row over 131 076 tokens: 45.9 -> 46.9 us), and the output's 2-norm error falls from 2.6e-3 to the 1.7e-3
// that its own rounding is.  With more rows, and in the bfloat16 kernels, one part is kept: the products and vector work are the bound there.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "lf_rollout.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct KvqAttnArgs {
  const uint16_t *Q, *Kx, *Vx;
  uint16_t* O;
  const uint8_t *kc, *vc, *ks, *vs;
  const int32_t* idx;
  int64_t q_stride_tok, q_stride_head, k_stride_tok, k_stride_head, v_stride_tok, v_stride_head, o_stride_tok, o_stride_head;
  int capacity, cached, extra;
  int n, nb, n_q, n_k, nb_cached;   // lists: blocks [0, nb_cached) lie in the cache
  int list_len, q_len, parts;
  float c;                          // scale * log2(e)
  float* state_o;
  float2* state_ml;
};

constexpr int kWaves = 4;
constexpr float kMostSum = 16384.0f;  // a larger sum of a tile's P moves the reference: P is 2^8 on the mean then, far from overflow

#define LDS_PTR(T, p) ((__attribute__((address_space(3))) T*)(p))

union Frag {
  u32x4 x;
  bf16x2 p[4];
  bf16x8 v;
};

// 8 codes to 8 values.
__device__ __forceinline__ Frag decode(uint32_t code, float scale) {
  Frag f;
  f.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0);
  f.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1);
  f.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2);
  f.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
  return f;
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }   // 255: the conversion gives NaN

// Up to 64 tokens side by side; cnt = 0: none.
struct Tile {
  int tok, cnt;
};

template <int D, int NQ, int RG, bool LISTS>
__global__ __launch_bounds__(64 * kWaves, 2) void lf_kvq_attn_kernel(KvqAttnArgs a) {
  constexpr int KS = D / 32;          // steps of the first product, 8 channels of a lane each
  constexpr int MB = D / 16;          // tiles of 16 channels of the second
  constexpr int CW = D / 32;          // words of codes of a lane and token (D / 4 channels)
  constexpr int CH = D / 8;           // 16-byte chunks of a row in LDS
  constexpr int VI = D / 64;          // scaled groups of half a tile's V for a lane
  constexpr int SL = kWaves / RG;     // tiles at a time
  constexpr bool TWO = NQ == 1;       // P in two bfloat16 parts: up to 16 rows
  __shared__ u32x4 stage[kWaves][32 * CH];
  __shared__ float2 ml[kWaves][16 * NQ];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rg = wave % RG, slot = wave / RG;
  const int col = lane & 15, kg = lane >> 4;
  const int part = blockIdx.x % a.parts, blk = blockIdx.x / a.parts;      // blk: (head, query block)
  const int h = LISTS ? blk / a.n_q : blk, r = LISTS ? blk % a.n_q : 0;
  int row0 = 0, rows = a.q_len;
  if constexpr (LISTS) {
    const int j = r % a.nb;
    row0 = r / a.nb * a.n + 64 * j;
    rows = min(64, a.n - 64 * j);
  }
  const int64_t hrow = (int64_t)h * a.capacity;
  const uint8_t* kc = a.kc + hrow * (D / 2);
  const uint8_t* vc = a.vc + hrow * (D / 2);
  const uint8_t* ks = a.ks + hrow * (D / 32);
  const uint8_t* vs = a.vs + hrow * (D / 32);
  const int32_t* list = LISTS ? a.idx + (int64_t)blk * a.list_len : nullptr;

  Frag qf[NQ][KS];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int row = row0 + min(16 * (NQ * rg + q) + col, rows - 1);
    const uint16_t* p = a.Q + (int64_t)h * a.q_stride_head + (int64_t)row * a.q_stride_tok + (D / 4) * kg;
#pragma unroll
    for (int u = 0; u < KS; ++u) qf[q][u].x = *reinterpret_cast<const u32x4*>(p + 8 * u);
  }

  // The tiles of this wavefront, in turn: every (parts SL)-th entry of the list, or block of 64 tokens; those in the cache (EXT = false), then
  // those behind it.
  const int held = (a.cached + 63) / 64;
  const int units = LISTS ? a.list_len : held + (a.extra + 63) / 64;
  const int stride = a.parts * SL;
  int at, ahead;                // the next entry, and for lists what it says
  auto begin = [&]() __attribute__((always_inline)) {
    at = part * SL + slot;
    ahead = LISTS && at < units ? list[at] : 0;
  };
  auto next = [&](bool ext) __attribute__((always_inline)) {
    Tile t = {0, 0};
    while (at < units && t.cnt == 0) {
      if constexpr (LISTS) {
        const int id = __builtin_amdgcn_readfirstlane(ahead);
        if (at + stride < units) ahead = list[at + stride];
        const int frame = id / a.nb, j = id - frame * a.nb;
        t.tok = (ext ? frame - a.nb_cached / a.nb : frame) * a.n + 64 * j;
        t.cnt = id >= (ext ? a.nb_cached : 0) && id < (ext ? a.n_k : a.nb_cached) ? min(64, a.n - 64 * j) : 0;
      } else if ((at >= held) == ext) {
        t.tok = 64 * (ext ? at - held : at);
        t.cnt = min(64, (ext ? a.extra : a.cached) - t.tok);
      }
      at += stride;
    }
    return t;
  };

  // The bytes of a tile: a lane's D/4 channels of four tokens of K, and its groups of V, half a tile at a time.
  uint32_t kw[4][CW], ksc[4], vw[2][VI][4], vsc[2][VI];
  auto load_k = [&](const Tile& t) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int row = t.tok + min(16 * s + col, t.cnt - 1);
      const uint8_t* p = kc + (uint32_t)(row * (D / 2) + (D / 8) * kg);
      if constexpr (CW == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        kw[s][0] = x.x; kw[s][1] = x.y; kw[s][2] = x.z; kw[s][3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        kw[s][0] = x.x; kw[s][1] = x.y;
      }
      ksc[s] = ks[(uint32_t)(row * (D / 32) + (D == 128 ? kg : kg >> 1))];
    }
  };
  auto load_v = [&](const Tile& t, int half) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const int item = 64 * i + lane, row = t.tok + min(32 * half + item / (D / 32), t.cnt - 1), grp = item % (D / 32);
      const uint4 x = *reinterpret_cast<const uint4*>(vc + (uint32_t)(row * (D / 2) + 16 * grp));
      vw[half][i][0] = x.x; vw[half][i][1] = x.y; vw[half][i][2] = x.z; vw[half][i][3] = x.w;
      vsc[half][i] = vs[(uint32_t)(row * (D / 32) + grp)];
    }
  };

  f32x4 oacc[NQ][MB];
  float m_run[NQ], l_run[NQ];
  bool first = true;
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    m_run[q] = -INFINITY;
    l_run[q] = 0.0f;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) oacc[q][mb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
  // Rows of V in LDS, 16-byte chunks swizzled for 16 neighbouring lanes that write one chunk (u) of every group of four rows (d = 64:
  // eight), and for 32 lanes of the transposing read that take 32 bytes (two chunks) of each of eight rows.  Pairs of chunks go by the row, the
  // place in a pair by the group; 16 rows on it is the same.  52 -> 49 us on 64 rows x 40 x 64 over 32 824 tokens.  Not free of conflicts:
  // 64 cycles of them a wavefront's tile at d = 64, 128 at d = 128, 39 % of the LDS cycles, as many as one of the two sides takes without any.
  auto swz = [](int row, int ch) __attribute__((always_inline)) {
    return ch ^ (CH == 16 ? (row & 7) << 1 : (row >> 1 & 3) << 1) ^ (ch >> 2 & 1);
  };
  u32x4* vt = stage[wave];
  auto own_lds = []() __attribute__((always_inline)) {    // this wavefront's own rows: LDS keeps its order, and the compiler its own
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  };

  auto tile = [&](auto ext_c, const Tile& cur, const Tile& then) __attribute__((always_inline)) {
    constexpr bool EXT = decltype(ext_c)::value;
    auto stage_v = [&](int half) __attribute__((always_inline)) {
      own_lds();
#pragma unroll
      for (int i = 0; i < VI; ++i) {
        const int item = 64 * i + lane, row = item / (D / 32), grp = item % (D / 32);
        u32x4 y[4];
        if constexpr (!EXT) {
#pragma unroll
          for (int u = 0; u < 4; ++u) y[u] = decode(vw[half][i][u], scale_of(vsc[half][i])).x;
        } else {
          const int tok = cur.tok + min(32 * half + row, cur.cnt - 1);
          const uint16_t* p = a.Vx + (int64_t)h * a.v_stride_head + (int64_t)tok * a.v_stride_tok + 32 * grp;
#pragma unroll
          for (int u = 0; u < 4; ++u) y[u] = *reinterpret_cast<const u32x4*>(p + 8 * u);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) vt[row * CH + swz(row, 4 * grp + u)] = y[u];
      }
      own_lds();
      if constexpr (!EXT) load_v(then, half);
    };
    f32x4 sacc[NQ][4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      Frag kf[KS];
      if constexpr (!EXT) {
#pragma unroll
        for (int u = 0; u < KS; ++u) kf[u] = decode(kw[s][u], scale_of(ksc[s]));
      } else {
        const int row = cur.tok + min(16 * s + col, cur.cnt - 1);
        const uint16_t* p = a.Kx + (int64_t)h * a.k_stride_head + (int64_t)row * a.k_stride_tok + (D / 4) * kg;
#pragma unroll
        for (int u = 0; u < KS; ++u) kf[u].x = *reinterpret_cast<const u32x4*>(p + 8 * u);
      }
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        sacc[q][s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < KS; ++u) sacc[q][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u].v, qf[q][u].v, sacc[q][s], 0, 0, 0);
      }
    }
    if constexpr (!EXT) load_k(then);
    stage_v(0);
    if (cur.cnt < 64) {       // (the tile's last token stands in for those behind it)
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * s + 4 * kg + i >= cur.cnt) sacc[q][s][i] = -INFINITY;
    }
    // P against the reference as it stands; where that is too low (or not set yet: the wavefront's first tile) it moves up to the maxima and P
    // is made again, before it has gone into any sum.
    float p[NQ][16];
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int i = 0; i < 16; ++i) p[q][i] = __builtin_amdgcn_exp2f(fmaf(sacc[q][i >> 2][i & 3], a.c, -m_run[q]));
    };
    bf16x8 pf[NQ][2], rest[2];
    f32x4 sum[NQ];
    auto sums = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
#pragma unroll
        for (int i = 0; i < 16; ++i) pf[q][i >> 3][i & 7] = (__bf16)p[q][i];
        sum[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int half = 0; half < 2; ++half) sum[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[q][half], sum[q], 0, 0, 0);
      }
    };
    bool move = first;
    if (!first) {
      weights();
      sums();
      bool past = false;
#pragma unroll
      for (int q = 0; q < NQ; ++q) past = past || sum[q][0] > kMostSum;
      move = __ballot(past) != 0ull;
    }
    if (move) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        float top = sacc[q][0][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, sacc[q][i >> 2][i & 3]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32)) * a.c;
        const float m_new = first ? top : fmaxf(m_run[q], top);
        const float alpha = first ? 0.0f : __builtin_amdgcn_exp2f(m_run[q] - m_new);
        m_run[q] = m_new;
        l_run[q] *= alpha;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 4; ++i) oacc[q][mb][i] *= alpha;
      }
      weights();
      sums();
      first = false;
    }
    if constexpr (TWO) {      // what P's rounding left off (only now: before the reference has moved P may be infinite)
#pragma unroll
      for (int i = 0; i < 16; ++i) rest[i >> 3][i & 7] = (__bf16)(p[0][i] - (float)pf[0][i >> 3][i & 7]);
#pragma unroll
      for (int half = 0; half < 2; ++half) sum[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, rest[half], sum[0], 0, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) l_run[q] += sum[q][0];
    auto product = [&](int half) __attribute__((always_inline)) {
      const uint16_t* v16 = reinterpret_cast<const uint16_t*>(vt);
      bf16x8 vf[MB];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        const int vrow = 4 * kg + (col >> 2), vcol = 16 * mb + 4 * (col & 3);
        const int off = (vrow * CH + swz(vrow, vcol >> 3)) * 8 + (vcol & 7);      // (16 rows on the swizzle is the same)
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(bf16x4, v16 + off));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(bf16x4, v16 + off + 16 * CH * 8));
        vf[mb] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int q = 0; q < NQ; ++q) oacc[q][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[mb], pf[q][half], oacc[q][mb], 0, 0, 0);
      }
      if constexpr (TWO) {      // (each sum's two products one behind the other: 48.1 us instead of 46.9)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) oacc[0][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[mb], rest[half], oacc[0][mb], 0, 0, 0);
      }
    };
    product(0);
    stage_v(1);
    product(1);
  };
  begin();
  Tile cur = next(false);
  if (cur.cnt > 0) {
    load_k(cur);
    load_v(cur, 0);
    load_v(cur, 1);
  }
  while (cur.cnt > 0) {
    const Tile then = next(false);
    // behind the last tile it is requested once more: loads that depend on a branch would make the waits of every tile wait for all of them
    tile(std::false_type{}, cur, then.cnt > 0 ? then : cur);
    cur = then;
  }
  if (a.extra > 0) {
    begin();
    for (Tile t = next(true); t.cnt > 0; t = next(true)) tile(std::true_type{}, t, t);
  }

  // The states of the SL wavefronts that have the same rows become one.
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    if (kg == 0) ml[wave][16 * q + col] = make_float2(m_run[q], l_run[q]);
  }
  __syncthreads();
  f32x4* buf = reinterpret_cast<f32x4*>(&stage[0][0]);        // MB tiles of four wavefronts, 64 lanes each: the whole stage
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    float M = -INFINITY, L = 0.0f;
#pragma unroll
    for (int w = 0; w < SL; ++w) M = fmaxf(M, ml[RG * w + rg][16 * q + col].x);
#pragma unroll
    for (int w = 0; w < SL; ++w) {
      const float2 x = ml[RG * w + rg][16 * q + col];
      L += x.x == -INFINITY ? 0.0f : x.y * __builtin_amdgcn_exp2f(x.x - M);
    }
    const float f = m_run[q] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[q] - M);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      f32x4 o = oacc[q][mb];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= f;
      buf[(mb * kWaves + wave) * 64 + lane] = o;
    }
    __syncthreads();
    const int row = 16 * (NQ * rg + q) + col;
#pragma unroll
    for (int k = 0; k < MB / SL; ++k) {
      const int mb = k * SL + slot;
      f32x4 o = buf[(mb * kWaves + rg) * 64 + lane];
#pragma unroll
      for (int w = 1; w < SL; ++w) {
        const f32x4 x = buf[(mb * kWaves + RG * w + rg) * 64 + lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += x[i];
      }
      if (a.parts == 1) {
        if (row < rows) {
          const float inv = L > 0.0f || L != L ? 1.0f / L : 0.0f;        // no token at all: zeros
          bf16x4 y;
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = (__bf16)(o[i] * inv);
          *reinterpret_cast<bf16x4*>(a.O + (int64_t)h * a.o_stride_head + (int64_t)(row0 + row) * a.o_stride_tok + 16 * mb + 4 * kg) = y;
        }
      } else {
        *reinterpret_cast<f32x4*>(a.state_o + (((int64_t)blockIdx.x * 16 * NQ * RG + row) * D + 16 * mb + 4 * kg)) = o;
      }
    }
    if (a.parts > 1 && slot == 0 && kg == 0) a.state_ml[(int64_t)blockIdx.x * 16 * NQ * RG + row] = make_float2(M, L);
    __syncthreads();
  }
}

// Joins the parts of a row: a workgroup each, its wavefronts taking every fourth part, lane p holding part p's weight (12 rows of 42 parts: 4 us, two
// loads one after the other and a launch; a wavefront a row, one part after the other: 13).
template <int D>
__global__ __launch_bounds__(64 * kWaves) void lf_kvq_join_kernel(KvqAttnArgs a, int rows_max, int tile_rows) {
  constexpr int W = D / 64;       // channels of a lane
  __shared__ float sums[kWaves][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blk = blockIdx.x / rows_max, i = blockIdx.x % rows_max;
  const int h = blk / a.n_q, r = blk % a.n_q;
  int row0 = 0, rows = a.q_len;
  if (a.idx) {
    const int j = r % a.nb;
    row0 = r / a.nb * a.n + 64 * j;
    rows = min(64, a.n - 64 * j);
  }
  if (i >= rows) return;
  const int64_t first = (int64_t)blk * a.parts * tile_rows + i;      // row of part 0; the others tile_rows apart
  float2 x = make_float2(-INFINITY, 0.0f);
  if (lane < a.parts) x = a.state_ml[first + (int64_t)lane * tile_rows];
  // a wavefront's parts are requested before the weights are known
  constexpr int N = LF_KVQ_MAX_PARTS / kWaves;
  float v[N][W], o[W];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int p = wave + kWaves * k;
#pragma unroll
    for (int e = 0; e < W; ++e) v[k][e] = p < a.parts ? a.state_o[(first + (int64_t)p * tile_rows) * D + W * lane + e] : 0.0f;
  }
  float M = x.x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
  const float wgt = x.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x.x - M);
#pragma unroll
  for (int e = 0; e < W; ++e) o[e] = 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float w = __shfl(wgt, wave + kWaves * k);       // 0 behind the last part
#pragma unroll
    for (int e = 0; e < W; ++e) o[e] = fmaf(w, v[k][e], o[e]);
  }
#pragma unroll
  for (int e = 0; e < W; ++e) sums[wave][W * lane + e] = o[e];
  __syncthreads();
  if (wave != 0) return;
  float L = wgt == 0.0f ? 0.0f : wgt * x.y;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) L += __shfl_xor(L, off);
  const float inv = L > 0.0f || L != L ? 1.0f / L : 0.0f;
  uint16_t* to = a.O + (int64_t)h * a.o_stride_head + (int64_t)(row0 + i) * a.o_stride_tok + W * lane;
#pragma unroll
  for (int e = 0; e < W; ++e) {
    float v = sums[0][W * lane + e];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += sums[w][W * lane + e];
    reinterpret_cast<__bf16*>(to)[e] = (__bf16)(v * inv);
  }
}

template <int D, bool LISTS>
void (*attn_kernel(int tiles))(KvqAttnArgs) {
  return tiles == 1 ? lf_kvq_attn_kernel<D, 1, 1, LISTS> : tiles == 2 ? lf_kvq_attn_kernel<D, 2, 1, LISTS> : lf_kvq_attn_kernel<D, 2, 2, LISTS>;
}

}  // namespace

int lf_launch_kvq_attn(const lf_kvq_call* c, void* stream) {
  const lf_kvq_parts p = lf_kvq_layout(c->cs);
  KvqAttnArgs a = {};
  a.Q = (const uint16_t*)c->Q;
  a.Kx = (const uint16_t*)c->K;
  a.Vx = (const uint16_t*)c->V;
  a.O = (uint16_t*)c->O;
  a.kc = c->cache + p.codes[0];
  a.vc = c->cache + p.codes[1];
  a.ks = c->cache + p.scales[0];
  a.vs = c->cache + p.scales[1];
  a.idx = c->indices;
  a.q_stride_tok = c->q_stride_tok; a.q_stride_head = c->q_stride_head;
  a.k_stride_tok = c->k_stride_tok; a.k_stride_head = c->k_stride_head;
  a.v_stride_tok = c->v_stride_tok; a.v_stride_head = c->v_stride_head;
  a.o_stride_tok = c->o_stride_tok; a.o_stride_head = c->o_stride_head;
  a.capacity = c->cs.capacity;
  a.cached = c->cached;
  a.extra = c->extra;
  a.n = c->n; a.nb = c->nb; a.n_q = c->n_q; a.n_k = c->n_k;
  a.nb_cached = c->indices ? c->cached / c->n * c->nb : 0;
  a.list_len = c->list_len;
  a.q_len = c->q_len;
  a.parts = c->parts;
  a.c = c->scale * 1.44269504088896340736f;
  const int tiles = lf_kvq_tiles(c->rows);
  const int64_t blocks = (int64_t)c->H * c->n_q;
  a.state_o = (float*)c->workspace;
  a.state_ml = (float2*)((float*)c->workspace + blocks * c->parts * 16 * tiles * c->d);
  hipStream_t st = (hipStream_t)stream;
  auto kernel = c->d == 128 ? (c->indices ? attn_kernel<128, true>(tiles) : attn_kernel<128, false>(tiles))
                            : (c->indices ? attn_kernel<64, true>(tiles) : attn_kernel<64, false>(tiles));
  hipError_t rc = lf_launch(kernel, dim3((unsigned)(blocks * c->parts)), dim3(64 * kWaves), 0, st, a);
  if (rc != hipSuccess) return LF_ERR_HIP;
  if (c->parts == 1) return LF_OK;
  const dim3 grid((unsigned)(blocks * c->rows));
  rc = c->d == 128 ? lf_launch(lf_kvq_join_kernel<128>, grid, dim3(64 * kWaves), 0, st, a, c->rows, 16 * tiles)
                   : lf_launch(lf_kvq_join_kernel<64>, grid, dim3(64 * kWaves), 0, st, a, c->rows, 16 * tiles);
  return rc == hipSuccess ? LF_OK : LF_ERR_HIP;
}
