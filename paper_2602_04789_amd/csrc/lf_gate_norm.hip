// Between two blocks: the block's output, normalised or not, gated onto the residual stream, and the norm of the stream with scale and shift.
//
//   p = B  or  B rb post_weight, rb = 1 / sqrt(mean(B^2) + eps);      Xout = X + rs gate p
//   n = (Xout - mean) r,  r = 1 / sqrt(var + eps)   (or without the mean);      Y = n f + shift,  f = weight (1 + scale)
//   backward, with u = dY f:  D = dXout + r (u - mean(u) - n mean(u n)),  dX = D,
//     e = rs gate D [post_weight],  dB = e  or  rb (e - bn mean(e bn)) with bn = B rb,
//     and sums over the rows of a group:  S = sum dY n,  Z = sum dY,  T = rs sum bn D,  from which the gradients of the tables follow
//     (dscale = weight S, dshift = Z, dgate = post_weight T, dweight = sum over groups of (1 + scale) S, dpost_weight = of gate T).
//
// HBM-bound: 8 bytes a value forward (bfloat16 stream), 12 backward.  A workgroup takes one row at a time and holds it in registers from the first
// sum to the stores, 8 channels of a thread side by side, so that every value is read once; the tables of the group stay in registers (forward)
// from row to row, and the next row is requested before the present one is summed.  Sums over a row go across the lanes of a wavefront and,
// where a row takes several, through LDS.  Sums over rows stay in registers over a slot (rows of one group); each slot leaves its sums, and a second
// launch adds the slots of a group in their order.  float32 throughout.
// Xout goes past the caches: it is wanted again behind the next block, and Y at once (32 760 rows of 1536, forward: 80 us, so 69; with a product of Y behind it 204 and
// 202; Y past the caches too 63, with the product 213).
//
// 32 760 rows of 5120: forward 247 us (1.34 GB, 5.4 TB/s), backward 434 and 12 for the sums (2.01 GB, 4.6 TB/s).  4680 rows of 1536: forward 12.6 us (57 MB).
// 4680 rows of 8192: forward 56 us, float32 stream 195 (96 registers spill; 94 at 4.9 TB/s).  One row: 2.7 us, the latency of its loads and sums.  1333 rows of 320, float32 stream, both ways: 4.6 + 7.0 + 4.2 + 2.9 us, four launches of little work.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "lf_blocks.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct NormArgs {
  const void *X, *B;
  const float *gate, *post, *weight, *scale, *shift;
  const int32_t* starts;
  void *Xout, *Y;
  const void *dY, *dXout;
  void *dX, *dB;
  float* part;
  int64_t x_stride, xo_stride, b_stride, y_stride, gate_stride, scale_stride, shift_stride;
  int L, C, groups, group_len, rows, per_group, layer;
  float eps, rs;
};

// The sum over a wavefront, in all of its lanes: rows of 16 lanes by rotation, then neighbouring rows and halves by exchange.
template <int CTRL> __device__ __forceinline__ float turned(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float row_sum16(float v) {
  v += turned<0x128>(v);      // row_ror:8, 4, 2, 1
  v += turned<0x124>(v);
  v += turned<0x122>(v);
  v += turned<0x121>(v);
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  v = row_sum16(v);
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

constexpr int kMaxWaves = 16;
// Sums over the workgroup.  `turn` counts the calls: they use two places in turn, so that one barrier a sum is enough.
struct RowSum {
  float (*place)[2][kMaxWaves];
  int waves, wave, turn;
  template <int N> __device__ __forceinline__ void operator()(float (&v)[N]) {
    static_assert(N <= 2, "two sums at a time");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if (waves == 1) return;
    float (*p)[kMaxWaves] = place[turn & 1];
    ++turn;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) p[i][wave] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {         // a lane of 16 for each wavefront
      const int w = threadIdx.x & 15;
      v[i] = row_sum16(w < waves ? p[i][w] : 0.0f);
    }
  }
};

// 8 values of the stream (bfloat16 or float32) and of a table.
template <bool F32> struct Raw { uint4 u; };
template <> struct Raw<true> { f32x4 a, b; };

template <bool F32> __device__ __forceinline__ Raw<F32> load_raw(const void* base, int64_t at) {
  Raw<F32> r;
  if constexpr (F32) {
    const f32x4* p = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(base) + at);
    r.a = p[0];
    r.b = p[1];
  } else {
    r.u = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(base) + at);
  }
  return r;
}
template <bool F32> __device__ __forceinline__ void unpack(const Raw<F32>& r, float (&x)[8]) {
  if constexpr (F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = r.a[e];
      x[4 + e] = r.b[e];
    }
  } else {
    const uint32_t w[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}
template <bool F32> __device__ __forceinline__ Raw<F32> pack(const float (&x)[8]) {
  Raw<F32> r;
  if constexpr (F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r.a[e] = x[e];
      r.b[e] = x[4 + e];
    }
  } else {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (__bf16)x[e];
    r.u = __builtin_bit_cast(uint4, o);
  }
  return r;
}
template <bool F32, bool PAST = false> __device__ __forceinline__ void store_raw(void* base, int64_t at, const Raw<F32>& r) {      // PAST: the caches
  if constexpr (F32) {
    f32x4* p = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(base) + at);
    if constexpr (PAST) {
      __builtin_nontemporal_store(r.a, p);
      __builtin_nontemporal_store(r.b, p + 1);
    } else {
      p[0] = r.a;
      p[1] = r.b;
    }
  } else {
    f32x4* p = reinterpret_cast<f32x4*>(reinterpret_cast<uint16_t*>(base) + at);
    if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(f32x4, r.u), p);
    else *p = __builtin_bit_cast(f32x4, r.u);
  }
}
__device__ __forceinline__ void load_table(const float* p, float (&t)[8]) {
  const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    t[e] = a[e];
    t[4 + e] = b[e];
  }
}
// weight (1 + scale) of a chunk
__device__ __forceinline__ void load_factor(const NormArgs& a, int g, int ch, float (&f)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = 1.0f;
  if (a.scale) {
    float t[8];
    load_table(a.scale + (int64_t)g * a.scale_stride + ch, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] += t[e];
  }
  if (a.weight) {
    float t[8];
    load_table(a.weight + ch, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= t[e];
  }
}
// The first token of group g (of the end for g = groups), inside the tensor whatever `starts` holds.
__device__ __forceinline__ int group_start(const NormArgs& a, int g) {
  return min(max(a.starts[g], 0), a.L);
}

constexpr int most_threads(int nc) { return nc == 2 ? 1024 : 256; }

template <int NC, bool F32, int AHEAD>
__global__ __launch_bounds__(most_threads(NC)) void lf_gate_norm_kernel(NormArgs a) {
  __shared__ float place[2][2][kMaxWaves];
  RowSum row_sum = {place, (int)blockDim.x >> 6, (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), 0};
  const int r0 = blockIdx.x * a.rows;
  int end = min(a.L, r0 + a.rows), r = r0, g = 0, g_end = 0;
  if (a.group_len > 0) {
    g = r / a.group_len;
    g_end = (int)min((int64_t)a.L, ((int64_t)g + 1) * a.group_len);
  } else {
    r = max(r, group_start(a, 0));
    end = min(end, group_start(a, a.groups));
    int lo = 0, hi = a.groups;             // the last group that begins at r or before it
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (group_start(a, mid) <= r) lo = mid; else hi = mid;
    }
    g = lo;
    g_end = group_start(a, g + 1);
  }
  if (r >= end) return;
  int ch[NC];
  bool in[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = 8 * (int)(threadIdx.x + i * blockDim.x);
    in[i] = c < a.C;
    ch[i] = in[i] ? c : 0;
  }
  const bool has_b = a.B != nullptr, post = a.post != nullptr;
  Raw<F32> xn[AHEAD][NC];           // rows r, r + 1, ..
  Raw<false> bn[AHEAD][NC];
  auto request = [&](int row, int to) __attribute__((always_inline)) {
    row = min(row, end - 1);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      xn[to][i] = load_raw<F32>(a.X, (int64_t)row * a.x_stride + ch[i]);
      if (has_b) bn[to][i] = load_raw<false>(a.B, (int64_t)row * a.b_stride + ch[i]);
    }
  };
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) request(r + k, k);
  float f[NC][8], sh[NC][8], ga[NC][8];
  int have = -1;
  const float count = (float)a.C;
  for (; r < end; ++r) {
    while (r >= g_end && g + 1 < a.groups) {
      ++g;
      g_end = a.group_len > 0 ? (int)min((int64_t)a.L, ((int64_t)g + 1) * a.group_len) : group_start(a, g + 1);
    }
    float x[NC][8], b[NC][8];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      unpack<F32>(xn[0][i], x[i]);
      if (has_b) unpack<false>(bn[0][i], b[i]);
#pragma unroll
      for (int k = 1; k < AHEAD; ++k) {
        xn[k - 1][i] = xn[k][i];
        if (has_b) bn[k - 1][i] = bn[k][i];
      }
    }
    if (g != have) {
      have = g;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        load_factor(a, g, ch[i], f[i]);
        if (a.shift) load_table(a.shift + (int64_t)g * a.shift_stride + ch[i], sh[i]);
        if (a.gate) load_table(a.gate + (int64_t)g * a.gate_stride + ch[i], ga[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ga[i][e] = a.gate ? ga[i][e] * a.rs : a.rs;
          if (!a.shift) sh[i][e] = 0.0f;
        }
      }
    }
    if (r + AHEAD < end) request(r + AHEAD, AHEAD - 1);
    if (has_b) {
      if (post) {
        float ss[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          float s = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fmaf(b[i][e], b[i][e], s);
          ss[0] += in[i] ? s : 0.0f;
        }
        row_sum(ss);
        const float rb = 1.0f / sqrtf(ss[0] / count + a.eps);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          float w[8];
          load_table(a.post + ch[i], w);
#pragma unroll
          for (int e = 0; e < 8; ++e) b[i][e] *= rb * w[e];
        }
      }
#pragma unroll
      for (int i = 0; i < NC; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = fmaf(ga[i][e], b[i][e], x[i][e]);
        const Raw<F32> o = pack<F32>(x[i]);
        if (in[i]) store_raw<F32, true>(a.Xout, (int64_t)r * a.xo_stride + ch[i], o);
        unpack<F32>(o, x[i]);
      }
    }
    float mean = 0.0f;
    if (a.layer) {
      float s[1] = {0.0f};
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        float t = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) t += x[i][e];
        s[0] += in[i] ? t : 0.0f;
      }
      row_sum(s);
      mean = s[0] / count;
    }
    float ss[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[i][e] -= mean;
        s = fmaf(x[i][e], x[i][e], s);
      }
      ss[0] += in[i] ? s : 0.0f;
    }
    row_sum(ss);
    const float inv = 1.0f / sqrtf(ss[0] / count + a.eps);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = fmaf(x[i][e] * inv, f[i][e], sh[i][e]);
      if (in[i]) store_raw<false>(a.Y, (int64_t)r * a.y_stride + ch[i], pack<false>(x[i]));
    }
  }
}

// The group and the rows of a slot of the backward kernel.
struct Slot {
  int g, r0, r1;
};
__device__ __forceinline__ int64_t slot_of(const NormArgs& a, int g) {     // the first slot of group g: `starts` of any values gives any order
  return (int64_t)group_start(a, g) / a.rows + g;
}
__device__ __forceinline__ Slot find_slot(const NormArgs& a, int64_t s) {
  Slot t;
  if (a.group_len > 0) {
    t.g = (int)(s / a.per_group);
    const int64_t first = (int64_t)t.g * a.group_len, r0 = first + (s % a.per_group) * a.rows;
    t.r0 = (int)min(r0, (int64_t)a.L);
    t.r1 = (int)min(min(r0 + a.rows, first + a.group_len), (int64_t)a.L);
    return t;
  }
  int lo = 0, hi = a.groups;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (slot_of(a, mid) <= s) lo = mid; else hi = mid;
  }
  t.g = lo;
  const int64_t i = s - slot_of(a, lo), r0 = (int64_t)group_start(a, lo) + i * a.rows;
  const int last = group_start(a, lo + 1);
  t.r0 = i < 0 ? last : (int)min(r0, (int64_t)last);
  t.r1 = (int)min((int64_t)t.r0 + a.rows, (int64_t)last);
  return t;
}

// How a workgroup of the backward kernel takes the rows of its slot.
//   kRow      one at a time, the next two on their way
//   kWaves    one for each of its four wavefronts (narrow rows: no barrier, and the four leave one set of sums)
//   kWide     one at a time, for rows of more than 6 144 channels: values stay packed and are unpacked where they are used, tables are read from
//             memory, and nothing is on its way.  All the same 128 registers, as 1 024 threads have, are too few: 86 to 172 spill, and scratch bounds
//             it (4680 rows of 8192 399 us, with post_weight 688, 94 at 4.9 TB/s; of 16 384 589 and 1090, 188)
enum NormForm { kRow, kWaves, kWide };

template <int NC, bool F32, int FORM, bool POST>
__global__ __launch_bounds__(FORM == kWide ? 1024 : 256) void lf_gate_norm_bwd_kernel(NormArgs a) {
  constexpr int AHEAD = FORM == kWide ? 1 : 2;
  constexpr bool KEPT = FORM != kWide;
  __shared__ float place[2][2][kMaxWaves];
  const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowSum row_sum = {place, FORM == kWaves ? 1 : (int)blockDim.x >> 6, wave, 0};
  const Slot slot = find_slot(a, blockIdx.x);
  if (slot.r0 >= slot.r1) return;
  const int step = FORM == kWaves ? 4 : 1, begin = slot.r0 + (FORM == kWaves ? wave : 0);
  const int tid = FORM == kWaves ? threadIdx.x & 63 : threadIdx.x, across = FORM == kWaves ? 64 : blockDim.x;
  int ch[NC];
  bool in[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = 8 * (tid + i * across);
    in[i] = c < a.C;
    ch[i] = in[i] ? c : 0;
  }
  const bool has_b = a.B != nullptr;
  const float count = (float)a.C;
  // What a thread without channels in a chunk holds is zeros: its dY, D and B add nothing.
  Raw<F32> xn[AHEAD][NC] = {}, on[AHEAD][NC] = {};
  Raw<false> bn[AHEAD][NC] = {}, yn[AHEAD][NC] = {};
  auto request = [&](int row, int to) __attribute__((always_inline)) {
    row = min(row, slot.r1 - 1);
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (in[i]) {
        xn[to][i] = load_raw<F32>(a.Xout, (int64_t)row * a.xo_stride + ch[i]);
        if (a.dXout) on[to][i] = load_raw<F32>(a.dXout, (int64_t)row * a.xo_stride + ch[i]);
        if (a.dY) yn[to][i] = load_raw<false>(a.dY, (int64_t)row * a.y_stride + ch[i]);
        if (has_b) bn[to][i] = load_raw<false>(a.B, (int64_t)row * a.b_stride + ch[i]);
      }
  };
  if constexpr (FORM != kWide) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) request(begin + k * step, k);
  }
  float S[NC][8], Z[NC][8], T[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) S[i][e] = Z[i][e] = T[i][e] = 0.0f;
  // the group's factors: of Y, and of B
  auto factors_y = [&](int i, float (&f)[8]) __attribute__((always_inline)) { load_factor(a, slot.g, ch[i], f); };
  auto factors_b = [&](int i, float (&ga)[8]) __attribute__((always_inline)) {
    if (a.gate) load_table(a.gate + (int64_t)slot.g * a.gate_stride + ch[i], ga);
    float w[8];
    if constexpr (POST) load_table(a.post + ch[i], w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      ga[e] = a.gate ? ga[e] * a.rs : a.rs;
      if constexpr (POST) ga[e] *= w[e];
    }
  };
  constexpr int KN = KEPT ? NC : 1;         // what is kept over the slot, or over a row: chunks
  float f[KN][8], ga[KN][8];
  if constexpr (KEPT) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      factors_y(i, f[i]);
      factors_b(i, ga[i]);
    }
  }
  for (int r = begin; r < slot.r1; r += step) {
    Raw<F32> xr[NC], orw[NC];
    Raw<false> br[NC], yr[NC];
    if constexpr (FORM == kWide) request(r, 0);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      xr[i] = xn[0][i];
      orw[i] = on[0][i];
      br[i] = bn[0][i];
      yr[i] = yn[0][i];
#pragma unroll
      for (int k = 1; k < AHEAD; ++k) {
        xn[k - 1][i] = xn[k][i];
        on[k - 1][i] = on[k][i];
        bn[k - 1][i] = bn[k][i];
        yn[k - 1][i] = yn[k][i];
      }
    }
    float n[KN][8], u[KN][8];
    // the row's mean, and the squares of B
    float first[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      float (&m)[8] = n[KEPT ? i : 0];
      unpack<F32>(xr[i], m);
#pragma unroll
      for (int e = 0; e < 8; ++e) first[0] += m[e];
      if constexpr (POST) {
        float b[8];
        unpack<false>(br[i], b);
#pragma unroll
        for (int e = 0; e < 8; ++e) first[1] = fmaf(b[e], b[e], first[1]);
      }
    }
    if constexpr (FORM != kWide) {
      if (r + AHEAD * step < slot.r1) request(r + AHEAD * step, AHEAD - 1);
    }
    if (a.layer || POST) row_sum(first);
    const float mean = a.layer ? first[0] / count : 0.0f;
    const float rb = POST ? 1.0f / sqrtf(first[1] / count + a.eps) : 1.0f;
    float ss[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      float (&m)[8] = n[KEPT ? i : 0];
      if constexpr (!KEPT) unpack<F32>(xr[i], m);
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[e] -= mean;
        s = fmaf(m[e], m[e], s);
      }
      ss[0] += in[i] ? s : 0.0f;
    }
    row_sum(ss);
    const float inv = 1.0f / sqrtf(ss[0] / count + a.eps);
    // n and dY f of a chunk
    auto values = [&](int i, bool first_time) __attribute__((always_inline)) {
      float (&m)[8] = n[KEPT ? i : 0];
      float (&w)[8] = u[KEPT ? i : 0];
      if constexpr (!KEPT) {
        unpack<F32>(xr[i], m);
        factors_y(i, f[0]);
      } else if (!first_time) {
        return;
      }
      float dy[8];
      unpack<false>(yr[i], dy);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[e] = KEPT ? m[e] * inv : (m[e] - mean) * inv;
        w[e] = dy[e] * f[KEPT ? i : 0][e];
        if (first_time) {
          S[i][e] = fmaf(dy[e], m[e], S[i][e]);
          Z[i][e] += dy[e];
        }
      }
    };
    float means[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      values(i, true);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        means[0] += u[KEPT ? i : 0][e];
        means[1] = fmaf(u[KEPT ? i : 0][e], n[KEPT ? i : 0][e], means[1]);
      }
    }
    row_sum(means);
    const float mu = a.layer ? means[0] / count : 0.0f, mun = means[1] / count;
    float eb[1] = {0.0f};
    float E[NC][8];              // what goes on to B
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      values(i, false);
      float D[8], b[8];
      unpack<F32>(orw[i], D);
      unpack<false>(br[i], b);
      if constexpr (!KEPT) {
        if (has_b) factors_b(i, ga[0]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) D[e] = fmaf(inv, fmaf(-n[KEPT ? i : 0][e], mun, u[KEPT ? i : 0][e] - mu), D[e]);
      if (in[i]) store_raw<F32>(a.dX, (int64_t)r * a.xo_stride + ch[i], pack<F32>(D));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (POST) b[e] *= rb;
        T[i][e] = fmaf(b[e], D[e], T[i][e]);
        E[i][e] = D[e] * ga[KEPT ? i : 0][e];
        if constexpr (POST) eb[0] = fmaf(E[i][e], b[e], eb[0]);      // (zero without channels: b is)
      }
    }
    if (has_b) {
      if constexpr (POST) {
        row_sum(eb);
        const float m = eb[0] / count;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          float b[8];
          unpack<false>(br[i], b);
#pragma unroll
          for (int e = 0; e < 8; ++e) E[i][e] = rb * fmaf(-b[e] * rb, m, E[i][e]);
        }
      }
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (in[i]) store_raw<false>(a.dB, (int64_t)r * a.b_stride + ch[i], pack<false>(E[i]));
    }
  }
  if (!a.part) return;
  float* p = a.part + (int64_t)blockIdx.x * 3 * a.C;
  if constexpr (FORM == kWaves) {       // the four wavefronts' sums become one, in their order
    __shared__ float both[3][NC * 8][64];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if (wave > 0) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) both[wave - 1][8 * i + e][tid] = k == 0 ? S[i][e] : k == 1 ? Z[i][e] : T[i][e];
      }
      __syncthreads();
      if (wave == 0) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float& v = k == 0 ? S[i][e] : k == 1 ? Z[i][e] : T[i][e];
            v = v + both[0][8 * i + e][tid] + both[1][8 * i + e][tid] + both[2][8 * i + e][tid];
          }
      }
      __syncthreads();
    }
    if (wave > 0) return;
  }
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (in[i]) {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        f32x4 lo, hi;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[e] = k == 0 ? S[i][e] : k == 1 ? Z[i][e] : T[i][e];
          hi[e] = k == 0 ? S[i][4 + e] : k == 1 ? Z[i][4 + e] : T[i][4 + e];
        }
        f32x4* to = reinterpret_cast<f32x4*>(p + (int64_t)k * a.C + ch[i]);
        to[0] = lo;
        to[1] = hi;
      }
    }
}

struct SumArgs {
  NormArgs n;
  int groups;            // of the tables: those past n.groups have no tokens
  float *dgate, *dscale, *dshift;
  float* sums;           // [groups][2][C]: S and T, for the weights; or null
  float *dweight, *dpost;
};
// A group's slots: 16 channels of a workgroup, its rows of threads (16, or 64 for groups of many slots) taking a slot in turn, four of them at a time, and joined
// in their order.  dweight = sum over groups of (1 + scale) S, dpost_weight = of gate T: here where there is one group, else in a launch of their
// own (both ways, without it and with it: 4680 rows of 1536 in one group 43.5 and 45.3 us; a workgroup that goes through three groups 47.2 and 46.7, eight 53.2 and 44.7).
template <int kSumRows>
__global__ __launch_bounds__(16 * kSumRows) void lf_gate_norm_sum_kernel(SumArgs b) {
  const NormArgs& a = b.n;
  __shared__ float s[3][kSumRows][17];
  const int col = threadIdx.x & 15, c = blockIdx.x * 16 + col, row = threadIdx.x >> 4;
  for (int g = blockIdx.y; g < b.groups; g += gridDim.y) {
    int64_t first, many;
    if (a.group_len > 0) {
      const int64_t rows = min((int64_t)a.group_len, (int64_t)a.L - (int64_t)g * a.group_len);
      first = (int64_t)g * a.per_group;
      many = rows > 0 ? (rows + a.rows - 1) / a.rows : 0;
    } else {
      const int n = group_start(a, g + 1) - group_start(a, g);
      first = slot_of(a, g);
      many = n > 0 ? ((int64_t)n + a.rows - 1) / a.rows : 0;
    }
    float v[3] = {0.0f, 0.0f, 0.0f};
    if (c < a.C) {
      const float* p = a.part + first * 3 * a.C + c;
      for (int64_t i = row; i < many; i += 4 * kSumRows) {
        float y[4][3];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int k = 0; k < 3; ++k) y[u][k] = i + u * kSumRows < many ? p[((i + u * kSumRows) * 3 + k) * a.C] : 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int k = 0; k < 3; ++k) v[k] += y[u][k];
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k][row][col] = v[k];
    __syncthreads();
    if (row < 3) {              // a sum each: three rows of threads
      float t = 0.0f;
#pragma unroll
      for (int i = 0; i < kSumRows; ++i) t += s[row][i][col];
      const int64_t at = (int64_t)g * a.C + c;
      const bool has = g < a.groups, only = has && a.groups == 1;
      if (c < a.C) {
        if (row == 0) {
          if (b.dscale) b.dscale[at] = a.weight ? t * a.weight[c] : t;
          if (only && b.dweight) b.dweight[c] = a.scale ? (1.0f + a.scale[c]) * t : t;
          else if (b.sums && has) b.sums[2 * (int64_t)g * a.C + c] = t;
        } else if (row == 1) {
          if (b.dshift) b.dshift[at] = t;
        } else {
          t *= a.rs;
          if (b.dgate) b.dgate[at] = a.post ? t * a.post[c] : t;
          if (only && b.dpost) b.dpost[c] = a.gate ? a.gate[c] * t : t;
          else if (b.sums && has) b.sums[(2 * (int64_t)g + 1) * a.C + c] = t;
        }
      }
    }
  }
}
__global__ __launch_bounds__(256) void lf_gate_norm_weight_kernel(SumArgs b) {
  const NormArgs& a = b.n;
  __shared__ float s[2][16][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), lane = threadIdx.x >> 4;
  float v[2] = {0.0f, 0.0f};
  if (c < a.C) {
    for (int g = lane; g < a.groups; g += 16) {
      const float S = b.sums[2 * (int64_t)g * a.C + c], T = b.sums[(2 * (int64_t)g + 1) * a.C + c];
      v[0] = fmaf(a.scale ? 1.0f + a.scale[(int64_t)g * a.scale_stride + c] : 1.0f, S, v[0]);
      v[1] = fmaf(a.gate ? a.gate[(int64_t)g * a.gate_stride + c] : 1.0f, T, v[1]);
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) s[k][lane][threadIdx.x & 15] = v[k];
  __syncthreads();
  if (lane != 0 || c >= a.C) return;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += s[k][i][threadIdx.x & 15];
    v[k] = t;
  }
  if (b.dweight) b.dweight[c] = v[0];
  if (b.dpost) b.dpost[c] = v[1];
}

NormArgs args_of(const lf_norm_call* c) {
  const lf_norm_shape* s = c->s;
  NormArgs a = {};
  a.X = c->X; a.B = c->B;
  a.gate = c->gate; a.post = c->post_weight; a.weight = c->weight; a.scale = c->scale; a.shift = c->shift;
  a.starts = c->starts;
  a.Xout = c->Xout; a.Y = c->Y;
  a.dY = c->dY; a.dXout = c->dXout; a.dX = c->dX; a.dB = c->dB;
  a.x_stride = s->x_stride; a.xo_stride = s->xo_stride; a.b_stride = s->b_stride; a.y_stride = s->y_stride;
  a.gate_stride = s->gate_stride; a.scale_stride = s->scale_stride; a.shift_stride = s->shift_stride;
  a.L = s->tokens; a.C = s->channels; a.groups = s->groups; a.group_len = s->group_len;
  a.layer = s->kind == LF_NORM_LAYER;
  a.eps = s->eps; a.rs = s->residual_scale;
  return a;
}

}  // namespace

int lf_launch_gate_norm(const lf_norm_call* c, void* stream) {
  NormArgs a = args_of(c);
  lf_norm_lay l;
  a.rows = lf_norm_fwd_rows(c->s, &l);
  const bool f32 = c->s->stream_dtype == LF_F32;
  auto kernel = l.nc == 1 ? (f32 ? lf_gate_norm_kernel<1, true, 1> : lf_gate_norm_kernel<1, false, 1>)
              : l.nc == 2 ? (f32 ? lf_gate_norm_kernel<2, true, 1> : lf_gate_norm_kernel<2, false, 1>)
                          : (f32 ? lf_gate_norm_kernel<3, true, 2> : lf_gate_norm_kernel<3, false, 2>);
  const unsigned blocks = (unsigned)((a.L - 1) / a.rows + 1);
  return lf_launch(kernel, dim3(blocks), dim3(l.threads), 0, (hipStream_t)stream, a) == hipSuccess ? LF_OK : LF_ERR_HIP;
}

int lf_launch_gate_norm_bwd(const lf_norm_call* c, void* stream) {
  const lf_norm_slots n = lf_norm_bwd_slots(c->s);
  NormArgs a = args_of(c);
  a.rows = n.rows;
  a.per_group = n.per_group;
  const bool sums = c->dgate || c->dpost_weight || c->dweight || c->dscale || c->dshift;
  a.part = sums ? c->workspace : nullptr;
  const bool f32 = c->s->stream_dtype == LF_F32;
  auto pick = [&](auto post) {
    constexpr bool P = decltype(post)::value;
    if (n.waves)
      return n.lay.nc == 1 ? (f32 ? lf_gate_norm_bwd_kernel<1, true, kWaves, P> : lf_gate_norm_bwd_kernel<1, false, kWaves, P>)
           : n.lay.nc == 2 ? (f32 ? lf_gate_norm_bwd_kernel<2, true, kWaves, P> : lf_gate_norm_bwd_kernel<2, false, kWaves, P>)
                           : (f32 ? lf_gate_norm_bwd_kernel<3, true, kWaves, P> : lf_gate_norm_bwd_kernel<3, false, kWaves, P>);
    return n.lay.nc == 3 ? (f32 ? lf_gate_norm_bwd_kernel<3, true, kRow, P> : lf_gate_norm_bwd_kernel<3, false, kRow, P>)
                         : (f32 ? lf_gate_norm_bwd_kernel<2, true, kWide, P> : lf_gate_norm_bwd_kernel<2, false, kWide, P>);
  };
  auto kernel = c->post_weight ? pick(std::true_type{}) : pick(std::false_type{});
  hipStream_t st = (hipStream_t)stream;
  if (lf_launch(kernel, dim3((unsigned)n.slots), dim3(n.waves ? 256 : n.lay.threads), 0, st, a) != hipSuccess) return LF_ERR_HIP;
  if (!sums) return LF_OK;
  const bool weights = a.groups > 1 && (c->dweight || c->dpost_weight), many = n.slots > 64 * (int64_t)a.groups;
  const SumArgs b = {a, c->groups, c->dgate, c->dscale, c->dshift, weights ? c->workspace + n.slots * 3 * a.C : nullptr, c->dweight, c->dpost_weight};
  const unsigned across = (unsigned)(a.C + 15) / 16;
  const dim3 grid(across, (unsigned)(c->groups < 4096 ? c->groups : 4096));
  if ((many ? lf_launch(lf_gate_norm_sum_kernel<64>, grid, dim3(1024), 0, st, b) : lf_launch(lf_gate_norm_sum_kernel<16>, grid, dim3(256), 0, st, b)) != hipSuccess)
    return LF_ERR_HIP;
  if (!weights) return LF_OK;
  return lf_launch(lf_gate_norm_weight_kernel, dim3(across), dim3(256), 0, st, b) == hipSuccess ? LF_OK : LF_ERR_HIP;
}
