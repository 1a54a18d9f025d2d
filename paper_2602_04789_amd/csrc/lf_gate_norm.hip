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
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

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
__device__ __forceinline__ float wave_sum(float v) {
  v += turned<0x128>(v);      // row_ror:8, 4, 2, 1
  v += turned<0x124>(v);
  v += turned<0x122>(v);
  v += turned<0x121>(v);
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
    for (int i = 0; i < N; ++i) {
      float s = p[i][0];
      for (int w = 1; w < waves; ++w) s += p[i][w];
      v[i] = s;
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
template <bool F32> __device__ __forceinline__ void store_raw(void* base, int64_t at, const Raw<F32>& r) {
  if constexpr (F32) {
    f32x4* p = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(base) + at);
    p[0] = r.a;
    p[1] = r.b;
  } else {
    *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(base) + at) = r.u;
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

constexpr int most_threads(int nc) { return nc == 1 ? 640 : nc == 2 ? 1024 : 256; }

template <int NC, bool F32>
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
  Raw<F32> xn[NC];
  Raw<false> bn[NC];
  auto request = [&](int row) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      xn[i] = load_raw<F32>(a.X, (int64_t)row * a.x_stride + ch[i]);
      if (has_b) bn[i] = load_raw<false>(a.B, (int64_t)row * a.b_stride + ch[i]);
    }
  };
  request(r);
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
      unpack<F32>(xn[i], x[i]);
      if (has_b) unpack<false>(bn[i], b[i]);
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
    if (r + 1 < end) request(r + 1);
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
        if (in[i]) store_raw<F32>(a.Xout, (int64_t)r * a.xo_stride + ch[i], o);
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

template <int NC, bool F32>
__global__ __launch_bounds__(most_threads(NC)) void lf_gate_norm_bwd_kernel(NormArgs a) {
  __shared__ float place[2][2][kMaxWaves];
  RowSum row_sum = {place, (int)blockDim.x >> 6, (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), 0};
  const Slot slot = find_slot(a, blockIdx.x);
  if (slot.r0 >= slot.r1) return;
  int ch[NC];
  bool in[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = 8 * (int)(threadIdx.x + i * blockDim.x);
    in[i] = c < a.C;
    ch[i] = in[i] ? c : 0;
  }
  const bool has_b = a.B != nullptr, post = a.post != nullptr;
  const float count = (float)a.C;
  Raw<F32> xn[NC], on[NC];
  Raw<false> bn[NC], yn[NC];
  auto request = [&](int row) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      xn[i] = load_raw<F32>(a.Xout, (int64_t)row * a.xo_stride + ch[i]);
      if (a.dXout) on[i] = load_raw<F32>(a.dXout, (int64_t)row * a.xo_stride + ch[i]);
      if (a.dY) yn[i] = load_raw<false>(a.dY, (int64_t)row * a.y_stride + ch[i]);
      if (has_b) bn[i] = load_raw<false>(a.B, (int64_t)row * a.b_stride + ch[i]);
    }
  };
  request(slot.r0);
  float S[NC][8], Z[NC][8], T[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) S[i][e] = Z[i][e] = T[i][e] = 0.0f;
  for (int r = slot.r0; r < slot.r1; ++r) {
    float n[NC][8], dy[NC][8], D[NC][8], b[NC][8];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      unpack<F32>(xn[i], n[i]);
      if (a.dXout) unpack<F32>(on[i], D[i]);
      if (a.dY) unpack<false>(yn[i], dy[i]);
      if (has_b) unpack<false>(bn[i], b[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!a.dXout) D[i][e] = 0.0f;
        if (!a.dY) dy[i][e] = 0.0f;
        if (!in[i]) n[i][e] = dy[i][e] = D[i][e] = b[i][e] = 0.0f;
      }
    }
    if (r + 1 < slot.r1) request(r + 1);
    // the row's mean, and its squares (of B too)
    float first[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      float s = 0.0f, q = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s += n[i][e];
        if (post) q = fmaf(b[i][e], b[i][e], q);
      }
      first[0] += s;
      first[1] += q;
    }
    if (a.layer || post) row_sum(first);
    const float mean = a.layer ? first[0] / count : 0.0f;
    const float rb = post ? 1.0f / sqrtf(first[1] / count + a.eps) : 1.0f;
    float ss[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[i][e] -= mean;
        s = fmaf(n[i][e], n[i][e], s);
      }
      ss[0] += in[i] ? s : 0.0f;
    }
    row_sum(ss);
    const float inv = 1.0f / sqrtf(ss[0] / count + a.eps);
    float means[2] = {0.0f, 0.0f};
    float f[NC][8];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      load_factor(a, slot.g, ch[i], f[i]);
      float s = 0.0f, q = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[i][e] = in[i] ? n[i][e] * inv : 0.0f;
        S[i][e] = fmaf(dy[i][e], n[i][e], S[i][e]);
        Z[i][e] += dy[i][e];
        dy[i][e] *= f[i][e];
        s += dy[i][e];
        q = fmaf(dy[i][e], n[i][e], q);
      }
      means[0] += s;
      means[1] += q;
    }
    row_sum(means);
    const float mu = a.layer ? means[0] / count : 0.0f, mun = means[1] / count;
    float eb[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NC; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) D[i][e] = fmaf(inv, fmaf(-n[i][e], mun, dy[i][e] - mu), D[i][e]);
      if (in[i]) store_raw<F32>(a.dX, (int64_t)r * a.xo_stride + ch[i], pack<F32>(D[i]));
      if (has_b) {
        float ga[8], w[8];
        if (a.gate) load_table(a.gate + (int64_t)slot.g * a.gate_stride + ch[i], ga);
        if (post) load_table(a.post + ch[i], w);
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          D[i][e] *= a.rs;
          b[i][e] *= rb;
          T[i][e] = fmaf(b[i][e], D[i][e], T[i][e]);
          if (a.gate) D[i][e] *= ga[e];
          if (post) D[i][e] *= w[e];
          s = fmaf(D[i][e], b[i][e], s);
        }
        eb[0] += in[i] ? s : 0.0f;
      }
    }
    if (has_b) {
      if (post) row_sum(eb);
      const float m = post ? eb[0] / count : 0.0f;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) D[i][e] = rb * fmaf(-b[i][e], m, D[i][e]);
        if (in[i]) store_raw<false>(a.dB, (int64_t)r * a.b_stride + ch[i], pack<false>(D[i]));
      }
    }
  }
  if (!a.part) return;
  float* p = a.part + (int64_t)blockIdx.x * 3 * a.C;
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
  float *dgate, *dscale, *dshift;
  float* sums;           // [groups][2][C]: S and T, for the weights; or null
};
// A group's slots: 16 channels of a workgroup, its 16 rows of threads taking every 16th slot and joined in their order.
__global__ __launch_bounds__(256) void lf_gate_norm_sum_kernel(SumArgs b) {
  const NormArgs& a = b.n;
  __shared__ float s[3][16][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), lane = threadIdx.x >> 4;
  for (int g = blockIdx.y; g < a.groups; g += gridDim.y) {
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
      for (int64_t i = lane; i < many; i += 16) {
        const float* p = a.part + (first + i) * 3 * a.C + c;
#pragma unroll
        for (int k = 0; k < 3; ++k) v[k] += p[(int64_t)k * a.C];
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k][lane][threadIdx.x & 15] = v[k];
    __syncthreads();
    if (lane == 0 && c < a.C) {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) t += s[k][i][threadIdx.x & 15];
        v[k] = t;
      }
      const int64_t at = (int64_t)g * a.C + c;
      if (b.dscale) b.dscale[at] = a.weight ? v[0] * a.weight[c] : v[0];
      if (b.dshift) b.dshift[at] = v[1];
      if (b.dgate) b.dgate[at] = a.post ? v[2] * a.post[c] : v[2];
      if (b.sums) {
        b.sums[2 * (int64_t)g * a.C + c] = v[0];
        b.sums[(2 * (int64_t)g + 1) * a.C + c] = v[2];
      }
    }
  }
}
// dweight = sum over groups of (1 + scale) S, dpost_weight = of gate T.
__global__ __launch_bounds__(256) void lf_gate_norm_weight_kernel(SumArgs b, float* dweight, float* dpost) {
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
  if (dweight) dweight[c] = v[0];
  if (dpost) dpost[c] = v[1];
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
  auto kernel = l.nc == 1 ? (f32 ? lf_gate_norm_kernel<1, true> : lf_gate_norm_kernel<1, false>)
              : l.nc == 2 ? (f32 ? lf_gate_norm_kernel<2, true> : lf_gate_norm_kernel<2, false>)
                          : (f32 ? lf_gate_norm_kernel<3, true> : lf_gate_norm_kernel<3, false>);
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
  auto kernel = n.lay.nc == 1 ? (f32 ? lf_gate_norm_bwd_kernel<1, true> : lf_gate_norm_bwd_kernel<1, false>)
              : n.lay.nc == 2 ? (f32 ? lf_gate_norm_bwd_kernel<2, true> : lf_gate_norm_bwd_kernel<2, false>)
                              : (f32 ? lf_gate_norm_bwd_kernel<3, true> : lf_gate_norm_bwd_kernel<3, false>);
  hipStream_t st = (hipStream_t)stream;
  if (lf_launch(kernel, dim3((unsigned)n.slots), dim3(n.lay.threads), 0, st, a) != hipSuccess) return LF_ERR_HIP;
  if (!sums) return LF_OK;
  const bool weights = c->dweight || c->dpost_weight;
  SumArgs b = {a, c->dgate, c->dscale, c->dshift, weights ? c->workspace + n.slots * 3 * a.C : nullptr};
  const unsigned across = (unsigned)(a.C + 15) / 16;
  if (lf_launch(lf_gate_norm_sum_kernel, dim3(across, (unsigned)(a.groups < 8192 ? a.groups : 8192)), dim3(256), 0, st, b) != hipSuccess)
    return LF_ERR_HIP;
  if (!weights) return LF_OK;
  return lf_launch(lf_gate_norm_weight_kernel, dim3(across), dim3(256), 0, st, b, c->dweight, c->dpost_weight) == hipSuccess ? LF_OK : LF_ERR_HIP;
}
