// RMSNorm, then rotary positions over three axes, written head-major, and the gradients of both.
//
//   forward   y = R(theta) (x inv g),  inv = 1 / sqrt(mean(x^2) + eps),  theta_i = pos[axis(i)] freq[i]
//   backward  z = R(-theta) dy;  dg = sum over tokens of z (x inv);  u = z g;
//             dx = inv (u - (x inv) mean(u x inv)),  the mean over the channels that the norm takes
//
// HBM-bound: the forward reads and writes 2 bytes an element, the backward reads 4 and writes 2.  The angles are made from
// 12 bytes a token instead of being read as two float tables of d/2 (512 bytes a token at d = 128, as much as one more head).
//
// A thread owns the 16-byte chunk `cih` (8 channels) of up to NI heads of one token, so it makes that chunk's angles once for
// all of them.  The CH = d/8 chunks of a head are neighbouring lanes of one wavefront (64 is a multiple of CH): a head's
// sums are taken across CH lanes, and the partner of a channel pair (i, i + d/2) is CH/2 lanes away.  Sums over all heads of a
// token go through LDS.  All arithmetic is float32 but for the angles: they are products of float64, reduced to
// half a turn either way there, so far positions keep their phase.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lf_rollout.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct AxesArgs {
  const uint16_t* X;
  const float* g;
  const int32_t* pos;
  const double* freq;
  uint16_t* Y;           // forward: written
  const uint16_t* dY;    // backward
  uint16_t* dX;
  float* part;           // [blocks][H d]
  int64_t x_stride_tok, y_stride_tok, y_stride_head;
  int H, L, across_heads, pairing;
  int axis1, axis2;      // first pair of the second and of the third axis
  int hpt, tt;           // heads side by side, tokens of a workgroup
  float eps;
};

__device__ __forceinline__ void unpack8(const uint4& u, float (&x)[8]) {
  x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xffff0000u);
  x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xffff0000u);
  x[4] = __uint_as_float(u.z << 16); x[5] = __uint_as_float(u.z & 0xffff0000u);
  x[6] = __uint_as_float(u.w << 16); x[7] = __uint_as_float(u.w & 0xffff0000u);
}

// Cosine and sine of pos * freq.  In turns, less the nearest whole number, in float64; the hardware's functions take turns and are off by
// 2^-22.9 at the most on [-1/2, 1/2] (4 194 304 values), as a float32 series would be.
__device__ __forceinline__ void angle(int pos, double freq, float& c, float& s) {
  const double t = (double)pos * (freq * 0.15915494309189533577);   // 1 / (2 pi)
  const float x = (float)(t - __builtin_rint(t));
  c = __builtin_amdgcn_cosf(x);
  s = __builtin_amdgcn_sinf(x);
}

// The angles of a thread's chunk: pairs (2i, 2i + 1) are four to a chunk; of pairs (i, i + d/2) a chunk holds one side of eight.
template <int CH, int PAIRING>
__device__ __forceinline__ void angles(const AxesArgs& a, int tok, int cih, float (&cs)[PAIRING ? 8 : 4], float (&sn)[PAIRING ? 8 : 4]) {
  constexpr int N = PAIRING ? 8 : 4;
  const int i0 = PAIRING ? 8 * (cih % (CH / 2)) : 4 * cih;
  const int32_t* p = a.pos + 3 * (int64_t)tok;
  const int p0 = p[0], p1 = p[1], p2 = p[2];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int i = i0 + e;
    angle(i < a.axis1 ? p0 : i < a.axis2 ? p1 : p2, a.freq[i], cs[e], sn[e]);
  }
}

// Exchanges among the CH lanes of a head (8 or 16, inside a row of 16) without LDS: quad_perm 0xb1 and 0x4e are lane ^ 1 and ^ 2, 0x1b is ^ 3,
// row_half_mirror (0x141) is ^ 7, row_ror:n (0x120 + n) rotates the row.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int CH> __device__ __forceinline__ float partner(float v) {      // of lane ^ CH/2
  if constexpr (CH == 16) return dpp<0x128>(v);
  else return dpp<0x1b>(dpp<0x141>(v));
}
template <int CH> __device__ __forceinline__ float head_sum(float v) {     // in all CH lanes
  if constexpr (CH == 16) {
    v += dpp<0x128>(v);
    v += dpp<0x124>(v);
    v += dpp<0x122>(v);
    v += dpp<0x121>(v);
  } else {
    v += dpp<0x141>(v);
    v += dpp<0xb1>(v);
    v += dpp<0x4e>(v);
  }
  return v;
}

// Turns a chunk by its angles (SIGN = 1) or back (-1).
template <int CH, int PAIRING, int SIGN>
__device__ __forceinline__ void turn(const float (&y)[8], const float (&cs)[PAIRING ? 8 : 4], const float (&sn)[PAIRING ? 8 : 4],
                                     int cih, float (&r)[8]) {
  if constexpr (PAIRING == 0) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float s = SIGN * sn[p];
      r[2 * p] = y[2 * p] * cs[p] - y[2 * p + 1] * s;
      r[2 * p + 1] = y[2 * p] * s + y[2 * p + 1] * cs[p];
    }
  } else {
    const bool first = cih < CH / 2;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float other = partner<CH>(y[e]);
      const float s = first ? -SIGN * sn[e] : SIGN * sn[e];
      r[e] = y[e] * cs[e] + other * s;
    }
  }
}

// Written past the caches: rows of 256 bytes at d = 128, scattered over the heads, were what the kernels waited for (forward, us: 4 680 tokens
// of 12 heads 8.7 -> 7.2, of 40 heads 22.8 -> 17.2; 32 760 tokens of 12 heads of 64 24.5 -> 17.6).  Nontemporal loads of X bring nothing.
__device__ __forceinline__ void store8(uint16_t* at, const float (&r)[8]) {
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = (__bf16)r[e];
  __builtin_nontemporal_store(o, reinterpret_cast<bf16x8*>(at));
}

template <int D, int NI, int PAIRING>
__global__ __launch_bounds__(512) void lf_rope_axes_kernel(AxesArgs a) {
  constexpr int CH = D / 8;
  extern __shared__ float red[];
  const int cih = threadIdx.x % CH, hp = threadIdx.x / CH % a.hpt, tl = threadIdx.x / CH / a.hpt;
  const int tok = blockIdx.x * a.tt + tl;
  const bool there = tl < a.tt && tok < a.L;
  const int t = there ? tok : a.L - 1;          // threads without a token read the last one and write nothing
  const uint16_t* xrow = a.X + (int64_t)t * a.x_stride_tok + 8 * cih;
  uint4 xr[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int h = hp + i * a.hpt;
    xr[i] = h < a.H ? *reinterpret_cast<const uint4*>(xrow + h * D) : make_uint4(0, 0, 0, 0);
  }
  float cs[PAIRING ? 8 : 4], sn[PAIRING ? 8 : 4];
  angles<CH, PAIRING>(a, t, cih, cs, sn);

  float ss[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    float x[8];
    unpack8(xr[i], x);
    ss[i] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss[i] = fmaf(x[e], x[e], ss[i]);
  }
  float n = (float)D;
  if (a.across_heads) {
    float all = 0.0f;
#pragma unroll
    for (int i = 0; i < NI; ++i) all += ss[i];
    all = head_sum<CH>(all);
    if (cih == 0 && tl < a.tt) red[tl * a.hpt + hp] = all;
    __syncthreads();
    all = 0.0f;
    if (tl < a.tt)
      for (int j = 0; j < a.hpt; ++j) all += red[tl * a.hpt + j];
#pragma unroll
    for (int i = 0; i < NI; ++i) ss[i] = all;
    n = (float)(a.H * D);
  } else {
#pragma unroll
    for (int i = 0; i < NI; ++i) ss[i] = head_sum<CH>(ss[i]);
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int h = hp + i * a.hpt;
    const bool real = h < a.H;
    const float* gp = a.g + (real ? h : 0) * D + 8 * cih;
    const float4 g0 = *reinterpret_cast<const float4*>(gp), g1 = *reinterpret_cast<const float4*>(gp + 4);
    const float gg[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
    const float inv = 1.0f / sqrtf(ss[i] / n + a.eps);
    float x[8], r[8];
    unpack8(xr[i], x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * gg[e];
    turn<CH, PAIRING, 1>(x, cs, sn, cih, r);
    if (there && real) store8(a.Y + (int64_t)h * a.y_stride_head + (int64_t)tok * a.y_stride_tok + 8 * cih, r);
  }
}

// The gradients.  A workgroup takes every gridDim.x-th group of tt tokens and holds what its channels of g get in registers; at
// the end the tt tokens' shares are added up through LDS, in ascending order, and the workgroup's row goes to `part`.
template <int D, int NI, int PAIRING>
__global__ __launch_bounds__(512) void lf_rope_axes_bwd_kernel(AxesArgs a) {
  constexpr int CH = D / 8;
  extern __shared__ float red[];
  const int cih = threadIdx.x % CH, hp = threadIdx.x / CH % a.hpt, tl = threadIdx.x / CH / a.hpt;
  float acc[NI][8];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[i][e] = 0.0f;
  float gg[NI][8];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int h = hp + i * a.hpt;
    const float* gp = a.g + (h < a.H ? h : 0) * D + 8 * cih;
    const float4 g0 = *reinterpret_cast<const float4*>(gp), g1 = *reinterpret_cast<const float4*>(gp + 4);
    gg[i][0] = g0.x; gg[i][1] = g0.y; gg[i][2] = g0.z; gg[i][3] = g0.w;
    gg[i][4] = g1.x; gg[i][5] = g1.y; gg[i][6] = g1.z; gg[i][7] = g1.w;
  }
  const int groups = (a.L - 1) / a.tt + 1;
  for (int grp = blockIdx.x; grp < groups; grp += gridDim.x) {
    const int tok = grp * a.tt + tl;
    const bool there = tl < a.tt && tok < a.L;
    const int t = there ? tok : a.L - 1;
    const uint16_t* xrow = a.X + (int64_t)t * a.x_stride_tok + 8 * cih;
    const uint16_t* yrow = a.dY + (int64_t)t * a.y_stride_tok + 8 * cih;
    uint4 xr[NI], yr[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int h = hp + i * a.hpt;
      const bool real = there && h < a.H;
      xr[i] = real ? *reinterpret_cast<const uint4*>(xrow + h * D) : make_uint4(0, 0, 0, 0);
      yr[i] = real ? *reinterpret_cast<const uint4*>(yrow + (int64_t)h * a.y_stride_head) : make_uint4(0, 0, 0, 0);
    }
    float cs[PAIRING ? 8 : 4], sn[PAIRING ? 8 : 4];
    angles<CH, PAIRING>(a, t, cih, cs, sn);
    float ss[NI], ux[NI], z[NI][8];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float x[8], y[8];
      unpack8(xr[i], x);
      unpack8(yr[i], y);
      turn<CH, PAIRING, -1>(y, cs, sn, cih, z[i]);
      ss[i] = ux[i] = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss[i] = fmaf(x[e], x[e], ss[i]);
        ux[i] = fmaf(z[i][e] * gg[i][e], x[e], ux[i]);
      }
    }
    float n = (float)D;
    if (a.across_heads) {
      float s = 0.0f, u = 0.0f;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        s += ss[i];
        u += ux[i];
      }
      s = head_sum<CH>(s);
      u = head_sum<CH>(u);
      __syncthreads();      // the sums of the tokens before have been read
      if (cih == 0 && tl < a.tt) {
        red[2 * (tl * a.hpt + hp)] = s;
        red[2 * (tl * a.hpt + hp) + 1] = u;
      }
      __syncthreads();
      s = u = 0.0f;
      if (tl < a.tt)
        for (int j = 0; j < a.hpt; ++j) {
          s += red[2 * (tl * a.hpt + j)];
          u += red[2 * (tl * a.hpt + j) + 1];
        }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        ss[i] = s;
        ux[i] = u;
      }
      n = (float)(a.H * D);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        ss[i] = head_sum<CH>(ss[i]);
        ux[i] = head_sum<CH>(ux[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int h = hp + i * a.hpt;
      // threads without a token add nothing to dg: with eps = 0 their 1 / sqrt(0) times their zeros would be NaN
      const float inv = there ? 1.0f / sqrtf(ss[i] / n + a.eps) : 0.0f;
      const float mean = ux[i] * inv / n;
      float x[8], r[8];
      unpack8(xr[i], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xn = x[e] * inv;
        acc[i][e] = fmaf(z[i][e], xn, acc[i][e]);
        r[e] = inv * (z[i][e] * gg[i][e] - xn * mean);
      }
      if (there && h < a.H) store8(a.dX + (int64_t)tok * a.x_stride_tok + h * D + 8 * cih, r);
    }
  }
  // red[tl][channel]: the tokens' shares side by side, then one thread adds up a channel's
  __syncthreads();
  const int cols = a.hpt * D;                   // channels of one of a thread's heads, side by side
#pragma unroll
  for (int i = 0; i < NI; ++i)
    if (tl < a.tt) {
      float* to = red + (i * a.tt + tl) * cols + hp * D + 8 * cih;
      *reinterpret_cast<float4*>(to) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
      *reinterpret_cast<float4*>(to + 4) = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
    }
  __syncthreads();
  float* row = a.part + (int64_t)blockIdx.x * a.H * D;
  for (int c = threadIdx.x; c < a.H * D; c += blockDim.x) {
    const float* from = red + c / cols * a.tt * cols + c % cols;
    float v = 0.0f;
    for (int j = 0; j < a.tt; ++j) v += from[j * cols];
    row[c] = v;
  }
}

// dg[c] = sum over the rows of `part`, in a fixed order.  A workgroup takes 16 channels, 16 lanes side by side read one row's.
constexpr int kSumCols = 16, kSumRows = 64;
static_assert(LF_AXES_MAX_BLOCKS % kSumRows == 0, "every thread adds up the same number of rows");
__global__ __launch_bounds__(kSumCols * kSumRows) void lf_rope_axes_dg_kernel(const float* part, int rows, int cols, float* dg) {
  __shared__ float red[kSumRows][kSumCols + 1];
  const int lc = threadIdx.x % kSumCols, lr = threadIdx.x / kSumCols;
  const int c = blockIdx.x * kSumCols + lc;     // cols is a multiple of 64
  float v[LF_AXES_MAX_BLOCKS / kSumRows], s = 0.0f;
#pragma unroll
  for (int k = 0; k < LF_AXES_MAX_BLOCKS / kSumRows; ++k) v[k] = lr + k * kSumRows < rows ? part[(int64_t)(lr + k * kSumRows) * cols + c] : 0.0f;
#pragma unroll
  for (int k = 0; k < LF_AXES_MAX_BLOCKS / kSumRows; ++k) s += v[k];
  red[lr][lc] = s;
  for (int half = kSumRows / 2; half > 0; half /= 2) {
    __syncthreads();
    if (lr < half) red[lr][lc] += red[lr + half][lc];
  }
  if (lr == 0) dg[c] = red[0][lc];
}

AxesArgs axes_args(const void* X, const float* g, const int32_t* pos, const double* freq, const lf_axes_shape* p) {
  AxesArgs a = {};
  a.X = (const uint16_t*)X;
  a.g = g;
  a.pos = pos;
  a.freq = freq;
  a.x_stride_tok = p->x_stride_tok;
  a.y_stride_tok = p->y_stride_tok;
  a.y_stride_head = p->y_stride_head;
  a.H = p->heads;
  a.L = p->tokens;
  a.across_heads = p->across_heads;
  a.pairing = p->pairing;
  a.axis1 = p->pairs[0];
  a.axis2 = p->pairs[0] + p->pairs[1];
  a.eps = p->eps;
  return a;
}

template <int D, int NI>
void (*kernel_of(bool bwd, int pairing))(AxesArgs) {
  if (bwd) return pairing ? lf_rope_axes_bwd_kernel<D, NI, 1> : lf_rope_axes_bwd_kernel<D, NI, 0>;
  return pairing ? lf_rope_axes_kernel<D, NI, 1> : lf_rope_axes_kernel<D, NI, 0>;
}
template <int D>
void (*kernel_for(bool bwd, int pairing, int ni))(AxesArgs) {
  return ni == 1 ? kernel_of<D, 1>(bwd, pairing) : ni == 2 ? kernel_of<D, 2>(bwd, pairing) : kernel_of<D, 4>(bwd, pairing);
}

}  // namespace

int lf_launch_rope_axes(const void* X, const float* g, const int32_t* pos, const double* freq, const lf_axes_shape* p, void* Y,
                        void* stream) {
  AxesArgs a = axes_args(X, g, pos, freq, p);
  a.Y = (uint16_t*)Y;
  const lf_axes_lay l = lf_lay_axes_fwd(a.H, p->head_dim, a.L);
  a.hpt = l.hpt;
  a.tt = l.tt;
  const unsigned grid = (unsigned)((a.L - 1) / l.tt + 1);
  const size_t lds = a.across_heads ? sizeof(float) * l.tt * l.hpt : 0;
  const hipError_t rc = lf_launch(p->head_dim == 128 ? kernel_for<128>(false, a.pairing, l.ni) : kernel_for<64>(false, a.pairing, l.ni),
                                  dim3(grid), dim3(l.threads), lds, (hipStream_t)stream, a);
  return rc == hipSuccess ? LF_OK : LF_ERR_HIP;
}

int lf_launch_rope_axes_bwd(const void* X, const float* g, const int32_t* pos, const double* freq, const lf_axes_shape* p,
                            const void* dY, void* dX, float* dg, float* part, void* stream) {
  AxesArgs a = axes_args(X, g, pos, freq, p);
  a.dY = (const uint16_t*)dY;
  a.dX = (uint16_t*)dX;
  a.part = part;
  const lf_axes_lay l = lf_lay_axes_bwd(a.H, p->head_dim);
  a.hpt = l.hpt;
  a.tt = l.tt;
  const int blocks = lf_axes_bwd_blocks(a.H, p->head_dim, a.L);
  const size_t sums = a.across_heads ? 2 * sizeof(float) * l.tt * l.hpt : 0;
  const size_t shares = sizeof(float) * l.ni * l.tt * l.hpt * p->head_dim;      // at most 64 KiB: 512 threads of four heads
  hipStream_t st = (hipStream_t)stream;
  hipError_t rc = lf_launch(p->head_dim == 128 ? kernel_for<128>(true, a.pairing, l.ni) : kernel_for<64>(true, a.pairing, l.ni),
                            dim3(blocks), dim3(l.threads), sums > shares ? sums : shares, st, a);
  if (rc != hipSuccess) return LF_ERR_HIP;
  const int cols = a.H * p->head_dim;
  rc = lf_launch(lf_rope_axes_dg_kernel, dim3(cols / kSumCols), dim3(kSumCols * kSumRows), 0, st, (const float*)part, blocks, cols, dg);
  return rc == hipSuccess ? LF_OK : LF_ERR_HIP;
}
