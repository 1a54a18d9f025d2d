// The norm over the gradients of all parameters, and their scaling to a largest norm.
//
//   norm = sqrt(sum x^2),   out = x min(1, max_norm / (norm + eps))
//
// HBM-bound: all values are read for the norm, then read and written once more (in place only where the factor is below 1).  A workgroup takes
// a share of one tensor (16 384 to 65 536 values), so tensors of any sizes fill the chip alike; the tensors' addresses travel as
// kernel arguments, so nothing is copied to the device and a captured call keeps them.  Squares are summed in binary64 (a bfloat16 square needs 16 bits, so
// rounding sets in where a thread's sum is 2^37 times its terms), one sum a share, and the shares are added in a fixed order.
//
// The scaling goes from the last share to the first, so what the norm read last is still in the last-level cache, and its stores pass the caches by.
// 270 tensors of 850 million bfloat16 values, into others: 960 us (5.1 GB, 5.3 TB/s; 1007 us in the order of the
// norm, 980 us backwards with ordinary stores).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "lf_blocks.h"

namespace {

// Tensors of a launch, in kernel arguments of up to 4 KB; fewer make a call shorter on the host (two launches of 18 tensors: by 1.9 us).
constexpr int kMany = 120, kFew = 24;
constexpr int kThreads = 256;

struct Tensor {
  const void* data;
  void* out;
  int64_t numel;
};
template <int N> struct Batch {
  Tensor t[N];
  int32_t first[N + 1];         // shares before tensor i, in the launch
  uint8_t dtype[N];             // bit 0: data is float32, bit 1: out is
  int32_t count;
  int64_t chunk;
  const double* part;           // of the launch's first share (norm), of all shares (scale)
  int64_t parts;
  const float* factor;          // scale, where a launch of its own has made it
  float* norm;
  float max_norm, eps;
  int32_t write_norm;
};
static_assert(sizeof(Batch<kMany>) <= 4000, "kernel arguments");

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Tensors are aligned to their elements only; the memory path takes 16 bytes from any address.
typedef u32x4 __attribute__((aligned(2))) u32x4_any2;
typedef f32x4 __attribute__((aligned(4))) f32x4_any4;

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double s[kThreads / 64];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) v += s[w];
  return v;
}

// The tensor of a share of the launch, and its values [at, at + n); BACK: the last share of a tensor first.
template <bool BACK, int N> __device__ __forceinline__ int share_of(const Batch<N>& b, int share, int64_t& at, int64_t& n) {
  int lo = 0, hi = b.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (b.first[mid] <= share) lo = mid; else hi = mid;
  }
  at = (int64_t)(BACK ? b.first[lo + 1] - 1 - share : share - b.first[lo]) * b.chunk;
  n = min(b.chunk, b.t[lo].numel - at);
  return lo;
}

template <bool F32> __device__ __forceinline__ void load8(const void* base, int64_t at, float (&x)[8]) {
  if constexpr (F32) {
    const f32x4_any4* p = reinterpret_cast<const f32x4_any4*>(reinterpret_cast<const float*>(base) + at);
    const f32x4 a = p[0], b = p[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = a[e];
      x[4 + e] = b[e];
    }
  } else {
    const u32x4 w = *reinterpret_cast<const u32x4_any2*>(reinterpret_cast<const uint16_t*>(base) + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}
template <bool F32> __device__ __forceinline__ float load1(const void* base, int64_t at) {
  if constexpr (F32) return reinterpret_cast<const float*>(base)[at];
  else return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(base)[at] << 16);
}
template <bool F32> __device__ __forceinline__ void store8(void* base, int64_t at, const float (&x)[8]) {
  if constexpr (F32) {
    f32x4_any4* p = reinterpret_cast<f32x4_any4*>(reinterpret_cast<float*>(base) + at);
    __builtin_nontemporal_store(f32x4_any4{x[0], x[1], x[2], x[3]}, p);
    __builtin_nontemporal_store(f32x4_any4{x[4], x[5], x[6], x[7]}, p + 1);
  } else {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (__bf16)x[e];
    __builtin_nontemporal_store((u32x4_any2)__builtin_bit_cast(u32x4, o), reinterpret_cast<u32x4_any2*>(reinterpret_cast<uint16_t*>(base) + at));
  }
}
template <bool F32> __device__ __forceinline__ void store1(void* base, int64_t at, float x) {
  if constexpr (F32) reinterpret_cast<float*>(base)[at] = x;
  else reinterpret_cast<__bf16*>(base)[at] = (__bf16)x;
}

template <bool F32> __device__ __forceinline__ double squares(const void* data, int64_t at, int64_t n) {
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  const int64_t whole = n & ~(int64_t)7;
#pragma unroll 4
  for (int64_t i = 8 * threadIdx.x; i < whole; i += 8 * kThreads) {
    float x[8];
    load8<F32>(data, at + i, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e & 3] = fma((double)x[e], (double)x[e], s[e & 3]);
  }
  if (threadIdx.x < n - whole) {
    const double x = load1<F32>(data, at + whole + threadIdx.x);
    s[0] = fma(x, x, s[0]);
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

template <int N> __global__ __launch_bounds__(kThreads) void lf_grad_square_kernel(Batch<N> b) {
  int64_t at, n;
  const int i = share_of<false>(b, blockIdx.x, at, n);
  const double s = block_sum(b.dtype[i] & 1 ? squares<true>(b.t[i].data, at, n) : squares<false>(b.t[i].data, at, n));
  if (threadIdx.x == 0) const_cast<double*>(b.part)[blockIdx.x] = s;
}

// min(1, max_norm / (norm + eps)) from the sum of squares, 1 where that is not finite; the norm to `norm` if asked for.
__device__ __forceinline__ float factor_of(double sum, float max_norm, float eps, float* norm) {
  const double n = sqrt(sum);
  if (norm) *norm = (float)n;
  if (!(n < (double)INFINITY)) return 1.0f;
  const double f = (double)max_norm / (n + (double)eps);
  return f < 1.0 ? (float)f : 1.0f;
}
__device__ __forceinline__ double sum_parts(const double* part, int64_t parts) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < parts; i += 16 * kThreads) {        // loads at once: 13 000 parts 19 us one after another
    double v[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = part[min(i + k * kThreads, parts - 1)];
#pragma unroll
    for (int k = 0; k < 16; ++k) s += i + k * kThreads < parts ? v[k] : 0.0;
  }
  return block_sum(s);
}
__global__ __launch_bounds__(kThreads) void lf_grad_norm_kernel(const double* part, int64_t parts, float max_norm, float eps, float* norm, float* factor) {
  const double s = sum_parts(part, parts);
  if (threadIdx.x == 0) *factor = factor_of(s, max_norm, eps, norm);
}

template <bool F32, bool OUT32> __device__ __forceinline__ void scaled(const void* data, void* out, int64_t at, int64_t n, float f) {
  const int64_t whole = n & ~(int64_t)7;
#pragma unroll 4
  for (int64_t i = 8 * threadIdx.x; i < whole; i += 8 * kThreads) {
    float x[8];
    load8<F32>(data, at + i, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= f;
    store8<OUT32>(out, at + i, x);
  }
  if (threadIdx.x < n - whole) store1<OUT32>(out, at + whole + threadIdx.x, f * load1<F32>(data, at + whole + threadIdx.x));
}

template <int N> __global__ __launch_bounds__(kThreads) void lf_grad_scale_kernel(Batch<N> b) {
  float f;
  if (b.factor) {
    f = *b.factor;
  } else {
    const double s = sum_parts(b.part, b.parts);
    f = factor_of(s, b.max_norm, b.eps, b.write_norm && blockIdx.x == 0 && threadIdx.x == 0 ? b.norm : nullptr);
  }
  int64_t at, n;
  const int i = share_of<true>(b, blockIdx.x, at, n);
  const void* data = b.t[i].data;
  void* out = b.t[i].out;
  if (data == out && f == 1.0f) return;
  switch (b.dtype[i]) {
    case 0: scaled<false, false>(data, out, at, n, f); break;
    case 1: scaled<true, false>(data, out, at, n, f); break;
    case 2: scaled<false, true>(data, out, at, n, f); break;
    default: scaled<true, true>(data, out, at, n, f);
  }
}

template <int N>
int launch(const lf_grad_tensor* t, int32_t count, int64_t numel, float max_norm, float eps, float* norm, double* part, hipStream_t st) {
  const int64_t chunk = lf_grad_chunk(numel);
  Batch<N> b;
  auto launch_all = [&](auto kernel, bool square) {
    int64_t done = 0;           // shares of the launches before
    bool first = true;
    for (int32_t i = 0; i < count;) {
      b.count = 0;
      b.first[0] = 0;
      for (; i < count && b.count < N; ++i) {
        const lf_grad_tensor& x = t[square ? i : count - 1 - i];
        if (x.numel == 0) continue;
        void* out = x.out ? x.out : const_cast<void*>(x.data);
        if (!square && out == x.data && max_norm == INFINITY) continue;         // the factor is 1 whatever the norm is
        const int64_t shares = (x.numel + chunk - 1) / chunk;
        if (b.count > 0 && b.first[b.count] + shares > (1 << 23)) break;    // a grid has less than 2^32 threads
        b.t[b.count] = {x.data, out, x.numel};
        b.dtype[b.count] = (uint8_t)((x.dtype == LF_F32 ? 1 : 0) | ((x.out ? x.out_dtype : x.dtype) == LF_F32 ? 2 : 0));
        b.first[b.count + 1] = (int32_t)(b.first[b.count] + shares);
        ++b.count;
      }
      if (b.count == 0) break;
      b.chunk = chunk;
      if (square) b.part = part + done;
      b.write_norm = first;
      first = false;
      if (lf_launch(kernel, dim3((unsigned)b.first[b.count]), dim3(kThreads), 0, st, b) != hipSuccess) return (int64_t)-1;
      done += b.first[b.count];
    }
    return done;
  };
  b.norm = norm;
  b.max_norm = max_norm;
  b.eps = eps;
  b.factor = nullptr;
  b.parts = 0;
  const int64_t parts = launch_all(lf_grad_square_kernel<N>, true);
  if (parts < 0) return LF_ERR_HIP;
  b.part = part;
  b.parts = parts;
  bool writes = false;
  for (int32_t i = 0; i < count; ++i) writes = writes || (t[i].numel > 0 && ((t[i].out && t[i].out != t[i].data) || max_norm != INFINITY));
  // Few shares are added by every workgroup of the scaling launch by itself, more of them (or without that launch) by a launch of their own (with and
  // without it, us: 75 shares 7.6 and 6.7, 768 shares 13.2 and 12.7, four times as many 25.0 and 26.8).
  if (!writes || parts > 1024) {
    float* factor = reinterpret_cast<float*>(part + lf_grad_most_chunks(count, numel));
    if (lf_launch(lf_grad_norm_kernel, dim3(1), dim3(kThreads), 0, st, (const double*)part, parts, max_norm, eps, norm, factor) != hipSuccess)
      return LF_ERR_HIP;
    b.factor = factor;
  }
  return writes && launch_all(lf_grad_scale_kernel<N>, false) < 0 ? LF_ERR_HIP : LF_OK;
}

}  // namespace

int lf_launch_grad_clip(const lf_grad_tensor* t, int32_t count, int64_t numel, float max_norm, float eps, float* norm, double* part,
                        void* stream) {
  return (count <= kFew ? launch<kFew> : launch<kMany>)(t, count, numel, max_norm, eps, norm, part, (hipStream_t)stream);
}
