// Keys and values in 4 bits: into the cache and out of it.
//
// 32 channels of a token share a scale s, the smallest power of two with max|x| <= 7 s (at least 2^-126), and a code holds x / s
// rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (sign and magnitude; ties to the even code; 6 .. 7 go to 6, which is
// as near as the next step, 8, would be).  A power of two makes x / s exact, so a code depends on no rounding but its own, and
// the instructions that convert between such codes and bfloat16 take the scale as an operand.  The kernels move bytes: an element is 2
// bytes on one side and 17/32 on the other.  4 680 tokens of 12 x 128, K and V:
// 7.2 us in, 7.0 out (36 MB each, partly out of the caches); 32 760 of them written for the bfloat16 attention: 254 MB in 53 us, 4.7 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lf_rollout.h"

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct KvqArgs {
  uint16_t* rows[2];             // K, V in bfloat16
  int64_t stride_tok[2], stride_head[2];
  uint8_t* codes[2];
  uint8_t* scales[2];
  int H, capacity, first, tokens;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

union Pair {
  uint32_t u;
  bf16x2 v;
};

// A thread takes 8 channels, the four lanes of a group agree on its scale.
template <int D>
__global__ __launch_bounds__(256) void lf_kvq_append_kernel(KvqArgs a) {
  constexpr int CH = D / 8;
  const int item = blockIdx.x * 256 + threadIdx.x;
  const int t = item / CH, c = item % CH;
  if (t >= a.tokens) return;                        // all lanes of a group leave together
  const int h = blockIdx.y % a.H, which = blockIdx.y / a.H;
  const uint4 x = *reinterpret_cast<const uint4*>(a.rows[which] + (int64_t)h * a.stride_head[which] + (int64_t)t * a.stride_tok[which] + 8 * c);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t top = 0;                                 // the largest magnitude's bits: bfloat16 magnitudes order as integers
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
    top = max(top, max(lo, hi));
  }
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  // top = m 2^(E - 127), m = 1 + low 7 bits / 128: m <= 1.75 fits with 2^(E - 127 - 2), a larger one with twice that
  int e = (int)(top >> 7) - ((top & 0x7fu) > 96u ? 1 : 2);
  e = max(e, 1);
  const bool fine = top < 0x7f80u;
  const float scale = __uint_as_float((uint32_t)e << 23);
  uint32_t code = 0;
  Pair p;
  p.u = w[0]; code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, p.v, scale, 0);
  p.u = w[1]; code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, p.v, scale, 1);
  p.u = w[2]; code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, p.v, scale, 2);
  p.u = w[3]; code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, p.v, scale, 3);
  const int64_t row = (int64_t)h * a.capacity + a.first + t;
  *reinterpret_cast<uint32_t*>(a.codes[which] + row * (D / 2) + 4 * c) = fine ? code : 0u;     // (past the caches: 45 -> 50 us)
  if (c % 4 == 0) a.scales[which][row * (D / 32) + c / 4] = (uint8_t)(fine ? e : 255);
}

// 8 codes to 8 bfloat16 values; scale byte 255 gives NaN.
__device__ __forceinline__ uint4 values8(uint32_t code, uint32_t byte) {
  const float scale = __uint_as_float(byte << 23);
  Pair p[4];
  p[0].v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0);
  p[1].v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1);
  p[2].v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2);
  p[3].v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
  return make_uint4(p[0].u, p[1].u, p[2].u, p[3].u);
}

template <int D>
__global__ __launch_bounds__(256) void lf_kvq_read_kernel(KvqArgs a) {
  constexpr int CH = D / 8;
  const int item = blockIdx.x * 256 + threadIdx.x;
  const int t = item / CH, c = item % CH;
  if (t >= a.tokens) return;
  const int h = blockIdx.y % a.H, which = blockIdx.y / a.H;
  const int64_t row = (int64_t)h * a.capacity + a.first + t;
  const uint32_t code = *reinterpret_cast<const uint32_t*>(a.codes[which] + row * (D / 2) + 4 * c);
  const uint4 y = values8(code, a.scales[which][row * (D / 32) + c / 4]);
  // past the caches: 4 680 tokens of 40 heads stored and read 45.0 -> 43.7 us
  __builtin_nontemporal_store(u32x4{y.x, y.y, y.z, y.w}, reinterpret_cast<u32x4*>(a.rows[which] + (int64_t)h * a.stride_head[which] + (int64_t)t * a.stride_tok[which] + 8 * c));
}

// The rows that the bfloat16 attention kernels read: tokens [0, tokens) from the cache, tokens [tokens, total) from K and V.
struct ExpandArgs {
  const uint8_t *codes[2], *scales[2];
  const uint16_t* more[2];
  int64_t stride_tok[2], stride_head[2];
  uint16_t* out[2];              // [H][total][d]
  int H, capacity, tokens, total;
};
template <int D>
__global__ __launch_bounds__(256) void lf_kvq_expand_kernel(ExpandArgs a) {
  constexpr int CH = D / 8;
  const int item = blockIdx.x * 256 + threadIdx.x;
  const int t = item / CH, c = item % CH;
  if (t >= a.total) return;
  const int h = blockIdx.y % a.H, which = blockIdx.y / a.H;
  uint4 y;
  if (t < a.tokens) {
    const int64_t row = (int64_t)h * a.capacity + t;
    y = values8(*reinterpret_cast<const uint32_t*>(a.codes[which] + row * (D / 2) + 4 * c), a.scales[which][row * (D / 32) + c / 4]);
  } else {
    y = *reinterpret_cast<const uint4*>(a.more[which] + (int64_t)h * a.stride_head[which] + (int64_t)(t - a.tokens) * a.stride_tok[which] + 8 * c);
  }
  // (the attention reads it next: past the caches the call takes 369 us instead of 364 on the last chunk of the 12-head rollout)
  *reinterpret_cast<uint4*>(a.out[which] + ((int64_t)h * a.total + t) * D + 8 * c) = y;
}

KvqArgs kvq_args(const void* K, const void* V, const lf_kvq_shape* s, const lf_kvq_rows* r, const uint8_t* cache) {
  const lf_kvq_parts p = lf_kvq_layout(*s);
  KvqArgs a;
  a.rows[0] = (uint16_t*)K;
  a.rows[1] = (uint16_t*)V;
  a.stride_tok[0] = r->k_stride_tok;
  a.stride_tok[1] = r->v_stride_tok;
  a.stride_head[0] = r->k_stride_head;
  a.stride_head[1] = r->v_stride_head;
  for (int i = 0; i < 2; ++i) {
    a.codes[i] = const_cast<uint8_t*>(cache) + p.codes[i];
    a.scales[i] = const_cast<uint8_t*>(cache) + p.scales[i];
  }
  a.H = s->heads;
  a.capacity = s->capacity;
  a.first = r->first;
  a.tokens = r->tokens;
  return a;
}

dim3 grid_of(const lf_kvq_shape* s, int tokens) {
  return dim3((unsigned)(((int64_t)tokens * (s->head_dim / 8) + 255) / 256), (unsigned)(2 * s->heads));
}

}  // namespace

int lf_launch_kvq_append(const void* K, const void* V, const lf_kvq_shape* s, const lf_kvq_rows* r, uint8_t* cache, void* stream) {
  const KvqArgs a = kvq_args(K, V, s, r, cache);
  const hipError_t rc = lf_launch(s->head_dim == 128 ? lf_kvq_append_kernel<128> : lf_kvq_append_kernel<64>, grid_of(s, r->tokens),
                                  dim3(256), 0, (hipStream_t)stream, a);
  return rc == hipSuccess ? LF_OK : LF_ERR_HIP;
}

int lf_launch_kvq_read(const uint8_t* cache, const lf_kvq_shape* s, const lf_kvq_rows* r, void* K, void* V, void* stream) {
  const KvqArgs a = kvq_args(K, V, s, r, cache);
  const hipError_t rc = lf_launch(s->head_dim == 128 ? lf_kvq_read_kernel<128> : lf_kvq_read_kernel<64>, grid_of(s, r->tokens),
                                  dim3(256), 0, (hipStream_t)stream, a);
  return rc == hipSuccess ? LF_OK : LF_ERR_HIP;
}

int lf_launch_kvq_expand(const lf_kvq_call* c, uint16_t* K, uint16_t* V, void* stream) {
  const lf_kvq_parts p = lf_kvq_layout(c->cs);
  ExpandArgs a;
  for (int i = 0; i < 2; ++i) {
    a.codes[i] = c->cache + p.codes[i];
    a.scales[i] = c->cache + p.scales[i];
  }
  a.more[0] = (const uint16_t*)c->K;
  a.more[1] = (const uint16_t*)c->V;
  a.stride_tok[0] = c->k_stride_tok;
  a.stride_tok[1] = c->v_stride_tok;
  a.stride_head[0] = c->k_stride_head;
  a.stride_head[1] = c->v_stride_head;
  a.out[0] = K;
  a.out[1] = V;
  a.H = c->H;
  a.capacity = c->cs.capacity;
  a.tokens = c->cached;
  a.total = c->cached + c->extra;
  const hipError_t rc = lf_launch(c->d == 128 ? lf_kvq_expand_kernel<128> : lf_kvq_expand_kernel<64>, grid_of(&c->cs, a.total),
                                  dim3(256), 0, (hipStream_t)stream, a);
  return rc == hipSuccess ? LF_OK : LF_ERR_HIP;
}
