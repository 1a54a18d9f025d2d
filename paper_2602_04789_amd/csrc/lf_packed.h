// Shared by the kernels of the packed attention: arguments, where a sequence lies and what its rows see, tiles in LDS.
#ifndef LF_PACKED_H
#define LF_PACKED_H

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "lf_blocks.h"
#include "lf_slots.h"

struct PackedArgs {
  const uint16_t *Q, *K, *V, *dO;
  uint16_t *O, *dQ, *dK, *dV;
  float *lse2, *ndelta, *nlse;   // nlse: -lse2 / c
  const int32_t *q_start, *kv_start;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;
  int H, Hk, G, seqs, q_len, kv_len, unit;
  int slots, parts, part_tokens;
  float c, scale;       // softmax_scale log2 e, softmax_scale
  float* state_o;       // divided calls: [tile][part][rows][D], unnormalised
  float2* state_ml;     //                [tile][part][rows], (reference, sum)
};

PackedArgs lf_packed_args(const lf_packed_call* c);
int lf_launch_packed_attn_wide(PackedArgs a, hipStream_t st);
int lf_launch_packed_dkv_wide(const PackedArgs& a, hipStream_t st);
int lf_launch_packed_join(const PackedArgs& a, int d, int tile_rows, bool few, hipStream_t st);

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int int32x4 __attribute__((ext_vector_type(4)));

union Frag {
  u32x4 u;
  bf16x8 v;
};

#define LDS_PTR(T, p) ((__attribute__((address_space(3))) T*)(p))

constexpr int vmcnt_imm(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }

// A sequence: rows [q0, q0 + nq), tokens [k0, k0 + nk).  Inside the tensors whatever the arrays hold.
struct Span {
  int q0, nq, k0, nk;
};
__device__ __forceinline__ int clamped(int at, int len) { return min(max(at, 0), len); }
__device__ __forceinline__ Span span_of(const PackedArgs& a, int b) {
  Span s;
  s.q0 = clamped(a.q_start[b], a.q_len);
  s.nq = max(clamped(a.q_start[b + 1], a.q_len) - s.q0, 0);
  s.k0 = clamped(a.kv_start[b], a.kv_len);
  s.nk = max(clamped(a.kv_start[b + 1], a.kv_len) - s.k0, 0);
  return s;
}

// Tiles of `rows` rows of all sequences without a table of them: place b < seqs is the first tile of sequence b, and behind those come the other tiles
// of each sequence.  With 64 sequences or fewer these are counted, so places that hold nothing are the last ones (workgroups that end at once at every
// second or fourth place leave half or three quarters of the chip idle: the dispatcher gives the shader engines workgroups in turn; 16 sequences of 240
// rows, 8 heads: 1065 us, and counted 351).  With more sequences those of sequence b start at floor(start_b / rows), which leaves as many places as it has or
// more.  `mul`: rows of a start's unit.  Returns the sequence, and the tile in it, of a place; a place that holds none gives a tile behind its
// sequence's last one, or -1.
__device__ __forceinline__ int others_upto(int x) {       // inclusive sum over the lanes
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);      // row_shr:1, 2, 4, 8: inside 16 lanes
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // row_bcast:15 into the second and fourth 16, :31 into the upper half
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
__device__ __forceinline__ int64_t place_of(int start, int len, int mul, int shift) { return (int64_t)clamped(start, len) * mul >> shift; }
__device__ __forceinline__ int find_tile(const int32_t* start, int seqs, int len, int mul, int rows, int place, int& tile) {
  const int shift = __builtin_ctz(rows);
  tile = 0;
  if (place < seqs) return place;
  place -= seqs;
  tile = 1 + place;
  if (seqs == 1) return 0;
  const int lane = threadIdx.x & 63;
  if (seqs <= 64) {
    int others = 0;
    if (lane < seqs) {
      const int64_t n = (int64_t)max(clamped(start[lane + 1], len) - clamped(start[lane], len), 0) * mul;
      others = (int)min(max((n - 1) >> shift, (int64_t)0), (int64_t)1 << 24);        // (a grid has fewer: starts of any values add up to less than 2^31)
    }
    const int upto = others_upto(others);
    const unsigned long long behind = __ballot(upto > place);
    if (behind == 0ull) {
      tile = -1;
      return 0;
    }
    const int b = __builtin_amdgcn_readfirstlane(__ffsll((long long)behind) - 1);
    tile = 1 + place - __builtin_amdgcn_readlane(upto - others, b);
    return b;
  }
  int lo = 0, hi = seqs;
  while (hi - lo > 64) {
    const int mid = (lo + hi) >> 1;
    if (place_of(start[mid], len, mul, shift) <= place) lo = mid; else hi = mid;
  }
  const int b = lo + lane;
  const unsigned long long below = __ballot(b < hi && place_of(start[min(b, seqs)], len, mul, shift) <= place);
  const int seq = lo + __builtin_amdgcn_readfirstlane(63 - __clzll((long long)(below | 1ull)));
  tile = below == 0ull ? -1 : 1 + (int)(place - place_of(__builtin_amdgcn_readfirstlane(start[seq]), len, mul, shift));
  return seq;
}

// How many of its sequence's tokens row i sees.
__device__ __forceinline__ int row_limit(const Span& s, int unit, int i) {
  if (unit == 0) return s.nk;
  const int p = s.nk - s.nq + i;
  if (p < 0) return 0;
  return (int)min((int64_t)s.nk, ((int64_t)(p / unit) + 1) * unit);
}
// The first row that sees token j (rows see a token or all rows behind them do).
__device__ __forceinline__ int first_row(const Span& s, int unit, int j) {
  if (unit == 0) return 0;
  return (int)max((int64_t)0, (int64_t)(j / unit) * unit - s.nk + s.nq);
}
// How a divided tile's tokens [0, seen) are shared: tokens of a part.
__device__ __forceinline__ int part_len(const PackedArgs& a, int seen) {
  return max(a.part_tokens, ((seen + a.parts - 1) / a.parts + 63) / 64 * 64);
}

// 16-byte chunks of a row in LDS, swizzled for two ways of reading.  Rows: 16 lanes take one chunk of 16 neighbouring rows.
template <int CH> __device__ __forceinline__ int row_swz(int row, int ch) { return ch ^ (CH == 16 ? row & 15 : (row >> 1) & 7); }

// Rows [.., + count) of a tensor as a buffer: what lies behind them reads as zeros.
__device__ __forceinline__ int32x4 rows_rsrc(const uint16_t* base, int64_t first, int count, uint32_t row_bytes) {
  int32x4 rs;
  const uint64_t b = (uint64_t)base + (uint64_t)first * row_bytes;
  rs[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)b);
  rs[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32));      // stride 0: raw buffer
  rs[2] = __builtin_amdgcn_readfirstlane((int)((uint32_t)max(count, 0) * row_bytes));
  rs[3] = 0x00020000;
  return rs;
}
// N loads of 1 KB each of a wavefront, memory to LDS: load i goes to lds + 1024 i, and `off[i]` has 1024 (i mod 4) taken off.
template <int N> __device__ __forceinline__ void fetch(int32x4 rs_, uint32_t lds, const uint32_t* off) {
  const int32x4 rs = aged(rs_);
  const uint32_t at = __builtin_amdgcn_readfirstlane(lds);
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                   "buffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                   "buffer_load_dwordx4 %2, %5, 0 offen offset:1024 lds\n\t"
                   "buffer_load_dwordx4 %3, %5, 0 offen offset:2048 lds\n\t"
                   "buffer_load_dwordx4 %4, %5, 0 offen offset:0xc00 lds"
                   :: "s"(at + 1024u * i), "v"(off[i]), "v"(off[i + 1]), "v"(off[i + 2]), "v"(off[i + 3]), "s"(rs) : "memory", "m0");
  } else if constexpr (N == 2) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %2, %3, 0 offen offset:1024 lds"
                 :: "s"(at), "v"(off[0]), "v"(off[1]), "s"(rs) : "memory", "m0");
  } else {
    static_assert(N == 1, "one, two or a multiple of four");
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(at), "v"(off[0]), "s"(rs) : "memory", "m0");
  }
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)LDS_PTR(void, (void*)p); }

// Orders LDS accesses of the workgroup; loads to LDS are waited for by the wavefront that made them, ahead of it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}

}  // namespace
#endif
