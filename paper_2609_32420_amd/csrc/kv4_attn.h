// What the kernels of attention over 4-bit cached keys and values share.
#pragma once

#include "internal.h"

#include <math.h>

namespace carnator {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxChunks = 256;
constexpr int kShortJoin = 32;  // parts that join_kernel loads at once
// Growth of the running maximum (log2 units) below which O and l keep their
// scale: P may then reach 2^8, harmless in fp32 and bf16.
constexpr float kSlack = 8.f;

// Two channels (or tokens) of byte SEL of `codes` as bf16, under the exponent
// bits of `scale` (the conversion reads no other bit of it).
template <int SEL>
__device__ inline uint32_t pair_of(uint32_t codes, uint32_t scale) {
  return __builtin_bit_cast(uint32_t,
                            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, __builtin_bit_cast(float, scale), SEL));
}
// Eight channels: four bytes under one scale.
__device__ inline bf16x8 eight_of(uint32_t codes, uint32_t scale) {
  return __builtin_bit_cast(bf16x8, u32x4{pair_of<0>(codes, scale), pair_of<1>(codes, scale),
                                          pair_of<2>(codes, scale), pair_of<3>(codes, scale)});
}

// 1 / l; 0 where nothing was seen.
__device__ inline float inverse(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN; }
// Natural log-sum-exp from a reference m (log2 units) and the sum beside it:
// reference, exponent and log2 of the mantissa are added in fp64, since the
// first two can be large where the result is small.
__device__ inline float lse_of(float m, float l) {
  const double l2 = (double)m + (double)__builtin_amdgcn_frexp_expf(l) + (double)__log2f(__builtin_amdgcn_frexp_mantf(l));
  return l > 0.f ? (float)(l2 * 0.69314718055994531) : l == 0.f ? -INFINITY : NAN;
}

// What a request's queries are and see.
struct Span {
  int q0;     // first query row
  int m;      // queries (before max_q), for the causal limit
  int rows;   // query rows times heads of a cached head
  int kv;     // tokens
  __device__ int limit(const Kv4Attn &a, int i) const {  // tokens that query i sees
    return a.causal ? min(max(kv - m + i + 1, 0), kv) : kv;
  }
};
__device__ inline Span span_from(const Kv4Attn &a, int q0, int q1, int kv) {
  Span s;
  s.q0 = min(max(q0, 0), a.n_rows);
  s.m = min(max(q1, s.q0), a.n_rows) - s.q0;
  s.rows = min(s.m, a.max_q) * a.group;
  s.kv = min(max(kv, 0), a.width << a.c.shift);
  return s;
}
// Of a request that all lanes ask for, and of each lane's own.
__device__ inline Span span_of(const Kv4Attn &a, int b) {
  return span_from(a, __builtin_amdgcn_readfirstlane(a.q_start[b]), __builtin_amdgcn_readfirstlane(a.q_start[b + 1]),
                   __builtin_amdgcn_readfirstlane(a.kv_len[b]));
}
__device__ inline Span lane_span_of(const Kv4Attn &a, int b) {
  return span_from(a, a.q_start[b], a.q_start[b + 1], a.kv_len[b]);
}
// Tokens that the last of 16 NT rows from row0 on sees: what a tile walks.
__device__ inline int tile_end(const Kv4Attn &a, const Span &s, int row0, int rows) {
  return s.limit(a, (min(row0 + rows, s.rows) - 1) / a.group);
}

// How a kernel cuts its share of a call, the requests of more than `over` and at
// most `upto` rows: tiles of tile_rows rows, and parts of the key axis of `chunk`
// tokens whose results another kernel joins.
struct Cut {
  int over, upto;
  int tile_rows, tiles, chunk, chunks;
  int turns;  // of the kernel for many rows: a turn is a tile of every request
  int items;  // tiles of its grid, each found in the turns by its number; 0: the grid holds the turns
  int columns;  // parts that the grid holds, and results of a row; a workgroup takes every columns-th part
  int span;   // rows of a request and cached head that parts are kept for; 0: parts are kept by query row
  __device__ bool has(const Span &s) const { return s.rows > over && s.rows <= upto; }
};
constexpr int kFindBatch = 1024;  // requests among which a tile is found by its number at a time
// Workgroups of a cut.
inline int64_t tile_groups(const Kv4Attn &a, const Cut &cut) {
  return (cut.items ? (int64_t)cut.items : (int64_t)cut.turns * a.batch) * a.c.heads * cut.columns;
}
// Empty turns before a request's tiles: those of a request that ends `late` tiles'
// tokens before the table does are that much later, so that a causal batch goes by
// what its tiles see.
template <int ROWS>
__device__ inline int late_of(const Kv4Attn &a, const Cut &cut, const Span &s) {
  return cut.turns > cut.tiles ? (int)((int64_t)((a.width << a.c.shift) - s.kv) * a.group / ROWS) : 0;
}
// Results of the parts: outputs [..][columns][d] not yet divided, (reference,
// rounded sum, sum) beside them, by query row and head or, where that is less (a
// padded batch, or one of few rows to a request), by request, cached head and row.
struct Parts {
  float *o;
  float4 *ml;
};
__device__ inline int64_t part_of(const Kv4Attn &a, const Cut &cut, const Span &s, int b, int h, int row, int i, int hd) {
  return (cut.span ? ((int64_t)b * a.c.heads + h) * cut.span + row : (int64_t)(s.q0 + i) * a.heads + hd) * cut.columns;
}

// The kernel for many rows (kv4_tile_kernels.hip), without the joining; its first or
// last few_groups workgroups take the batch's requests of few rows.
hipError_t launch_kv4_tiles(const Kv4Attn &a, const Cut &few, const Parts &few_parts, int few_groups, const Cut &cut,
                            const Parts &parts, hipStream_t s);

}  // namespace carnator
