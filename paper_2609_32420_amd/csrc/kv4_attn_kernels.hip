// Attention over cached keys and values in 4 bits: the kernel for requests of few
// rows alone (its work is in kv4_rows.h), the joining of parts of the key axis, and
// how a call is launched.
#include "kv4_cut.h"
#include "kv4_rows.h"

namespace carnator {
namespace {

template <int D, int NT, bool SPLIT>
__global__ void __launch_bounds__(64 * kWaves, NT * D <= 128 ? 3 : 2)
rows_kernel(Kv4Attn a, Cut cut, Parts parts) {
  extern __shared__ float lds_rows[];
  rows_body<D, NT, SPLIT, kWaves>(a, cut, parts, (int)blockIdx.x, lds_rows);
}

// Query i of request b, by its number: most to a request (most > 0), or by its row
// (a ragged batch has far fewer of these).
struct Query {
  int b, i;  // b < 0: of no request
};
__device__ inline Query query_of(const Kv4Attn &a, int64_t id, int most) {
  if (most) return Query{(int)(id / most) < a.batch ? (int)(id / most) : -1, (int)(id % most)};
  int b = 0, end = a.batch;
  if (id >= a.n_rows || id < a.q_start[0] || id >= a.q_start[end]) return Query{-1, 0};
  while (end - b > 1) {  // q_start[b] <= id < q_start[end]
    const int mid = (b + end) >> 1;
    if (a.q_start[mid] <= id) b = mid;
    else end = mid;
  }
  return Query{b, (int)id - max(a.q_start[b], 0)};
}

// Joins the parts of a query row and head, in their order: a wave sums every
// fourth part, 64 lanes over the channels.  SHORT: 32 parts at most, whose loads are
// all under way while the factors are formed (16 requests, 64 heads on 8 cached
// ones over 3000 tokens 19.5 -> 18.7 us a call; with 78 parts it costs 1 us instead).
template <int D, bool SHORT>
__global__ void __launch_bounds__(64 * kWaves)
join_kernel(Kv4Attn a, Cut few, Parts few_parts, Cut many, Parts many_parts, int most) {
  constexpr int C = D / 64;  // channels of a lane
  __shared__ float factor[SHORT ? 1 : kMaxChunks];
  __shared__ float sums[kWaves][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int hd = (int)blockIdx.x % a.heads;
  const Query query = query_of(a, (int)blockIdx.x / a.heads, most);
  const int b = __builtin_amdgcn_readfirstlane(query.b), i = __builtin_amdgcn_readfirstlane(query.i);
  if (b < 0) return;
  const Span sp = span_of(a, b);
  if (i * a.group >= sp.rows) return;
  // a single request is of many rows however few it has
  const bool is_many = many.has(sp);
  const Cut &cut = is_many ? many : few;
  const Parts &parts = is_many ? many_parts : few_parts;
  const int row = i * a.group + hd % a.group;
  const int end = tile_end(a, sp, row - row % cut.tile_rows, cut.tile_rows);
  if (end <= cut.chunk) return;
  const int n = min((end + cut.chunk - 1) / cut.chunk, cut.columns);
  const int64_t at = part_of(a, cut, sp, b, hd / a.group, row, i, hd);
  constexpr int EARLY = SHORT ? kShortJoin / kWaves : 1;
  float4 first = make_float4(-INFINITY, 0.f, 0.f, 0.f);
  if (lane < n) first = parts.ml[at + lane];
  float early[EARLY][C] = {};
  if constexpr (SHORT) {
#pragma unroll
    for (int e = 0; e < EARLY; ++e)
      if (wave + kWaves * e < n)
#pragma unroll
        for (int x = 0; x < C; ++x) early[e][x] = parts.o[(at + wave + kWaves * e) * D + 64 * x + lane];
  }
  float m = first.x;
  if constexpr (!SHORT)
    for (int c = lane + 64; c < n; c += 64) m = fmaxf(m, parts.ml[at + c].x);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
  const float ref = m == -INFINITY ? 0.f : m;
  const float f0 = __builtin_amdgcn_exp2f(first.x - ref);
  float l = first.y * f0, le = first.z * f0;
  if constexpr (!SHORT) {
    if (wave == 0) factor[lane] = f0;
    for (int c = lane + 64; c < n; c += 64) {
      const float4 x = parts.ml[at + c];
      const float f = __builtin_amdgcn_exp2f(x.x - ref);
      if (wave == 0) factor[c] = f;
      l += x.y * f;
      le += x.z * f;
    }
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    l += __shfl_xor(l, s);
    le += __shfl_xor(le, s);
  }
  float o[C] = {};
  if constexpr (SHORT) {
#pragma unroll
    for (int e = 0; e < EARLY; ++e) {
      const float f = __shfl(f0, wave + kWaves * e);  // 0 behind the last part
#pragma unroll
      for (int x = 0; x < C; ++x) o[x] += f * early[e][x];
    }
  } else {
    __syncthreads();
#pragma unroll 4
    for (int c = wave; c < n; c += kWaves) {
      const float f = factor[c];
#pragma unroll
      for (int x = 0; x < C; ++x) o[x] += f * parts.o[(at + c) * D + 64 * x + lane];
    }
  }
#pragma unroll
  for (int x = 0; x < C; ++x) sums[wave][64 * x + lane] = o[x];
  __syncthreads();
  if (threadIdx.x < D) {
    const int c = threadIdx.x;
    const float v = ((sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c])) * inverse(l);
    a.out[(int64_t)(sp.q0 + i) * a.ost + (int64_t)hd * a.osh + c] = __builtin_bit_cast(uint16_t, (__bf16)v);
  }
  if (a.lse && threadIdx.x == 0) a.lse[(int64_t)(sp.q0 + i) * a.heads + hd] = lse_of(m, le);
}

// The same for few parts of many rows: D / 4 lanes take a query row and head, no
// lane waits for another, and the loads of eight parts are under way at once
// (64 requests of 4 queries, 16 heads on 2 over 2048 tokens: 20.6 -> 20.2 us a call).
template <int D>
__global__ void __launch_bounds__(256)
join_few_kernel(Kv4Attn a, Cut few, Parts few_parts, Cut many, Parts many_parts, int most) {
  constexpr int LANES = D / 4;
  int64_t id = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const int c4 = 4 * (threadIdx.x % LANES);
  const int hd = (int)(id % a.heads);
  const Query query = query_of(a, id / a.heads, most);
  const int b = query.b, i = query.i;
  if (b < 0) return;
  const Span sp = lane_span_of(a, b);  // a workgroup may hold rows of two requests
  if (i * a.group >= sp.rows) return;
  const bool is_many = many.has(sp);
  const Cut cut = is_many ? many : few;
  const Parts parts = is_many ? many_parts : few_parts;
  const int row = i * a.group + hd % a.group;
  const int end = tile_end(a, sp, row - row % cut.tile_rows, cut.tile_rows);
  if (end <= cut.chunk) return;
  const int n = min((end + cut.chunk - 1) / cut.chunk, cut.columns);
  const int64_t at = part_of(a, cut, sp, b, hd / a.group, row, i, hd);
  float m = -INFINITY, l = 0.f, le = 0.f;
  f32x4 o = {};
  for (int c0 = 0; c0 < n; c0 += 8) {  // eight parts' loads at once
    float4 x[8];
    f32x4 v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
      v[e] = f32x4{};
      if (c0 + e < n) {
        x[e] = parts.ml[at + c0 + e];
        v[e] = *reinterpret_cast<const f32x4 *>(parts.o + (at + c0 + e) * D + c4);
      }
    }
    float top = m;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e].x);
    const float ref = top == -INFINITY ? 0.f : top;
    const float al = __builtin_amdgcn_exp2f(m - ref);
    m = top;
    l *= al;
    le *= al;
    o *= al;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = __builtin_amdgcn_exp2f(x[e].x - ref);
      l += x[e].y * f;
      le += x[e].z * f;
      o += v[e] * f;
    }
  }
  const float inv = inverse(l);
  bf16x4 w;
#pragma unroll
  for (int x = 0; x < 4; ++x) w[x] = (__bf16)(o[x] * inv);
  *reinterpret_cast<bf16x4 *>(a.out + (int64_t)(sp.q0 + i) * a.ost + (int64_t)hd * a.osh + c4) = w;
  if (a.lse && c4 == 0) a.lse[(int64_t)(sp.q0 + i) * a.heads + hd] = lse_of(m, le);
}

template <int D, int NT>
hipError_t launch_rows(const Kv4Attn &a, const Cut &cut, const Parts &parts, hipStream_t s) {
  static_assert(kWaves == 4, "256 threads, as most_threads has them");
  const size_t lds = rows_lds(D, NT, kWaves);
  const int64_t grid = few_groups(a, cut);
  const auto f = cut.chunks > 1 ? &rows_kernel<D, NT, true> : &rows_kernel<D, NT, false>;
  const hipError_t e = allow_lds(reinterpret_cast<const void *>(f), lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(f, dim3((unsigned)grid), dim3(64 * kWaves), lds, s, a, cut, parts);
  return hipGetLastError();
}

Parts parts_at(const Kv4Attn &a, const Cut &cut, char *at) {
  return Parts{reinterpret_cast<float *>(at), reinterpret_cast<float4 *>(at + outputs_bytes(a, cut))};
}

hipError_t launch_join(const Kv4Attn &a, const Cut &few, const Parts &fp, const Cut &many, const Parts &mp, hipStream_t s) {
  const Joined join = joined(a, few, many);
  if (join.queries == 0) return hipSuccess;
  const int64_t n = join.queries * a.heads;
  const int most = join.most;
  const bool d128 = a.c.d == 128;
  if (joins_few(few, many, n)) {
    const dim3 grid((unsigned)up(n, 1024 / a.c.d));
    if (d128) hipLaunchKernelGGL(join_few_kernel<128>, grid, dim3(256), 0, s, a, few, fp, many, mp, most);
    else hipLaunchKernelGGL(join_few_kernel<64>, grid, dim3(256), 0, s, a, few, fp, many, mp, most);
  } else {
    const bool is_short = (many.tiles > 0 && many.columns > few.columns ? many.columns : few.columns) <= kShortJoin;
    const auto f = d128 ? (is_short ? &join_kernel<128, true> : &join_kernel<128, false>)
                        : (is_short ? &join_kernel<64, true> : &join_kernel<64, false>);
    hipLaunchKernelGGL(f, dim3((unsigned)n), dim3(64 * kWaves), 0, s, a, few, fp, many, mp, most);
  }
  return hipGetLastError();
}

}  // namespace

int64_t kv4_attn_threads(const Kv4Attn &a) { return most_threads(a, cuts(a)); }

size_t kv4_attn_scratch_bytes(const Kv4Attn &a) {
  const auto [few, many] = cuts(a);
  return parts_bytes(a, few) + parts_bytes(a, many);
}

hipError_t launch_kv4_attn(const Kv4Attn &a, void *scratch, hipStream_t s) {
  const auto [few, many] = cuts(a);
  char *at = static_cast<char *>(scratch);
  const Parts fp = parts_at(a, few, at), mp = parts_at(a, many, at + parts_bytes(a, few));
  hipError_t e;
  const bool d128 = a.c.d == 128;
  if (many.tiles > 0)
    e = launch_kv4_tiles(a, few, fp, (int)few_groups(a, few), many, mp, s);
  else if (few.tile_rows == 16)
    e = d128 ? launch_rows<128, 1>(a, few, fp, s) : launch_rows<64, 1>(a, few, fp, s);
  else if (few.tile_rows == 32)
    e = d128 ? launch_rows<128, 2>(a, few, fp, s) : launch_rows<64, 2>(a, few, fp, s);
  else
    e = launch_rows<64, 4>(a, few, fp, s);
  if (e != hipSuccess) return e;
  return launch_join(a, few, fp, many, mp, s);
}

}  // namespace carnator
