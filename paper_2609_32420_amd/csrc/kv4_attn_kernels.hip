// Attention over cached keys and values in 4 bits: the kernel for requests of few
// rows alone (its work is in kv4_rows.h), the joining of parts of the key axis, and
// how a call is cut and launched.
#include "kv4_rows.h"

namespace carnator {
namespace {

template <int D, int NT, bool SPLIT>
__global__ void __launch_bounds__(64 * kWaves, NT == 1 ? 3 : 2)
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
  const int n = (end + cut.chunk - 1) / cut.chunk;
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
  const int n = (end + cut.chunk - 1) / cut.chunk;
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

// Workgroups for the requests of few rows.
int64_t few_groups(const Kv4Attn &a, const Cut &cut) { return (int64_t)a.batch * a.c.heads * cut.columns; }

template <int D, int NT>
hipError_t launch_rows(const Kv4Attn &a, const Cut &cut, const Parts &parts, hipStream_t s) {
  const size_t lds = rows_lds(D, NT, kWaves);
  const int64_t grid = few_groups(a, cut);
  const auto f = cut.chunks > 1 ? &rows_kernel<D, NT, true> : &rows_kernel<D, NT, false>;
  const hipError_t e = allow_lds(reinterpret_cast<const void *>(f), lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(f, dim3((unsigned)grid), dim3(64 * kWaves), lds, s, a, cut, parts);
  return hipGetLastError();
}

constexpr int kMaxParts = 64;  // parts of the requests of many rows
constexpr int kFewGroups = 8192;  // workgroups for the requests of few rows

int64_t up(int64_t x, int64_t y) { return (x + y - 1) / y; }

// Rows of a request, at most.
int64_t most_rows(const Kv4Attn &a) { return (int64_t)a.max_q * a.group; }

// Rows of a request up to which it is of few rows.  At d = 128 the outputs of 64
// rows do not fit the registers of two waves a SIMD (8 heads, 16,000 tokens, 48
// rows: 35 us with one wave a SIMD, 23 in the other kernel); at d = 64 they do, but
// not those of the three that the other kernel runs with.
int few_rows(const Kv4Attn &a) { return a.c.d == 64 && most_rows(a) <= 64 ? 64 : 32; }

// Cuts the key axis into parts of `chunk` tokens (a multiple of 128).
void set_chunk(Cut &cut, int64_t reach, int64_t chunk) {
  if (chunk * kMaxChunks < reach) chunk = up(reach, kMaxChunks * 128) * 128;
  cut.chunk = (int)chunk;
  cut.chunks = (int)up(reach, chunk);
}

// Keeps parts by request where that takes less than by query row.
void set_span(const Kv4Attn &a, Cut &cut, int64_t rows) {
  if (rows * a.batch * a.c.heads < (int64_t)a.n_rows * a.heads) cut.span = (int)rows;
}

// The requests of few rows.  One workgroup takes 0.7 us for its four waves' 128
// tokens, and three of them fit a CU, so the axis is cut for about 640
// workgroups; parts of 128 tokens to 1536 (longer ones balance ragged lengths
// worse and save nothing).  The second kernel costs 3 us: axes of 512 tokens
// stay whole, those of 1024 where there are more than 64 workgroups.  us at d =
// 128 with parts of 128 / 256 / 512 / 1024 / 2048 tokens / whole:
//   8 heads, 512 tokens: 8.5 / 9.3 / - / - / - / 7.3
//   8 heads, 1024: 8.7 / 9.2 / 10.6 / - / - / 9.9
//   8 heads, 4096: 9.0 / 9.5 / 10.8 / 13.4 / 18.8 / 26
//   32 heads, 4096: 13.6 / 11.3 / 11.4 / 13.5 / 18.8 / 26
//   128 heads, 1024: 15.9 / 12.5 / 12.8 / - / - / 10.1
//   192 heads, 4096: 39.5 / 30.2 / 26.8 / 25.4 / 27.8 / 30.3
//   128 heads, 16,384: 121 / 85 / 69 / 57 / 60 / 120
// The lengths are on the device: the table's width is what the axis may reach.
// Beside requests of many rows that keep the chip for at least twice as long
// as a whole axis takes (many_us, 0 without them, or where they are joined anyway)
// it stays whole too: a prompt of 2000 beside 60 single tokens, 32 / 8 heads, d = 128,
// 4000 cached 113 -> 103 us.
// A table may be far wider than what is cached: of more than 8192 workgroups, some
// thousand of which start to find nothing in a microsecond, the grid holds the
// first parts, and a workgroup goes on to later ones.  48 requests of 1000 tokens,
// 32 / 8 heads, d = 128, a table for 131,072: 43.6 us without, 18.6 so.
Cut few_cut(const Kv4Attn &a, double many_us) {
  const int64_t rows = most_rows(a) < few_rows(a) ? most_rows(a) : few_rows(a);
  const int nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const int64_t reach = (int64_t)a.width << a.c.shift;
  const int64_t base = (int64_t)a.batch * a.c.heads;
  Cut cut{0, few_rows(a), 16 * nt, 1, (int)reach, 1, 1, 0, 1, 0};
  set_span(a, cut, rows);
  if (reach <= 512 || (reach <= 1024 && base > 64) ||
      (reach <= 8192 && 2 * 0.7 / 128 * (double)reach <= many_us))
    return cut;
  const int64_t chunk = up(up(reach * base, 640), 128) * 128;
  set_chunk(cut, reach, chunk > 1536 ? 1536 : chunk);
  const int64_t columns = kFewGroups / base > 1 ? kFewGroups / base : 1;
  cut.columns = (int)(cut.chunks < columns ? cut.chunks : columns);
  return cut;
}

// The requests of more rows (tiles is 0 where there can be none).  Parts of the
// key axis fill CUs that the tiles leave empty and even out the last round, and
// cost their outputs' way through memory.  At d = 128 a tile is 128 rows, two
// workgroups to a CU, or 256, one of eight waves that convert a stage once where
// two would do it twice: 12 heads of 4680 rows over 32,760 tokens 940 -> 840 us,
// 40 of 1000 over 16,000 347 -> 319, but 12 requests of 24 heads, 798 rows and
// 1427 tokens (a last tile nearly empty, start and end of a workgroup beside
// nothing) 195 -> 241 and 8 of 400 over 2000 24.5 -> 28.1.  Taken are the tile
// and the number of parts with the least time by this.  A token of a tile takes
// 20, 27 ns with one or two workgroups on the CU (d = 64: 14.6, 19, 28.6 with up to
// three), 24.6 and 4 us at the start with 256 rows.  Past two rounds half a one
// is added, since workgroups do not end together.  A part of a tile adds 0.03 us
// (0.015) to the joining, which begins at 6 us.  Over 70 calls drawn over the
// whole range the choice is within 1 % of the better tile's time (geometric
// mean; 15 % at worst).  Per call at d = 128, whole / in parts of 512 / 2048 / 4096
// tokens, 128 rows:
//   8 tiles, 2000 tokens: 50 / 25 / - / - us (17 in parts of 128)
//   60 tiles, 16,000: 317 / 109 / 86 / 103
//   192 tiles, 16,000: 319 / 325 / 238 / 240
//   444 tiles, 32,000: 863 / 1416 / 984 / 931
// A ragged batch has tiles of all lengths, the longest first: it takes as long as
// the longest (the requests of most rows see two thirds of the table, say) or as
// the work, three tenths of the table for each, on all slots (parts cost 1.3 times
// as much there); over 40 such calls drawn over the whole range that is within 4 %
// of the best cut (geometric mean; 23 % at worst).  Tiles of 256 rows leave the
// requests of few rows in the same grid two thirds of the waves, so they are for
// batches of mostly long requests.  5 prompts, 9622 queries, 16 / 4 heads, d = 128:
// 174 us with 256 rows, 196 with 128; one of 4096 beside 30 of a token and 8000 cached
// 149 in three parts of 256 rows, 106 whole with 128.
// Rows: d = 64; d = 128, 128 and 256 rows.  Columns: one, two, three workgroups on the CU.
constexpr double kTokenUs[3][3] = {{0.0146, 0.019, 0.0286}, {0.020, 0.027, 0.027}, {0.0246, 0.0246, 0.0246}};
Cut many_cut(const Kv4Attn &a, double *whole_us) {
  *whole_us = 0;
  const int64_t reach = (int64_t)a.width << a.c.shift;
  Cut cut{few_rows(a), 0x7FFFFFFF, 128, 0, (int)reach, 1, 0, 0, 0, 0};
  if (most_rows(a) <= few_rows(a)) return cut;
  set_span(a, cut, most_rows(a));
  if (a.batch == 1) cut.over = 0;  // a single request is left to this kernel however few rows it has
  const bool d128 = a.c.d == 128;
  const bool ragged = (int64_t)a.max_q * a.batch > a.n_rows;
  const int64_t long_ones = a.n_rows / a.max_q;
  const bool large = d128 && (!ragged || a.batch <= 4 * long_ones);
  double best = 1e300;
  for (int rows = 128; rows <= (large ? 256 : 128); rows *= 2) {
    const int64_t tiles = up(most_rows(a), rows);
    // tiles that hold rows, about: all of them where every request has max_q
    // queries; else the requests' sum is n_rows, and the last tiles half empty of
    // twice as many requests as could be that long
    const int64_t halves = a.batch / 2 < long_ones ? a.batch / 2 : long_ones;
    const int64_t all = tiles * a.batch, held = up((int64_t)a.n_rows * a.group, rows) + halves;
    const int64_t base = (!ragged || all < held ? all : held) * a.c.heads;
    const int fit = rows == 256 ? 1 : d128 ? 2 : 3;  // workgroups on a CU
    const double *token = kTokenUs[rows == 256 ? 2 : d128];
    const double start = rows != 256 ? 0 : ragged ? 8 : 4, part = (d128 ? 0.03 : 0.015) * (ragged ? 1.3 : 1);
    for (int64_t n = 1; n <= kMaxParts && (n == 1 || reach >= n * 128); ++n) {
      const int64_t chunk = n == 1 ? reach : up(up(reach, n), 128) * 128;
      const int64_t groups = base * n, round = 256 * fit;
      const int64_t on_cu = up(groups, 256) < fit ? up(groups, 256) : fit;
      const double rounds = groups <= 2 * round ? (double)up(groups, round) : (double)groups / round + 0.5;
      const double work = ragged ? (double)base * 0.3 * (double)reach * token[fit - 1] / (double)round : 0;
      const double seen = 0.65 * (double)reach < (double)chunk ? 0.65 * (double)reach : (double)chunk;
      const double longest = 0.5 * (token[0] + token[fit - 1]) * seen + start;
      const double us = (!ragged ? rounds * (token[on_cu - 1] * (double)chunk + start) : longest > work ? longest : work) +
                        (n > 1 ? 6 + part * (double)groups : 0);
      if (us < best) {
        best = us;
        cut.tile_rows = rows;
        cut.tiles = (int)tiles;
        cut.chunk = (int)chunk;
        cut.chunks = (int)up(reach, chunk);
      }
    }
  }
  if (cut.chunks == 1 && cut.over > 0) *whole_us = best;
  cut.turns = cut.tiles;
  if (a.causal && a.batch > 1 && reach * a.group <= 4 * most_rows(a))
    cut.turns += (int)(reach * a.group / cut.tile_rows);
  // Ragged batches: the turns hold many tiles that there are not, each a workgroup
  // that starts to find nothing; the rows leave at most `most` (a part of a tile a
  // request, of those with more than `over` rows).  Finding a tile by its number
  // takes a workgroup half a microsecond.  A prompt of 4096 beside 30 single tokens,
  // 16 / 4 heads, 8000 cached: d = 64 117 -> 94 us, d = 128 (with the choices above)
  // 424 -> 103.
  const int64_t rows = (int64_t)a.n_rows * a.group, some = rows / (cut.over + 1);
  const int64_t most = rows / cut.tile_rows + (some < a.batch ? some : a.batch);
  if (a.batch > 1 && a.batch <= kFindBatch && 2 * (int64_t)cut.turns * a.batch > 3 * most) cut.items = (int)(most ? most : 1);
  return cut;
}

struct Cuts {
  Cut few, many;
};
Cuts cuts(const Kv4Attn &a) {
  double whole_us;
  const Cut many = many_cut(a, &whole_us);
  return Cuts{few_cut(a, whole_us), many};
}

// Scratch of a cut: the parts' outputs, then their references and sums.
size_t part_count(const Kv4Attn &a, const Cut &cut) {
  return (cut.span ? (size_t)cut.span * a.batch * a.c.heads : (size_t)a.n_rows * a.heads) * cut.chunks;
}
size_t outputs_bytes(const Kv4Attn &a, const Cut &cut) { return align_up(part_count(a, cut) * a.c.d * 4); }
size_t parts_bytes(const Kv4Attn &a, const Cut &cut) {
  if (cut.chunks == 1 || cut.tiles == 0) return 0;
  return outputs_bytes(a, cut) + align_up(part_count(a, cut) * 16);
}
// Queries that a second kernel looks at, and of them `most` to a request (0: by row).
struct Joined {
  int64_t queries;
  int most;
};
Joined joined(const Kv4Attn &a, const Cut &few, const Cut &many) {
  int most = a.max_q;
  if (!(many.tiles > 0 && many.chunks > 1)) {
    if (many.over == 0 || few.chunks == 1) return Joined{0, 0};
    if (few.upto < most_rows(a)) most = few.upto / a.group;
  }
  const int64_t all = (int64_t)most * a.batch;
  return 2 * all > 3 * (int64_t)a.n_rows ? Joined{a.n_rows, 0} : Joined{all, most};
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
  const int parts = many.tiles > 0 && many.chunks > 1 ? many.chunks : few.chunks;
  if (parts <= 16 && n >= 2048) {
    const dim3 grid((unsigned)up(n, 1024 / a.c.d));
    if (d128) hipLaunchKernelGGL(join_few_kernel<128>, grid, dim3(256), 0, s, a, few, fp, many, mp, most);
    else hipLaunchKernelGGL(join_few_kernel<64>, grid, dim3(256), 0, s, a, few, fp, many, mp, most);
  } else {
    const bool is_short = (many.tiles > 0 && many.chunks > few.chunks ? many.chunks : few.chunks) <= kShortJoin;
    const auto f = d128 ? (is_short ? &join_kernel<128, true> : &join_kernel<128, false>)
                        : (is_short ? &join_kernel<64, true> : &join_kernel<64, false>);
    hipLaunchKernelGGL(f, dim3((unsigned)n), dim3(64 * kWaves), 0, s, a, few, fp, many, mp, most);
  }
  return hipGetLastError();
}

}  // namespace

int64_t kv4_attn_workgroups(const Kv4Attn &a) {
  const auto [few, many] = cuts(a);
  const int64_t main = few_groups(a, few) + tile_groups(a, many);
  const int64_t join = joined(a, few, many).queries * a.heads;
  return main > join ? main : join;
}

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
    e = launch_kv4_tiles(a, few, fp, many.over == 0 ? 0 : (int)few_groups(a, few), many, mp, s);
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
