// How a call of attention over 4-bit cached keys and values is cut into workgroups:
// host code on the call's sizes alone, since the lengths are on the device.
#pragma once

#include "kv4_attn.h"

namespace carnator {

constexpr int kMaxParts = 64;     // parts of the requests of many rows
constexpr int kFewGroups = 8192;  // workgroups for the requests of few rows
// Bytes for the parts of the requests of many rows: 1.5 million rows' at d = 128 (23
// rounds of workgroups), of whose parts the best number gains little.  us with any
// number / so / with a third of it: 24 heads, 12,270 queries, 100,000 tokens 14,400 /
// 14,400 / 15,450; 12 heads, 2 requests of 3615, 107,000 tokens 4970 / 4970 / 5380;
// 32 / 8 heads, 8 of 4096 over 5000 tokens, a table for 131,072, 1820 / 1670 / 1670.
constexpr int64_t kPartsBytes = (int64_t)3 << 28;

// Workgroups for the requests of few rows.
inline int64_t few_groups(const Kv4Attn &a, const Cut &cut) { return (int64_t)a.batch * a.c.heads * cut.columns; }

inline int64_t up(int64_t x, int64_t y) { return (x + y - 1) / y; }

// Rows of a request, at most.
inline int64_t most_rows(const Kv4Attn &a) { return (int64_t)a.max_q * a.group; }

// Rows of a request up to which it is of few rows.  At d = 128 the outputs of 64
// rows do not fit the registers of two waves a SIMD (8 heads, 16,000 tokens, 48
// rows: 35 us with one wave a SIMD, 23 in the other kernel); at d = 64 they do, but
// not those of the three that the other kernel runs with.
inline int few_rows(const Kv4Attn &a) { return a.c.d == 64 && most_rows(a) <= 64 ? 64 : 32; }

// Cuts the key axis into parts of `chunk` tokens (a multiple of 128).
inline void set_chunk(Cut &cut, int64_t reach, int64_t chunk) {
  if (chunk * kMaxChunks < reach) chunk = up(reach, kMaxChunks * 128) * 128;
  cut.chunk = (int)chunk;
  cut.chunks = (int)up(reach, chunk);
}

// Keeps parts by request where that takes less than by query row.
inline void set_span(const Kv4Attn &a, Cut &cut, int64_t rows) {
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
// first parts, and a workgroup goes on to later ones with its running sums, so that
// results number the workgroups; past 4096 requests and heads the axis is whole.
// 48 requests of 1000 tokens, 32 / 8 heads, d = 128, a table for 131,072: 43.6 us
// without, 18.6 so.  With a result for every part instead, 200 requests of 600
// tokens take 39.7 us (now 34.0) and 291 MB of scratch (17), 600 of up to 8000
// under a tight table 354 (296) and 61 MB (none).
inline Cut few_cut(const Kv4Attn &a, double many_us) {
  const int64_t rows = most_rows(a) < few_rows(a) ? most_rows(a) : few_rows(a);
  const int nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const int64_t reach = (int64_t)a.width << a.c.shift;
  const int64_t base = (int64_t)a.batch * a.c.heads;
  Cut cut{0, few_rows(a), 16 * nt, 1, (int)reach, 1, 1, 0, 1, 0};
  set_span(a, cut, rows);
  if (reach <= 512 || (reach <= 1024 && base > 64) ||
      (reach <= 8192 && 2 * 0.7 / 128 * (double)reach <= many_us))
    return cut;
  const int64_t columns = kFewGroups / base;
  if (columns < 2) return cut;
  const int64_t chunk = up(up(reach * base, 640), 128) * 128;
  set_chunk(cut, reach, chunk > 1536 ? 1536 : chunk);
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
inline Cut many_cut(const Kv4Attn &a, double *whole_us) {
  *whole_us = 0;
  const int64_t reach = (int64_t)a.width << a.c.shift;
  Cut cut{few_rows(a), 0x7FFFFFFF, 128, 0, (int)reach, 1, 0, 0, 1, 0};
  if (most_rows(a) <= few_rows(a)) return cut;
  set_span(a, cut, most_rows(a));
  if (a.batch == 1) cut.over = 0;  // a single request is left to this kernel however few rows it has
  const bool d128 = a.c.d == 128;
  const bool ragged = (int64_t)a.max_q * a.batch > a.n_rows;
  const int64_t long_ones = a.n_rows / a.max_q;
  const bool large = d128 && (!ragged || a.batch <= 4 * long_ones);
  const int64_t part_bytes = (cut.span ? (int64_t)cut.span * a.batch * a.c.heads : (int64_t)a.n_rows * a.heads) *
                             (4 * a.c.d + 16);
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
    for (int64_t n = 1; n <= kMaxParts && (n == 1 || (reach >= n * 128 && n * part_bytes <= kPartsBytes)); ++n) {
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
        cut.chunks = cut.columns = (int)up(reach, chunk);
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
  // takes a workgroup half a microsecond for each 1024 requests before it.  A prompt
  // of 4096 beside 30 single tokens, 16 / 4 heads, 8000 cached: d = 64 117 -> 94 us,
  // d = 128 (with the choices above) 424 -> 103; one of 8192 beside 1024, 32 / 8
  // heads, d = 64, a table for 16,384: 7461 -> 541.
  const int64_t rows = (int64_t)a.n_rows * a.group, some = rows / (cut.over + 1);
  const int64_t most = rows / cut.tile_rows + (some < a.batch ? some : a.batch);
  if (a.batch > 1 && 2 * (int64_t)cut.turns * a.batch > 3 * most) cut.items = (int)(most ? most : 1);
  return cut;
}

struct Cuts {
  Cut few, many;
};
inline Cuts cuts(const Kv4Attn &a) {
  double whole_us;
  const Cut many = many_cut(a, &whole_us);
  // with no request left to it, the cut of few rows has neither workgroups nor parts
  return Cuts{many.over == 0 ? Cut{0, 0, 16, 0, many.chunk, 1, 0, 0, 0, 0} : few_cut(a, whole_us), many};
}

// Scratch of a cut: the parts' outputs, then their references and sums.
inline size_t part_count(const Kv4Attn &a, const Cut &cut) {
  return (cut.span ? (size_t)cut.span * a.batch * a.c.heads : (size_t)a.n_rows * a.heads) * cut.columns;
}
inline size_t outputs_bytes(const Kv4Attn &a, const Cut &cut) { return align_up(part_count(a, cut) * a.c.d * 4); }
inline size_t parts_bytes(const Kv4Attn &a, const Cut &cut) {
  if (cut.columns <= 1 || cut.tiles == 0) return 0;
  return outputs_bytes(a, cut) + align_up(part_count(a, cut) * 16);
}
// Queries that a second kernel looks at, and of them `most` to a request (0: by row).
struct Joined {
  int64_t queries;
  int most;
};
inline Joined joined(const Kv4Attn &a, const Cut &few, const Cut &many) {
  int most = a.max_q;
  if (!(many.tiles > 0 && many.chunks > 1)) {
    if (many.over == 0 || few.chunks == 1) return Joined{0, 0};
    if (few.upto < most_rows(a)) most = few.upto / a.group;
  }
  const int64_t all = (int64_t)most * a.batch;
  return 2 * all > 3 * (int64_t)a.n_rows ? Joined{a.n_rows, 0} : Joined{all, most};
}
// Whether n rows and heads are joined by the kernel for few parts of many.
inline bool joins_few(const Cut &few, const Cut &many, int64_t n) {
  return (many.tiles > 0 && many.columns > 1 ? many.columns : few.columns) <= 16 && n >= 2048;
}

// Threads of a call's largest launch.
inline int64_t most_threads(const Kv4Attn &a, const Cuts &c) {
  const int64_t main = (few_groups(a, c.few) + tile_groups(a, c.many)) * (c.many.tile_rows == 256 ? 512 : 256);
  const int64_t n = joined(a, c.few, c.many).queries * a.heads;
  const int64_t join = (joins_few(c.few, c.many, n) ? up(n, 1024 / a.c.d) : n) * 256;
  return main > join ? main : join;
}

}  // namespace carnator
