// Attention over cached keys and values in 4 bits for many query rows of a
// request (prompts, frames): the products bind, not the cache's bytes.
//
// A workgroup takes 32 WAVES rows of one request and cached head (a row is a
// query token and one of the query heads that share the cached head), 32 to a
// wave, and walks the request's pages in stages of 64 tokens.  All of its
// threads convert a stage to bf16 once, into LDS: K by token, V by channel, so
// that both are read back as MFMA operands with 16-byte reads.  S^T = K Q^T and
// O^T += V^T P^T run on bf16 MFMA 32x32x16 with fp32 accumulation: every score
// of a query is in one lane pair, and with bits 2 and 3 of a key's row swapped
// the score accumulators are the B operand of the second product.  The softmax
// keeps a running maximum and sum per query (fp32, exp2 domain).
//
// A wave issues vector instructions while its own MFMAs run, so iteration j is
// one stream of MFMA slots with a share of the other work behind each: first O
// += V(j-1)^T P(j-1)^T beside the maximum and half of the exponentials of S(j),
// then S(j+1) beside the other half and beside the conversion of K(j+2) and
// V(j), whose bytes were loaded during the iteration before.
//
// What bounds it is the issue of its instructions: beside an MFMA of 32 cycles a
// wave issues 6.0 vector ones (d = 128; 12.8 at d = 64), and MFMAs are under way
// 53 % (37) of the time, vector instructions 53 % (74), LDS 36 % (33).  12 heads, d =
// 128, 4680 queries over 32,760 tokens (942 GFLOP): 840 to 930 us with eight waves
// on a stage, 940 to 980 with four (twice the conversions).  At d = 64 the softmax
// is twice as much beside an MFMA, so three workgroups on a CU hide more of it
// than two: 1319 -> 1248 us for 8 requests of 16 heads (4 cached) over 8192 tokens,
// 4096 queries each.
#include "kv4_rows.h"

#include <math.h>

#include <type_traits>

namespace carnator {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kKeys = 64;  // tokens of a stage

// Waits for this wave's LDS accesses (not for its loads from memory), then
// meets the other waves.
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// MFMA row -> token inside 32: swap bits 2 and 3.
__device__ inline int perm32(int rr) { return (rr & ~12) | ((rr & 4) << 1) | ((rr & 8) >> 1); }

// The values of x in the two lanes that hold a query, in the same order in both.
__device__ inline float2 halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline void anchor(float x) { asm volatile("" ::"v"(x)); }

// 16-byte chunk c of row r sits at c ^ swizzle(r): the lanes that are served
// together read consecutive rows at one chunk.
template <int CHUNKS>
__device__ inline int swizzle(int r) {
  if constexpr (CHUNKS == 16) return r & 15;
  else return (r >> 1) & 7;
}

template <int D, int WAVES>
struct TileCfg {
  static constexpr int THREADS = 64 * WAVES;
  static constexpr int UNITS = 4 * D / THREADS;  // 8-byte units of K, and of V, that a thread converts
  static constexpr int RB = 2 * D;               // bytes of a K row
  static constexpr int TB = kKeys * RB;          // a converted tile of K or V
  static constexpr int POISON = 4 * TB;          // K slots 0, 1; V slots 0, 1; then token masks
  static constexpr int NT = 2;                   // tiles of rows_body in the same workgroups
  static constexpr int OWN = POISON + 2 * (D / 32) * 8;
  static constexpr int FEW = rows_lds(D, NT, WAVES);
  static constexpr int LDS = OWN > FEW ? OWN : FEW;
  static_assert(UNITS >= 1, "a thread converts at least a unit");
};

// Sum over a wave's lanes, in every lane.
__device__ inline int wave_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return __builtin_amdgcn_readlane(x, 63);
}

// Turn and request of tile `item` of the requests from base on (64 K of them) in the
// order of the turns, where a request has `late` empty ones before its tiles;
// request -1, and item counted down, where it lies behind their last.  A lane
// holds the requests base + lane + 64 k, k < K.
template <int ROWS, int K>
__device__ inline int2 find_tile(const Kv4Attn &a, const Cut &cut, int base, int &item) {
  const int lane = threadIdx.x & 63;
  int n[K], late[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    n[k] = late[k] = 0;
    const int b = base + lane + 64 * k;
    if (base + 64 * k < a.batch && b < a.batch) {
      const Span sp = lane_span_of(a, b);
      if (cut.has(sp)) n[k] = (sp.rows + ROWS - 1) / ROWS;
      late[k] = late_of<ROWS>(a, cut, sp);
    }
  }
  const auto before = [&](int t) {  // tiles of the turns before t
    int s = 0;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (base + 64 * k < a.batch) s += min(max(t - late[k], 0), n[k]);
    return wave_sum(s);
  };
  int t = 0, end = cut.turns, first = 0;
  const int all = before(end);
  if (item >= all) {
    item -= all;
    return make_int2(0, -1);
  }
  while (end - t > 1) {  // before(t) <= item < before(end)
    const int mid = (t + end) >> 1, s = before(mid);
    if (s <= item) {
      t = mid;
      first = s;
    } else {
      end = mid;
    }
  }
  int left = item - first, b = -1;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (base + 64 * k >= a.batch) break;
    const uint64_t in = __ballot(t >= late[k] && t - late[k] < n[k]);
    const int count = __builtin_popcountll(in);
    if (b < 0 && left < count) {
      const int rank = __builtin_amdgcn_mbcnt_hi((unsigned)(in >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)in, 0));
      b = base + 64 * k + __builtin_ctzll(__ballot((in >> lane & 1) && rank == left));
    }
    left -= count;
  }
  return make_int2(t, b);
}

template <int D, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, D == 64 ? 3 : 2)
tile_kernel(Kv4Attn a, Cut few, Parts few_parts, int few_first, Cut cut, Parts parts) {
  using C = TileCfg<D, WAVES>;
  constexpr int UN = C::UNITS;
  constexpr int ROWS = 32 * WAVES;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int group = a.c.heads * cut.chunks * (cut.items ? 1 : a.batch), groups = cut.items ? cut.items : cut.turns;
  const int place = (int)blockIdx.x - few_first;
  int turn_of = place / group;
  if (place < 0 || turn_of >= groups) {  // requests of few rows (a launch of their own would cost more than they)
    const int id = place < 0 ? (int)blockIdx.x : place - groups * group;
    rows_body<D, C::NT, true, WAVES>(a, few, few_parts, id, reinterpret_cast<float *>(lds));
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  // The tiles that see most first.  Workgroups go to the eight XCDs in turn, so
  // the heads, requests and parts of a tile are rotated from tile to tile where
  // their number is even: otherwise the long ones of a ragged batch, or the early
  // parts of a causal one, would all meet on a few XCDs.
  int id = place - turn_of * group;
  if (group % 2 == 0) id = (id + turn_of) % group;
  const int h = id % a.c.heads;
  id /= a.c.heads;
  int b, chunk = id;
  if (cut.items) {
    int2 found;
    if (a.batch <= 64) {
      found = find_tile<ROWS, 1>(a, cut, 0, turn_of);
    } else {
      found = find_tile<ROWS, kFindBatch / 64>(a, cut, 0, turn_of);
      for (int base = kFindBatch; found.y < 0 && base < a.batch; base += kFindBatch)
        found = find_tile<ROWS, kFindBatch / 64>(a, cut, base, turn_of);
    }
    turn_of = found.x;
    b = found.y;
    if (b < 0) return;
  } else {
    b = id % a.batch;
    chunk = id / a.batch;
  }
  const Span sp = span_of(a, b);
  const int late = late_of<ROWS>(a, cut, sp);
  const int tile = (sp.rows + ROWS - 1) / ROWS - 1 - (turn_of - late);
  const int row0 = tile * ROWS;
  if (!cut.has(sp) || turn_of < late || tile < 0) return;
  const int end = tile_end(a, sp, row0, ROWS);
  const int k_first = chunk * cut.chunk;
  if (k_first >= end && chunk > 0) return;
  const bool whole = end <= cut.chunk;
  const int k_end = min(end, k_first + cut.chunk);
  const int seen_by_all = sp.limit(a, row0 / a.group);

  // ---- Q (B operand): query l32, channels 16 t + 8 hh .. + 8
  const int row = row0 + 32 * wave + l32;
  const int qi = row / a.group, hd = h * a.group + row - qi * a.group;
  const bool live = row < sp.rows;
  const int limit = min(live ? sp.limit(a, qi) : sp.kv, k_end);
  // tokens that every row of the wave sees
  const int wave_all = min(row0 + 32 * wave < sp.rows ? sp.limit(a, (row0 + 32 * wave) / a.group) : sp.kv, k_end);
  bf16x8 qf[D / 16];
  {
    const uint16_t *qp = a.q.data + (int64_t)(sp.q0 + qi) * a.q.st + (int64_t)hd * a.q.sh + 8 * hh;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      u32x4 w = {};
      if (live) w = *reinterpret_cast<const u32x4 *>(qp + 16 * t);
      qf[t] = __builtin_bit_cast(bf16x8, w);
    }
  }
  f32x16 o[D / 32];
#pragma unroll
  for (int mo = 0; mo < D / 32; ++mo)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[mo][r] = 0.f;
  float mrun = -INFINITY, lsum = 0.f, alpha = 1.f;

  // ---- the stages: positions of those that have a page
  const int block = 1 << a.c.shift;
  const int rec = kv4_head_bytes(D, block);
  const int codes = kv4_codes(D, block), scales = kv4_scales(D, block);
  int entry0 = k_first >> a.c.shift, entry = -1;
  auto look = [&]() {
    entry = -1;
    if (entry0 + lane < a.width) entry = a.table[(int64_t)b * a.width + entry0 + lane];
  };
  look();
  struct Stage {
    int k;     // first token; k_end and beyond: none
    int page;
  };
  auto next = [&](int k) __attribute__((always_inline)) {
    Stage s{k, 0};
    for (; s.k < k_end; s.k += kKeys) {
      int at = (s.k >> a.c.shift) - entry0;
      if (at >= 64) {
        entry0 += at;
        at = 0;
        look();
      }
      s.page = __builtin_amdgcn_readlane(entry, at);
      if ((unsigned)s.page < (unsigned)a.c.n_pages) break;
    }
    return s;
  };

  // ---- what a thread loads and converts: 8-byte units u = thread + i THREADS;
  // of K: 16 channels 16 (u % (D / 16)) of token u / (D / 16); of V: channel
  // pair u % (D / 2) of octet u / (D / 2)
  struct Raw {
    uint2 w[UN];
    uint32_t ks[UN];
    uint2 vs[UN];
  };
  // Unit i lies THREADS i units on: TOK i tokens of K, OCT i octets of V; in LDS
  // that leaves K's swizzle as it is and flips bit 2 of an octet's chunk.
  constexpr int TOK = C::THREADS / (D / 16), OCT = C::THREADS / (D / 2);
  static_assert(UN == 1 || (UN == 2 && TOK % 16 == 0 && OCT == 4), "offsets of a second unit");
  const int tok0 = threadIdx.x / (D / 16), part0 = threadIdx.x % (D / 16);
  const int oct0 = threadIdx.x / (D / 2), pair0 = threadIdx.x % (D / 2);
  const unsigned off = 8 * threadIdx.x;
  const unsigned ks_off = tok0 * (D / 32) + part0 / 2, vs_off = (oct0 * (D / 32) + pair0 / 16) * 8;
  const unsigned k_to = tok0 * C::RB + (((2 * part0) ^ swizzle<D / 8>(tok0)) << 4);
  const unsigned v_to = 2 * C::TB + 2 * pair0 * 128 + ((oct0 ^ swizzle<8>(2 * pair0)) << 4);
  auto load_k = [&](Raw &x, const Stage &s) __attribute__((always_inline)) {
    if (s.k >= k_end) return;
    const unsigned char *base = a.c.pages + ((int64_t)s.page * a.c.heads + h) * rec;
    const int tp = s.k & (block - 1);
    const unsigned char *kb = base + tp * (D / 2), *ks = base + codes + tp * (D / 32);
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      x.w[i] = *reinterpret_cast<const uint2 *>(kb + (off + i * 8 * C::THREADS));
      x.ks[i] = ks[ks_off + i * TOK * (D / 32)];
    }
  };
  auto load_v = [&](Raw &x, const Stage &s) __attribute__((always_inline)) {
    if (s.k >= k_end) {
#pragma unroll
      for (int i = 0; i < UN; ++i) x.w[i] = x.vs[i] = make_uint2(0, 0);
      return;
    }
    const unsigned char *base = a.c.pages + ((int64_t)s.page * a.c.heads + h) * rec;
    const int tp = s.k & (block - 1);
    const unsigned char *vb = base + codes + scales + tp * (D / 2), *vs = base + 2 * codes + scales + tp * (D / 32);
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      x.w[i] = *reinterpret_cast<const uint2 *>(vb + (off + i * 8 * C::THREADS));
      x.vs[i] = *reinterpret_cast<const uint2 *>(vs + (vs_off + i * OCT * (D / 32) * 8));
    }
  };
  // a K unit's half x: eight channels
  auto put_k = [&](const Raw &x, int i, int half, int slot) __attribute__((always_inline)) {
    const bf16x8 w = eight_of(half ? x.w[i].y : x.w[i].x, x.ks[i] << 23);
    *reinterpret_cast<bf16x8 *>(lds + (k_to ^ (half << 4)) + i * TOK * C::RB + slot * C::TB) = w;
  };
  // a V unit: eight tokens of two channels, told apart
  auto conv_v = [&](const Raw &x, int i, int half, uint32_t (&t)[8]) __attribute__((always_inline)) {
    const uint32_t w = half ? x.w[i].y : x.w[i].x, s = half ? x.vs[i].y : x.vs[i].x;
    t[4 * half + 0] = pair_of<0>(w, s << 23);
    t[4 * half + 1] = pair_of<1>(w, s << 15);
    t[4 * half + 2] = pair_of<2>(w, s << 7);
    t[4 * half + 3] = pair_of<3>(w, s >> 1);
  };
  auto put_v = [&](const uint32_t (&t)[8], int i, int ch, int slot) __attribute__((always_inline)) {
    const uint32_t sel = ch ? 0x07060302u : 0x05040100u;
    const u32x4 w = {__builtin_amdgcn_perm(t[1], t[0], sel), __builtin_amdgcn_perm(t[3], t[2], sel),
                     __builtin_amdgcn_perm(t[5], t[4], sel), __builtin_amdgcn_perm(t[7], t[6], sel)};
    *reinterpret_cast<u32x4 *>(lds + (v_to ^ (i << 6)) + ch * 128 + slot * C::TB) = w;
  };
  // Stage of which a row does not see all: tokens whose V is NaN, or behind the
  // last one, get the scale byte 0 (P is 0 there, which they would turn into
  // NaN); the ones that are NaN are noted by group of 32 channels, for the rows
  // that see them.
  auto clean_v = [&](Raw &x, int k, int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int oct = oct0 + i * OCT;
      uint32_t nan = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t &w = e < 4 ? x.vs[i].x : x.vs[i].y;
        const uint32_t byte = 0xFFu << (8 * (e & 3));
        const bool in = k + 8 * oct + e < sp.kv, is_nan = (w & byte) == byte;
        if (is_nan && in) nan |= 1u << e;
        if (is_nan || !in) w &= ~byte;
      }
      if (pair0 % 16 == 0) lds[C::POISON + (slot * (D / 32) + pair0 / 16) * 8 + oct] = (unsigned char)nan;
    }
  };
  auto poison = [&](int k, int slot) __attribute__((always_inline)) {
    const int see = limit - k;
    const uint64_t vis = see >= 64 ? ~0ull : see <= 0 ? 0ull : (1ull << see) - 1;
#pragma unroll
    for (int mo = 0; mo < D / 32; ++mo) {
      const uint64_t m = *reinterpret_cast<const uint64_t *>(lds + C::POISON + (slot * (D / 32) + mo) * 8);
      if (m & vis)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[mo][r] = NAN;
    }
  };

  // ---- operand reads: K row perm32(l32), chunk 2 t + hh; V^T row 32 mo + l32, chunk 2 tp + hh
  int kread[D / 16], vread[4];
  {
    const int kr = perm32(l32);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) kread[t] = kr * C::RB + (((2 * t + hh) ^ swizzle<D / 8>(kr)) << 4);
#pragma unroll
    for (int tp = 0; tp < 4; ++tp) vread[tp] = 2 * C::TB + l32 * 128 + (((2 * tp + hh) ^ swizzle<8>(l32)) << 4);
  }
  auto mask = [&](f32x16 (&s)[2], int mt, int k0) __attribute__((always_inline)) {
    const int see = limit - k0 - 8 * hh;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (32 * mt + 16 * (r >> 3) + 4 * ((r >> 2) & 1) + (r & 3) >= see) s[mt][r] = -INFINITY;
  };

  struct Soft {
    float m0, m1, sub, s0, s1;
  };
  auto sm_max = [&](Soft &st, const f32x16 (&s)[2], int x) __attribute__((always_inline)) {
    st.m0 = __builtin_fmaxf(__builtin_fmaxf(st.m0, s[x >> 4][x & 15]), s[x >> 4][(x + 1) & 15]);
    st.m1 = __builtin_fmaxf(__builtin_fmaxf(st.m1, s[x >> 4][(x + 2) & 15]), s[x >> 4][(x + 3) & 15]);
    anchor(st.m0);
    anchor(st.m1);
  };
  auto sm_alpha = [&](Soft &st) __attribute__((always_inline)) {
    const float2 hv = halves(__builtin_fmaxf(st.m0, st.m1));
    const float top = __builtin_fmaxf(hv.x, hv.y) * a.c2;
    const float mnew = top > mrun + kSlack ? top : mrun;
    const float al = __builtin_amdgcn_exp2f(mnew == -INFINITY ? 0.f : mrun - mnew);
    alpha *= al;
    lsum *= al;
    mrun = mnew;
    st.sub = mnew == -INFINITY ? 0.f : mnew;
    anchor(st.sub);
    anchor(lsum);
  };
  auto sm_exp = [&](Soft &st, const f32x16 (&s)[2], u32x4 (&p)[4], int x) __attribute__((always_inline)) {
    const float v0 = __builtin_amdgcn_exp2f(fmaf(s[x >> 4][x & 15], a.c2, -st.sub));
    const float v1 = __builtin_amdgcn_exp2f(fmaf(s[x >> 4][(x + 1) & 15], a.c2, -st.sub));
    const bf16x2 pp = {(__bf16)v0, (__bf16)v1};
    // P is rounded as in rows_part; the sum is that of the unrounded P, for the
    // outputs too.  With one of the rounded P beside it for these (a convex
    // combination again) 21 frames at d = 128 took 942 us instead of 902, 8 requests
    // of 4096 queries over 8192 tokens at d = 64 1345 instead of 1265.
    p[x >> 3][(x & 7) >> 1] = __builtin_bit_cast(uint32_t, pp);
    st.s0 += v0;
    st.s1 += v1;
    anchor(__builtin_bit_cast(float, pp));
    anchor(st.s0);
    anchor(st.s1);
  };
  auto sm_done = [&](Soft &st) __attribute__((always_inline)) {
    lsum += st.s0 + st.s1;
    st.s0 = st.s1 = 0.f;
    anchor(lsum);
  };
  auto rescale = [&]() __attribute__((always_inline)) {
    if (__ballot(alpha != 1.f)) {
#pragma unroll
      for (int mo = 0; mo < D / 32; ++mo)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[mo][r] *= alpha;
      alpha = 1.f;
    }
  };

  constexpr int PF = 4;               // operand reads run this many slots ahead
  constexpr int NPV = 4 * (D / 32);   // MFMAs of a P.V
  constexpr int NQK = 2 * (D / 16);   // MFMAs of a Q.K

  // S, P and the walk.  P(j) takes the place of P(j-1): its first half is formed
  // when the products of the other's are done.
  f32x16 s[2];
  u32x4 p[4];
  Soft st{-INFINITY, -INFINITY, 0.f, 0.f, 0.f};
  auto iterate = [&](auto odd, const Stage &sj, const Stage &s1, Raw &kraw, Raw &vraw, int k_prev) __attribute__((always_inline)) {
    constexpr int VS = decltype(odd)::value ? 0 : 1, KS = VS;  // slots of V(j-1) and K(j+1)
    constexpr int VW = 1 - VS, KW = 1 - KS;                   // of V(j) and K(j+2)
    st.m0 = st.m1 = -INFINITY;
    if (sj.k + kKeys > seen_by_all) clean_v(vraw, sj.k, VW);
    {
      bf16x8 vf[NPV];
      auto vrd = [&](int i) __attribute__((always_inline)) {
        vf[i] = *reinterpret_cast<const bf16x8 *>(lds + vread[i / (D / 32)] + VS * C::TB + (i % (D / 32)) * 32 * 128);
      };
      constexpr int NC = 8 + 1 + 8;  // maxima, alpha, exponentials of the first tile
      static_assert(9 * NPV / 17 >= NPV / 2, "P is formed where it has been used");
#pragma unroll
      for (int i = 0; i < PF; ++i) vrd(i);
#pragma unroll
      for (int sl = 0; sl < NPV; ++sl) {
        if (sl + PF < NPV) vrd(sl + PF);
        const int tp = sl / (D / 32), mo = sl % (D / 32);
        o[mo] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[sl], __builtin_bit_cast(bf16x8, p[tp]), o[mo], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if (c * NPV / NC != sl) continue;
          if (c < 8) sm_max(st, s, 4 * c);
          else if (c < 9) sm_alpha(st);
          else sm_exp(st, s, p, 2 * (c - 9));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (k_prev + kKeys > seen_by_all) poison(k_prev, VS);
    }
    {
      bf16x8 kf[NQK];
      uint32_t tv[UN][8];
      auto krd = [&](int i) __attribute__((always_inline)) {
        kf[i] = *reinterpret_cast<const bf16x8 *>(lds + kread[i % (D / 16)] + KS * C::TB + (i / (D / 16)) * 32 * C::RB);
      };
#pragma unroll
      for (int i = 0; i < PF; ++i) krd(i);
      constexpr int HALF = NQK / 2;
      constexpr int NE = 8 + 1;      // exponentials of the second tile, sums
      constexpr int ND = 6 * UN;     // conversions
#pragma unroll
      for (int sl = 0; sl < NQK; ++sl) {
        if (sl + PF < NQK) krd(sl + PF);
        const int mt = sl / (D / 16), t = sl % (D / 16);
        if (t == 0) s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[sl], qf[t], f32x16{}, 0, 0, 0);
        else s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[sl], qf[t], s[mt], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < NE; ++c) {
          if (c * HALF / NE != sl) continue;
          if (c < 8) sm_exp(st, s, p, 16 + 2 * c);
          else sm_done(st);
        }
#pragma unroll
        for (int c = 0; c < ND; ++c) {
          if (HALF + c * HALF / ND != sl) continue;
          const int i = c / 6, w = c % 6;
          if (w < 2) put_k(kraw, i, w, KW);
          else if (w < 4) conv_v(vraw, i, w - 2, tv[i]);
          else put_v(tv[i], i, w - 4, VW);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (s1.k + kKeys > wave_all) {
        mask(s, 0, s1.k);
        mask(s, 1, s1.k);
      }
    }
  };

  Stage s0 = next(k_first);
  if (s0.k < k_end) {
    Stage s1 = next(s0.k + kKeys), s2 = next(s1.k + kKeys);
    Raw kr{}, vr{};
    auto put_all = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        put_k(kr, i, 0, slot);
        put_k(kr, i, 1, slot);
      }
    };
    load_k(kr, s0);
    put_all(0);
    load_k(kr, s1);
    put_all(1);
    load_k(kr, s2);
    load_v(vr, s0);
    // stage -1: nothing, in the slot of odd stages
#pragma unroll
    for (int i = 0; i < C::TB / 16 / C::THREADS; ++i)
      *reinterpret_cast<u32x4 *>(lds + 3 * C::TB + (threadIdx.x + i * C::THREADS) * 16) = u32x4{};
#pragma unroll
    for (int t = 0; t < 4; ++t) p[t] = u32x4{};
    lds_barrier();
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int t = 0; t < D / 16; ++t) {
        const bf16x8 k = *reinterpret_cast<const bf16x8 *>(lds + kread[t] + mt * 32 * C::RB);
        s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[t], t ? s[mt] : f32x16{}, 0, 0, 0);
      }
    if (s0.k + kKeys > wave_all) {
      mask(s, 0, s0.k);
      mask(s, 1, s0.k);
    }
    int k_prev = -kKeys;
    // iteration j: s0 = stage j, s1, s2 the next ones; kr, vr hold K(j+2), V(j).
    // Iterations come in pairs; one past the last stage sees no token.
    auto advance = [&]() __attribute__((always_inline)) {
      k_prev = s0.k;
      s0 = s1;
      s1 = s2;
      s2 = next(s2.k + kKeys);
      load_k(kr, s2);
      load_v(vr, s0);
    };
    auto turn = [&](auto odd) __attribute__((always_inline)) {
      lds_barrier();
      rescale();
      iterate(odd, s0, s1, kr, vr, k_prev);
      advance();
    };
    if (row0 + 32 * wave >= sp.rows) {
      // a wave without rows (the last tile of a request) converts its share
      int slot = 0;
      do {
        lds_barrier();
        if (s0.k + kKeys > seen_by_all) clean_v(vr, s0.k, slot);
#pragma unroll
        for (int i = 0; i < UN; ++i) {
          uint32_t tv[8];
          put_k(kr, i, 0, slot);
          put_k(kr, i, 1, slot);
          conv_v(vr, i, 0, tv);
          conv_v(vr, i, 1, tv);
          put_v(tv, i, 0, slot);
          put_v(tv, i, 1, slot);
        }
        advance();
        slot ^= 1;
      } while (s0.k < k_end || slot == 1);
      lds_barrier();
      return;
    }
    do {
      turn(std::false_type{});
      turn(std::true_type{});
    } while (s0.k < k_end);
    // P.V of the last stage, an odd one
    lds_barrier();
    rescale();
#pragma unroll
    for (int tp = 0; tp < 4; ++tp)
#pragma unroll
      for (int mo = 0; mo < D / 32; ++mo) {
        const bf16x8 v = *reinterpret_cast<const bf16x8 *>(lds + vread[tp] + C::TB + mo * 32 * 128);
        o[mo] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, p[tp]), o[mo], 0, 0, 0);
      }
    if (k_prev + kKeys > seen_by_all) poison(k_prev, 1);
  }

  // ---- outputs: channels 32 mo + 8 g + 4 hh + i
  const float2 lh = halves(lsum);
  const float l = lh.x + lh.y;
  if (!live) return;
  if (!whole) {
    const int64_t at = part_of(a, cut, sp, b, h, row, qi, hd) + chunk;
#pragma unroll
    for (int mo = 0; mo < D / 32; ++mo)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(parts.o + at * D + 32 * mo + 8 * g + 4 * hh) =
            f32x4{o[mo][4 * g], o[mo][4 * g + 1], o[mo][4 * g + 2], o[mo][4 * g + 3]};
    if (hh == 0) parts.ml[at] = make_float4(mrun, l, l, 0.f);
    return;
  }
  const float inv = inverse(l);
  uint16_t *op = a.out + (int64_t)(sp.q0 + qi) * a.ost + (int64_t)hd * a.osh + 4 * hh;
#pragma unroll
  for (int mo = 0; mo < D / 32; ++mo)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (__bf16)(o[mo][4 * g + i] * inv);
      *reinterpret_cast<bf16x4 *>(op + 32 * mo + 8 * g) = w;
    }
  if (a.lse && hh == 0) a.lse[(int64_t)(sp.q0 + qi) * a.heads + hd] = lse_of(mrun, l);
}

template <int D, int WAVES>
hipError_t launch(const Kv4Attn &a, const Cut &few, const Parts &few_parts, int few_groups, const Cut &cut,
                  const Parts &parts, hipStream_t s) {
  using C = TileCfg<D, WAVES>;
  const hipError_t e = allow_lds(reinterpret_cast<const void *>(&tile_kernel<D, WAVES>), C::LDS);
  if (e != hipSuccess) return e;
  const int64_t grid = tile_groups(a, cut) + few_groups;
  // what is not cut begins first, what is cut fills the end
  const int few_first = few.chunks == 1 ? few_groups : 0;
  hipLaunchKernelGGL((tile_kernel<D, WAVES>), dim3((unsigned)grid), dim3(C::THREADS), C::LDS, s, a, few, few_parts,
                     few_first, cut, parts);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_tiles(const Kv4Attn &a, const Cut &few, const Parts &few_parts, int few_groups, const Cut &cut,
                            const Parts &parts, hipStream_t s) {
  if (a.c.d == 64) return launch<64, 4>(a, few, few_parts, few_groups, cut, parts, s);
  return cut.tile_rows == 256 ? launch<128, 8>(a, few, few_parts, few_groups, cut, parts, s)
                              : launch<128, 4>(a, few, few_parts, few_groups, cut, parts, s);
}

}  // namespace carnator
