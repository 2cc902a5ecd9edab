// Attention over cached keys and values in 4 bits (Sec. 3.3: tokens outside the
// active region keep their cached computation), for each request's queries over
// the pages that its table names.
//
// A workgroup takes one request, one cached head and up to 16 NT query rows (a
// row is a query token and one of the query heads that share the cached head,
// so the cache is read once for all of them).  Its four waves take 32 tokens in
// turn.  S = K Q^T and O^T += V^T P^T run on bf16 MFMA 16x16x32 with fp32
// accumulation, one pass with a running maximum and sum per query (fp32, exp2
// domain).  Nothing passes through LDS: a lane's 16 bytes of K are one token's
// 32 channels under one scale, which is its A operand once converted (the
// channels are dealt to the four products in the same order for Q), and a
// lane's bytes of V are the eight tokens of an octet for two channels, which
// are an A operand of V^T each once the two are told apart.  Rows of a K tile
// are permuted so that the scores of eight consecutive tokens end in one lane,
// as the B operand of the second product.
#include "kv4_attn.h"

namespace carnator {
namespace {

constexpr int kWaves = 4;
constexpr int kStep = 32;  // tokens of a wave's step

// What a wave reads of 32 tokens.
template <int D>
struct Raw {
  u32x4 k[2];        // 16 (8 at d = 64) bytes of a token
  uint32_t ks[2];    // their scale
  u32x4 v[D / 64];   // two channel pairs of an octet
  uint2 vs[D / 64];  // the octet's scales
};

template <int D, int NT, bool SPLIT>
__global__ void __launch_bounds__(64 * kWaves, NT == 1 ? 3 : 2)
rows_kernel(Kv4Attn a, Cut cut, Parts parts) {
  constexpr int TQ = D / 32;        // products of a key tile
  constexpr int CPL = D / 4;        // channels of a lane
  constexpr int NV = D / 64;        // 64-channel parts of V
  extern __shared__ float lds_o[];  // [2][NT * NV * 16][64] outputs, then [2][NT][3][64] references and sums
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, j = lane >> 4;
  int id = (int)blockIdx.x;
  const int h = id % a.c.heads;
  id /= a.c.heads;
  const int tile = id % cut.tiles;
  id /= cut.tiles;
  const int b = id % a.batch, chunk = SPLIT ? id / a.batch : 0;
  const Span sp = span_of(a, b);
  const int row0 = tile * 16 * NT;
  if (!cut.has(sp) || row0 >= sp.rows) return;
  const int end = tile_end(a, sp, row0, 16 * NT);  // tokens that a row of the tile sees
  const int k_first = SPLIT ? chunk * cut.chunk : 0;
  if (k_first >= end && chunk > 0) return;
  const bool whole = !SPLIT || end <= cut.chunk;  // nothing to join
  const int k_end = SPLIT ? min(end, k_first + cut.chunk) : end;
  const int seen_by_all = sp.limit(a, row0 / a.group);

  // ---- Q: query column r of each 16, channels CPL j + 8 t .. + 8
  bf16x8 qf[NT][TQ];
  int limit[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = row0 + 16 * n + r;
    const int i = row / a.group, hd = h * a.group + row - i * a.group;
    const bool live = row < sp.rows;
    limit[n] = live ? sp.limit(a, i) : sp.kv;
    const uint16_t *qp = a.q.data + (int64_t)(sp.q0 + i) * a.q.st + (int64_t)hd * a.q.sh + CPL * j;
#pragma unroll
    for (int t = 0; t < TQ; ++t) {
      u32x4 w = {};
      if (live) w = *reinterpret_cast<const u32x4 *>(qp + 8 * t);
      qf[n][t] = __builtin_bit_cast(bf16x8, w);
    }
  }

  f32x4 o[NT][NV][4];
  float mrun[NT], lrun[NT], lexact[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    mrun[n] = -INFINITY;
    lrun[n] = lexact[n] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int p = 0; p < 4; ++p) o[n][v][p] = f32x4{};
  }

  const int block = 1 << a.c.shift;
  const int rec = kv4_head_bytes(D, block);
  const int codes = kv4_codes(D, block), scales = kv4_scales(D, block);
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};

  // ---- the wave's steps: pages come from the table 64 entries at a time
  int entry0 = k_first >> a.c.shift;  // of lane 0
  int entry = -1;
  auto look = [&]() {
    entry = -1;
    if (entry0 + lane < a.width) entry = a.table[(int64_t)b * a.width + entry0 + lane];
  };
  look();
  int page = -1;
  // the first of the wave's steps from k0 on that has a page
  auto next = [&](int k0) {
    for (; k0 < k_end; k0 += kWaves * kStep) {
      int at = (k0 >> a.c.shift) - entry0;
      if (at >= 64) {
        entry0 += at;
        at = 0;
        look();
      }
      page = __builtin_amdgcn_readlane(entry, at);
      if ((unsigned)page < (unsigned)a.c.n_pages) break;
    }
    return k0;
  };
  // K: tile T, MFMA row r is token 8 (r >> 2) + 4 T + (r & 3); V: octet j,
  // channels 64 v + 4 r .. + 4
  // (unsigned offsets from a scalar address: no 64-bit vector additions)
  const unsigned k_tok = 8 * (r >> 2) + (r & 3);
  const unsigned k_off = k_tok * (D / 2) + CPL / 2 * j, ks_off = k_tok * (D / 32) + j * CPL / 32;
  const unsigned v_off = (j * (D / 2) + 2 * r) * 8, vs_off = (j * (D / 32) + (r >> 3)) * 8;
  auto load = [&](Raw<D> &x, int k0) {
    const unsigned char *base = a.c.pages + ((int64_t)page * a.c.heads + h) * rec;
    const int tp = k0 & (block - 1);
    const unsigned char *kb = base + tp * (D / 2), *ks = base + codes + tp * (D / 32);
    const unsigned char *vb = base + codes + scales + tp * (D / 2), *vs = base + 2 * codes + scales + tp * (D / 32);
#pragma unroll
    for (int T = 0; T < 2; ++T) {
      if constexpr (D == 128) {
        x.k[T] = *reinterpret_cast<const u32x4 *>(kb + (k_off + 4 * T * (D / 2)));
      } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(kb + (k_off + 4 * T * (D / 2)));
        x.k[T] = u32x4{w.x, w.y, 0, 0};
      }
      x.ks[T] = ks[ks_off + 4 * T * (D / 32)];
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      x.v[v] = *reinterpret_cast<const u32x4 *>(vb + (v_off + 256 * v));
      x.vs[v] = *reinterpret_cast<const uint2 *>(vs + (vs_off + 16 * v));
    }
  };
  auto step = [&](const Raw<D> &x, int k0) {
    bf16x8 kf[2][TQ];
#pragma unroll
    for (int T = 0; T < 2; ++T)
#pragma unroll
      for (int t = 0; t < TQ; ++t) kf[T][t] = eight_of(x.k[T][t], x.ks[T] << 23);
    uint2 vs[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) vs[v] = x.vs[v];
    const bool part = k0 + kStep > seen_by_all;  // a row does not see all of the tokens
    uint32_t poison[NV] = {};  // tokens whose V is NaN in this lane's output channels
    if (part) {
      // A token out of a row's sight has P = 0 there, which NaN (or what lies
      // behind the last token) would still turn into NaN: its scale becomes that
      // of byte 0.  Rows that see it get their NaN afterwards.
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        uint32_t nan = 0;  // of this lane's octet and group of 32 channels
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t &w = e < 4 ? vs[v].x : vs[v].y;
          const uint32_t byte = 0xFFu << (8 * (e & 3));
          const bool in = k0 + 8 * j + e < sp.kv, is_nan = (w & byte) == byte;
          if (is_nan && in) nan |= 1u << e;
          if (is_nan || !in) w &= ~byte;
        }
        // outputs 64 v + 16 j + ..: group 2 v + (j >> 1), read by lanes 8 (j >> 1) .. + 8 of each octet
        uint32_t p0 = 0, p1 = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          p0 |= (uint32_t)__builtin_amdgcn_readlane((int)nan, 16 * g) << (8 * g);
          p1 |= (uint32_t)__builtin_amdgcn_readlane((int)nan, 16 * g + 8) << (8 * g);
        }
        poison[v] = j < 2 ? p0 : p1;
      }
    }
    // ---- scores, softmax
    u32x4 p[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      f32x4 s[2];
#pragma unroll
      for (int T = 0; T < 2; ++T) {
        s[T] = f32x4{};
#pragma unroll
        for (int t = 0; t < TQ; ++t) s[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[T][t], qf[n][t], s[T], 0, 0, 0);
      }
      if (part) {
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (k0 + 8 * j + 4 * T + i >= limit[n]) s[T][i] = -INFINITY;
      }
      float mx = s[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i >> 2][i & 3]);
      mx *= a.c2;
      if (__ballot(mx > mrun[n] + kSlack)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mnew = mx > mrun[n] + kSlack ? mx : mrun[n];
        const float al = __builtin_amdgcn_exp2f(mnew == -INFINITY ? 0.f : mrun[n] - mnew);
        mrun[n] = mnew;
        lrun[n] *= al;
        lexact[n] *= al;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int q = 0; q < 4; ++q) o[n][v][q] *= al;
      }
      const float sub = mrun[n] == -INFINITY ? 0.f : mrun[n];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e >> 1][2 * (e & 1)], a.c2, -sub));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[e >> 1][2 * (e & 1) + 1], a.c2, -sub));
        const bf16x2 pp = {(__bf16)p0, (__bf16)p1};
        p[n][e] = __builtin_bit_cast(uint32_t, pp);
        // the outputs are divided by the sum of what is multiplied with V: a
        // convex combination of its rows; the LSE takes the unrounded sum
        lrun[n] = __builtin_amdgcn_fdot2_f32_bf16(pp, ones, lrun[n], false);
        lexact[n] += p0 + p1;
      }
    }
    // ---- O^T += V^T P^T
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int pr = 0; pr < 2; ++pr) {
        const uint32_t w0 = x.v[v][2 * pr], w1 = x.v[v][2 * pr + 1];  // tokens 0-3, 4-7 of a channel pair
        const uint32_t lo = vs[v].x, hi = vs[v].y;
        const uint32_t t0 = pair_of<0>(w0, lo << 23), t1 = pair_of<1>(w0, lo << 15), t2 = pair_of<2>(w0, lo << 7),
                       t3 = pair_of<3>(w0, lo >> 1), t4 = pair_of<0>(w1, hi << 23), t5 = pair_of<1>(w1, hi << 15),
                       t6 = pair_of<2>(w1, hi << 7), t7 = pair_of<3>(w1, hi >> 1);
#pragma unroll
        for (int ch = 0; ch < 2; ++ch) {
          const uint32_t sel = ch ? 0x07060302u : 0x05040100u;
          const u32x4 w = {__builtin_amdgcn_perm(t1, t0, sel), __builtin_amdgcn_perm(t3, t2, sel),
                           __builtin_amdgcn_perm(t5, t4, sel), __builtin_amdgcn_perm(t7, t6, sel)};
#pragma unroll
          for (int n = 0; n < NT; ++n)
            o[n][v][2 * pr + ch] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, p[n]), o[n][v][2 * pr + ch], 0, 0, 0);
        }
      }
    if (part) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int see = limit[n] - k0;
          const uint32_t vis = see >= 32 ? ~0u : see <= 0 ? 0u : (1u << see) - 1;
          if (poison[v] & vis)
#pragma unroll
            for (int q = 0; q < 4; ++q) o[n][v][q] = f32x4{NAN, NAN, NAN, NAN};
        }
      }
    }
  };
  // the loads of a step are under way during the one before
  Raw<D> even, odd;
  const int stride = kWaves * kStep;
  int k0 = next(k_first + wave * kStep);
  if (k0 < k_end) {
    load(even, k0);
    int k1 = next(k0 + stride);
    while (k1 < k_end) {
      load(odd, k1);
      step(even, k0);
      k0 = next(k1 + stride);
      if (k0 < k_end) load(even, k0);
      step(odd, k1);
      k1 = next(k0 + stride);
    }
    if (k0 < k_end) step(even, k0);
  }
  // ---- sums over the lanes of a query, then the waves' parts in a fixed order
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    lrun[n] += __shfl_xor(lrun[n], 16);
    lrun[n] += __shfl_xor(lrun[n], 32);
    lexact[n] += __shfl_xor(lexact[n], 16);
    lexact[n] += __shfl_xor(lexact[n], 32);
  }
  float *ml = lds_o + 2 * NT * NV * 16 * 64;
  auto put = [&](int slot) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      ml[((slot * NT + n) * 3 + 0) * 64 + lane] = mrun[n];
      ml[((slot * NT + n) * 3 + 1) * 64 + lane] = lrun[n];
      ml[((slot * NT + n) * 3 + 2) * 64 + lane] = lexact[n];
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            lds_o[((((slot * NT + n) * NV + v) * 4 + q) * 4 + i) * 64 + lane] = o[n][v][q][i];
    }
  };
  auto add = [&](int slot) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float m2 = ml[((slot * NT + n) * 3 + 0) * 64 + lane];
      const float m = fmaxf(mrun[n], m2);
      const float ref = m == -INFINITY ? 0.f : m;
      const float f1 = __builtin_amdgcn_exp2f(mrun[n] - ref), f2 = __builtin_amdgcn_exp2f(m2 - ref);
      mrun[n] = m;
      lrun[n] = lrun[n] * f1 + ml[((slot * NT + n) * 3 + 1) * 64 + lane] * f2;
      lexact[n] = lexact[n] * f1 + ml[((slot * NT + n) * 3 + 2) * 64 + lane] * f2;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            o[n][v][q][i] = o[n][v][q][i] * f1 + lds_o[((((slot * NT + n) * NV + v) * 4 + q) * 4 + i) * 64 + lane] * f2;
    }
  };
  if (wave >= 2) put(wave - 2);
  __syncthreads();
  if (wave < 2) add(wave);
  __syncthreads();
  if (wave == 1) put(0);
  __syncthreads();
  if (wave != 0) return;
  add(0);

  // ---- outputs: channels 64 v + 16 j + 4 i + q
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = row0 + 16 * n + r;
    if (row >= sp.rows) continue;
    const int i = row / a.group, hd = h * a.group + row - i * a.group;
    if (SPLIT && !whole) {
      const int64_t at = ((int64_t)(sp.q0 + i) * a.heads + hd) * cut.chunks + chunk;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          *reinterpret_cast<f32x4 *>(parts.o + at * D + 64 * v + 16 * j + 4 * x) =
              f32x4{o[n][v][0][x], o[n][v][1][x], o[n][v][2][x], o[n][v][3][x]};
      if (j == 0) parts.ml[at] = make_float4(mrun[n], lrun[n], lexact[n], 0.f);
      continue;
    }
    const float inv = inverse(lrun[n]);
    uint16_t *op = a.out + (int64_t)(sp.q0 + i) * a.ost + (int64_t)hd * a.osh + 16 * j;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bf16x8 w;
#pragma unroll
        for (int x = 0; x < 8; ++x) w[x] = (__bf16)(o[n][v][x & 3][2 * half + (x >> 2)] * inv);
        *reinterpret_cast<bf16x8 *>(op + 64 * v + 8 * half) = w;
      }
    if (a.lse && j == 0) a.lse[(int64_t)(sp.q0 + i) * a.heads + hd] = lse_of(mrun[n], lexact[n]);
  }
}

// Joins the parts of a query row and head, in their order: a wave sums every
// fourth part, 64 lanes over the channels.
template <int D>
__global__ void __launch_bounds__(64 * kWaves)
join_kernel(Kv4Attn a, Cut cut, Parts parts) {
  constexpr int C = D / 64;  // channels of a lane
  __shared__ float factor[kMaxChunks];
  __shared__ float sums[kWaves][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int id = (int)blockIdx.x;
  const int hd = id % a.heads;
  id /= a.heads;
  const int b = id % a.batch, i = id / a.batch;
  const Span sp = span_of(a, b);
  if (!cut.has(sp) || i * a.group >= sp.rows) return;
  const int row = i * a.group + hd % a.group;
  const int end = tile_end(a, sp, row - row % cut.tile_rows, cut.tile_rows);
  if (end <= cut.chunk) return;
  const int n = (end + cut.chunk - 1) / cut.chunk;
  const int64_t at = ((int64_t)(sp.q0 + i) * a.heads + hd) * cut.chunks;
  float m = -INFINITY;
  for (int c = lane; c < n; c += 64) m = fmaxf(m, parts.ml[at + c].x);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f, le = 0.f;
  for (int c = lane; c < n; c += 64) {
    const float4 x = parts.ml[at + c];
    const float f = __builtin_amdgcn_exp2f(x.x - ref);
    if (wave == 0) factor[c] = f;
    l += x.y * f;
    le += x.z * f;
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    l += __shfl_xor(l, s);
    le += __shfl_xor(le, s);
  }
  __syncthreads();
  float o[C] = {};
#pragma unroll 4
  for (int c = wave; c < n; c += kWaves) {
    const float f = factor[c];
#pragma unroll
    for (int x = 0; x < C; ++x) o[x] += f * parts.o[(at + c) * D + 64 * x + lane];
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

// The same for few parts of many rows: D / 4 lanes take a query row and head, and
// no lane waits for another.
template <int D>
__global__ void __launch_bounds__(256)
join_few_kernel(Kv4Attn a, Cut cut, Parts parts, int most) {
  constexpr int LANES = D / 4;
  int64_t id = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const int c4 = 4 * (threadIdx.x % LANES);
  const int hd = (int)(id % a.heads);
  id /= a.heads;
  const int i = (int)(id % most), b = (int)(id / most);
  if (b >= a.batch) return;
  Span sp;  // of this lane's request (a workgroup may hold rows of two)
  sp.q0 = min(max(a.q_start[b], 0), a.n_rows);
  sp.m = min(max(a.q_start[b + 1], sp.q0), a.n_rows) - sp.q0;
  sp.rows = min(sp.m, a.max_q) * a.group;
  sp.kv = min(max(a.kv_len[b], 0), a.width << a.c.shift);
  if (!cut.has(sp) || i * a.group >= sp.rows) return;
  const int row = i * a.group + hd % a.group;
  const int end = tile_end(a, sp, row - row % cut.tile_rows, cut.tile_rows);
  if (end <= cut.chunk) return;
  const int n = (end + cut.chunk - 1) / cut.chunk;
  const int64_t at = ((int64_t)(sp.q0 + i) * a.heads + hd) * cut.chunks;
  float m = -INFINITY;
  for (int c = 0; c < n; ++c) m = fmaxf(m, parts.ml[at + c].x);
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f, le = 0.f;
  f32x4 o = {};
#pragma unroll 4
  for (int c = 0; c < n; ++c) {
    const float4 x = parts.ml[at + c];
    const f32x4 v = *reinterpret_cast<const f32x4 *>(parts.o + (at + c) * D + c4);
    const float f = __builtin_amdgcn_exp2f(x.x - ref);
    l += x.y * f;
    le += x.z * f;
    o += v * f;
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
  const size_t lds = (size_t)2 * NT * (D / 64 * 16 + 3) * 64 * 4;
  const int64_t grid = (int64_t)cut.tiles * a.batch * a.c.heads * cut.chunks;
  const auto f = cut.chunks > 1 ? &rows_kernel<D, NT, true> : &rows_kernel<D, NT, false>;
  const hipError_t e = allow_lds(reinterpret_cast<const void *>(f), lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(f, dim3((unsigned)grid), dim3(64 * kWaves), lds, s, a, cut, parts);
  return hipGetLastError();
}

constexpr int kMaxParts = 64;  // parts of the requests of many rows

int64_t up(int64_t x, int64_t y) { return (x + y - 1) / y; }

// Rows of a request, at most.
int64_t most_rows(const Kv4Attn &a) { return (int64_t)a.max_q * a.group; }

// Rows of a request up to which rows_kernel takes it: at d = 128 the outputs of
// 64 rows do not fit the registers of two waves a SIMD (8 heads, 16,000 tokens,
// 48 rows: 35 us with one wave a SIMD, 23 in the other kernel).
int few_rows(const Kv4Attn &a) { return a.c.d == 128 ? 32 : 64; }

// Cuts the key axis into parts of `chunk` tokens (a multiple of 128).
void set_chunk(Cut &cut, int64_t reach, int64_t chunk) {
  if (chunk * kMaxChunks < reach) chunk = up(reach, kMaxChunks * 128) * 128;
  cut.chunk = (int)chunk;
  cut.chunks = (int)up(reach, chunk);
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
Cut few_cut(const Kv4Attn &a) {
  const int64_t rows = most_rows(a) < few_rows(a) ? most_rows(a) : few_rows(a);
  const int nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const int64_t reach = (int64_t)a.width << a.c.shift;
  const int64_t base = (int64_t)a.batch * a.c.heads;
  Cut cut{0, few_rows(a), 16 * nt, 1, (int)reach, 1, 1};
  if (reach <= 512 || (reach <= 1024 && base > 64)) return cut;
  const int64_t chunk = up(up(reach * base, 640), 128) * 128;
  set_chunk(cut, reach, chunk > 1536 ? 1536 : chunk);
  return cut;
}

// The requests of more rows (tiles is 0 where there can be none).  Parts of the
// key axis fill CUs that the tiles leave empty and even out the last round, and
// cost their outputs' way through memory; their number is the one with the least
// time by this: a token of a tile takes 27 ns (19 at d = 64) with two workgroups
// on the CU and 20 (14.6) with one, so 512 workgroups are a round
// (half a one more than their number says, past two); a part of a
// tile adds 0.03 us (half at d = 64) to the joining, which begins at 6 us.  Per call at d =
// 128, whole / in parts of 512 / 2048 / 4096 tokens:
//   8 tiles, 2000 tokens: 50 / 25 / - / - us (17 in parts of 128)
//   60 tiles, 16,000: 317 / 109 / 86 / 103
//   192 tiles, 16,000: 319 / 325 / 238 / 240
//   444 tiles, 32,000: 863 / 1416 / 984 / 931
Cut many_cut(const Kv4Attn &a) {
  const int64_t reach = (int64_t)a.width << a.c.shift;
  Cut cut{few_rows(a), 0x7FFFFFFF, kTileRows, 0, (int)reach, 1, 0};
  if (most_rows(a) <= few_rows(a)) return cut;
  if (a.batch == 1) cut.over = 0;  // a single request is left to this kernel however few rows it has
  cut.tiles = (int)up(most_rows(a), kTileRows);
  // tiles that hold rows, about: the requests' sum is at most n_rows
  const int64_t all = (int64_t)cut.tiles * a.batch, held = up((int64_t)a.n_rows * a.group, kTileRows);
  const int64_t base = (all < held ? all : held) * a.c.heads;
  const double two = a.c.d == 128 ? 0.027 : 0.019, one = a.c.d == 128 ? 0.020 : 0.0146;
  const double part = a.c.d == 128 ? 0.03 : 0.015;
  double best = 1e300;
  for (int64_t n = 1; n <= kMaxParts && (n == 1 || reach >= n * 128); ++n) {
    const int64_t chunk = n == 1 ? reach : up(up(reach, n), 128) * 128;
    const double rounds = base * n <= 256 ? one / two : base * n <= 1024 ? (double)up(base * n, 512)
                                                                         : (double)(base * n) / 512 + 0.5;
    const double us = rounds * two * (double)chunk + (n > 1 ? 6 + part * (double)(base * n) : 0);
    if (us < best) {
      best = us;
      cut.chunk = (int)chunk;
      cut.chunks = (int)up(reach, chunk);
    }
  }
  cut.turns = cut.tiles;
  if (a.causal && a.batch > 1 && reach * a.group <= 4 * most_rows(a))
    cut.turns += (int)(reach * a.group / kTileRows);
  return cut;
}

// Scratch of a cut: the parts' outputs, then their references and sums.
size_t outputs_bytes(const Kv4Attn &a, const Cut &cut) {
  return align_up((size_t)a.n_rows * a.heads * cut.chunks * a.c.d * 4);
}
size_t parts_bytes(const Kv4Attn &a, const Cut &cut) {
  if (cut.chunks == 1 || cut.tiles == 0) return 0;
  return outputs_bytes(a, cut) + align_up((size_t)a.n_rows * a.heads * cut.chunks * 16);
}
int64_t workgroups(const Kv4Attn &a, const Cut &cut) {
  const int64_t main = (int64_t)cut.turns * a.batch * a.c.heads * cut.chunks;
  const int64_t join = cut.chunks > 1 ? (int64_t)a.max_q * a.batch * a.heads : 0;
  return main > join ? main : join;
}
Parts parts_at(const Kv4Attn &a, const Cut &cut, char *at) {
  return Parts{reinterpret_cast<float *>(at), reinterpret_cast<float4 *>(at + outputs_bytes(a, cut))};
}

hipError_t launch_join(const Kv4Attn &a, const Cut &cut, const Parts &parts, hipStream_t s) {
  // rows of the requests that it joins
  const int most = cut.upto < most_rows(a) ? cut.upto / a.group : a.max_q;
  const int64_t n = (int64_t)most * a.batch * a.heads;
  const bool d128 = a.c.d == 128;
  if (cut.chunks <= 16 && n >= 2048) {
    const dim3 grid((unsigned)up(n, 1024 / a.c.d));
    if (d128) hipLaunchKernelGGL(join_few_kernel<128>, grid, dim3(256), 0, s, a, cut, parts, most);
    else hipLaunchKernelGGL(join_few_kernel<64>, grid, dim3(256), 0, s, a, cut, parts, most);
  } else if (d128) {
    hipLaunchKernelGGL(join_kernel<128>, dim3((unsigned)n), dim3(64 * kWaves), 0, s, a, cut, parts);
  } else {
    hipLaunchKernelGGL(join_kernel<64>, dim3((unsigned)n), dim3(64 * kWaves), 0, s, a, cut, parts);
  }
  return hipGetLastError();
}

}  // namespace

int64_t kv4_attn_workgroups(const Kv4Attn &a) {
  const int64_t x = workgroups(a, few_cut(a)), y = workgroups(a, many_cut(a));
  return x > y ? x : y;
}

size_t kv4_attn_scratch_bytes(const Kv4Attn &a) { return parts_bytes(a, few_cut(a)) + parts_bytes(a, many_cut(a)); }

hipError_t launch_kv4_attn(const Kv4Attn &a, void *scratch, hipStream_t s) {
  const Cut few = few_cut(a), many = many_cut(a);
  char *at = static_cast<char *>(scratch);
  hipError_t e = hipSuccess;
  if (many.tiles > 0) {
    const Parts parts = parts_at(a, many, at + parts_bytes(a, few));
    if ((e = launch_kv4_tiles(a, many, parts, s)) != hipSuccess) return e;
    if (many.chunks > 1 && (e = launch_join(a, many, parts, s)) != hipSuccess) return e;
    if (many.over == 0) return e;
  }
  const Parts parts = parts_at(a, few, at);
  const bool d128 = a.c.d == 128;
  switch (few.tile_rows) {
    case 16: e = d128 ? launch_rows<128, 1>(a, few, parts, s) : launch_rows<64, 1>(a, few, parts, s); break;
    case 32: e = d128 ? launch_rows<128, 2>(a, few, parts, s) : launch_rows<64, 2>(a, few, parts, s); break;
    default: e = launch_rows<64, 4>(a, few, parts, s);
  }
  if (e != hipSuccess || few.chunks == 1) return e;
  return launch_join(a, few, parts, s);
}

}  // namespace carnator
