// Attention over cached keys and values in 4 bits (Sec. 3.3: tokens outside the
// active region keep their cached computation), for each request's queries over
// the pages that its table names.
//
// A workgroup takes one request, one cached head and up to 16 NT query rows (a row
// is a query token and one of the query heads that share the cached head, so the
// cache is read once for all of them). Its waves take 32 tokens in turn. S = K Q^T
// and O^T += V^T P^T run on bf16 MFMA 16x16x32 with fp32 accumulation, one pass
// with a running maximum and sum per query (fp32, exp2 domain). Nothing passes
// through LDS: a lane's 16 bytes of K are one token's 32 channels under one scale,
// which is its A operand once converted (the channels are dealt to the four
// products in the same order for Q), and a lane's bytes of V are the eight tokens
// of an octet for two channels, which are an A operand of V^T each once the two
// are told apart. Rows of a K tile are permuted so that the scores of eight
// consecutive tokens end in one lane, as the B operand of the second product.
//
// Bound by the cache's bytes where there are many: 24 heads, d = 128, one query
// over 119,056 tokens (389 MB) 75 us, 5.2 TB/s (the loads alone 71, the rest alone
// 54); 47 requests of 32 / 8 heads and a query, 238,000 tokens in all (258 MB) 60
// us.  A step's loads are issued one step ahead, and three waves fit a SIMD (two:
// 112 us for the first, 86 with three before the axis was cut as now).  A short
// cache is the latency of a launch and of one step: 12 heads, 77 tokens 4.7 us.
#pragma once

#include "kv4_attn.h"

namespace carnator {

constexpr int kWaves = 4;  // of a workgroup of the kernel for few rows alone
constexpr int kStep = 32;  // tokens of a wave's step

// LDS of rows_body.
constexpr int rows_lds(int d, int nt, int waves) { return waves / 2 * nt * (d / 64 * 16 + 3) * 64 * 4; }

// What a wave reads of 32 tokens.
template <int D>
struct Raw {
  u32x4 k[2];        // 16 (8 at d = 64) bytes of a token
  uint32_t ks[2];    // their scale
  u32x4 v[D / 64];   // two channel pairs of an octet
  uint2 vs[D / 64];  // the octet's scales
};

// Request b, cached head h; SPLIT: of its key axis the parts column, column +
// cut.columns, .. in turn, under one running maximum and sum.
template <int D, int NT, bool SPLIT, int WAVES>
__device__ __attribute__((always_inline)) inline void rows_part(const Kv4Attn &a, const Cut &cut, const Parts &parts,
                                                                const Span &sp, int b, int h, int column, float *lds_o) {
  constexpr int TQ = D / 32;        // products of a key tile
  constexpr int CPL = D / 4;        // channels of a lane
  constexpr int NV = D / 64;        // 64-channel parts of V
  // lds_o: [WAVES / 2][NT * NV * 16][64] outputs, then [WAVES / 2][NT][3][64] references and sums
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, j = lane >> 4;
  constexpr int row0 = 0;
  const int end = tile_end(a, sp, row0, 16 * NT);  // tokens that a row of the tile sees
  const bool whole = !SPLIT || end <= cut.chunk;  // nothing to join
  int part = SPLIT ? column * cut.chunk : 0, part_end = SPLIT ? min(end, part + cut.chunk) : end;
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
  int entry0 = part >> a.c.shift;  // of lane 0
  int entry = -1;
  auto look = [&]() {
    entry = -1;
    if (entry0 + lane < a.width) entry = a.table[(int64_t)b * a.width + entry0 + lane];
  };
  look();
  int page = -1;
  // the first of the wave's steps from k0 on that has a page; end and beyond: none
  auto next = [&](int k0) {
    for (; k0 < end; k0 += WAVES * kStep) {
      if constexpr (SPLIT) {
        while (k0 >= part_end) {  // on to the workgroup's next part
          part = (int)min((unsigned)part + (unsigned)(cut.columns * cut.chunk), (unsigned)end);
          if (part == end) return end;
          part_end = min(end, part + cut.chunk);
          k0 = part + wave * kStep;
        }
      }
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
        // P is rounded to bf16 (by 2^-9 of itself at most) for the matrix cores, whose
        // fp32 rate is a sixteenth: outputs are then 0.0018 from fp64 (relative, norms)
        // over 77 tokens where fp32 weights leave 0.0017, 0.0014 for both over 119,056.
        // The outputs are divided by the sum of what is multiplied with V: a convex
        // combination of its rows; the LSE takes the unrounded sum
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
  const int stride = WAVES * kStep;
  int k0 = next(part + wave * kStep);
  if (k0 < end) {
    load(even, k0);
    int k1 = next(k0 + stride);
    while (k1 < end) {
      load(odd, k1);
      step(even, k0);
      k0 = next(k1 + stride);
      if (k0 < end) load(even, k0);
      step(odd, k1);
      k1 = next(k0 + stride);
    }
    if (k0 < end) step(even, k0);
  }
  // ---- sums over the lanes of a query, then the waves' parts in a fixed order
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    lrun[n] += __shfl_xor(lrun[n], 16);
    lrun[n] += __shfl_xor(lrun[n], 32);
    lexact[n] += __shfl_xor(lexact[n], 16);
    lexact[n] += __shfl_xor(lexact[n], 32);
  }
  float *ml = lds_o + WAVES / 2 * NT * NV * 16 * 64;
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
#pragma unroll
  for (int w = WAVES / 2; w > 1; w /= 2) {
    if (wave >= w && wave < 2 * w) put(wave - w);
    __syncthreads();
    if (wave < w) add(wave);
    __syncthreads();
  }
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
      const int64_t at = part_of(a, cut, sp, b, h, row, i, hd) + column;
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

// Workgroup `id` of a grid of heads x batch x columns.
template <int D, int NT, bool SPLIT, int WAVES>
__device__ __attribute__((always_inline)) inline void rows_body(const Kv4Attn &a, const Cut &cut, const Parts &parts, int id,
                                                                float *lds_o) {
  const int h = id % a.c.heads;
  id /= a.c.heads;
  const int b = id % a.batch;
  const Span sp = span_of(a, b);
  if (!cut.has(sp)) return;
  if constexpr (!SPLIT) {
    rows_part<D, NT, false, WAVES>(a, cut, parts, sp, b, h, 0, lds_o);
  } else {
    const int column = id / a.batch;
    if (column > 0 && column * cut.chunk >= tile_end(a, sp, 0, 16 * NT)) return;
    rows_part<D, NT, true, WAVES>(a, cut, parts, sp, b, h, column, lds_o);
  }
}

}  // namespace carnator
