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
#include "internal.h"

#include <math.h>

namespace carnator {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kStep = 32;  // tokens of a wave's step
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
__device__ inline Span span_of(const Kv4Attn &a, int b) {
  Span s;
  s.q0 = min(max(a.q_start[b], 0), a.n_rows);
  s.m = min(max(a.q_start[b + 1], s.q0), a.n_rows) - s.q0;
  s.rows = min(s.m, a.max_q) * a.group;
  s.kv = min(max(a.kv_len[b], 0), a.width << a.c.shift);
  return s;
}

template <int D, int NT>
__global__ void __launch_bounds__(64 * kWaves, 2)
rows_kernel(Kv4Attn a, int tiles) {
  constexpr int TQ = D / 32;        // products of a key tile
  constexpr int CPL = D / 4;        // channels of a lane
  constexpr int NV = D / 64;        // 64-channel parts of V
  extern __shared__ float lds_o[];  // [2][NT * NV * 16][64] outputs, then [2][NT][2][64] maxima and sums
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, j = lane >> 4;
  const int tile = (int)blockIdx.x % tiles;
  const int bh = (int)blockIdx.x / tiles;
  const int b = bh / a.c.heads, h = bh - b * a.c.heads;
  const Span sp = span_of(a, b);
  const int row0 = tile * 16 * NT;
  if (row0 >= sp.rows) return;

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
  // tokens that every row of the tile sees, and that one of them sees
  const int seen_by_all = sp.limit(a, row0 / a.group);
  const int end = sp.limit(a, (min(row0 + 16 * NT, sp.rows) - 1) / a.group);

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
  for (int k0 = wave * kStep; k0 < end; k0 += kWaves * kStep) {
    const int page = __builtin_amdgcn_readfirstlane(a.table[(int64_t)b * a.width + (k0 >> a.c.shift)]);
    if ((unsigned)page >= (unsigned)a.c.n_pages) continue;
    const unsigned char *base = a.c.pages + ((int64_t)page * a.c.heads + h) * rec;
    const int tp = k0 & (block - 1);
    // ---- K: tile T, MFMA row r is token 8 (r >> 2) + 4 T + (r & 3)
    bf16x8 kf[2][TQ];
#pragma unroll
    for (int T = 0; T < 2; ++T) {
      const int tok = tp + 8 * (r >> 2) + 4 * T + (r & 3);
      const uint32_t sc = (uint32_t)base[codes + tok * (D / 32) + j * CPL / 32] << 23;
      if constexpr (D == 128) {
        const u32x4 w = *reinterpret_cast<const u32x4 *>(base + tok * (D / 2) + 16 * j);
#pragma unroll
        for (int t = 0; t < TQ; ++t) kf[T][t] = eight_of(w[t], sc);
      } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(base + tok * (D / 2) + 8 * j);
        kf[T][0] = eight_of(w.x, sc);
        kf[T][1] = eight_of(w.y, sc);
      }
    }
    // ---- V: octet j; channels 64 v + 4 r .. + 4 (two pairs)
    u32x4 vw[NV];
    uint2 vs[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const unsigned char *vb = base + codes + scales;
      vw[v] = *reinterpret_cast<const u32x4 *>(vb + (((tp >> 3) + j) * (D / 2) + 32 * v + 2 * r) * 8);
      vs[v] = *reinterpret_cast<const uint2 *>(vb + codes + (((tp >> 3) + j) * (D / 32) + 2 * v + (r >> 3)) * 8);
    }
    const bool part = k0 + kStep > seen_by_all;  // a row does not see all of the tokens
    uint32_t poison[NV][2] = {};  // tokens whose V is NaN, of the two groups of a part
    if (part) {
      // A token out of a row's sight has P = 0 there, which NaN (or what lies
      // behind the last token) would still turn into NaN: its scale becomes that
      // of byte 0.  Rows that see it get their NaN afterwards.
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t &w = e < 4 ? vs[v].x : vs[v].y;
          const uint32_t byte = 0xFFu << (8 * (e & 3));
          const bool nan = (w & byte) == byte;
          const bool in = k0 + 8 * j + e < sp.kv;
          const uint64_t bad = __ballot(nan && in);
          if (nan || !in) w &= ~byte;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            poison[v][0] |= (bad >> (16 * g) & 0xFF) ? 1u << (8 * g + e) : 0u;
            poison[v][1] |= (bad >> (16 * g + 8) & 0xFF) ? 1u << (8 * g + e) : 0u;
          }
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
        const uint32_t w0 = vw[v][2 * pr], w1 = vw[v][2 * pr + 1];  // tokens 0-3, 4-7 of a channel pair
        const uint32_t x = vs[v].x, y = vs[v].y;
        const uint32_t t0 = pair_of<0>(w0, x << 23), t1 = pair_of<1>(w0, x << 15), t2 = pair_of<2>(w0, x << 7),
                       t3 = pair_of<3>(w0, x >> 1), t4 = pair_of<0>(w1, y << 23), t5 = pair_of<1>(w1, y << 15),
                       t6 = pair_of<2>(w1, y << 7), t7 = pair_of<3>(w1, y >> 1);
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
        const uint32_t mine = j < 2 ? poison[v][0] : poison[v][1];  // of this lane's output channels
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int see = limit[n] - k0;
          const uint32_t vis = see >= 32 ? ~0u : see <= 0 ? 0u : (1u << see) - 1;
          if (mine & vis)
#pragma unroll
            for (int q = 0; q < 4; ++q) o[n][v][q] = f32x4{NAN, NAN, NAN, NAN};
        }
      }
    }
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
    const float inv = lrun[n] > 0.f ? 1.f / lrun[n] : lrun[n] == 0.f ? 0.f : NAN;
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
    if (a.lse && j == 0) {
      // reference, exponent and log2 of the mantissa in fp64: the first two
      // can be large where the LSE is small
      const double l2 = (double)mrun[n] + (double)__builtin_amdgcn_frexp_expf(lexact[n]) +
                        (double)__log2f(__builtin_amdgcn_frexp_mantf(lexact[n]));
      a.lse[(int64_t)(sp.q0 + i) * a.heads + hd] =
          lexact[n] > 0.f ? (float)(l2 * 0.69314718055994531) : lexact[n] == 0.f ? -INFINITY : NAN;
    }
  }
}

template <int D, int NT>
hipError_t launch_rows(const Kv4Attn &a, hipStream_t s) {
  const int64_t rows = (int64_t)a.max_q * a.group;
  const int64_t tiles = (rows + 16 * NT - 1) / (16 * NT);
  const size_t lds = (size_t)2 * NT * (D / 64 * 16 + 3) * 64 * 4;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&rows_kernel<D, NT>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((rows_kernel<D, NT>), dim3((unsigned)(tiles * a.batch * a.c.heads)), dim3(64 * kWaves), lds, s, a,
                     (int)tiles);
  return hipGetLastError();
}

}  // namespace

int64_t kv4_attn_workgroups(const Kv4Attn &a) {
  return ((int64_t)a.max_q * a.group + 63) / 64 * a.batch * a.c.heads;
}

size_t kv4_attn_scratch_bytes(const Kv4Attn &) { return 0; }

hipError_t launch_kv4_attn(const Kv4Attn &a, void *, hipStream_t s) {
  return a.c.d == 128 ? launch_rows<128, 4>(a, s) : launch_rows<64, 4>(a, s);
}

}  // namespace carnator
