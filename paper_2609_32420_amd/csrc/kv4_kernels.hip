// Cached keys and values in 4 bits (Sec. 3.3: tokens outside the active region
// keep their cached computation): where new tokens go (page plan), writing them
// (store) and reading them back as bf16 (load).  The attention over the pages
// is in kv4_attn_kernels.hip.
//
// All three are bound by HBM at size and by their launch when small.  The
// format puts 32 channels of a token under one power of two, so a value is
// converted by one instruction for two channels in either direction
// (v_cvt_scalef32_pk_fp4_bf16 and its inverse take the exponent of an fp32
// scale; rounding, saturation and the NaN scale are those of the format,
// checked on gfx950 for every bf16 value and scale).
#include "internal.h"

#include <type_traits>

namespace carnator {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- page plan

constexpr int kPlanSlots = 4;  // consecutive slots of a thread

// Exclusive scan of x over the T threads of a workgroup, sums cut at cap (x, cap
// <= 2^31 - 1), and the total.  tmp: one value per wave; the next call with the
// same tmp has to lie behind another barrier.
template <int T>
__device__ inline unsigned scan_cut(unsigned x, unsigned cap, unsigned *tmp, unsigned *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned inc = min(x, cap);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned y = __shfl_up(inc, o);
    if (lane >= o) inc = min(inc + y, cap);
  }
  if (lane == 63) tmp[wave] = inc;
  __syncthreads();
  unsigned before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < T / 64; ++w) {
    if (w < wave) before = min(before + tmp[w], cap);
    sum = min(sum + tmp[w], cap);
  }
  *total = sum;
  const unsigned y = __shfl_up(inc, 1);
  return min(before + (lane ? y : 0u), cap);
}

// Every workgroup scans the lengths by itself, R to a thread (a batch is a few KB
// in L2), so that one launch does: a second one costs more than the
// scans.  Workgroup 0 writes what there is per request, every workgroup the slots
// of its tokens; a page is entered in the table by the token that it begins
// with.  4096 requests, 580,000 tokens: 11.8 us with 1024 threads (35 with 256
// that each scanned consecutive requests); 64 requests of a token: 4.6 us (7.2).
template <int T, int R>
__global__ void __launch_bounds__(T)
plan_kernel(const int32_t *__restrict__ kv_len, const int32_t *__restrict__ new_len, int batch,
            int32_t *__restrict__ table, int width, const int32_t *__restrict__ free_pages, int n_free, int shift,
            int32_t *__restrict__ q_start, int32_t *__restrict__ kv_len_out, int32_t *__restrict__ slots,
            int32_t *__restrict__ positions, int n_slots, int32_t *__restrict__ counts) {
  extern __shared__ int lds_plan[];
  int *start = lds_plan;              // [batch + 1]
  int *first = lds_plan + batch + 1;  // [batch]
  __shared__ unsigned tmp[2][T / 64];
  __shared__ unsigned long long left;
  const int most = width << shift;
  auto clamped = [&](int kv) { return min(max(kv, 0), most); };
  auto full_of = [&](int kv) { return (int)(((int64_t)kv + (1 << shift) - 1) >> shift); };

  // ---- starts of the requests' new tokens, first new page of each
  if (threadIdx.x == 0) left = 0;
  const unsigned cap = (unsigned)n_slots;
  unsigned total = 0, pages = 0;
  unsigned long long lack = 0;
  for (int base = 0; base < batch; base += T * R) {
    const int b0 = base + (int)threadIdx.x * R;
    int wish[R], kv[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int b = min(b0 + i, batch - 1);
      wish[i] = new_len[b];
      kv[i] = kv_len[b];
    }
    unsigned sum = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      wish[i] = b0 + i < batch ? max(wish[i], 0) : 0;
      kv[i] = clamped(kv[i]);
      sum = min(sum + min((unsigned)wish[i], cap), cap);
    }
    unsigned all;
    unsigned at[R + 1], page[R + 1];
    at[0] = min(total + scan_cut<T>(sum, cap, tmp[0], &all), cap);
    total = min(total + all, cap);
    int want[R];
    sum = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      at[i + 1] = min(at[i] + min((unsigned)wish[i], cap), cap);
      const int n = (int)(at[i + 1] - at[i]);
      const int end = (int)min((int64_t)width, ((int64_t)kv[i] + n + (1 << shift) - 1) >> shift);
      want[i] = max(end - full_of(kv[i]), 0);
      sum += want[i];
    }
    page[0] = pages + scan_cut<T>(sum, 0x7FFFFFFFu, tmp[1], &all);
    pages += all;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int b = b0 + i;
      page[i + 1] = page[i] + want[i];
      if (b >= batch) continue;
      start[b] = (int)at[i];
      first[b] = (int)page[i];
      if (blockIdx.x == 0) {
        const int64_t reach = min((int64_t)width, (int64_t)full_of(kv[i]) + max(n_free - (int)page[i], 0));
        const int placed = (int)min((int64_t)(at[i + 1] - at[i]), max((reach << shift) - kv[i], (int64_t)0));
        q_start[b] = (int)at[i];
        kv_len_out[b] = kv[i] + placed;
        lack += (unsigned long long)(wish[i] - placed);
      }
    }
  }
  if (threadIdx.x == 0) start[batch] = (int)total;
  if (blockIdx.x == 0) {
    if (lack) atomicAdd(&left, lack);
    __syncthreads();
    if (threadIdx.x == 0) {
      q_start[batch] = (int)total;
      counts[0] = (int)total;
      counts[1] = (int)min(pages, (unsigned)n_free);
      counts[2] = (int)min(left, (unsigned long long)0x7FFFFFFF);
    }
  }
  __syncthreads();

  // ---- the tokens
  const int64_t step = (int64_t)gridDim.x * T * kPlanSlots;
  for (int64_t t0 = ((int64_t)blockIdx.x * T + threadIdx.x) * kPlanSlots; t0 < n_slots; t0 += step) {
    int b = 0;
    if (t0 < total) {  // the request of slot t0: the last with start <= t0
      int hi = batch;
      while (hi - b > 1) {
        const int mid = (b + hi) >> 1;
        if (start[mid] <= t0) b = mid;
        else hi = mid;
      }
    }
    int slot[kPlanSlots], pos[kPlanSlots];
#pragma unroll
    for (int i = 0; i < kPlanSlots; ++i) {
      const int64_t t = t0 + i;
      slot[i] = pos[i] = -1;
      if (t >= total) continue;
      while (start[b + 1] <= t) ++b;
      const int kv = clamped(kv_len[b]);
      const int64_t p = (int64_t)kv + (t - start[b]);  // < 2^32
      pos[i] = (int)min(p, (int64_t)0x7FFFFFFF);
      const int64_t k = p >> shift;
      if (k >= width) continue;
      const int full = full_of(kv);
      int page;
      if (k < full) {
        page = table[(int64_t)b * width + k];
      } else {
        const int64_t f = (int64_t)first[b] + (k - full);
        if (f >= n_free) continue;
        page = free_pages[f];
        if ((p & ((1 << shift) - 1)) == 0) table[(int64_t)b * width + k] = page;
      }
      if (page >= 0 && page <= (0x7FFFFFFF >> shift) - 1) slot[i] = (page << shift) + (int)(p & ((1 << shift) - 1));
    }
#pragma unroll
    for (int i = 0; i < kPlanSlots; ++i)
      if (t0 + i < n_slots) {
        slots[t0 + i] = slot[i];
        if (positions) positions[t0 + i] = pos[i];
      }
  }
}

// ---------------------------------------------------------------- store

// Scale byte of a group whose largest magnitude has the bf16 bits `most`:
// 1.m * 2^x <= 7 * 2^e = 1.75 * 2^(e + 2), so e = x - 2, one more where the
// mantissa passes 1.75.
__device__ inline unsigned scale_of(unsigned most) {
  if (most >= 0x7F80u) return 255;
  const int e = (int)(most >> 7) - 2 + ((most & 127) > 96 ? 1 : 0);
  return (unsigned)min(max(e, 2), 252);
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Codes of eight channels (bf16 bits in x) and the scale byte of the 32 that
// four neighbouring lanes hold.
__device__ inline uint2 quantise(const uint4 &x) {
  const auto magnitude = [](unsigned w) { return __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu); };
  const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(magnitude(x.x), magnitude(x.y)),
                                            __builtin_elementwise_max(magnitude(x.z), magnitude(x.w)));
  unsigned most = max((unsigned)m.x, (unsigned)m.y);
  most = max(most, (unsigned)__builtin_amdgcn_mov_dpp((int)most, 0xB1, 0xF, 0xF, false));  // quad_perm [1, 0, 3, 2]
  most = max(most, (unsigned)__builtin_amdgcn_mov_dpp((int)most, 0x4E, 0xF, 0xF, false));  // quad_perm [2, 3, 0, 1]
  const unsigned scale = scale_of(most);
  const float s = __uint_as_float(scale << 23);
  unsigned c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2, x.x), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.y), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.z), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.w), s, 3);
  return make_uint2(c, scale);
}

// A wave takes K or V of eight rows of 64 / (D / 8) heads, a lane eight channels
// of each.  K goes out four bytes a lane and row.  V lies by octets of tokens: rows
// that fill an octet (consecutive slots from a multiple of 8 on, as a prompt's
// rows have them, at whatever row it begins) are transposed in registers and
// stored 32 bytes a lane; other rows go out byte by byte.  Such a run belongs to
// the wave whose eight rows hold its first one, which finds them all from the
// slots of these rows and of the eight on either side.  `subs` waves share the
// eight rows of a small call, to wait for fewer of them in turn: 31 rows of 8
// heads 4.1 us (8.0 with one wave).  32,760 rows of 12 heads, d = 128 (201 MB read,
// 53 written): 66 us from HBM, 3.9 TB/s, bound by the reads (55 without the stores);
// 49 where part of the rows is still in the Infinity Cache.
template <int D>
__global__ void __launch_bounds__(256)
store_kernel(Kv4 c, Rows k, Rows v, int n_rows, const int32_t *__restrict__ slots, int subs, int64_t waves) {
  constexpr int LANES = D / 8, HEADS = 64 / LANES;
  const int block = 1 << c.shift;
  const int64_t limit = (int64_t)c.n_pages << c.shift;
  const int rec = kv4_head_bytes(D, block);
  const int codes = kv4_codes(D, block), scales = kv4_scales(D, block);
  const int lane = threadIdx.x & 63, l = lane % LANES, q = l & 3, g = l >> 2;
  const int parts = (c.heads + HEADS - 1) / HEADS;
  for (int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < waves;
       w += (int64_t)gridDim.x * 4) {
    int64_t oct = w >> 1;
    const bool is_v = w & 1;
    const Rows x = is_v ? v : k;
    const int sub = (int)(oct % subs);
    oct /= subs;
    const int64_t part = oct % parts;
    oct /= parts;
    const int head = (int)part * HEADS + lane / LANES;
    const bool live = head < c.heads;
    // slots of rows 8 oct - 8 + lane, lanes 0 to 23
    const int64_t r0 = 8 * oct - 8;
    int slot = -1;
    if (lane < 24 && r0 + lane >= 0 && r0 + lane < n_rows) {
      slot = slots[r0 + lane];
      if ((unsigned)slot >= (uint64_t)limit) slot = -1;
    }
    const int after = __shfl_down(slot, 1);
    const uint64_t valid = __ballot(slot >= 0);
    const uint64_t begins = __ballot(slot >= 0 && (slot & 7) == 0);
    uint64_t run = __ballot(slot >= 0 && lane < 23 && after == slot + 1);  // the next row has the next slot
    run &= run >> 1;
    run &= run >> 2;
    run = begins & run & (run >> 3) & 0x1FFFF;  // seven times in turn
    uint64_t in_run = run | run << 1;
    in_run |= in_run << 2;
    in_run |= in_run << 4;

    // rows first + e of the window, e in mask; whole: they are a run
    auto put = [&](int first, unsigned mask, bool whole) {
      uint4 raw[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        raw[e] = make_uint4(0, 0, 0, 0);
        if ((mask >> e & 1) && live)
          raw[e] = *reinterpret_cast<const uint4 *>(x.data + (r0 + first + e) * x.st + head * x.sh + 8 * l);
      }
      unsigned d[8], sc[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint2 y = quantise(raw[e]);
        d[e] = y.x;
        sc[e] = y.y;
      }
      if (!live) return;
      auto place = [&](int s) { return c.pages + ((int64_t)(s >> c.shift) * c.heads + head) * rec; };
      if (is_v && whole) {
        const int s = __builtin_amdgcn_readlane(slot, first), t = s & (block - 1);
        unsigned char *dst = place(s) + codes + scales;
        unsigned o[4][2];  // channel pair, tokens 0-3 and 4-7
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const unsigned a = __builtin_amdgcn_perm(d[4 * h + 1], d[4 * h], 0x05010400u);
          const unsigned b = __builtin_amdgcn_perm(d[4 * h + 3], d[4 * h + 2], 0x05010400u);
          const unsigned cc = __builtin_amdgcn_perm(d[4 * h + 1], d[4 * h], 0x07030602u);
          const unsigned dd = __builtin_amdgcn_perm(d[4 * h + 3], d[4 * h + 2], 0x07030602u);
          o[0][h] = __builtin_amdgcn_perm(b, a, 0x05040100u);
          o[1][h] = __builtin_amdgcn_perm(b, a, 0x07060302u);
          o[2][h] = __builtin_amdgcn_perm(dd, cc, 0x05040100u);
          o[3][h] = __builtin_amdgcn_perm(dd, cc, 0x07060302u);
        }
        uint4 *to = reinterpret_cast<uint4 *>(dst + ((t >> 3) * (D / 2) + 4 * l) * 8);
        to[0] = make_uint4(o[0][0], o[0][1], o[1][0], o[1][1]);
        to[1] = make_uint4(o[2][0], o[2][1], o[3][0], o[3][1]);
        if (q == 0)
          *reinterpret_cast<uint2 *>(dst + codes + ((t >> 3) * (D / 32) + g) * 8) = make_uint2(
              sc[0] | sc[1] << 8 | sc[2] << 16 | sc[3] << 24, sc[4] | sc[5] << 8 | sc[6] << 16 | sc[7] << 24);
        return;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!(mask >> e & 1)) continue;
        const int s = __builtin_amdgcn_readlane(slot, first + e), t = s & (block - 1);
        unsigned char *dst = place(s);
        if (is_v) {
          dst += codes + scales;
          unsigned char *to = dst + ((t >> 3) * (D / 2) + 4 * l) * 8 + (t & 7);
#pragma unroll
          for (int b = 0; b < 4; ++b) to[8 * b] = (unsigned char)(d[e] >> (8 * b));
          if (q == (e & 3)) dst[codes + ((t >> 3) * (D / 32) + g) * 8 + (t & 7)] = (unsigned char)sc[e];
        } else {
          *reinterpret_cast<unsigned *>(dst + t * (D / 2) + 4 * l) = d[e];
          if (q == (e & 3)) dst[codes + t * (D / 32) + g] = (unsigned char)sc[e];
        }
      }
    };
    const unsigned own = (unsigned)(run >> 8) & 0xFF;  // at most one begins here
    if (own && sub == 0) put(8 + __builtin_ctz(own), 0xFF, true);
    const unsigned rest = (unsigned)((valid & ~in_run) >> 8) & (subs == 1 ? 0xFFu : 3u << (2 * sub));
    if (rest) put(8, rest, false);
  }
}

// ---------------------------------------------------------------- load

template <int SEL>
__device__ inline unsigned value_pair(unsigned codes, unsigned scale) {
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, __uint_as_float(scale << 23), SEL));
}

// A thread reads eight channels of eight consecutive tokens (an octet of V, as
// it lies; eight rows of K) and writes 16 bytes of each token: 16 (8) lanes
// cover a token's row, consecutive octets follow.  STREAM: outputs past the L2s (4
// MB each) go out as nontemporal stores, which leave what else is cached where it
// is: 17,776 tokens of 48 heads, d = 64, 60 % of the pages (38 MB read, 141
// written) 44.9 -> 31.4 us (5.7 TB/s), 32,760 of 12 heads, d = 128 (54 and 201) 47.6
// -> 42.4.
template <int D, bool STREAM>
__global__ void __launch_bounds__(256)
load_kernel(Kv4 c, const int32_t *__restrict__ table, int batch, int width, const int32_t *__restrict__ kv_len, int n,
            uint16_t *__restrict__ ko, int64_t ksb, int64_t ksh, int64_t ksn, uint16_t *__restrict__ vo, int64_t vsb,
            int64_t vsh, int64_t vsn, int per, int64_t groups) {
  constexpr int CH = D / 8;      // threads of an octet
  constexpr int OCT = 256 / CH;  // octets of a workgroup
  const int block = 1 << c.shift;
  const int rec = kv4_head_bytes(D, block);
  const int codes = kv4_codes(D, block), scales = kv4_scales(D, block);
  const int c8 = threadIdx.x % CH;
  auto put = [](uint16_t *to, const u32x4 &w) {
    if constexpr (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(to));
    else *reinterpret_cast<u32x4 *>(to) = w;
  };
  for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
    const int bh = (int)(g / per);
    const int b = bh / c.heads, h = bh - b * c.heads;
    const int64_t t0 = ((g - (int64_t)bh * per) * OCT + threadIdx.x / CH) * 8;
    const int kv = min(min(max(kv_len[b], 0), width << c.shift), n);
    if (t0 >= kv) continue;
    const int page = table[(int64_t)b * width + (t0 >> c.shift)];
    if ((unsigned)page >= (unsigned)c.n_pages) continue;
    const unsigned char *base = c.pages + ((int64_t)page * c.heads + h) * rec;
    const int tp = (int)t0 & (block - 1);
    unsigned kw[8], ks[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      kw[e] = *reinterpret_cast<const unsigned *>(base + (tp + e) * (D / 2) + 4 * c8);
      ks[e] = base[codes + (tp + e) * (D / 32) + c8 / 4];
    }
    const unsigned char *vb = base + codes + scales;
    const uint4 v0 = *reinterpret_cast<const uint4 *>(vb + ((tp >> 3) * (D / 2) + 4 * c8) * 8);
    const uint4 v1 = *reinterpret_cast<const uint4 *>(vb + ((tp >> 3) * (D / 2) + 4 * c8) * 8 + 16);
    const uint2 vs = *reinterpret_cast<const uint2 *>(vb + codes + ((tp >> 3) * (D / 32) + c8 / 4) * 8);
    const int valid = (int)min((int64_t)8, kv - t0);
    uint16_t *kp = ko + b * ksb + h * ksh + t0 * ksn + 8 * c8;
    uint16_t *vp = vo + b * vsb + h * vsh + t0 * vsn + 8 * c8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e >= valid) break;
      put(kp + e * ksn, u32x4{value_pair<0>(kw[e], ks[e]), value_pair<1>(kw[e], ks[e]), value_pair<2>(kw[e], ks[e]),
                              value_pair<3>(kw[e], ks[e])});
    }
    auto v_row = [&](auto sel, int e, unsigned p0, unsigned p1, unsigned p2, unsigned p3, unsigned sw) {
      constexpr int S = decltype(sel)::value;
      if (e >= valid) return;
      const unsigned sc = (sw >> (8 * S)) & 255u;
      put(vp + e * vsn, u32x4{value_pair<S>(p0, sc), value_pair<S>(p1, sc), value_pair<S>(p2, sc),
                              value_pair<S>(p3, sc)});
    };
    v_row(std::integral_constant<int, 0>{}, 0, v0.x, v0.z, v1.x, v1.z, vs.x);
    v_row(std::integral_constant<int, 1>{}, 1, v0.x, v0.z, v1.x, v1.z, vs.x);
    v_row(std::integral_constant<int, 2>{}, 2, v0.x, v0.z, v1.x, v1.z, vs.x);
    v_row(std::integral_constant<int, 3>{}, 3, v0.x, v0.z, v1.x, v1.z, vs.x);
    v_row(std::integral_constant<int, 0>{}, 4, v0.y, v0.w, v1.y, v1.w, vs.y);
    v_row(std::integral_constant<int, 1>{}, 5, v0.y, v0.w, v1.y, v1.w, vs.y);
    v_row(std::integral_constant<int, 2>{}, 6, v0.y, v0.w, v1.y, v1.w, vs.y);
    v_row(std::integral_constant<int, 3>{}, 7, v0.y, v0.w, v1.y, v1.w, vs.y);
  }
}

// Workgroups of a launch whose kernel walks the rest of its work in a loop.
constexpr int64_t kMaxGrid = (int64_t)1 << 22;

}  // namespace

hipError_t launch_page_plan(const int32_t *kv_len, const int32_t *new_len, int batch, int32_t *table, int width,
                            const int32_t *free_pages, int n_free, int shift, int32_t *q_start, int32_t *kv_len_out,
                            int32_t *slots, int32_t *positions, int n_slots, int32_t *counts, hipStream_t s) {
  const size_t lds = (size_t)(2 * batch + 1) * 4;
  // few requests and tokens: a small workgroup starts and meets sooner
  const bool small = batch <= 256 && n_slots <= 4096;
  const auto f = small ? &plan_kernel<256, 1> : &plan_kernel<1024, 4>;
  const int threads = small ? 256 : 1024;
  const hipError_t e = allow_lds(reinterpret_cast<const void *>(f), lds);
  if (e != hipSuccess) return e;
  const int64_t need = ((int64_t)n_slots + threads * kPlanSlots - 1) / (threads * kPlanSlots);
  const unsigned grid = (unsigned)(need < 1 ? 1 : need > 512 ? 512 : need);
  hipLaunchKernelGGL(f, dim3(grid), dim3(threads), lds, s, kv_len, new_len, batch, table, width, free_pages, n_free,
                     shift, q_start, kv_len_out, slots, positions, n_slots, counts);
  return hipGetLastError();
}

hipError_t launch_kv4_store(Kv4 c, Rows k, Rows v, int n_rows, const int32_t *slots, hipStream_t s) {
  const int heads = 512 / c.d;  // of a wave
  const int64_t octets = ((int64_t)n_rows + 7) / 8 * ((c.heads + heads - 1) / heads);
  const int subs = octets <= 256 ? 4 : 1;  // 8 waves of each, 2048 in all: a wave a SIMD
  const int64_t waves = 2 * octets * subs, need = (waves + 3) / 4;
  const dim3 grid((unsigned)(need < kMaxGrid ? need : kMaxGrid));
  if (c.d == 128) hipLaunchKernelGGL(store_kernel<128>, grid, dim3(256), 0, s, c, k, v, n_rows, slots, subs, waves);
  else hipLaunchKernelGGL(store_kernel<64>, grid, dim3(256), 0, s, c, k, v, n_rows, slots, subs, waves);
  return hipGetLastError();
}

hipError_t launch_kv4_load(Kv4 c, const int32_t *table, int batch, int width, const int32_t *kv_len, int n,
                           uint16_t *ko, int64_t ksb, int64_t ksh, int64_t ksn, uint16_t *vo, int64_t vsb, int64_t vsh,
                           int64_t vsn, hipStream_t s) {
  const int64_t reach = (int64_t)width << c.shift;
  const int64_t most = n < reach ? n : reach;
  const int tokens = 8 * 256 / (c.d / 8);  // of a workgroup
  const int64_t per = (most + tokens - 1) / tokens;
  const int64_t groups = per * batch * c.heads;
  const dim3 grid((unsigned)(groups < kMaxGrid ? groups : kMaxGrid));
  const bool stream = groups * tokens * c.d * 4 > ((int64_t)32 << 20);
  const auto f = c.d == 128 ? (stream ? &load_kernel<128, true> : &load_kernel<128, false>)
                            : (stream ? &load_kernel<64, true> : &load_kernel<64, false>);
  hipLaunchKernelGGL(f, grid, dim3(256), 0, s, c, table, batch, width, kv_len, n, ko, ksb, ksh, ksn, vo, vsb, vsh, vsn,
                     (int)per, groups);
  return hipGetLastError();
}

}  // namespace carnator
