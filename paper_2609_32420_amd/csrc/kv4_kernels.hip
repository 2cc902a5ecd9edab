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

// ---------------------------------------------------------------- page plan

constexpr int kPlanThreads = 256;
constexpr int kPlanSlots = 4;  // consecutive slots of a thread

// Exclusive scan of x over the workgroup, sums cut at cap (x, cap <= 2^31 - 1).
// tmp: one value per wave; returns the total in *total.
__device__ inline unsigned scan_cut(unsigned x, unsigned cap, unsigned *tmp, unsigned *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned inc = min(x, cap);
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned y = __shfl_up(inc, o);
    if (lane >= o) inc = min(inc + y, cap);
  }
  __syncthreads();
  if (lane == 63) tmp[wave] = inc;
  __syncthreads();
  unsigned before = 0, sum = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before = min(before + tmp[w], cap);
    sum = min(sum + tmp[w], cap);
  }
  *total = sum;
  const unsigned y = __shfl_up(inc, 1);
  return min(before + (lane ? y : 0u), cap);
}

// Every workgroup scans the lengths by itself (a batch is a few KB in L2), so
// that one launch does: a second one costs more than the scans.  Workgroup 0
// writes what there is per request, every workgroup the slots of its tokens;
// a page is entered in the table by the token that it begins with.
__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(const int32_t *__restrict__ kv_len, const int32_t *__restrict__ new_len, int batch,
            int32_t *__restrict__ table, int width, const int32_t *__restrict__ free_pages, int n_free, int shift,
            int32_t *__restrict__ q_start, int32_t *__restrict__ kv_len_out, int32_t *__restrict__ slots,
            int32_t *__restrict__ positions, int n_slots, int32_t *__restrict__ counts) {
  extern __shared__ int lds_plan[];
  int *start = lds_plan;              // [batch + 1]
  int *first = lds_plan + batch + 1;  // [batch]
  __shared__ unsigned tmp[kPlanThreads / 64];
  __shared__ unsigned long long left;
  const int per = (batch + kPlanThreads - 1) / kPlanThreads;
  const int b0 = min((int)threadIdx.x * per, batch), b1 = min(b0 + per, batch);
  const int most = width << shift;
  auto held = [&](int b) { return min(max(kv_len[b], 0), most); };

  // ---- starts of the requests' new tokens
  unsigned sum = 0, total;
  for (int b = b0; b < b1; ++b) sum = min(sum + (unsigned)min(max(new_len[b], 0), n_slots), (unsigned)n_slots);
  unsigned at = scan_cut(sum, n_slots, tmp, &total);
  for (int b = b0; b < b1; ++b) {
    start[b] = (int)at;
    at = min(at + (unsigned)min(max(new_len[b], 0), n_slots), (unsigned)n_slots);
  }
  if (threadIdx.x == 0) start[batch] = (int)total;
  __syncthreads();
  // ---- first new page of each request
  auto want_of = [&](int b) {
    const int kv = held(b), n = start[b + 1] - start[b];
    const int full = (int)(((int64_t)kv + (1 << shift) - 1) >> shift);
    const int end = (int)min((int64_t)width, ((int64_t)kv + n + (1 << shift) - 1) >> shift);
    return (unsigned)max(end - full, 0);
  };
  sum = 0;
  for (int b = b0; b < b1; ++b) sum += want_of(b);
  unsigned pages;
  at = scan_cut(sum, 0x7FFFFFFFu, tmp, &pages);
  for (int b = b0; b < b1; ++b) {
    first[b] = (int)at;
    at += want_of(b);
  }
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) left = 0;
    __syncthreads();
    unsigned long long lack = 0;
    for (int b = b0; b < b1; ++b) {
      const int kv = held(b), n = start[b + 1] - start[b];
      const int64_t full = ((int64_t)kv + (1 << shift) - 1) >> shift;
      const int64_t end = min((int64_t)width, full + max(n_free - first[b], 0));
      const int placed = (int)min((int64_t)n, max((end << shift) - kv, (int64_t)0));
      q_start[b] = start[b];
      kv_len_out[b] = kv + placed;
      lack += (unsigned long long)(max(new_len[b], 0) - placed);
    }
    atomicAdd(&left, lack);
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
  const int64_t step = (int64_t)gridDim.x * kPlanThreads * kPlanSlots;
  for (int64_t t0 = ((int64_t)blockIdx.x * kPlanThreads + threadIdx.x) * kPlanSlots; t0 < n_slots; t0 += step) {
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
      const int kv = held(b);
      const int64_t p = (int64_t)kv + (t - start[b]);  // < 2^32
      pos[i] = (int)min(p, (int64_t)0x7FFFFFFF);
      const int64_t k = p >> shift;
      if (k >= width) continue;
      const int full = (int)(((int64_t)kv + (1 << shift) - 1) >> shift);
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

// Largest of the 16 lanes of a DPP row, in every lane.
__device__ inline unsigned row_max(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, false));   // quad_perm [1, 0, 3, 2]
  x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, false));   // quad_perm [2, 3, 0, 1]
  x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, false));  // row_half_mirror
  x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, false));  // row_mirror
  return x;
}

// Scale byte of a group whose largest magnitude has the bf16 bits `most`:
// 1.m * 2^x <= 7 * 2^e = 1.75 * 2^(e + 2), so e = x - 2, one more where the
// mantissa passes 1.75.
__device__ inline unsigned scale_of(unsigned most) {
  if (most >= 0x7F80u) return 255;
  const int e = (int)(most >> 7) - 2 + ((most & 127) > 96 ? 1 : 0);
  return (unsigned)min(max(e, 2), 252);
}

// Byte of two channels (bf16 bits in x) under a scale byte.
__device__ inline unsigned code_pair(unsigned x, unsigned scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2, x), __uint_as_float(scale << 23), 0) &
         255u;
}

// A thread quantises two channels of a head in eight consecutive rows, so its
// eight V bytes are one store where the rows' slots are an aligned run (rows of
// a prompt); 16 neighbouring lanes hold a scale's 32 channels.  K bytes are
// exchanged inside each four lanes, which then store four bytes of one row.
template <int D>
__global__ void __launch_bounds__(256)
store_kernel(Kv4 c, Rows k, Rows v, int n_rows, const int32_t *__restrict__ slots, int64_t items) {
  const unsigned per = (unsigned)c.heads * (D / 2);  // threads of eight rows
  const int block = 1 << c.shift;
  const int64_t limit = (int64_t)c.n_pages << c.shift;
  const int rec = kv4_head_bytes(D, block);
  const int codes = kv4_codes(D, block), scales = kv4_scales(D, block);
  for (int64_t base = (int64_t)blockIdx.x * 256; base < items; base += (int64_t)gridDim.x * 256) {
    // the rest of a division by workgroup, then by thread in 32 bits
    const int64_t o0 = base / per;
    const unsigned r0 = (unsigned)(base - o0 * per) + threadIdx.x;
    const int64_t oct = o0 + r0 / per;
    const unsigned in = r0 % per;
    const int head = in / (D / 2), pair = in % (D / 2);
    const int64_t row0 = 8 * oct;
    auto slot_at = [&](int64_t row) {
      const int s = row < n_rows ? slots[row] : -1;
      return (unsigned)s < (uint64_t)limit ? s : -1;
    };
    int slot[8];
    unsigned xk[8], xv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      slot[e] = slot_at(row0 + e);
      xk[e] = xv[e] = 0;
      if (slot[e] >= 0) {
        xk[e] = *reinterpret_cast<const unsigned *>(k.data + (row0 + e) * k.st + head * k.sh + 2 * pair);
        xv[e] = *reinterpret_cast<const unsigned *>(v.data + (row0 + e) * v.st + head * v.sh + 2 * pair);
      }
    }
    unsigned bk[2] = {0, 0}, bv[2] = {0, 0}, sk[2] = {0, 0}, sv[2] = {0, 0};  // byte e: row e
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned ak = row_max(max(xk[e] & 0x7FFFu, (xk[e] >> 16) & 0x7FFFu));
      const unsigned av = row_max(max(xv[e] & 0x7FFFu, (xv[e] >> 16) & 0x7FFFu));
      const unsigned ck = scale_of(ak), cv = scale_of(av);
      bk[e >> 2] |= code_pair(xk[e], ck) << (8 * (e & 3));
      bv[e >> 2] |= code_pair(xv[e], cv) << (8 * (e & 3));
      sk[e >> 2] |= ck << (8 * (e & 3));
      sv[e >> 2] |= cv << (8 * (e & 3));
    }
    auto place = [&](int s) {
      return c.pages + ((int64_t)(s >> c.shift) * c.heads + head) * rec;
    };
    const int lane = threadIdx.x & 63;
    // K: lane q of four takes rows q and 4 + q
    const unsigned q = lane & 3;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const unsigned a0 = __builtin_amdgcn_mov_dpp((int)bk[half], 0x00, 0xF, 0xF, false);
      const unsigned a1 = __builtin_amdgcn_mov_dpp((int)bk[half], 0x55, 0xF, 0xF, false);
      const unsigned a2 = __builtin_amdgcn_mov_dpp((int)bk[half], 0xAA, 0xF, 0xF, false);
      const unsigned a3 = __builtin_amdgcn_mov_dpp((int)bk[half], 0xFF, 0xF, 0xF, false);
      const unsigned lo = __builtin_amdgcn_perm(a1, a0, 0x0C0C0000u | (4 + q) << 8 | q);
      const unsigned hi = __builtin_amdgcn_perm(a3, a2, 0x00000C0Cu | (4 + q) << 24 | q << 16);
      const int s = slot_at(row0 + 4 * half + q);
      if (s >= 0)
        *reinterpret_cast<unsigned *>(place(s) + (s & (block - 1)) * (D / 2) + (pair & ~3)) = lo | hi;
    }
    // V
    bool run = slot[0] >= 0 && (slot[0] & 7) == 0;
#pragma unroll
    for (int e = 1; e < 8; ++e) run = run && slot[e] == slot[0] + e;
    if (run) {
      *reinterpret_cast<uint2 *>(place(slot[0]) + codes + scales +
                                 (((slot[0] & (block - 1)) >> 3) * (D / 2) + pair) * 8) = make_uint2(bv[0], bv[1]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (slot[e] >= 0) {
          const int t = slot[e] & (block - 1);
          place(slot[e])[codes + scales + ((t >> 3) * (D / 2) + pair) * 8 + (t & 7)] =
              (unsigned char)(bv[e >> 2] >> (8 * (e & 3)));
        }
    }
    // scales: lanes 0 to 7 of a group K's of row e, lanes 8 to 15 V's
    {
      const int e = lane & 7, g = pair / 16;
      const int s = slot_at(row0 + e);
      if (s >= 0) {
        const int t = s & (block - 1);
        const bool isk = (lane & 8) == 0;
        const unsigned w = isk ? (e < 4 ? sk[0] : sk[1]) : (e < 4 ? sv[0] : sv[1]);
        const int off = isk ? codes + t * (D / 32) + g
                            : 2 * codes + scales + ((t >> 3) * (D / 32) + g) * 8 + (t & 7);
        place(s)[off] = (unsigned char)(w >> (8 * (e & 3)));
      }
    }
  }
}

// ---------------------------------------------------------------- load

template <int SEL>
__device__ inline unsigned value_pair(unsigned codes, unsigned scale) {
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, __uint_as_float(scale << 23), SEL));
}

// A thread reads eight channels of eight consecutive tokens (an octet of V, as
// it lies; eight rows of K) and writes 16 bytes of each token: 16 (8) lanes
// cover a token's row, consecutive octets follow.
template <int D>
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
      *reinterpret_cast<uint4 *>(kp + e * ksn) = make_uint4(value_pair<0>(kw[e], ks[e]), value_pair<1>(kw[e], ks[e]),
                                                            value_pair<2>(kw[e], ks[e]), value_pair<3>(kw[e], ks[e]));
    }
    auto v_row = [&](auto sel, int e, unsigned p0, unsigned p1, unsigned p2, unsigned p3, unsigned sw) {
      constexpr int S = decltype(sel)::value;
      if (e >= valid) return;
      const unsigned sc = (sw >> (8 * S)) & 255u;
      *reinterpret_cast<uint4 *>(vp + e * vsn) =
          make_uint4(value_pair<S>(p0, sc), value_pair<S>(p1, sc), value_pair<S>(p2, sc), value_pair<S>(p3, sc));
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
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&plan_kernel),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (kMaxPlanBatch * 2 + 1) * 4);
  if (e != hipSuccess) return e;
  const int64_t need = ((int64_t)n_slots + kPlanThreads * kPlanSlots - 1) / (kPlanThreads * kPlanSlots);
  const unsigned grid = (unsigned)(need < 1 ? 1 : need > 512 ? 512 : need);
  hipLaunchKernelGGL(plan_kernel, dim3(grid), dim3(kPlanThreads), lds, s, kv_len, new_len, batch, table, width,
                     free_pages, n_free, shift, q_start, kv_len_out, slots, positions, n_slots, counts);
  return hipGetLastError();
}

hipError_t launch_kv4_store(Kv4 c, Rows k, Rows v, int n_rows, const int32_t *slots, hipStream_t s) {
  const int64_t items = ((int64_t)n_rows + 7) / 8 * c.heads * (c.d / 2);
  const int64_t need = (items + 255) / 256;
  const dim3 grid((unsigned)(need < kMaxGrid ? need : kMaxGrid));
  if (c.d == 128) hipLaunchKernelGGL(store_kernel<128>, grid, dim3(256), 0, s, c, k, v, n_rows, slots, items);
  else hipLaunchKernelGGL(store_kernel<64>, grid, dim3(256), 0, s, c, k, v, n_rows, slots, items);
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
  if (c.d == 128)
    hipLaunchKernelGGL(load_kernel<128>, grid, dim3(256), 0, s, c, table, batch, width, kv_len, n, ko, ksb, ksh, ksn,
                       vo, vsb, vsh, vsn, (int)per, groups);
  else
    hipLaunchKernelGGL(load_kernel<64>, grid, dim3(256), 0, s, c, table, batch, width, kv_len, n, ko, ksb, ksh, ksn,
                       vo, vsb, vsh, vsn, (int)per, groups);
  return hipGetLastError();
}

}  // namespace carnator
