// Rows of keys and values into the 8-bit committed cache: e4m3 codes with one
// power-of-two scale per page and head, for the keys and for the values.
//
// Row x of a page becomes the codes of x * 2^-k, rounded to nearest even, with
// 2^k the smallest power of two that brings the page's largest entry to 448 (the
// largest e4m3 value) or below.  A power of two, because e4m3 is a floating
// format: another scale would gain no precision, and a scale that grows with
// later rows changes earlier codes only where they fall below its normal range.
// Memory-bound: 6 bytes per entry of a row.  One wavefront per page, layer, head
// and kind, so that the largest entry never leaves it.
#include "co_kernels.h"

namespace co {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kStoreWaves = 4;        // wavefronts per workgroup
constexpr int kStoreFill = 2048;      // wavefronts (of two kinds) that fill the chip

// 2^-(b - 127), exactly.
__device__ __forceinline__ float unscale(int b) {
  return __uint_as_float(static_cast<uint32_t>(254 - b) << 23);
}

// Two codes in the low or high half of w; what is not finite becomes NaN.
template <bool HI>
__device__ __forceinline__ uint32_t code2(float x, float y, uint32_t w) {
  return static_cast<uint32_t>(
      __builtin_amdgcn_cvt_pk_fp8_f32(x, y, static_cast<int>(w), HI));
}

// Four codes as they read under a scale 2^-d times as fine.
__device__ __forceinline__ uint32_t recode4(uint32_t w, float f) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
  const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
  return code2<true>(b[0] * f, b[1] * f, code2<false>(a[0] * f, a[1] * f, 0));
}

__device__ __forceinline__ float lo_f(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float hi_f(uint32_t p) { return __uint_as_float(p & 0xFFFF0000u); }

// Keys of one page: rows r .. r + n - 1 of head `row0` into slots t0 .. t0 + n - 1
// of the page at `page` ([16][HD] codes).  A lane takes 8 dims of every
// RPI-th slot: whole rows are read and written.
template <int HD>
__device__ void store_keys(const uint16_t* rows, int64_t row_stride, int t0, int n, uint8_t* page,
                           uint8_t* scale, int lane) {
  constexpr int LPR = HD / 8, RPI = 64 / LPR, NI = kPage / RPI;   // lanes per row, rows at once
  const int rr = lane / LPR, d = (lane % LPR) * 8;
  u32x4 x[NI];
  u32x2 old[NI];
  uint32_t top = 0;
  const int before = t0 > 0 ? *scale : 0;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int j = i * RPI + rr - t0;
    x[i] = u32x4{0, 0, 0, 0};
    old[i] = u32x2{0, 0};
    if (j >= 0 && j < n) x[i] = *reinterpret_cast<const u32x4*>(rows + j * row_stride + d);
    else if (t0 > 0) old[i] = *reinterpret_cast<const u32x2*>(page + (i * RPI + rr) * HD + d);
  }
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = finite_max_bf16(top, x[i][e]);
  const int b = max(before, scale_byte_e4m3(static_cast<uint32_t>(wave_max(top)) << 16));
  const float f = unscale(b);
  const bool finer = t0 > 0 && b > before;
  const float g = finer ? __uint_as_float(static_cast<uint32_t>(max(0, 127 + before - b)) << 23) : 0.f;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int t = i * RPI + rr, j = t - t0;
    u32x2* to = reinterpret_cast<u32x2*>(page + t * HD + d);
    if (j >= 0 && j < n) {
      u32x2 w;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        w[e] = code2<true>(lo_f(x[i][2 * e + 1]) * f, hi_f(x[i][2 * e + 1]) * f,
                           code2<false>(lo_f(x[i][2 * e]) * f, hi_f(x[i][2 * e]) * f, 0));
      *to = w;
    } else if (t0 == 0) {
      *to = u32x2{0, 0};
    } else if (finer) {
      *to = u32x2{recode4(old[i][0], g), recode4(old[i][1], g)};
    }
  }
  if (lane == 0) *scale = static_cast<uint8_t>(b);
}

// Values of one page ([HD][16] codes): a lane takes HD / 64 dims of all slots, so
// that the page's other order costs nothing but 2- or 4-byte reads of the rows.
template <int HD>
__device__ void store_values(const uint16_t* rows, int64_t row_stride, int t0, int n, uint8_t* page,
                             uint8_t* scale, int lane) {
  constexpr int ND = HD / 64;   // dims per lane
  uint32_t x[kPage];
  u32x4 old[ND];
  uint32_t top = 0;
  const int before = t0 > 0 ? *scale : 0;
#pragma unroll
  for (int t = 0; t < kPage; ++t) {
    const int j = t - t0;   // uniform
    x[t] = 0;
    if (j >= 0 && j < n) {
      if constexpr (ND == 2) x[t] = *reinterpret_cast<const uint32_t*>(rows + j * row_stride + 2 * lane);
      else x[t] = rows[j * row_stride + lane];
    }
  }
  u32x4* to = reinterpret_cast<u32x4*>(page) + ND * lane;
#pragma unroll
  for (int d = 0; d < ND; ++d) old[d] = t0 > 0 ? to[d] : u32x4{0, 0, 0, 0};
#pragma unroll
  for (int t = 0; t < kPage; ++t) top = finite_max_bf16(top, x[t]);
  const int b = max(before, scale_byte_e4m3(static_cast<uint32_t>(wave_max(top)) << 16));
  const float f = unscale(b);
  const bool finer = t0 > 0 && b > before;
  const float g = finer ? __uint_as_float(static_cast<uint32_t>(max(0, 127 + before - b)) << 23) : 0.f;
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    u32x4 w;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float v[4];
      uint32_t take = 0;   // bytes that rows go to
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = 4 * q + e;
        v[e] = (d == 0 ? lo_f(x[t]) : hi_f(x[t])) * f;
        if (t >= t0 && t < t0 + n) take |= 0xFFu << (8 * e);
      }
      const uint32_t c = code2<true>(v[2], v[3], code2<false>(v[0], v[1], 0));
      const uint32_t keep = finer ? recode4(old[d][q], g) : old[d][q];
      w[q] = (c & take) | (keep & ~take);
    }
    to[d] = w;
  }
  if (lane == 0) *scale = static_cast<uint8_t>(b);
}

// Wavefront (group, kind): the pages whose first row lies in rows group * per ..
// + per - 1, keys (kind 0) or values, of (layer, head) blockIdx.y.
template <int HD>
__global__ __launch_bounds__(64 * kStoreWaves) void store_kv8_kernel(StoreArgs a, int per) {
  const int lane = threadIdx.x & 63;
  const int unit = blockIdx.x * kStoreWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kind = unit & 1, r0 = (unit >> 1) * per;
  if (r0 >= a.M) return;
  const int layer = blockIdx.y / a.Hkv, g = blockIdx.y % a.Hkv;
  // A page's rows are consecutive with consecutive slots; its first one is where
  // that run begins.
  const int rl = r0 + lane;
  int32_t d = -1, prev = -1;
  if (lane < per && rl < a.M) {
    d = a.row_dst[rl];
    prev = rl > 0 ? a.row_dst[rl - 1] : -1;
  }
  const bool inside = d >= 0 && d / kPage < a.num_pages;
  if (d >= 0 && !inside && blockIdx.y == 0 && kind == 0) set_status(a.status, CO_ERR_PAGE_RANGE);
  uint64_t firsts = __ballot(inside && (d % kPage == 0 || prev != d - 1));
  const int64_t row_stride = static_cast<int64_t>(a.Hkv) * HD;
  const uint16_t* src = static_cast<const uint16_t*>(kind ? a.v_rows : a.k_rows) +
                        static_cast<int64_t>(layer) * a.M * row_stride + g * HD;
  uint8_t* pages = static_cast<uint8_t*>(kind ? a.v_pages : a.k_pages);
  uint8_t* scales = kind ? a.v_scale : a.k_scale;
  while (firsts) {
    const int l = __ffsll(static_cast<long long>(firsts)) - 1;
    firsts &= firsts - 1;
    const int r = r0 + l, d0 = __builtin_amdgcn_readlane(d, l), t0 = d0 % kPage;
    const bool same = lane < kPage - t0 && r + lane < a.M && a.row_dst[r + lane] == d0 + lane;
    const int n = __ffsll(static_cast<long long>(~__ballot(same))) - 1;
    const int64_t at = (static_cast<int64_t>(layer) * a.num_pages + d0 / kPage) * a.Hkv + g;
    const uint16_t* rows = src + r * row_stride;
    if (kind == 0) store_keys<HD>(rows, row_stride, t0, n, pages + at * (kPage * HD), scales + at, lane);
    else store_values<HD>(rows, row_stride, t0, n, pages + at * (kPage * HD), scales + at, lane);
  }
}

}  // namespace

hipError_t launch_store_kv8(const StoreArgs& a, hipStream_t stream) {
  if (a.M == 0) return hipSuccess;
  // Rows per wavefront: as many as leave kStoreFill wavefronts, up to a page's sixteen.
  // Few rows in flight are latency (pages one after the other in a wavefront), many
  // wavefronts that find no page's first row are not free: 16252 rows of prompts, 5
  // layers of 8 heads of 128: 206 us at 1, 137 at 4, 94 at 16 (5.3 TB/s); windows of 32
  // sequences with 3 of 16 rows committed 17, 10 and 6.4 us.
  int per = 1;
  while (per < kPage && static_cast<int64_t>(a.M) * a.L * a.Hkv / per >= kStoreFill) per *= 2;
  const int64_t units = 2 * ((static_cast<int64_t>(a.M) + per - 1) / per);
  const dim3 grid(static_cast<uint32_t>((units + kStoreWaves - 1) / kStoreWaves), a.L * a.Hkv);
  if (a.hd == 64) hipLaunchKernelGGL(store_kv8_kernel<64>, grid, dim3(64 * kStoreWaves), 0, stream, a, per);
  else hipLaunchKernelGGL(store_kv8_kernel<128>, grid, dim3(64 * kStoreWaves), 0, stream, a, per);
  return hipGetLastError();
}

}  // namespace co
