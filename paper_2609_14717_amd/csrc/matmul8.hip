// Products of 8-bit integers with a scale for each row of both operands, and the rows'
// quantisation.
//
//   code[i][k] = rint(127 x[i][k] / a_i), a_i = max_k |x[i][k]|, scale_i = a_i / 127
//   out[i][j]  = float(sum_k a[i][k] w[j][k]) (a_scale[i] w_scale[j]) + bias[j]
//
// Sums are exact: int32, for k up to 131008.
#include "co_store.h"

namespace co {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

constexpr float kLeast = 0x1.fcp-120f;   // 127 * 2^-126: smallest magnitude that scales a row

// -------------------------------------------------------------- quantisation

// One code: 127 x / a to the nearest integer, ties to even (the fp64 quotient's rounding
// cannot reach a middle of two integers that the exact quotient, of two 24-bit numbers, does
// not lie on).
__device__ __forceinline__ int code_of(float x, float a) {
  return static_cast<int>(rint(static_cast<double>(x) * 127.0 / static_cast<double>(a)));
}

// Largest of the workgroup's values, in every thread.
template <int NT>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* red) {
  v = static_cast<uint32_t>(wave_max(static_cast<int>(v)));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = max(v, red[w]);
  return v;
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Eight elements as fp32.
__device__ __forceinline__ void eight(const uint16_t* p, float (&x)[8]) {
  const u16x8 v = *reinterpret_cast<const u16x8*>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = bf2f(v[e]);
}
__device__ __forceinline__ void eight(const float* p, float (&x)[8]) {
  const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = lo[e];
    x[4 + e] = hi[e];
  }
}

// The scale of a row and what its entries are multiplied by; bad: not finite.
struct RowScale {
  float a, r, scale;
  bool bad;
  __device__ __forceinline__ explicit RowScale(uint32_t top) {
    bad = top >= 0x7F800000u;
    a = fmaxf(__uint_as_float(bad ? 0u : top), kLeast);
    r = 127.f / a;
    scale = bad ? NAN : a / 127.f;
  }
  // x r, r = 127 / a, is off from the quotient by up to 2^-16 (127 times two roundings): added
  // to 1.5 * 2^23 it leaves the nearest integer in the sum's low bits.  Where one of the eight
  // comes within 2^-14 of a middle, the quotients decide.
  __device__ __forceinline__ void codes(const float (&x)[8], int8_t* out) const {
    constexpr float kMagic = 12582912.f;
    uint32_t w[2], n[8];
    float far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = fmaf(x[e], r, kMagic);
      far = fmaxf(far, fabsf(fmaf(x[e], r, kMagic - t)));
      n[e] = __float_as_uint(t);
    }
    if (far > 0.5f - 0x1p-14f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) n[e] = static_cast<uint32_t>(code_of(x[e], a));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // the low bytes of four words: pairs, then both pairs
      const uint32_t lo = __builtin_amdgcn_perm(n[4 * h + 1], n[4 * h], 0x0C0C0400u);
      const uint32_t hi = __builtin_amdgcn_perm(n[4 * h + 3], n[4 * h + 2], 0x0C0C0400u);
      w[h] = bad ? 0u : (lo | hi << 16);
    }
    *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
  }
};

// One workgroup per row, which it holds in registers (Q times eight entries a thread) from
// the search for its largest magnitude to its codes; Q = 0: rows of any length, read twice
// (their columns are counted without a sign: the step behind the last may pass 2^31).
// Magnitudes compare as their bits, infinities and NaNs as the largest.  Memory traffic bounds
// it in the limit; at the sizes of a round its three steps one behind the other do: 512 bf16
// rows of 20480 13.6 us (2.3 TB/s), 544 of 4096 5.4, one of 768 2.4 (here and at the other
// kernels: averages under the profiler, where no other kind is named).
template <typename T, int NT, int Q>
__global__ __launch_bounds__(NT) void quantize_rows_kernel(const T* x, int cols, int8_t* codes,
                                                           float* scale) {
  __shared__ uint32_t red[NT / 64];
  const int64_t row = blockIdx.x;
  const T* xr = x + row * cols;
  int8_t* cr = codes + row * cols;
  uint32_t top = 0;
  if constexpr (Q > 0) {
    float v[Q][8];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = (q * NT + threadIdx.x) * 8;
      if (c < cols) eight(xr + c, v[q]);
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if ((q * NT + threadIdx.x) * 8 < cols)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[q][e]));
    const RowScale s(block_max<NT>(top, red));
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = (q * NT + threadIdx.x) * 8;
      if (c < cols) s.codes(v[q], cr + c);
    }
    if (threadIdx.x == 0) scale[row] = s.scale;
  } else {
    const uint32_t end = cols;
    float v[8];
    for (uint32_t c = threadIdx.x * 8; c < end; c += NT * 8) {
      eight(xr + c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[e]));
    }
    const RowScale s(block_max<NT>(top, red));
    for (uint32_t c = threadIdx.x * 8; c < end; c += NT * 8) {
      eight(xr + c, v);
      s.codes(v, cr + c);
    }
    if (threadIdx.x == 0) scale[row] = s.scale;
  }
}

template <typename T>
void launch_quantize_t(const T* x, int64_t rows, int cols, int8_t* codes, float* scale, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(rows));
  auto launch = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, x, cols, codes, scale);
  };
  // as many threads as hold a row
  if (cols <= 2048) launch(quantize_rows_kernel<T, 256, 1>, 256);
  else if (cols <= 8192) launch(quantize_rows_kernel<T, 512, 2>, 512);
  else if (cols <= 32768) launch(quantize_rows_kernel<T, 1024, 4>, 1024);
  else launch(quantize_rows_kernel<T, 1024, 0>, 1024);
}

// ------------------------------------------------------------------- product

__device__ __forceinline__ i32x16 mfma_i8(i32x4 a, i32x4 b, i32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

__device__ __forceinline__ i32x4 mfma_i8(i32x4 a, i32x4 b, i32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

// One result; the operations are rounded one by one.
__device__ __forceinline__ float scaled(int sum, float sa, float sw) {
#pragma clang fp contract(off)
  return static_cast<float>(sum) * (sa * sw);
}

__device__ __forceinline__ float scaled(int sum, float sa, float sw, float bias) {
#pragma clang fp contract(off)
  const float v = static_cast<float>(sum) * (sa * sw);
  return v + bias;
}

template <typename T> __device__ __forceinline__ void put(T* p, float v);
template <> __device__ __forceinline__ void put<float>(float* p, float v) { *p = v; }
template <> __device__ __forceinline__ void put<uint16_t>(uint16_t* p, float v) {
  *p = static_cast<uint16_t>(cvt_pk_bf16(v, v));
}

// Workgroups are dealt to the eight XCDs in turn: renumbered, each XCD gets a run of
// consecutive indices, whose shared panels then stay in its L2.
__device__ __forceinline__ int xcd_run(int t, int total) {
  const int q = total >> 3, r = total & 7, x = t & 7;
  return x * q + min(x, r) + (t >> 3);
}

// Where results go: plain rows, or (X = KvDest) the K/V rows of the projection.  Each C
// columns of a tile are then C / 2 rotation pairs of a head: their low halves, then their high
// ones, so that whoever has a tile's row has both of a pair.
struct PlainRows {};

template <int C, typename X>
__device__ __forceinline__ int column(const X& x, int n0, int c) {
  if constexpr (sizeof(X) > 1) {
    const int t = c & -C, j = c & (C - 1);
    return n0 + t / x.hd * x.hd + t % x.hd / 2 + j % (C / 2) + j / (C / 2) * (x.hd / 2);
  }
  return n0 + c;
}

// Few rows (16 MT of them): bound by reading the weights once.  A workgroup's NW
// wavefronts share 16 TN columns and split K: a wavefront takes every NW-th unit of 256
// bytes of K, straight into the operand registers of v_mfma_i32_16x16x64_i8 (lane l holds
// row or column l % 16, 16 k from 16 (l / 16) on; result register r is row 4 (l / 16) + r,
// column l % 16), the next unit's loads in flight while one is multiplied.  The NW partial
// tiles are added in LDS: whole numbers, so the order does not matter.  One launch, so the
// kernel of the smallest products: 1 x 256 x 768 2.8 us, 16 x 2048 x 4096 6.2 (its K/V rows
// rotated and stored 7.8: with 16 wavefronts, which have 128 registers a lane, that form keeps
// 100 bytes a lane in scratch).
constexpr int kUnit = 256;

template <int MT, int TN, int NW, typename T, typename X>
__global__ __launch_bounds__(64 * NW) void matmul_i8_few_kernel(MatmulI8Args g, X x) {
  __shared__ __align__(16) int red[NW][MT * TN * 256];
  __shared__ double inv_tab[sizeof(X) > 1 ? 64 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n0 = static_cast<int>(blockIdx.x) * 16 * TN;
  const int quad = (lane >> 4) * 16;
  const int8_t* pa[MT];
  const int8_t* pw[TN];
#pragma unroll
  for (int i = 0; i < MT; ++i)
    pa[i] = g.A + static_cast<int64_t>(min(16 * i + (lane & 15), g.M - 1)) * g.K + quad;
#pragma unroll
  for (int j = 0; j < TN; ++j)
    pw[j] = g.W + static_cast<int64_t>(min(column<16>(x, 0, n0 + 16 * j + (lane & 15)), g.N - 1)) * g.K + quad;
  if constexpr (sizeof(X) > 1)
    if (tid < x.hd / 2) inv_tab[tid] = rope_table<uint16_t>(x, tid);
  i32x4 acc[MT][TN] = {};
  struct Unit {
    i32x4 a[4][MT], w[4][TN];
  };
  const int units = g.K / kUnit;
  auto load = [&](int u, Unit& f) {
    const int64_t k = static_cast<int64_t>(u) * kUnit;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int j = 0; j < TN; ++j) f.w[t][j] = *reinterpret_cast<const i32x4*>(pw[j] + k + 64 * t);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int i = 0; i < MT; ++i) f.a[t][i] = *reinterpret_cast<const i32x4*>(pa[i] + k + 64 * t);
    }
  };
  auto compute = [&](const Unit& f) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma_i8(f.a[t][i], f.w[t][j], acc[i][j]);
  };
  Unit f0, f1;
  int u = wave;
  if (u < units) load(u, f0);
  while (u < units) {
    if (u + NW < units) load(u + NW, f1);
    compute(f0);
    u += NW;
    if (u >= units) break;
    if (u + NW < units) load(u + NW, f0);
    compute(f1);
    u += NW;
  }
  for (int k = units * kUnit + 64 * wave; k < g.K; k += 64 * NW) {   // up to three steps of 64
    i32x4 w[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) w[j] = *reinterpret_cast<const i32x4*>(pw[j] + k);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const i32x4 a = *reinterpret_cast<const i32x4*>(pa[i] + k);
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = mfma_i8(a, w[j], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        red[wave][(16 * i + 4 * (lane >> 4) + r) * (16 * TN) + 16 * j + (lane & 15)] = acc[i][j][r];
  __syncthreads();
  if constexpr (sizeof(X) > 1) {
    // four pairs a thread, rows side by side (a value page has a dim's tokens next to each other)
    for (int o = tid; o < MT * TN * 32; o += 64 * NW) {
      const int row = o % (16 * MT), h = o / (16 * MT) % 2, j = o / (32 * MT);
      const int32_t dst = row < g.M && n0 + 16 * j < g.N ? x.row_dst[row] : kSkip;
      if (dst == kSkip) continue;
      const int at = row * (16 * TN) + 16 * j + 4 * h, col = column<16>(x, 0, n0 + 16 * j + 4 * h);
      i32x4 a = {}, b = {};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        a += *reinterpret_cast<const i32x4*>(&red[w][at]);
        b += *reinterpret_cast<const i32x4*>(&red[w][at + 8]);
      }
      const float sa = g.a_scale[row];
      float lo[4], hi[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = scaled(a[i], sa, g.w_scale[col + i]);
        hi[i] = scaled(b[i], sa, g.w_scale[col + x.hd / 2 + i]);
      }
      kv_store<uint16_t, 4>(x, row, dst, x.row_pos[row], col / x.hd, col % x.hd, lo, hi, inv_tab);
    }
    return;
  }
  for (int o = tid; o < MT * TN * 256; o += 64 * NW) {
    const int row = o / (16 * TN), col = n0 + o % (16 * TN);
    if (row >= g.M || col >= g.N) continue;
    int sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum += red[w][o];
    const float sa = g.a_scale[row], sw = g.w_scale[col];
    put(static_cast<T*>(g.out) + static_cast<int64_t>(row) * g.N + col,
        g.bias ? scaled(sum, sa, sw, g.bias[col]) : scaled(sum, sa, sw));
  }
}

// Columns col .. col + C - 1 of a row that starts anywhere, those below N.
template <int C, typename E, typename V>
__device__ __forceinline__ void put_cols(E* row, int col, int N, const V& v) {
  typedef E out_t __attribute__((ext_vector_type(C), aligned(sizeof(E))));
  if (col + C <= N) {
    *reinterpret_cast<out_t*>(row + col) = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < C; ++i)
    if (col + i < N) row[col + i] = v[i];
}

// Few rows through LDS: a workgroup's four wavefronts take 16 columns each and share 16 MT
// rows; K advances in stages of 256 bytes a row (long runs of memory) through a ring of NS,
// and is split over workgroups until the chip is full.  The weights are the first operand: a
// lane ends with row l % 16 and four columns from 4 (l / 16) on.  17 x 128000 x 4096 104-107 us:
// 5.0 TB/s of weights, a large copy's rate (reads alone reach 5.7-5.9); the same by registers,
// each wavefront reading 256-byte pieces of 16 rows, 127.  16 x 4096 x 20480, parts left to the
// reader, 14.7 us.
template <int MT, int NS, typename T>
__global__ __launch_bounds__(256) void matmul_i8_stream_kernel(MatmulI8Args g, int tiles_n, int k_per_split) {
  constexpr int ROWS = 64 + 16 * MT, STAGE = ROWS * kUnit;
  constexpr int LPW = ROWS / 16;                 // 1 KiB loads (four rows) of a wavefront, a stage
  static_assert(LPW * (NS - 1) < 64 && NS >= 2 && NS <= 4, "vmcnt");
  __shared__ __align__(16) unsigned char smem[NS * STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = static_cast<int>(blockIdx.x % tiles_n) * 64, sp = blockIdx.x / tiles_n;
  const int kbeg = sp * k_per_split, klen = min(g.K - kbeg, k_per_split);
  const int nk = (klen + kUnit - 1) / kUnit;
  const int8_t* src[LPW];
  int chunk[LPW];
#pragma unroll
  for (int j = 0; j < LPW; ++j) {
    const int row = (LPW * wave + j) * 4 + (lane >> 4);
    chunk[j] = ((lane & 15) ^ (row & 15)) * 16;
    src[j] = (row < 64 ? g.W + static_cast<int64_t>(min(n0 + row, g.N - 1)) * g.K
                       : g.A + static_cast<int64_t>(min(row - 64, g.M - 1)) * g.K) + kbeg;
  }
  const uint32_t ring = lds_addr(smem);
  auto issue = [&](int kt) {
    const uint32_t st = ring + (kt % NS) * STAGE + LPW * wave * 1024;
    const int left = klen - kt * kUnit;
    if (left >= kUnit) {
#pragma unroll
      for (int j = 0; j < LPW; ++j) lds_dma16_opaque(src[j] + kt * kUnit + chunk[j], st + j * 1024);
    } else {   // chunks past the end are not read: they take the first
#pragma unroll
      for (int j = 0; j < LPW; ++j)
        lds_dma16_opaque(src[j] + kt * kUnit + (chunk[j] < left ? chunk[j] : 0), st + j * 1024);
    }
  };
  auto wait_stage = [&](int ahead) {
    if (NS >= 4 && ahead >= 3) wait_vm_lgkm_barrier<(NS >= 4 ? 3 * LPW : 0)>();
    else if (NS >= 3 && ahead >= 2) wait_vm_lgkm_barrier<(NS >= 3 ? 2 * LPW : 0)>();
    else if (ahead >= 1) wait_vm_lgkm_barrier<LPW>();
    else wait_vm_lgkm_barrier<0>();
  };
  i32x4 acc[MT] = {};
  auto step = [&](const unsigned char* st, int h) {
    const int off = (lane & 15) * kUnit + (((4 * h + (lane >> 4)) ^ (lane & 15)) << 4);
    const i32x4 w = *reinterpret_cast<const i32x4*>(st + 16 * wave * kUnit + off);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const i32x4 a = *reinterpret_cast<const i32x4*>(st + (64 + 16 * i) * kUnit + off);
      acc[i] = mfma_i8(w, a, acc[i]);
    }
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < nk) issue(s);
  for (int kt = 0; kt < nk; ++kt) {
    wait_stage(min(NS - 2, nk - 1 - kt));
    // (every wavefront is done with stage kt - 1: its slot takes stage kt + NS - 1)
    if (kt + NS - 1 < nk) issue(kt + NS - 1);
    const unsigned char* st = smem + (kt % NS) * STAGE;
    const int steps = min(klen - kt * kUnit, kUnit) / 64;
    if (steps == 4) {
#pragma unroll
      for (int h = 0; h < 4; ++h) step(st, h);
    } else {
      for (int h = 0; h < steps; ++h) step(st, h);
    }
  }
  const int col = n0 + 16 * wave + 4 * (lane >> 4);
  const bool parts = gridDim.x > static_cast<unsigned>(tiles_n);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int row = 16 * i + (lane & 15);
    if (row >= g.M) continue;
    if (parts) {
      put_cols<4>(static_cast<int*>(g.ws) + (static_cast<int64_t>(sp) * g.M + row) * g.N, col, g.N, acc[i]);
      continue;
    }
    const float sa = g.a_scale[row];
    T* out = static_cast<T*>(g.out) + static_cast<int64_t>(row) * g.N;
    f32x4 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = min(col + q, g.N - 1);
      v[q] = g.bias ? scaled(acc[i][q], sa, g.w_scale[c], g.bias[c]) : scaled(acc[i][q], sa, g.w_scale[c]);
    }
    if constexpr (sizeof(T) == 4) {
      put_cols<4>(out, col, g.N, v);
    } else {
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      const u32x2 w = {cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
      put_cols<4>(out, col, g.N, __builtin_bit_cast(u16x4, w));
    }
  }
}

// Its parts of K, rows by rows, added up and scaled.
template <typename T>
__global__ __launch_bounds__(256) void sum_rows_i8_kernel(MatmulI8Args g, int splits) {
  const int64_t n = static_cast<int64_t>(g.M) * g.N;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= n) return;
  const int* part = static_cast<const int*>(g.ws);
  int sum = 0;
  for (int s = 0; s < splits; ++s) sum += part[s * n + i];
  const int row = static_cast<int>(i / g.N), col = static_cast<int>(i % g.N);
  const float sa = g.a_scale[row], sw = g.w_scale[col];
  put(static_cast<T*>(g.out) + i, g.bias ? scaled(sum, sa, sw, g.bias[col]) : scaled(sum, sa, sw));
}

// Many rows: a tile of BM x BN outputs, eight wavefronts (2 x 4) of TMW x TNW tiles of
// v_mfma_i32_32x32x32_i8 (lane l holds row or column l % 32, 16 k from 16 (l / 32) on).
// The weights are its first operand, so that a lane ends with one output row, l % 32, and
// in registers 4 q .. 4 q + 3 four columns next to each other, from 8 q + 4 (l / 32) on,
// which go to memory from the registers.  K advances in
// stages of 128 bytes (whole cache lines: stages of 64 fetch every line twice) through a
// ring of NS in LDS, filled by direct-to-LDS loads that the compiler does not see: a
// wavefront waits for its own with an exact count and a barrier publishes a stage.  The
// 16-byte chunks of a staged row are permuted by row / 2, so that 16 lanes reading a
// fragment hit 16 bank groups.  Fragments of a step of 32 k are read while the step before
// multiplies.
// Bound by the matrix instructions and the LDS reads that feed them.  8192^3 486 us, 2.26 POP/s;
// 544 x 128000 x 4096, bf16 results, 337 us, 1.69 POP/s: three row tiles of 192 hold 544 (6 %),
// and the 139 MB of results leave no time of their own, for one workgroup fills a compute unit;
// 512 x 4096 x 20480 in four parts 56 + 9; 512 x 10240 x 4096 34, with rotation and stores of
// K/V rows 42.  The first by calls one behind the other, as the following: the library's 440 with
// int32 results, this kernel's with fp32 results 512; the second 332, with fp32 results 360, the
// library's 388; stages of 64 bytes 469, results by way of LDS 421.
constexpr int kStageK = 128;

// A wavefront's 32 x 32 results: scaled, the bias added, stored.
template <typename T>
__device__ __forceinline__ void put_tile(const MatmulI8Args& g, const i32x16& acc, int row, float sa,
                                         int n0, int lane, const float* col_scale, const float* col_bias) {
#pragma clang fp contract(off)
  f32x4 v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = 8 * q + 4 * (lane >> 5);
    const f32x4 sw = *reinterpret_cast<const f32x4*>(col_scale + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[q][i] = scaled(acc[4 * q + i], sa, sw[i]);
    if (g.bias) {
      const f32x4 bv = *reinterpret_cast<const f32x4*>(col_bias + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[q][i] = v[q][i] + bv[i];
    }
  }
  T* out = static_cast<T*>(g.out) + static_cast<int64_t>(row) * g.N;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (row < g.M) put_cols<4>(out, n0 + 8 * q + 4 * (lane >> 5), g.N, v[q]);
  } else {
    // lanes l and l ^ 32 hold every other four columns of a row: exchanged, each has eight
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      const auto lo = __builtin_amdgcn_permlane32_swap(cvt_pk_bf16(v[q][0], v[q][1]),
                                                       cvt_pk_bf16(v[q + 1][0], v[q + 1][1]), false, false);
      const auto hi = __builtin_amdgcn_permlane32_swap(cvt_pk_bf16(v[q][2], v[q][3]),
                                                       cvt_pk_bf16(v[q + 1][2], v[q + 1][3]), false, false);
      const u32x4 w = {static_cast<uint32_t>(lo[0]), static_cast<uint32_t>(hi[0]),
                       static_cast<uint32_t>(lo[1]), static_cast<uint32_t>(hi[1])};
      if (row < g.M) put_cols<8>(out, n0 + 8 * q + 8 * (lane >> 5), g.N, __builtin_bit_cast(u16x8, w));
    }
  }
}

// Tile r of a part of K: groups of up to four row tiles sweep the column tiles, so that
// consecutive indices share panels of both operands.
template <int BM, int BN>
__device__ __forceinline__ void tile_of(int r, int tiles_m, int tiles_n, int* m0, int* n0) {
  const int gm = min(4, tiles_m), grp = r / (gm * tiles_n);
  const int gsz = min(gm, tiles_m - grp * gm), rg = r % (gm * tiles_n);
  *m0 = (grp * gm + rg % gsz) * BM;
  *n0 = rg / gsz * BN;
}

// A wavefront's 32 x 32 results of the K/V product: scaled, rotated and stored.
__device__ __forceinline__ void put_pairs(const MatmulI8Args& g, const KvDest& e, const i32x16& acc, int row,
                                          float sa, int n0, int cb, int lane, const float* col_scale,
                                          const double* inv_tab) {
  const int seg = n0 / e.hd + cb / e.hd;
  if (row >= g.M || seg * e.hd >= g.N) return;
  const int32_t dst = e.row_dst[row];
  if (dst == kSkip) return;
  const int pos = e.row_pos[row];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int c = 8 * q + 4 * (lane >> 5);
    float lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = scaled(acc[4 * q + i], sa, col_scale[c + i]);
      hi[i] = scaled(acc[4 * q + 8 + i], sa, col_scale[c + 16 + i]);
    }
    kv_store<uint16_t, 4>(e, row, dst, pos, seg, cb % e.hd / 2 + c, lo, hi, inv_tab);
  }
}

template <int TMW, int TNW, int NS, typename T, typename X>
__global__ __launch_bounds__(512, 1) void matmul_i8_wide_kernel(MatmulI8Args g, X x, int tiles_m,
                                                                int tiles_n, int k_per_split) {
  constexpr int BM = 64 * TMW, BN = 128 * TNW, ROWS = BM + BN, STAGE = ROWS * kStageK;
  constexpr int LPW = ROWS / 64;                         // 1 KiB loads of a wavefront, a stage
  static_assert(LPW * (NS - 1) < 64 && NS >= 2 && NS <= 4, "vmcnt");
  static_assert(NS * STAGE + 8 * BN + 512 <= 160 * 1024, "LDS");
  __shared__ __align__(16) unsigned char smem[NS * STAGE];
  __shared__ __align__(16) float col_scale[BN], col_bias[BN];
  __shared__ double inv_tab[sizeof(X) > 1 ? 64 : 1];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int t = xcd_run(blockIdx.x, gridDim.x);   // parts of K one after the other
  const int per_split = tiles_m * tiles_n;
  const int sp = t / per_split;
  int m0, n0;
  tile_of<BM, BN>(t % per_split, tiles_m, tiles_n, &m0, &n0);
  const int kbeg = sp * k_per_split;
  const int klen = min(g.K - kbeg, k_per_split);
  const int nk = (klen + kStageK - 1) / kStageK;
  const bool half = (klen & 64) != 0;                    // the last stage is half a one

  // load j of the wavefront fills rows 8 (LPW wave + j) .. + 7
  const int8_t* src[LPW];
#pragma unroll
  for (int j = 0; j < LPW; ++j) {
    const int row = (LPW * wave + j) * 8 + lane / 8;
    const int chunk = (lane & 7) ^ ((row >> 1) & 7);
    const int8_t* base = row < BM ? g.A + static_cast<int64_t>(min(m0 + row, g.M - 1)) * g.K
                                  : g.W + static_cast<int64_t>(min(column<32>(x, n0, row - BM), g.N - 1)) * g.K;
    src[j] = base + kbeg + chunk * 16;
  }
  // chunks past a half stage are not read: they take the half before
  auto back = [&](int j) {
    const int row = (LPW * wave + j) * 8 + lane / 8;
    return (((lane & 7) ^ ((row >> 1) & 7)) & 4) << 4;
  };
  const uint32_t ring = lds_addr(smem);
  auto issue = [&](int kt) {
    const uint32_t st = ring + (kt % NS) * STAGE + LPW * wave * 1024;
    if (half && kt + 1 == nk) {
#pragma unroll
      for (int j = 0; j < LPW; ++j) lds_dma16_opaque(src[j] + kt * kStageK - back(j), st + j * 1024);
    } else {
#pragma unroll
      for (int j = 0; j < LPW; ++j) lds_dma16_opaque(src[j] + kt * kStageK, st + j * 1024);
    }
  };
  // Waits until the stage `ahead` stages before the newest one issued has landed.
  auto wait_stage = [&](int ahead) {
    if (NS >= 4 && ahead >= 3) wait_vm_lgkm_barrier<(NS >= 4 ? 3 * LPW : 0)>();
    else if (NS >= 3 && ahead >= 2) wait_vm_lgkm_barrier<(NS >= 3 ? 2 * LPW : 0)>();
    else if (ahead >= 1) wait_vm_lgkm_barrier<LPW>();
    else wait_vm_lgkm_barrier<0>();
  };

  i32x16 acc[TMW][TNW] = {};
  const int frow = (lane & 31) * kStageK;
  const int fswz = ((lane & 31) >> 1) & 7;
  struct Frags {
    i32x4 a[TMW], b[TNW];
  };
  auto load = [&](int kt, int h, Frags& f) {
    const unsigned char* st = smem + (kt % NS) * STAGE;
    const int off = frow + (((2 * h + (lane >> 5)) ^ fswz) << 4);
#pragma unroll
    for (int a = 0; a < TMW; ++a)
      f.a[a] = *reinterpret_cast<const i32x4*>(st + (wm * TMW + a) * 32 * kStageK + off);
#pragma unroll
    for (int b = 0; b < TNW; ++b)
      f.b[b] = *reinterpret_cast<const i32x4*>(st + (BM + (wn * TNW + b) * 32) * kStageK + off);
  };
  auto settle = [&](Frags& f) {   // the LDS reads are waited for here, not at the products
#pragma unroll
    for (int a = 0; a < TMW; ++a) asm volatile("" : "+v"(f.a[a]));
#pragma unroll
    for (int b = 0; b < TNW; ++b) asm volatile("" : "+v"(f.b[b]));
  };
  auto compute = [&](const Frags& f) {
#pragma unroll
    for (int a = 0; a < TMW; ++a)
#pragma unroll
      for (int b = 0; b < TNW; ++b) acc[a][b] = mfma_i8(f.b[b], f.a[a], acc[a][b]);
  };

  for (int c = tid; c < BN; c += 512) {   // (read behind the main loop's barriers)
    const int col = min(column<32>(x, n0, c), g.N - 1);
    col_scale[c] = g.w_scale[col];
    col_bias[c] = g.bias ? g.bias[col] : 0.f;
  }
  if constexpr (sizeof(X) > 1)
    if (tid < x.hd / 2) inv_tab[tid] = rope_table<uint16_t>(x, tid);
#pragma unroll
  for (int s = 0; s < NS; ++s)
    if (s < nk) issue(s);
  Frags f0, f1;
  wait_stage(min(NS - 1, nk - 1));
  load(0, 0, f0);
  const int whole = half ? nk - 1 : nk;
  for (int kt = 0; kt < whole; ++kt) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      Frags& cur = (h & 1) ? f1 : f0;
      Frags& nxt = (h & 1) ? f0 : f1;
      if (h < 3) load(kt, h + 1, nxt);
      __builtin_amdgcn_sched_barrier(0);
      compute(cur);
      __builtin_amdgcn_sched_barrier(0);
      if (h == 2) {
        // every wavefront holds the rest of stage kt: its slot takes stage kt + NS
        settle(nxt);
        if (kt + 1 < nk) {
          wait_stage(min(NS - 2, nk - 2 - kt));
          if (kt + NS < nk) issue(kt + NS);
          load(kt + 1, 0, cur);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  if (half) {
    load(nk - 1, 1, f1);
    compute(f0);
    compute(f1);
  }

  if (gridDim.x > static_cast<unsigned>(per_split)) {
    // a part of K: the sums to the workspace in the order of the registers, 16 bytes a lane
    i32x4* part = reinterpret_cast<i32x4*>(g.ws) + static_cast<int64_t>(t) * (BM * BN / 4) + tid;
#pragma unroll
    for (int a = 0; a < TMW; ++a)
#pragma unroll
      for (int b = 0; b < TNW; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          part[((a * TNW + b) * 4 + q) * 512] = i32x4{acc[a][b][4 * q], acc[a][b][4 * q + 1],
                                                      acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
    return;
  }
#pragma unroll
  for (int a = 0; a < TMW; ++a) {
    const int row = m0 + (wm * TMW + a) * 32 + (lane & 31);
    const float sa = row < g.M ? g.a_scale[row] : 0.f;
#pragma unroll
    for (int b = 0; b < TNW; ++b) {
      const int cb = (wn * TNW + b) * 32;
      if constexpr (sizeof(X) > 1)
        put_pairs(g, x, acc[a][b], row, sa, n0, cb, lane, col_scale + cb, inv_tab);
      else
        put_tile<T>(g, acc[a][b], row, sa, n0 + cb, lane, col_scale + cb, col_bias + cb);
    }
  }
}

// The parts of K of one 32 x 32 tile for each wavefront, added up, scaled and stored: memory
// traffic and a launch, 9 us for 512 x 4096 (the call with the product 60; parts by rows of the
// result 65).
template <int TMW, int TNW, typename T, typename X>
__global__ __launch_bounds__(512) void sum_parts_i8_kernel(MatmulI8Args g, X x, int tiles_m,
                                                           int tiles_n, int splits) {
  constexpr int BM = 64 * TMW, BN = 128 * TNW;
  __shared__ __align__(16) float col_scale[BN], col_bias[BN];
  __shared__ double inv_tab[sizeof(X) > 1 ? 64 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 2, wn = wave & 3;
  const int frag = blockIdx.x % (TMW * TNW), r0 = blockIdx.x / (TMW * TNW);
  int m0, n0;
  tile_of<BM, BN>(r0, tiles_m, tiles_n, &m0, &n0);
  for (int c = tid; c < BN; c += 512) {
    const int col = min(column<32>(x, n0, c), g.N - 1);
    col_scale[c] = g.w_scale[col];
    col_bias[c] = g.bias ? g.bias[col] : 0.f;
  }
  if constexpr (sizeof(X) > 1)
    if (tid < x.hd / 2) inv_tab[tid] = rope_table<uint16_t>(x, tid);
  const int64_t step = static_cast<int64_t>(tiles_m) * tiles_n * (BM * BN / 4);
  const i32x4* part = reinterpret_cast<const i32x4*>(g.ws) + static_cast<int64_t>(r0) * (BM * BN / 4) +
                      frag * 4 * 512 + tid;
  i32x4 sum[4] = {};
  for (int s = 0; s < splits; ++s) {
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] += part[s * step + q * 512];
  }
  __syncthreads();
  i32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = sum[r >> 2][r & 3];
  const int a = frag / TNW, b = frag % TNW;
  const int row = m0 + (wm * TMW + a) * 32 + (lane & 31);
  const int cb = (wn * TNW + b) * 32;
  const float sa = row < g.M ? g.a_scale[row] : 0.f;
  if constexpr (sizeof(X) > 1) put_pairs(g, x, acc, row, sa, n0, cb, lane, col_scale + cb, inv_tab);
  else put_tile<T>(g, acc, row, sa, n0 + cb, lane, col_scale + cb, col_bias + cb);
}

// Tile variants of the wide kernel; kFew: the kernel for few rows.
constexpr int kVariants = 8, kFew = kVariants, kStream = kVariants + 1;
constexpr int kBM[kVariants] = {256, 256, 128, 192, 128, 64, 64, 192};
constexpr int kBN[kVariants] = {256, 128, 256, 256, 128, 256, 128, 128};

template <int TMW, int TNW, int NS, typename T, typename X>
void launch_wide_t(const MatmulI8Args& g, const X& x, const MatmulI8Plan& p, hipStream_t stream) {
  const int tm = (g.M + 64 * TMW - 1) / (64 * TMW), tn = (g.N + 128 * TNW - 1) / (128 * TNW);
  hipLaunchKernelGGL((matmul_i8_wide_kernel<TMW, TNW, NS, T, X>), dim3(static_cast<unsigned>(p.workgroups)),
                     dim3(512), 0, stream, g, x, tm, tn, p.k_per_split);
  if (p.splits > 1)
    hipLaunchKernelGGL((sum_parts_i8_kernel<TMW, TNW, T, X>), dim3(static_cast<unsigned>(tm) * tn * TMW * TNW),
                       dim3(512), 0, stream, g, x, tm, tn, p.splits);
}

template <typename T, typename X>
hipError_t launch_wide(const MatmulI8Args& g, const X& x, const MatmulI8Plan& p, hipStream_t stream) {
  switch (p.variant) {
    case 0: launch_wide_t<4, 2, 2, T>(g, x, p, stream); break;
    case 1: launch_wide_t<4, 1, 3, T>(g, x, p, stream); break;
    case 2: launch_wide_t<2, 2, 3, T>(g, x, p, stream); break;
    case 3: launch_wide_t<3, 2, 2, T>(g, x, p, stream); break;
    case 4: launch_wide_t<2, 1, 4, T>(g, x, p, stream); break;
    case 5: launch_wide_t<1, 2, 3, T>(g, x, p, stream); break;
    case 6: launch_wide_t<1, 1, 4, T>(g, x, p, stream); break;
    default: launch_wide_t<3, 1, 3, T>(g, x, p, stream); break;
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_stream(const MatmulI8Args& g, const MatmulI8Plan& p, bool keep_parts, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(p.workgroups)), block(256);
  const int tn = (g.N + 63) / 64, k = p.k_per_split;
  if (g.M <= 16) hipLaunchKernelGGL((matmul_i8_stream_kernel<1, 4, T>), grid, block, 0, stream, g, tn, k);
  else if (g.M <= 32) hipLaunchKernelGGL((matmul_i8_stream_kernel<2, 3, T>), grid, block, 0, stream, g, tn, k);
  else hipLaunchKernelGGL((matmul_i8_stream_kernel<4, 2, T>), grid, block, 0, stream, g, tn, k);
  if (p.splits > 1 && !keep_parts) {
    const int64_t n = static_cast<int64_t>(g.M) * g.N;
    hipLaunchKernelGGL(sum_rows_i8_kernel<T>, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256),
                       0, stream, g, p.splits);
  }
  return hipGetLastError();
}

template <int MT, int TN, typename T, typename X>
hipError_t launch_few_nw(const MatmulI8Args& g, const X& x, const MatmulI8Plan& p, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(p.workgroups));
  if constexpr (TN == 1) {   // (32 columns: the plan has eight at most)
    if (p.waves == 16) {
      hipLaunchKernelGGL((matmul_i8_few_kernel<MT, TN, 16, T, X>), grid, dim3(1024), 0, stream, g, x);
      return hipGetLastError();
    }
  }
  if (p.waves == 8) hipLaunchKernelGGL((matmul_i8_few_kernel<MT, TN, 8, T, X>), grid, dim3(512), 0, stream, g, x);
  else hipLaunchKernelGGL((matmul_i8_few_kernel<MT, TN, 4, T, X>), grid, dim3(256), 0, stream, g, x);
  return hipGetLastError();
}

template <typename T, typename X>
hipError_t launch_few(const MatmulI8Args& g, const X& x, const MatmulI8Plan& p, hipStream_t stream) {
  if (g.M <= 16)
    return p.cols == 2 ? launch_few_nw<1, 2, T>(g, x, p, stream) : launch_few_nw<1, 1, T>(g, x, p, stream);
  return p.cols == 2 ? launch_few_nw<2, 2, T>(g, x, p, stream) : launch_few_nw<2, 1, T>(g, x, p, stream);
}

}  // namespace

hipError_t launch_quantize_i8(const void* x, int64_t rows, int cols, int dtype, int8_t* codes,
                              float* scale, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  if (dtype == CO_DTYPE_BF16) launch_quantize_t(static_cast<const uint16_t*>(x), rows, cols, codes, scale, stream);
  else launch_quantize_t(static_cast<const float*>(x), rows, cols, codes, scale, stream);
  return hipGetLastError();
}

constexpr int kFewRows = 32;

MatmulI8Plan plan_matmul_i8(int M, int N, int K, int num_cus) {
  MatmulI8Plan p{};
  p.splits = 1;
  p.k_per_split = K;
  const int64_t force = tuning(CO_TUNE_MATMUL_I8);
  if (M <= 64 && (force < 0 || force >= kFew)) {
    const int64_t tiles = (static_cast<int64_t>(N) + 63) / 64;
    int split = 1;
    while (tiles * split < 2 * num_cus && K / (split * 2) >= 2 * kUnit) split *= 2;
    // A split stream's parts are added up by a second launch; the registers' kernel has none,
    // but reads the rows' codes once for 16 columns.  us, by registers and by stream:
    // 16 x 2048 x 4096 6.9, 9.6; 16 x 10240 x 4096 14.7, 15.2; 12 x 4339 x 7680 16.2, 13.3;
    // 16 x 4096 x 20480 26.0, 22.6; 4 x 1218 x 16448 11.5, 15.0; 1 x 20 x 11584 7.7, 8.2;
    // 1 x 155 x 704 3.7, 4.8; unsplit 17 x 128000 x 4096 127, 104.  The stream against 64-row tiles: unsplit
    // 64 x 128000 x 4096 130, 113; split 64 x 4096 x 20480 25.6, 29.3; 39 x 468 x 3136 8.6, 10.2;
    // 60 x 20911 x 11264 70, 56.
    const bool few = force < 0 ? (split > 1 || tiles < num_cus) && static_cast<int64_t>(K) * M <= 81920
                               : force == kFew;
    if (M <= kFewRows && few) {
      p.variant = kFew;
      // columns of a workgroup / 16: two (the rows' codes are read once for both) where that
      // leaves two workgroups to a compute unit
      p.cols = N >= 64 * num_cus ? 2 : 1;
      p.workgroups = (N + 16 * p.cols - 1) / (16 * p.cols);
      // wavefronts: enough of them on the chip, each with a unit of K or more (32 columns are
      // two workgroups to a compute unit or more, so eight)
      p.waves = 4;
      while (p.waves < 16 && p.workgroups * p.waves < 16ll * num_cus && K / kUnit > p.waves) p.waves *= 2;
      return p;
    }
    if (force < 0 ? M <= kFewRows || (split > 1 && tiles * 4 <= num_cus) : force == kStream) {
      p.variant = kStream;
      p.k_per_split = ((K + split - 1) / split + kUnit - 1) / kUnit * kUnit;
      p.splits = (K + p.k_per_split - 1) / p.k_per_split;
      p.workgroups = tiles * p.splits;
      p.ws_bytes = p.splits > 1 ? (static_cast<size_t>(p.splits) * M * N * 4 + 255) / 256 * 256 : 0;
      return p;
    }
  }
  // The tile and split of K with the least time by a model: rounds of workgroups over the compute
  // units at the rate that each tile reached on a large product (256 x 256 taken as 2.05e15 a
  // second on 256 units, the others as shares of it), 256 k more for a workgroup's start and end,
  // or the weights' bytes, once from memory and once for every row tile, if they take longer; parts
  // written and read, and a launch.  (The rows' bytes are in neither term.)  Over a sweep of sizes,
  // 1 to 4096 rows and 16 to 131072 columns, every variant timed, its choice takes 1.03 to 1.05
  // times the best variant's time on average; small tiles win where large ones leave units idle
  // (us: 512 x 10240 x 4096 with 192 x 128 34, the best of the others 38).
  double best = 1e30;
  for (int v = 0; v < kVariants; ++v) {
    if (force >= 0 && force < kFew && force != v) continue;
    const int64_t tm = (static_cast<int64_t>(M) + kBM[v] - 1) / kBM[v];
    const int64_t tiles = tm * ((static_cast<int64_t>(N) + kBN[v] - 1) / kBN[v]);
    for (int s = 1; s <= 8; ++s) {
      const int kps = ((K + s - 1) / s + 63) / 64 * 64;
      if (s > 1 && (kps < 512 || (K + kps - 1) / kps != s || static_cast<int64_t>(M) * N * s > (1ll << 28)))
        continue;
      const int64_t wgs = tiles * s, waves = (wgs + num_cus - 1) / num_cus;
      constexpr double kEff[kVariants] = {1.0, 0.8, 0.85, 0.95, 0.7, 0.6, 0.55, 0.78};
      const double t_mfma = static_cast<double>(waves) * kBM[v] * kBN[v] * (kps + 256.0) * 2.0 / (8.0e12 * kEff[v]);
      const double t_mem = static_cast<double>(tm) * N * K / 8.0e12 + static_cast<double>(N) * K / 8e12;
      const double t_part = s > 1 ? static_cast<double>(s) * M * N * 8.0 / 4.0e12 + 3e-6 : 0.0;
      const double t = (t_mfma > t_mem ? t_mfma : t_mem) + t_part;
      if (t < best) {
        best = t;
        p.variant = v;
        p.splits = s;
        p.k_per_split = kps;
        p.workgroups = wgs;
      }
    }
  }
  p.ws_bytes = p.splits > 1 ? static_cast<size_t>(p.workgroups) * kBM[p.variant] * kBN[p.variant] * 4 : 0;
  return p;
}

// keep_parts: the stream's parts of K stay in the workspace, rows by rows.
static hipError_t launch_product(const MatmulI8Args& g, const MatmulI8Plan& p, bool keep_parts,
                                 hipStream_t stream) {
  if (g.M == 0 || g.N == 0) return hipSuccess;
  if (p.variant == kStream)
    return g.dtype == CO_DTYPE_BF16 ? launch_stream<uint16_t>(g, p, keep_parts, stream)
                                    : launch_stream<float>(g, p, keep_parts, stream);
  if (p.variant == kFew)
    return g.dtype == CO_DTYPE_BF16 ? launch_few<uint16_t>(g, PlainRows{}, p, stream)
                                    : launch_few<float>(g, PlainRows{}, p, stream);
  return g.dtype == CO_DTYPE_BF16 ? launch_wide<uint16_t>(g, PlainRows{}, p, stream)
                                  : launch_wide<float>(g, PlainRows{}, p, stream);
}

hipError_t launch_matmul_i8(const MatmulI8Args& g, const MatmulI8Plan& p, hipStream_t stream) {
  return launch_product(g, p, false, stream);
}

// -------------------------------------------- projection with 8-bit weights
//
// quantise, F's product, its rows finished and quantised, the K/V product, rows stored.  The
// stream kernel's parts of K are added up by the kernel that reads them.

namespace {

// A product's results: fp32, or parts of its sums with the scales (splits > 0).
struct Product {
  const float* y;          // [M][N]
  const int* part;         // [splits][M][N]
  const float* a_scale;    // [M]
  const float* w_scale;    // [N]
  int M, N, splits;
  __device__ __forceinline__ f32x4 four(int64_t row, int col) const {
#pragma clang fp contract(off)
    const int64_t at = row * N + col;
    if (splits == 0) return *reinterpret_cast<const f32x4*>(y + at);
    i32x4 sum = {};
    int s = 0;
    for (; s + 4 <= splits; s += 4) {   // four loads in flight
#pragma unroll
      for (int q = 0; q < 4; ++q)
        sum += *reinterpret_cast<const i32x4*>(part + (s + q) * static_cast<int64_t>(M) * N + at);
    }
    for (; s < splits; ++s) sum += *reinterpret_cast<const i32x4*>(part + s * static_cast<int64_t>(M) * N + at);
    const float sa = a_scale[row];
    const f32x4u sw = *reinterpret_cast<const f32x4u*>(w_scale + col);   // (aligned to an element)
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = scaled(sum[i], sa, sw[i]);
    return v;
  }
};

template <int NT>
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) v += red[w];
  return v;
}

// A row of z from F's product: F E on a carry row, the optional RMS norm, its codes.  Q
// times eight entries of it stay in a thread's registers; Q = 0: rows of any length by way
// of `spill` [M][d] (which may be the product's own fp32 results), without a norm: rows of more
// than kNormMaxCols have none.  A chain of a row's loads,
// one or two sums over the workgroup, and its stores: 5.9 us for 16 rows of 4096, 6.3 for 512.
template <int NT, int Q>
__global__ __launch_bounds__(NT) void z_codes_kernel(Product p, float* spill, const float* fe,
                                                     const float* gain, const int32_t* row_dst,
                                                     int8_t* codes, float* scale) {
#pragma clang fp contract(off)
  __shared__ float red[NT / 64];
  __shared__ uint32_t redu[NT / 64];
  const int64_t row = blockIdx.x;
  const int d = p.N;
  const bool carry = fe && is_carry_row(row_dst[row]);
  int8_t* cr = codes + row * d;
  float* sr = spill + row * d;
  constexpr int QN = Q > 0 ? Q : 1;
  float v[QN][8];
  auto read = [&](int c, float (&x)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 z = p.four(row, c + 4 * h);
      if (carry) z += *reinterpret_cast<const f32x4*>(fe + c + 4 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = z[i];
    }
  };
  float ss = 0.f, r = 1.f;
  uint32_t top = 0;
  auto squares = [&](const float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
  };
  auto normed = [&](int c, float (&x)[8]) {
    if (gain) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] * r * gain[c + e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, magnitude(x[e]));
  };
  if constexpr (Q > 0) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = (q * NT + threadIdx.x) * 8;
      if (c < d) {
        read(c, v[q]);
        squares(v[q]);
      }
    }
    if (gain) r = rsqrtf(block_sum<NT>(ss, red) / static_cast<float>(d) + kRmsEps);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = (q * NT + threadIdx.x) * 8;
      if (c < d) normed(c, v[q]);
    }
    const RowScale s(block_max<NT>(top, redu));
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = (q * NT + threadIdx.x) * 8;
      if (c < d) s.codes(v[q], cr + c);
    }
    if (threadIdx.x == 0) scale[row] = s.scale;
  } else {
    for (int c = threadIdx.x * 8; c < d; c += NT * 8) {
      read(c, v[0]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sr[c + e] = v[0][e];
        top = max(top, magnitude(v[0][e]));
      }
    }
    const RowScale s(block_max<NT>(top, redu));
    for (int c = threadIdx.x * 8; c < d; c += NT * 8) {   // (a thread reads what it wrote)
      eight(sr + c, v[0]);
      s.codes(v[0], cr + c);
    }
    if (threadIdx.x == 0) scale[row] = s.scale;
  }
}

// Rows of the K/V product to their destinations: one head segment of some rows a workgroup,
// four rotation pairs a thread.  Keys: the lanes of a row side by side (its dims lie next to
// each other).  Values: rows side by side, for their pages have a dim's sixteen tokens next
// to each other (two bytes a token; dims side by side 23 us, rows 12 us for 512 rows of five
// layers).
__global__ __launch_bounds__(256) void store_rows_i8_kernel(Product p, KvDest e) {
  __shared__ double inv_tab[64];
  const int half = e.hd / 2, lanes = half / 4, rows = 256 / lanes;   // 16 or 8 lanes a row
  if (threadIdx.x < half) inv_tab[threadIdx.x] = rope_table<uint16_t>(e, threadIdx.x);
  __syncthreads();
  const int segs = p.N / e.hd, seg = blockIdx.x % segs;
  const bool value = (seg / e.Hkv & 1) != 0;
  const int tid = threadIdx.x;
  const int row = static_cast<int>(blockIdx.x / segs) * rows + (value ? tid % rows : tid / lanes);
  const int i0 = (value ? tid / rows : tid % lanes) * 4;
  if (row >= p.M) return;                  // (a key's lanes of a row leave together)
  const int32_t dst = e.row_dst[row];
  if (dst == kSkip) return;
  const f32x4 a = p.four(row, seg * e.hd + i0), b = p.four(row, seg * e.hd + half + i0);
  float lo[4], hi[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    lo[q] = a[q];
    hi[q] = b[q];
  }
  k_norm<4>(e, seg, i0, lanes, lo, hi);
  kv_store<uint16_t, 4>(e, row, dst, e.row_pos[row], seg, i0, lo, hi, inv_tab);
}

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t project_i8_ws_bytes(int M, int Dcat, int d, int n_kv, int num_cus) {
  const int wide = Dcat > d ? Dcat : d, out = d > n_kv ? d : n_kv;
  const size_t pf = plan_matmul_i8(M, d, Dcat, num_cus).ws_bytes;
  const size_t pk = plan_matmul_i8(M, n_kv, d, num_cus).ws_bytes;
  return pad256(static_cast<size_t>(M) * wide) + pad256(static_cast<size_t>(M) * 4) +
         pad256(static_cast<size_t>(M) * out * 4) + (pf > pk ? pf : pk);
}

hipError_t launch_project_i8(const ProjectI8Args& a, int num_cus, hipStream_t stream) {
  if (a.M == 0) return hipSuccess;
  const int n_kv = 2 * a.dst.L * a.dst.Hkv * a.dst.hd;
  const int wide = a.Dcat > a.d ? a.Dcat : a.d, out = a.d > n_kv ? a.d : n_kv;
  char* ws = static_cast<char*>(a.ws);
  int8_t* codes = reinterpret_cast<int8_t*>(ws);
  float* scale = reinterpret_cast<float*>(ws + pad256(static_cast<size_t>(a.M) * wide));
  float* y = reinterpret_cast<float*>(reinterpret_cast<char*>(scale) + pad256(static_cast<size_t>(a.M) * 4));
  MatmulI8Args g{};
  g.M = a.M;
  g.dtype = CO_DTYPE_F32;
  g.A = codes;
  g.a_scale = scale;
  g.out = y;
  g.ws = reinterpret_cast<char*>(y) + pad256(static_cast<size_t>(a.M) * out * 4);
  auto product = [&](int N, int K, const int8_t* w, const float* w_scale, Product* p) {
    g.N = N;
    g.K = K;
    g.W = w;
    g.w_scale = w_scale;
    const MatmulI8Plan plan = plan_matmul_i8(g.M, N, K, num_cus);
    const bool parts = plan.variant == kStream && plan.splits > 1;
    *p = Product{y, static_cast<const int*>(g.ws), scale, w_scale, g.M, N, parts ? plan.splits : 0};
    return launch_product(g, plan, parts, stream);
  };
  hipError_t err = launch_quantize_i8(a.hidden, a.M, a.Dcat, CO_DTYPE_BF16, codes, scale, stream);
  if (err != hipSuccess) return err;
  Product p;
  if ((err = product(a.d, a.Dcat, a.wf, a.wf_scale, &p)) != hipSuccess) return err;
  auto finish = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, dim3(a.M), dim3(threads), 0, stream, p, y, a.fe, a.znorm, a.dst.row_dst, codes, scale);
  };
  static_assert(kNormMaxCols <= 16384, "a norm's rows are in registers");
  if (a.d <= 2048) finish(z_codes_kernel<256, 1>, 256);
  else if (a.d <= 4096) finish(z_codes_kernel<512, 1>, 512);
  else if (a.d <= 16384) finish(z_codes_kernel<1024, 2>, 1024);
  else finish(z_codes_kernel<1024, 0>, 1024);
  const MatmulI8Plan kv = plan_matmul_i8(a.M, n_kv, a.d, num_cus);
  if (kv.variant != kStream && a.dst.knorm == nullptr) {   // tiles rotate and store their rows
    g.N = n_kv;
    g.K = a.d;
    g.W = a.wkv;
    g.w_scale = a.wkv_scale;
    return kv.variant == kFew ? launch_few<float>(g, a.dst, kv, stream) : launch_wide<float>(g, a.dst, kv, stream);
  }
  if ((err = product(n_kv, a.d, a.wkv, a.wkv_scale, &p)) != hipSuccess) return err;
  const int per = 1024 / (a.dst.hd / 2);   // rows of a workgroup
  hipLaunchKernelGGL(store_rows_i8_kernel,
                     dim3(static_cast<unsigned>((a.M + per - 1) / per) * (n_kv / a.dst.hd)), dim3(256), 0,
                     stream, p, a.dst);
  return hipGetLastError();
}

}  // namespace co
