// Products of 8-bit integers with a scale for each row of both operands, and the rows'
// quantisation.
//
//   code[i][k] = rint(127 x[i][k] / a_i), a_i = max_k |x[i][k]|, scale_i = a_i / 127
//   out[i][j]  = float(sum_k a[i][k] w[j][k]) (a_scale[i] w_scale[j]) + bias[j]
//
// Sums are exact: int32, for k up to 131008.
#include "co_kernels.h"

namespace co {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr float kLeast = 0x1.fcp-120f;   // 127 * 2^-126: smallest magnitude that scales a row

// -------------------------------------------------------------- quantisation

// One code: 127 x / a to the nearest integer, ties to even, exactly: where the fp32
// product with r = 127 / a (off by up to 2^-16) is too close to the middle of two
// integers, the quotient in fp64 decides (its rounding cannot reach a middle that the
// exact quotient, of two 24-bit numbers, does not lie on).
__device__ __forceinline__ int code_of(float x, float a, float r) {
#pragma clang fp contract(off)
  const float t = x * r;
  const float n = rintf(t);
  if (fabsf(fabsf(t - n) - 0.5f) < 0x1p-14f)
    return static_cast<int>(rint(static_cast<double>(x) * 127.0 / static_cast<double>(a)));
  return static_cast<int>(n);
}

// One workgroup per row: its largest magnitude, then its codes.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* x, int cols, int8_t* codes,
                                                            float* scale) {
  __shared__ uint32_t red[4];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  const T* xr = x + row * cols;
  auto get = [&](int c) {
    if constexpr (sizeof(T) == 2) return bf2f(xr[c]); else return xr[c];
  };
  uint32_t top = 0;   // magnitudes compare as their bits; infinities and NaNs are largest
  for (int c = tid; c < cols; c += 256) top = max(top, __float_as_uint(get(c)) & 0x7FFFFFFFu);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), off)));
  if ((tid & 63) == 0) red[tid >> 6] = top;
  __syncthreads();
  top = max(max(red[0], red[1]), max(red[2], red[3]));
  const bool fine = top < 0x7F800000u;
  const float a = fmaxf(__uint_as_float(top), kLeast), r = 127.f / a;
  int8_t* cr = codes + row * cols;
  for (int c = tid; c < cols; c += 256) cr[c] = fine ? static_cast<int8_t>(code_of(get(c), a, r)) : 0;
  if (tid == 0) scale[row] = fine ? a / 127.f : NAN;
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

// Few rows (16 MT of them): bound by reading the weights once.  A workgroup's NW
// wavefronts share 16 TN columns and split K: a wavefront takes every NW-th unit of 256
// bytes of K, straight into the operand registers of v_mfma_i32_16x16x64_i8 (lane l holds
// row or column l % 16, 16 k from 16 (l / 16) on; result register r is row 4 (l / 16) + r,
// column l % 16), the next unit's loads in flight while one is multiplied.  The NW partial
// tiles are added in LDS: whole numbers, so the order does not matter.
constexpr int kUnit = 256;

template <int MT, int TN, int NW, typename T>
__global__ __launch_bounds__(64 * NW) void matmul_i8_few_kernel(MatmulI8Args g) {
  __shared__ int red[NW][MT * TN * 256];
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
    pw[j] = g.W + static_cast<int64_t>(min(n0 + 16 * j + (lane & 15), g.N - 1)) * g.K + quad;
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
constexpr int kStageK = 128;

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

template <int TMW, int TNW, int NS, typename T>
__global__ __launch_bounds__(512, 1) void matmul_i8_wide_kernel(MatmulI8Args g, int tiles_m,
                                                                int tiles_n, int k_per_split) {
  constexpr int BM = 64 * TMW, BN = 128 * TNW, ROWS = BM + BN, STAGE = ROWS * kStageK;
  constexpr int LPW = ROWS / 64;                         // 1 KiB loads of a wavefront, a stage
  static_assert(LPW * (NS - 1) < 64 && NS >= 2 && NS <= 4, "vmcnt");
  static_assert(NS * STAGE + 8 * BN <= 160 * 1024, "LDS");
  __shared__ __align__(16) unsigned char smem[NS * STAGE];
  __shared__ __align__(16) float col_scale[BN], col_bias[BN];

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
                                  : g.W + static_cast<int64_t>(min(n0 + row - BM, g.N - 1)) * g.K;
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
    const int col = min(n0 + c, g.N - 1);
    col_scale[c] = g.w_scale[col];
    col_bias[c] = g.bias ? g.bias[col] : 0.f;
  }
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
      put_tile<T>(g, acc[a][b], row, sa, n0 + cb, lane, col_scale + cb, col_bias + cb);
    }
  }
}

// The parts of K of one 32 x 32 tile for each wavefront, added up, scaled and stored.
template <int TMW, int TNW, typename T>
__global__ __launch_bounds__(512) void sum_parts_i8_kernel(MatmulI8Args g, int tiles_m, int tiles_n,
                                                           int splits) {
  constexpr int BM = 64 * TMW, BN = 128 * TNW;
  __shared__ __align__(16) float col_scale[BN], col_bias[BN];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 2, wn = wave & 3;
  const int frag = blockIdx.x % (TMW * TNW), r0 = blockIdx.x / (TMW * TNW);
  int m0, n0;
  tile_of<BM, BN>(r0, tiles_m, tiles_n, &m0, &n0);
  for (int c = tid; c < BN; c += 512) {
    const int col = min(n0 + c, g.N - 1);
    col_scale[c] = g.w_scale[col];
    col_bias[c] = g.bias ? g.bias[col] : 0.f;
  }
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
  put_tile<T>(g, acc, row, row < g.M ? g.a_scale[row] : 0.f, n0 + cb, lane, col_scale + cb, col_bias + cb);
}

// Tile variants of the wide kernel; kFew: the kernel for few rows.
constexpr int kVariants = 7, kFew = kVariants;
constexpr int kBM[kVariants] = {256, 256, 128, 192, 128, 64, 64};
constexpr int kBN[kVariants] = {256, 128, 256, 256, 128, 256, 128};

template <int TMW, int TNW, int NS, typename T>
void launch_wide_t(const MatmulI8Args& g, const MatmulI8Plan& p, hipStream_t stream) {
  const int tm = (g.M + 64 * TMW - 1) / (64 * TMW), tn = (g.N + 128 * TNW - 1) / (128 * TNW);
  hipLaunchKernelGGL((matmul_i8_wide_kernel<TMW, TNW, NS, T>), dim3(static_cast<unsigned>(p.workgroups)),
                     dim3(512), 0, stream, g, tm, tn, p.k_per_split);
  if (p.splits > 1)
    hipLaunchKernelGGL((sum_parts_i8_kernel<TMW, TNW, T>), dim3(static_cast<unsigned>(tm) * tn * TMW * TNW),
                       dim3(512), 0, stream, g, tm, tn, p.splits);
}

template <typename T>
hipError_t launch_wide(const MatmulI8Args& g, const MatmulI8Plan& p, hipStream_t stream) {
  switch (p.variant) {
    case 0: launch_wide_t<4, 2, 2, T>(g, p, stream); break;
    case 1: launch_wide_t<4, 1, 3, T>(g, p, stream); break;
    case 2: launch_wide_t<2, 2, 3, T>(g, p, stream); break;
    case 3: launch_wide_t<3, 2, 2, T>(g, p, stream); break;
    case 4: launch_wide_t<2, 1, 4, T>(g, p, stream); break;
    case 5: launch_wide_t<1, 2, 3, T>(g, p, stream); break;
    default: launch_wide_t<1, 1, 4, T>(g, p, stream); break;
  }
  return hipGetLastError();
}

template <int MT, int TN, typename T>
hipError_t launch_few_nw(const MatmulI8Args& g, const MatmulI8Plan& p, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(p.workgroups));
  if constexpr (MT * TN <= 2) {   // (more tiles need more than the 128 registers of sixteen wavefronts)
    if (p.waves == 16) {
      hipLaunchKernelGGL((matmul_i8_few_kernel<MT, TN, 16, T>), grid, dim3(1024), 0, stream, g);
      return hipGetLastError();
    }
  }
  if (p.waves == 8) hipLaunchKernelGGL((matmul_i8_few_kernel<MT, TN, 8, T>), grid, dim3(512), 0, stream, g);
  else hipLaunchKernelGGL((matmul_i8_few_kernel<MT, TN, 4, T>), grid, dim3(256), 0, stream, g);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_few(const MatmulI8Args& g, const MatmulI8Plan& p, hipStream_t stream) {
  if (g.M <= 16) {
    if (p.cols == 4) return launch_few_nw<1, 4, T>(g, p, stream);
    if (p.cols == 2) return launch_few_nw<1, 2, T>(g, p, stream);
    return launch_few_nw<1, 1, T>(g, p, stream);
  }
  if (p.cols == 4) return launch_few_nw<2, 4, T>(g, p, stream);
  if (p.cols == 2) return launch_few_nw<2, 2, T>(g, p, stream);
  return launch_few_nw<2, 1, T>(g, p, stream);
}

}  // namespace

hipError_t launch_quantize_i8(const void* x, int64_t rows, int cols, int dtype, int8_t* codes,
                              float* scale, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(rows)), block(256);
  if (dtype == CO_DTYPE_BF16)
    hipLaunchKernelGGL(quantize_rows_kernel<uint16_t>, grid, block, 0, stream,
                       static_cast<const uint16_t*>(x), cols, codes, scale);
  else
    hipLaunchKernelGGL(quantize_rows_kernel<float>, grid, block, 0, stream,
                       static_cast<const float*>(x), cols, codes, scale);
  return hipGetLastError();
}

constexpr int kFewRows = 32;

MatmulI8Plan plan_matmul_i8(int M, int N, int K, int num_cus) {
  MatmulI8Plan p{};
  p.splits = 1;
  p.k_per_split = K;
  const int64_t force = tuning(CO_TUNE_MATMUL_I8);
  if (force < 0 ? M <= kFewRows : force == kFew && M <= kFewRows) {
    p.variant = kFew;
    // columns of a workgroup: as many (the rows' codes are read once for them) as leave
    // two workgroups to a compute unit
    p.cols = N >= 128 * num_cus ? 4 : (N >= 64 * num_cus ? 2 : 1);
    p.workgroups = (N + 16 * p.cols - 1) / (16 * p.cols);
    // wavefronts: enough of them on the chip, each with a unit of K or more
    p.waves = 4;
    while (p.waves < 16 && p.workgroups * p.waves < 16ll * num_cus && K / kUnit > p.waves) p.waves *= 2;
    if (p.cols * (M > 16 ? 2 : 1) > 2 && p.waves == 16) p.waves = 8;
    return p;
  }
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
      constexpr double kEff[kVariants] = {1.0, 0.8, 0.85, 0.95, 0.7, 0.6, 0.45};
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

hipError_t launch_matmul_i8(const MatmulI8Args& g, const MatmulI8Plan& p, hipStream_t stream) {
  if (g.M == 0 || g.N == 0) return hipSuccess;
  if (p.variant == kFew)
    return g.dtype == CO_DTYPE_BF16 ? launch_few<uint16_t>(g, p, stream) : launch_few<float>(g, p, stream);
  return g.dtype == CO_DTYPE_BF16 ? launch_wide<uint16_t>(g, p, stream) : launch_wide<float>(g, p, stream);
}

// -------------------------------------------- projection with 8-bit weights

namespace {

// A row of z: F(E) on carried rows, the optional RMS norm, then its codes.
__global__ __launch_bounds__(256) void z_codes_kernel(float* z, int d, const float* fe,
                                                      const float* gain, const int32_t* row_dst,
                                                      int8_t* codes, float* scale) {
#pragma clang fp contract(off)
  __shared__ float red[4];
  __shared__ uint32_t redu[4];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  float* zr = z + row * d;
  const int32_t dst = row_dst[row];
  const bool carry = fe && dst < 0 && dst != kSkip;
  float ss = 0.f;
  for (int c = tid; c < d; c += 256) {
    const float v = carry ? zr[c] + fe[c] : zr[c];
    zr[c] = v;
    ss += v * v;
  }
  float r = 1.f;
  if (gain) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
    if ((tid & 63) == 0) red[tid >> 6] = ss;
    __syncthreads();
    r = rsqrtf(((red[0] + red[1]) + (red[2] + red[3])) / static_cast<float>(d) + 1e-6f);
  }
  uint32_t top = 0;
  for (int c = tid; c < d; c += 256) {
    float v = zr[c];
    if (gain) zr[c] = v = v * r * gain[c];
    top = max(top, __float_as_uint(v) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), off)));
  if ((tid & 63) == 0) redu[tid >> 6] = top;
  __syncthreads();
  top = max(max(redu[0], redu[1]), max(redu[2], redu[3]));
  const bool fine = top < 0x7F800000u;
  const float a = fmaxf(__uint_as_float(top), kLeast), q = 127.f / a;
  int8_t* cr = codes + row * d;
  for (int c = tid; c < d; c += 256) cr[c] = fine ? static_cast<int8_t>(code_of(zr[c], a, q)) : 0;
  if (tid == 0) scale[row] = fine ? a / 127.f : NAN;
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
  const int wide = a.Dcat > a.d ? a.Dcat : a.d;
  char* ws = static_cast<char*>(a.ws);
  int8_t* codes = reinterpret_cast<int8_t*>(ws);
  float* scale = reinterpret_cast<float*>(ws + pad256(static_cast<size_t>(a.M) * wide));
  float* y = reinterpret_cast<float*>(reinterpret_cast<char*>(scale) + pad256(static_cast<size_t>(a.M) * 4));
  const int out = a.d > n_kv ? a.d : n_kv;
  hipError_t err = launch_quantize_i8(a.hidden, a.M, a.Dcat, CO_DTYPE_BF16, codes, scale, stream);
  if (err != hipSuccess) return err;
  MatmulI8Args g{};
  g.M = a.M;
  g.N = a.d;
  g.K = a.Dcat;
  g.dtype = CO_DTYPE_F32;
  g.A = codes;
  g.a_scale = scale;
  g.W = a.wf;
  g.w_scale = a.wf_scale;
  g.out = y;
  g.ws = reinterpret_cast<char*>(y) + pad256(static_cast<size_t>(a.M) * out * 4);
  if ((err = launch_matmul_i8(g, plan_matmul_i8(g.M, g.N, g.K, num_cus), stream)) != hipSuccess) return err;
  hipLaunchKernelGGL(z_codes_kernel, dim3(a.M), dim3(256), 0, stream, y, a.d, a.fe, a.znorm,
                     a.dst.row_dst, codes, scale);
  g.N = n_kv;
  g.K = a.d;
  g.W = a.wkv;
  g.w_scale = a.wkv_scale;
  if ((err = launch_matmul_i8(g, plan_matmul_i8(g.M, g.N, g.K, num_cus), stream)) != hipSuccess) return err;
  return launch_store_products(y, 1, a.M, n_kv, a.dst, stream);
}

}  // namespace co
