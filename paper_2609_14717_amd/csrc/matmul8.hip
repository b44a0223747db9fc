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

__device__ __forceinline__ float scaled(int sum, float sa, float sw) {
#pragma clang fp contract(off)
  return static_cast<float>(sum) * (sa * sw);
}

// A wavefront: 32 x 32 outputs, fragments from memory.  Lane l holds 16 k of row l % 32
// of each operand; result register r is column l % 32 of row 8 (r / 4) + 4 (l / 32) + r % 4.
template <typename T>
__global__ __launch_bounds__(256) void matmul_i8_kernel(MatmulI8Args g, int tiles_n) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int m0 = static_cast<int>(blockIdx.x / tiles_n) * 64 + (wave >> 1) * 32;
  const int n0 = static_cast<int>(blockIdx.x % tiles_n) * 64 + (wave & 1) * 32;
  const int am = min(m0 + (lane & 31), g.M - 1), bn = min(n0 + (lane & 31), g.N - 1);
  const int8_t* pa = g.A + static_cast<int64_t>(am) * g.K + (lane >> 5) * 16;
  const int8_t* pb = g.W + static_cast<int64_t>(bn) * g.K + (lane >> 5) * 16;
  i32x16 acc = {};
  for (int k = 0; k < g.K; k += 32)
    acc = mfma_i8(*reinterpret_cast<const i32x4*>(pa + k), *reinterpret_cast<const i32x4*>(pb + k), acc);
  const int col = n0 + (lane & 31);
  if (col >= g.N) return;
  const float sw = g.w_scale[col];
  const float bias = g.bias ? g.bias[col] : 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int row = m0 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
    if (row >= g.M) continue;
    float v = scaled(acc[r], g.a_scale[row], sw);
    if (g.bias) v = v + bias;
    T* out = static_cast<T*>(g.out) + static_cast<int64_t>(row) * g.N + col;
    if constexpr (sizeof(T) == 2) *out = static_cast<T>(cvt_pk_bf16(v, v)); else *out = v;
  }
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

MatmulI8Plan plan_matmul_i8(int M, int N, int K, int num_cus) {
  (void)K;
  (void)num_cus;
  MatmulI8Plan p{};
  p.workgroups = static_cast<int64_t>((M + 63) / 64) * ((N + 63) / 64);
  p.ws_bytes = 0;
  return p;
}

hipError_t launch_matmul_i8(const MatmulI8Args& g, const MatmulI8Plan& p, hipStream_t stream) {
  if (g.M == 0 || g.N == 0) return hipSuccess;
  const int tiles_n = (g.N + 63) / 64;
  const dim3 grid(static_cast<unsigned>(p.workgroups)), block(256);
  if (g.dtype == CO_DTYPE_BF16)
    hipLaunchKernelGGL(matmul_i8_kernel<uint16_t>, grid, block, 0, stream, g, tiles_n);
  else
    hipLaunchKernelGGL(matmul_i8_kernel<float>, grid, block, 0, stream, g, tiles_n);
  return hipGetLastError();
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
  (void)num_cus;
  return pad256(static_cast<size_t>(M) * wide) + pad256(static_cast<size_t>(M) * 4) +
         pad256(static_cast<size_t>(M) * out * 4);
}

hipError_t launch_project_i8(const ProjectI8Args& a, int num_cus, hipStream_t stream) {
  if (a.M == 0) return hipSuccess;
  const int n_kv = 2 * a.dst.L * a.dst.Hkv * a.dst.hd;
  const int wide = a.Dcat > a.d ? a.Dcat : a.d;
  char* ws = static_cast<char*>(a.ws);
  int8_t* codes = reinterpret_cast<int8_t*>(ws);
  float* scale = reinterpret_cast<float*>(ws + pad256(static_cast<size_t>(a.M) * wide));
  float* y = reinterpret_cast<float*>(reinterpret_cast<char*>(scale) + pad256(static_cast<size_t>(a.M) * 4));
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
