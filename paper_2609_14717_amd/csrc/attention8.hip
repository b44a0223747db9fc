// Block attention over ctx = [C ; U] with the committed segment C in the 8-bit
// cache (e4m3 codes, one power-of-two scale per page, head and kind), the carry
// segment U and the block's own rows S in bf16: one online softmax over all of
// them, as drafter_block_attention_ext.
//
// One workgroup per query row and KV head: thread t scores key t of a chunk of
// 256, then the chunk's values are added up, a thread per dim.
#include "co_kernels.h"

namespace co {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float code_value(uint8_t c) {
  return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(c), 0);
}
__device__ __forceinline__ float scale_value(uint8_t b) {
  return __uint_as_float(static_cast<uint32_t>(b) << 23);
}

template <int HD>
__global__ __launch_bounds__(256) void attn_kv8_kernel(AttnArgs a) {
  __shared__ float q[HD], p[256], red[8], part[256];
  const int t = threadIdx.x, G = a.Hq / a.Hkv;
  const int n = blockIdx.x, s = blockIdx.y, g = blockIdx.z % a.Hkv, ll = blockIdx.z / a.Hkv;
  const int layer = a.layer_begin + ll, i = n / G;
  int ctx = a.ctx_len[s], carry = a.carry_len[s];
  const bool ok = ctx >= 0 && ctx <= a.max_pages * kPage && carry >= 0 && carry <= a.CP * kPage;
  if (!ok) {
    if (t == 0) set_status(a.status, CO_ERR_LENGTH);
    ctx = carry = 0;
  }
  const int own = a.k_self && ok ? a.B : 0, keys = ctx + carry + own;
  const int64_t row = ((static_cast<int64_t>(ll) * a.S + s) * a.B + i) * a.Hq + g * G + n % G;
  auto rotated = [&](const uint16_t* x, int d, int pos) {
    const int h = d % (HD / 2);
    float c = 1.f, sn = 0.f;
    rope_cos_sin_rev(pos, a.rope_inv[h] * kInv2Pi, &c, &sn);
    return d < HD / 2 ? bf2f(x[h]) * c - bf2f(x[h + HD / 2]) * sn
                      : bf2f(x[h + HD / 2]) * c + bf2f(x[h]) * sn;
  };
  if (t < HD) {
    const uint16_t* Q = static_cast<const uint16_t*>(a.q) + row * HD;
    const float x = (a.flags & CO_Q_PREROTATED) ? bf2f(Q[t]) : rotated(Q, t, ctx + i);
    q[t] = x * rsqrtf(static_cast<float>(HD)) * kLog2e;
  }
  float M = -INFINITY, l = 0.f, lu = 0.f, ls = 0.f, acc = 0.f;
  auto head = [&](int page) { return (static_cast<int64_t>(layer) * a.num_pages + page) * a.Hkv + g; };
  auto carry_head = [&](int c) {
    return ((static_cast<int64_t>(layer) * a.S + s) * a.CP + c / kPage) * a.Hkv + g;
  };
  const int32_t* pt = a.page_table + static_cast<int64_t>(s) * a.max_pages;
  const int64_t self0 = ((static_cast<int64_t>(ll) * a.S + s) * a.B * a.Hkv + g) * HD;
  __syncthreads();
  for (int k0 = 0; k0 < keys; k0 += 256) {
    const int k = k0 + t;
    float sc = -INFINITY;
    if (k < ctx) {
      const int page = pt[k / kPage];
      if (page < 0 || page >= a.num_pages) {
        set_status(a.status, CO_ERR_PAGE_RANGE);
      } else {
        const uint8_t* x = static_cast<const uint8_t*>(a.k_cache) + (head(page) * kPage + k % kPage) * HD;
        float v = 0.f;
        for (int d = 0; d < HD; ++d) v = fmaf(q[d], code_value(x[d]), v);
        sc = v * scale_value(a.k_scale[head(page)]);
      }
    } else if (k < ctx + carry) {
      const int c = k - ctx;
      const uint16_t* x = static_cast<const uint16_t*>(a.k_carry) + (carry_head(c) * kPage + c % kPage) * HD;
      sc = 0.f;
      for (int d = 0; d < HD; ++d) sc = fmaf(q[d], bf2f(x[d]), sc);
    } else if (k < keys) {
      const int c = k - ctx - carry;
      const uint16_t* x = static_cast<const uint16_t*>(a.k_self) + self0 + static_cast<int64_t>(c) * a.Hkv * HD;
      sc = 0.f;
      for (int d = 0; d < HD; ++d) sc = fmaf(q[d], bf2f(f2bf(rotated(x, d, ctx + c))), sc);
    }
    auto reduce = [&](float v, bool mx) {   // over the workgroup
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const float u = __shfl_xor(v, o);
        v = mx ? fmaxf(v, u) : v + u;
      }
      __syncthreads();
      if ((t & 63) == 0) red[t >> 6] = v;
      __syncthreads();
      return mx ? fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]))
                : (red[0] + red[1]) + (red[2] + red[3]);
    };
    const float m = fmaxf(M, reduce(sc, true)), base = m == -INFINITY ? 0.f : m;
    const float e = exp2f(sc - base), f = M == -INFINITY ? 0.f : exp2f(M - base);
    M = m;
    l = l * f + reduce(e, false);
    lu = lu * f + reduce(k >= ctx && k < ctx + carry ? e : 0.f, false);
    ls = ls * f + reduce(k >= ctx + carry ? e : 0.f, false);
    p[t] = e;
    __syncthreads();
    acc *= f;
    const int d = t % HD;
    for (int j = t / HD; j < 256 && k0 + j < keys; j += 256 / HD) {
      const int kk = k0 + j;
      float v = 0.f;
      if (kk < ctx) {
        const int page = pt[kk / kPage];
        if (page < 0 || page >= a.num_pages) continue;
        v = code_value(static_cast<const uint8_t*>(a.v_cache)[(head(page) * HD + d) * kPage + kk % kPage]) *
            scale_value(a.v_scale[head(page)]);
      } else if (kk < ctx + carry) {
        const int c = kk - ctx;
        v = bf2f(static_cast<const uint16_t*>(a.v_carry)[(carry_head(c) * HD + d) * kPage + c % kPage]);
      } else {
        v = bf2f(static_cast<const uint16_t*>(a.v_self)[self0 + static_cast<int64_t>(kk - ctx - carry) * a.Hkv * HD + d]);
      }
      acc = fmaf(p[j], v, acc);
    }
    __syncthreads();
  }
  part[t] = acc;
  __syncthreads();
  if (t < HD) {
    float o = 0.f;
    for (int j = 0; j < 256 / HD; ++j) o += part[t + j * HD];
    static_cast<uint16_t*>(a.out)[row * HD + t] = f2bf(l > 0.f ? o / l : 0.f);
  }
  if (t == 0 && a.lse) a.lse[row] = l > 0.f ? (M + log2f(l)) * kLn2 : -INFINITY;
  if (t == 0 && a.mass) a.mass[row] = l - ls > 0.f ? lu / (l - ls) : 0.f;
}

}  // namespace

hipError_t launch_attention_kv8(const AttnArgs& a, const AttnPlan& p, int layer_count,
                                hipStream_t stream) {
  (void)p;
  if (a.S == 0 || layer_count == 0) return hipSuccess;
  const dim3 grid(a.B * (a.Hq / a.Hkv), a.S, layer_count * a.Hkv);
  if (a.hd == 64) hipLaunchKernelGGL(attn_kv8_kernel<64>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(attn_kv8_kernel<128>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace co
