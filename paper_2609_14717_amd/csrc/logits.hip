// From a model's logits to what a verification takes: the history of the tokens that a
// request has seen, the rules on its logits (penalties for repeated tokens, biases,
// grammar masks) and the probabilities at its temperature.
//
// A verified window has several rows of logits per sequence; row j comes after the
// proposals before it, so that these count as generated there.  For token v of row j,
// with c = how often v was generated (history and window):
//   x = x > 0 ? x / r : x * r        if v was seen (prompt, history or window)
//   x = x - f c;  x = x - p          if c > 0
//   x = x + bias                     if v has one
//   x = -inf                         if the row's mask forbids v
// each operation rounded to fp32 on its own, so that equal logits stay equal.  Probabilities
// are exp((x - max) / T) / sum, in fp32.
//
// All of it is bound by memory: a logit is read and a logit or a probability written.
#include "co_kernels.h"

namespace co {

namespace {

constexpr int kVec = 8;                     // tokens of a thread: one byte of a mask
constexpr int kChunk = 256 * kVec;          // of a workgroup at a time
constexpr int kRowsMax = 8;                 // rows of a sequence that a workgroup takes together

typedef uint16_t u16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

enum { kRules = 0, kStats = 1, kProbs = 2 };

constexpr float kNone = -INFINITY;

// Eight elements v .. v + 7 of a row that starts anywhere, `pad` from V on.
template <typename T> struct Vec;
template <> struct Vec<uint16_t> {
  u16x8u x;
  __device__ __forceinline__ float get(int e) const { return bf2f(x[e]); }
};
template <> struct Vec<float> {
  f32x4u lo, hi;
  __device__ __forceinline__ float get(int e) const { return e < 4 ? lo[e & 3] : hi[e & 3]; }
};

__device__ __forceinline__ void load8(const uint16_t* p, int v, int V, Vec<uint16_t>* o,
                                      uint16_t pad) {
  if (v + kVec <= V) {
    o->x = *reinterpret_cast<const u16x8u*>(p + v);
    return;
  }
#pragma unroll
  for (int e = 0; e < kVec; ++e) o->x[e] = v + e < V ? p[v + e] : pad;
}

__device__ __forceinline__ void load8(const float* p, int v, int V, Vec<float>* o, float pad) {
  if (v + kVec <= V) {
    o->lo = *reinterpret_cast<const f32x4u*>(p + v);
    o->hi = *reinterpret_cast<const f32x4u*>(p + v + 4);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    o->lo[e] = v + e < V ? p[v + e] : pad;
    o->hi[e] = v + e + 4 < V ? p[v + e + 4] : pad;
  }
}

template <typename T> __device__ __forceinline__ T lowest();
template <> __device__ __forceinline__ uint16_t lowest<uint16_t>() { return 0xFF80u; }
template <> __device__ __forceinline__ float lowest<float>() { return kNone; }

__device__ __forceinline__ void store8(float* p, int v, int V, const float (&x)[kVec]) {
  if (v + kVec <= V) {
    *reinterpret_cast<f32x4u*>(p + v) = f32x4u{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4u*>(p + v + 4) = f32x4u{x[4], x[5], x[6], x[7]};
    return;
  }
#pragma unroll
  for (int e = 0; e < kVec; ++e)
    if (v + e < V) p[v + e] = x[e];
}

__device__ __forceinline__ void store8(uint16_t* p, int v, int V, const float (&x)[kVec]) {
  u16x8u o;
#pragma unroll
  for (int e = 0; e < kVec; e += 2) {
    const uint32_t w = cvt_pk_bf16(x[e], x[e + 1]);
    o[e] = static_cast<uint16_t>(w);
    o[e + 1] = static_cast<uint16_t>(w >> 16);
  }
  if (v + kVec <= V) {
    *reinterpret_cast<u16x8u*>(p + v) = o;
    return;
  }
#pragma unroll
  for (int e = 0; e < kVec; ++e)
    if (v + e < V) p[v + e] = o[e];
}

// The penalties on one logit that was seen; c: how often generated.
__device__ __forceinline__ float penalise(float x, int c, float rep, float freq, float pres) {
#pragma clang fp contract(off)
  x = x > 0.f ? x / rep : x * rep;
  if (c > 0) {
    const float fc = freq * static_cast<float>(c);
    x = x - fc;
    x = x - pres;
  }
  return x;
}

// exp2 of non-positive arguments; 0 at -inf
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// log2(e) / T, kept finite and above 0; 0 for a greedy sequence (T <= 0 or NaN).
__device__ __forceinline__ float row_slope(const float* temperature, int s) {
  const float t = temperature ? temperature[s] : 1.f;
  if (!(t > 0.f)) return 0.f;
  return fminf(fmaxf(1.44269504088896341f / t, 0x1p-126f), 0x1.fffffep+127f);
}

// What a part of a row holds: its largest logit, where it first is, and the sum of
// exp2((x - m) k).
struct Part {
  float m, l;
  int at;
};

__device__ __forceinline__ Part join(const Part& a, const Part& b, float k) {
  Part r;
  const bool other = b.m > a.m || (b.m == a.m && b.at < a.at);
  r.m = other ? b.m : a.m;
  r.at = other ? b.at : a.at;
  // (equal largest values, infinite ones among them, keep their sums as they are)
  const float la = a.m == r.m ? a.l : a.l * exp2_fast((a.m - r.m) * k);
  const float lb = b.m == r.m ? b.l : b.l * exp2_fast((b.m - r.m) * k);
  r.l = la + lb;
  return r;
}

__device__ __forceinline__ Part shfl_part(const Part& p, int mask) {
  return Part{__shfl_xor(p.m, mask), __shfl_xor(p.l, mask), __shfl_xor(p.at, mask)};
}

// One workgroup: chunks of tokens of one sequence, up to kRowsMax of its rows together, so
// that the history words and biases of a token are read once for them and every thread has
// as many loads in flight as there are rows.
template <typename T, int KIND>
__global__ __launch_bounds__(256) void rows_kernel(LogitArgs a) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int b = blockIdx.x;
  const int grp = b % a.groups;
  b /= a.groups;
  const int tile = b % a.tiles, s = b / a.tiles;
  const int j0 = grp * a.rows_per, nr = min(a.rows_per, a.R - j0);
  const int V = a.V;
  const int64_t row0 = static_cast<int64_t>(s) * a.R + j0;
  const T* logits = static_cast<const T*>(a.logits) + row0 * V;
  const bool first = tile == 0 && grp == 0 && tid == 0;   // reports what concerns a sequence

  const bool penalties = a.seen != nullptr;
  const float rep = a.repetition ? a.repetition[s] : 1.f;
  const float freq = a.frequency ? a.frequency[s] : 0.f;
  const float pres = a.presence ? a.presence[s] : 0.f;
  const int32_t* draft = a.draft && penalties ? a.draft + static_cast<int64_t>(s) * a.B : nullptr;
  if (KIND != kProbs && draft && tile == 0 && grp == 0)
    for (int i = tid; i < a.R - 1; i += 256)
      if (static_cast<uint32_t>(draft[i]) >= static_cast<uint32_t>(V))
        set_status(a.status, CO_ERR_TOKEN);
  int b0 = 0, b1 = 0;
  if (a.bias_start) {
    b0 = a.bias_start[s];
    b1 = a.bias_start[s + 1];
    if (b0 < 0 || b1 < b0 || b1 > a.num_bias) {
      if (first) set_status(a.status, CO_ERR_LENGTH);
      b0 = b1 = 0;
    }
  }
  int mask[kRowsMax];   // >= 0: the row's mask, -1: none, -2: no such mask, nothing allowed
#pragma unroll
  for (int r = 0; r < kRowsMax; ++r) {
    mask[r] = a.mask_row && r < nr ? max(-1, a.mask_row[row0 + r]) : -1;
    if (mask[r] >= a.num_masks) {
      mask[r] = -2;
      if (tid == 0) set_status(a.status, CO_ERR_MASK);
    }
  }
  const int64_t mask_bytes = static_cast<int64_t>((V + 31) / 32) * 4;

  __shared__ int last[kChunk];
  __shared__ Part parts[4][kRowsMax];
  __shared__ Part whole[kRowsMax];
  const float k = KIND == kRules ? 0.f : row_slope(a.temperature, s);

  Part acc[kRowsMax];
  if constexpr (KIND == kStats) {
#pragma unroll
    for (int r = 0; r < kRowsMax; ++r) acc[r] = Part{kNone, 0.f, INT32_MAX};
  }
  if constexpr (KIND == kProbs) {
    // the row's parts joined: its largest logit and one over its sum
    for (int r = wave; r < nr; r += 4) {
      Part p{kNone, 0.f, INT32_MAX};
      for (int t = lane; t < a.tiles; t += 64) {
        const float4 w = a.ws[(row0 + r) * a.tiles + t];
        p = join(p, Part{w.x, w.y, __float_as_int(w.z)}, k);
      }
#pragma unroll
      for (int x = 32; x >= 1; x >>= 1) p = join(p, shfl_part(p, x), k);
      if (lane == 0) {
        p.l = p.l > 0.f ? 1.f / p.l : 0.f;
        whole[r] = p;
        if (tile == 0 && a.top) a.top[row0 + r] = p.m > kNone ? p.at : -1;
      }
    }
    __syncthreads();
  }

  for (int c = 0; c < a.chunks; ++c) {
    const int base = (tile * a.chunks + c) * kChunk;
    if (base >= V) break;
    const int v = base + tid * kVec;
    // the last entry of each token of the chunk in the sequence's list of biases
    if (b1 > b0) {
      __syncthreads();
      for (int i = tid; i < kChunk; i += 256) last[i] = 0;
      __syncthreads();
      for (int i = b0 + tid; i < b1; i += 256) {
        const int t = a.bias_tok[i];
        if (static_cast<uint32_t>(t) >= static_cast<uint32_t>(V)) set_status(a.status, CO_ERR_TOKEN);
        else if (t >= base && t - base < kChunk) atomicMax(&last[t - base], i + 1 - b0);
      }
      __syncthreads();
    }
    if (v >= V) continue;

    Vec<T> x[kRowsMax];
#pragma unroll
    for (int r = 0; r < kRowsMax; ++r)
      if (r < nr) load8(logits + static_cast<int64_t>(r) * V, v, V, &x[r], lowest<T>());
    uint8_t allowed[kRowsMax];
#pragma unroll
    for (int r = 0; r < kRowsMax; ++r) {
      allowed[r] = mask[r] == -2 ? 0 : 0xFF;
      if (mask[r] >= 0)
        allowed[r] = reinterpret_cast<const uint8_t*>(a.mask_bits)[mask[r] * mask_bytes + v / 8];
    }
    int cnt[kVec];
    uint32_t known = 0;        // bit e: token v + e was seen
    if (penalties) {
      Vec<uint16_t> w;
      load8(a.seen + static_cast<int64_t>(s) * V, v, V, &w, 0);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        cnt[e] = w.x[e] & 0x7FFF;
        known |= (w.x[e] != 0 ? 1u : 0u) << e;
      }
    }
    auto add = [&](int t) {    // one more proposal
      const uint32_t e0 = static_cast<uint32_t>(t - v);
      if (e0 >= kVec) return;
#pragma unroll
      for (int e = 0; e < kVec; ++e) cnt[e] += static_cast<int>(e0) == e ? 1 : 0;
      known |= 1u << e0;
    };
    if (draft)
      for (int i = 0; i < j0; ++i) add(draft[i]);
    float bias[kVec];
    uint32_t biased = 0;
    if (b1 > b0) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const int i = last[tid * kVec + e];
        bias[e] = 0.f;
        if (i > 0) {
          bias[e] = a.bias_val[b0 + i - 1];
          biased |= 1u << e;
        }
      }
    }

#pragma unroll
    for (int r = 0; r < kRowsMax; ++r) {
      if (r >= nr) continue;
      if (draft && r > 0) add(draft[j0 + r - 1]);
      float y[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) y[e] = x[r].get(e);
      if (known) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (known >> e & 1) y[e] = penalise(y[e], cnt[e], rep, freq, pres);
      }
      if (biased) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (biased >> e & 1) y[e] = y[e] + bias[e];
      }
      if (allowed[r] != 0xFF) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (!(allowed[r] >> e & 1)) y[e] = kNone;
      }
      if constexpr (KIND == kRules) {
        store8(static_cast<T*>(a.out) + (row0 + r) * V, v, V, y);
        continue;
      }
      // a NaN is left out, as if its token were masked
#pragma unroll
      for (int e = 0; e < kVec; ++e) y[e] = y[e] == y[e] ? y[e] : kNone;
      if constexpr (KIND == kStats) {
        float top = y[0];
#pragma unroll
        for (int e = 1; e < kVec; ++e) top = fmaxf(top, y[e]);
        Part& p = acc[r];
        if (top > p.m) {
          int at = 0;
#pragma unroll
          for (int e = kVec - 1; e >= 0; --e) at = y[e] == top ? e : at;
          p.l = p.m > kNone ? p.l * exp2_fast((p.m - top) * k) : 0.f;
          p.m = top;
          p.at = v + at;
        }
        if (p.m > kNone) {
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            p.l += y[e] == p.m ? 1.f : exp2_fast((y[e] - p.m) * k);
        }
      } else {
        const Part p = whole[r];
        if (k > 0.f && p.m > kNone) {
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            y[e] = (y[e] == p.m ? 1.f : exp2_fast((y[e] - p.m) * k)) * p.l;
        } else {   // greedy, or nothing left
#pragma unroll
          for (int e = 0; e < kVec; ++e) y[e] = p.m > kNone && v + e == p.at ? 1.f : 0.f;
        }
        store8(a.probs + (row0 + r) * V, v, V, y);
      }
    }
  }

  if constexpr (KIND == kStats) {
#pragma unroll
    for (int r = 0; r < kRowsMax; ++r) {
      if (r >= nr) continue;
      Part p = acc[r];
#pragma unroll
      for (int x = 32; x >= 1; x >>= 1) p = join(p, shfl_part(p, x), k);
      if (lane == 0) parts[wave][r] = p;
    }
    __syncthreads();
    if (tid < nr) {
      Part p = parts[0][tid];
      for (int w = 1; w < 4; ++w) p = join(p, parts[w][tid], k);
      a.ws[(row0 + tid) * a.tiles + tile] = float4{p.m, p.l, __int_as_float(p.at), 0.f};
    }
  }
}

// ---------------------------------------------------------------- history

constexpr int kTile = 8192;   // tokens whose counts a workgroup holds

// How many of a sequence's tokens count; -1: the length is wrong.
__device__ __forceinline__ int token_count(const CountArgs& a, int s) {
  const int n = a.len ? a.len[s] : a.width;
  return n < 0 || n > a.width ? -1 : n;
}

__device__ __forceinline__ uint16_t counted(uint16_t word, uint32_t n, uint32_t flags) {
  if (flags & CO_COUNT_PROMPT) return word | 0x8000u;
  const uint32_t c = min((word & 0x7FFFu) + n, 0x7FFFu);
  return static_cast<uint16_t>((word & 0x8000u) | c);
}

// A tile of one sequence's words: the tokens that fall into it are counted in LDS, then
// the tile is written whole (a row that starts afresh), or its touched words are.  Every
// word has one writer.
__global__ __launch_bounds__(256) void count_tile_kernel(CountArgs a) {
  __shared__ uint32_t cnt[kTile];
  const int tid = threadIdx.x;
  const int tile = blockIdx.x % a.tiles, s = blockIdx.x / a.tiles;
  const int n = token_count(a, s);
  if (n < 0 && tile == 0 && tid == 0) set_status(a.status, CO_ERR_LENGTH);
  if (n <= 0) return;
  const int base = tile * kTile, here = min(kTile, a.V - base);
  for (int i = tid; i < here; i += 256) cnt[i] = 0;
  __syncthreads();
  const int32_t* tok = a.tokens + static_cast<int64_t>(s) * a.width;
  for (int i = tid; i < n; i += 256) {
    const int t = tok[i];
    if (t >= a.V) set_status(a.status, CO_ERR_TOKEN);
    else if (t >= base && t - base < here) atomicAdd(&cnt[t - base], 1u);
  }
  __syncthreads();
  uint16_t* row = a.seen + static_cast<int64_t>(s) * a.V + base;
  if (a.flags & CO_COUNT_FRESH) {
    for (int i = tid; i < here; i += 256) row[i] = cnt[i] ? counted(0, cnt[i], a.flags) : 0;
  } else {
    for (int i = tid; i < here; i += 256)
      if (cnt[i]) row[i] = counted(row[i], cnt[i], a.flags);
  }
}

// Up to 64 tokens of a sequence in one wavefront: the first lane of each token counts the
// others that hold it and writes its word.
__global__ __launch_bounds__(256) void count_few_kernel(CountArgs a) {
  const int lane = threadIdx.x & 63;
  const int s = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (s >= a.S) return;
  const int n = token_count(a, s);
  if (n < 0 && lane == 0) set_status(a.status, CO_ERR_LENGTH);
  if (n <= 0) return;
  int t = lane < n ? a.tokens[static_cast<int64_t>(s) * a.width + lane] : -1;
  if (t >= a.V) {
    set_status(a.status, CO_ERR_TOKEN);
    t = -1;
  }
  uint32_t same = 0;
  bool owner = t >= 0;
  for (int i = 0; i < n; ++i) {
    const bool eq = __builtin_amdgcn_readlane(t, i) == t;
    same += eq ? 1 : 0;
    if (eq && i < lane) owner = false;
  }
  if (owner) {
    uint16_t* w = a.seen + static_cast<int64_t>(s) * a.V + t;
    *w = counted(*w, same, a.flags);
  }
}

template <typename T>
hipError_t launch_rows(const LogitArgs& a, int kind, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.S) * a.tiles * a.groups)), block(256);
  if (kind == kRules) {
    hipLaunchKernelGGL((rows_kernel<T, kRules>), grid, block, 0, stream, a);
  } else {
    hipLaunchKernelGGL((rows_kernel<T, kStats>), grid, block, 0, stream, a);
    hipLaunchKernelGGL((rows_kernel<T, kProbs>), grid, block, 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace

LogitPlan plan_logits(int S, int R, int V, int num_cus) {
  LogitPlan p{};
  p.groups = (R + kRowsMax - 1) / kRowsMax;
  p.rows_per = (R + p.groups - 1) / p.groups;
  p.groups = (R + p.rows_per - 1) / p.rows_per;
  const int64_t all = (static_cast<int64_t>(V) + kChunk - 1) / kChunk;
  // as many chunks to a workgroup as leave eight workgroups to every compute unit
  int64_t chunks = all * S * p.groups / (8 * num_cus);
  chunks = chunks < 1 ? 1 : (chunks > 8 ? 8 : chunks);
  p.chunks = static_cast<int>(chunks);
  p.tiles = static_cast<int>((all + chunks - 1) / chunks);
  p.workgroups = static_cast<int64_t>(S) * p.groups * p.tiles;
  p.ws_bytes = (static_cast<size_t>(S) * R * p.tiles * sizeof(float4) + 255) / 256 * 256;
  return p;
}

hipError_t launch_logit_rules(const LogitArgs& a, int dtype, hipStream_t stream) {
  if (a.S == 0) return hipSuccess;
  return dtype == CO_DTYPE_BF16 ? launch_rows<uint16_t>(a, kRules, stream)
                                : launch_rows<float>(a, kRules, stream);
}

hipError_t launch_probabilities(const LogitArgs& a, int dtype, hipStream_t stream) {
  if (a.S == 0) return hipSuccess;
  return dtype == CO_DTYPE_BF16 ? launch_rows<uint16_t>(a, kProbs, stream)
                                : launch_rows<float>(a, kProbs, stream);
}

int64_t count_workgroups(int S, int V) {
  return static_cast<int64_t>(S) * ((static_cast<int64_t>(V) + kTile - 1) / kTile);
}

hipError_t launch_count_tokens(CountArgs a, hipStream_t stream) {
  if (a.S == 0 || a.width == 0) return hipSuccess;
  if (a.width <= 64 && !(a.flags & CO_COUNT_FRESH)) {
    hipLaunchKernelGGL(count_few_kernel, dim3((a.S + 3) / 4), dim3(256), 0, stream, a);
  } else {
    a.tiles = static_cast<int>((static_cast<int64_t>(a.V) + kTile - 1) / kTile);
    hipLaunchKernelGGL(count_tile_kernel, dim3(static_cast<unsigned>(count_workgroups(a.S, a.V))),
                       dim3(256), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace co
