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
// All of it is bound by memory: a logit is read and a logit or a probability written.  What
// is done for every token is therefore kept to a few operations: its mask bit, the largest
// value, an exponential.  The tokens that have a history, a proposal or a bias are special;
// there are hundreds of them among a hundred thousand, but several in every run that a
// wavefront takes, so that testing for them in place would run their code (a division among
// it) almost everywhere.  They are masked out of the run, listed once for a workgroup's tile
// and taken one each by its threads, as are the up to seven tokens behind the last whole
// vector of a row.
//
// Probabilities read a row of more than 16384 logits twice (largest logit and sum first).  One
// of 128000 fp32 logits takes all of a compute unit's registers; one of bf16 logits would fit
// (63 of the 128 that 1024 threads have each), which has not been measured.  Measured (kernels:
// averages under the profiler): rules on 64 rows of 128000 fp32 logits, about 1800 special
// tokens each, 20 us, 4.1 TB/s; on 8 rows of 32001 bf16 logits of 11 sequences 9.6 us, a chain
// of loads from the history to the first row.  Probabilities of 17 rows of 128000 bf16 logits
// for 32 sequences 142 us: first pass 62, second 81; without any rule 120, which is 4.6 TB/s
// over both passes.  The special tokens (1800 a sequence) are the rest: the
// first pass lists them for every four rows and leaves their marks and logits for the second.
#include "co_kernels.h"

namespace co {

namespace {

constexpr int kVec = 8;                     // tokens of a thread: one byte of a mask
// Such vectors of a thread: with four the two rows in flight take 141 to 153 registers, and
// three workgroups share a compute unit (rules on 64 x 128000 25.8 us, with two 21.6).
constexpr int kVecs = 2;
// Rows of a sequence that a workgroup takes: its special tokens' logits of all of them are in
// registers, and more workgroups share a compute unit the fewer they are, while each lists them
// once more (32 x 17 x 128000, probabilities, with 2 to 6 and 9 rows: 151, 144, 142, 160, 147,
// 169 us; 100 x 17 x 12000 with 2 to 5: 88, 86, 77, 88).
constexpr int kRowsMax = 4;

enum { kRules = 0, kStats = 1, kProbs = 2, kWhole = 3 };

constexpr float kNone = -INFINITY;

__device__ __forceinline__ float widen(uint16_t v) { return bf2f(v); }
__device__ __forceinline__ float widen(float v) { return v; }

// Eight elements next to each other, at any address of an element.
template <typename T>
struct Vec {
  typedef T vec __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
  vec x;
  __device__ __forceinline__ void load(const T* p) { x = *reinterpret_cast<const vec*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<vec*>(p) = x; }
};

// (Stores that bypass the caches are slower: a second pass of 98 us took 109.)
__device__ __forceinline__ void store8(float* p, const float (&x)[kVec]) {
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
  *reinterpret_cast<vec*>(p) = vec{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<vec*>(p + 4) = vec{x[4], x[5], x[6], x[7]};
}

__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(uint16_t* p, float x) { *p = static_cast<uint16_t>(cvt_pk_bf16(x, x)); }

template <typename T> constexpr T kLowest = T(-INFINITY);
template <> constexpr uint16_t kLowest<uint16_t> = 0xFF80u;

// y where bit e of `allowed` is set, minus infinity elsewhere: a bit field extract and an
// insert (written out, the compiler makes five operations of the latter).
__device__ __forceinline__ float masked(float y, uint32_t allowed, int e) {
  const int m = __builtin_amdgcn_sbfe(static_cast<int>(allowed), e, 1);
  float r;
  asm("v_bfi_b32 %0, %1, %2, %3" : "=v"(r) : "v"(m), "v"(y), "v"(kNone));
  return r;
}

// The same for 16-bit logits two at a time; m: all ones where a token is allowed.
__device__ __forceinline__ uint32_t masked2(uint32_t x, uint32_t m) {
  uint32_t r;
  asm("v_bfi_b32 %0, %1, %2, %3" : "=v"(r) : "v"(m), "v"(x), "v"(0xFF80FF80u));
  return r;
}
__device__ __forceinline__ uint32_t pair_mask(uint32_t allowed, int pair) {
  return (allowed >> (2 * pair) & 1 ? 0xFFFFu : 0u) | (allowed >> (2 * pair + 1) & 1 ? 0xFFFF0000u : 0u);
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

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// log2(e) / T, kept finite and above 0; greedy sequences (T <= 0 or NaN) have any.
__device__ __forceinline__ float row_slope(const float* temperature, int s, bool* greedy) {
  const float t = temperature ? temperature[s] : 1.f;
  *greedy = !(t > 0.f);
  return *greedy ? 1.f : fminf(fmaxf(1.44269504088896341f / t, 0x1p-126f), 0x1.fffffep+127f);
}

// What a part of a row holds: its largest logit, the sum of exp2((x - m) k), and where the
// largest is: the first vector of eight that has it, and the first special token that is it
// (INT32_MAX: none).
struct Part {
  float m, l;
  int vec, one;
};

constexpr int kNowhere = INT32_MAX;

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, false));
}

__device__ __forceinline__ float wave_max_f(float v) {
  v = fmaxf(v, dpp<0x128>(v));   // rotations within 16 lanes: by 8, 4, 2, 1
  v = fmaxf(v, dpp<0x124>(v));
  v = fmaxf(v, dpp<0x122>(v));
  v = fmaxf(v, dpp<0x121>(v));
  return max_across_rows(v);
}

__device__ __forceinline__ float wave_sum_f(float v) {
  v += dpp<0x128>(v);
  v += dpp<0x124>(v);
  v += dpp<0x122>(v);
  v += dpp<0x121>(v);
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ int wave_min(int v) { return INT32_MAX - wave_max(INT32_MAX - v); }

// The wavefront's parts joined, in every lane.
__device__ __forceinline__ Part wave_join(const Part& p, float k) {
  Part r;
  r.m = wave_max_f(p.m);
  // (equal largest values, infinite ones among them, keep their sums as they are)
  r.l = wave_sum_f(p.m == r.m ? p.l : p.l * exp2_fast((p.m - r.m) * k));
  r.vec = wave_min(p.m == r.m ? p.vec : kNowhere);
  r.one = wave_min(p.m == r.m ? p.one : kNowhere);
  return r;
}

// One more special token.  A NaN is left out, as if it were masked.
__device__ __forceinline__ void take(Part& p, float y, int v, float k) {
  if (y > p.m) {
    p.l = p.m > kNone ? p.l * exp2_fast((p.m - y) * k) : 0.f;
    p.m = y;
    p.one = v;
  } else if (y == p.m) {
    p.one = min(p.one, v);
  }
  if (y > kNone) p.l += y == p.m ? 1.f : exp2_fast((y - p.m) * k);
}

// A row's largest logit, one over its sum (0: nothing left) and its lowest largest token.
struct Whole {
  float m, inv;
  int at;
};

template <int N>
__device__ __forceinline__ void shares(const Whole& p, float (&y)[N], int v, float k, bool greedy) {
  if (greedy || p.m == INFINITY || p.inv == 0.f) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      y[e] = p.inv == 0.f ? 0.f : (greedy ? (v + e == p.at ? 1.f : 0.f) : (y[e] == p.m ? p.inv : 0.f));
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] = fmaxf(exp2_fast((y[e] - p.m) * k) * p.inv, 0.f);   // (NaN: 0)
}

// A special token of a tile.
struct Entry {
  int v;                 // token
  uint32_t word;         // its history
  float bias;
  bool biased;
  uint32_t proposed[2];  // bit i: the window's proposal i is this token (of the first 64)
};

// The biased tokens of a tile are found again by a table in LDS: place of a token, then the next
// ones.  Lists of more tokens than such steps find are walked (us for 16 rows of 4886 tokens and
// up to 300 biases, two sequences: walked 104, by the table 15; 17
// rows of 2919 with every rule, 113 sequences: 217, 72).  Every biased token of a tile walks the
// whole list there, so that its time is tokens times entries (one row of 128000 tokens with 300,
// 8000, 16000, 32000 and 128000 different biased tokens: rules 6, 21, 890, 3000, 36000 us,
// probabilities twice that).
constexpr int kSteps = 32;
template <int SLOTS>
__device__ __forceinline__ int slot_of(int t) {
  return static_cast<int>(static_cast<uint32_t>(t) * 2654435769u >> 20) & (SLOTS - 1);
}

// One workgroup: a tile of tokens of one sequence, C vectors of eight a thread, in rows one
// after the other, the next row's logits in flight.
// Special tokens of all rows come first, so that the rows' loop has nothing to wait for but
// its own loads.  kProbs finds up to NT of them in the workspace (at six rows a workgroup
// the call above takes 147 us; 160 when it listed them again, and one sequence of 17 rows 19.0 in
// place of 16.8); it lists those of a
// tile that has more.
//   kRules: rules on logits.  kStats: each tile's largest logit and sum; kProbs: the tiles'
//   parts joined, and the probabilities.  kWhole: both, where a row is one tile.
template <typename T, int KIND, int NT, int C>
__global__ __launch_bounds__(NT) void rows_kernel(LogitArgs a) {
  constexpr int kTokens = NT * kVec * C, kWaves = NT / 64, kBlock = 64 * kVec;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int b = blockIdx.x;
  const int grp = b % a.groups;
  b /= a.groups;
  const int tile = b % a.tiles, s = b / a.tiles;
  const int j0 = grp * a.rows_per, nr = min(a.rows_per, a.R - j0);
  const int V = a.V;
  const int64_t row0 = static_cast<int64_t>(s) * a.R + j0;
  const T* logits = static_cast<const T*>(a.logits) + row0 * V;
  const bool reports = KIND != kProbs && tile == 0 && grp == 0;   // what concerns a sequence

  __shared__ uint32_t special[kTokens / 32], with_bias[kTokens / 32];   // a bit a token
  __shared__ uint16_t list[kTokens];
  constexpr int kSlots = NT == 1024 ? 4096 : 512;
  __shared__ int bias_key[kSlots], bias_order[kSlots];   // token of the tile, its last entry
  __shared__ int walked, listed[kWaves];                 // walked: not all found a place
  constexpr int kParts = KIND == kStats || KIND == kWhole ? kRowsMax * kWaves : 1;
  __shared__ Part parts[kParts];                 // of the wavefronts
  constexpr int kLanes = KIND == kStats || KIND == kWhole ? kRowsMax * NT : 1;
  __shared__ float one_m[kLanes], one_l[kLanes]; // of each thread's special tokens
  __shared__ int one_at[kLanes];
  __shared__ Whole whole[kRowsMax];
  __shared__ float own_special[KIND == kRules || KIND == kProbs ? kRowsMax * NT : 1];
  bool greedy = false;
  const float k = KIND == kRules ? 0.f : row_slope(a.temperature, s, &greedy);

  // Vector c of this thread: whole where full(c); others are loaded from the row's last whole
  // one, so that no load is behind a branch, and masked.
  // Tiles interleave in blocks of a wavefront's 512 tokens: frequent tokens have low numbers,
  // and a tile of them alone would have most of the special ones (32 x 17 x 128000: tiles of
  // tokens next to each other 183 us, interleaved 171, with 16-bit logits masked in pairs).
  auto vec = [&](int c) { return ((c * kWaves + wave) * a.tiles + tile) * kBlock + lane * kVec; };
  auto token_of = [&](int t) { return ((t / kBlock) * a.tiles + tile) * kBlock + t % kBlock; };
  auto in_tile = [&](int v) {   // the inverse; -1: another tile's
    const int b = v / kBlock;
    return b % a.tiles == tile ? b / a.tiles * kBlock + v % kBlock : -1;
  };
  auto full = [&](int c) { return vec(c) + kVec <= V; };
  auto at_vec = [&](int c) { return min(vec(c), V - kVec); };
  const bool vectors = V >= kVec;
  const int64_t mask_bytes = static_cast<int64_t>((V + 31) / 32) * 4;
  // What hangs on nothing but the indices is loaded first, all at once.
  int mask_held = a.mask_row && lane < nr ? a.mask_row[row0 + lane] : -1;
  const uint16_t* seen = a.seen ? a.seen + static_cast<int64_t>(s) * V : nullptr;
  const int32_t* draft = a.draft && a.seen ? a.draft + static_cast<int64_t>(s) * a.B : nullptr;
  const int before = draft ? j0 + nr - 1 : 0;              // proposals that some row has behind it
  const int held = lane < before ? draft[lane] : -1;       // lane i holds number i, later ones are read
  int b0 = 0, b1 = 0;
  if (a.bias_start) {
    b0 = a.bias_start[s];
    b1 = a.bias_start[s + 1];
  }
  Vec<uint16_t> w[C];
  auto load_history = [&]() {
    if (seen && vectors) {
#pragma unroll
      for (int c = 0; c < C; ++c) w[c].load(seen + at_vec(c));
    }
  };
  // kProbs: the marks of special tokens are those of the pass before (where there is nothing to
  // mark but the tokens behind the last vector, they are made again: no load to wait for)
  const bool kept = a.seen || a.bias_start;
  uint8_t* marks = a.marks + static_cast<int64_t>(blockIdx.x) * (kTokens / 8) + tid;
  uint32_t mine[C];           // of this thread's vectors
  if (KIND == kProbs && kept) {
#pragma unroll
    for (int c = 0; c < C; ++c) mine[c] = marks[c * NT];
  }
  if constexpr (KIND != kProbs) load_history();
  struct Row {
    Vec<T> x[C];
    uint32_t allowed[C];   // (words: bytes would be packed, and waited for, as they arrive)
  };
  auto load = [&](int r, Row& o) {
    if (!vectors) return;
    const T* p = logits + static_cast<int64_t>(r) * V;
#pragma unroll
    for (int c = 0; c < C; ++c) o.x[c].load(p + at_vec(c));
  };
  Row cur, next;
  load(0, cur);
  const float rep = a.repetition ? a.repetition[s] : 1.f;
  const float freq = a.frequency ? a.frequency[s] : 0.f;
  const float pres = a.presence ? a.presence[s] : 0.f;

  // lane r holds the mask of row r: >= 0, or -1: none, -2: no such mask, nothing is allowed
  mask_held = max(-1, mask_held);
  if (mask_held >= a.num_masks) {
    mask_held = -2;
    if (KIND != kProbs) set_status(a.status, CO_ERR_MASK);
  }
  auto mask_of = [&](int r) { return __builtin_amdgcn_readlane(mask_held, r); };
  auto bits_of = [&](int m) { return reinterpret_cast<const uint8_t*>(a.mask_bits) + m * mask_bytes; };
  auto load_mask = [&](int r, Row& o) {
    // (what is so without a mask first: written behind a branch, it would wait for every load in
    // flight: at six rows a workgroup 153 us for the call above, 147 so)
    const int m = mask_of(r);
    uint32_t without = m == -1 ? 0xFF : 0;
    asm volatile("" : "+v"(without));
#pragma unroll
    for (int c = 0; c < C; ++c) o.allowed[c] = without;
    if (m >= 0 && vectors) {
      const uint8_t* bits = bits_of(m);
#pragma unroll
      for (int c = 0; c < C; ++c) o.allowed[c] = bits[at_vec(c) / kVec];
    }
  };
  load_mask(0, cur);

  // ---- the tile's special tokens
  auto proposal_held = [&](int i) { return i == lane && i < before ? held : draft[i]; };
  const bool right = b0 >= 0 && b1 >= b0 && b1 <= a.num_bias;
  if (!right && reports && tid == 0) set_status(a.status, CO_ERR_LENGTH);
  const int n_bias = right ? b1 - b0 : 0;
  uint8_t* special8 = reinterpret_cast<uint8_t*>(special);
  int own_tok = -1;           // of bias number tid
  if (KIND != kProbs && tid < n_bias) own_tok = a.bias_tok[b0 + tid];
  // Marks them, with those that have a bias.
  auto mark = [&]() {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      uint32_t m = 0;
      if (full(c)) {
        if (seen) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) m |= (w[c].x[e] != 0 ? 1u : 0u) << e;
        }
      } else if (vec(c) < V) {
        m = (1u << (V - vec(c))) - 1;
      }
      special8[c * NT + tid] = static_cast<uint8_t>(m);
      reinterpret_cast<uint8_t*>(with_bias)[c * NT + tid] = 0;
    }
    if (tid == 0) walked = 0;
    if (n_bias > 0) {
      for (int i = tid; i < kSlots; i += NT) bias_key[i] = bias_order[i] = -1;
    }
    if (n_bias > 0 || draft) {
      __syncthreads();
      for (int i = tid; i < (reports && draft ? a.R - 1 : before); i += NT) {
        const int d = proposal_held(i);
        if (static_cast<uint32_t>(d) >= static_cast<uint32_t>(V)) {
          if (reports) set_status(a.status, CO_ERR_TOKEN);
        } else if (i < before) {
          const int t = in_tile(d);
          if (t >= 0) atomicOr(&special[t >> 5], 1u << (t & 31));
        }
      }
      for (int i = tid; i < n_bias; i += NT) {
        const int d = KIND != kProbs && i == tid ? own_tok : a.bias_tok[b0 + i];
        if (static_cast<uint32_t>(d) >= static_cast<uint32_t>(V)) {
          if (reports) set_status(a.status, CO_ERR_TOKEN);
        } else if (const int t = in_tile(d); t >= 0) {
          atomicOr(&special[t >> 5], 1u << (t & 31));
          atomicOr(&with_bias[t >> 5], 1u << (t & 31));
          int h = slot_of<kSlots>(t), step = 0;
          for (; step < kSteps; ++step) {
            const int was = atomicCAS(&bias_key[h], -1, t);
            if (was == -1 || was == t) break;
            h = (h + 1) & (kSlots - 1);
          }
          if (step < kSteps) atomicMax(&bias_order[h], i);
          else walked = 1;
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) mine[c] = special8[c * NT + tid];
  };
  if (KIND != kProbs || !kept) mark();
  uint32_t plain[C];          // tokens of a vector that are not special
  int own = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    plain[c] = full(c) ? mine[c] ^ 0xFF : 0;
    own += __builtin_popcount(mine[c]);
  }
  uint32_t pairs[sizeof(T) == 2 ? C : 1][4];   // 16-bit logits: the masks of `plain`
  if constexpr (sizeof(T) == 2 && KIND != kRules) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int q = 0; q < 4; ++q) pairs[c][q] = pair_mask(vectors ? plain[c] : 0, q);
  }
  const int upto = wave_scan(own);
  if (lane == 63) listed[wave] = upto;
  __syncthreads();
  int start = upto - own, n = 0;   // of this thread's tokens in the list
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    start += w < wave ? listed[w] : 0;
    n += listed[w];
  }
  if (KIND != kProbs || n > NT) {
    if constexpr (KIND == kProbs) {   // (the list is walked again behind the rows)
      load_history();
      mark();
    }
    int at = start;
#pragma unroll
    for (int c = 0; c < C; ++c)
      for (uint32_t m = mine[c]; m != 0; m &= m - 1)
        list[at++] = static_cast<uint16_t>((c * NT + tid) * kVec + __builtin_ctz(m));
    __syncthreads();
  }

  // number i of the list; the last entry of a token in the list of biases counts
  auto entry = [&](int i) {
    Entry e{};
    const int t = list[i];
    e.v = token_of(t);
    e.word = seen ? seen[e.v] : 0;
    e.biased = with_bias[t >> 5] >> (t & 31) & 1;
    if (e.biased) {
      int order = -1;
      if (walked == 0) {
        int h = slot_of<kSlots>(t);
        for (int step = 0; step < kSteps && bias_key[h] != t; ++step) h = (h + 1) & (kSlots - 1);
        order = bias_order[h];
      } else {
#pragma unroll 8
        for (int j = 0; j < n_bias; ++j) order = a.bias_tok[b0 + j] == e.v ? j : order;
      }
      e.bias = a.bias_val[b0 + order];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
      for (int j = 32 * h; j < min(before, 32 * h + 32); ++j)
        e.proposed[h] |= __builtin_amdgcn_readlane(held, j) == e.v ? 1u << (j & 31) : 0;
    return e;
  };
  // its logit x after the rules, in row r; `allowed`: its byte of the row's mask
  auto ruled = [&](const Entry& e, int r, float x, uint32_t allowed) {
    const int j = j0 + r;       // proposals behind the row
    uint32_t count = e.word & 0x7FFFu;
    count += __builtin_popcount(e.proposed[0] & (j < 32 ? (1u << j) - 1 : ~0u));
    if (j > 32) count += __builtin_popcount(e.proposed[1] & (j < 64 ? (1u << (j - 32)) - 1 : ~0u));
    for (int i = 64; i < (draft ? j : 0); ++i) count += draft[i] == e.v ? 1 : 0;
    if (e.word != 0 || count != 0) x = penalise(x, static_cast<int>(min(count, 0x7FFFu)), rep, freq, pres);
    if (e.biased) x = x + e.bias;
    return allowed >> (e.v % 8) & 1 ? x : kNone;
  };
  // Every special token of this wavefront's share (one a lane, the rest idle) in every row:
  // f(r, number in the list, token, its logit after the rules).  Its logits and mask bytes of
  // all rows are loaded together.
  auto each_special = [&](int from, int to, auto&& f) {
    for (int i0 = from + wave * 64; i0 < to; i0 += NT) {
      const bool on = i0 + lane < n;
      const Entry e = entry(min(i0 + lane, n - 1));   // (by all lanes: it reads across them)
      T x[kRowsMax];
      uint32_t allowed[kRowsMax];
#pragma unroll
      for (int q = 0; q < kRowsMax; ++q) x[q] = logits[static_cast<int64_t>(min(q, nr - 1)) * V + e.v];
#pragma unroll
      for (int q = 0; q < kRowsMax; ++q) allowed[q] = 0xFF;
      if (a.mask_row && a.num_masks > 0) {   // (rows without a mask read the first one's)
#pragma unroll
        for (int q = 0; q < kRowsMax; ++q) allowed[q] = bits_of(max(0, mask_of(min(q, nr - 1))))[e.v / 8];
      }
#pragma unroll 1
      for (int r = 0; r < nr; ++r) {
        T xr = x[0];
        uint32_t ar = allowed[0];
#pragma unroll
        for (int q = 1; q < kRowsMax; ++q) {
          xr = q == r ? x[q] : xr;
          ar = q == r ? allowed[q] : ar;
        }
        const int m = mask_of(r);
        const float y = ruled(e, r, widen(xr), m >= 0 ? ar : (m == -1 ? 0xFF : 0));
        if (on) f(r, i0 + lane, e.v, y);
      }
    }
  };

  // Which token a part's largest is, by the lanes of a wavefront: the first of its vector's
  // eight that is neither masked nor special, or a special one before it.
  auto place = [&](const Part& p, int r) {
    if (p.vec == kNowhere) return p.one;
    const int v = p.vec + (lane & 7), t = in_tile(v), m = mask_of(r);
    const uint32_t allowed = m >= 0 ? bits_of(m)[v / 8] >> (v % 8) & 1 : (m == -1 ? 1 : 0);
    const bool is = allowed && !(special[t >> 5] >> (t & 31) & 1) &&
                    widen(logits[static_cast<int64_t>(r) * V + v]) == p.m;
    const unsigned long long found = __ballot(is) & 0xFF;
    return min(p.one, p.vec + __ffsll(static_cast<long long>(found)) - 1);
  };
  const Part nothing{kNone, 0.f, kNowhere, kNowhere};
  if constexpr (KIND == kProbs) {
    // the rows' parts joined
    for (int r = wave; r < nr; r += kWaves) {
      Part p = nothing;
      for (int t = lane; t < a.tiles; t += 64) {
        const float4 w = a.ws[(row0 + r) * a.tiles + t];
        const int at = __float_as_int(w.z);
        if (w.x > p.m) {
          p.l = p.m > kNone ? p.l * exp2_fast((p.m - w.x) * k) : 0.f;
          p.m = w.x;
          p.one = at;
        } else if (w.x == p.m) {
          p.one = min(p.one, at);
        }
        if (w.x > kNone) p.l += w.x == p.m ? w.y : w.y * exp2_fast((w.x - p.m) * k);
      }
      p = wave_join(p, k);
      if (lane == 0) {
        whole[r] = Whole{p.m, p.m > kNone ? 1.f / p.l : 0.f, p.one};
        if (tile == 0 && a.top) a.top[row0 + r] = p.m > kNone ? p.one : -1;
      }
    }
    __syncthreads();
  }

  if constexpr (KIND == kStats || KIND == kWhole) {
    // (a thread has every NT-th of the list, and joins them by itself)
    each_special(0, n, [&](int r, int i, int v, float y) {
      const int o = r * NT + tid;
      Part p = nothing;
      if (i >= NT) p = Part{one_m[o], one_l[o], kNowhere, one_at[o]};
      take(p, y, v, k);
      one_m[o] = p.m;
      one_l[o] = p.l;
      one_at[o] = p.one;
    });
  }
  auto result = [&](int r, int v, float x) {
    if constexpr (KIND == kRules) return x;
    float y[1] = {x};
    shares(whole[r], y, v, k, greedy);
    return y[0];
  };
  // The first NT special tokens after the rules wait in LDS, row by row, for the thread that
  // stores the vectors that hold them.  It stores rules behind its own vector (later, the lines
  // that they lie in would be in memory already, and be fetched to be changed); probabilities it
  // puts into the vector before.  (Either is slower the other way: rules on 64 x 128000 bf16
  // 17.3 us, 16.0; probabilities of 32 x 17 x 128000 164, 160.)
  auto each_own = [&](int r, int c, auto&& f) {   // f(place in vector c, logit)
    int i = start;
#pragma unroll
    for (int b = 0; b < C; ++b) i += b < c ? __builtin_popcount(mine[b]) : 0;
    for (uint32_t m = mine[c]; m != 0 && i < NT; m &= m - 1, ++i) f(__builtin_ctz(m), own_special[r * NT + i]);
  };
  if constexpr (KIND == kProbs) {   // the first pass left them
    float y[kRowsMax];
    if (n > NT) {
      each_special(0, NT, [&](int r, int i, int, float x) { own_special[r * NT + i] = x; });
    } else if (tid < n) {
#pragma unroll
      for (int q = 0; q < kRowsMax; ++q) y[q] = a.ruled[((row0 + min(q, nr - 1)) * a.tiles + tile) * NT + tid];
#pragma unroll
      for (int q = 0; q < kRowsMax; ++q) own_special[q * NT + tid] = y[q];
    }
    __syncthreads();
  }

  // kRules, kProbs: the first NT special tokens before the rows, the others behind them
#pragma unroll 1
  for (int phase = 0; phase < (KIND == kStats ? 1 : 2); ++phase) {
    if constexpr (KIND == kRules) {
      if (phase == 0) {
        each_special(0, min(n, NT), [&](int r, int i, int, float x) { own_special[r * NT + i] = x; });
        __syncthreads();
      }
    }
    if (KIND != kStats && phase == 1) {
      each_special(KIND == kWhole ? 0 : NT, n, [&](int r, int, int v, float x) {
        const float y = result(r, v, x);
        if constexpr (KIND == kRules) store1(static_cast<T*>(a.out) + (row0 + r) * V + v, y);
        else a.probs[(row0 + r) * V + v] = y;
      });
      break;
    }
#pragma unroll 1
    for (int r = 0; r < nr; ++r) {
      if (r + 1 < nr) {
        load(r + 1, next);
        load_mask(r + 1, next);
      }
      T* out = static_cast<T*>(a.out) + (row0 + r) * V;
      float* probs = a.probs + (row0 + r) * V;
      if constexpr (KIND == kRules) {
        // what is not special is forbidden or stays as it is (where it is, in place)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if (!full(c)) continue;
          const uint32_t allowed = (cur.allowed[c] | ~plain[c]) & 0xFF;
          if (allowed == 0xFF && out == logits + static_cast<int64_t>(r) * V) continue;
#pragma unroll
          for (int e = 0; e < kVec; ++e) cur.x[c].x[e] = allowed >> e & 1 ? cur.x[c].x[e] : kLowest<T>;
          cur.x[c].store(out + vec(c));
        }
      } else {
        float y[C][kVec], top = kNone;
        int where = kNowhere;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if constexpr (sizeof(T) == 2) {
            typedef uint16_t plain8 __attribute__((ext_vector_type(8)));
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            const u32x4 x = __builtin_bit_cast(u32x4, static_cast<plain8>(cur.x[c].x));
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const uint32_t z = masked2(x[q], pairs[c][q]);
              y[c][2 * q] = __uint_as_float(z << 16);
              y[c][2 * q + 1] = __uint_as_float(z & 0xFFFF0000u);
            }
            if (mask_of(r) != -1) {
#pragma unroll
              for (int e = 0; e < kVec; ++e) y[c][e] = masked(y[c][e], cur.allowed[c], e);
            }
          } else {
            const uint32_t allowed = vectors ? cur.allowed[c] & plain[c] : 0;
#pragma unroll
            for (int e = 0; e < kVec; ++e) y[c][e] = widen(cur.x[c].x[e]);
            if (__any(allowed != 0xFF)) {
#pragma unroll
              for (int e = 0; e < kVec; ++e) y[c][e] = masked(y[c][e], allowed, e);
            }
          }
          if constexpr (KIND == kProbs) {
            if (full(c)) {
              each_own(r, c, [&](int at, float x) {
#pragma unroll
                for (int e = 0; e < kVec; ++e) y[c][e] = e == at ? x : y[c][e];
              });
              shares(whole[r], y[c], vec(c), k, greedy);
              store8(probs + vec(c), y[c]);
            } else {
              each_own(r, c, [&](int e, float x) { probs[vec(c) + e] = result(r, vec(c) + e, x); });
            }
          } else {
            float most = y[c][0];
#pragma unroll
            for (int e = 1; e < kVec; ++e) most = fmaxf(most, y[c][e]);
            where = most > top ? vec(c) : where;
            top = fmaxf(top, most);
          }
        }
        if constexpr (KIND != kProbs) {
          Part p = nothing;   // of this thread's special tokens
          if (tid < n) p = Part{one_m[r * NT + tid], one_l[r * NT + tid], kNowhere, one_at[r * NT + tid]};
          Part w;   // the wavefront's
          w.m = wave_max_f(fmaxf(top, p.m));
          w.l = 0.f;
          if (__builtin_amdgcn_readfirstlane(w.m > kNone)) {
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
              for (int e = 0; e < kVec; ++e) sum += exp2_fast((y[c][e] - w.m) * k);
            if (sum != sum) {   // a NaN, or infinities, which count 1 each
              sum = 0.f;
#pragma unroll
              for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                  if (y[c][e] == y[c][e]) sum += y[c][e] == w.m ? 1.f : exp2_fast((y[c][e] - w.m) * k);
            }
            if (p.m > kNone) sum += p.m == w.m ? p.l : p.l * exp2_fast((p.m - w.m) * k);
            w.l = wave_sum_f(sum);
          }
          w.vec = wave_min(top == w.m ? where : kNowhere);
          w.one = wave_min(p.m == w.m ? p.one : kNowhere);
          if (lane == 0) parts[r * kWaves + wave] = w;
          if constexpr (KIND == kWhole) {
            __syncthreads();
            const Part q = wave_join(lane < kWaves ? parts[r * kWaves + lane] : nothing, k);
            const int at = q.m > kNone ? place(q, r) : -1;
            const Whole all{q.m, q.m > kNone ? 1.f / q.l : 0.f, at};
            if (tid == 0) {
              whole[r] = all;
              if (a.top) a.top[row0 + r] = at;
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
              if (!full(c)) continue;
              shares(all, y[c], vec(c), k, greedy);
              store8(probs + vec(c), y[c]);
            }
          }
        }
      }
      if constexpr (KIND == kRules) {
#pragma unroll
        for (int c = 0; c < C; ++c) each_own(r, c, [&](int e, float x) { store1(out + vec(c) + e, x); });
      }
      cur = next;
    }
    __syncthreads();
    if ((KIND == kRules || KIND == kProbs) && n <= NT) break;
  }

  if constexpr (KIND == kStats) {
    if (kept) {
#pragma unroll
      for (int c = 0; c < C; ++c) marks[c * NT] = special8[c * NT + tid];
    }
    if (n <= NT && tid < n)
      for (int r = 0; r < nr; ++r) a.ruled[((row0 + r) * a.tiles + tile) * NT + tid] = one_m[r * NT + tid];
    for (int r = wave; r < nr; r += kWaves) {
      const Part p = wave_join(lane < kWaves ? parts[r * kWaves + lane] : nothing, k);
      const int at = p.m > kNone ? place(p, r) : kNowhere;
      if (lane == 0) a.ws[(row0 + r) * a.tiles + tile] = float4{p.m, p.l, __int_as_float(at), 0.f};
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

// Every token of a sequence, four to a load where they are aligned: f(token).
template <int NT, typename F>
__device__ __forceinline__ void each_token(const int32_t* tok, int n, F&& f) {
  const int tid = threadIdx.x;
  int done = 0;
  if ((reinterpret_cast<uintptr_t>(tok) & 15) == 0) {
    const int4* four = reinterpret_cast<const int4*>(tok);
    for (int i = tid; i < n / 4; i += NT) {
      const int4 t = four[i];
      f(t.x);
      f(t.y);
      f(t.z);
      f(t.w);
    }
    done = n & ~3;
  }
  for (int i = done + tid; i < n; i += NT) f(tok[i]);
}

// Bound by writing the words of fresh rows (2 bytes a token of the vocabulary), and by the
// latency of a launch otherwise: 64 prompts of up to 8192 of 128000 tokens 6.2 us, 2.7 TB/s.
//
// A tile of one sequence's words: the tokens that fall into it are counted in LDS, then the
// tile is written whole (a row that starts afresh), or its touched words are.  Every word
// has one writer, and whole numbers are added, so the order does not matter.
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
  each_token<256>(a.tokens + static_cast<int64_t>(s) * a.width, n, [&](int t) {
    if (t >= a.V) set_status(a.status, CO_ERR_TOKEN);
    else if (t >= base && t - base < here) atomicAdd(&cnt[t - base], 1u);
  });
  __syncthreads();
  uint16_t* row = a.seen + static_cast<int64_t>(s) * a.V + base;
  for (int i = tid; i < here; i += 256) {
    const uint16_t old = a.flags & CO_COUNT_FRESH || !cnt[i] ? 0 : row[i];
    if (cnt[i]) row[i] = counted(old, cnt[i], 0);
    else if (a.flags & CO_COUNT_FRESH) row[i] = 0;
  }
}

// The same for prompts, of which a bit a token is all there is to know: tiles of up to
// 65536 tokens, so that the tokens are read few times over.
constexpr int kPromptTile = 65536;

__global__ __launch_bounds__(512) void mark_tile_kernel(CountArgs a, int size) {
  __shared__ uint32_t bits[kPromptTile / 32];
  const int tid = threadIdx.x;
  const int tile = blockIdx.x % a.tiles, s = blockIdx.x / a.tiles;
  const int n = token_count(a, s);
  if (n < 0 && tile == 0 && tid == 0) set_status(a.status, CO_ERR_LENGTH);
  if (n <= 0) return;
  const int base = tile * size, here = min(size, a.V - base);
  for (int i = tid; i < size / 32; i += 512) bits[i] = 0;
  __syncthreads();
  each_token<512>(a.tokens + static_cast<int64_t>(s) * a.width, n, [&](int t) {
    if (t >= a.V) set_status(a.status, CO_ERR_TOKEN);
    else if (t >= base && t - base < here) atomicOr(&bits[(t - base) >> 5], 1u << (t & 31));
  });
  __syncthreads();
  uint16_t* row = a.seen + static_cast<int64_t>(s) * a.V + base;
  const uint8_t* byte = reinterpret_cast<const uint8_t*>(bits);
  if (a.flags & CO_COUNT_FRESH) {
    for (int i = tid; i < here / kVec; i += 512) {
      Vec<uint16_t> w;
#pragma unroll
      for (int e = 0; e < kVec; ++e) w.x[e] = static_cast<uint16_t>((byte[i] >> e & 1) << 15);
      w.store(row + i * kVec);
    }
    for (int i = (here & ~(kVec - 1)) + tid; i < here; i += 512)
      row[i] = static_cast<uint16_t>((bits[i >> 5] >> (i & 31) & 1) << 15);
  } else {
    for (int i = tid; i < (here + 31) / 32; i += 512)
      for (uint32_t m = bits[i]; m != 0; m &= m - 1) row[32 * i + __builtin_ctz(m)] |= 0x8000u;
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
hipError_t launch_rows(const LogitArgs& a, bool rules, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.S) * a.tiles * a.groups));
  if (rules) {
    hipLaunchKernelGGL((rows_kernel<T, kRules, 256, kVecs>), grid, dim3(256), 0, stream, a);
  } else if (a.tiles == 1 && a.V <= 256 * kVec) {
    hipLaunchKernelGGL((rows_kernel<T, kWhole, 256, 1>), grid, dim3(256), 0, stream, a);
  } else if (a.tiles == 1) {
    hipLaunchKernelGGL((rows_kernel<T, kWhole, 1024, 2>), grid, dim3(1024), 0, stream, a);
  } else {
    hipLaunchKernelGGL((rows_kernel<T, kStats, 256, kVecs>), grid, dim3(256), 0, stream, a);
    hipLaunchKernelGGL((rows_kernel<T, kProbs, 256, kVecs>), grid, dim3(256), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace

LogitPlan plan_logits(int S, int R, int V, int num_cus, bool rules) {
  LogitPlan p{};
  // rows that one workgroup holds take one launch and are read once (us by tiles, whole:
  // 1 x 17 x 16000 22.2, 21.1; 32 x 17 x 16000 61.2, 52.8; 32 x 17 x 4000 42.3, 40.6)
  const bool whole = !rules && V <= 1024 * kVec * 2;
  const int tile = whole ? V : 256 * kVec * kVecs;
  p.threads = whole && V > 256 * kVec ? 1024 : 256;
  p.tiles = static_cast<int>((static_cast<int64_t>(V) + tile - 1) / tile);
  // Rows together (what is special is listed once for them) as long as so many workgroups are
  // left to every compute unit: tiles 4 (us at 1, 4, 16, bf16 rows by tokens with 2000 tokens of
  // history: 4 x 17 x 128000 41.9, 36.0, 40.4; 8 x 17 x 32000 39.4, 31.2, 31.1), rows whole 1 of
  // 1024 threads (at 1, 2, 4: 32 x 17 x 4000 40.4, 46.9, 46.9; 100 x 17 x 12000 96.4, 91.9, 126.5)
  // or 2 of 256 (100 x 17 x 1000 35.2, 28.3, 31.7).
  const int left = !whole ? 4 : (p.threads == 1024 ? 1 : 2);
  int64_t per = static_cast<int64_t>(p.tiles) * S * R / (left * num_cus);
  per = per < 1 ? 1 : (per > kRowsMax ? kRowsMax : per);
  p.groups = (R + static_cast<int>(per) - 1) / static_cast<int>(per);
  p.rows_per = (R + p.groups - 1) / p.groups;
  p.groups = (R + p.rows_per - 1) / p.rows_per;
  p.workgroups = static_cast<int64_t>(S) * p.groups * p.tiles;
  // parts of the rows; where there are several, also marks and values of special tokens
  const size_t parts = static_cast<size_t>(S) * R * p.tiles;
  p.marks_at = (parts * sizeof(float4) + 255) / 256 * 256;
  p.ruled_at = p.marks_at + (whole ? 0 : static_cast<size_t>(p.workgroups) * (tile / 8));
  p.ws_bytes = p.ruled_at + (whole ? 0 : parts * 256 * sizeof(float));
  return p;
}

hipError_t launch_logit_rules(const LogitArgs& a, int dtype, hipStream_t stream) {
  if (a.S == 0) return hipSuccess;
  return dtype == CO_DTYPE_BF16 ? launch_rows<uint16_t>(a, true, stream) : launch_rows<float>(a, true, stream);
}

hipError_t launch_probabilities(const LogitArgs& a, int dtype, hipStream_t stream) {
  if (a.S == 0) return hipSuccess;
  return dtype == CO_DTYPE_BF16 ? launch_rows<uint16_t>(a, false, stream) : launch_rows<float>(a, false, stream);
}

int64_t count_workgroups(int S, int V) {
  return static_cast<int64_t>(S) * ((static_cast<int64_t>(V) + kTile - 1) / kTile);
}

hipError_t launch_count_tokens(CountArgs a, int num_cus, hipStream_t stream) {
  if (a.S == 0 || a.width == 0) return hipSuccess;
  // us for prompts, proposals and corrections of 256 sequences, the latter two by tiles 23.7, by
  // wavefronts 10.9
  if (a.width <= 64 && !(a.flags & CO_COUNT_FRESH)) {
    hipLaunchKernelGGL(count_few_kernel, dim3((a.S + 3) / 4), dim3(256), 0, stream, a);
  } else if (a.flags & CO_COUNT_PROMPT) {
    // tiles as large as leave a workgroup to every compute unit, from kTile on (us of the same
    // three calls with 128000 tokens, prompts up to 8192: 4 sequences, tiles of 65536 9.5, of 8192
    // 8.2; 64 sequences, tiles of 65536 13.1, of 32768 12.4)
    int size = kPromptTile;
    while (size > kTile && static_cast<int64_t>(a.S) * ((a.V + int64_t{size} - 1) / size) < num_cus) size /= 2;
    a.tiles = static_cast<int>((static_cast<int64_t>(a.V) + size - 1) / size);
    hipLaunchKernelGGL(mark_tile_kernel, dim3(static_cast<unsigned>(a.S) * a.tiles), dim3(512), 0, stream, a,
                       size);
  } else {
    a.tiles = static_cast<int>((static_cast<int64_t>(a.V) + kTile - 1) / kTile);
    hipLaunchKernelGGL(count_tile_kernel, dim3(static_cast<unsigned>(count_workgroups(a.S, a.V))),
                       dim3(256), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace co
