// Page tables and slot maps from request lengths, on the device: the pages that
// every sequence holds follow its length (carryover_assign_pages), and packed
// rows get their positions and committed slots (carryover_slot_map).  Next to
// the paper, which leaves the cache's paging to the serving stack.
//
// Pages change hands by number.  Released pages are numbered 0 .. R - 1 in
// (sequence, logical page) order, places to fill 0 .. T - 1 likewise; place k
// takes released page k, or (k >= R) entry free + R - 1 - k of the free list,
// and released page k >= T goes to that entry.  Every page that moves is so
// read and written by one thread, no entry is both read and written, and going
// back to the lengths before restores table and list exactly.
#include <algorithm>

#include "co_kernels.h"

namespace co {

namespace {

constexpr int kScanThreads = 1024;
constexpr int kSlotThreads = 256, kSlotRows = 4;   // rows per thread of the slot map
constexpr int kSlotSeqs = 4096;                    // sequences whose starts fit in LDS

// What a sequence holds and needs; an error leaves it as it is.
struct Need {
  int held, need, err;
};

__device__ __forceinline__ Need seq_need(const PagesArgs& a, int s) {
  const int h = a.held[s], w = a.want[s];
  const int64_t n = w > 0 ? (static_cast<int64_t>(w) + a.reserve + kPage - 1) / kPage : 0;
  if (h < 0 || h > a.max_pages) return {0, 0, CO_ERR_LENGTH};
  if (w < 0) return {h, h, CO_ERR_LENGTH};
  if (n > a.max_pages) return {h, h, CO_ERR_CAPACITY};
  return {h, static_cast<int>(n), CO_OK};
}

// The moves of one call: sequence s moves its places [lo, hi), out of its row
// (bit 31 of `to` set) or into it, the first one numbered `first`; `grow` is the
// number of its first place to fill.
struct Moves {
  int *lo, *hi, *first, *grow;   // [S] each
  int released, taken, have;     // R, T, free + R
};

// One workgroup: numbers every sequence's moves and writes the new holdings.
// Thread t takes ceil(S / 1024) sequences in a row.  sh: 2 * 16 ints of LDS.
__device__ void number_moves(const PagesArgs& a, Moves& m, int* sh) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int per = (a.S + kScanThreads - 1) / kScanThreads;
  const int s0 = min(a.S, t * per), s1 = min(a.S, s0 + per);
  const int c = a.free_count[0];   // read by every thread before it changes below
  int back = 0, more = 0;
  for (int s = s0; s < s1; ++s) {
    const Need n = seq_need(a, s);
    if (n.err != CO_OK) set_status(a.status, n.err);
    back += max(0, n.held - n.need);
    more += max(0, n.need - n.held);
  }
  int bi = back, mi = more;   // inclusive over the wavefront
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int b = __shfl_up(bi, o), g = __shfl_up(mi, o);
    if (lane >= o) {
      bi += b;
      mi += g;
    }
  }
  if (lane == 63) {
    sh[wave] = bi;
    sh[16 + wave] = mi;
  }
  __syncthreads();
  int R = 0, bx = bi - back, mx = mi - more;   // bx, mx: before this thread's sequences
#pragma unroll
  for (int w = 0; w < kScanThreads / 64; ++w) {
    const int b = sh[w], g = sh[16 + w];
    R += b;
    bx += w < wave ? b : 0;
    mx += w < wave ? g : 0;
  }
  // free + released, in 64 bits: more than the pool's pages cannot be true, and nothing changes
  const bool ok = c >= 0 && static_cast<int64_t>(c) + R <= a.num_pages;
  if (!ok && t == 0) set_status(a.status, CO_ERR_POOL);
  const int have = ok ? c + R : 0;
  int T = 0;
  for (int s = s0; s < s1; ++s) {
    const Need n = seq_need(a, s);
    const int b = max(0, n.held - n.need), g = max(0, n.need - n.held);
    const bool fits = mx + g <= have;   // in order: none after the first that does not fit
    if (ok && g > 0 && !fits) set_status(a.status, CO_ERR_POOL);
    const bool out = ok && b > 0, in = ok && g > 0 && fits;
    m.lo[s] = out ? n.need : n.held;
    m.hi[s] = in ? n.need : n.held;
    m.first[s] = out ? static_cast<int>(0x80000000u | static_cast<uint32_t>(bx)) : mx;
    m.grow[s] = mx;
    if (out || in) a.held[s] = n.need;
    if (in) T = mx + g;
    bx += b;
    mx += g;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) T = max(T, __shfl_xor(T, o));
  __syncthreads();   // sh is read
  if (lane == 0) sh[wave] = T;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kScanThreads / 64; ++w) T = max(T, sh[w]);
  m.released = ok ? R : 0;
  m.taken = T;
  m.have = have;
  if (ok && t == 0) a.free_count[0] = have - T;
}

// Place p of sequence s, in [lo, hi), changes hands.  An id that is no page's moves as
// the others do, so that going back undoes it too.  Returns the id (0: none moved here):
// a thread reports the largest of its ids once, which costs one instruction a move.
__device__ __forceinline__ uint32_t move_page(const PagesArgs& a, const Moves& m, int s, int p, int lo,
                                          int first) {
  const bool out = first < 0;
  const int k = (first & 0x7FFFFFFF) + p - lo;
  int32_t* at = a.table + static_cast<int64_t>(s) * a.max_pages + p;
  if (!out) {
    // (entries from R on: the rest come with a released page)
    if (k < m.released) return 0;
    const int32_t id = a.free_pages[m.have - 1 - k];
    *at = id;
    return id;
  }
  const int32_t id = *at;
  *at = -1;
  if (k < m.taken) {   // to the place of the same number
    int l = 0, r = a.S;   // the last sequence whose places start at or before k
    while (r - l > 1) {
      const int mid = (l + r) >> 1;
      if (m.grow[mid] <= k) l = mid;
      else r = mid;
    }
    a.table[static_cast<int64_t>(l) * a.max_pages + m.lo[l] + k - m.grow[l]] = id;
  } else {
    a.free_pages[m.have - 1 - k] = id;   // (have: at most num_pages)
  }
  return id;
}

__device__ __forceinline__ void report_ids(const PagesArgs& a, uint32_t largest) {
  if (largest >= static_cast<uint32_t>(a.num_pages)) set_status(a.status, CO_ERR_PAGE_RANGE);
}

// Both steps in one workgroup: a power of two of threads to each sequence, so many that all
// sequences have theirs in up to kTurns turns.  A turn and a thread's move are chains of loads: fewer
// turns suit steps where few pages move, more threads per sequence those where whole
// requests do.  Two turns against four (us, graph replays): 64 sequences of 512-8000
// positions in a decoding step 4.1 / 4.5, all changed 17.7 / 13.7; 634 of 50-178, all changed, 8.7 / 7.9
// (a wavefront per sequence, 40 turns: 24).
constexpr int kTurns = 2;

__global__ __launch_bounds__(kScanThreads) void assign_pages_kernel(PagesArgs a) {
  __shared__ int sh[32], lds[4 * kAssignSeqs];
  Moves m{lds, lds + kAssignSeqs, lds + 2 * kAssignSeqs, lds + 3 * kAssignSeqs, 0, 0, 0};
  number_moves(a, m, sh);
  __syncthreads();
  const int w = min(31 - __clz(kScanThreads), 31 - __clz(kTurns * kScanThreads / a.S));   // S: 1 .. kAssignSeqs
  static_assert(kAssignSeqs <= kScanThreads, "a thread at least");
  uint32_t ids = 0;
  for (int s = threadIdx.x >> w; s < a.S; s += kScanThreads >> w) {
    const int lo = m.lo[s], hi = m.hi[s], first = m.first[s];
    for (int p = lo + (threadIdx.x & ((1 << w) - 1)); p < hi; p += 1 << w) ids = max(ids, move_page(a, m, s, p, lo, first));
  }
  report_ids(a, ids);
}

// Or in two launches, the moves by a thread per place of the table.
__global__ __launch_bounds__(kScanThreads) void assign_scan_kernel(PagesArgs a) {
  __shared__ int sh[32];
  int* w = a.ws + kAssignHdr;
  Moves m{w, w + a.S, w + 2 * a.S, w + 3 * a.S, 0, 0, 0};
  number_moves(a, m, sh);
  if (threadIdx.x == 0) {
    a.ws[0] = m.released;
    a.ws[1] = m.taken;
    a.ws[2] = m.have;
  }
}

template <bool LDS>   // the sequences' first places, which released pages search, fit there
__global__ __launch_bounds__(256) void assign_move_kernel(PagesArgs a) {
  __shared__ int grow[LDS ? kAssignSeqs : 1];
  int* w = a.ws + kAssignHdr;
  Moves m{w, w + a.S, w + 2 * a.S, w + 3 * a.S, a.ws[0], a.ws[1], a.ws[2]};
  const int s = blockIdx.x, p = blockIdx.y * 256 + threadIdx.x;
  const int lo = m.lo[s];
  if constexpr (LDS) {
    for (int i = threadIdx.x; i < a.S; i += 256) grow[i] = m.grow[i];
    m.grow = grow;
    __syncthreads();
  }
  if (p >= lo && p < m.hi[s]) report_ids(a, move_page(a, m, s, p, lo, m.first[s]));
}

// Position and slot of packed rows: row r belongs to the last sequence that
// starts at or before it.  A thread takes kSlotRows rows in a row: one search, then
// on over the sequences' ends.  LDS: the starts fit there, and every workgroup
// sees whether one decreases: no row gets a slot then, for which row is whose is not
// defined (beyond, slot_starts_kernel looks afterwards).
template <bool LDS>
__global__ __launch_bounds__(kSlotThreads) void slot_map_kernel(SlotMapArgs a) {
  __shared__ int32_t lds[LDS ? kSlotSeqs + 1 : 1];
  const int32_t* start = a.row_start;
  bool bad = false;
  if constexpr (LDS) {
    __shared__ int down[kSlotThreads / 64];   // a word per wavefront: one barrier for all
    const int lane = threadIdx.x & 63;
    bool mine = false;
#pragma unroll 4
    for (int i = threadIdx.x; i <= a.S; i += kSlotThreads) {
      const int32_t v = a.row_start[i], before = a.row_start[max(i - 1, 0)];
      lds[i] = v;
      mine |= before > v;
    }
    const bool any = __any(mine);
    if (lane == 0) down[threadIdx.x >> 6] = any;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSlotThreads / 64; ++w) bad |= down[w] != 0;
    if (bad && threadIdx.x == 0) set_status(a.status, CO_ERR_LENGTH);
    start = lds;
  }
  const int64_t r0 = (static_cast<int64_t>(blockIdx.x) * kSlotThreads + threadIdx.x) * kSlotRows;
  if (r0 >= a.num_rows) return;
  int s = -1, end = a.S;   // start[s] <= r0 < start[end], with -1 and S + 1 as the ends
  ++end;
  while (end - s > 1) {
    const int mid = (s + end) >> 1;
    if (start[mid] <= r0) s = mid;
    else end = mid;
  }
  int32_t pos[kSlotRows], dst[kSlotRows];
#pragma unroll
  for (int i = 0; i < kSlotRows; ++i) {
    const int64_t r = r0 + i;
    pos[i] = 0;
    dst[i] = kSkip;
    if (bad || r >= a.num_rows) continue;
    // on to the row's sequence by steps that double, then bisected: a run of n
    // sequences without rows (free slots of a server) costs 2 log n reads
    int next = min(s + 1, a.S + 1);
    for (int step = 2; next <= a.S && start[next] <= r; step *= 2) {
      s = next;
      next = min(s + step, a.S + 1);
    }
    while (next - s > 1) {
      const int mid = (s + next) >> 1;
      if (start[mid] <= r) s = mid;
      else next = mid;
    }
    if (s < 0 || s >= a.S) continue;   // (rows before the first sequence and behind the last)
    const int32_t p0 = a.pos0[s];
    const int64_t p = p0 + (r - start[s]);
    if (p0 < 0) {
      set_status(a.status, CO_ERR_LENGTH);
    } else if (p >= static_cast<int64_t>(a.max_pages) * kPage) {
      set_status(a.status, CO_ERR_CAPACITY);
    } else {
      const int32_t id = a.table[static_cast<int64_t>(s) * a.max_pages + p / kPage];
      if (id < 0 || id >= a.num_pages) {
        set_status(a.status, CO_ERR_PAGE_RANGE);
      } else {
        pos[i] = static_cast<int32_t>(p);
        dst[i] = id * kPage + pos[i] % kPage;
      }
    }
  }
  typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
  static_assert(kSlotRows == 4, "one store");
  if (a.wide && r0 + kSlotRows <= a.num_rows) {
    *reinterpret_cast<i32x4*>(a.row_pos + r0) = i32x4{pos[0], pos[1], pos[2], pos[3]};
    *reinterpret_cast<i32x4*>(a.row_dst + r0) = i32x4{dst[0], dst[1], dst[2], dst[3]};
    return;
  }
#pragma unroll
  for (int i = 0; i < kSlotRows; ++i) {
    if (r0 + i >= a.num_rows) return;
    a.row_pos[r0 + i] = pos[i];
    a.row_dst[r0 + i] = dst[i];
  }
}

// Starts that do not fit in LDS, behind the map: a thread per start looks for one that
// decreases.  The workgroup of the first such start takes every row's slot back.
__global__ __launch_bounds__(kSlotThreads) void slot_starts_kernel(SlotMapArgs a) {
  const int i0 = blockIdx.x * kSlotThreads, i = i0 + threadIdx.x;   // S: at most 2^30
  auto falls = [&](int k) { return a.row_start[k] > a.row_start[k + 1]; };
  if (!__syncthreads_or(i < a.S && falls(i) ? 1 : 0)) return;
  if (threadIdx.x == 0) set_status(a.status, CO_ERR_LENGTH);
  for (int k0 = 0; k0 < i0; k0 += kSlotThreads)
    if (__syncthreads_or(falls(k0 + static_cast<int>(threadIdx.x)) ? 1 : 0)) return;
  for (int64_t r = threadIdx.x; r < a.num_rows; r += kSlotThreads) {
    a.row_pos[r] = 0;
    a.row_dst[r] = kSkip;
  }
}

}  // namespace

size_t assign_ws_bytes(int S) {
  return (kAssignHdr + 4 * static_cast<size_t>(S)) * 4 + 255 & ~static_cast<size_t>(255);
}

hipError_t launch_assign_pages(const PagesArgs& a, hipStream_t stream) {
  if (a.S == 0) return hipSuccess;
  if (a.S <= kAssignSeqs && static_cast<int64_t>(a.S) * a.max_pages <= kAssignPlaces) {
    hipLaunchKernelGGL(assign_pages_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(assign_scan_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const dim3 grid(a.S, (a.max_pages + 255) / 256);
  if (a.S <= kAssignSeqs) hipLaunchKernelGGL(assign_move_kernel<true>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(assign_move_kernel<false>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_slot_map(const SlotMapArgs& a, hipStream_t stream) {
  if (a.num_rows == 0) return hipSuccess;
  const int per = kSlotThreads * kSlotRows;
  const dim3 grid((static_cast<unsigned>(a.num_rows) + per - 1) / per);   // (past 2^31 - per rows too)
  if (a.S <= kSlotSeqs) {
    hipLaunchKernelGGL(slot_map_kernel<true>, grid, dim3(kSlotThreads), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(slot_map_kernel<false>, grid, dim3(kSlotThreads), 0, stream, a);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const unsigned blocks = (static_cast<unsigned>(a.S) + kSlotThreads - 1) / kSlotThreads;
  hipLaunchKernelGGL(slot_starts_kernel, dim3(blocks), dim3(kSlotThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace co
