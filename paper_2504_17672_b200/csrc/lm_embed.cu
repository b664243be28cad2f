// Embedding lookup with scaling, and its gradient by sorted tokens (include/cocodc_lm.h).

#include "lm_common.cuh"

#include <type_traits>

using namespace cocodc_lm_impl;

namespace {

// W elements of one type, loaded or stored as 16-byte accesses (or one of W * sizeof(T) bytes); W = 1: the element alone
template <typename T, int W> struct Pack {
  float v[W];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (W == 1) {
      v[0] = to_f32(*p);
    } else {
      constexpr int bytes = W * (int)sizeof(T);
      alignas(16) T e[W];
      if constexpr (bytes == 8) *reinterpret_cast<uint2*>(e) = *reinterpret_cast<const uint2*>(p);
      else for (int i = 0; i < bytes / 16; ++i) reinterpret_cast<uint4*>(e)[i] = reinterpret_cast<const uint4*>(p)[i];
      for (int i = 0; i < W; ++i) v[i] = to_f32(e[i]);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (W == 1) {
      *p = from_f32<T>(v[0]);
    } else {
      constexpr int bytes = W * (int)sizeof(T);
      alignas(16) T e[W];
      for (int i = 0; i < W; ++i) e[i] = from_f32<T>(v[i]);
      if constexpr (bytes == 8) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(e);
      else for (int i = 0; i < bytes / 16; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(e)[i];
    }
  }
};

// the same as it came from memory, converted when it is used
template <typename T, int W> struct Raw {
  alignas(16) T e[W];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (W == 1) e[0] = *p;
    else
      for (int i = 0; i < W * (int)sizeof(T) / 16; ++i) reinterpret_cast<uint4*>(e)[i] = load16(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ float at(int i) const { return to_f32(e[i]); }
};

// W sums of one thread, in shared or global scratch
template <int W> __device__ __forceinline__ void put(float* to, const float (&v)[W]) {
  if constexpr (W % 4 == 0)
    for (int i = 0; i < W; i += 4) *reinterpret_cast<float4*>(to + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  else
    for (int i = 0; i < W; ++i) to[i] = v[i];
}
template <int W, bool GLOBAL> __device__ __forceinline__ void get(float (&v)[W], const float* from) {
  if constexpr (W % 4 == 0)
    for (int i = 0; i < W; i += 4) {
      const float4 x = GLOBAL ? __ldcg(reinterpret_cast<const float4*>(from + i)) : *reinterpret_cast<const float4*>(from + i);
      v[i] = x.x; v[i + 1] = x.y; v[i + 2] = x.z; v[i + 3] = x.w;
    }
  else
    for (int i = 0; i < W; ++i) v[i] = GLOBAL ? __ldcg(from + i) : from[i];
}

// ---- lookup ------------------------------------------------------------------------------------
// A gather: bound by memory, and at fp32 tables by what L2 gives the SMs beside the writes: 65536 rows of 1024 in 36 us fp32 to
// bfloat16 (134 MB written, 268 MB gathered, 64 MB of them from DRAM), 28 us bfloat16 to
// bfloat16; 65536 rows of 777, element by element, in 104 us; 8 rows of 768 in 1.4 us (in a graph).  `lanes` neighbouring lanes (a power of two, up to a warp) take up to U packs of W elements each
// of one token's row, all loads before the first store; a longer row is several items.
template <typename TIn, typename TOut, int W, int U>
__global__ void __launch_bounds__(256) k_embed(const TIn* table, long long table_stride, long long V,
                                               unsigned packs, int lanes_log2, unsigned items_per_row, const void* ids,
                                               int is64, long long T, float scale, TOut* y, long long y_stride,
                                               int* status) {
  wait_for_previous();
  may_follow();
  const int lanes = 1 << lanes_log2, sub = threadIdx.x & (lanes - 1);
  const long long items = T * items_per_row, step = (long long)gridDim.x * 256 >> lanes_log2;
  for (long long item = ((long long)blockIdx.x * 256 + threadIdx.x) >> lanes_log2; item < items; item += step) {
    const long long t = items_per_row == 1 ? item : item / items_per_row;
    const unsigned first = (unsigned)(item - t * items_per_row) * (U << lanes_log2) + sub;
    const long long v = token_at(ids, is64, t, V, status);
    const TIn* from = table + v * table_stride;
    TOut* to = y + t * y_stride;
    Raw<TIn, W> x[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const unsigned col = first + (i << lanes_log2);
      if (v >= 0 && col < packs) x[i].load(from + (long long)col * W);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const unsigned col = first + (i << lanes_log2);
      if (col >= packs) continue;
      Pack<TOut, W> out;
#pragma unroll
      for (int k = 0; k < W; ++k) out.v[k] = v < 0 ? 0.f : scale * x[i].at(k);
      out.store(to + (long long)col * W);
    }
  }
}

// ---- gradient, step 1: the tokens in order of their rows ------------------------------------------
// The table's rows are dealt to B bins (a power of two), row v to bin v mod B, so that the frequent tokens, whose ids
// tend to lie together, end up in different bins; the sorted order is by (bin, row, token position).  One CTA per bin finds its
// tokens itself by walking over all T ids; no CTA waits for another.  A warp walks over its contiguous part of the
// ids and appends the hits, in order, to a list in shared memory; ids in lower bins are counted: their number is where this
// bin begins.  The hits counted per (row, warp), a prefix sum over the counts gives every row's and warp's first
// position, and a second run over the lists (over the ids, where a list was too short) places the tokens: equal ids
// stay in the order of their positions because a warp's part precedes the next warp's.
// Every CTA reads all ids, from L2 after the first: 128 CTAs and 65536 tokens of 4 bytes make 34 MB.  Measured, zero rows
// included: 28 us for 4099 tokens and 50257 rows of 768 (of which 22 us are the zeros, 144 MB), 29 us for 65536 tokens
// and 32000 rows of 1024 (20 us the walk: issue slots and shared memory, not bytes).
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxBinRows = 768;
constexpr int kBinPitch = kSortWarps + 1;              // counters of a warp's lanes fall into different banks
constexpr int kListLength = 512;                       // hits that a warp keeps, at most 128 of them new per step
constexpr int kRowBits = 10;                           // of a list entry; the others hold the position in the warp's part
constexpr long long kMostTokens = 1ll << (32 - kRowBits + 5);
constexpr long long kMostRows = 1ll << 30;
static_assert(kMaxBinRows <= 1 << kRowBits, "a bin's rows do not fit a list entry");

struct GradArgs {
  const void* ids;
  int is64;
  int T;
  long long V, D;
  int bins_log2, bin_rows;
  int accumulate;
  float scale;
  const void* dy;
  long long dy_stride;
  void* dtable;
  long long dtable_stride;
  int dtable_esize;
  int dtable_wide;    // rows start on 16-byte boundaries
  int* row_start;     // [bins * bin_rows + 1] first sorted position of every row, in sorted order
  int2* sorted;       // [T] (token position, row) in sorted order
  float* partial;     // [tiles][2][padded D]: sums of the rows that a tile shares with its neighbours
  int* arrived;       // [tiles][column blocks]: tiles that have left their part of the row that begins in the tile
  long long n_arrived;
  int positions;      // sorted positions of one group of a tile
  long long pitch;    // padded D
  int* status;
};
// where a row comes in the sorted order
__device__ __forceinline__ int order_of(const GradArgs& a, int row) {
  return (row & ((1 << a.bins_log2) - 1)) * a.bin_rows + (row >> a.bins_log2);
}

struct SortShared {
  unsigned list[kSortWarps][kListLength];              // position in the warp's part << kRowBits | row of the bin
  int scratch[kSortWarps];
  int again;                                           // a list was too short
  int cnt[];                                           // [bin_rows][kBinPitch]
};

template <typename I>
__global__ void __launch_bounds__(kSortThreads) k_embed_sort(const GradArgs a) {
  wait_for_previous();
  may_follow();
  extern __shared__ __align__(16) unsigned char dyn[];
  SortShared& sh = *reinterpret_cast<SortShared*>(dyn);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int bin = blockIdx.x, mask = (1 << a.bins_log2) - 1;
  const int part = ((a.T + kSortWarps - 1) / kSortWarps + 127) / 128 * 128;       // T <= kMostTokens: no overflow
  const int t0 = warp * part, t1 = min(a.T, t0 + part);
  const I* ids = static_cast<const I*>(a.ids);
  const bool wide = ((uintptr_t)ids & 15) == 0;

  for (int i = tid; i < a.bin_rows * kBinPitch; i += kSortThreads) sh.cnt[i] = 0;
  for (long long i = (long long)bin * kSortThreads + tid; i < a.n_arrived; i += (long long)gridDim.x * kSortThreads)
    a.arrived[i] = 0;
  if (tid == 0) sh.again = 0;
  __syncthreads();

  // f on hits [0, n) of the warp's list, 32 at a time: token position, row (-1: none), the lanes with the same row
  const auto each = [&](int n, auto&& f) {
    __syncwarp();
    for (int i = 0; i < n; i += 32) {
      const unsigned e = sh.list[warp][min(i + lane, n - 1)];
      const int row = i + lane < n ? (int)(e & ((1u << kRowBits) - 1)) : -1;
      f(t0 + (int)(e >> kRowBits), row, __match_any_sync(~0u, row));
      __syncwarp();
    }
  };
  int below = 0, hits = 0;
  bool flushed = false;
  const auto walk = [&](auto&& f) {
    hits = 0;
    I v[4], next[4];
    const auto fetch = [&](int t) {                    // lane l takes ids t + 4 l .. t + 4 l + 3
      const int first = t + lane * 4;
      if (wide && first + 4 <= t1) {
        constexpr int words = 4 * sizeof(I) / 16;
        for (int i = 0; i < words; ++i) reinterpret_cast<uint4*>(next)[i] = load16(reinterpret_cast<const uint4*>(ids + first) + i);
      } else {
        for (int i = 0; i < 4; ++i) next[i] = first + i < t1 ? ids[first + i] : I(-1);
      }
    };
    fetch(t0);
    for (int t = t0; t < t1; t += 128) {
      const int first = t + lane * 4;
      for (int i = 0; i < 4; ++i) v[i] = next[i];
      if (t + 128 < t1) fetch(t + 128);                // on its way while this step is worked on
      unsigned mine = 0;
      bool bad = false;
      for (int i = 0; i < 4; ++i) {
        using U = typename std::make_unsigned<I>::type;
        const bool there = (U)v[i] < (U)a.V;           // false for negative ids too
        bad |= v[i] >= (I)a.V;
        const int b = there ? (int)v[i] & mask : mask + 1;
        below += b < bin;
        mine |= (unsigned)(b == bin) << i;
      }
      if (bad) record(a.status, COCODC_ERR_INVALID_ARG);
      const unsigned with = __ballot_sync(~0u, mine != 0);
      if (!with) continue;
      const int n = __popc(mine);
      const unsigned under = (1u << lane) - 1;
      int before = __popc(with & under), all = __popc(with);
      if (__any_sync(~0u, n > 1))
        for (int i = 2; i <= 4; ++i) {
          const unsigned m = __ballot_sync(~0u, n >= i);
          before += __popc(m & under);
          all += __popc(m);
        }
      if (mine)
        for (int i = 0; i < 4; ++i)
          if (mine >> i & 1) sh.list[warp][hits + before++] = (unsigned)(first + i - t0) << kRowBits | (unsigned)(v[i] >> a.bins_log2);
      hits += all;
      if (hits > kListLength - 128) {
        each(hits, f);
        hits = 0;
        flushed = true;
      }
    }
  };
  const auto count = [&](int, int row, unsigned same) {
    if (row >= 0 && lane == __ffs(same) - 1) sh.cnt[row * kBinPitch + warp] += __popc(same);
  };
  walk(count);
  each(hits, count);
  if (flushed && lane == 0) sh.again = 1;

  for (int o = 16; o; o >>= 1) below += __shfl_xor_sync(~0u, below, o);
  if (lane == 0) sh.scratch[warp] = below;
  __syncthreads();
  int at = 0;                                          // of the bin, then of the thread's row
  for (int w = 0; w < kSortWarps; ++w) at += sh.scratch[w];
  __syncthreads();
  int total = 0;
  if (tid < a.bin_rows)
    for (int w = 0; w < kSortWarps; ++w) total += sh.cnt[tid * kBinPitch + w];
  int incl = total;
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(~0u, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) sh.scratch[warp] = incl;
  __syncthreads();
  at += incl - total;
  for (int w = 0; w < warp; ++w) at += sh.scratch[w];
  if (tid < a.bin_rows) {
    a.row_start[bin * a.bin_rows + tid] = at;
    if (bin == mask && tid == a.bin_rows - 1) a.row_start[(bin + 1) * a.bin_rows] = at + total;
    int run = at;
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = sh.cnt[tid * kBinPitch + w];
      sh.cnt[tid * kBinPitch + w] = run;
      run += c;
    }
    sh.cnt[tid * kBinPitch + kSortWarps] = total;      // the padding word keeps the row's count
  }
  __syncthreads();

  const auto place = [&](int t, int row, unsigned same) {
    const int leader = __ffs(same) - 1;
    int base = 0;
    if (row >= 0 && lane == leader) {
      base = sh.cnt[row * kBinPitch + warp];
      sh.cnt[row * kBinPitch + warp] = base + __popc(same);
    }
    base = __shfl_sync(~0u, base, leader);
    if (row >= 0) a.sorted[base + __popc(same & ((1u << lane) - 1))] = make_int2(t, (row << a.bins_log2) + bin);
  };
  if (sh.again) walk(place);
  each(hits, place);

  // Rows that no token names: zeros.  (Written by CTAs of the next launch, beside the sums, they took 4 us longer at
  // 50257 x 768 and 2 us longer at 32000 x 1024.)
  if (!a.accumulate) {
    const long long bytes = a.D * a.dtable_esize, n16 = a.dtable_wide ? bytes / 16 : 0;
    for (int r = warp; r < a.bin_rows; r += kSortWarps) {
      const long long v = ((long long)r << a.bins_log2) + bin;
      if (v >= a.V || sh.cnt[r * kBinPitch + kSortWarps]) continue;
      char* p = static_cast<char*>(a.dtable) + v * a.dtable_stride * a.dtable_esize;
      for (long long i = lane; i < n16; i += 32) reinterpret_cast<uint4*>(p)[i] = make_uint4(0, 0, 0, 0);
      for (long long i = n16 * 16 + lane * a.dtable_esize; i < bytes; i += 32 * a.dtable_esize) {
        if (a.dtable_esize == 4) *reinterpret_cast<float*>(p + i) = 0.f;
        else *reinterpret_cast<unsigned short*>(p + i) = 0;
      }
    }
  }
}

// ---- gradient, step 2: the sums -----------------------------------------------------------------
// A CTA takes a tile of kGroups * positions consecutive entries of the sorted order, so the work is even however the
// tokens are distributed: each of its groups of threads sums its own run of entries, one column pack per thread, and
// starts a new sum where the row changes.  A row that lies inside one group is written at once.  Rows that cross group
// boundaries are joined in shared memory in order; those that cross tile boundaries leave their parts in the
// workspace, and the tile that arrives last at the row's counter adds all parts in tile order (nobody waits).
// Measured: 45 us for 65536 gradients of 1024 bfloat16 (134 MB read, 79 MB written: 4.7 TB/s), 13 us for 4099 of 768.  The
// time not spent on bytes goes into the joins, most tiles begin and end inside a frequent token's row.  Eight loads
// ahead instead of four spilled (62 us).
constexpr int kGroups = 4;
constexpr int kAhead = 4;      // loads in flight per thread

template <typename TIn, typename TOut, int W>
__global__ void __launch_bounds__(kGroups * 128, 2) k_embed_sum(const GradArgs a) {
  wait_for_previous();
  may_follow();
  extern __shared__ __align__(16) float part[];                       // [kGroups][2][threads of a group][W]: head, tail
  __shared__ int pending_row[2], is_last[2], pending_first[2], pending_parts[2];
  __shared__ int edge[2 * kGroups + 2];                 // rows of: the entry before the tile, each group's first and last, the entry after
  const int width = blockDim.x / kGroups, group = threadIdx.x / width, c = threadIdx.x % width;
  const long long col = ((long long)blockIdx.y * width + c) * W;
  const bool active = col < a.D;
  const int n = a.row_start[a.bin_rows << a.bins_log2];
  const int tile = blockIdx.x, span = kGroups * a.positions, begin = tile * span;
  if (begin >= n) return;
  const TIn* dy = static_cast<const TIn*>(a.dy) + (active ? col : 0);
  TOut* out = static_cast<TOut*>(a.dtable) + (active ? col : 0);

  float acc[W];
  const auto clear = [&] { for (int k = 0; k < W; ++k) acc[k] = 0.f; };
  const auto write_row = [&](int row) {
    if (!active) return;
    Pack<TOut, W> o;
    TOut* p = out + (long long)row * a.dtable_stride;
    if (a.accumulate) {
      o.load(p);
      for (int k = 0; k < W; ++k) o.v[k] += a.scale * acc[k];
    } else {
      for (int k = 0; k < W; ++k) o.v[k] = a.scale * acc[k];
    }
    o.store(p);
  };
  float* head = part + ((group * 2) * width + c) * W;
  float* tail = part + ((group * 2 + 1) * width + c) * W;

  const int p0 = min(n, begin + group * a.positions), p1 = min(n, p0 + a.positions);
  if (p0 < p1) {
    // lane i holds entry i of the group: its row, where its gradient starts, and whether a row begins there
    const int lane = threadIdx.x & 31, entries = p1 - p0;
    const int2 mine = lane < entries ? a.sorted[p0 + lane] : make_int2(0, -1);
    const int left = p0 > 0 ? a.sorted[p0 - 1].y : -1, right = p1 < n ? a.sorted[p1].y : -1;
    const long long offset = mine.x * a.dy_stride;
    const int before = __shfl_up_sync(~0u, mine.y, 1);
    const unsigned starts = __ballot_sync(~0u, lane > 0 && mine.y != before);
    const int row_in = __shfl_sync(~0u, mine.y, 0), row_out = __shfl_sync(~0u, mine.y, entries - 1);
    bool open = left == row_in;                          // the current sum continues a row of the group before
    const bool goes_on = right == row_out;
    if (c == 0) {
      edge[1 + 2 * group] = row_in;
      edge[2 + 2 * group] = row_out;
      if (group == 0) edge[0] = left;
      if (p1 == min(n, begin + span)) {
        edge[1 + 2 * kGroups] = right;
        for (int g = group + 1; g < kGroups; ++g) edge[1 + 2 * g] = edge[2 + 2 * g] = -1;   // groups without entries
      }
      // the rows that cross the tile's ends: where they begin and how many tiles share them
      for (int s = 0; s < 2; ++s) {
        const int row = s == 0 ? (group == 0 && open ? row_in : -1) : (p1 == min(n, begin + span) && goes_on ? row_out : -1);
        if (row < 0) continue;
        const int g = order_of(a, row);
        pending_first[s] = a.row_start[g] / span;
        pending_parts[s] = (a.row_start[g + 1] - 1) / span - pending_first[s] + 1;
      }
    }
    clear();
    for (int p = 0; p < entries; p += kAhead) {
      Raw<TIn, W> x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const long long at = __shfl_sync(~0u, offset, (p + i) & 31);
        if (p + i < entries) x[i].load(dy + at);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (p + i >= entries) break;
        if (starts >> (p + i) & 1) {
          if (open) put<W>(head, acc);
          else write_row(__shfl_sync(~0u, mine.y, p + i - 1));
          open = false;
          clear();
        }
        for (int k = 0; k < W; ++k) acc[k] += x[i].at(k);
      }
    }
    float* to = open ? head : goes_on ? tail : nullptr;
    if (to) put<W>(to, acc);
    else write_row(row_out);
  }
  if (threadIdx.x < 2) pending_row[threadIdx.x] = -1;
  __syncthreads();

  // rows that cross groups: joined in order by the first group's threads
  if (group == 0) {
    bool running = false, outside = false;               // a sum is open; it began in an earlier tile
    int row = -1;
    const auto leave = [&](int slot) {                   // slot 0: begun in an earlier tile, 1: begun here
      if (active) put<W>(a.partial + ((long long)tile * 2 + slot) * a.pitch + col, acc);
      if (c == 0) pending_row[slot] = row;
      __threadfence();
    };
    for (int g = 0; g < kGroups && edge[1 + 2 * g] >= 0; ++g) {
      const int row_in = edge[1 + 2 * g], row_out = edge[2 + 2 * g];
      const int follower = g + 1 < kGroups && edge[3 + 2 * g] >= 0 ? edge[3 + 2 * g] : edge[1 + 2 * kGroups];
      const bool left = edge[2 * g] == row_in, right = follower == row_out, through = left && right && row_in == row_out;
      if (left) {
        if (!running) { clear(); running = true; outside = true; row = row_in; }
        float h[W];
        get<W, false>(h, part + ((g * 2) * width + c) * W);
        for (int k = 0; k < W; ++k) acc[k] += h[k];
        if (!through) {
          if (outside) leave(0);
          else write_row(row);
          running = false;
        }
      }
      if (right && !running) {
        get<W, false>(acc, part + ((g * 2 + 1) * width + c) * W);
        running = true;
        outside = false;
        row = row_out;
      }
    }
    if (running) leave(outside ? 0 : 1);
  }
  __syncthreads();

  // rows that cross tiles: the last of their tiles to arrive adds the parts
  if (threadIdx.x < 2) {
    const int row = pending_row[threadIdx.x];
    int last = 0;
    if (row >= 0) {
      __threadfence();
      last = atomicAdd(&a.arrived[(long long)pending_first[threadIdx.x] * gridDim.y + blockIdx.y], 1) ==
             pending_parts[threadIdx.x] - 1;
      __threadfence();
    }
    is_last[threadIdx.x] = last;
  }
  __syncthreads();
  for (int s = 0; s < 2; ++s) {
    if (!is_last[s]) continue;
    const int row = pending_row[s], first = pending_first[s], parts = pending_parts[s];
    clear();
    const int j1 = (int)((long long)parts * (group + 1) / kGroups);
    if (active)
      for (int j = (int)((long long)parts * group / kGroups); j < j1; j += 4) {
        float x[4][W];
        for (int i = 0; i < 4; ++i)
          if (j + i < j1) get<W, true>(x[i], a.partial + ((long long)(first + j + i) * 2 + (j + i == 0 ? 1 : 0)) * a.pitch + col);
        for (int i = 0; i < 4; ++i)
          if (j + i < j1) for (int k = 0; k < W; ++k) acc[k] += x[i][k];
      }
    put<W>(head, acc);
    __syncthreads();
    if (group == 0) {
      for (int g = 1; g < kGroups; ++g) {
        float h[W];
        get<W, false>(h, part + ((g * 2) * width + c) * W);
        for (int k = 0; k < W; ++k) acc[k] += h[k];
      }
      write_row(row);
    }
    __syncthreads();
  }
}

// Sorted entries per group (a lane each): 32 amortise the boundaries; with few tokens fewer, so that there are tiles for all SMs.  (148, a
// B200's: the size of a workspace is asked for without a handle.)
int positions_for(int64_t T) {
  int p = 32;
  while (p > 4 && T < (int64_t)148 * 2 * kGroups * p) p /= 2;
  return p;
}

uint64_t up16(uint64_t n) { return (n + 15) / 16 * 16; }
// 128 bins (one CTA per SM: every CTA reads all ids, so twice as many took 7 us longer at 65536 tokens), fewer for a smaller
// table, more where a bin's rows would not fit shared memory
int bins_log2_for(int64_t V) {
  int l = 0;
  while (l < 7 && (int64_t(1) << l) < V) ++l;
  while ((V + (int64_t(1) << l) - 1) >> l > kMaxBinRows) ++l;
  return l;
}
// At least more than half of an SM's shared memory: a block that starts while the previous kernel ends must not join
// another one on an SM that happens to be free first (65536 tokens: 77 -> 96 us for the whole gradient)
unsigned sort_smem(int bin_rows) {
  const unsigned need = (unsigned)sizeof(SortShared) + bin_rows * kBinPitch * 4, alone = 120 * 1024;
  return need > alone ? need : alone;
}
int64_t bin_rows_for(int64_t V) { return (V + (int64_t(1) << bins_log2_for(V)) - 1) >> bins_log2_for(V); }
int64_t starts_for(int64_t V) { return (bin_rows_for(V) << bins_log2_for(V)) + 1; }
int64_t padded(int64_t D) { return (D + 7) / 8 * 8; }
int64_t tiles_for(int64_t T) { return (T + kGroups * positions_for(T) - 1) / (kGroups * positions_for(T)); }

}  // namespace

namespace cocodc_lm_impl {
bool embed_prepare() {
  const int most = (int)sort_smem(kMaxBinRows);
  return cudaFuncSetAttribute(k_embed_sort<int>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) == cudaSuccess &&
         cudaFuncSetAttribute(k_embed_sort<long long>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) == cudaSuccess;
}
}  // namespace cocodc_lm_impl

extern "C" {

cocodc_status cocodc_lm_embed(cocodc_lm* lm, const void* table, int32_t table_type, int64_t table_stride, int64_t V,
                              int64_t D, const void* ids, int32_t ids_type, int64_t T, float scale, void* y,
                              int32_t y_type, int64_t y_stride, void* stream) {
  if (!lm || !sane(V) || !sane(D) || !sane(T) || V < 1 || D < 1 || D > INT32_MAX || !known_type(table_type) || !known_type(y_type) ||
      (ids_type != COCODC_I32 && ids_type != COCODC_I64) || table_stride < D || y_stride < D || !sane(table_stride) ||
      !sane(y_stride))
    return COCODC_ERR_INVALID_ARG;
  if (T == 0) return COCODC_OK;
  if (!table || !ids || !y) return COCODC_ERR_INVALID_ARG;
  const int es = type_bytes(table_type), ys = type_bytes(y_type);
  if (!on_boundary(table, es) || !on_boundary(y, ys) || !on_boundary(ids, index_bytes(ids_type))) return COCODC_ERR_ALIGNMENT;
  const Span sy = span(y, T, y_stride, D, ys);
  if (meet(sy, span(table, V, table_stride, D, es)) || meet(sy, span(ids, 1, T, T, index_bytes(ids_type))))
    return COCODC_ERR_ALIAS;
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = rows_aligned(table, table_stride, es) && rows_aligned(y, y_stride, ys) && D % 8 == 0;
  return with_type(table_type, [&](auto in) {
    return with_type(y_type, [&](auto out) {
      using TIn = decltype(in);
      using TOut = decltype(out);
      const auto run = [&](auto kernel, int W, int U) {
        const unsigned packs = (unsigned)(D / W);
        int lanes_log2 = 0;
        while (lanes_log2 < 5 && (1u << lanes_log2) < packs) ++lanes_log2;
        const unsigned per_row = (packs + (U << lanes_log2) - 1) / (U << lanes_log2);
        const long long blocks = (((T * per_row) << lanes_log2) + 255) / 256;
        return start(lm, kernel, (unsigned)(blocks < (1 << 30) ? blocks : (1 << 30)), 256, 0, st, 1,
                     static_cast<const TIn*>(table), table_stride, V, packs, lanes_log2, per_row, ids, ids_type == COCODC_I64, T,
                     scale, static_cast<TOut*>(y), y_stride, lm->d_status);
      };
      // few packs: one per thread, so that they spread over the SMs.  65536 x 1024 in us at U = 2 / 4: fp32 to bf16 40.9 / 36.6,
      // bf16 to bf16 33.3 / 28.6, fp32 to fp32 66.0 / 71.8
      constexpr int U = sizeof(TIn) + sizeof(TOut) == 8 ? 2 : 4;
      if (!wide) return run(k_embed<TIn, TOut, 1, 4>, 1, 4);
      if (T * (D / 8) < (long long)lm->sm_count * 2048) return run(k_embed<TIn, TOut, 8, 1>, 8, 1);
      return run(k_embed<TIn, TOut, 8, U>, 8, U);
    });
  });
}

uint64_t cocodc_lm_embed_grad_workspace(int64_t V, int64_t D, int64_t T) {
  if (V < 0 || D < 0 || T < 0 || V > kMostRows || D > INT32_MAX || T > kMostTokens) return 0;
  const uint64_t tiles = (uint64_t)tiles_for(T);
  return up16((uint64_t)starts_for(V) * sizeof(int)) + up16((uint64_t)T * sizeof(int2)) + tiles * 2 * padded(D) * sizeof(float) +
         up16(tiles * (uint64_t)((D + 31) / 32) * sizeof(int));
}

cocodc_status cocodc_lm_embed_grad(cocodc_lm* lm, const void* dy, int32_t dy_type, int64_t dy_stride, const void* ids,
                                   int32_t ids_type, int64_t T, int64_t V, int64_t D, float scale, int32_t accumulate,
                                   void* dtable, int32_t dtable_type, int64_t dtable_stride, void* workspace,
                                   uint64_t workspace_bytes, void* stream) {
  if (!lm || !sane(V) || !sane(D) || !sane(T) || V < 1 || D < 1 || D > INT32_MAX || T > kMostTokens || V > kMostRows || !dtable ||
      !known_type(dy_type) || !known_type(dtable_type) || (ids_type != COCODC_I32 && ids_type != COCODC_I64) ||
      dy_stride < D || dtable_stride < D || !sane(dy_stride) || !sane(dtable_stride))
    return COCODC_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < cocodc_lm_embed_grad_workspace(V, D, T)) return COCODC_ERR_INVALID_ARG;
  if (T > 0 && (!dy || !ids)) return COCODC_ERR_INVALID_ARG;
  const int es = type_bytes(dy_type), gs = type_bytes(dtable_type);
  if (!on_boundary(dy, es) || !on_boundary(dtable, gs) || !on_boundary(ids, index_bytes(ids_type)) ||
      !on_boundary(workspace, 16))
    return COCODC_ERR_ALIGNMENT;
  const Span sw = span(workspace, 1, (int64_t)workspace_bytes, (int64_t)workspace_bytes, 1);
  const Span sg = span(dtable, V, dtable_stride, D, gs), sy = span(dy, T, dy_stride, D, es);
  const Span si = span(ids, T ? 1 : 0, T, T, index_bytes(ids_type));
  if (meet(sg, sy) || meet(sg, si) || meet(sw, sg) || meet(sw, sy) || meet(sw, si)) return COCODC_ERR_ALIAS;
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  GradArgs a{};
  a.ids = ids;
  a.is64 = ids_type == COCODC_I64;
  a.T = (int)T;
  a.V = V;
  a.D = D;
  a.accumulate = accumulate != 0;
  a.scale = scale;
  a.dy = dy;
  a.dy_stride = dy_stride;
  a.dtable = dtable;
  a.dtable_stride = dtable_stride;
  a.dtable_esize = gs;
  const int64_t tiles = tiles_for(T);
  char* at = static_cast<char*>(workspace);
  const auto take = [&](uint64_t bytes) { char* p = at; at += up16(bytes); return p; };
  a.row_start = reinterpret_cast<int*>(take((uint64_t)starts_for(V) * sizeof(int)));
  a.sorted = reinterpret_cast<int2*>(take((uint64_t)T * sizeof(int2)));
  a.partial = reinterpret_cast<float*>(take((uint64_t)tiles * 2 * padded(D) * sizeof(float)));
  a.arrived = reinterpret_cast<int*>(at);
  a.status = lm->d_status;
  a.positions = positions_for(T);
  a.pitch = padded(D);
  a.dtable_wide = rows_aligned(dtable, dtable_stride, gs);
  // 16 bytes of dy per thread where rows of both matrices start on 16-byte boundaries and hold whole packs
  const int W = rows_aligned(dy, dy_stride, es) && a.dtable_wide && D % (16 / es) == 0 ? 16 / es : 1;
  const long long packs = D / W;
  const int width = packs >= 128 ? 128 : (int)((packs + 31) / 32 * 32);
  const long long columns = (packs + width - 1) / width;
  if (columns > 65535) return COCODC_ERR_INVALID_ARG;
  a.n_arrived = tiles * columns;
  a.bins_log2 = bins_log2_for(V);
  a.bin_rows = (int)bin_rows_for(V);
  const unsigned bins = 1u << a.bins_log2, smem_sort = sort_smem(a.bin_rows);
  const cocodc_status sorted = a.is64 ? start(lm, k_embed_sort<long long>, bins, kSortThreads, smem_sort, st, 1, a)
                                      : start(lm, k_embed_sort<int>, bins, kSortThreads, smem_sort, st, 1, a);
  if (sorted != COCODC_OK || T == 0) return sorted;
  return with_type(dy_type, [&](auto in) {
    return with_type(dtable_type, [&](auto out) {
      using TIn = decltype(in);
      using TOut = decltype(out);
      const dim3 grid((unsigned)tiles, (unsigned)columns);
      const unsigned smem = kGroups * 2 * width * W * sizeof(float);
      return W > 1 ? start(lm, k_embed_sum<TIn, TOut, 16 / (int)sizeof(TIn)>, grid, kGroups * width, smem, st, 1, a)
                   : start(lm, k_embed_sum<TIn, TOut, 1>, grid, kGroups * width, smem, st, 1, a);
    });
  });
}

}  // extern "C"
