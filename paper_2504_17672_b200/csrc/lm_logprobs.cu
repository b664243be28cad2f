// Log probabilities of given tokens with entropy and top alternatives, and their gradient (include/cocodc_lm.h).

#include "lm_common.cuh"

#include <type_traits>

using namespace cocodc_lm_impl;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr float kMostScale = 1e30f;   // times log2 e still finite
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A logit as a 32-bit number with the same order (NaN above +Inf, -0 equal to +0), and with the position behind it
// as one 64-bit number: larger logits first, equal ones by ascending position.  Every key is above 0 and below ~0
// (also a NaN at position 0).
__device__ __forceinline__ unsigned ordered(float x) {
  if (x != x) return 0xffffffffu;
  const unsigned b = __float_as_uint(x + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ unsigned long long key_of(float x, unsigned j) {
  return ((unsigned long long)ordered(x) << 32) | (0xfffffffeu - j);
}
__device__ __forceinline__ unsigned position_of(unsigned long long key) { return 0xfffffffeu - (unsigned)key; }

__device__ __forceinline__ unsigned long long warp_max(unsigned long long k) {
  const unsigned hi = (unsigned)(k >> 32), best = __reduce_max_sync(~0u, hi);
  const unsigned lo = __reduce_max_sync(~0u, hi == best ? (unsigned)k : 0u);
  return ((unsigned long long)best << 32) | lo;
}

struct RowArgs {
  const void* logits;
  long long stride, T;
  unsigned V;
  const void* targets;
  int targets64;
  float scale;
  float *logp, *entropy, *lse;
  int top_k;
  int* top_ids;
  float* top_logp;
  int* status;
};

// ---- pairs of fp32 numbers: one instruction for two ----------------------------------------------
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float lo, float hi) {
  f32x2 v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
  return v;
}
__device__ __forceinline__ void split(f32x2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 v;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}

// ---- sixteen bytes of a row ---------------------------------------------------------------------
// Logits below -kFar take part in the sums as -kFar (-Inf would turn 0 * d into NaN in the entropy's sum).  That is exact
// where their exponentials are 0 either way: where the largest logit is above -kFar / 2 and c kFar / 2 is above 200;
// anything else goes the careful way.  kFar is a power of two, so that c * kFar is c's bits and -kFar's distance to itself is 0; it
// is finite times the largest c, and masks of -1e9 and lower lie beyond it.
template <typename T> struct Words;
template <> struct Words<float> {
  static constexpr int n = 4;
  static constexpr float kFar = 0x1p27f;
  float e[4];
  __device__ __forceinline__ void set(uint4 w) {
    const float f[4] = {__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)};
    for (int i = 0; i < 4; ++i) asm("max.NaN.f32 %0, %1, %2;" : "=f"(e[i]) : "f"(f[i]), "f"(-kFar));
  }
  static __device__ __forceinline__ uint4 far() { const unsigned v = __float_as_uint(-kFar); return make_uint4(v, v, v, v); }
  __device__ __forceinline__ float at(int i) const { return e[i]; }
  __device__ __forceinline__ f32x2 two(int i) const { return pair_of(e[2 * i], e[2 * i + 1]); }
  static __device__ __forceinline__ f32x2 pair(const uint4& w, int i) {   // two logits as they are
    return i ? pair_of(__uint_as_float(w.z), __uint_as_float(w.w)) : pair_of(__uint_as_float(w.x), __uint_as_float(w.y));
  }
  __device__ __forceinline__ float largest() const { return fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3])); }
};
template <> struct Words<__nv_bfloat16> {
  static constexpr int n = 8;
  static constexpr float kFar = 0x1p27f;
  __nv_bfloat162 e[4];
  static __device__ __forceinline__ __nv_bfloat162 low() { return __float2bfloat162_rn(-kFar); }
  __device__ __forceinline__ void set(uint4 w) {
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
    for (int i = 0; i < 4; ++i) e[i] = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&u[i]), low());
  }
  static __device__ __forceinline__ uint4 far() {
    const __nv_bfloat162 l = low();
    const unsigned v = *reinterpret_cast<const unsigned*>(&l);
    return make_uint4(v, v, v, v);
  }
  __device__ __forceinline__ float at(int i) const { return i & 1 ? __high2float(e[i / 2]) : __low2float(e[i / 2]); }
  static __device__ __forceinline__ f32x2 widen(unsigned u) {   // a bfloat16 is the upper half of the same fp32 number
    return pair_of(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  }
  __device__ __forceinline__ f32x2 two(int i) const { return widen(*reinterpret_cast<const unsigned*>(&e[i])); }
  static __device__ __forceinline__ f32x2 pair(const uint4& w, int i) { return widen(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w); }
  __device__ __forceinline__ float largest() const {
    const __nv_bfloat162 m = __hmax2(__hmax2(e[0], e[1]), __hmax2(e[2], e[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
};
template <> struct Words<__half> {
  static constexpr int n = 8;
  static constexpr float kFar = 0x1p15f;
  __half2 e[4];
  static __device__ __forceinline__ __half2 low() { return __float2half2_rn(-kFar); }
  __device__ __forceinline__ void set(uint4 w) {
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
    for (int i = 0; i < 4; ++i) e[i] = __hmax2_nan(*reinterpret_cast<const __half2*>(&u[i]), low());
  }
  static __device__ __forceinline__ uint4 far() {
    const __half2 l = low();
    const unsigned v = *reinterpret_cast<const unsigned*>(&l);
    return make_uint4(v, v, v, v);
  }
  __device__ __forceinline__ float at(int i) const { return i & 1 ? __high2float(e[i / 2]) : __low2float(e[i / 2]); }
  static __device__ __forceinline__ f32x2 widen(__half2 v) {
    const float2 f = __half22float2(v);
    return pair_of(f.x, f.y);
  }
  __device__ __forceinline__ f32x2 two(int i) const { return widen(e[i]); }
  static __device__ __forceinline__ f32x2 pair(const uint4& w, int i) {
    const unsigned u = i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
    return widen(*reinterpret_cast<const __half2*>(&u));
  }
  __device__ __forceinline__ float largest() const {
    const __half2 m = __hmax2(__hmax2(e[0], e[1]), __hmax2(e[2], e[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
};

// What a part of a row comes to, in base 2: m the largest logit, s = sum 2^(c (x - m)), u = sum c (x - m) 2^(c (x - m)).
// The walk measures every logit against c m as it is rounded (one fma a logit), which is off by up to half a unit in the last place of
// c m, another amount for every thread's m.  So parts of a walk are joined by the distance of these shifts, and only the CTA's sums are
// taken to c m itself (to_largest): everything after that is measured against the largest logit, and logits that share a
// large offset lose no digits to it.
struct Stats {
  float m, s, u;
};
// Below this a shift's rounding changes the exponents by at most 32; from about 2^31 on it could take a sum to 0 or Inf.
constexpr float kMostShift = 0x1p30f;
__device__ __forceinline__ float shift_of(float m, float c) { return __fmul_rn(m, c); }   // never contracted into an fma
__device__ __forceinline__ Stats to_largest(const Stats& x, float c) {
  const float off = fmaf(x.m, c, -shift_of(x.m, c)), f = exp2f(-off);
  return Stats{x.m, x.s * f, (x.u - off * x.s) * f};
}
// c (x - m), of two logits' halves, whose distance cannot overflow
__device__ __forceinline__ float distance(float x, float m, float c) { return (0.5f * x - 0.5f * m) * (c + c); }
// Two parts measured against their largest logits.
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b, float c) {
  const float m = fmaxf(a.m, b.m);
  // the offsets are bounded so that 0 * offset stays 0; a part without sum keeps its zeros
  const float da = fmaxf(a.m == m ? 0.f : distance(a.m, m, c), -1e4f), db = fmaxf(b.m == m ? 0.f : distance(b.m, m, c), -1e4f);
  const float fa = fast_exp2(da), fb = fast_exp2(db);
  return Stats{m, a.s * fa + b.s * fb, (a.u + da * a.s) * fa + (b.u + db * b.s) * fb};
}
// All lanes' parts at once, measured against their shifts: scaled to the warp's largest, then summed; lanes without a part hold
// m = -Inf, s = u = 0.  (Lanes with one m in common are only summed, whatever they are measured against.)
__device__ __forceinline__ Stats warp_join(Stats x, float c) {
  const unsigned top = __reduce_max_sync(~0u, ordered(x.m));
  const float m = value_of(top);
  const float d = fmaxf(x.m == m ? 0.f : shift_of(x.m, c) - shift_of(m, c), -1e4f), f = fast_exp2(d);
  x.u = (x.u + d * x.s) * f;
  x.s *= f;
  for (int o = 16; o; o >>= 1) {
    x.s += __shfl_xor_sync(~0u, x.s, o);
    x.u += __shfl_xor_sync(~0u, x.u, o);
  }
  return Stats{m, x.s, x.u};
}
__device__ __forceinline__ Stats block_join(Stats x, float c, Stats* scratch) {
  x = warp_join(x, c);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
  __syncthreads();
  const int lane = threadIdx.x & 31;
  return warp_join(lane < kWarps ? scratch[lane] : Stats{-INFINITY, 0.f, 0.f}, c);
}

// The careful way: any values, any number of them, element by element.  [j0, j1) of the row.
template <typename T>
__device__ __noinline__ Stats careful_stats(const T* row, unsigned j0, unsigned j1, float c, Stats* scratch) {
  Stats x{-INFINITY, 0.f, 0.f};
  for (unsigned j = j0 + threadIdx.x; j < j1; j += kThreads) {
    x.m = fmaxf(x.m, to_f32(row[j]));
  }
  for (int o = 16; o; o >>= 1) x.m = fmaxf(x.m, __shfl_xor_sync(~0u, x.m, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5].m = x.m;
  __syncthreads();
  for (int w = 0; w < kWarps; ++w) x.m = fmaxf(x.m, scratch[w].m);
  for (unsigned j = j0 + threadIdx.x; j < j1; j += kThreads) {
    const float v = to_f32(row[j]);
    if (v == -INFINITY) continue;
    const float d = distance(v, x.m, c), e = exp2f(d);
    x.s += e;
    if (e != 0.f) x.u += e * d;
  }
  return block_join(x, c, scratch);
}
// The k largest keys of [j0, j1), in descending order in list[0 .. k): k walks, element by element.  1333 x 32000 fp32 with eight, where a
// row takes this way: 49 -> 370-450 us; one row of 50257 bfloat16, some of whose eight parts do: 13 -> 25 us.
template <typename T>
__device__ __noinline__ void careful_top(const T* row, unsigned j0, unsigned j1, int k, unsigned long long* list,
                                         unsigned long long* scratch) {
  unsigned long long last = ~0ull;
  for (int i = 0; i < k; ++i) {
    unsigned long long best = 0;
    for (unsigned j = j0 + threadIdx.x; j < j1; j += kThreads) {
      const unsigned long long q = key_of(to_f32(row[j]), j);
      if (q < last && q > best) best = q;
    }
    best = warp_max(best);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = best;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) best = scratch[w] > best ? scratch[w] : best;
    last = best;
    if (threadIdx.x == 0) list[i] = best;
  }
  __syncthreads();
}

// One warp, one value per lane (0: none): the k largest, descending, to list[0 .. k) (0 where there are no more).
__device__ __forceinline__ void warp_largest(unsigned v, int k, unsigned* list) {
  const int lane = threadIdx.x & 31;
  for (int i = 0; i < k; ++i) {
    const unsigned best = __reduce_max_sync(~0u, v), holders = __ballot_sync(~0u, v == best);
    if (lane == __ffs(holders) - 1) v = 0;
    if (lane == 0) list[i] = best;
  }
}
// One warp: the k-th largest of list[0 .. n), n <= 256, counting equal ones separately.
__device__ __forceinline__ unsigned warp_kth(const unsigned* list, int n, int k) {
  const int lane = threadIdx.x & 31;
  unsigned held[8], best = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) held[j] = lane + 32 * j < n ? list[lane + 32 * j] : 0;
  for (int i = 0; i < k; ++i) {
    unsigned mine = held[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) mine = max(mine, held[j]);
    best = __reduce_max_sync(~0u, mine);
    const unsigned holders = __ballot_sync(~0u, mine == best);
    if (lane == __ffs(holders) - 1) {
      bool gone = false;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!gone && held[j] == best) { held[j] = 0; gone = true; }
      }
    }
  }
  return best;
}

// One warp: the k largest of keys[0 .. n), descending, to list[0 .. k) (0 where there are no more).
template <int PER> __device__ __forceinline__ void warp_top_held(const unsigned long long* keys, int n, int k, unsigned long long* list) {
  const int lane = threadIdx.x & 31;
  unsigned long long held[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) held[j] = lane + 32 * j < n ? keys[lane + 32 * j] : 0;
  __syncwarp();
  for (int i = 0; i < k; ++i) {
    unsigned long long best = held[0];
#pragma unroll
    for (int j = 1; j < PER; ++j) best = held[j] > best ? held[j] : best;
    best = warp_max(best);
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (held[j] == best) held[j] = 0;
    if (lane == 0) list[i] = best;
  }
  __syncwarp();
}
__device__ __forceinline__ void warp_top(const unsigned long long* keys, int n, int k, unsigned long long* list) {
  if (n <= 64) return warp_top_held<2>(keys, n, k, list);
  if (n <= 256) return warp_top_held<8>(keys, n, k, list);
  const int lane = threadIdx.x & 31;
  unsigned long long last = ~0ull;
  for (int i = 0; i < k; ++i) {
    unsigned long long best = 0;
    for (int j = lane; j < n; j += 32)
      if (keys[j] < last && keys[j] > best) best = keys[j];
    last = best = warp_max(best);
    if (lane == 0) list[i] = best;
  }
  __syncwarp();
}

constexpr int kUnroll = 4;           // 16-byte loads in flight per thread (fp32 rows without alternatives: 6, see k_logprobs)
constexpr int kCandidates = 1024;
constexpr int kMaxTop = COCODC_LM_MAX_TOP;

template <int N, bool PARTIAL> struct Batch {     // words of a step; PARTIAL: some may lie beyond the end
  static constexpr int value = N;
  static constexpr bool partial = PARTIAL;
};

struct RowShared {
  Stats scratch[kWarps];
  Stats part;                                       // this CTA's part of the row, read by the cluster's first CTA
  unsigned long long warp_keys[kWarps];
  unsigned lists[kWarps * kMaxTop];                 // the warps' largest thread maxima
  unsigned long long top[kMaxTop];                  // this CTA's part's largest keys
  unsigned long long candidates[kCandidates];
  unsigned long long gathered[8 * kMaxTop], merged[kMaxTop];   // first CTA: the parts' lists, the row's
  int flagged[kThreads], n_flagged, n_candidates;
  unsigned tau;
};

// A row is read once: bound by memory, closely followed by the issue slots (7 instructions a logit: unpacking, fma, exponential,
// two sums, maximum).  8192 x 50257 bfloat16 in 145-153 us (5.4-5.7 TB/s), 1333 x 32000 fp32 with five alternatives in
// 35 us, one row of 50257 with eight in 8.1 us, without in 4.0 (in a graph).  Each thread keeps (m, s, u) of its own elements, rescaled when its largest logit grows, in
// batches of kUnroll 16-byte words; the parts are joined through shuffles and shared memory, and between the CTAs of a cluster (a row is
// split over 1 to 8 CTAs, so that few rows still fill the GPU) through distributed shared memory.
//
// Where nothing stands in the way, the alternatives cost the walk nothing: tau, the k-th largest of the threads' largest logits, is not above the k-th
// largest logit, so every alternative lies with a thread whose largest logit is at least tau.  Only what those threads saw
// is read again (from L2), and of it only logits >= tau are sorted, by value and position.  The careful way instead: rows (of a few
// rows, parts of a row) with a NaN or +Inf, with fewer threads that hold a logit above -kFar than alternatives, with more than
// kCandidates equal logits at the border, and those whose sums have to be taken with care.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) k_logprobs(const RowArgs a, int parts) {
  wait_for_previous();
  may_follow();
  using W = Words<T>;
  // loads in flight per thread: six at fp32 (4000 x 50257: 130 -> 120 us); with alternatives, or twice the logits per word, the
  // registers that takes cost more CTAs than it gives (bf16: 70 -> 81 us)
  constexpr int kAhead = sizeof(T) == 4 && !TOP ? 6 : kUnroll;
  __shared__ RowShared sh;
  const long long t = blockIdx.x / parts;
  const int part = blockIdx.x - (int)(t * parts);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  const float c = a.scale * kLog2e;

  // [j0, j1): this CTA's part; whole 16-byte words from `base` on, what is left at the row's ends goes element by element
  const unsigned lead = min(a.V, (unsigned)((16 - ((uintptr_t)row & 15)) & 15) / (unsigned)sizeof(T));
  const unsigned words = (a.V - lead) / W::n, per = (words + parts - 1) / parts;
  const unsigned w0 = min(words, part * per), w1 = min(words, w0 + per), n = w1 - w0;
  const unsigned j0 = part == 0 ? 0 : lead + w0 * W::n, j1 = part == parts - 1 ? a.V : lead + w1 * W::n;
  const unsigned base = lead + w0 * W::n, tail = lead + w1 * W::n;
  const uint4* src = reinterpret_cast<const uint4*>(row + base);

  // the target's logit is on its way before the walk
  long long y = -1;
  float target = 0.f;
  if (a.logp && part == 0 && tid == 0) {
    y = token_at(a.targets, a.targets64, t, a.V, a.status);
    if (y >= 0) target = to_f32(row[y]);
  }
  Stats x{-W::kFar, 0.f, 0.f};
  f32x2 s2 = 0, u2 = 0;                                      // sums of the even and the odd elements
  f32x2 less2 = pair_of(-shift_of(x.m, c), -shift_of(x.m, c));   // minus the shift, twice
  const auto less = [&] {
    float lo, hi;
    split(less2, lo, hi);
    return lo;
  };
  const f32x2 c2 = pair_of(c, c);
  const auto raise = [&](float m) {
    const float to = shift_of(m, c), d = fmaxf(-(less() + to), -1e4f), f = exp2f(d);
    u2 = mul2(fma2(pair_of(d, d), s2, u2), pair_of(f, f));
    s2 = mul2(s2, pair_of(f, f));
    x.m = m;
    less2 = pair_of(-to, -to);
  };
  const auto add = [&](f32x2 v) {
    const f32x2 d = fma2(v, c2, less2);
    float lo, hi;
    split(d, lo, hi);
    const f32x2 e = pair_of(fast_exp2(lo), fast_exp2(hi));
    s2 = add2(s2, e);
    u2 = fma2(e, d, u2);
  };
  const auto single = [&](unsigned j) {
    float v;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(to_f32(row[j])), "f"(-W::kFar));
    if (v > x.m) raise(v);
    const float d = fmaf(v, c, less()), e = fast_exp2(d);
    s2 = add2(s2, pair_of(e, 0.f));
    u2 = add2(u2, pair_of(e * d, 0.f));
  };
  if (j0 + tid < base) single(j0 + tid);
  const auto words_at = [&](unsigned i, auto count) {
    constexpr int N = decltype(count)::value;
    uint4 raw[N];
    W w[N];
#pragma unroll
    for (int k = 0; k < N; ++k) raw[k] = !count.partial || i + k * kThreads < n ? load16(src + i + k * kThreads) : W::far();
#pragma unroll
    for (int k = 0; k < N; ++k) w[k].set(raw[k]);
    float m = w[0].largest();
#pragma unroll
    for (int k = 1; k < N; ++k) m = fmaxf(m, w[k].largest());
    if (m > x.m) raise(m);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int q = 0; q < W::n / 2; ++q) add(w[k].two(q));
  };
  unsigned i = tid;
  for (; i + (kAhead - 1) * kThreads < n; i += kThreads * kAhead) words_at(i, Batch<kAhead, false>());
  if (i + kThreads < n) words_at(i, Batch<kAhead, true>());   // the last words in one round trip
  else if (i < n) words_at(i, Batch<1, false>());
  if (tail + tid < j1) single(tail + tid);
  {
    float lo, hi;
    split(s2, lo, hi);
    x.s = lo + hi;
    split(u2, lo, hi);
    x.u = lo + hi;
  }
  // the thread's largest logit; 0: nothing above -kFar
  const unsigned largest = TOP && x.m > -W::kFar ? ordered(x.m) : 0;
  if (TOP) {
    warp_largest(largest, a.top_k, sh.lists + warp * a.top_k);
    if (tid == 0) sh.n_flagged = sh.n_candidates = 0;
  }
  x = block_join(x, c, sh.scratch);
  // a NaN or +Inf, nothing but very low logits, a very small scale, a very large product of scale and largest logit: once more, with
  // care (also the alternatives)
  const bool careful = !(x.m > -W::kFar / 2) || !(x.s + fabsf(x.u) < INFINITY) || !(c * (W::kFar / 2) > 200.f) ||
                       !(fabsf(shift_of(x.m, c)) < kMostShift);
  x = careful ? careful_stats(row, j0, j1, c, sh.scratch) : to_largest(x, c);

  if (TOP) {
    bool done = false;
    if (!careful) {
      if (warp == 0) {
        const unsigned t0 = warp_kth(sh.lists, kWarps * a.top_k, a.top_k);
        if (lane == 0) sh.tau = t0;
      }
      __syncthreads();
      const unsigned tau = sh.tau;
      // tau 0: fewer threads than alternatives hold anything; leave it to the careful way
      if (tau != 0) {
        if (largest >= tau) sh.flagged[atomicAdd(&sh.n_flagged, 1)] = tid;
        __syncthreads();
        const auto offer = [&](float v, unsigned j) {
          if (ordered(v) < tau) return;
          const int slot = atomicAdd(&sh.n_candidates, 1);
          if (slot < kCandidates) sh.candidates[slot] = key_of(v, j);
        };
        for (int f = warp; f < sh.n_flagged; f += kWarps) {
          const unsigned who = sh.flagged[f];
          if (lane == 0 && j0 + who < base) offer(to_f32(row[j0 + who]), j0 + who);
          if (lane == 1 && tail + who < j1) offer(to_f32(row[tail + who]), tail + who);
          for (unsigned i = who + lane * kThreads; i < n; i += 32 * kThreads) {
            W w;
            w.set(load16(src + i));
            if (ordered(w.largest()) < tau) continue;
#pragma unroll
            for (int q = 0; q < W::n; ++q) offer(w.at(q), base + i * W::n + q);
          }
        }
        __syncthreads();
        // many equal logits at the border may not fit the list
        done = sh.n_candidates <= kCandidates;
        if (done && warp == 0) warp_top(sh.candidates, sh.n_candidates, a.top_k, sh.top);
      }
    }
    if (!done) careful_top(row, j0, j1, a.top_k, sh.top, sh.warp_keys);
  }

  // the parts of the row come together in the cluster's first CTA
  const unsigned long long* top = sh.top;
  if (parts > 1) {
    if (tid == 0) sh.part = x;
    cluster_barrier();
    if (part == 0) {
      if (tid == 0) {
        const unsigned here = (unsigned)__cvta_generic_to_shared(&sh.part);
        for (int p = 1; p < parts; ++p) {
          unsigned there;
          Stats y;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(p));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(y.m) : "r"(there));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(y.s) : "r"(there + 4));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(y.u) : "r"(there + 8));
          x = join(x, y, c);
        }
      }
      if (TOP) {
        const unsigned here = (unsigned)__cvta_generic_to_shared(sh.top);
        for (int i = tid; i < parts * a.top_k; i += kThreads) {
          unsigned there;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here + i % a.top_k * 8), "r"(i / a.top_k));
          asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(sh.gathered[i]) : "r"(there));
        }
        __syncthreads();
        if (warp == 0) warp_top(sh.gathered, parts * a.top_k, a.top_k, sh.merged);
        top = sh.merged;
      }
    }
    // the others' shared memory stays until it has been read
    cluster_barrier();
    if (part != 0) return;
  }

  if (warp != 0) return;
  const bool empty = x.m == -INFINITY && x.s == 0.f;
  const float log_s = __shfl_sync(~0u, empty ? -INFINITY : kLn2 * log2f(x.s), 0), m = __shfl_sync(~0u, x.m, 0);
  const bool none = __shfl_sync(~0u, (int)empty, 0);
  const auto logp_of = [&](float v) { return none ? -INFINITY : distance(v, m, a.scale) - log_s; };
  if (lane == 0) {
    if (a.lse) a.lse[t] = none ? -INFINITY : __fmul_rn(m, a.scale) + log_s;
    if (a.entropy) a.entropy[t] = none ? 0.f : log_s - kLn2 * (x.u / x.s);
    if (a.logp) a.logp[t] = y < 0 ? 0.f : logp_of(target);
  }
  if (TOP && lane < a.top_k) {
    a.top_ids[t * a.top_k + lane] = (int)position_of(top[lane]);
    a.top_logp[t * a.top_k + lane] = logp_of(value_of((unsigned)(top[lane] >> 32)));
  }
}

struct GradArgs {
  const void* logits;
  long long stride, T;
  unsigned V;
  const void* targets;
  int targets64;
  float scale;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* dlogits;
  long long dstride;
  int* status;
};

// One read and one write of every logit: bound by memory (8192 x 50257 bfloat16 in 278-281 us, 5.9 TB/s).  A CTA takes a row or
// an even part of it: seven CTAs to a row, each with its own set-up, took 303 us.
template <typename T> struct Out;   // packs results the way Words unpacks logits
template <> struct Out<float> {
  static __device__ __forceinline__ uint4 of(const float (&d)[4]) {
    return make_uint4(__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3]));
  }
};
template <typename T2, typename F> __device__ __forceinline__ uint4 pack8(const float (&d)[8], F&& pair) {
  unsigned u[4];
  for (int i = 0; i < 4; ++i) {
    const T2 v = pair(d[2 * i], d[2 * i + 1]);
    u[i] = *reinterpret_cast<const unsigned*>(&v);
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}
template <> struct Out<__nv_bfloat16> {
  static __device__ __forceinline__ uint4 of(const float (&d)[8]) {
    return pack8<__nv_bfloat162>(d, [](float x, float y) { return __floats2bfloat162_rn(x, y); });
  }
};
template <> struct Out<__half> {
  static __device__ __forceinline__ uint4 of(const float (&d)[8]) {
    return pack8<__half2>(d, [](float x, float y) { return __floats2half2_rn(x, y); });
  }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 8) k_logprobs_grad(const GradArgs a, unsigned chunks) {
  wait_for_previous();
  may_follow();
  constexpr int n = 16 / sizeof(T);
  const long long t = blockIdx.x / chunks;
  const unsigned chunk = blockIdx.x - (unsigned)(t * chunks);
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  T* out = static_cast<T*>(a.dlogits) + t * a.dstride;
  const long long y = a.dlogp ? token_at(a.targets, a.targets64, t, a.V, a.status) : -1;
  const float lse = a.lse[t];
  // the scale goes into the coefficients; a row without valid probabilities (lse NaN or beyond fp32's range) gets NaN everywhere
  float g = y >= 0 ? a.scale * a.dlogp[t] : 0.f;
  const float h = a.dentropy ? a.scale * a.dentropy[t] : 0.f, H = a.dentropy ? a.entropy[t] : 0.f;
  if (!(lse < INFINITY)) g = NAN;
  const bool none = lse == -INFINITY;
  // -p (g + h (log p + H)), the bracket as one fma of log p; log p is kept above -1e4, where p is 0, so that a masked logit's -Inf
  // does not meet that 0.  The product with the scale is rounded before lse is taken off, as it was in lse: the largest logit's
  // log p is then never above 0, while in one fma the product's rounding would stay and be exponentiated.  (As single products: of a
  // product of pairs and a sum of pairs that fma is made all the same.)
  const f32x2 lse2 = pair_of(-lse, -lse), log2e2 = pair_of(kLog2e, kLog2e),
              slope = pair_of(-h, -h), level = pair_of(-fmaf(h, H, g), -fmaf(h, H, g));
  const auto slope2 = [&](f32x2 x) {
    float lo, hi;
    split(x, lo, hi);
    split(add2(pair_of(__fmul_rn(lo, a.scale), __fmul_rn(hi, a.scale)), lse2), lo, hi);
    const f32x2 lp = pair_of(fmaxf(lo, -1e4f), fmaxf(hi, -1e4f));
    split(mul2(lp, log2e2), lo, hi);
    const f32x2 p = pair_of(fast_exp2(lo), fast_exp2(hi));
    return mul2(p, fma2(slope, lp, level));
  };
  const auto single = [&](unsigned j) {
    float d, other;
    split(slope2(pair_of(to_f32(row[j]), 0.f)), d, other);
    out[j] = from_f32<T>(none ? 0.f : d + (j == y ? g : 0.f));
  };
  if (((uintptr_t)row ^ (uintptr_t)out) & 15) {         // no common 16-byte boundaries
    const unsigned per = (a.V + chunks - 1) / chunks, j1 = min((unsigned long long)a.V, (chunk + 1ull) * per);
    for (unsigned long long j = (unsigned long long)chunk * per + threadIdx.x; j < j1; j += kThreads) single((unsigned)j);
    return;
  }
  const unsigned lead = min(a.V, (unsigned)((16 - ((uintptr_t)row & 15)) & 15) / (unsigned)sizeof(T));
  const unsigned words = (a.V - lead) / n, tail = lead + words * n;
  if (chunk == 0 && threadIdx.x < lead) single(threadIdx.x);
  if (chunk == chunks - 1 && tail + threadIdx.x < a.V) single(tail + threadIdx.x);
  const uint4* src = reinterpret_cast<const uint4*>(row + lead);
  uint4* dst = reinterpret_cast<uint4*>(out + lead);
  // the row's words dealt evenly to its CTAs
  const unsigned per = (words + chunks - 1) / chunks, end = min(words, (chunk + 1) * per);
  const long long hit_word = y < (long long)lead || y >= (long long)tail ? -1 : (y - lead) / n;
  // neither the logits nor the gradient are needed again soon (streaming accesses: 310 -> 293 us at 8192 x 50257, when the rest took longer)
  const auto words_at = [&](unsigned i, auto count) {
    constexpr int N = decltype(count)::value;
    uint4 raw[N];
#pragma unroll
    for (int k = 0; k < N; ++k) raw[k] = __ldcs(src + i + k * kThreads);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float d[n];
#pragma unroll
      for (int q = 0; q < n / 2; ++q) split(slope2(Words<T>::pair(raw[k], q)), d[2 * q], d[2 * q + 1]);
      if (i + k * kThreads == hit_word) {
        const int hit = (int)(y - lead) % n;
#pragma unroll
        for (int q = 0; q < n; ++q) d[q] += q == hit ? g : 0.f;
      }
      __stcs(dst + i + k * kThreads, Out<T>::of(d));
    }
  };
  unsigned i = chunk * per + threadIdx.x;
  if (none) {
    for (; i < end; i += kThreads) dst[i] = make_uint4(0, 0, 0, 0);
    return;
  }
  for (; i + (kUnroll - 1) * kThreads < end; i += kThreads * kUnroll) words_at(i, std::integral_constant<int, kUnroll>());
  for (; i < end; i += kThreads) words_at(i, std::integral_constant<int, 1>());
}

}  // namespace

extern "C" {

cocodc_status cocodc_lm_logprobs(cocodc_lm* lm, const void* logits, int32_t type, int64_t stride, int64_t T, int64_t V,
                                 const void* targets, int32_t targets_type, float scale, float* logp, float* entropy,
                                 float* lse, int32_t top_k, int32_t* top_ids, float* top_logp, void* stream) {
  if (!lm || !known_type(type) || !sane(T) || T > INT32_MAX || V < 1 || V > INT32_MAX || stride < V || !sane(stride) ||
      !(scale > 0.f && scale <= kMostScale) || top_k < 0 || top_k > COCODC_LM_MAX_TOP || top_k > V)
    return COCODC_ERR_INVALID_ARG;
  if (T == 0) return COCODC_OK;
  if ((targets == nullptr) != (logp == nullptr) || (top_k > 0) != (top_ids != nullptr) || (top_k > 0) != (top_logp != nullptr) ||
      (targets && targets_type != COCODC_I32 && targets_type != COCODC_I64))
    return COCODC_ERR_INVALID_ARG;
  if (!logits || (!logp && !entropy && !lse && top_k == 0)) return COCODC_ERR_INVALID_ARG;
  const int es = type_bytes(type);
  if (!on_boundary(logits, es) || (targets && !on_boundary(targets, index_bytes(targets_type))) || !on_boundary(logp, 4) ||
      !on_boundary(entropy, 4) || !on_boundary(lse, 4) || !on_boundary(top_ids, 4) || !on_boundary(top_logp, 4))
    return COCODC_ERR_ALIGNMENT;
  const Span in[2] = {span(logits, T, stride, V, es), span(targets, 1, T, T, targets ? index_bytes(targets_type) : 1)};
  const Span out[5] = {span(logp, 1, T, T, 4), span(entropy, 1, T, T, 4), span(lse, 1, T, T, 4),
                       span(top_ids, top_k ? T : 0, top_k, top_k, 4), span(top_logp, top_k ? T : 0, top_k, top_k, 4)};
  for (int i = 0; i < 5; ++i) {
    if (meet(out[i], in[0]) || meet(out[i], in[1])) return COCODC_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return COCODC_ERR_ALIAS;
  }
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  const RowArgs a{logits, stride, T, (unsigned)V, targets, targets_type == COCODC_I64, scale, logp, entropy, lse,
                  top_k, top_ids, top_logp, lm->d_status};
  // few rows: each over as many CTAs (a cluster) as it takes to give every SM one, but at least 4 KB of the row to each; to
  // give every SM two where 48 KB remain to each (200 rows of 50257 fp32: 20 -> 14.5 us; with shorter parts the joining costs
  // more: 64 rows of 50257 bf16 5.5 -> 6.5 us)
  int parts = 1;
  while (parts < 8 && T * parts < lm->sm_count && V * es >= 8192 * parts) parts *= 2;
  while (parts < 8 && T * parts < 2 * lm->sm_count && V * es >= 2 * 49152 * parts) parts *= 2;
  if (T > INT32_MAX / parts) return COCODC_ERR_INVALID_ARG;
  return with_type(type, [&](auto x) {
    using E = decltype(x);
    return start(lm, top_k ? k_logprobs<E, true> : k_logprobs<E, false>, (unsigned)(T * parts), kThreads, 0,
                 static_cast<cudaStream_t>(stream), (unsigned)parts, a, parts);
  });
}

cocodc_status cocodc_lm_logprobs_grad(cocodc_lm* lm, const void* logits, int32_t type, int64_t stride, int64_t T,
                                      int64_t V, const void* targets, int32_t targets_type, float scale,
                                      const float* lse, const float* entropy, const float* dlogp,
                                      const float* dentropy, void* dlogits, int64_t dlogits_stride, void* stream) {
  if (!lm || !known_type(type) || !sane(T) || T > INT32_MAX || V < 1 || V > INT32_MAX || stride < V || !sane(stride) ||
      dlogits_stride < V || !sane(dlogits_stride) || !(scale > 0.f && scale <= kMostScale))
    return COCODC_ERR_INVALID_ARG;
  if (T == 0) return COCODC_OK;
  if (!logits || !lse || !dlogits || (!dlogp && !dentropy) || (targets == nullptr) != (dlogp == nullptr) ||
      (dentropy && !entropy) || (targets && targets_type != COCODC_I32 && targets_type != COCODC_I64))
    return COCODC_ERR_INVALID_ARG;
  const int es = type_bytes(type);
  if (!on_boundary(logits, es) || !on_boundary(dlogits, es) || !on_boundary(lse, 4) || !on_boundary(entropy, 4) ||
      !on_boundary(dlogp, 4) || !on_boundary(dentropy, 4) || (targets && !on_boundary(targets, index_bytes(targets_type))))
    return COCODC_ERR_ALIGNMENT;
  const Span out = span(dlogits, T, dlogits_stride, V, es);
  const bool in_place = dlogits == logits && dlogits_stride == stride;
  if ((!in_place && meet(out, span(logits, T, stride, V, es))) ||
      meet(out, span(targets, 1, T, T, targets ? index_bytes(targets_type) : 1)) || meet(out, span(lse, 1, T, T, 4)) ||
      meet(out, span(entropy, 1, T, T, 4)) || meet(out, span(dlogp, 1, T, T, 4)) || meet(out, span(dentropy, 1, T, T, 4)))
    return COCODC_ERR_ALIAS;
  // whole rows amortise what a CTA does once per row; few rows are split so that there are CTAs for all SMs, down to the
  // four 16-byte words that a thread has in flight
  const long long most = (V * es + kThreads * kUnroll * 16 - 1) / (kThreads * kUnroll * 16);
  const long long wanted = (16LL * lm->sm_count + T - 1) / T;
  const long long chunks = wanted < most ? wanted : most, blocks = T * chunks;
  if (blocks > INT32_MAX) return COCODC_ERR_INVALID_ARG;
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  const GradArgs a{logits, stride, T, (unsigned)V, targets, targets_type == COCODC_I64, scale, lse, entropy, dlogp,
                   dentropy, dlogits, dlogits_stride, lm->d_status};
  return with_type(type, [&](auto x) {
    return start(lm, k_logprobs_grad<decltype(x)>, (unsigned)blocks, kThreads, 0, static_cast<cudaStream_t>(stream), 1, a,
                 (unsigned)chunks);
  });
}

}  // extern "C"
