// The root-mean-square norm with the residual's addition and its gradient (include/cocodc_lm.h).

#include "lm_mma.cuh"

#include <type_traits>

using namespace cocodc_lm_impl;

namespace {

constexpr int kThreads = 256;
constexpr float kMost8 = 448.f, kLeastScale = 1e-30f;

// ---- elements ----------------------------------------------------------------------------------------
// Eight elements of a row as they lie in memory, fetched before they are needed.
template <typename T> struct Raw8 { uint4 q[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ Raw8<T> fetch8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.q[i] = load16(p + i * (16 / sizeof(T)));
  return r;
}
__device__ __forceinline__ void widen(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[4 * i] = __uint_as_float(r.q[i].x);
    v[4 * i + 1] = __uint_as_float(r.q[i].y);
    v[4 * i + 2] = __uint_as_float(r.q[i].z);
    v[4 * i + 3] = __uint_as_float(r.q[i].w);
  }
}
template <typename T> __device__ __forceinline__ void widen(const Raw8<T>& r, float (&v)[8]) {
  const unsigned w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same_v<T, __nv_bfloat16>) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
}
template <typename T> __device__ __forceinline__ Raw8<T> narrow8(const float (&v)[8]) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      r.q[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
  } else {
    r.q[0] = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
  }
  return r;
}
// fp32: both halves of a 32-byte sector in one store where its address allows (65536 x 1024 with fp32 sums: 140 -> 134 us)
template <typename T> __device__ __forceinline__ void store_raw(T* p, const Raw8<T>& r) {
  if constexpr (sizeof(T) == 4) {
    if ((reinterpret_cast<unsigned long long>(p) & 31) == 0) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r.q[0].x), "r"(r.q[0].y), "r"(r.q[0].z), "r"(r.q[0].w),
                   "r"(r.q[1].x), "r"(r.q[1].y), "r"(r.q[1].z), "r"(r.q[1].w) : "memory");
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = r.q[i];
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]) { store_raw(p, narrow8<T>(v)); }
// x + u, rounded to u's type: of one 16-bit type by pairs, otherwise in fp32 and then by pairs
template <typename X, typename S> __device__ __forceinline__ Raw8<S> sum8(const Raw8<X>& x, const Raw8<S>& u) {
  if constexpr (std::is_same_v<X, S> && sizeof(S) == 2) {
    using Two = std::conditional_t<std::is_same_v<S, __half>, __half2, __nv_bfloat162>;
    const auto add = [](unsigned a, unsigned b) {
      const Two v = __hadd2(*reinterpret_cast<const Two*>(&a), *reinterpret_cast<const Two*>(&b));
      return *reinterpret_cast<const unsigned*>(&v);
    };
    Raw8<S> r;
    r.q[0] = make_uint4(add(x.q[0].x, u.q[0].x), add(x.q[0].y, u.q[0].y), add(x.q[0].z, u.q[0].z), add(x.q[0].w, u.q[0].w));
    return r;
  } else {
    float v[8], q[8];
    widen(x, v);
    widen(u, q);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += q[i];
    return narrow8<S>(v);
  }
}
// two numbers to the nearest e4m3, the first in the lower byte
__device__ __forceinline__ unsigned narrow_e4m3(float a, float b) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
// v / scale rounded once (v times the inverse is up to an ulp off, which at a border gives another code), by Markstein's division: the rounded inverse
// by a Newton step from an approximate one, then what the product with it leaves of v divided too.  scale is normal, or infinite: finite numbers
// then become 0, infinite ones NaN.  4099 x 3200: 19.3 us, 18.5 with the product alone.
struct Divide {
  float scale, inv;
  __device__ __forceinline__ explicit Divide(float s) : scale(s < INFINITY ? s : 0.f) {
    inv = __fdividef(1.f, s);
    inv = fmaf(fmaf(-scale, inv, 1.f), inv, inv);
  }
  __device__ __forceinline__ float operator()(float v) const {
    const float q = v * inv;
    return fmaf(fmaf(-q, scale, v), inv, q);
  }
  // a pair by packed instructions, as e4m3 codes
  __device__ __forceinline__ unsigned codes(float a, float b) const {
    asm("{\n .reg .b64 v, i, s, q, r;\n mov.b64 v, {%0, %1};\n mov.b64 i, {%2, %2};\n mov.b64 s, {%3, %3};\n mul.rn.f32x2 q, v, i;\n"
        " fma.rn.f32x2 r, q, s, v;\n fma.rn.f32x2 q, r, i, q;\n mov.b64 {%0, %1}, q;\n}" : "+f"(a), "+f"(b) : "f"(inv), "f"(-scale));
    return narrow_e4m3(a, b);
  }
};
__device__ __forceinline__ float load_as(const void* p, int type, long long i) {
  return type == COCODC_F32    ? static_cast<const float*>(p)[i]
         : type == COCODC_BF16 ? to_f32(static_cast<const __nv_bfloat16*>(p)[i])
                               : to_f32(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_as(void* p, int type, long long i, float v) {
  if (type == COCODC_F32) static_cast<float*>(p)[i] = v;
  else if (type == COCODC_BF16) static_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(v);
  else if (type == COCODC_F16) static_cast<__half*>(p)[i] = from_f32<__half>(v);
  else static_cast<unsigned char*>(p)[i] = (unsigned char)narrow_e4m3(v, 0.f);
}

// ---- a row in registers ---------------------------------------------------------------------------------
// A group of G threads (whole warps, as many as the row's columns fill) holds a row, 8 P columns each; a block has as many groups as
// make 256 threads, and each strides on by itself.  Where rows are whole packs of eight columns on 16-byte boundaries (WIDE) a thread's columns are such
// packs, otherwise single ones G apart, so that neighbours read neighbours either way.
template <int P, bool WIDE> struct Row {
  int G, t;                                          // threads of the group, this one's number
  __device__ __forceinline__ int column(int p, int i) const { return WIDE ? (p * G + t) * 8 + i : (p * 8 + i) * G + t; }
};
// Rows on their way (WIDE): a ring of stages in shared memory for each group, filled by bulk copies of whole rows, up to three arrays' rows to a stage.
// A stage is read into registers before the row's sum is joined, and filled again right after.  A wait that gives up lets its
// warp go on (the group's barriers need all of them) without writing anything.
constexpr int kMostStages = 3;
struct Ring {
  unsigned base, bar, bytes, stages, turn, issued;
  volatile int* stop;
  bool ok;
  __device__ __forceinline__ unsigned stage() const { return base + turn % stages * bytes; }
  __device__ __forceinline__ unsigned barrier() const { return bar + turn % stages * 8; }
  // the copies in flight land before the block leaves its shared memory (who issued them has waited for all of them as long as it is ok)
  __device__ __forceinline__ void drain() const {
    for (unsigned i = issued > stages ? issued - stages : 0; i < issued; ++i) bar_drain(bar + i % stages * 8, (i / stages) & 1);
  }
  // one answer for a warp, whose lanes go on together
  __device__ __forceinline__ void wait() { ok = __all_sync(~0u, bar_wait(barrier(), (turn / stages) & 1, stop)) && ok; }
};
__device__ __forceinline__ Ring ring_of(unsigned char* memory, unsigned long long (*bars)[kMostStages], int* stop, int group, unsigned bytes, unsigned stages) {
  return Ring{smem_addr(memory) + group * stages * bytes, smem_addr(&bars[group][0]), bytes, stages, 0, 0, stop, true};
}
__device__ __forceinline__ void ring_start(unsigned long long (*bars)[kMostStages], int* stop) {
  if (threadIdx.x < kThreads / 32 * kMostStages) bar_init(smem_addr(&bars[0][0]) + threadIdx.x * 8, 1);
  if (threadIdx.x == 0) *stop = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncthreads();
}
// All threads of the block: a wait that gave up is recorded whichever warp's it was, since the group's others may have been in time.
__device__ __forceinline__ void ring_end(const Ring& ring, bool issuer, int* status) {
  if (issuer && !ring.ok) ring.drain();
  __syncthreads();
  if (threadIdx.x == 0 && *ring.stop) record(status, COCODC_ERR_TIMEOUT);
}
template <typename T> __device__ __forceinline__ Raw8<T> staged8(unsigned at) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i)
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.q[i].x), "=r"(r.q[i].y), "=r"(r.q[i].z), "=r"(r.q[i].w) : "r"(at + i * 16));
  return r;
}

// Pack p of a row from its place in a stage; columns behind the row's end are zero.
template <typename T, int P> __device__ __forceinline__ void get(const Row<P, true>& r, unsigned staged, int D, int p, float (&v)[8]) {
  const int c = r.column(p, 0);
  if (c < D) widen(staged8<T>(staged + c * (unsigned)sizeof(T)), v);
  else
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
}
// Rows that are not whole packs: a row's columns on their way in registers (gradient of 10392 x 601 bf16: 33 us, 60 without).
template <typename T, int P, bool WIDE> struct Ahead {
  T one[WIDE ? 1 : P * 8];
  __device__ __forceinline__ void fetch(const Row<P, WIDE>& r, const T* row, int D) {
    if constexpr (!WIDE) {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) one[p * 8 + i] = r.column(p, i) < D ? row[r.column(p, i)] : from_f32<T>(0.f);
    }
  }
  __device__ __forceinline__ void get(int p, float (&v)[8]) const {
    if constexpr (!WIDE) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = to_f32(one[p * 8 + i]);
    }
  }
};
template <typename T, int P, bool WIDE> __device__ __forceinline__ void put(const Row<P, WIDE>& r, T* row, int D, int p, const float (&v)[8]) {
  if (WIDE) {
    if (r.column(p, 0) < D) store8(row + r.column(p, 0), v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (r.column(p, i) < D) row[r.column(p, i)] = from_f32<T>(v[i]);
  }
}
template <int P, bool WIDE> __device__ __forceinline__ void put_type(const Row<P, WIDE>& r, void* y, int type, long long at, int D, int p, const float (&v)[8]) {
  if (type == COCODC_F32) put<float>(r, static_cast<float*>(y) + at, D, p, v);
  else if (type == COCODC_BF16) put<__nv_bfloat16>(r, static_cast<__nv_bfloat16*>(y) + at, D, p, v);
  else put<__half>(r, static_cast<__half*>(y) + at, D, p, v);
}
// The weights of a thread's columns, read once for all of its rows.
template <int P, bool WIDE> __device__ __forceinline__ void fetch_weight(const Row<P, WIDE>& r, const void* w, int type, int D, float (&v)[P][8]) {
  const auto take = [&](auto e) {
    using T = decltype(e);
    const T* p0 = static_cast<const T*>(w);
    if (WIDE && (reinterpret_cast<unsigned long long>(w) & 15) == 0) {
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (r.column(p, 0) < D) widen(fetch8(p0 + r.column(p, 0)), v[p]);
        else
#pragma unroll
          for (int i = 0; i < 8; ++i) v[p][i] = 0.f;
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[p][i] = r.column(p, i) < D ? to_f32(p0[r.column(p, i)]) : 0.f;
    }
  };
  if (type == COCODC_F32) take(float());
  else if (type == COCODC_BF16) take(__nv_bfloat16());
  else take(__half());
}

struct Plus { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct Most { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };
// Sums or maxima over the threads of a row's group.  Above a warp they meet in shared memory, in two buffers in turn: one barrier of
// the group each.
struct Join {
  float (*cell)[kThreads / 32];                      // [2][...]
  int group, G;
  int turn = 0;
  __device__ __forceinline__ void barrier() const {
    __syncwarp();
    if (G > 32) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(G) : "memory");
  }
  template <typename F> __device__ __forceinline__ float operator()(float v, F f) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(~0u, v, o));
    if (G > 32) {
      const int first = group * (G / 32);
      if (threadIdx.x % 32 == 0) cell[turn][threadIdx.x / 32] = v;
      barrier();
      if (G == 64) {
        v = f(cell[turn][first], cell[turn][first + 1]);
      } else {
        v = cell[turn][first + min((int)threadIdx.x % 8, G / 32 - 1)];
        if constexpr (std::is_same_v<F, Plus>) v = (int)threadIdx.x % 8 < G / 32 ? v : 0.f;
#pragma unroll
        for (int o = 4; o; o >>= 1) v = f(v, __shfl_xor_sync(~0u, v, o));
      }
      turn ^= 1;
    }
    return v;
  }
};
struct NormArgs {
  const void *x, *residual, *weight;
  long long x_stride, r_stride, t_stride, y_stride;
  long long T;
  int D, G, stages, weight_type, y_type, groups;   // G: threads of a row; groups: scales of a row (0: y is not in 8 bits)
  float eps;
  void *total, *y;
  float *y_scale, *rstd;
  int* status;
};

// 2 ulp from the approximate root, 1 from the reciprocal of D
__device__ __forceinline__ float rms_scale(float sum, float inv_d, float eps) { return rsqrtf(fmaf(sum, inv_d, eps)); }
__device__ __forceinline__ float scale_8(float most) { return fmaxf(most * (1.f / kMost8), kLeastScale); }

// Bound by memory: x and residual read, total and y written once.  Rows wait in shared memory rather than in registers (with the next row in
// registers, two blocks of 128 registers an SM: 135 us), P = 2 leaves three blocks an SM; the 8-bit output costs 28 instructions an element and
// seven rounds of rows at 4099.  Measured: 65536 x 1024 bf16 with fp32 sums 128 us (6.3 TB/s, 96 % of the copy rate); 4099 x 3200 in
// 8 bits 19.3 us (4.8 TB/s); one row of 2048 5.3 us alone with cold caches.
template <typename X, typename S, int P, bool WIDE>
__global__ void __launch_bounds__(kThreads, P == 4 || !WIDE ? 2 : 3) k_norm(const NormArgs a) {
  extern __shared__ __align__(128) unsigned char memory[];
  __shared__ float cell[2][kThreads / 32];
  __shared__ unsigned long long bars[kThreads / 32][kMostStages];
  __shared__ int shared_stop;
  __shared__ unsigned most[WIDE ? 1 : kThreads * P * 8 / 128 + kThreads / 32];   // a group's largest magnitudes: column order is not the threads'
  const int group = threadIdx.x / a.G;
  const Row<P, WIDE> r{a.G, (int)threadIdx.x % a.G};
  Join join{cell, group, a.G};
  const int D = a.D;
  const float inv_d = 1.f / D;
  const unsigned x_bytes = D * (unsigned)sizeof(X), s_bytes = a.residual ? D * (unsigned)sizeof(S) : 0;
  Ring ring = ring_of(memory, bars, &shared_stop, group, x_bytes + s_bytes, a.stages);
  if (WIDE) ring_start(bars, &shared_stop);
  wait_for_previous();
  may_follow();
  const int rows = blockDim.x / a.G;
  const long long step = (long long)gridDim.x * rows;
  long long row = (long long)blockIdx.x * rows + group;
  const X* const x = static_cast<const X*>(a.x);
  const S* const u = static_cast<const S*>(a.residual);
  const auto fetch = [&](long long t, unsigned stage, unsigned bar) {
    bar_expect(bar, x_bytes + s_bytes);
    bulk_load(stage, x + t * a.x_stride, x_bytes, bar);
    if (u) bulk_load(stage + x_bytes, u + t * a.r_stride, s_bytes, bar);
  };
  if (WIDE && r.t == 0)
    for (; ring.issued < ring.stages && row + ring.issued * step < a.T; ++ring.issued)
      fetch(row + ring.issued * step, ring.base + ring.issued * ring.bytes, ring.bar + ring.issued * 8);
  float w[P][8];
  fetch_weight(r, a.weight, a.weight_type, D, w);
  Ahead<X, P, WIDE> ahead_x;
  Ahead<S, P, WIDE> ahead_u;
  const auto fetch_ahead = [&](long long t) {
    if (WIDE || t >= a.T) return;
    ahead_x.fetch(r, x + t * a.x_stride, D);
    if (u) ahead_u.fetch(r, u + t * a.r_stride, D);
  };
  fetch_ahead(row);
  for (; row < a.T; row += step) {
    if (WIDE) ring.wait();
    const unsigned stage = ring.stage();
    S* const total = static_cast<S*>(a.total) + row * a.t_stride;
    float v[P][8], sum = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if constexpr (WIDE) {
        const int c = r.column(p, 0);
        const unsigned at = stage + c * (unsigned)sizeof(X);
        if (c >= D) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[p][i] = 0.f;
        } else if (u) {
          const Raw8<S> both = sum8(staged8<X>(at), staged8<S>(stage + x_bytes + c * (unsigned)sizeof(S)));
          if (ring.ok) store_raw(total + c, both);
          widen(both, v[p]);
        } else {
          widen(staged8<X>(at), v[p]);
        }
      } else {
        ahead_x.get(p, v[p]);
        if (u) {
          float q[8];
          ahead_u.get(p, q);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[p][i] = to_f32(from_f32<S>(v[p][i] + q[i]));
          put<S>(r, total, D, p, v[p]);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[p][i], v[p][i], sum);
    }
    fetch_ahead(row + step);
    const float rstd = rms_scale(join(sum, Plus()), inv_d, a.eps);
    if (WIDE) {                                                     // all of the group have read the stage
      __syncwarp();
      if (r.t == 0 && ring.ok && row + a.stages * step < a.T) {
        fetch(row + a.stages * step, stage, ring.barrier());
        ++ring.issued;
      }
      ++ring.turn;
    }
    if (!ring.ok) {
      if (a.groups == 1) join(0.f, Most());                         // the group's barrier
      continue;
    }
    if (a.rstd && r.t == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[p][i] = v[p][i] * rstd * w[p][i];
    if (a.groups == 0) {
#pragma unroll
      for (int p = 0; p < P; ++p) put_type(r, a.y, a.y_type, row * a.y_stride, D, p, v[p]);
      continue;
    }
    unsigned char* y = static_cast<unsigned char*>(a.y) + row * a.y_stride;
    float top = 0.f;
    if (a.groups == 1) {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[p][i]));
      top = scale_8(join(top, Most()));
      if (r.t == 0) a.y_scale[row] = top;
    }
    if constexpr (WIDE) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = r.column(p, 0);
        float scale = top;
        if (a.groups > 1) {                                         // sixteen neighbours hold 128 columns
          scale = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) scale = fmaxf(scale, fabsf(v[p][i]));
#pragma unroll
          for (int o = 8; o; o >>= 1) scale = fmaxf(scale, __shfl_xor_sync(~0u, scale, o));
          scale = scale_8(scale);
          if (r.t % 16 == 0 && c < D) a.y_scale[row * a.groups + c / 128] = scale;
        }
        const Divide by(scale);
        if (c < D) {
          const unsigned lo = by.codes(v[p][0], v[p][1]) | by.codes(v[p][2], v[p][3]) << 16;
          const unsigned hi = by.codes(v[p][4], v[p][5]) | by.codes(v[p][6], v[p][7]) << 16;
          *reinterpret_cast<uint2*>(y + c) = make_uint2(lo, hi);
        }
      }
    } else {
      unsigned* mine = most + group * ((kThreads * P * 8 / 128) / rows + 1);
      if (a.groups > 1) {                                           // as whole numbers: the order of the updates changes nothing
        for (int i = r.t; i < a.groups; i += a.G) mine[i] = 0;
        join.barrier();
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (r.column(p, i) < D && !isnan(v[p][i])) atomicMax(&mine[r.column(p, i) / 128], __float_as_uint(fabsf(v[p][i])));
        join.barrier();
        for (int i = r.t; i < a.groups; i += a.G) a.y_scale[row * a.groups + i] = scale_8(__uint_as_float(mine[i]));
      }
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = r.column(p, i);
          if (c < D) y[c] = (unsigned char)narrow_e4m3(Divide(a.groups > 1 ? scale_8(__uint_as_float(mine[c / 128])) : top)(v[p][i]), 0.f);
        }
      if (a.groups > 1) join.barrier();                             // before the next row's maxima
    }
  }
  if (WIDE) ring_end(ring, r.t == 0, a.status);
}

// Rows too long for registers: read again after their sum is known; one block a row.
template <typename X, typename S> __global__ void __launch_bounds__(kThreads) k_norm_long(const NormArgs a) {
  wait_for_previous();
  may_follow();
  __shared__ float cell[2][kThreads / 32];
  Join join{cell, 0, kThreads};
  const int D = a.D;                                 // columns are counted from the row's end, -D to -1: D may be 2^31 - 1, and a step beyond it no int
  for (long long row = blockIdx.x; row < a.T; row += gridDim.x) {
    const X* x = static_cast<const X*>(a.x) + row * a.x_stride + D;
    const S* r = static_cast<const S*>(a.residual) + row * a.r_stride + D;
    S* total = static_cast<S*>(a.total) + row * a.t_stride + D;
    const auto value = [&](int c) { return a.residual ? to_f32(total[c]) : to_f32(x[c]); };
    float sum = 0.f;
    for (int c = (int)threadIdx.x - D; c < 0; c += kThreads) {
      if (a.residual) total[c] = from_f32<S>(to_f32(x[c]) + to_f32(r[c]));
      sum = fmaf(value(c), value(c), sum);
    }
    const float rstd = rms_scale(join(sum, Plus()), 1.f / a.D, a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    const auto result = [&](int c) { return value(c) * rstd * load_as(a.weight, a.weight_type, (long long)D + c); };
    if (a.groups == 0) {
      for (int c = (int)threadIdx.x - D; c < 0; c += kThreads) store_as(a.y, a.y_type, row * a.y_stride + D + c, result(c));
      continue;
    }
    const auto finish = [&](int from, int to, float scale, int at, int pace) {
      const Divide by(scale);
      for (int c = from + at; c < to; c += pace) store_as(a.y, COCODC_E4M3, row * a.y_stride + D + c, by(result(c)));
    };
    if (a.groups == 1) {
      float m = 0.f;
      for (int c = (int)threadIdx.x - D; c < 0; c += kThreads) m = fmaxf(m, fabsf(result(c)));
      const float scale = scale_8(join(m, Most()));
      if (threadIdx.x == 0) a.y_scale[row] = scale;
      finish(-D, 0, scale, threadIdx.x, kThreads);
      continue;
    }
    // a warp takes a group at a time; the columns of its lanes are not those that they summed
    __syncthreads();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (int g = warp; g < a.groups; g += kThreads / 32) {
      const int from = g * 128 - D, to = min(0, from + 128);
      float m = 0.f;
      for (int c = from + lane; c < to; c += 32) m = fmaxf(m, fabsf(result(c)));
#pragma unroll
      for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
      const float scale = scale_8(m);
      if (lane == 0) a.y_scale[row * a.groups + g] = scale;
      finish(from, to, scale, lane, 32);
    }
  }
}

struct NormGradArgs {
  const void *dy, *total, *weight, *dtotal;
  long long dy_stride, t_stride, dt_stride, dx_stride;
  long long T;
  int D, G, stages, weight_type;
  const float* rstd;
  void* dx;
  float* parts;             // [blocks][D]: the blocks' sums of dweight, or NULL
  int* status;
};

// Bound by memory; a thread keeps its columns' sums of dweight in registers over all of its rows.  65536 x 1024 bf16 with dtotal: 92 us with
// k_norm_weight (5.9 TB/s, 90 % of the copy rate), 99 us with the rows in registers.
template <typename Y, typename S, int P, bool WIDE>
__global__ void __launch_bounds__(kThreads, P == 4 ? 1 : 2) k_norm_grad(const NormGradArgs a) {
  extern __shared__ __align__(128) unsigned char memory[];
  __shared__ float cell[2][kThreads / 32];
  __shared__ unsigned long long bars[kThreads / 32][kMostStages];
  __shared__ int shared_stop;
  const int group = threadIdx.x / a.G, rows = blockDim.x / a.G;
  const Row<P, WIDE> r{a.G, (int)threadIdx.x % a.G};
  Join join{cell, group, a.G};
  const int D = a.D;
  const float inv_d = 1.f / D;
  const unsigned y_bytes = D * (unsigned)sizeof(Y), s_bytes = D * (unsigned)sizeof(S), all = y_bytes + s_bytes * (a.dtotal ? 2 : 1);
  Ring ring = ring_of(memory, bars, &shared_stop, group, all, a.stages);
  if (WIDE) ring_start(bars, &shared_stop);
  wait_for_previous();
  may_follow();
  const long long step = (long long)gridDim.x * rows;
  long long row = (long long)blockIdx.x * rows + group;
  const Y* const dy = static_cast<const Y*>(a.dy);
  const S *const s = static_cast<const S*>(a.total), *const dt = static_cast<const S*>(a.dtotal);
  const auto fetch = [&](long long t, unsigned stage, unsigned bar) {
    bar_expect(bar, all);
    bulk_load(stage, dy + t * a.dy_stride, y_bytes, bar);
    bulk_load(stage + y_bytes, s + t * a.t_stride, s_bytes, bar);
    if (dt) bulk_load(stage + y_bytes + s_bytes, dt + t * a.dt_stride, s_bytes, bar);
  };
  if (WIDE && r.t == 0)
    for (; ring.issued < ring.stages && row + ring.issued * step < a.T; ++ring.issued)
      fetch(row + ring.issued * step, ring.base + ring.issued * ring.bytes, ring.bar + ring.issued * 8);
  float w[P][8], dw[P][8] = {};
  fetch_weight(r, a.weight, a.weight_type, D, w);
  float next = row < a.T ? a.rstd[row] : 0.f;
  Ahead<Y, P, WIDE> ahead_y;
  Ahead<S, P, WIDE> ahead_s, ahead_t;
  const auto fetch_ahead = [&](long long t) {
    if (WIDE || t >= a.T) return;
    ahead_y.fetch(r, dy + t * a.dy_stride, D);
    ahead_s.fetch(r, s + t * a.t_stride, D);
    if (dt) ahead_t.fetch(r, dt + t * a.dt_stride, D);
  };
  fetch_ahead(row);
  for (; row < a.T; row += step) {
    const float k = next;
    if (row + step < a.T) next = a.rstd[row + step];
    if (WIDE) ring.wait();
    const unsigned stage = ring.stage();
    float g[P][8], h[P][8], sum = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if constexpr (WIDE) {
        get<Y>(r, stage, D, p, g[p]);
        get<S>(r, stage + y_bytes, D, p, h[p]);
      } else {
        ahead_y.get(p, g[p]);
        ahead_s.get(p, h[p]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[p][i] *= k;
        dw[p][i] = fmaf(g[p][i], h[p][i], dw[p][i]);
        g[p][i] *= w[p][i];
        sum = fmaf(g[p][i], h[p][i], sum);
      }
    }
    const float mean = join(sum, Plus()) * inv_d;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      float q[8] = {};
      if (dt) {
        if constexpr (WIDE) get<S>(r, stage + y_bytes + s_bytes, D, p, q);
        else ahead_t.get(p, q);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) g[p][i] = fmaf(k, fmaf(-h[p][i], mean, g[p][i]), q[i]);
      if (p == P - 1) fetch_ahead(row + step);
      if (a.dx && ring.ok) put<S>(r, static_cast<S*>(a.dx) + row * a.dx_stride, D, p, g[p]);
    }
    if (WIDE) {
      join.barrier();                                               // all of the group have read the stage
      if (r.t == 0 && ring.ok && row + a.stages * step < a.T) {
        fetch(row + a.stages * step, stage, ring.barrier());
        ++ring.issued;
      }
      ++ring.turn;
    }
  }
  if (WIDE) ring_end(ring, r.t == 0, a.status);
  float* const shared_parts = reinterpret_cast<float*>(memory);      // [rows of the block][D] where it has more than one
  if (!a.parts) return;
  float* out = a.parts + (long long)blockIdx.x * D;
  float* mine = rows == 1 ? out : shared_parts + group * D;
  if (rows > 1) __syncthreads();                                     // the stages have been read
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (r.column(p, i) < D) mine[r.column(p, i)] = dw[p][i];
  if (rows == 1) return;
  __syncthreads();
  for (int c = threadIdx.x; c < D; c += blockDim.x) {
    float sum = 0.f;
    for (int i = 0; i < rows; ++i) sum += shared_parts[i * D + c];
    out[c] = sum;
  }
}

// Rows too long for registers; the block's sums of dweight stay in memory.
template <typename Y, typename S> __global__ void __launch_bounds__(kThreads) k_norm_grad_long(const NormGradArgs a) {
  wait_for_previous();
  may_follow();
  __shared__ float cell[2][kThreads / 32];
  Join join{cell, 0, kThreads};
  const int D = a.D;                                 // columns from the row's end, as in k_norm_long
  float* part = a.parts ? a.parts + ((long long)blockIdx.x + 1) * D : nullptr;
  if (part)
    for (int c = (int)threadIdx.x - D; c < 0; c += kThreads) part[c] = 0.f;
  for (long long row = blockIdx.x; row < a.T; row += gridDim.x) {
    const Y* dy = static_cast<const Y*>(a.dy) + row * a.dy_stride + D;
    const S* s = static_cast<const S*>(a.total) + row * a.t_stride + D;
    const S* dt = static_cast<const S*>(a.dtotal) + row * a.dt_stride + D;
    S* dx = static_cast<S*>(a.dx) + row * a.dx_stride + D;
    const float k = a.rstd[row];
    float sum = 0.f;
    for (int c = (int)threadIdx.x - D; c < 0; c += kThreads) {
      const float g = to_f32(dy[c]), h = to_f32(s[c]) * k;
      if (part) part[c] = fmaf(g, h, part[c]);
      sum = fmaf(g * load_as(a.weight, a.weight_type, (long long)D + c), h, sum);
    }
    const float mean = join(sum, Plus()) / a.D;
    if (a.dx)
      for (int c = (int)threadIdx.x - D; c < 0; c += kThreads) {
        const float g = to_f32(dy[c]) * load_as(a.weight, a.weight_type, (long long)D + c), h = to_f32(s[c]) * k;
        dx[c] = from_f32<S>(fmaf(k, fmaf(-h, mean, g), a.dtotal ? to_f32(dt[c]) : 0.f));
      }
  }
}

// The blocks' sums of dweight added in order: a block takes 32 columns, each of its 32 warps every 32nd part.
__global__ void __launch_bounds__(1024) k_norm_weight(const float* parts, int count, int D, void* out, int type, int accumulate) {
  wait_for_previous();
  may_follow();
  __shared__ float cell[32][33];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const long long c = (long long)blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (c < D) {
#pragma unroll 8
    for (int i = warp; i < count; i += 32) sum += parts[(long long)i * D + c];
  }
  cell[warp][lane] = sum;
  __syncthreads();
  if (warp || c >= D) return;
  sum = accumulate ? load_as(out, type, c) : 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) sum += cell[i][lane];
  store_as(out, type, c, sum);
}

// Columns that 256 threads hold: 32 each in packs, 8 one by one (more take more registers than there are)
int64_t longest(bool wide) { return wide ? 8192 : 2048; }
constexpr int kGradBlocks = 592;                    // at most, four for each SM of a B200 (the workspace's size is asked for without a handle)

// Calls f with the element types (x and the sum) that two type codes stand for.
template <typename F> cocodc_status with_types(int32_t x, int32_t s, F&& f) {
  if (x == COCODC_F32) return f(float(), float());
  if (x == COCODC_BF16) return s == COCODC_F32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
  return s == COCODC_F32 ? f(__half(), float()) : f(__half(), __half());
}
constexpr unsigned kSharedOfSm = 227 * 1024, kMostShared = kSharedOfSm - 4096;      // of an SM; of a block, beside what the kernels declare
template <int N> using Int = std::integral_constant<int, N>;

unsigned grid_for(const cocodc_lm* lm, int64_t T, int rows, int per_sm) {
  const int64_t blocks = (T + rows - 1) / rows, most = (int64_t)lm->sm_count * per_sm;
  return (unsigned)(blocks < most ? blocks : most);
}
// Blocks of a kernel that an SM holds, by registers and shared memory.  A kernel's registers are asked for once.
int per_sm(std::atomic<int>& known, const void* kernel, int threads, unsigned shared) {
  int regs = known.load(std::memory_order_relaxed);
  if (regs == 0) {
    cudaFuncAttributes f;
    if (cudaFuncGetAttributes(&f, kernel) != cudaSuccess) {
      cudaGetLastError();
      return 1;
    }
    regs = (f.numRegs + 7) / 8 * 8;
    known.store(regs, std::memory_order_relaxed);
  }
  const int by_regs = 65536 / (regs * threads), by_memory = (int)(kSharedOfSm / (shared + 2048)), most = 2048 / threads;
  const int blocks = by_regs < by_memory ? by_regs : by_memory;
  return blocks < 1 ? 1 : blocks < most ? blocks : most;
}

// Calls f(packs of a thread, whether wide, threads of a row, rows of a block).  Two packs a thread leave registers for two blocks and more on an SM;
// one where rows are few and their latency is what counts.
template <typename F> cocodc_status with_shape(const cocodc_lm* lm, int64_t T, int64_t D, bool wide, F&& f) {
  const auto go = [&](auto p) {
    constexpr int P = decltype(p)::value;
    const int G = (int)((D + 8 * P * 32 - 1) / (8 * P * 32)) * 32, rows = G >= kThreads ? 1 : kThreads / G;
    if constexpr (P == 1)
      if (!wide) return f(p, std::false_type(), G, rows);
    return f(p, std::true_type(), G, rows);
  };
  if (!wide || D <= 256 || (T <= 2 * lm->sm_count && D <= 2048)) return go(Int<1>());
  return D <= 4096 ? go(Int<2>()) : go(Int<4>());
}
// Stages of a group's ring: what the loads of an SM need to be on their way at a time, but no more than there are rows.
int stages_for(unsigned bytes, int rows, int blocks_by_regs, int64_t T, unsigned grid_rows) {
  const unsigned part = kSharedOfSm / blocks_by_regs - 2048, share = part < kMostShared ? part : kMostShared;
  int n = (int)(share / (bytes * rows));
  n = n > kMostStages ? kMostStages : n < 2 ? 2 : n;
  const int64_t each = (T + grid_rows - 1) / grid_rows;
  return each < n ? (int)(each < 1 ? 1 : each) : n;
}

// Starts a kernel that walks over rows with a ring of `bytes` a row (0: none).
template <typename K, typename A>
cocodc_status start_rows(cocodc_lm* lm, std::atomic<int>& regs, K kernel, A& a, int G, int rows, unsigned bytes, unsigned more, bool waves, int most_blocks, unsigned* blocks,
                         cudaStream_t st) {
  const int by_regs = per_sm(regs, reinterpret_cast<const void*>(kernel), G * rows, more);
  a.G = G;
  a.stages = bytes ? stages_for(bytes, rows, by_regs, a.T, (unsigned)rows * by_regs * lm->sm_count) : 1;
  unsigned shared = bytes * rows * a.stages;
  if (shared < more) shared = more;
  int resident = per_sm(regs, reinterpret_cast<const void*>(kernel), G * rows, shared);
  // up to four times as many blocks as are resident, as long as each keeps eight rounds of rows: those of an SM that is ahead do not wait for the others'
  // last rows (65536 x 1024: 134 -> 127 us; at 4099 x 3200, ten rounds of resident blocks, four times as many cost 23.4 -> 27.6 us)
  const int64_t rounds = a.T / ((int64_t)rows * resident * lm->sm_count), times = rounds / 8;
  if (waves) resident *= (int)(times < 1 ? 1 : times > 4 ? 4 : times);
  *blocks = grid_for(lm, a.T, rows, resident);
  if (*blocks > (unsigned)most_blocks) *blocks = (unsigned)most_blocks;
  return start(lm, kernel, *blocks, G * rows, shared, st, 1, a);
}

}  // namespace

namespace cocodc_lm_impl {
bool norm_prepare() {
  bool ok = true;
  const auto allow = [&](auto kernel) {
    ok = ok && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared) == cudaSuccess;
  };
  for (int32_t x : {COCODC_F32, COCODC_BF16, COCODC_F16})
    for (int32_t s : {x, (int32_t)COCODC_F32})
      with_types(x, s, [&](auto xt, auto st) {
        using X = decltype(xt);
        using S = decltype(st);
        allow(k_norm<X, S, 1, true>);
        allow(k_norm<X, S, 2, true>);
        allow(k_norm<X, S, 4, true>);
        allow(k_norm_grad<X, S, 1, true>);
        allow(k_norm_grad<X, S, 2, true>);
        allow(k_norm_grad<X, S, 4, true>);
        return COCODC_OK;
      });
  return ok;
}
}  // namespace cocodc_lm_impl

extern "C" {

cocodc_status cocodc_lm_norm(cocodc_lm* lm, const void* x, int32_t x_type, int64_t x_stride, const void* residual,
                             int64_t residual_stride, int32_t sum_type, const void* weight, int32_t weight_type, int64_t T,
                             int64_t D, float eps, void* total, int64_t total_stride, void* y, int32_t y_type, int64_t y_stride,
                             float* y_scale, int64_t scale_group, float* rstd, void* stream) {
  const bool eight = y_type == COCODC_E4M3, sum = residual || total;
  if (!lm || !known_type(x_type) || !known_type(weight_type) || !(known_type(y_type) || eight) || !sane(T) || D < 1 || D > INT32_MAX ||
      !(eps >= 0.f && eps <= 3.4e38f) || x_stride < D || !sane(x_stride) || y_stride < D || !sane(y_stride) ||
      (eight ? (scale_group != 0 && scale_group != 128) : scale_group != 0))
    return COCODC_ERR_INVALID_ARG;
  if (sum && ((sum_type != x_type && sum_type != COCODC_F32) || residual_stride < D || !sane(residual_stride) || total_stride < D ||
              !sane(total_stride)))
    return COCODC_ERR_INVALID_ARG;
  if (T == 0) return COCODC_OK;
  if (!x || !weight || !y || !residual != !total || !eight != !y_scale) return COCODC_ERR_INVALID_ARG;
  const int xb = type_bytes(x_type), sb = sum ? type_bytes(sum_type) : xb, yb = eight ? 1 : type_bytes(y_type), wb = type_bytes(weight_type);
  if (!on_boundary(x, xb) || !on_boundary(residual, sb) || !on_boundary(total, sb) || !on_boundary(y, yb) || !on_boundary(weight, wb) ||
      !on_boundary(y_scale, 4) || !on_boundary(rstd, 4))
    return COCODC_ERR_ALIGNMENT;
  const int64_t groups = eight ? (scale_group ? (D + 127) / 128 : 1) : 0;
  const Span in[3] = {span(x, T, x_stride, D, xb), span(residual, T, residual_stride, D, sb), span(weight, 1, D, D, wb)};
  const Span out[4] = {span(total, T, total_stride, D, sb), span(y, T, y_stride, D, yb), span(y_scale, T, groups, groups, 4), span(rstd, 1, T, T, 4)};
  const bool in_place = residual && total == residual && total_stride == residual_stride;
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 3; ++j)
      if (!(in_place && i == 0 && j == 1) && meet(out[i], in[j])) return COCODC_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return COCODC_ERR_ALIAS;
  }
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  NormArgs a{x, residual, weight, x_stride, residual_stride, total_stride, y_stride, T, (int)D, 0, 0, weight_type, y_type, (int)groups, eps,
                   total, y, y_scale, rstd, lm->d_status};
  const bool wide = D % 8 == 0 && rows_aligned(x, x_stride, xb) && (!sum || (rows_aligned(residual, residual_stride, sb) && rows_aligned(total, total_stride, sb))) &&
                    (eight ? on_boundary(y, 8) && y_stride % 8 == 0 : rows_aligned(y, y_stride, yb));
  return with_types(x_type, sum ? sum_type : x_type, [&](auto xt, auto s) {
    using X = decltype(xt);
    using S = decltype(s);
    if (D > longest(wide)) return start(lm, k_norm_long<X, S>, grid_for(lm, T, 1, 8), kThreads, 0, st, 1, a);
    return with_shape(lm, T, D, wide, [&](auto p, auto w, int G, int rows) {
      static std::atomic<int> regs{0};
      unsigned blocks;
      return start_rows(lm, regs, k_norm<X, S, decltype(p)::value, decltype(w)::value>, a, G, rows,
                        decltype(w)::value ? (unsigned)D * (unsigned)(sizeof(X) + (sum ? sizeof(S) : 0)) : 0, 0, true, INT32_MAX, &blocks, st);
    });
  });
}

uint64_t cocodc_lm_norm_grad_workspace(int64_t T, int64_t D) {
  if (!sane(T) || D < 1 || D > INT32_MAX) return 0;
  return 16 + (uint64_t)(T < kGradBlocks ? T : kGradBlocks) * (uint64_t)D * sizeof(float);
}

cocodc_status cocodc_lm_norm_grad(cocodc_lm* lm, const void* dy, int32_t dy_type, int64_t dy_stride, const void* total,
                                  int32_t total_type, int64_t total_stride, const void* weight, int32_t weight_type,
                                  const float* rstd, int64_t T, int64_t D, const void* dtotal, int64_t dtotal_stride, void* dx,
                                  int64_t dx_stride, void* dweight, int32_t dweight_type, int32_t accumulate, void* workspace,
                                  uint64_t workspace_bytes, void* stream) {
  if (!lm || !known_type(dy_type) || (total_type != dy_type && total_type != COCODC_F32) || !known_type(weight_type) || !sane(T) || D < 1 ||
      D > INT32_MAX || dy_stride < D || !sane(dy_stride) || total_stride < D || !sane(total_stride) ||
      (dtotal && (dtotal_stride < D || !sane(dtotal_stride))) || (dx && (dx_stride < D || !sane(dx_stride))) ||
      (dweight && !known_type(dweight_type)))
    return COCODC_ERR_INVALID_ARG;
  if (!dx && !dweight) return T == 0 ? COCODC_OK : COCODC_ERR_INVALID_ARG;
  if (T > 0 && (!dy || !total || !weight || !rstd)) return COCODC_ERR_INVALID_ARG;
  if (dweight && (!workspace || workspace_bytes < cocodc_lm_norm_grad_workspace(T, D))) return COCODC_ERR_INVALID_ARG;
  const int yb = type_bytes(dy_type), sb = type_bytes(total_type), wb = type_bytes(weight_type), db = dweight ? type_bytes(dweight_type) : 4;
  if (!on_boundary(dy, yb) || !on_boundary(total, sb) || !on_boundary(dtotal, sb) || !on_boundary(dx, sb) || !on_boundary(weight, wb) ||
      !on_boundary(dweight, db) || !on_boundary(rstd, 4) || (dweight && !on_boundary(workspace, 16)))
    return COCODC_ERR_ALIGNMENT;
  const Span in[5] = {span(dy, T, dy_stride, D, yb), span(total, T, total_stride, D, sb), span(weight, 1, D, D, wb), span(rstd, 1, T, T, 4),
                      span(dtotal, T, dtotal_stride, D, sb)};
  const Span out[3] = {span(dx, T, dx_stride, D, sb), span(dweight, 1, D, D, db),
                       dweight ? span(workspace, 1, (int64_t)workspace_bytes, (int64_t)workspace_bytes, 1) : Span{0, 0, 0, 0}};
  const bool in_place = dx && dx == dtotal && dx_stride == dtotal_stride;
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 5; ++j)
      if (!(in_place && i == 0 && j == 4) && meet(out[i], in[j])) return COCODC_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return COCODC_ERR_ALIAS;
  }
  if (T == 0 && (!dweight || accumulate)) return COCODC_OK;
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  NormGradArgs a{dy, total, weight, dtotal, dy_stride, total_stride, dtotal_stride, dx_stride, T, (int)D, 0, 0, weight_type, rstd, dx,
                       dweight ? static_cast<float*>(workspace) : nullptr, lm->d_status};
  const bool wide = D % 8 == 0 && rows_aligned(dy, dy_stride, yb) && rows_aligned(total, total_stride, sb) && (!dtotal || rows_aligned(dtotal, dtotal_stride, sb)) &&
                    (!dx || rows_aligned(dx, dx_stride, sb));
  unsigned blocks = 0;
  cocodc_status status = COCODC_OK;
  if (T > 0) {
    status = with_types(dy_type, total_type, [&](auto yt, auto s) {
      using Y = decltype(yt);
      using S = decltype(s);
      if (D > longest(wide)) {
        blocks = grid_for(lm, T, 1, 4);
        if (blocks > kGradBlocks) blocks = kGradBlocks;
        return start(lm, k_norm_grad_long<Y, S>, blocks, kThreads, 0, st, 1, a);
      }
      return with_shape(lm, T, D, wide, [&](auto p, auto w, int G, int rows) {
        static std::atomic<int> regs{0};
        return start_rows(lm, regs, k_norm_grad<Y, S, decltype(p)::value, decltype(w)::value>, a, G, rows,
                          decltype(w)::value ? (unsigned)D * (unsigned)(sizeof(Y) + sizeof(S) * (dtotal ? 2 : 1)) : 0,
                          dweight && rows > 1 ? rows * (unsigned)D * 4 : 0, false, kGradBlocks, &blocks, st);
      });
    });
  }
  if (status != COCODC_OK || !dweight) return status;
  return start(lm, k_norm_weight, (unsigned)((D + 31) / 32), 1024, 0, st, 1, static_cast<const float*>(workspace), (int)blocks, (int)D, dweight,
               dweight_type, accumulate ? 1 : 0);
}

}  // extern "C"
