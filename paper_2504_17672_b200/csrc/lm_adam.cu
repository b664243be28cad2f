// The AdamW step over many tensors (include/cocodc_lm.h).

#include "lm_common.cuh"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

using namespace cocodc_lm_impl;

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kUnit = COCODC_LM_ADAM_BLOCK;          // elements that a warp takes at a time and that share a scale: 8 for each lane
constexpr float kMost8 = 448.f, kLeastScale = 1e-30f;
__device__ __forceinline__ float scale_8(unsigned most) { return fmaxf(__fmul_rn(__uint_as_float(most), 1.f / kMost8), kLeastScale); }

struct Tensor {                                      // as the kernel reads it
  float* p;
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  void* copy;
  long long n;
  int grad_type, copy_type;
  float decay;
  int position;                                      // in the plan
  int wide;                                          // every array starts where vector accesses may
  long long first;                                   // number of its first unit among all tensors' units
};

}  // namespace

struct cocodc_lm_adam {
  int device = 0, bits = 32;
  long long units = 0;
  int count = 0;
  Tensor* d_tensors = nullptr;
};

namespace {

struct AdamArgs {
  const Tensor* tensors;                             // those with elements; `position` of each is its place in the plan
  int count;
  long long units;
  float b1, c1, b2, c2, eps;                         // c = 1 - b
  float k1, k2;                                      // where the step and the rate are known on the host
  double lr, beta1, beta2;
  long long step;
  const long long* step_at;
  const float *grad_scale, *lr_scale;
  unsigned seed;
  int* status;
};

// One round of multiplications and shifts that spreads every bit over the word (the 32-bit finaliser with Appleby's constants).
__host__ __device__ __forceinline__ unsigned mix(unsigned x) {
  x = (x ^ x >> 16) * 0x85EBCA6Bu;
  x = (x ^ x >> 13) * 0xC2B2AE35u;
  return x ^ x >> 16;
}
constexpr unsigned kGolden = 0x9E3779B9u;

// ---- pairs of fp32 numbers: one instruction for two, each rounded on its own --------------------------
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float lo, float hi) {
  f32x2 v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
  return v;
}
__device__ __forceinline__ float2 halves(f32x2 v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 v;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ f32x2 mul2_cut(f32x2 a, f32x2 b) {
  f32x2 v;
  asm("mul.rz.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ f32x2 both(float x) { return pair_of(x, x); }
// one by one: the two instructions of a packed product and sum come out of the assembler as one, which rounds once
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  const float2 x = halves(a), y = halves(b);
  return pair_of(__fadd_rn(x.x, y.x), __fadd_rn(x.y, y.y));
}

// A number times 2^-120 (a unit's largest magnitude was brought to 448 before) to an e4m3 code in the highest byte, without its sign: up with
// probability (what is cut off) / (spacing).  There the exponents of e4m3 are those of fp32, below its smallest normal number too (2^-126
// here and there), so that the code is what stands above the lowest 20 bits; 16 random bits, here bytes 1 and 2, are added to
// those.  Below that number the product with 2^-120 is cut, not rounded: rounded it could reach the next code without them.  The number may be 448 + 3 ulp: no carry comes of it.
__device__ __forceinline__ unsigned code_of(float x, unsigned random) { return (__float_as_uint(x) << 4) + random; }
__device__ __forceinline__ float2 widen_e4m3(unsigned short v) {
  unsigned h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(v));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ float load_grad(const void* p, int type, long long i) {
  return type == COCODC_F32    ? static_cast<const float*>(p)[i]
         : type == COCODC_BF16 ? to_f32(static_cast<const __nv_bfloat16*>(p)[i])
                               : to_f32(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ unsigned narrow2(int type, float2 v) {
  if (type == COCODC_BF16) {
    const __nv_bfloat162 h = __float22bfloat162_rn(v);
    return *reinterpret_cast<const unsigned*>(&h);
  }
  const __half2 h = __float22half2_rn(v);
  return *reinterpret_cast<const unsigned*>(&h);
}
__device__ __forceinline__ uint2 load8(const void* p) {
  uint2 v;
  asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ unsigned load4(const void* p) {
  unsigned v;
  asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
// the larger magnitude; NaN if one is
__device__ __forceinline__ float larger(float a, float b) {
  float v;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(a), "f"(fabsf(b)));
  return v;
}
__device__ __forceinline__ float inverse(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ unsigned finite_magnitude(float x) {
  const unsigned b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// A lane's eight elements of a unit: 4 l .. 4 l + 3 and 128 + 4 l .. 128 + 4 l + 3, so that neighbours read neighbours in every width.
struct Eight { f32x2 p[4], m[4], v[4], g[4]; };
__device__ __forceinline__ int place(int e, int lane) { return e / 4 * 128 + lane * 4 + e % 4; }

// A unit's numbers on their way.
template <bool EIGHT> struct RawUnit {
  uint4 p[2], g[2];
  uint4 m[EIGHT ? 1 : 2], v[EIGHT ? 1 : 2];          // EIGHT: codes in x and y
  float ms, vs;
};
// A lane's addresses in a unit of the tensor (first: the unit's first element + 4 l).
struct At {
  float* p;
  const char* g;
  char *m, *v, *c;
  float *ms, *vs;
};
constexpr int kAhead = kWarps * kUnit;               // elements from a warp's unit to its next
template <bool EIGHT, int AHEAD> __device__ __forceinline__ void fetch(RawUnit<EIGHT>& r, const At& a, int grad_type) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = AHEAD + h * 128;
    r.p[h] = load16(a.p + i);
    if (grad_type == COCODC_F32) {
      r.g[h] = load16(a.g + i * 4);
    } else {
      const uint2 q = load8(a.g + i * 2);
      r.g[h].x = q.x;
      r.g[h].y = q.y;
    }
    if (EIGHT) {
      (h ? r.m[0].y : r.m[0].x) = load4(a.m + i);
      (h ? r.v[0].y : r.v[0].x) = load4(a.v + i);
    } else {
      r.m[h] = load16(a.m + i * 4);
      r.v[h] = load16(a.v + i * 4);
    }
  }
  if (EIGHT) {
    r.ms = a.ms[AHEAD / kUnit];
    r.vs = a.vs[AHEAD / kUnit];
  }
}
__device__ __forceinline__ void spread4(const uint4& r, f32x2* v) {
  v[0] = pair_of(__uint_as_float(r.x), __uint_as_float(r.y));
  v[1] = pair_of(__uint_as_float(r.z), __uint_as_float(r.w));
}
template <bool EIGHT> __device__ __forceinline__ void spread(const RawUnit<EIGHT>& r, int grad_type, Eight& x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    spread4(r.p[h], x.p + 2 * h);
    if (grad_type == COCODC_F32) {
      spread4(r.g[h], x.g + 2 * h);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const unsigned w = i ? r.g[h].y : r.g[h].x;
        if (grad_type == COCODC_BF16) {
          x.g[2 * h + i] = pair_of(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
        } else {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
          x.g[2 * h + i] = pair_of(f.x, f.y);
        }
      }
    }
    if (EIGHT) {
      const unsigned cm = h ? r.m[0].y : r.m[0].x, cv = h ? r.v[0].y : r.v[0].x;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 fm = widen_e4m3((unsigned short)(cm >> 16 * i)), fv = widen_e4m3((unsigned short)(cv >> 16 * i));
        x.m[2 * h + i] = pair_of(fm.x, fm.y);
        x.v[2 * h + i] = pair_of(fv.x, fv.y);
      }
    } else {
      spread4(r.m[h], x.m + 2 * h);
      spread4(r.v[h], x.v + 2 * h);
    }
  }
}

// The step of a lane's eight elements.  EIGHT: m and v come as codes, which ms and vs scale, and leave as codes of four elements each with new scales.
struct Factors { f32x2 gs, b1, c1, b2, c2, k1, k2, eps, keep; };
template <bool EIGHT>
__device__ __forceinline__ void step_of(Eight& x, const Factors& f, float& ms, float& vs, unsigned key, unsigned (&mc)[2], unsigned (&vc)[2]) {
  f32x2 root[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (EIGHT) {
      x.m[i] = mul2(x.m[i], both(ms));
      x.v[i] = mul2(x.v[i], both(vs));
      x.v[i] = mul2(x.v[i], x.v[i]);
    }
    const f32x2 g = mul2(x.g[i], f.gs);
    x.m[i] = add2(mul2(x.m[i], f.b1), mul2(g, f.c1));
    x.v[i] = add2(mul2(x.v[i], f.b2), mul2(mul2(g, f.c2), g));
    const float2 v = halves(x.v[i]);
    root[i] = pair_of(__fsqrt_rn(v.x), __fsqrt_rn(v.y));
    const float2 d = halves(add2(mul2(root[i], f.k2), f.eps));
    x.p[i] = add2(mul2(x.p[i], f.keep), mul2(mul2(x.m[i], f.k1), pair_of(inverse(d.x), inverse(d.y))));        // k1 is negative
  }
  if constexpr (!EIGHT) return;
  float top_m = 0.f, top_v = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 m = halves(x.m[i]), r = halves(root[i]);
    top_m = larger(larger(top_m, m.x), m.y);
    top_v = larger(larger(top_v, r.x), r.y);
  }
  unsigned most_m = __reduce_max_sync(~0u, __float_as_uint(top_m)), most_v = __reduce_max_sync(~0u, __float_as_uint(top_v));
  const bool odd = max(most_m, most_v) >= 0x7f800000u;               // a number that is not finite, somewhere in the unit
  if (odd) {
    most_m = most_v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 m = halves(x.m[i]), r = halves(root[i]);
      most_m = max(most_m, max(finite_magnitude(m.x), finite_magnitude(m.y)));
      most_v = max(most_v, max(finite_magnitude(r.x), finite_magnitude(r.y)));
    }
    most_m = __reduce_max_sync(~0u, most_m);
    most_v = __reduce_max_sync(~0u, most_v);
  }
  ms = scale_8(most_m);
  vs = scale_8(most_v);
  const f32x2 im = both(__frcp_rn(ms)), iv = both(__frcp_rn(vs)), low = both(0x1p-120f);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    unsigned cm[4], cv[4], sign[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 m = halves(x.m[2 * h + i]), r = halves(root[2 * h + i]);
      const float2 y = halves(mul2_cut(mul2(x.m[2 * h + i], im), low)), z = halves(mul2_cut(mul2(root[2 * h + i], iv), low));
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int n = 2 * i + j;
        const unsigned bits = mix(key + (unsigned)(h * 128 + n) * kGolden);
        cm[n] = code_of(j ? y.y : y.x, __byte_perm(bits, 0, 0x4104));
        // a root above zero (none is below 2^-75) stays above zero
        cv[n] = max(code_of(j ? z.y : z.x, __byte_perm(bits, 0, 0x4324)), min(__float_as_uint(j ? r.y : r.x), 1u << 24));
        sign[n] = __float_as_uint(j ? m.y : m.x);
        if (odd) {
          if (finite_magnitude(j ? m.y : m.x) == 0 && (j ? m.y : m.x) != 0.f) cm[n] = 0x7f000000u;
          if (finite_magnitude(j ? r.y : r.x) == 0 && (j ? r.y : r.x) != 0.f) cv[n] = 0x7f000000u;
        }
      }
    }
    const auto pack = [](const unsigned* c) { return __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410); };
    mc[h] = (pack(cm) & 0x7f7f7f7fu) | (pack(sign) & 0x80808080u);
    vc[h] = pack(cv);
  }
}

constexpr int kSoon = 3;                             // units of a warp

// Read once, written once: bound by memory, with states in 8 bits as much by instructions (68 an element, of them 11 for random bits and 9 for the root).
// The units of all tensors form one row, of which each block takes an equal part and its warps one unit in turn: a warp walks from tensor to
// tensor, and the next unit's numbers are on their way while it works on one.  Measured: 124M elements in 12 blocks of layers, fp32 gradients and
// states, 540 us (6.4 TB/s, 98 % of the copy rate); 187M with 8-bit states, bf16 gradients and copies 584-594 us (5.1 TB/s).  Tried for the 8-bit
// states: rings of asynchronous copies by lanes (718 us) or of bulk copies by warps (614 us, and 580 us for the 32-bit ones); loads with a
// condition for the last, ragged units (660 us).  Where tensors are small the walk shows: a warp's first unit of a tensor waits for its loads
// (6.3M elements with 8-bit states: 25 us in 11 tensors, 42 us in 82, most of them with ragged ends).
template <bool EIGHT> __global__ void __launch_bounds__(kThreads, EIGHT ? 4 : 3) k_adamw(const AdamArgs a) {
  wait_for_previous();
  may_follow();
  __shared__ float factors[2];
  __shared__ double shared_lr;
  if (threadIdx.x == 0) {
    factors[0] = a.k1;
    factors[1] = a.k2;
    shared_lr = a.lr;
    if (a.step_at || a.lr_scale) {
      long long step = a.step_at ? *a.step_at : a.step;
      if (step < 1) {
        record(a.status, COCODC_ERR_INVALID_ARG);
        step = 1;
      }
      if (a.lr_scale) shared_lr = a.lr * (double)*a.lr_scale;
      factors[0] = (float)(shared_lr / (1.0 - pow(a.beta1, (double)step)));
      factors[1] = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)step)));
    }
  }
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const unsigned step_bits = (unsigned)max(a.step_at ? *a.step_at : a.step, 1ll);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const long long last = a.units * (blockIdx.x + 1) / gridDim.x;
  const long long from = a.units * blockIdx.x / gridDim.x;
  long long unit = from + warp;
  // the tensor of the block's first unit: the last one that begins at or before it (all looked at together: a search by halves waits for a load at each)
  int number = -1;
  for (int i = 0; i < a.count; i += kThreads) number += __syncthreads_count(i + (int)threadIdx.x < a.count && a.tensors[i + threadIdx.x].first <= from);
  Factors f;
  f.gs = both(gs);
  f.b1 = both(a.b1);
  f.c1 = both(a.c1);
  f.b2 = both(a.b2);
  f.c2 = both(a.c2);
  f.k1 = both(-factors[0]);
  f.k2 = both(factors[1]);
  f.eps = both(a.eps);
  for (; unit < last; ++number) {
    const Tensor t = a.tensors[number];
    const long long units = (t.n + kUnit - 1) / kUnit, end = min(last, t.first + units) - t.first;
    const long long wide_end = t.wide ? min(end, t.n / kUnit) : 0;     // units before this one are whole and aligned
    long long own = unit - t.first;
    if (own >= end) continue;
    f.keep = both((float)(1.0 - shared_lr * (double)t.decay));
    unsigned seed = mix(a.seed + kGolden) ^ step_bits;
    seed = mix((mix(seed + kGolden) ^ (unsigned)t.position) + kGolden);
    const auto key_of = [&](long long u) { return mix((seed ^ (unsigned)u) + kGolden) + (unsigned)(lane * 4) * kGolden; };
    RawUnit<EIGHT> raw;
    Eight x;
    unsigned mc[2], vc[2];
    float ms = 0.f, vs = 0.f;
    if (own < wide_end) {
      const long long i = own * kUnit + lane * 4;
      const int gb = t.grad_type == COCODC_F32 ? 4 : 2, sb = EIGHT ? 1 : 4;
      At at{t.p + i, static_cast<const char*>(t.grad) + i * gb, static_cast<char*>(t.m) + i * sb, static_cast<char*>(t.v) + i * sb,
            t.copy ? static_cast<char*>(t.copy) + i * 2 : nullptr, EIGHT ? t.m_scale + own : nullptr, EIGHT ? t.v_scale + own : nullptr};
      fetch<EIGHT, 0>(raw, at, t.grad_type);
      // states in 8 bits: 2 KB a unit and warp are too few on their way, and registers for more there are none.  The lines of later units are brought to
      // L2 by a lane each: 8 of the parameters, up to 8 of the gradients, 2 of each state.
      const int line = lane < 8 ? lane : lane < 16 ? lane - 8 : lane < 18 ? lane - 16 : lane - 18;
      const int width = lane < 8 ? 4 : lane < 16 ? gb : sb;
      const char* soon = lane < 8 ? reinterpret_cast<const char*>(t.p) : lane < 16 ? static_cast<const char*>(t.grad) : lane < 18 ? static_cast<const char*>(t.m) : static_cast<const char*>(t.v);
      soon += (own + kSoon * kWarps) * kUnit * width + line * 128;
      const bool helps = EIGHT && lane < 20 && line * 128 < kUnit * width;
      for (; own < wide_end; own += kWarps) {
        if (EIGHT) {
          if (helps && own + kSoon * kWarps < wide_end) asm volatile("prefetch.global.L2 [%0];" ::"l"(soon));
          soon += kAhead * width;
        }
        spread(raw, t.grad_type, x);
        ms = raw.ms;
        vs = raw.vs;
        if (own + kWarps < wide_end) fetch<EIGHT, kAhead>(raw, at, t.grad_type);
        step_of<EIGHT>(x, f, ms, vs, key_of(own), mc, vc);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 p0 = halves(x.p[2 * h]), p1 = halves(x.p[2 * h + 1]);
          *reinterpret_cast<float4*>(at.p + h * 128) = make_float4(p0.x, p0.y, p1.x, p1.y);
          if (EIGHT) {
            *reinterpret_cast<unsigned*>(at.m + h * 128) = mc[h];
            *reinterpret_cast<unsigned*>(at.v + h * 128) = vc[h];
          } else {
            const float2 m0 = halves(x.m[2 * h]), m1 = halves(x.m[2 * h + 1]), v0 = halves(x.v[2 * h]), v1 = halves(x.v[2 * h + 1]);
            *reinterpret_cast<float4*>(at.m + h * 512) = make_float4(m0.x, m0.y, m1.x, m1.y);
            *reinterpret_cast<float4*>(at.v + h * 512) = make_float4(v0.x, v0.y, v1.x, v1.y);
          }
          if (at.c) *reinterpret_cast<uint2*>(at.c + h * 256) = make_uint2(narrow2(t.copy_type, p0), narrow2(t.copy_type, p1));
        }
        if (EIGHT && lane == 0) {
          *at.ms = ms;
          *at.vs = vs;
        }
        at.p += kAhead;
        at.g += kAhead * gb;
        at.m += kAhead * sb;
        at.v += kAhead * sb;
        if (at.c) at.c += kAhead * 2;
        if (EIGHT) {
          at.ms += kWarps;
          at.vs += kWarps;
        }
      }
    }
    // a last unit that is not whole, or a tensor that is not aligned: element by element
    for (; own < end; own += kWarps) {
      const long long base = own * kUnit;
      const int here = (int)min((long long)kUnit, t.n - base);
      float p[8], g[8], m[8], v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int o = place(e, lane);
        p[e] = g[e] = m[e] = v[e] = 0.f;
        if (o >= here) continue;
        p[e] = t.p[base + o];
        g[e] = load_grad(t.grad, t.grad_type, base + o);
        if (EIGHT) {
          m[e] = widen_e4m3(static_cast<const unsigned char*>(t.m)[base + o]).x;
          v[e] = widen_e4m3(static_cast<const unsigned char*>(t.v)[base + o]).x;
        } else {
          m[e] = static_cast<const float*>(t.m)[base + o];
          v[e] = static_cast<const float*>(t.v)[base + o];
        }
      }
      if (EIGHT) {
        ms = t.m_scale[own];
        vs = t.v_scale[own];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x.p[i] = pair_of(p[2 * i], p[2 * i + 1]);
        x.g[i] = pair_of(g[2 * i], g[2 * i + 1]);
        x.m[i] = pair_of(m[2 * i], m[2 * i + 1]);
        x.v[i] = pair_of(v[2 * i], v[2 * i + 1]);
      }
      step_of<EIGHT>(x, f, ms, vs, key_of(own), mc, vc);
      if (EIGHT && lane == 0) {
        t.m_scale[own] = ms;
        t.v_scale[own] = vs;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int o = place(e, lane);
        if (o >= here) continue;
        const float2 pp = halves(x.p[e / 2]), pm = halves(x.m[e / 2]), pv = halves(x.v[e / 2]);
        const float q = e % 2 ? pp.y : pp.x;
        t.p[base + o] = q;
        if (EIGHT) {
          static_cast<unsigned char*>(t.m)[base + o] = (unsigned char)(mc[e / 4] >> e % 4 * 8);
          static_cast<unsigned char*>(t.v)[base + o] = (unsigned char)(vc[e / 4] >> e % 4 * 8);
        } else {
          static_cast<float*>(t.m)[base + o] = e % 2 ? pm.y : pm.x;
          static_cast<float*>(t.v)[base + o] = e % 2 ? pv.y : pv.x;
        }
        if (t.copy) static_cast<unsigned short*>(t.copy)[base + o] = (unsigned short)narrow2(t.copy_type, make_float2(q, 0.f));
      }
    }
    unit = t.first + own;
  }
}

cocodc_status check(const cocodc_lm_tensor* tensors, int64_t count, int32_t bits, std::vector<Tensor>& out, long long* total) {
  struct Array { Span s; bool written; };
  std::vector<Array> arrays;
  const int state = bits == 8 ? 1 : 4;
  for (int64_t i = 0; i < count; ++i) {
    const cocodc_lm_tensor& t = tensors[i];
    if (t.n < 0 || t.n > (int64_t(1) << 38) || !known_type(t.grad_type) || (t.copy && t.copy_type != COCODC_BF16 && t.copy_type != COCODC_F16) ||
        !(t.decay >= 0.f && std::isfinite(t.decay)) || t.reserved != 0)
      return COCODC_ERR_INVALID_ARG;
    const int64_t units = (t.n + kUnit - 1) / kUnit;
    if (t.n > 0 && (!t.p || !t.grad || !t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale)))) return COCODC_ERR_INVALID_ARG;
    if (bits != 8 && (t.m_scale || t.v_scale)) return COCODC_ERR_INVALID_ARG;
    const int gb = type_bytes(t.grad_type);
    if (!on_boundary(t.p, 4) || !on_boundary(t.grad, gb) || !on_boundary(t.m, state) || !on_boundary(t.v, state) || !on_boundary(t.copy, 2) ||
        !on_boundary(t.m_scale, 4) || !on_boundary(t.v_scale, 4))
      return COCODC_ERR_ALIGNMENT;
    arrays.push_back({span(t.p, 1, t.n, t.n, 4), true});
    arrays.push_back({span(t.m, 1, t.n, t.n, state), true});
    arrays.push_back({span(t.v, 1, t.n, t.n, state), true});
    arrays.push_back({span(t.m_scale, 1, units, units, 4), true});
    arrays.push_back({span(t.v_scale, 1, units, units, 4), true});
    arrays.push_back({span(t.copy, 1, t.n, t.n, 2), true});
    arrays.push_back({span(t.grad, 1, t.n, t.n, gb), false});
    const bool wide = on_boundary(t.p, 16) && on_boundary(t.grad, gb == 4 ? 16 : 8) && on_boundary(t.m, 4 * state) && on_boundary(t.v, 4 * state) &&
                      on_boundary(t.copy, 8);
    if (units) out.push_back({t.p, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.n, t.grad_type, t.copy_type, t.decay, (int)i, wide ? 1 : 0, *total});
    *total += units;
  }
  // in order of their first bytes, an array that is written begins behind all before it, a gradient behind all written ones before it
  std::sort(arrays.begin(), arrays.end(), [](const Array& x, const Array& y) { return x.s.lo < y.s.lo; });
  uintptr_t end = 0, written = 0;
  for (const Array& x : arrays) {
    if (x.s.lo >= x.s.hi) continue;
    if (x.s.lo < (x.written ? end : written)) return COCODC_ERR_ALIAS;
    end = std::max(end, x.s.hi);
    if (x.written) written = std::max(written, x.s.hi);
  }
  return COCODC_OK;
}

}  // namespace

extern "C" {

cocodc_status cocodc_lm_adam_create(cocodc_lm_adam** out, cocodc_lm* lm, const cocodc_lm_tensor* tensors, int64_t count, int32_t state_bits) {
  if (!out) return COCODC_ERR_INVALID_ARG;
  *out = nullptr;
  if (!lm || count < 0 || count > (1 << 20) || (count && !tensors) || (state_bits != 32 && state_bits != 8)) return COCODC_ERR_INVALID_ARG;
  try {
    std::vector<Tensor> t;
    long long units = 0;
    const cocodc_status status = check(tensors, count, state_bits, t, &units);
    if (status != COCODC_OK) return status;
    DeviceScope scope(lm->device);
    if (!scope.ok) return COCODC_ERR_CUDA;
    cocodc_lm_adam* plan = new cocodc_lm_adam();
    plan->device = lm->device;
    plan->bits = state_bits;
    plan->units = units;
    plan->count = (int)t.size();
    if (units) {
      const cocodc_status got = allocate(&plan->d_tensors, t.size() * sizeof(Tensor));
      if (got != COCODC_OK) {
        delete plan;
        return got;
      }
      // the copy may return before it has arrived, and a step on another stream does not wait for it
      if (cudaMemcpy(plan->d_tensors, t.data(), t.size() * sizeof(Tensor), cudaMemcpyHostToDevice) != cudaSuccess ||
          cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess) {
        cudaGetLastError();
        cudaFree(plan->d_tensors);
        delete plan;
        return COCODC_ERR_CUDA;
      }
    }
    *out = plan;
    return COCODC_OK;
  } catch (...) {                                    // no memory on the host
    return COCODC_ERR_NOMEM;
  }
}

cocodc_status cocodc_lm_adam_destroy(cocodc_lm_adam* plan) {
  if (!plan) return COCODC_OK;
  DeviceScope scope(plan->device);
  const bool ok = scope.ok && cudaFree(plan->d_tensors) == cudaSuccess;
  delete plan;
  return ok ? COCODC_OK : COCODC_ERR_CUDA;
}

cocodc_status cocodc_lm_adamw(cocodc_lm* lm, const cocodc_lm_adam* plan, double lr, double beta1, double beta2, double eps, int64_t step,
                              const int64_t* step_at, const float* grad_scale, const float* lr_scale, int64_t seed, void* stream) {
  if (!lm || !plan || plan->device != lm->device || !std::isfinite(lr) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) ||
      !(eps == 0 || (eps >= 0x1p-126 && eps <= 0x1p125)) || (!step_at && step < 1))         // a smaller eps would be 0 for the approximate inverse, with a larger one that is 0
    return COCODC_ERR_INVALID_ARG;
  if (!on_boundary(step_at, 8) || !on_boundary(grad_scale, 4) || !on_boundary(lr_scale, 4)) return COCODC_ERR_ALIGNMENT;
  if (plan->units == 0) return COCODC_OK;
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  const AdamArgs a{plan->d_tensors, plan->count, plan->units, (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps,
                   (float)(lr / (1.0 - std::pow(beta1, (double)step))), (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step))), lr, beta1, beta2, step, reinterpret_cast<const long long*>(step_at), grad_scale, lr_scale,
                   (unsigned)seed ^ mix((unsigned)((uint64_t)seed >> 32)), lm->d_status};
  const long long blocks = (plan->units + kWarps - 1) / kWarps, most = (long long)lm->sm_count * (plan->bits == 8 ? 4 : 3);
  const unsigned grid = (unsigned)(blocks < most ? blocks : most);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return plan->bits == 8 ? start(lm, k_adamw<true>, grid, kThreads, 0, st, 1, a) : start(lm, k_adamw<false>, grid, kThreads, 0, st, 1, a);
}

}  // extern "C"
