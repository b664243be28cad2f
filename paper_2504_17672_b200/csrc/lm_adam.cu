// The AdamW step over many tensors (include/cocodc_lm.h).

#include "lm_common.cuh"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

using namespace cocodc_lm_impl;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
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
  double lr, beta1, beta2;
  long long step;
  const long long* step_at;
  const float *grad_scale, *lr_scale;
  unsigned seed;
  int* status;
};

// One round of multiplications and shifts that spreads every bit over the word (the 32-bit finaliser with Appleby's constants).
__device__ __forceinline__ unsigned mix(unsigned x) {
  x = (x ^ x >> 16) * 0x85EBCA6Bu;
  x = (x ^ x >> 13) * 0xC2B2AE35u;
  return x ^ x >> 16;
}
constexpr unsigned kGolden = 0x9E3779B9u;

// A number x of a unit's largest magnitude 448 to an e4m3 code in the highest byte, without its sign: up with probability (what is cut off) /
// (spacing).  Times 2^-120 the exponents of e4m3 are those of fp32, numbers below its smallest normal one too (2^-126 here and there), so that the
// code is what stands above the lowest 20 bits; 16 random bits, here bytes 1 and 2, are added to those.  x may be 448 + 3 ulp: no carry comes of it.
__device__ __forceinline__ unsigned code_of(float x, unsigned random) {
  return (__float_as_uint(__fmul_rn(x, 0x1p-120f)) << 4) + random;
}
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
__device__ __forceinline__ unsigned narrow2(int type, float a, float b) {
  if (type == COCODC_BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const unsigned*>(&v);
  }
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&v);
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

// A unit's numbers on their way: lane l has its elements 4 l .. 4 l + 3 and 128 + 4 l .. 128 + 4 l + 3, so that neighbours read neighbours in
// every width.
template <bool EIGHT> struct RawUnit {
  uint4 p[2], g[2];
  uint4 m[EIGHT ? 1 : 2], v[EIGHT ? 1 : 2];          // EIGHT: codes in x and y
  float ms, vs;
};
template <bool EIGHT> __device__ __forceinline__ void fetch(RawUnit<EIGHT>& r, const Tensor& t, long long unit, int lane) {
  const long long base = unit * kUnit + lane * 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const long long i = base + h * 128;
    r.p[h] = load16(t.p + i);
    if (t.grad_type == COCODC_F32) {
      r.g[h] = load16(static_cast<const float*>(t.grad) + i);
    } else {
      const uint2 q = load8(static_cast<const unsigned short*>(t.grad) + i);
      r.g[h].x = q.x;
      r.g[h].y = q.y;
    }
    if (EIGHT) {
      (h ? r.m[0].y : r.m[0].x) = load4(static_cast<const unsigned char*>(t.m) + i);
      (h ? r.v[0].y : r.v[0].x) = load4(static_cast<const unsigned char*>(t.v) + i);
    } else {
      r.m[h] = load16(static_cast<const float*>(t.m) + i);
      r.v[h] = load16(static_cast<const float*>(t.v) + i);
    }
  }
  if (EIGHT) {
    r.ms = t.m_scale[unit];
    r.vs = t.v_scale[unit];
  }
}
__device__ __forceinline__ void spread4(const uint4& r, float* v) {
  v[0] = __uint_as_float(r.x);
  v[1] = __uint_as_float(r.y);
  v[2] = __uint_as_float(r.z);
  v[3] = __uint_as_float(r.w);
}
template <bool EIGHT>
__device__ __forceinline__ void spread(const RawUnit<EIGHT>& r, int grad_type, float (&p)[8], float (&g)[8], float (&m)[8], float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    spread4(r.p[h], p + 4 * h);
    float* pg = g + 4 * h;
    if (grad_type == COCODC_F32) {
      spread4(r.g[h], pg);
    } else if (grad_type == COCODC_BF16) {
      pg[0] = __uint_as_float(r.g[h].x << 16);
      pg[1] = __uint_as_float(r.g[h].x & 0xffff0000u);
      pg[2] = __uint_as_float(r.g[h].y << 16);
      pg[3] = __uint_as_float(r.g[h].y & 0xffff0000u);
    } else {
      const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&r.g[h].x)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&r.g[h].y));
      pg[0] = f0.x;
      pg[1] = f0.y;
      pg[2] = f1.x;
      pg[3] = f1.y;
    }
    if (EIGHT) {
      const unsigned cm = h ? r.m[0].y : r.m[0].x, cv = h ? r.v[0].y : r.v[0].x;
      const float2 m0 = widen_e4m3((unsigned short)cm), m1 = widen_e4m3((unsigned short)(cm >> 16));
      const float2 v0 = widen_e4m3((unsigned short)cv), v1 = widen_e4m3((unsigned short)(cv >> 16));
      m[4 * h] = m0.x; m[4 * h + 1] = m0.y; m[4 * h + 2] = m1.x; m[4 * h + 3] = m1.y;
      v[4 * h] = v0.x; v[4 * h + 1] = v0.y; v[4 * h + 2] = v1.x; v[4 * h + 3] = v1.y;
    } else {
      spread4(r.m[h], m + 4 * h);
      spread4(r.v[h], v + 4 * h);
    }
  }
}

// Read once, written once: bound by memory.  The units of all tensors form one row, of which each block takes an equal part and its warps one unit
// in turn: a warp walks from tensor to tensor, and the next unit's numbers are on their way while it works on one.
template <bool EIGHT> __global__ void __launch_bounds__(kThreads, EIGHT ? 3 : 2) k_adamw(const AdamArgs a) {
  wait_for_previous();
  may_follow();
  __shared__ float factors[2];
  __shared__ double shared_lr;
  if (threadIdx.x == 0) {
    long long step = a.step_at ? *a.step_at : a.step;
    if (step < 1) {
      record(a.status, COCODC_ERR_INVALID_ARG);
      step = 1;
    }
    const double lr = a.lr_scale ? a.lr * (double)*a.lr_scale : a.lr;
    factors[0] = (float)(lr / (1.0 - pow(a.beta1, (double)step)));
    factors[1] = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)step)));
    shared_lr = lr;
  }
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const unsigned step_bits = (unsigned)(a.step_at ? *a.step_at : a.step);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const long long last = a.units * (blockIdx.x + 1) / gridDim.x;
  long long unit = a.units * blockIdx.x / gridDim.x + warp;
  // the tensor of the warp's first unit: the last one that begins at or before it
  int at = 0;
  for (int n = a.count; n > 1;) {
    const int half = n / 2;
    if (a.tensors[at + half].first <= unit) at += half;
    n -= half;
  }
  long long behind = a.tensors[at].first + (a.tensors[at].n + kUnit - 1) / kUnit;      // the unit behind the tensor's last
  const auto whole = [&](const Tensor& t, long long u) { return t.wide && (u - t.first + 1) * kUnit <= t.n; };
  RawUnit<EIGHT> raw;
  if (unit < last && whole(a.tensors[at], unit)) fetch(raw, a.tensors[at], unit - a.tensors[at].first, lane);
  __syncthreads();
  const float k1 = factors[0], k2 = factors[1];
  while (unit < last) {
    const Tensor& t = a.tensors[at];
    const long long own = unit - t.first, base = own * kUnit;
    const bool wide = whole(t, unit);
    const float keep = (float)(1.0 - shared_lr * (double)t.decay);
    float p[8], g[8], m[8], v[8], ms = 0.f, vs = 0.f;
    const int here = (int)min((long long)kUnit, t.n - base);
    if (wide) {
      spread(raw, t.grad_type, p, g, m, v);
      ms = raw.ms;
      vs = raw.vs;
    } else {
      if (EIGHT) {
        ms = t.m_scale[own];
        vs = t.v_scale[own];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int o = e / 4 * 128 + lane * 4 + e % 4;
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
    }
    // the next unit's
    const int now = at;
    unit += kWarps;
    while (unit < last && unit >= behind) {
      ++at;
      behind = a.tensors[at].first + (a.tensors[at].n + kUnit - 1) / kUnit;
    }
    if (unit < last && whole(a.tensors[at], unit)) fetch(raw, a.tensors[at], unit - a.tensors[at].first, lane);
    float root[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (EIGHT) {
        m[e] = __fmul_rn(m[e], ms);
        v[e] = __fmul_rn(v[e], vs);
        v[e] = __fmul_rn(v[e], v[e]);
      }
      const float gr = __fmul_rn(g[e], gs);
      m[e] = __fadd_rn(__fmul_rn(m[e], a.b1), __fmul_rn(gr, a.c1));
      v[e] = __fadd_rn(__fmul_rn(v[e], a.b2), __fmul_rn(__fmul_rn(gr, a.c2), gr));
      root[e] = __fsqrt_rn(v[e]);
      p[e] = __fadd_rn(__fmul_rn(p[e], keep), -__fmul_rn(__fmul_rn(m[e], k1), inverse(__fadd_rn(__fmul_rn(root[e], k2), a.eps))));
    }
    unsigned mc[2], vc[2];                             // codes of four elements each
    if (EIGHT) {
      float top_m = 0.f, top_v = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        top_m = larger(top_m, m[e]);
        top_v = larger(top_v, root[e]);
      }
      unsigned most_m = __reduce_max_sync(~0u, __float_as_uint(top_m)), most_v = __reduce_max_sync(~0u, __float_as_uint(top_v));
      const bool odd = max(most_m, most_v) >= 0x7f800000u;             // a number that is not finite, somewhere in the unit
      if (odd) {
        most_m = most_v = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          most_m = max(most_m, finite_magnitude(m[e]));
          most_v = max(most_v, finite_magnitude(root[e]));
        }
        most_m = __reduce_max_sync(~0u, most_m);
        most_v = __reduce_max_sync(~0u, most_v);
      }
      ms = scale_8(most_m);
      vs = scale_8(most_v);
      const float im = __fdiv_rn(1.f, ms), iv = __fdiv_rn(1.f, vs);
      unsigned key = mix(a.seed + kGolden) ^ step_bits;
      key = mix(key + kGolden) ^ (unsigned)a.tensors[now].position;
      key = mix(key + kGolden) ^ (unsigned)own;
      key = mix(key + kGolden) + (unsigned)(lane * 4) * kGolden;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        unsigned cm[4], cv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = h * 4 + i;
          const unsigned bits = mix(key + (unsigned)(h * 128 + i) * kGolden);
          cm[i] = code_of(__fmul_rn(m[e], im), __byte_perm(bits, 0, 0x4104));
          // a root above zero (none is below 2^-75) stays above zero
          cv[i] = max(code_of(__fmul_rn(root[e], iv), __byte_perm(bits, 0, 0x4324)), min(__float_as_uint(root[e]), 1u << 24));
          if (odd) {
            if (finite_magnitude(m[e]) == 0 && m[e] != 0.f) cm[i] = 0x7f000000u;
            if (finite_magnitude(root[e]) == 0 && root[e] != 0.f) cv[i] = 0x7f000000u;
          }
        }
        const auto pack = [](const unsigned* c) { return __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410); };
        unsigned sign[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sign[i] = __float_as_uint(m[h * 4 + i]);
        mc[h] = (pack(cm) & 0x7f7f7f7fu) | (pack(sign) & 0x80808080u);
        vc[h] = pack(cv);
      }
    }
    const Tensor& d = a.tensors[now];
    if (EIGHT && lane == 0) {
      d.m_scale[own] = ms;
      d.v_scale[own] = vs;
    }
    if (wide) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const long long i = base + h * 128 + lane * 4;
        const float *pp = p + 4 * h, *pm = m + 4 * h, *pv = v + 4 * h;
        *reinterpret_cast<float4*>(d.p + i) = make_float4(pp[0], pp[1], pp[2], pp[3]);
        if (EIGHT) {
          *reinterpret_cast<unsigned*>(static_cast<unsigned char*>(d.m) + i) = mc[h];
          *reinterpret_cast<unsigned*>(static_cast<unsigned char*>(d.v) + i) = vc[h];
        } else {
          *reinterpret_cast<float4*>(static_cast<float*>(d.m) + i) = make_float4(pm[0], pm[1], pm[2], pm[3]);
          *reinterpret_cast<float4*>(static_cast<float*>(d.v) + i) = make_float4(pv[0], pv[1], pv[2], pv[3]);
        }
        if (d.copy)
          *reinterpret_cast<uint2*>(static_cast<unsigned short*>(d.copy) + i) =
              make_uint2(narrow2(d.copy_type, pp[0], pp[1]), narrow2(d.copy_type, pp[2], pp[3]));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int o = e / 4 * 128 + lane * 4 + e % 4;
        if (o >= here) continue;
        d.p[base + o] = p[e];
        if (EIGHT) {
          static_cast<unsigned char*>(d.m)[base + o] = (unsigned char)(mc[e / 4] >> e % 4 * 8);
          static_cast<unsigned char*>(d.v)[base + o] = (unsigned char)(vc[e / 4] >> e % 4 * 8);
        } else {
          static_cast<float*>(d.m)[base + o] = m[e];
          static_cast<float*>(d.v)[base + o] = v[e];
        }
        if (d.copy) static_cast<unsigned short*>(d.copy)[base + o] = (unsigned short)narrow2(d.copy_type, p[e], 0.f);
      }
    }
  }
}

cocodc_status check(const cocodc_lm_tensor* tensors, int64_t count, int32_t bits, std::vector<Tensor>& out, long long* total) {
  struct Array { Span s; bool written; };
  std::vector<Array> arrays;
  const int state = bits == 8 ? 1 : 4;
  for (int64_t i = 0; i < count; ++i) {
    const cocodc_lm_tensor& t = tensors[i];
    if (t.n < 0 || t.n > (int64_t(1) << 38) || !known_type(t.grad_type) || (t.copy && t.copy_type != COCODC_BF16 && t.copy_type != COCODC_F16) ||
        !(t.decay >= 0.f && t.decay <= 1e30f) || t.reserved != 0)
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
      const bool ok = cudaMalloc(&plan->d_tensors, t.size() * sizeof(Tensor)) == cudaSuccess &&
                      cudaMemcpy(plan->d_tensors, t.data(), t.size() * sizeof(Tensor), cudaMemcpyHostToDevice) == cudaSuccess;
      if (!ok) {
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
      !(eps >= 0 && eps <= 1) || (!step_at && step < 1))
    return COCODC_ERR_INVALID_ARG;
  if (!on_boundary(step_at, 8) || !on_boundary(grad_scale, 4) || !on_boundary(lr_scale, 4)) return COCODC_ERR_ALIGNMENT;
  if (plan->units == 0) return COCODC_OK;
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  const AdamArgs a{plan->d_tensors, plan->count, plan->units, (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps,
                   lr, beta1, beta2, step, reinterpret_cast<const long long*>(step_at), grad_scale, lr_scale, (unsigned)seed, lm->d_status};
  const long long blocks = (plan->units + kWarps - 1) / kWarps, most = (long long)lm->sm_count * (plan->bits == 8 ? 3 : 2);
  const unsigned grid = (unsigned)(blocks < most ? blocks : most);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return plan->bits == 8 ? start(lm, k_adamw<true>, grid, kThreads, 0, st, 1, a) : start(lm, k_adamw<false>, grid, kThreads, 0, st, 1, a);
}

}  // extern "C"
