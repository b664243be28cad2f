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
constexpr int kTileUnits = 16;                       // a block's share: 4096 elements of one tensor
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
  int wide;                                          // every array starts where vector accesses may
};
struct Tile { int tensor, first; };                  // first: its first unit

}  // namespace

struct cocodc_lm_adam {
  int device = 0, bits = 32;
  long long tiles = 0;
  Tensor* d_tensors = nullptr;
  Tile* d_tiles = nullptr;
};

namespace {

struct AdamArgs {
  const Tensor* tensors;
  const Tile* tiles;
  long long count;
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

// x in [0, 448] to an e4m3 code, up with probability (what is cut off) / (spacing): bits holds 16 random ones.  From 2^-6 on
// they are added below the three bits of mantissa that stay; below, the codes are multiples of 2^-9.
__device__ __forceinline__ unsigned round_8(float x, unsigned bits) {
  const unsigned cut = ((__float_as_uint(x) + (bits << 4)) >> 20) - (120u << 3);
  const float u = __uint_as_float(0x3f800000u | bits << 7) - 1.f;
  const unsigned whole = __float_as_uint(__fadd_rz(fmaf(x, 512.f, u), 8388608.f)) & 15u;      // floor of a number below 16
  return x < 0.015625f ? whole : cut;
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
// finite magnitudes as whole numbers, whose order is theirs; 0 for the others
__device__ __forceinline__ unsigned magnitude(float x) {
  const unsigned b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// A warp takes a unit: lane l has its elements 4 l .. 4 l + 3 and 128 + 4 l .. 128 + 4 l + 3, so that neighbours read neighbours in
// every width.  Read once, written once: bound by memory.
template <bool EIGHT> __global__ void __launch_bounds__(kThreads) k_adamw(const AdamArgs a) {
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
  __syncthreads();
  const float k1 = factors[0], k2 = factors[1], gs = a.grad_scale ? *a.grad_scale : 1.f;
  const double lr = shared_lr;
  const unsigned step_bits = (unsigned)(a.step_at ? *a.step_at : a.step);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (long long at = blockIdx.x; at < a.count; at += gridDim.x) {
    const Tile tile = a.tiles[at];
    const Tensor t = a.tensors[tile.tensor];
    const float keep = (float)(1.0 - lr * (double)t.decay);
    const long long units = (t.n + kUnit - 1) / kUnit;
    for (long long unit = (long long)tile.first + warp; unit < min(units, (long long)tile.first + kTileUnits); unit += kWarps) {
      const long long base = unit * kUnit;
      const int here = (int)min((long long)kUnit, t.n - base);
      const bool wide = t.wide && here == kUnit;
      float p[8], g[8], m[8], v[8];
      float ms = 0.f, vs = 0.f;
      if (EIGHT) {
        ms = t.m_scale[unit];
        vs = t.v_scale[unit];
      }
      if (wide) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const long long i = base + h * 128 + lane * 4;
          const uint4 rp = load16(t.p + i);
          uint4 rg, rm, rv;
          if (t.grad_type == COCODC_F32) {
            rg = load16(static_cast<const float*>(t.grad) + i);
          } else {
            const uint2 q = load8(static_cast<const unsigned short*>(t.grad) + i);
            rg = make_uint4(q.x, q.y, 0, 0);
          }
          if (EIGHT) {
            rm.x = load4(static_cast<const unsigned char*>(t.m) + i);
            rv.x = load4(static_cast<const unsigned char*>(t.v) + i);
          } else {
            rm = load16(static_cast<const float*>(t.m) + i);
            rv = load16(static_cast<const float*>(t.v) + i);
          }
          float *pp = p + 4 * h, *pg = g + 4 * h, *pm = m + 4 * h, *pv = v + 4 * h;
          pp[0] = __uint_as_float(rp.x); pp[1] = __uint_as_float(rp.y); pp[2] = __uint_as_float(rp.z); pp[3] = __uint_as_float(rp.w);
          if (t.grad_type == COCODC_F32) {
            pg[0] = __uint_as_float(rg.x); pg[1] = __uint_as_float(rg.y); pg[2] = __uint_as_float(rg.z); pg[3] = __uint_as_float(rg.w);
          } else if (t.grad_type == COCODC_BF16) {
            pg[0] = __uint_as_float(rg.x << 16); pg[1] = __uint_as_float(rg.x & 0xffff0000u);
            pg[2] = __uint_as_float(rg.y << 16); pg[3] = __uint_as_float(rg.y & 0xffff0000u);
          } else {
            const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&rg.x)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&rg.y));
            pg[0] = f0.x; pg[1] = f0.y; pg[2] = f1.x; pg[3] = f1.y;
          }
          if (EIGHT) {
            const float2 m0 = widen_e4m3((unsigned short)rm.x), m1 = widen_e4m3((unsigned short)(rm.x >> 16));
            const float2 v0 = widen_e4m3((unsigned short)rv.x), v1 = widen_e4m3((unsigned short)(rv.x >> 16));
            pm[0] = m0.x; pm[1] = m0.y; pm[2] = m1.x; pm[3] = m1.y;
            pv[0] = v0.x; pv[1] = v0.y; pv[2] = v1.x; pv[3] = v1.y;
          } else {
            pm[0] = __uint_as_float(rm.x); pm[1] = __uint_as_float(rm.y); pm[2] = __uint_as_float(rm.z); pm[3] = __uint_as_float(rm.w);
            pv[0] = __uint_as_float(rv.x); pv[1] = __uint_as_float(rv.y); pv[2] = __uint_as_float(rv.z); pv[3] = __uint_as_float(rv.w);
          }
        }
      } else {
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
        p[e] = __fadd_rn(__fmul_rn(p[e], keep), -__fdividef(__fmul_rn(m[e], k1), __fadd_rn(__fmul_rn(root[e], k2), a.eps)));
      }
      unsigned mc[8], vc[8];
      if (EIGHT) {
        unsigned top_m = 0, top_v = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int o = e / 4 * 128 + lane * 4 + e % 4;
          if (o < here) {
            top_m = max(top_m, magnitude(m[e]));
            top_v = max(top_v, magnitude(root[e]));
          }
        }
        top_m = __reduce_max_sync(~0u, top_m);
        top_v = __reduce_max_sync(~0u, top_v);
        ms = scale_8(top_m);
        vs = scale_8(top_v);
        const float im = __fdiv_rn(1.f, ms), iv = __fdiv_rn(1.f, vs);
        unsigned key = mix(a.seed + kGolden) ^ step_bits;
        key = mix(key + kGolden) ^ (unsigned)tile.tensor;
        key = mix(key + kGolden) ^ (unsigned)unit;
        key = mix(key + kGolden);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const unsigned bits = mix(key + (unsigned)(e / 4 * 128 + lane * 4 + e % 4) * kGolden);
          mc[e] = round_8(fminf(__fmul_rn(fabsf(m[e]), im), kMost8), bits & 0xffffu) | (__float_as_uint(m[e]) >> 24 & 0x80u);
          vc[e] = round_8(fminf(__fmul_rn(root[e], iv), kMost8), bits >> 16);
          if (root[e] > 0.f) vc[e] = max(vc[e], 1u);
          if (magnitude(m[e]) == 0 && m[e] != 0.f) mc[e] = 0x7f;
          if (magnitude(root[e]) == 0 && root[e] != 0.f) vc[e] = 0x7f;
        }
        if (lane == 0) {
          t.m_scale[unit] = ms;
          t.v_scale[unit] = vs;
        }
      }
      if (wide) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const long long i = base + h * 128 + lane * 4;
          const float *pp = p + 4 * h, *pm = m + 4 * h, *pv = v + 4 * h;
          *reinterpret_cast<float4*>(t.p + i) = make_float4(pp[0], pp[1], pp[2], pp[3]);
          if (EIGHT) {
            const unsigned *qm = mc + 4 * h, *qv = vc + 4 * h;
            *reinterpret_cast<unsigned*>(static_cast<unsigned char*>(t.m) + i) = qm[0] | qm[1] << 8 | qm[2] << 16 | qm[3] << 24;
            *reinterpret_cast<unsigned*>(static_cast<unsigned char*>(t.v) + i) = qv[0] | qv[1] << 8 | qv[2] << 16 | qv[3] << 24;
          } else {
            *reinterpret_cast<float4*>(static_cast<float*>(t.m) + i) = make_float4(pm[0], pm[1], pm[2], pm[3]);
            *reinterpret_cast<float4*>(static_cast<float*>(t.v) + i) = make_float4(pv[0], pv[1], pv[2], pv[3]);
          }
          if (t.copy)
            *reinterpret_cast<uint2*>(static_cast<unsigned short*>(t.copy) + i) =
                make_uint2(narrow2(t.copy_type, pp[0], pp[1]), narrow2(t.copy_type, pp[2], pp[3]));
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int o = e / 4 * 128 + lane * 4 + e % 4;
          if (o >= here) continue;
          t.p[base + o] = p[e];
          if (EIGHT) {
            static_cast<unsigned char*>(t.m)[base + o] = (unsigned char)mc[e];
            static_cast<unsigned char*>(t.v)[base + o] = (unsigned char)vc[e];
          } else {
            static_cast<float*>(t.m)[base + o] = m[e];
            static_cast<float*>(t.v)[base + o] = v[e];
          }
          if (t.copy) static_cast<unsigned short*>(t.copy)[base + o] = (unsigned short)narrow2(t.copy_type, p[e], 0.f);
        }
      }
    }
  }
}

cocodc_status check(const cocodc_lm_tensor* tensors, int64_t count, int32_t bits, std::vector<Tensor>& out, std::vector<Tile>& tiles) {
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
    out.push_back({t.p, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.n, t.grad_type, t.copy_type, t.decay, wide ? 1 : 0});
    for (int64_t u = 0; u < units; u += kTileUnits) tiles.push_back({(int)i, (int)u});
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
    std::vector<Tile> tiles;
    const cocodc_status status = check(tensors, count, state_bits, t, tiles);
    if (status != COCODC_OK) return status;
    DeviceScope scope(lm->device);
    if (!scope.ok) return COCODC_ERR_CUDA;
    cocodc_lm_adam* plan = new cocodc_lm_adam();
    plan->device = lm->device;
    plan->bits = state_bits;
    plan->tiles = (long long)tiles.size();
    if (plan->tiles) {
      const bool ok = cudaMalloc(&plan->d_tensors, t.size() * sizeof(Tensor)) == cudaSuccess &&
                      cudaMalloc(&plan->d_tiles, tiles.size() * sizeof(Tile)) == cudaSuccess &&
                      cudaMemcpy(plan->d_tensors, t.data(), t.size() * sizeof(Tensor), cudaMemcpyHostToDevice) == cudaSuccess &&
                      cudaMemcpy(plan->d_tiles, tiles.data(), tiles.size() * sizeof(Tile), cudaMemcpyHostToDevice) == cudaSuccess;
      if (!ok) {
        cudaGetLastError();
        cudaFree(plan->d_tensors);
        cudaFree(plan->d_tiles);
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
  bool ok = scope.ok && cudaFree(plan->d_tensors) == cudaSuccess;
  ok = scope.ok && cudaFree(plan->d_tiles) == cudaSuccess && ok;
  delete plan;
  return ok ? COCODC_OK : COCODC_ERR_CUDA;
}

cocodc_status cocodc_lm_adamw(cocodc_lm* lm, const cocodc_lm_adam* plan, double lr, double beta1, double beta2, double eps, int64_t step,
                              const int64_t* step_at, const float* grad_scale, const float* lr_scale, int64_t seed, void* stream) {
  if (!lm || !plan || plan->device != lm->device || !std::isfinite(lr) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) ||
      !(eps >= 0 && eps <= 1) || (!step_at && step < 1))
    return COCODC_ERR_INVALID_ARG;
  if (!on_boundary(step_at, 8) || !on_boundary(grad_scale, 4) || !on_boundary(lr_scale, 4)) return COCODC_ERR_ALIGNMENT;
  if (plan->tiles == 0) return COCODC_OK;
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  const AdamArgs a{plan->d_tensors, plan->d_tiles, plan->tiles, (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps,
                   lr, beta1, beta2, step, reinterpret_cast<const long long*>(step_at), grad_scale, lr_scale, (unsigned)seed, lm->d_status};
  const long long most = (long long)lm->sm_count * 4;
  const unsigned grid = (unsigned)(plan->tiles < most ? plan->tiles : most);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return plan->bits == 8 ? start(lm, k_adamw<true>, grid, kThreads, 0, st, 1, a) : start(lm, k_adamw<false>, grid, kThreads, 0, st, 1, a);
}

}  // extern "C"
