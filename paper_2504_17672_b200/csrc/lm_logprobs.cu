// Log probabilities of given tokens with entropy and top alternatives, and their gradient (include/cocodc_lm.h).

#include "lm_common.cuh"

using namespace cocodc_lm_impl;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A logit as a 32-bit number with the same order (NaN above +Inf, -0 equal to +0), and with the position behind it
// as one 64-bit number: larger logits first, equal ones by ascending position.  Every key is above 0 and below ~0
// (also a NaN at position 0).
__device__ __forceinline__ unsigned ordered(float x) {
  if (x != x) return 0xffffffffu;
  const unsigned b = __float_as_uint(x + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
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

__device__ __forceinline__ float block_reduce(float v, float* scratch, bool is_max) {
  for (int o = 16; o; o >>= 1) {
    const float w = __shfl_xor_sync(~0u, v, o);
    v = is_max ? fmaxf(v, w) : v + w;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  v = scratch[0];
  for (int w = 1; w < kWarps; ++w) v = is_max ? fmaxf(v, scratch[w]) : v + scratch[w];
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_logprobs(const RowArgs a) {
  __shared__ float scratch[kWarps];
  __shared__ unsigned long long best[kWarps];
  const long long t = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float m = -INFINITY;
  for (unsigned j = tid; j < a.V; j += kThreads) m = fmaxf(m, to_f32(row[j]));
  m = block_reduce(m, scratch, true);
  float s = 0.f, u = 0.f;
  const float c = a.scale * kLog2e;
  for (unsigned j = tid; j < a.V; j += kThreads) {
    const float x = to_f32(row[j]);
    if (x == -INFINITY) continue;
    const float d = (x - m) * c, e = exp2f(d);
    s += e;
    if (e != 0.f) u += e * d;      // a far lower logit: d may be -Inf, e * d is 0
  }
  s = block_reduce(s, scratch, false);
  u = block_reduce(u, scratch, false);
  const bool empty = m == -INFINITY && s == 0.f;
  const float lse = empty ? -INFINITY : m * a.scale + logf(s);
  if (tid == 0) {
    if (a.lse) a.lse[t] = lse;
    if (a.entropy) a.entropy[t] = empty ? 0.f : kLn2 * (log2f(s) - u / s);
    if (a.logp) {
      const long long y = token_at(a.targets, a.targets64, t, a.V, a.status);
      a.logp[t] = y < 0 ? 0.f : empty ? -INFINITY : to_f32(row[y]) * a.scale - lse;
    }
  }
  unsigned long long last = ~0ull;
  for (int i = 0; i < a.top_k; ++i) {
    unsigned long long k = 0;
    for (unsigned j = tid; j < a.V; j += kThreads) {
      const unsigned long long q = key_of(to_f32(row[j]), j);
      if (q < last && q > k) k = q;
    }
    k = warp_max(k);
    __syncthreads();
    if (lane == 0) best[warp] = k;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) k = best[w] > k ? best[w] : k;
    last = k;
    if (tid == 0 && k != 0) {
      const unsigned j = position_of(k);
      a.top_ids[t * a.top_k + i] = (int)j;
      a.top_logp[t * a.top_k + i] = empty ? -INFINITY : to_f32(row[j]) * a.scale - lse;
    }
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

constexpr int kGradElems = 2048;   // elements of a row that one CTA takes

template <typename T>
__global__ void __launch_bounds__(kThreads) k_logprobs_grad(const GradArgs a) {
  const long long chunks = (a.V + kGradElems - 1LL) / kGradElems;
  const long long t = blockIdx.x / chunks;
  const unsigned j0 = (unsigned)(blockIdx.x - t * chunks) * kGradElems;
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  T* out = static_cast<T*>(a.dlogits) + t * a.dstride;
  const long long y = a.dlogp ? token_at(a.targets, a.targets64, t, a.V, a.status) : -1;
  const float lse = a.lse[t];
  const float g = y >= 0 ? a.dlogp[t] : 0.f;
  const float h = a.dentropy ? a.dentropy[t] : 0.f, H = a.dentropy ? a.entropy[t] : 0.f;
  for (unsigned j = j0 + threadIdx.x; j < a.V && j < j0 + kGradElems; j += kThreads) {
    float d = 0.f;
    if (lse != -INFINITY) {
      const float lp = to_f32(row[j]) * a.scale - lse, p = expf(lp);
      if (lp != -INFINITY) d = -p * (g + h * (lp + H));
      if (j == y) d += g;
    }
    out[j] = from_f32<T>(a.scale * d);
  }
}

}  // namespace

namespace cocodc_lm_impl {
bool logprobs_prepare() { return true; }
}  // namespace cocodc_lm_impl

extern "C" {

cocodc_status cocodc_lm_logprobs(cocodc_lm* lm, const void* logits, int32_t type, int64_t stride, int64_t T, int64_t V,
                                 const void* targets, int32_t targets_type, float scale, float* logp, float* entropy,
                                 float* lse, int32_t top_k, int32_t* top_ids, float* top_logp, void* stream) {
  if (!lm || !known_type(type) || !sane(T) || T > INT32_MAX || V < 1 || V > INT32_MAX || stride < V || !sane(stride) ||
      !(scale > 0.f) || scale > 3.4e38f || top_k < 0 || top_k > COCODC_LM_MAX_TOP || top_k > V)
    return COCODC_ERR_INVALID_ARG;
  if ((targets == nullptr) != (logp == nullptr) || (top_k > 0 && T > 0) != (top_ids != nullptr && top_logp != nullptr) ||
      (targets && targets_type != COCODC_I32 && targets_type != COCODC_I64))
    return COCODC_ERR_INVALID_ARG;
  if (T == 0) return COCODC_OK;
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
  with_type(type, [&](auto x) {
    k_logprobs<decltype(x)><<<(unsigned)T, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
    return true;
  });
  return launched(lm);
}

cocodc_status cocodc_lm_logprobs_grad(cocodc_lm* lm, const void* logits, int32_t type, int64_t stride, int64_t T,
                                      int64_t V, const void* targets, int32_t targets_type, float scale,
                                      const float* lse, const float* entropy, const float* dlogp,
                                      const float* dentropy, void* dlogits, int64_t dlogits_stride, void* stream) {
  if (!lm || !known_type(type) || !sane(T) || T > INT32_MAX || V < 1 || V > INT32_MAX || stride < V || !sane(stride) ||
      dlogits_stride < V || !sane(dlogits_stride) || !(scale > 0.f) || scale > 3.4e38f)
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
  const long long blocks = T * ((V + kGradElems - 1) / kGradElems);
  if (blocks > INT32_MAX) return COCODC_ERR_INVALID_ARG;
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  const GradArgs a{logits, stride, T, (unsigned)V, targets, targets_type == COCODC_I64, scale, lse, entropy, dlogp,
                   dentropy, dlogits, dlogits_stride, lm->d_status};
  with_type(type, [&](auto x) {
    k_logprobs_grad<decltype(x)><<<(unsigned)blocks, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
    return true;
  });
  return launched(lm);
}

}  // extern "C"
