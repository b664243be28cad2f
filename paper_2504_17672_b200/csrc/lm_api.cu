// Handle of the local step's operators (include/cocodc_lm.h): a status word and a launch counter.

#include "lm_common.cuh"

#include <cstring>
#include <new>
#include <tuple>
#include <type_traits>

using namespace cocodc_lm_impl;

namespace {
// The next word of a record, as what the parameter asks for.
struct Reader {
  const char* at;
  int64_t word() {
    int64_t w;
    std::memcpy(&w, at, 8);
    at += 8;
    return w;
  }
  template <typename T> T next() {
    if constexpr (std::is_pointer_v<T>) {
      return reinterpret_cast<T>(static_cast<uintptr_t>(word()));
    } else if constexpr (std::is_floating_point_v<T>) {
      const int64_t w = word();
      double d;
      std::memcpy(&d, &w, 8);
      return static_cast<T>(d);
    } else {
      return static_cast<T>(word());
    }
  }
};
template <typename... P> cocodc_status call(cocodc_status (*f)(cocodc_lm*, P...), cocodc_lm* lm, Reader r) {
  std::tuple<P...> args{r.next<P>()...};     // braces: read from left to right
  return std::apply([&](const P&... p) { return f(lm, p...); }, args);
}
}  // namespace

extern "C" {

cocodc_status cocodc_lm_create(cocodc_lm** lm_out, int32_t device) {
  if (!lm_out) return COCODC_ERR_INVALID_ARG;
  *lm_out = nullptr;
  int n_dev = 0;
  if (cudaGetDeviceCount(&n_dev) != cudaSuccess) return COCODC_ERR_CUDA;
  if (device < 0 || device >= n_dev) return COCODC_ERR_INVALID_ARG;
  DeviceScope scope(device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  cocodc_lm* lm = new (std::nothrow) cocodc_lm();
  if (!lm) return COCODC_ERR_NOMEM;
  lm->device = device;
  const cocodc_status got = cocodc_lm_impl::allocate(&lm->d_status, sizeof(int));
  if (got != COCODC_OK) {
    delete lm;
    return got;
  }
  bool ok = cudaDeviceGetAttribute(&lm->sm_count, cudaDevAttrMultiProcessorCount, device) == cudaSuccess;
  // cudaMemset may return before it is done, and calls on other streams do not wait for it
  ok = ok && cudaMemset(lm->d_status, 0, sizeof(int)) == cudaSuccess && cudaStreamSynchronize(cudaStreamLegacy) == cudaSuccess;
  ok = ok && embed_prepare() && glu_prepare() && head_prepare() && norm_prepare();
  if (!ok) {
    cudaGetLastError();
    cudaFree(lm->d_status);
    delete lm;
    return COCODC_ERR_CUDA;
  }
  *lm_out = lm;
  return COCODC_OK;
}

cocodc_status cocodc_lm_destroy(cocodc_lm* lm) {
  if (!lm) return COCODC_OK;
  DeviceScope scope(lm->device);
  const bool ok = scope.ok && cudaFree(lm->d_status) == cudaSuccess;
  delete lm;
  return ok ? COCODC_OK : COCODC_ERR_CUDA;
}

cocodc_status cocodc_lm_poll_status(cocodc_lm* lm, void* stream) {
  if (!lm) return COCODC_ERR_INVALID_ARG;
  DeviceScope scope(lm->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int word = 0;
  const auto failed = [] {
    cudaGetLastError();                                // reported here, nobody else is to find it
    return COCODC_ERR_CUDA;
  };
  if (!scope.ok || cudaMemcpyAsync(&word, lm->d_status, sizeof(int), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
      cudaStreamSynchronize(st) != cudaSuccess)
    return failed();
  // cleared only when something was read: an error that a call on another stream records meanwhile is not lost
  if (word != 0 && (cudaMemsetAsync(lm->d_status, 0, sizeof(int), st) != cudaSuccess ||
                    cudaStreamSynchronize(st) != cudaSuccess))
    return failed();
  return static_cast<cocodc_status>(word);
}

cocodc_status cocodc_lm_submit(cocodc_lm* lm, const void* record) {
  if (!lm || !record) return COCODC_ERR_INVALID_ARG;
  Reader r{static_cast<const char*>(record)};
  switch (r.word()) {
    case COCODC_LM_EMBED: return call(cocodc_lm_embed, lm, r);
    case COCODC_LM_EMBED_GRAD: return call(cocodc_lm_embed_grad, lm, r);
    case COCODC_LM_GLU: return call(cocodc_lm_glu, lm, r);
    case COCODC_LM_GLU_GRAD: return call(cocodc_lm_glu_grad, lm, r);
    case COCODC_LM_LOGPROBS: return call(cocodc_lm_logprobs, lm, r);
    case COCODC_LM_LOGPROBS_GRAD: return call(cocodc_lm_logprobs_grad, lm, r);
    case COCODC_LM_NORM: return call(cocodc_lm_norm, lm, r);
    case COCODC_LM_NORM_GRAD: return call(cocodc_lm_norm_grad, lm, r);
    case COCODC_LM_HEAD: return call(cocodc_lm_head, lm, r);
    case COCODC_LM_HEAD_GRAD: return call(cocodc_lm_head_grad, lm, r);
    case COCODC_LM_ADAMW: return call(cocodc_lm_adamw, lm, r);
  }
  return COCODC_ERR_INVALID_ARG;
}

int64_t cocodc_lm_launch_count(const cocodc_lm* lm) { return lm ? (int64_t)lm->launches.load() : 0; }

}  // extern "C"
