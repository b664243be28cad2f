// Embedding lookup with scaling, and its gradient by sorted tokens (include/cocodc_lm.h).

#include "lm_common.cuh"

using namespace cocodc_lm_impl;

namespace {

// ---- lookup ------------------------------------------------------------------------------------
template <typename TIn, typename TOut>
__global__ void __launch_bounds__(256) k_embed(const TIn* table, long long table_stride, long long V, long long D,
                                               const void* ids, int is64, long long T, float scale, TOut* y,
                                               long long y_stride, int* status) {
  const long long n = T * D;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long t = i / D, d = i - t * D;
    const long long v = token_at(ids, is64, t, V, status);
    y[t * y_stride + d] = from_f32<TOut>(v < 0 ? 0.f : scale * to_f32(table[v * table_stride + d]));
  }
}

// ---- gradient, step 1: the tokens sorted by id --------------------------------------------------
// One CTA owns the kBinRows (or fewer) consecutive table rows from lo on and finds their tokens itself by walking over all T ids
// twice; no CTA waits for another.  Walk 1 counts, per row and warp, how often the row occurs in the warp's contiguous
// part of the ids, and how many ids lie below lo (where this CTA's rows start in the sorted order).  A prefix sum
// over (row, warp) turns the counts into positions, and walk 2 places every token: equal ids stay in the order of
// their positions because a warp's part precedes the next warp's and ballots rank the lanes of a warp.
// All T ids are read by every CTA, from L2 after the first: at 65536 tokens of 4 bytes and 148 CTAs 39 MB a walk.
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxBinRows = 768;                       // (rows * 33 + 64) * 4 bytes of shared memory: 99 KB
constexpr int kBinPitch = kSortWarps + 1;              // counters of a warp's lanes fall into different banks

struct GradArgs {
  const void* ids;
  int is64;
  int T;
  long long V, D;
  int bin_rows;
  int accumulate;
  float scale;
  const void* dy;
  long long dy_stride;
  void* dtable;
  long long dtable_stride;
  int dtable_esize;
  int* row_start;     // [V + 1] first sorted position of every row
  int2* sorted;       // [T] (token position, row) in sorted order
  int* status;
};

__device__ __forceinline__ int block_sum(int v, int* scratch) {   // scratch: 32 ints
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  int s = 0;
  for (int w = 0; w < kSortWarps; ++w) s += scratch[w];
  __syncthreads();
  return s;
}

__global__ void __launch_bounds__(kSortThreads) k_embed_sort(const GradArgs a) {
  extern __shared__ int smem[];
  int* cnt = smem;                                   // [bin_rows][kBinPitch]
  int* scratch = smem + a.bin_rows * kBinPitch;      // [32]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long lo = (long long)blockIdx.x * a.bin_rows;
  const int rows = (int)min((long long)a.bin_rows, a.V - lo);
  const long long part = ((a.T + kSortWarps - 1LL) / kSortWarps + 31) / 32 * 32;
  const long long t0 = warp * part, t1 = min((long long)a.T, t0 + part);

  for (int i = tid; i < rows * kBinPitch; i += kSortThreads) cnt[i] = 0;
  __syncthreads();
  int below = 0;
  for (long long t = t0; t < t1; t += 32) {
    const long long v = t + lane < t1 ? token_at(a.ids, a.is64, t + lane, a.V, a.status) : -1;
    below += v >= 0 && v < lo;
    const bool mine = v >= lo && v < lo + rows;
    if (!__ballot_sync(~0u, mine)) continue;
    const int r = mine ? (int)(v - lo) : -1;
    const unsigned same = __match_any_sync(~0u, r);
    if (mine && lane == __ffs(same) - 1) cnt[r * kBinPitch + warp] += __popc(same);
    __syncwarp();
  }
  const int first = block_sum(below, scratch);
  __syncthreads();

  // positions: exclusive prefix over the rows of the bin, then over the warps inside a row
  int total = 0;
  if (tid < rows)
    for (int w = 0; w < kSortWarps; ++w) total += cnt[tid * kBinPitch + w];
  int incl = total;
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(~0u, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) scratch[warp] = incl;
  __syncthreads();
  int at = first + incl - total;
  for (int w = 0; w < warp; ++w) at += scratch[w];
  if (tid < rows) {
    a.row_start[lo + tid] = at;
    if (lo + tid == a.V - 1) a.row_start[a.V] = at + total;
    int run = at;
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = cnt[tid * kBinPitch + w];
      cnt[tid * kBinPitch + w] = run;
      run += c;
    }
    cnt[tid * kBinPitch + kSortWarps] = total;       // the padding word keeps the row's count
  }
  __syncthreads();

  // rows that no token names: zeros
  if (!a.accumulate) {
    for (int r = warp; r < rows; r += kSortWarps) {
      if (cnt[r * kBinPitch + kSortWarps]) continue;
      char* p = static_cast<char*>(a.dtable) + (lo + r) * a.dtable_stride * a.dtable_esize;
      if (a.dtable_esize == 4) for (long long i = lane; i < a.D; i += 32) reinterpret_cast<float*>(p)[i] = 0.f;
      else for (long long i = lane; i < a.D; i += 32) reinterpret_cast<unsigned short*>(p)[i] = 0;
    }
  }

  for (long long t = t0; t < t1; t += 32) {
    const long long v = t + lane < t1 ? token_at(a.ids, a.is64, t + lane, a.V, a.status) : -1;
    const bool mine = v >= lo && v < lo + rows;
    if (!__ballot_sync(~0u, mine)) continue;
    const int r = mine ? (int)(v - lo) : -1;
    const unsigned same = __match_any_sync(~0u, r);
    const int leader = __ffs(same) - 1;
    int base = 0;
    if (mine && lane == leader) {
      base = cnt[r * kBinPitch + warp];
      cnt[r * kBinPitch + warp] = base + __popc(same);
    }
    base = __shfl_sync(~0u, base, leader);
    if (mine) a.sorted[base + __popc(same & ((1u << lane) - 1))] = make_int2((int)(t + lane), (int)v);
    __syncwarp();
  }
}

// ---- gradient, step 2: the sums -----------------------------------------------------------------
template <typename TIn, typename TOut>
__global__ void __launch_bounds__(256) k_embed_sum(const GradArgs a) {
  const int lane = threadIdx.x & 31;
  const long long v = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (v >= a.V) return;
  const int p0 = a.row_start[v], p1 = a.row_start[v + 1];
  if (p0 == p1) return;
  for (long long d = lane; d < a.D; d += 32) {
    float s = 0.f;
    for (int p = p0; p < p1; ++p) s += to_f32(static_cast<const TIn*>(a.dy)[a.sorted[p].x * a.dy_stride + d]);
    TOut* out = static_cast<TOut*>(a.dtable) + v * a.dtable_stride + d;
    *out = from_f32<TOut>(a.accumulate ? to_f32(*out) + a.scale * s : a.scale * s);
  }
}

uint64_t up16(uint64_t n) { return (n + 15) / 16 * 16; }

}  // namespace

namespace cocodc_lm_impl {
bool embed_prepare() {
  return cudaFuncSetAttribute(k_embed_sort, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (kMaxBinRows * kBinPitch + 32) * 4) == cudaSuccess;
}
}  // namespace cocodc_lm_impl

extern "C" {

cocodc_status cocodc_lm_embed(cocodc_lm* lm, const void* table, int32_t table_type, int64_t table_stride, int64_t V,
                              int64_t D, const void* ids, int32_t ids_type, int64_t T, float scale, void* y,
                              int32_t y_type, int64_t y_stride, void* stream) {
  if (!lm || !sane(V) || !sane(D) || !sane(T) || V < 1 || D < 1 || !known_type(table_type) || !known_type(y_type) ||
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
  const long long blocks = (T * D + 255) / 256;
  with_type(table_type, [&](auto in) {
    return with_type(y_type, [&](auto out) {
      using TIn = decltype(in);
      using TOut = decltype(out);
      k_embed<TIn, TOut><<<(unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)), 256, 0, st>>>(
          static_cast<const TIn*>(table), table_stride, V, D, ids, ids_type == COCODC_I64, T, scale,
          static_cast<TOut*>(y), y_stride, lm->d_status);
      return true;
    });
  });
  return launched(lm);
}

uint64_t cocodc_lm_embed_grad_workspace(int64_t V, int64_t D, int64_t T) {
  if (!sane(V) || !sane(D) || !sane(T)) return 0;
  return up16((uint64_t)(V + 1) * sizeof(int)) + up16((uint64_t)T * sizeof(int2));
}

cocodc_status cocodc_lm_embed_grad(cocodc_lm* lm, const void* dy, int32_t dy_type, int64_t dy_stride, const void* ids,
                                   int32_t ids_type, int64_t T, int64_t V, int64_t D, float scale, int32_t accumulate,
                                   void* dtable, int32_t dtable_type, int64_t dtable_stride, void* workspace,
                                   uint64_t workspace_bytes, void* stream) {
  if (!lm || !sane(V) || !sane(D) || !sane(T) || V < 1 || D < 1 || T > INT32_MAX || V >= INT32_MAX || !dtable ||
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
  a.row_start = static_cast<int*>(workspace);
  a.sorted = reinterpret_cast<int2*>(static_cast<char*>(workspace) + up16((uint64_t)(V + 1) * sizeof(int)));
  a.status = lm->d_status;
  const long long per_sm = (V + lm->sm_count - 1) / lm->sm_count;
  a.bin_rows = (int)(per_sm < kMaxBinRows ? per_sm : kMaxBinRows);
  const unsigned bins = (unsigned)((V + a.bin_rows - 1) / a.bin_rows);
  k_embed_sort<<<bins, kSortThreads, (a.bin_rows * kBinPitch + 32) * 4, st>>>(a);
  if (T > 0)
    with_type(dy_type, [&](auto in) {
      return with_type(dtable_type, [&](auto out) {
        k_embed_sum<decltype(in), decltype(out)><<<(unsigned)((V + 7) / 8), 256, 0, st>>>(a);
        return true;
      });
    });
  return launched(lm, T > 0 ? 2 : 1);
}

}  // extern "C"
