// The output head with its loss, without keeping the logits, and its gradient (include/cocodc_lm.h).

#include "lm_head_tc.cuh"
#include "lm_plain.cuh"

#include <type_traits>

using namespace cocodc_lm_impl;

namespace {

constexpr int kSms = 148;                            // of a B200 (workspace sizes are asked for without a handle)

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }

// Columns of a tile of logits: multiples of `step` up to 256.  Tiles times their width in rounds of one per SM, plus what a tile
// costs beside its products, come out smallest.
int tile_width(int64_t T, int64_t V, int step) {
  const int64_t rows = up(T, kBM);
  int best = 256;
  int64_t least = INT64_MAX;
  for (int w = 256; w >= step; w -= step) {
    const int64_t cost = up(rows * up(V, w), kSms) * (w + 24);
    if (cost < least) {
      least = cost;
      best = w;
    }
  }
  return best;
}
int strip_width(int64_t T, int64_t V) { return tile_width(T, V, 16); }

// Any strides: 64 rows and a strip for each block, in pieces of 64 columns.
template <typename E>
__global__ void __launch_bounds__(256) k_head_plain(const HeadArgs a, const Operand<E> x, const Operand<E> w, long long D) {
  wait_for_previous();
  may_follow();
  __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
  const long long strip = blockIdx.x % a.strips, t0 = blockIdx.x / a.strips * kTile, v0 = strip * a.width, v1 = min(a.V, v0 + a.width);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  Stats own[4];
  long long target[4];
  for (int i = 0; i < 4; ++i) {
    own[i] = Stats{-INFINITY, 0.f};
    const long long t = t0 + ty * 4 + i;
    target[i] = a.targets && t < a.T ? raw_target(a.targets, a.targets64, t) : -1;
  }
  for (long long v = v0; v < v1; v += kTile) {
    float c[4][4] = {};
    accumulate(c, x, w, t0, a.T, v, v1, D, sa, sb);
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const long long col = v + tx * 4 + j, t = t0 + ty * 4 + i;
        if (col >= v1 || t >= a.T) continue;
        const float z = c[i][j] * a.scale2;
        const float m = fmaxf(own[i].m, z), k = shift_of(m);
        own[i] = Stats{m, own[i].s * fast_exp2(own[i].m - k) + fast_exp2(z - k)};
        if (col == target[i]) a.picked[t] = z;
      }
  }
  for (int i = 0; i < 4; ++i) {
    for (int o = 8; o; o >>= 1) {
      const float m = __shfl_xor_sync(~0u, own[i].m, o), s = __shfl_xor_sync(~0u, own[i].s, o);
      own[i] = join(own[i], Stats{m, s});
    }
    const long long t = t0 + ty * 4 + i;
    if (tx == 0 && t < a.T) a.stats[strip * a.T + t] = make_float2(own[i].m, own[i].s);
  }
}

// The strips of a row joined: eight rows a block, 32 threads each, that read by eight rows at a time (two times 197 strips of 1333 rows took 21 us with
// eight threads a row); few rows: one a block, all its threads, so that one round of loads does.
__device__ __forceinline__ Stats join_warp(Stats v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const float m = __shfl_xor_sync(~0u, v.m, o), s = __shfl_xor_sync(~0u, v.s, o);
    v = join(v, Stats{m, s});
  }
  return v;
}
template <int ROWS> __global__ void __launch_bounds__(256) k_head_join(const HeadArgs a, float* logp, float* lse, int* status) {
  wait_for_previous();
  may_follow();
  constexpr int kParts = 256 / ROWS;
  __shared__ Stats cell[8][33];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const long long t = (long long)blockIdx.x * ROWS + threadIdx.x % ROWS, row = (long long)blockIdx.x * ROWS + (ROWS == 1 ? 0 : warp);
  long long y = -1;
  float picked = 0.f;
  if (lane == 0 && row < a.T && (ROWS > 1 || warp == 0)) {            // on its way beside the strips
    if (logp) y = token_at(a.targets, a.targets64, row, a.V, status);
    if (y >= 0) picked = a.picked[row];
  }
  Stats all{-INFINITY, 0.f};
  if (t < a.T) {
    for (long long i = threadIdx.x / ROWS; i < a.strips; i += 8 * kParts) {
      float2 v[8];                                                    // together on their way
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = i + k * kParts < a.strips ? a.stats[(i + k * kParts) * a.T + t] : make_float2(-INFINITY, 0.f);
      float m = all.m;
#pragma unroll
      for (int k = 0; k < 8; ++k) m = fmaxf(m, v[k].x);
      const float shift = shift_of(m);
      float s = all.s * fast_exp2(all.m - shift);
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k].y * fast_exp2(v[k].x - shift);
      all = Stats{m, s};
    }
  }
  if (ROWS == 1) {
    all = join_warp(all);
    if (lane == 0) cell[0][warp] = all;
    __syncthreads();
    if (warp) return;
    all = lane < 8 ? cell[0][lane] : Stats{-INFINITY, 0.f};
  } else {
    cell[threadIdx.x % ROWS][threadIdx.x / ROWS] = all;
    __syncthreads();
    all = cell[warp][lane];
  }
  all = join_warp(all);
  if (lane || row >= a.T) return;
  const float log2sum = shift_of(all.m) + log2f(all.s);
  if (lse) lse[row] = log2sum * kLn2;
  if (logp) logp[row] = y < 0 ? 0.f : (log2sum == -INFINITY ? -INFINITY : (picked - log2sum) * kLn2);
}

// ---- gradient -------------------------------------------------------------------------------------
// The power of two that half-precision dz is taken at: factor[0], and its inverse.
__global__ void __launch_bounds__(1024) k_head_factor(const HeadArgs a, const float* dlogp, const float* dlse, float* factor) {
  wait_for_previous();
  may_follow();
  __shared__ unsigned cell[32];
  unsigned most = 0;
  for (long long t = threadIdx.x; t < a.T; t += 1024) {
    float v = dlse ? fabsf(dlse[t]) : 0.f;
    if (dlogp && raw_target(a.targets, a.targets64, t) >= 0) v += fabsf(dlogp[t]);
    if (v < INFINITY) most = max(most, __float_as_uint(v));         // not NaN either
  }
  most = __reduce_max_sync(~0u, most);
  if (threadIdx.x % 32 == 0) cell[threadIdx.x / 32] = most;
  __syncthreads();
  if (threadIdx.x) return;
  for (int i = 1; i < 32; ++i) most = max(most, cell[i]);
  int e = most ? 9 - ilogbf(__uint_as_float(most)) : 0;
  e = max(-120, min(120, e));
  factor[0] = ldexpf(1.f, e);
  factor[1] = ldexpf(1.f, -e);
}

template <typename E>
__global__ void __launch_bounds__(256) k_head_dz_plain(const DzArgs a, const Operand<E> x, const Operand<E> w, long long D) {
  wait_for_previous();
  may_follow();
  __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
  const long long tiles = (a.v1 - a.v0 + kTile - 1) / kTile;
  const long long v = a.v0 + blockIdx.x % tiles * kTile, t0 = blockIdx.x / tiles * kTile;
  float c[4][4] = {};
  accumulate(c, x, w, t0, a.T, v, a.v1, D, sa, sb);
  for (int i = 0; i < 4; ++i) {
    const long long t = t0 + threadIdx.x / 16 * 4 + i;
    if (t >= a.T) continue;
    const RowOf r = row_of(a, t);
    for (int j = 0; j < 4; ++j) {
      const long long col = v + threadIdx.x % 16 * 4 + j;
      if (col < a.v1) static_cast<E*>(a.dz)[t * a.pitch + col - a.v0] = from_f32<E>(dz_of(r, c[i][j] * a.scale2, col == r.y));
    }
  }
}

template <typename E> __device__ __forceinline__ void deliver(const Out& o, long long r, long long c, long long cols, float v) {
  if (o.sums && o.add) v += o.sums[r * cols + c];
  if (o.sums && !o.last) {
    o.sums[r * cols + c] = v;
    return;
  }
  v = Back(o)(v);
  if (o.type == COCODC_F32) {
    float* p = static_cast<float*>(o.out) + r * o.ld + c;
    *p = o.accumulate ? *p + v : v;
  } else {
    E* p = static_cast<E*>(o.out) + r * o.ld + c;
    *p = from_f32<E>(o.accumulate ? to_f32(*p) + v : v);
  }
}

template <typename E>
__global__ void __launch_bounds__(256) k_head_product_plain(const Operand<E> A, const Operand<E> B, long long M, long long N, long long K, const Out o) {
  wait_for_previous();
  may_follow();
  __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
  const long long tiles = (N + kTile - 1) / kTile;
  const long long n0 = blockIdx.x % tiles * kTile, m0 = blockIdx.x / tiles * kTile;
  float c[4][4] = {};
  accumulate(c, A, B, m0, M, n0, N, K, sa, sb);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const long long m = m0 + threadIdx.x / 16 * 4 + i, n = n0 + threadIdx.x % 16 * 4 + j;
      if (m < M && n < N) deliver<E>(o, m, n, N, c[i][j]);
    }
}

template <typename O> __global__ void __launch_bounds__(256) k_head_zero(O* out, long long ld, long long rows, long long cols) {
  wait_for_previous();
  may_follow();
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (long long)gridDim.x * 256)
    out[i / cols * ld + i % cols] = from_f32<O>(0.f);
}

// Columns of a piece of the vocabulary in the gradient: dz of a piece takes at most kPieceBytes, as long as that leaves 1024 columns.
constexpr int64_t kPieceBytes = int64_t(1) << 28, kLeastPiece = 1024;
int64_t piece_width(int64_t T, int64_t V) {
  int64_t w = T > 0 ? kPieceBytes / 2 / T / 256 * 256 : V;
  if (w < kLeastPiece) w = kLeastPiece;
  if (w >= V) return up(V, 64) * 64;
  const int64_t pieces = up(V, w);
  return up(up(V, pieces), 256) * 256;
}

template <typename F> cocodc_status with_half(int32_t type, F&& f) { return type == COCODC_BF16 ? f(__nv_bfloat16()) : f(__half()); }

bool sizes_ok(int64_t T, int64_t D, int64_t V) {
  const int64_t most = int64_t(1) << 48;             // elements of a matrix: byte counts stay far inside 64 bits
  return T >= 0 && T <= INT32_MAX && D >= 1 && D <= INT32_MAX && V >= 1 && V <= (int64_t(1) << 30) && T <= most / D && V <= most / D;
}
// a grid of tiles of `t` x `n` in one dimension
bool grid_of(int64_t rows, int64_t t, int64_t cols, int64_t n, unsigned* out) {
  const int64_t blocks = up(rows, t) * up(cols, n);
  *out = (unsigned)blocks;
  return blocks <= INT32_MAX;
}

// Parts of dx's contraction where its tiles are few: as many as there are SMs for each tile, with at least 16 k-blocks to a part.
int dx_width(int64_t D) { return D >= 256 ? 256 : (int)up(D, 64) * 64; }
int dx_parts(int64_t T, int64_t D, int64_t width) {
  if (T < 1) return 1;
  const int64_t tiles = up(T, kBM) * up(D, dx_width(D)), parts = kSms / tiles, most = up(width, kBK) / 16;
  const int64_t p = parts < most ? parts : most;
  return p < 2 ? 1 : (int)p;
}

struct GradLayout { uint64_t sums, dz, bytes; int64_t width; };
GradLayout grad_layout(int64_t T, int64_t D, int64_t V) {
  GradLayout l{};
  l.width = piece_width(T, V);
  const int parts = dx_parts(T, D, l.width);
  l.sums = 256;
  // whole tiles of 128 x dx_width for each part; the kernels for any strides need T x D of it
  l.dz = l.sums + (l.width < V || parts > 1 ? (uint64_t)parts * (uint64_t)up(T, kBM) * (uint64_t)up(D, dx_width(D)) * kBM * dx_width(D) * 4 : 0);
  l.bytes = l.dz + (uint64_t)T * (uint64_t)l.width * 2;
  return l;
}

// ---- tensor-core path: host side ----------------------------------------------------------------
bool map_f32(CUtensorMap* map, const void* p, int64_t stride, int64_t rows, int64_t cols) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 4};
  const cuuint32_t box[2] = {32, 32}, steps[2] = {1, 1};
  return g_encode.load()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<void*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The same memory as slabs of 64 columns, `count` of which (64 rows each) a copy brings at once: an MN-major operand of k-blocks of 64 in one
// copy instead of two or four.  For rows of whole slabs.
template <typename E> bool map_slabs(CUtensorMap* map, const void* p, int64_t stride, int64_t rows, int64_t cols, int count) {
  const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(cols / 64)}, strides[2] = {(cuuint64_t)stride * 2, 128};
  const cuuint32_t box[3] = {64, (cuuint32_t)kBK, (cuuint32_t)count}, steps[3] = {1, 1, 1};
  return g_encode.load()(map, IsBf16<E>::v ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(p), dims,
                         strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
int a_rows(int64_t T) { return T >= kBM ? kBM : (int)up(T, 8) * 8; }

template <typename E, int MODE> cocodc_status run_tc(cocodc_lm* lm, HeadTc& c, cudaStream_t st) {
  const long long tiles = MODE == HEAD_PRODUCTS ? (long long)c.job[0].tiles + c.job[1].tiles : (long long)c.m_tiles * c.n_tiles;
  if (tiles > INT32_MAX / 2) return COCODC_ERR_INVALID_ARG;
  c.status = lm->d_status;
  return start(lm, k_head_tc<E, MODE>, (unsigned)(tiles < lm->sm_count ? tiles : lm->sm_count), kHeadThreads, kHeadSmem, st, 1, c);
}
// A tile of logits: x [T][D] by rows of the table.
template <typename E>
bool logit_maps(HeadTc* c, const void* x, int64_t x_stride, const void* table, int64_t table_stride, int64_t T, int64_t D, int64_t V, int width) {
  c->width = width;
  c->a_bytes = a_rows(T) * kBK * 2;
  c->m_tiles = (int)up(T, kBM);
  c->k_blocks = (int)up(D, kBK);
  return map_of<E>(&c->a[0], x, x_stride, T, D, a_rows(T)) && map_of<E>(&c->b[0], table, table_stride, V, D, width);
}

}  // namespace

namespace cocodc_lm_impl {
bool head_prepare() {
  bool ok = true;
  const auto allow = [&](auto kernel) {
    ok = ok && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeadSmem) == cudaSuccess;
  };
  const auto allow_type = [&](auto e) {
    using E = decltype(e);
    allow(k_head_tc<E, HEAD_STATS>);
    allow(k_head_tc<E, HEAD_LONG>);
    allow(k_head_tc<E, HEAD_DZ>);
    allow(k_head_tc<E, HEAD_PRODUCTS>);
  };
  allow_type(__nv_bfloat16());
  allow_type(__half());
  return ok;
}
}  // namespace cocodc_lm_impl

extern "C" {

uint64_t cocodc_lm_head_workspace(int64_t T, int64_t D, int64_t V) {
  if (!sizes_ok(T, D, V)) return 0;
  return 16 + (uint64_t)T * 4 + 16 + (uint64_t)up(V, strip_width(T, V)) * 2 * (uint64_t)T * sizeof(float2);
}

cocodc_status cocodc_lm_head(cocodc_lm* lm, int32_t type, const void* x, int64_t x_stride, const void* table, int64_t table_stride,
                             int64_t T, int64_t D, int64_t V, const void* targets, int32_t targets_type, float scale,
                             float* logp, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!lm || (type != COCODC_BF16 && type != COCODC_F16) || !sizes_ok(T, D, V) || x_stride < D || !sane(x_stride) || table_stride < D ||
      !sane(table_stride) || !(scale > 0.f && scale <= kMostScale) || (targets && targets_type != COCODC_I32 && targets_type != COCODC_I64))
    return COCODC_ERR_INVALID_ARG;
  if (!logp != !targets || (!logp && !lse)) return T == 0 ? COCODC_OK : COCODC_ERR_INVALID_ARG;
  if (T == 0) return COCODC_OK;
  unsigned grid;                                      // of k_head_plain; k_head_tc has as many tiles at most
  if (!x || !table || !workspace || workspace_bytes < cocodc_lm_head_workspace(T, D, V) || !grid_of(T, kTile, V, strip_width(T, V), &grid))
    return COCODC_ERR_INVALID_ARG;
  const int ib = targets ? index_bytes(targets_type) : 4;
  if (!on_boundary(x, 2) || !on_boundary(table, 2) || !on_boundary(targets, ib) || !on_boundary(logp, 4) || !on_boundary(lse, 4) ||
      !on_boundary(workspace, 16))
    return COCODC_ERR_ALIGNMENT;
  const Span in[3] = {span(x, T, x_stride, D, 2), span(table, V, table_stride, D, 2), span(targets, 1, T, T, ib)};
  const Span out[3] = {span(logp, 1, T, T, 4), span(lse, 1, T, T, 4), span(workspace, 1, (int64_t)workspace_bytes, (int64_t)workspace_bytes, 1)};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 3; ++j)
      if (meet(out[i], in[j])) return COCODC_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return COCODC_ERR_ALIAS;
  }
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  HeadArgs a{};
  a.T = T;
  a.V = V;
  a.width = strip_width(T, V);
  a.strips = up(V, a.width);                          // parts of a row's statistics: one for each strip, on the tensor cores two
  a.scale2 = scale * kLog2e;
  a.targets = targets;
  a.targets64 = targets_type == COCODC_I64;
  a.picked = static_cast<float*>(workspace);
  a.stats = reinterpret_cast<float2*>(static_cast<char*>(workspace) + up(T, 4) * 16);
  const bool tensor = rows_aligned(x, x_stride, 2) && rows_aligned(table, table_stride, 2);
  const cocodc_status status = with_half(type, [&](auto e) {
    using E = decltype(e);
    if (tensor) {
      HeadTc c{};
      c.h = a;
      c.n_tiles = (int)a.strips;
      c.parts = (int)up(up(D, kBK), kPartBlocks);
      a.strips *= 2;
      if (!logit_maps<E>(&c, x, x_stride, table, table_stride, T, D, V, a.width)) return COCODC_ERR_CUDA;
      return c.k_blocks >= kLongBlocks ? run_tc<E, HEAD_LONG>(lm, c, st) : run_tc<E, HEAD_STATS>(lm, c, st);
    }
    const Operand<E> xo{static_cast<const E*>(x), x_stride, 1}, wo{static_cast<const E*>(table), table_stride, 1};
    return start(lm, k_head_plain<E>, grid, 256, 0, st, 1, a, xo, wo, (long long)D);
  });
  if (status != COCODC_OK) return status;
  return T <= 2 * kSms ? start(lm, k_head_join<1>, (unsigned)T, 256, 0, st, 1, a, logp, lse, lm->d_status)
                       : start(lm, k_head_join<8>, (unsigned)up(T, 8), 256, 0, st, 1, a, logp, lse, lm->d_status);
}

uint64_t cocodc_lm_head_grad_workspace(int64_t T, int64_t D, int64_t V) { return sizes_ok(T, D, V) ? grad_layout(T, D, V).bytes : 0; }

cocodc_status cocodc_lm_head_grad(cocodc_lm* lm, int32_t type, const void* x, int64_t x_stride, const void* table,
                                  int64_t table_stride, int64_t T, int64_t D, int64_t V, const void* targets, int32_t targets_type,
                                  float scale, const float* lse, const float* dlogp, const float* dlse, void* dx, int64_t dx_stride,
                                  void* dtable, int32_t dtable_type, int64_t dtable_stride, int32_t accumulate, void* workspace,
                                  uint64_t workspace_bytes, void* stream) {
  if (!lm || (type != COCODC_BF16 && type != COCODC_F16) || !sizes_ok(T, D, V) || x_stride < D || !sane(x_stride) || table_stride < D ||
      !sane(table_stride) || !(scale > 0.f && scale <= kMostScale) || (targets && targets_type != COCODC_I32 && targets_type != COCODC_I64) ||
      (dx && (dx_stride < D || !sane(dx_stride))) ||
      (dtable && (dtable_stride < D || !sane(dtable_stride) || (dtable_type != type && dtable_type != COCODC_F32))))
    return COCODC_ERR_INVALID_ARG;
  if (!dx && !dtable) return T == 0 ? COCODC_OK : COCODC_ERR_INVALID_ARG;
  if (T > 0 && (!x || !table || !lse || !dlogp != !targets || (!dlogp && !dlse) || !workspace ||
                workspace_bytes < cocodc_lm_head_grad_workspace(T, D, V)))
    return COCODC_ERR_INVALID_ARG;
  // grids of the kernels for any strides, tiles of the tensor-core kernel's products
  const GradLayout l = T > 0 ? grad_layout(T, D, V) : GradLayout{};
  unsigned g1 = 0, g2 = 0, g3 = 0;
  if (T > 0 && (!grid_of(T, kTile, l.width, kTile, &g1) || !grid_of(T, kTile, D, kTile, &g2) || !grid_of(l.width, kTile, D, kTile, &g3) ||
                up(T, kBM) * up(D, 64) > INT32_MAX / kSms || up(l.width, kBM) * up(D, 64) > INT32_MAX / 4))
    return COCODC_ERR_INVALID_ARG;
  const int ib = targets ? index_bytes(targets_type) : 4, wb = dtable_type == COCODC_F32 ? 4 : 2;
  if (!on_boundary(x, 2) || !on_boundary(table, 2) || !on_boundary(dx, 2) || !on_boundary(dtable, wb) || !on_boundary(targets, ib) ||
      !on_boundary(lse, 4) || !on_boundary(dlogp, 4) || !on_boundary(dlse, 4) || !on_boundary(workspace, 16))
    return COCODC_ERR_ALIGNMENT;
  const Span in[6] = {span(x, T, x_stride, D, 2), span(table, V, table_stride, D, 2), span(targets, 1, T, T, ib), span(lse, 1, T, T, 4),
                      span(dlogp, 1, T, T, 4), span(dlse, 1, T, T, 4)};
  const Span out[3] = {span(dx, T, dx_stride, D, 2), span(dtable, V, dtable_stride, D, wb),
                       T > 0 ? span(workspace, 1, (int64_t)workspace_bytes, (int64_t)workspace_bytes, 1) : Span{0, 0, 0, 0}};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 6; ++j)
      if (meet(out[i], in[j])) return COCODC_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return COCODC_ERR_ALIAS;
  }
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_half(type, [&](auto e) {
    using E = decltype(e);
    if (T == 0) {
      if (!dtable || accumulate) return COCODC_OK;
      const unsigned blocks = (unsigned)(up(V * D, 1024) < 65535 ? up(V * D, 1024) : 65535);
      return dtable_type == COCODC_F32
                 ? start(lm, k_head_zero<float>, blocks, 256, 0, st, 1, static_cast<float*>(dtable), (long long)dtable_stride, (long long)V, (long long)D)
                 : start(lm, k_head_zero<E>, blocks, 256, 0, st, 1, static_cast<E*>(dtable), (long long)dtable_stride, (long long)V, (long long)D);
    }
    char* ws = static_cast<char*>(workspace);
    DzArgs d{};
    d.T = T;
    d.V = V;
    d.scale2 = scale * kLog2e;
    d.targets = targets;
    d.targets64 = targets_type == COCODC_I64;
    d.lse = lse;
    d.dlogp = dlogp;
    d.dlse = dlse;
    d.dz = ws + l.dz;
    d.pitch = l.width;
    d.status = lm->d_status;
    if (type == COCODC_F16) {
      d.factor = reinterpret_cast<float*>(ws);
      HeadArgs h{};
      h.T = T;
      h.V = V;
      h.targets = targets;
      h.targets64 = d.targets64;
      const cocodc_status s = start(lm, k_head_factor, 1, 1024, 0, st, 1, h, dlogp, dlse, reinterpret_cast<float*>(ws));
      if (s != COCODC_OK) return s;
    }
    const bool tensor = rows_aligned(x, x_stride, 2) && rows_aligned(table, table_stride, 2) && (!dx || rows_aligned(dx, dx_stride, 2)) &&
                        (!dtable || rows_aligned(dtable, dtable_stride, wb));
    const int parts = tensor ? dx_parts(T, D, l.width) : 1;
    const E *xe = static_cast<const E*>(x), *we = static_cast<const E*>(table), *dz = reinterpret_cast<const E*>(ws + l.dz);
    for (int64_t v0 = 0; v0 < V; v0 += l.width) {
      d.v0 = v0;
      d.v1 = v0 + l.width < V ? v0 + l.width : V;
      const long long w = d.v1 - v0;
      const Out ow{static_cast<char*>(dtable) + v0 * dtable_stride * wb, dtable_type, accumulate ? 1 : 0, dtable_stride, nullptr, 0, 1, d.factor, scale};
      const Out ox{dx, type, 0, dx_stride, l.width < V || parts > 1 ? reinterpret_cast<float*>(ws + l.sums) : nullptr, v0 > 0,
                   d.v1 == V && parts == 1, d.factor, scale};
      if (tensor) {
        HeadTc c{};
        c.d = d;
        c.first_row = v0;
        c.counter = reinterpret_cast<int*>(ws + 64);
        const int width = tile_width(T, w, 64);
        c.n_tiles = (int)up(w, width);
        if (!logit_maps<E>(&c, x, x_stride, table, table_stride, T, D, V, width) || !map_of<E>(&c.c[0], d.dz, d.pitch, T, w, 32)) return COCODC_ERR_CUDA;
        cocodc_status s = run_tc<E, HEAD_DZ>(lm, c, st);
        if (s != COCODC_OK) return s;
        c.width = dx_width(D);
        const int n_tiles = (int)up(D, c.width);
        c.slabs = D % 64 == 0 ? c.width / 64 : 1;
        const auto map_b = [&](CUtensorMap* map, const void* p, int64_t stride, int64_t rows) {
          return c.slabs > 1 ? map_slabs<E>(map, p, stride, rows, D, c.slabs) : map_of<E>(map, p, stride, rows, D, kBK);
        };
        if (dtable) {
          HeadJob& j = c.job[0];
          j = HeadJob{(int)up(w, kBM), n_tiles, (int)up(T, kBK), 1, (int)up(w, kBM) * n_tiles, (int)w, (int)D, kABytes, ow};
          if (!map_slabs<E>(&c.a[0], d.dz, d.pitch, T, up(w, 64) * 64, kBM / 64) || !map_b(&c.b[0], x, x_stride, T) ||
              !(wb == 4 ? map_f32(&c.c[0], ow.out, dtable_stride, w, D) : map_of<E>(&c.c[0], ow.out, dtable_stride, w, D, 32)))
            return COCODC_ERR_CUDA;
        }
        if (dx) {
          HeadJob& j = c.job[1];
          const int tiles = (int)up(T, kBM) * n_tiles;
          j = HeadJob{(int)up(T, kBM), n_tiles, (int)up(w, kBK), parts, tiles * parts, (int)T, (int)D, c.a_bytes, ox};
          if (!map_of<E>(&c.a[1], d.dz, d.pitch, T, w, a_rows(T)) || !map_b(&c.b[1], table, table_stride, V) ||
              !map_of<E>(&c.c[1], dx, dx_stride, T, D, 32))
            return COCODC_ERR_CUDA;
        }
        c.first = c.job[1].tiles && (!c.job[0].tiles || (c.job[1].k_blocks + parts - 1) / parts > c.job[0].k_blocks) ? 1 : 0;
        s = run_tc<E, HEAD_PRODUCTS>(lm, c, st);
        if (s != COCODC_OK) return s;
        if (dx && parts > 1 && d.v1 == V)
          s = start(lm, k_head_add<E>, dim3((unsigned)(c.job[1].m_tiles * n_tiles * (kBM / 8)), (unsigned)up(c.width, 128)), 256, 0, st, 1, c);
        if (s != COCODC_OK) return s;
        continue;
      }
      grid_of(T, kTile, w, kTile, &g1);
      cocodc_status s = start(lm, k_head_dz_plain<E>, g1, 256, 0, st, 1, d, Operand<E>{xe, x_stride, 1}, Operand<E>{we, table_stride, 1}, (long long)D);
      if (s != COCODC_OK) return s;
      if (dtable) {
        grid_of(w, kTile, D, kTile, &g3);
        s = start(lm, k_head_product_plain<E>, g3, 256, 0, st, 1, Operand<E>{dz, 1, d.pitch}, Operand<E>{xe, 1, x_stride}, w, (long long)D, (long long)T, ow);
        if (s != COCODC_OK) return s;
      }
      if (dx) {
        s = start(lm, k_head_product_plain<E>, g2, 256, 0, st, 1, Operand<E>{dz, d.pitch, 1}, Operand<E>{we + v0 * table_stride, 1, table_stride},
                  (long long)T, (long long)D, w, ox);
        if (s != COCODC_OK) return s;
      }
    }
    return COCODC_OK;
  });
}

}  // extern "C"
