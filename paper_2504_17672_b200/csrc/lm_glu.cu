// The gated feed-forward block h = act(x Wg^T) * (x Wu^T) and its gradient (include/cocodc_lm.h).

#include "lm_glu_tc.cuh"
#include "lm_plain.cuh"

using namespace cocodc_lm_impl;

namespace cocodc_lm_impl {

constexpr float kLog2e = 1.4426950408889634f;

// act(g) = g * s(g) for both activations: s is the logistic function of g (SILU) or of 2z, z = sqrt(2/pi) (g + 0.044715 g^3)
// (GELU: (1 + tanh z) / 2 is that function of 2z).  The cubic is taken at g clamped to [-30, 30], where s has long
// been exactly 0 or 1, so that a large g cannot turn it into Inf (and its slope into 0 * Inf).
struct Activation { float value, slope; };
template <int ACT> __device__ __forceinline__ Activation activate(float g) {
  float z = g, dz = 1.f;
  if (ACT == COCODC_ACT_GELU) {
    const float k = 2.f * 0.7978845608028654f, b = 0.044715f;
    const float q = fminf(fmaxf(g, -30.f), 30.f);
    z = k * (q + b * q * q * q);
    dz = k * (1.f + 3.f * b * q * q);
  }
  const float s = __fdividef(1.f, 1.f + fast_exp2(-z * kLog2e));
  return Activation{g * s, s + g * (s * (1.f - s)) * dz};
}
template <int ACT> __device__ __forceinline__ float act_value(float g) { return activate<ACT>(g).value; }

}  // namespace cocodc_lm_impl

namespace {

// ---- products of any strides and sizes (lm_plain.cuh) --------------------------------------------------
template <typename T> struct PlainArgs {
  Operand<T> a[2], b[2];
  long long M, N, K;
  T* out[3];              // forward: h, gate, up; otherwise out[blockIdx.z]
  long long ld, ld_gu;
};

template <typename T, int ACT>
__global__ void __launch_bounds__(256) k_glu_plain(const PlainArgs<T> p) {
  wait_for_previous();
  may_follow();
  __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
  const long long m0 = (long long)blockIdx.x * kTile, n0 = (long long)blockIdx.y * kTile;
  float g[4][4] = {}, u[4][4] = {};
  accumulate(g, p.a[0], p.b[0], m0, p.M, n0, p.N, p.K, sa, sb);
  accumulate(u, p.a[0], p.b[1], m0, p.M, n0, p.N, p.K, sa, sb);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const long long m = m0 + threadIdx.x / 16 * 4 + i, n = n0 + threadIdx.x % 16 * 4 + j;
      if (m >= p.M || n >= p.N) continue;
      p.out[0][m * p.ld + n] = from_f32<T>(activate<ACT>(g[i][j]).value * u[i][j]);
      if (p.out[1]) {
        p.out[1][m * p.ld_gu + n] = from_f32<T>(g[i][j]);
        p.out[2][m * p.ld_gu + n] = from_f32<T>(u[i][j]);
      }
    }
}

// SUM: one output, both sources added (dx); otherwise source and output z (dwg, dwu)
template <typename T, bool SUM>
__global__ void __launch_bounds__(256) k_product_plain(const PlainArgs<T> p) {
  wait_for_previous();
  may_follow();
  __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
  const long long m0 = (long long)blockIdx.x * kTile, n0 = (long long)blockIdx.y * kTile;
  const int z = blockIdx.z;
  float c[4][4] = {};
  accumulate(c, p.a[z], p.b[z], m0, p.M, n0, p.N, p.K, sa, sb);
  if (SUM) accumulate(c, p.a[1], p.b[1], m0, p.M, n0, p.N, p.K, sa, sb);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const long long m = m0 + threadIdx.x / 16 * 4 + i, n = n0 + threadIdx.x % 16 * 4 + j;
      if (m < p.M && n < p.N) p.out[z][m * p.ld + n] = from_f32<T>(c[i][j]);
    }
}

// ---- few tokens -----------------------------------------------------------------------------------
// Bound by reading the weights once.  A CTA takes 8 columns of the output: the 16 rows of an mma.sync tile are 8 rows of
// Wg and the same 8 of Wu, so that a thread's accumulators hold gate and up of the same elements.  The warps share the
// contraction in blocks of 64 k, and every lane loads 32 consecutive bytes of a row of each matrix per block, straight
// into fragments: the k's of a lane's fragment places are permuted, the same way for weights and tokens, which a
// contraction does not notice.  The warps' sums meet in shared memory in fixed order.  TILES: groups of eight tokens.
// Four CTAs per SM (64 registers) for one group: 11.2 -> 9.6 us at 2048 x 5632, 36.9 -> 32.6 us at 4096 x 11008 (9.1 and 32 now, with early starts); two groups
// then spill, and run three.
constexpr int kFewWarps = 8;
// Up to 8 tokens always; up to 32 where tokens (in eights) x D x F stay below kFewProduct, us here / on tcgen05 tiles: 16 tokens,
// 2048 x 5632: 11.7 / 14.5, 3200 x 8640: 26.6 / 23.1; 32 tokens, 1024 x 2816: 6.6 / 9.1, 2048 x 5632: 16.3 / 14.9.
constexpr long long kFewProduct = 190 * 1000 * 1000;
bool few_tokens(int64_t T, int64_t D, int64_t F) {
  const int64_t rows = T <= 8 ? 8 : T <= 16 ? 16 : 32;
  return T <= 8 || (T <= 32 && D * F <= kFewProduct / rows);
}

template <typename E> __device__ __forceinline__ void mma16816(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3,
                                                               unsigned b0, unsigned b1);
template <> __device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], unsigned a0, unsigned a1, unsigned a2,
                                                                    unsigned a3, unsigned b0, unsigned b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16816<__half>(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3,
                                                             unsigned b0, unsigned b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// weights: read once, not kept in L1
__device__ __forceinline__ uint4 load_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// 8 elements of a row, zeros from the n-th on
template <typename E> __device__ __forceinline__ uint4 load_end(const E* p, int n) {
  alignas(16) E v[8];
  for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : from_f32<E>(0.f);
  return *reinterpret_cast<const uint4*>(v);
}

template <typename E> struct FewArgs {
  const E *x, *wg, *wu;
  long long x_stride, w_stride;
  int T, D, F;
  E *h, *gate, *up;
  long long h_stride, gu_stride;
};

template <typename E, int ACT, int TILES>
__global__ void __launch_bounds__(kFewWarps * 32, TILES == 1 ? 4 : TILES == 2 ? 3 : 2) k_glu_few(const FewArgs<E> p) {
  wait_for_previous();
  may_follow();
  constexpr int kBlocks = TILES <= 2 ? 4 : 2;                     // k blocks in flight per warp
  __shared__ float sums[kFewWarps][2][TILES * 8 * 8];             // [warp][gate, up][token, column]
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = lane / 4, q = lane % 4;
  const int f0 = blockIdx.x * 8;
  // columns and tokens outside are taken from the last one inside; what they give is not written
  const long long row = min(f0 + r, p.F - 1) * p.w_stride + q * 16;
  const E *wg = p.wg + row, *wu = p.wu + row, *tokens[TILES];
#pragma unroll
  for (int n = 0; n < TILES; ++n) tokens[n] = p.x + min(n * 8 + r, p.T - 1) * p.x_stride + q * 16;
  float c[TILES][4] = {};
  const auto multiply = [&](const uint4& g, const uint4& u, const uint4& x, int n) {
    mma16816<E>(c[n], g.x, u.x, g.y, u.y, x.x, x.y);
    mma16816<E>(c[n], g.z, u.z, g.w, u.w, x.z, x.w);
  };
  const auto blocks_at = [&](int b, auto count) {
    constexpr int N = decltype(count)::value;
    uint4 g[N][2], u[N][2], x[N][TILES][2];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int at = (b + i * kFewWarps) * 64 + k * 8;
        g[i][k] = load_once(wg + at);
        u[i][k] = load_once(wu + at);
#pragma unroll
        for (int n = 0; n < TILES; ++n) x[i][n][k] = load16(tokens[n] + at);
      }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int n = 0; n < TILES; ++n) multiply(g[i][k], u[i][k], x[i][n][k], n);
  };
  const int whole = p.D / 64;
  int b = warp;
  for (; b + (kBlocks - 1) * kFewWarps < whole; b += kFewWarps * kBlocks) blocks_at(b, std::integral_constant<int, kBlocks>());
  if (kBlocks > 2 && b + kFewWarps < whole) {
    blocks_at(b, std::integral_constant<int, 2>());
    b += 2 * kFewWarps;
  }
  for (; b < whole; b += kFewWarps) blocks_at(b, std::integral_constant<int, 1>());
  if (b == whole && p.D % 64) {                                   // the last, partial block
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int at = whole * 64 + k * 8, left = p.D - at - q * 16;
      const uint4 g = load_end(wg + at, left), u = load_end(wu + at, left);
#pragma unroll
      for (int n = 0; n < TILES; ++n) {
        const uint4 x = load_end(tokens[n] + at, left);
        __syncwarp();                                             // lanes load different numbers of elements; mma.sync takes them together
        multiply(g, u, x, n);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < TILES; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[warp][i >> 1][(n * 8 + q * 2 + (i & 1)) * 8 + r] = c[n][i];
  __syncthreads();
  static_assert(TILES * 64 <= kFewWarps * 32, "one output per thread");
  if (threadIdx.x >= TILES * 64) return;
  const int t = threadIdx.x / 8, f = f0 + threadIdx.x % 8;
  if (t >= p.T || f >= p.F) return;
  float gs = 0.f, us = 0.f;
#pragma unroll
  for (int w = 0; w < kFewWarps; ++w) {
    gs += sums[w][0][threadIdx.x];
    us += sums[w][1][threadIdx.x];
  }
  p.h[t * p.h_stride + f] = from_f32<E>(act_value<ACT>(gs) * us);
  if (p.gate) {
    p.gate[t * p.gu_stride + f] = from_f32<E>(gs);
    p.up[t * p.gu_stride + f] = from_f32<E>(us);
  }
}

// ---- the element-wise part of the gradient ------------------------------------------------------
// dg and du go to scratch of pitch F rounded up to 8 elements, so that its rows start on 16-byte boundaries.
// One read of dh, gate and up, one write of dg and du: bound by memory (8192 x 5632: 461 MB in 65 us, 7.1 TB/s with part of
// the writes still in L2).  WIDE: the inputs' rows start on 16-byte
// boundaries; a thread takes 8 columns (the last ones of a row one by one), otherwise one.
template <typename T, int ACT, bool WIDE>
__global__ void __launch_bounds__(256) k_glu_slope(const T* dh, long long dh_stride, const T* gate, const T* up,
                                                   long long gu_stride, long long rows, unsigned F, T* dg, T* du,
                                                   long long pitch) {
  wait_for_previous();
  may_follow();
  constexpr unsigned W = WIDE ? 8 : 1;
  const unsigned packs = (F + W - 1) / W;
  const long long blocks = (rows * packs + 255) / 256;
  const auto one = [&](float d, float g, float u, float& out_g, float& out_u) {
    const Activation x = activate<ACT>(g);
    out_g = d * u * x.slope;
    out_u = d * x.value;
  };
  for (long long b = blockIdx.x; b < blocks; b += gridDim.x) {
    const long long first = b * 256, row0 = first / packs;
    const unsigned rest = (unsigned)(first - row0 * packs) + threadIdx.x, down = rest / packs, f = (rest - down * packs) * W;
    const long long t = row0 + down;
    if (t >= rows) return;
    const T *pd = dh + t * dh_stride + f, *pg = gate + t * gu_stride + f, *pu = up + t * gu_stride + f;
    if (WIDE && f + 8 <= F) {
      const uint4 rd = load16(pd), rg = load16(pg), ru = load16(pu);
      const T *d = reinterpret_cast<const T*>(&rd), *g = reinterpret_cast<const T*>(&rg), *u = reinterpret_cast<const T*>(&ru);
      unsigned og[4], ou[4];
      for (int i = 0; i < 4; ++i) {
        float g0, g1, u0, u1;
        one(to_f32(d[2 * i]), to_f32(g[2 * i]), to_f32(u[2 * i]), g0, u0);
        one(to_f32(d[2 * i + 1]), to_f32(g[2 * i + 1]), to_f32(u[2 * i + 1]), g1, u1);
        og[i] = pack2<T>(g0, g1);
        ou[i] = pack2<T>(u0, u1);
      }
      *reinterpret_cast<uint4*>(dg + t * pitch + f) = make_uint4(og[0], og[1], og[2], og[3]);
      *reinterpret_cast<uint4*>(du + t * pitch + f) = make_uint4(ou[0], ou[1], ou[2], ou[3]);
    } else {
      for (unsigned i = 0; i < W && f + i < F; ++i) {
        float og, ou;
        one(to_f32(pd[i]), to_f32(pg[i]), to_f32(pu[i]), og, ou);
        dg[t * pitch + f + i] = from_f32<T>(og);
        du[t * pitch + f + i] = from_f32<T>(ou);
      }
    }
  }
}

template <typename F> void with_glu(int32_t type, int32_t act, F&& f) {
  if (type == COCODC_BF16) {
    if (act == COCODC_ACT_SILU) f(__nv_bfloat16(), std::integral_constant<int, COCODC_ACT_SILU>());
    else f(__nv_bfloat16(), std::integral_constant<int, COCODC_ACT_GELU>());
  } else {
    if (act == COCODC_ACT_SILU) f(__half(), std::integral_constant<int, COCODC_ACT_SILU>());
    else f(__half(), std::integral_constant<int, COCODC_ACT_GELU>());
  }
}

int tiles_of(int64_t n, int tile) { return (int)((n + tile - 1) / tile); }

// Parts of dx's contraction where its tiles leave at least half of the SMs without one: as many as there are SMs for each
// tile, with at least 16 k-blocks to a part.  One row of tiles takes narrow ones (more SMs read weights), more rows the
// widest (the tokens are read once per tile); 2048 x 5632 without parts, with parts of 64 and of 256 columns, us for the
// whole of dx: 128 tokens 57 / 28 / 35, 512 tokens 59 / 61 (no parts) / 41.
constexpr int kPartTiles = 148;                       // tiles x parts at most: a B200's SMs (the workspace's size is asked for without a handle)
int part_width(int64_t T) { return T <= kBM ? 64 : 256; }
int parts_for(int64_t T, int64_t D, int64_t F) {
  const long long tiles = (long long)tiles_of(T, kBM) * tiles_of(D, part_width(T)), blocks = 2ll * tiles_of(F, kBK);
  const long long parts = tiles > 0 ? kPartTiles / tiles : 1, most = blocks / 16;
  const long long p = parts < most ? parts : most;
  return p < 2 ? 1 : (int)p;
}
uint64_t part_bytes(int64_t T, int64_t D, int64_t F) {
  const int p = parts_for(T, D, F), w = part_width(T);
  return p < 2 ? 0 : (uint64_t)p * tiles_of(T, kBM) * tiles_of(D, w) * kBM * w * sizeof(float);
}

int64_t scratch_pitch(int64_t F) { return (F + 7) / 8 * 8; }

// ---- tensor-core path: host side ----------------------------------------------------------------
template <typename E, int MODE, int ACT, int BN> cocodc_status run_tc(cocodc_lm* lm, const TcArgs& a, cudaStream_t st) {
  const long long tiles = (long long)a.m_tiles * a.n_tiles * a.matrices, most = lm->sm_count;
  if (tiles > INT32_MAX / 2) return COCODC_ERR_INVALID_ARG;
  return start(lm, k_glu_tc<E, MODE, ACT, BN>, (unsigned)(tiles < most ? tiles : most), kTcThreads, TcShape<BN>::kSmem, st, 1, a);
}

int a_rows_for(int64_t T) { return T >= kBM ? kBM : (int)((T + 7) / 8 * 8); }
// Width of the tiles in columns of an output: the narrowest that still gives every tile an SM of its own (few tokens:
// more SMs read weights), and the widest once there are more tiles than SMs (fewer bytes per product).  Forward, us at widths
// 128 / 64 / 32: 128 tokens, 2048 x 5632: 19.0 / 15.4 / 16.1 (88 tiles of 64); 256 tokens: 19.5 / 25.1 / 24.4 (88 tiles of
// 128); 128 tokens, 1024 x 2816: 12.2 / 10.0 / 9.5 (88 tiles of 32).
int width_for(const cocodc_lm* lm, int64_t M, int64_t N, int widest) {
  for (int w = widest / 4; w < widest; w *= 2)
    if ((long long)tiles_of(M, kBM) * tiles_of(N, w) <= lm->sm_count) return w;
  return widest;
}

bool tiles_fit(int64_t rows, int64_t cols) { return (rows + kTile - 1) / kTile <= INT32_MAX && (cols + kTile - 1) / kTile <= 65535; }

}  // namespace

namespace cocodc_lm_impl {
bool glu_prepare() {
  if (!g_encode.load()) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || !fn) return false;
    g_encode.store(reinterpret_cast<EncodeTiled>(fn));
  }
  bool ok = true;
  const auto allow = [&](auto kernel, unsigned smem) {
    ok = ok && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess;
  };
  const auto allow_tc = [&](auto e, auto width) {
    using E = decltype(e);
    constexpr int BN = decltype(width)::value;
    allow(k_glu_tc<E, GLU_FWD, COCODC_ACT_SILU, BN>, TcShape<BN>::kSmem);
    allow(k_glu_tc<E, GLU_FWD, COCODC_ACT_GELU, BN>, TcShape<BN>::kSmem);
    allow(k_glu_tc<E, GLU_DX, 0, BN>, TcShape<BN>::kSmem);
    allow(k_glu_tc<E, GLU_DW, 0, BN>, TcShape<BN>::kSmem);
    if constexpr (BN != 128) allow(k_glu_tc<E, GLU_DX_PARTS, 0, BN>, TcShape<BN>::kSmem);
  };
  const auto allow_type = [&](auto e) {
    allow_tc(e, std::integral_constant<int, 256>());
    allow_tc(e, std::integral_constant<int, 128>());
    allow_tc(e, std::integral_constant<int, 64>());
  };
  allow_type(__nv_bfloat16());
  allow_type(__half());
  return ok;
}
}  // namespace cocodc_lm_impl

extern "C" {

cocodc_status cocodc_lm_glu(cocodc_lm* lm, int32_t act, int32_t type, const void* x, int64_t x_stride, const void* wg,
                            const void* wu, int64_t w_stride, int64_t T, int64_t D, int64_t F, void* h,
                            int64_t h_stride, void* gate, void* up, int64_t gu_stride, void* stream) {
  if (!lm || (act != COCODC_ACT_SILU && act != COCODC_ACT_GELU) || (type != COCODC_BF16 && type != COCODC_F16) ||
      !sane(T) || !sane(D) || !sane(F) || T > INT32_MAX || D < 1 || D > INT32_MAX || F < 1 || F > INT32_MAX ||
      x_stride < D || w_stride < D || h_stride < F || !sane(x_stride) || !sane(w_stride) || !sane(h_stride))
    return COCODC_ERR_INVALID_ARG;
  if (T == 0) return COCODC_OK;
  if ((gate == nullptr) != (up == nullptr) || (gate && (gu_stride < F || !sane(gu_stride)))) return COCODC_ERR_INVALID_ARG;
  if (!x || !wg || !wu || !h || !tiles_fit(T, F)) return COCODC_ERR_INVALID_ARG;
  for (const void* p : {x, wg, wu, (const void*)h, (const void*)gate, (const void*)up})
    if (!on_boundary(p, 2)) return COCODC_ERR_ALIGNMENT;
  const Span in[3] = {span(x, T, x_stride, D, 2), span(wg, F, w_stride, D, 2), span(wu, F, w_stride, D, 2)};
  const Span out[3] = {span(h, T, h_stride, F, 2), span(gate, T, gu_stride, F, 2), span(up, T, gu_stride, F, 2)};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 3; ++j)
      if (meet(out[i], in[j])) return COCODC_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return COCODC_ERR_ALIAS;
  }
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool tensor = rows_aligned(x, x_stride, 2) && rows_aligned(wg, w_stride, 2) && rows_aligned(wu, w_stride, 2) &&
                      rows_aligned(h, h_stride, 2) && (!gate || (rows_aligned(gate, gu_stride, 2) && rows_aligned(up, gu_stride, 2)));
  cocodc_status result = COCODC_OK;
  const bool few = few_tokens(T, D, F) && rows_aligned(x, x_stride, 2) && rows_aligned(wg, w_stride, 2) && rows_aligned(wu, w_stride, 2);
  with_glu(type, act, [&](auto e, auto a) {
    using E = decltype(e);
    if (few) {
      constexpr int A = decltype(a)::value;
      const FewArgs<E> p{static_cast<const E*>(x), static_cast<const E*>(wg), static_cast<const E*>(wu), x_stride, w_stride,
                         (int)T, (int)D, (int)F, static_cast<E*>(h), static_cast<E*>(gate), static_cast<E*>(up), h_stride, gu_stride};
      const unsigned grid = (unsigned)((F + 7) / 8);
      result = T <= 8    ? start(lm, k_glu_few<E, A, 1>, grid, kFewWarps * 32, 0, st, 1, p)
               : T <= 16 ? start(lm, k_glu_few<E, A, 2>, grid, kFewWarps * 32, 0, st, 1, p)
                         : start(lm, k_glu_few<E, A, 4>, grid, kFewWarps * 32, 0, st, 1, p);
      return;
    }
    if (tensor) {
      TcArgs c{};
      const int width = width_for(lm, T, F, 128);
      bool ok = map_of<E>(&c.a[0], x, x_stride, T, D, a_rows_for(T)) && map_of<E>(&c.b[0], wg, w_stride, F, D, width) &&
                map_of<E>(&c.b[1], wu, w_stride, F, D, width) && map_of<E>(&c.c[0], h, h_stride, T, F, 32);
      c.a_bytes = a_rows_for(T) * kBK * 2;
      if (gate) ok = ok && map_of<E>(&c.c[1], gate, gu_stride, T, F, 32) && map_of<E>(&c.c[2], up, gu_stride, T, F, 32);
      c.m_tiles = tiles_of(T, kBM);
      c.n_tiles = tiles_of(F, width);
      c.matrices = c.sources = 1;
      c.k_blocks = tiles_of(D, kBK);
      c.M = (int)T;
      c.N = (int)F;
      c.save = gate != nullptr;
      c.out[0] = h; c.out[1] = gate; c.out[2] = up;
      c.ld[0] = h_stride; c.ld[1] = c.ld[2] = gu_stride;
      c.status = lm->d_status;
      constexpr int A = decltype(a)::value;
      result = !ok            ? COCODC_ERR_CUDA
               : width == 128 ? run_tc<E, GLU_FWD, A, 256>(lm, c, st)
               : width == 64  ? run_tc<E, GLU_FWD, A, 128>(lm, c, st)
                              : run_tc<E, GLU_FWD, A, 64>(lm, c, st);
      return;
    }
    PlainArgs<E> p{};
    p.a[0] = {static_cast<const E*>(x), x_stride, 1};
    p.b[0] = {static_cast<const E*>(wg), w_stride, 1};
    p.b[1] = {static_cast<const E*>(wu), w_stride, 1};
    p.M = T; p.N = F; p.K = D;
    p.out[0] = static_cast<E*>(h);
    p.out[1] = static_cast<E*>(gate);
    p.out[2] = static_cast<E*>(up);
    p.ld = h_stride;
    p.ld_gu = gu_stride;
    const dim3 grid((unsigned)((T + kTile - 1) / kTile), (unsigned)((F + kTile - 1) / kTile));
    result = start(lm, k_glu_plain<E, decltype(a)::value>, grid, 256, 0, st, 1, p);
  });
  return result;
}

uint64_t cocodc_lm_glu_grad_workspace(int64_t T, int64_t D, int64_t F) {
  if (T < 0 || D < 0 || F < 0 || T > INT32_MAX || D > INT32_MAX || F > INT32_MAX) return 0;
  return 16 + 2 * (uint64_t)T * (uint64_t)scratch_pitch(F) * 2 + part_bytes(T, D, F);
}

cocodc_status cocodc_lm_glu_grad(cocodc_lm* lm, int32_t act, int32_t type, const void* dh, int64_t dh_stride,
                                 const void* gate, const void* up, int64_t gu_stride, const void* x, int64_t x_stride,
                                 const void* wg, const void* wu, int64_t w_stride, int64_t T, int64_t D, int64_t F,
                                 void* dx, int64_t dx_stride, void* dwg, void* dwu, int64_t dw_stride,
                                 void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!lm || (act != COCODC_ACT_SILU && act != COCODC_ACT_GELU) || (type != COCODC_BF16 && type != COCODC_F16) ||
      !sane(T) || !sane(D) || !sane(F) || T > INT32_MAX || D < 1 || D > INT32_MAX || F < 1 || F > INT32_MAX ||
      x_stride < D || w_stride < D || dh_stride < F || gu_stride < F || !sane(x_stride) || !sane(w_stride) ||
      !sane(dh_stride) || !sane(gu_stride) || (dx && (dx_stride < D || !sane(dx_stride))) ||
      (dwg == nullptr) != (dwu == nullptr) || (dwg && (dw_stride < D || !sane(dw_stride))))
    return COCODC_ERR_INVALID_ARG;
  if (!dx && !dwg) return T == 0 ? COCODC_OK : COCODC_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < cocodc_lm_glu_grad_workspace(T, D, F)) return COCODC_ERR_INVALID_ARG;
  if (T > 0 && (!dh || !gate || !up || (dwg && !x) || (dx && (!wg || !wu)))) return COCODC_ERR_INVALID_ARG;
  if (!tiles_fit(T, D) || !tiles_fit(F, D)) return COCODC_ERR_INVALID_ARG;
  for (const void* p : {dh, gate, up, x, wg, wu, (const void*)dx, (const void*)dwg, (const void*)dwu})
    if (!on_boundary(p, 2)) return COCODC_ERR_ALIGNMENT;
  if (!on_boundary(workspace, 16)) return COCODC_ERR_ALIGNMENT;
  const Span in[6] = {span(dh, T, dh_stride, F, 2), span(gate, T, gu_stride, F, 2), span(up, T, gu_stride, F, 2),
                      span(x, T, x_stride, D, 2), span(wg, F, w_stride, D, 2), span(wu, F, w_stride, D, 2)};
  const Span out[4] = {span(dx, T, dx_stride, D, 2), span(dwg, F, dw_stride, D, 2), span(dwu, F, dw_stride, D, 2),
                       span(workspace, 1, (int64_t)workspace_bytes, (int64_t)workspace_bytes, 1)};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 6; ++j)
      if (meet(out[i], in[j])) return COCODC_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return COCODC_ERR_ALIAS;
  }
  DeviceScope scope(lm->device);
  if (!scope.ok) return COCODC_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool tensor_dx = rows_aligned(wg, w_stride, 2) && rows_aligned(wu, w_stride, 2) && rows_aligned(dx, dx_stride, 2);
  const bool tensor_dw = rows_aligned(x, x_stride, 2) && rows_aligned(dwg, dw_stride, 2) && rows_aligned(dwu, dw_stride, 2);
  cocodc_status result = COCODC_OK;
  with_glu(type, act, [&](auto e, auto a) {
    using E = decltype(e);
    const int64_t pitch = scratch_pitch(F);
    E* dg = static_cast<E*>(workspace);
    E* du = dg + T * pitch;
    if (T > 0) {
      const bool wide = rows_aligned(dh, dh_stride, 2) && rows_aligned(gate, gu_stride, 2) && rows_aligned(up, gu_stride, 2);
      const auto slope = [&](auto kernel, int W) {
        const long long blocks = (T * ((F + W - 1) / W) + 255) / 256;
        return start(lm, kernel, (unsigned)(blocks < (1 << 30) ? blocks : (1 << 30)), 256, 0, st, 1,
                     static_cast<const E*>(dh), dh_stride, static_cast<const E*>(gate), static_cast<const E*>(up), gu_stride, T,
                     (unsigned)F, dg, du, pitch);
      };
      result = wide ? slope(k_glu_slope<E, decltype(a)::value, true>, 8) : slope(k_glu_slope<E, decltype(a)::value, false>, 1);
      if (result != COCODC_OK) return;                 // dg and du were not written
    }
    TcArgs c{};
    c.status = lm->d_status;
    c.splits = 1;
    c.N = (int)D;
    const auto run = [&](auto mode, int width) {
      constexpr int MODE = decltype(mode)::value;
      return width == 256 ? run_tc<E, MODE, 0, 256>(lm, c, st)
             : width == 128 ? run_tc<E, MODE, 0, 128>(lm, c, st)
                            : run_tc<E, MODE, 0, 64>(lm, c, st);
    };
    if (dx && T > 0 && tensor_dx) {
      const int splits = parts_for(T, D, F), width = splits > 1 ? part_width(T) : width_for(lm, T, D, 256);
      c.n_tiles = tiles_of(D, width);
      c.a_bytes = a_rows_for(T) * kBK * 2;
      c.splits = splits;
      c.parts = reinterpret_cast<float*>(du + T * pitch);
      const bool ok = map_of<E>(&c.a[0], dg, pitch, T, F, a_rows_for(T)) && map_of<E>(&c.a[1], du, pitch, T, F, a_rows_for(T)) &&
                      map_of<E>(&c.b[0], wg, w_stride, F, D, kBK) && map_of<E>(&c.b[1], wu, w_stride, F, D, kBK) &&
                      map_of<E>(&c.c[0], dx, dx_stride, T, D, 32);
      c.m_tiles = tiles_of(T, kBM);
      c.matrices = splits;
      c.sources = 2;
      c.out[0] = dx;
      c.ld[0] = dx_stride;
      c.k_blocks = tiles_of(F, kBK);
      c.M = (int)T;
      const auto in_parts = [&](auto w) {
        constexpr int BN = decltype(w)::value;
        const cocodc_status s = run_tc<E, GLU_DX_PARTS, 0, BN>(lm, c, st);
        return s != COCODC_OK ? s : start(lm, k_add_parts<E, BN>, (unsigned)(c.m_tiles * c.n_tiles * (kBM / 8)), 256, 0, st, 1, c);
      };
      result = !ok           ? COCODC_ERR_CUDA
               : splits == 1 ? run(std::integral_constant<int, GLU_DX>(), width)
               : width == 64 ? in_parts(std::integral_constant<int, 64>())
                             : in_parts(std::integral_constant<int, 256>());
    } else if (dx && T > 0) {
      PlainArgs<E> p{};
      p.a[0] = {dg, pitch, 1};
      p.a[1] = {du, pitch, 1};
      p.b[0] = {static_cast<const E*>(wg), 1, w_stride};
      p.b[1] = {static_cast<const E*>(wu), 1, w_stride};
      p.M = T; p.N = D; p.K = F;
      p.out[0] = static_cast<E*>(dx);
      p.ld = dx_stride;
      const dim3 grid((unsigned)((T + kTile - 1) / kTile), (unsigned)((D + kTile - 1) / kTile));
      result = start(lm, k_product_plain<E, true>, grid, 256, 0, st, 1, p);
    }
    if (result != COCODC_OK) return;
    if (dwg && tensor_dw && T > 0) {
      const int width = width_for(lm, 2 * F, D, 256);
      c.n_tiles = tiles_of(D, width);
      c.a_bytes = kABytes;
      const bool ok = map_of<E>(&c.a[0], dg, pitch, T, F, kBK) && map_of<E>(&c.a[1], du, pitch, T, F, kBK) &&
                      map_of<E>(&c.b[0], x, x_stride, T, D, kBK) && map_of<E>(&c.c[0], dwg, dw_stride, F, D, 32) &&
                      map_of<E>(&c.c[1], dwu, dw_stride, F, D, 32);
      c.m_tiles = tiles_of(F, kBM);
      c.matrices = 2;
      c.sources = 1;
      c.out[0] = dwg; c.out[1] = dwu;
      c.ld[0] = c.ld[1] = dw_stride;
      c.k_blocks = tiles_of(T, kBK);
      c.M = (int)F;
      result = ok ? run(std::integral_constant<int, GLU_DW>(), width) : COCODC_ERR_CUDA;
    } else if (dwg) {
      PlainArgs<E> p{};
      p.a[0] = {dg, 1, pitch};
      p.a[1] = {du, 1, pitch};
      p.b[0] = p.b[1] = {static_cast<const E*>(x), 1, x_stride};
      p.M = F; p.N = D; p.K = T;
      p.out[0] = static_cast<E*>(dwg);
      p.out[1] = static_cast<E*>(dwu);
      p.ld = dw_stride;
      const dim3 grid((unsigned)((F + kTile - 1) / kTile), (unsigned)((D + kTile - 1) / kTile), 2);
      result = start(lm, k_product_plain<E, false>, grid, 256, 0, st, 1, p);
    }
  });
  return result;
}

}  // extern "C"
