// Tensor-core kernel of the gated block: its forward pass and the two products of its gradient.
//
// Persistent, 128 x BN output tiles (M x N), k-blocks of 64:
//   warp 0   producer: TMA copies of the operands' tiles into a ring of shared-memory stages
//   warp 1   issuer: tcgen05.mma of each stage into one of two TMEM accumulators of BN columns
//   warps 2-5 epilogue: TMEM -> registers -> activation -> shared memory -> TMA store, while the other accumulator fills
// BN = 256 feeds the tensor cores best (one CTA per SM); narrower tiles are for few tokens, where there would be fewer
// tiles than SMs and the time goes into reading the weights.
// Forward: BN / 2 columns of F, the tile's B rows are the gate's weight rows followed by the up projection's, so a
// thread of the epilogue finds gate and up of one element in its own TMEM lane and the product needs no exchange.
// dx = dg Wg + du Wu: one accumulator, the k loop runs through both sources.  dw = d^T x: the tile index picks dg or du.
// The operands of the gradient whose contraction runs along rows are taken MN-major as they lie in memory.
// Measured: forward 8192 x 3200 x 8640 with gate and up kept 612-621 us alone (1.46-1.48 PFLOP/s, tensor pipe 81 % active) and 747-756 us
// back to back, where the power cap lowers the clock (without keeping them 687 us; a library product of the same size
// 645-685 us in the same loop); dx 270-276 us and dw 263-267 us alone at 8192 x 2048 x 5632 (1.40, 1.44 PFLOP/s).  Pairs of CTAs with
// 256 x 256 tiles (cta_group::2) and a second set of epilogue warps were built and gave nothing at these sizes.
// With few tokens dx has few tiles and a long contraction: it is cut into parts (GLU_DX_PARTS, the slowest tile index),
// whose fp32 sums k_add_parts adds in order.
// Ragged sizes: TMA fills what lies outside a matrix with zeros, and clips rows and whole 16-byte groups of columns
// when it writes; the last N mod 8 columns of an output leave by ordinary stores (a copy rounds them up to 16 bytes).
#pragma once

#include "lm_mma.cuh"

namespace cocodc_lm_impl {

enum { GLU_FWD = 0, GLU_DX = 1, GLU_DW = 2, GLU_DX_PARTS = 3 };

struct TcArgs {
  CUtensorMap a[2], b[2], c[3];
  int m_tiles, n_tiles;      // of one matrix
  int matrices;              // GLU_DW: 2; GLU_DX_PARTS: splits
  int k_blocks;              // of one source
  int sources;               // GLU_DX: 2
  int splits;                // GLU_DX_PARTS: parts of the contraction, whose sums go to `parts` in fp32
  float* parts;              // [splits][tile][128][BN]
  int M, N;                  // rows and columns of the outputs
  int a_bytes;               // of A's part of a stage: fewer than 128 tokens are loaded as they are
  int save;                  // GLU_FWD: also write gate and up (c[1], c[2])
  void* out[3];              // what c[] describes, for columns that a copy cannot write alone
  long long ld[3];
  int* status;
};

template <int BN> struct TcShape {
  static constexpr unsigned kBBytes = BN * kBK * 2, kStageBytes = kABytes + kBBytes;
  // one CTA per SM; wide tiles stage their outputs for TMA stores, narrow ones write them from registers
  static constexpr bool kStaged = BN >= 128;
  static constexpr int kStages = BN == 256 ? 4 : BN == 128 ? 6 : 8;
  static constexpr unsigned kSmem = 1024 + kStages * kStageBytes + (kStaged ? 4 * 2 * kOutBytes : 0);
};
// Tiles of consecutive rows that go through one column of tiles in turn.  Under the power cap, where fewer bytes from L2 mean
// a higher clock, 8 / 16 / 32 / 64 of them took 740 / 706 / 687 / 697 us forward (8192 x 3200 x 8640) and 8 / 16 / 32 took
// 708 / 724 / 717 us for the gradient (8192 x 2048 x 5632, all three launches).
template <int MODE> constexpr int kGroupM = MODE == GLU_FWD ? 32 : 8;

struct TcShared {
  unsigned long long full[8], empty[8], acc_full[2], acc_empty[2], drain;
  unsigned tmem;
  int stop;
};

struct TileAt { int z, m, n; };
// Tiles in groups of row tiles, inside a group column after column: CTAs that run together share operands in L2.
template <int MODE> __device__ __forceinline__ TileAt tile_at(const TcArgs& a, int tile) {
  TileAt t;
  const int per = a.m_tiles * a.n_tiles;
  t.z = tile / per;
  tile -= t.z * per;
  const int group = tile / (kGroupM<MODE> * a.n_tiles), first = group * kGroupM<MODE>;
  const int height = min(kGroupM<MODE>, a.m_tiles - first);
  tile -= group * kGroupM<MODE> * a.n_tiles;
  t.m = first + tile % height;
  t.n = tile / height;
  return t;
}

template <int ACT> __device__ __forceinline__ float act_value(float g);

// 64 staged columns of the warp's 32 rows leave for global memory; rows and columns outside are not written.
__device__ __forceinline__ void send(const TcArgs& a, int what, int x, int y, unsigned buf, int lane) {
  if (x + 64 <= a.N || a.N % 8 == 0) {
    fence_async_smem();
    __syncwarp();
    if (lane == 0) tma_store(&a.c[what], x, y, buf);
  } else if (y + lane < a.M) {
    unsigned short* row = static_cast<unsigned short*>(a.out[what]) + (y + lane) * a.ld[what] + x;
    for (int i = 0; i < a.N - x; ++i) {
      unsigned short v;
      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(buf + lane * 128 + (((i / 8) ^ (lane & 7)) << 4) + i % 8 * 2));
      row[i] = v;
    }
  }
  if (lane == 0) store_commit();
}
// 32 columns (packed in pairs) of a row straight to global memory; rows start on 16-byte boundaries
__device__ __forceinline__ void store_row(const TcArgs& a, int what, int x, int y, const unsigned (&v)[16]) {
  unsigned short* row = static_cast<unsigned short*>(a.out[what]) + y * a.ld[what] + x;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (x + q * 8 + 8 <= a.N) {
      reinterpret_cast<uint4*>(row)[q] = make_uint4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (x + q * 8 + i < a.N) row[q * 8 + i] = (unsigned short)(v[4 * q + i / 2] >> (i % 2 * 16));
    }
  }
}
template <typename E, int MODE, int ACT, int BN>
__global__ void __launch_bounds__(kTcThreads, 1) k_glu_tc(const __grid_constant__ TcArgs a) {
  extern __shared__ unsigned char dyn[];
  __shared__ TcShared sh;
  using S = TcShape<BN>;
  constexpr int kStages = S::kStages, kColumns = MODE == GLU_FWD ? BN / 2 : BN;   // of an output
  constexpr unsigned kStageBytes = S::kStageBytes, kBBytes = S::kBBytes;
  const unsigned base = (smem_addr(dyn) + 1023u) & ~1023u;
  const unsigned staging = base + kStages * kStageBytes;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  constexpr bool a_mn = MODE == GLU_DW, b_mn = MODE != GLU_FWD;
  const int tiles = a.m_tiles * a.n_tiles * a.matrices;
  const int blocks = a.k_blocks * a.sources;
  const auto first_block = [&](int z) { return MODE == GLU_DX_PARTS ? (int)((long long)blocks * z / a.splits) : 0; };
  constexpr bool kDx = MODE == GLU_DX || MODE == GLU_DX_PARTS;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      bar_init(smem_addr(&sh.full[s]), 1);
      bar_init(smem_addr(&sh.empty[s]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(smem_addr(&sh.acc_full[i]), 1);
      bar_init(smem_addr(&sh.acc_empty[i]), 4);
    }
    bar_init(smem_addr(&sh.drain), 1);
    sh.stop = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // Before TMEM is taken: a block that held it while it waited could starve a block of the kernel it waits for; and only
  // then may the next kernel's blocks come.
  wait_for_previous();
  if (warp == 1) tmem_alloc(smem_addr(&sh.tmem), 2 * BN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  may_follow();
  const unsigned tmem = sh.tmem;
  volatile int* stop = &sh.stop;

  if (warp == 0) {
    if (lane == 0) {
      long long it = 0;
      bool ok = true;
      for (int tile = blockIdx.x; ok && tile < tiles; tile += gridDim.x) {
        const TileAt t = tile_at<MODE>(a, tile);
        const int m0 = t.m * kBM, n0 = t.n * kColumns;
        const int kb0 = first_block(t.z), kb1 = MODE == GLU_DX_PARTS ? first_block(t.z + 1) : blocks;
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          const int s = (int)(it % kStages);
          ok = bar_wait(smem_addr(&sh.empty[s]), (unsigned)((it / kStages) & 1) ^ 1, stop);
          if (!ok) break;
          const unsigned full = smem_addr(&sh.full[s]), sa = base + s * kStageBytes, sb = sa + kABytes;
          const int src = kb >= a.k_blocks, k0 = (kb - src * a.k_blocks) * kBK;
          bar_expect(full, a.a_bytes + kBBytes);
          if (MODE == GLU_FWD) {
            tma_load(sa, &a.a[0], k0, m0, full);
            tma_load(sb, &a.b[0], k0, n0, full);
            tma_load(sb + kBBytes / 2, &a.b[1], k0, n0, full);
          } else {
            if (kDx) {
              tma_load(sa, &a.a[src], k0, m0, full);
            } else {
              for (int i = 0; i < kBM / 64; ++i) tma_load(sa + i * kSlab, &a.a[t.z], m0 + i * 64, k0, full);
            }
            for (int i = 0; i < BN / 64; ++i)
              tma_load(sb + i * kSlab, &a.b[kDx ? src : 0], n0 + i * 64, k0, full);
          }
        }
      }
      // the issuer's last arrivals come before the CTA leaves
      for (long long i = it > kStages ? it - kStages : 0; ok && i < it; ++i)
        ok = bar_wait(smem_addr(&sh.empty[i % kStages]), (unsigned)((i / kStages) & 1), stop);
      // given up: the copies in flight land before the CTA leaves its shared memory
      if (!ok)
        for (long long i = it > kStages ? it - kStages : 0; i < it; ++i)
          bar_drain(smem_addr(&sh.full[i % kStages]), (unsigned)((i / kStages) & 1));
    }
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr unsigned idesc = instr_desc<E>(kBM, BN, a_mn, b_mn);
      long long it = 0;
      int turn = 0;
      bool ok = true;
      for (int tile = blockIdx.x; ok && tile < tiles; tile += gridDim.x, ++turn) {
        const int acc = turn & 1, z = MODE == GLU_DX_PARTS ? tile / (a.m_tiles * a.n_tiles) : 0;
        const int kb0 = first_block(z), kb1 = MODE == GLU_DX_PARTS ? first_block(z + 1) : blocks;
        ok = bar_wait(smem_addr(&sh.acc_empty[acc]), (unsigned)((turn >> 1) & 1) ^ 1, stop);
        tc_fence_after();
        for (int kb = kb0; ok && kb < kb1; ++kb, ++it) {
          const int s = (int)(it % kStages);
          ok = bar_wait(smem_addr(&sh.full[s]), (unsigned)((it / kStages) & 1), stop);
          if (!ok) break;
          tc_fence_after();
          const unsigned sa = base + s * kStageBytes, sb = sa + kABytes;
          const unsigned long long da = tile_desc(sa, a_mn ? kSlab : 16), db = tile_desc(sb, b_mn ? kSlab : 16);
          for (int k = 0; k < kBK / 16; ++k)   // 16 k: 32 bytes along a K-major row, 16 rows of an MN-major tile
            tc_mma(tmem + acc * BN, da + (unsigned)(k * (a_mn ? 2048 : 32) >> 4), db + (unsigned)(k * (b_mn ? 2048 : 32) >> 4),
                   idesc, kb > kb0 || k > 0);
          tc_commit(smem_addr(&sh.empty[s]));
        }
        if (ok) tc_commit(smem_addr(&sh.acc_full[acc]));
      }
      if (!ok) {
        tc_commit(smem_addr(&sh.drain));
        bar_drain(smem_addr(&sh.drain), 0);
      }
    }
  } else {
    const int quarter = warp & 3, e = warp - 2;
    const unsigned out = staging + e * 2 * kOutBytes;
    int turn = 0, sent = 0;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++turn) {
      const int acc = turn & 1;
      const TileAt t = tile_at<MODE>(a, tile);
      const int row0 = t.m * kBM + quarter * 32, n0 = t.n * kColumns;
      if (!__all_sync(~0u, bar_wait(smem_addr(&sh.acc_full[acc]), (unsigned)((turn >> 1) & 1), stop))) break;
      tc_fence_after();
      const unsigned src = tmem + acc * BN + ((unsigned)(quarter * 32) << 16);
      if constexpr (MODE == GLU_DX_PARTS) {
        if (row0 < a.M)
          for (int col = 0; col < kColumns; col += 32) {
            float v[32];
            tmem_load32(v, src + col);
            tmem_wait_loads();
            float4* to = reinterpret_cast<float4*>(a.parts + ((long long)tile * kBM + quarter * 32 + lane) * BN + col);
            for (int i = 0; i < 8; ++i) to[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
          }
      } else if constexpr (S::kStaged) {
        // one staged tile of 64 columns after the other, two buffers in turn
        const int pieces = kColumns / 64 * (MODE == GLU_FWD && a.save ? 3 : 1);
        for (int p = 0; p < pieces; ++p) {
          const int chunk = MODE == GLU_FWD && a.save ? p / 3 : p, what = MODE == GLU_FWD && a.save ? p % 3 : 0;
          const unsigned buf = out + (sent & 1) * kOutBytes;
          const int x = n0 + chunk * 64;
          if (x >= a.N || row0 >= a.M) continue;
          if (lane == 0) store_wait_read<1>();
          __syncwarp();
          for (int half = 0; half < 2; ++half) {
            float v[32];
            unsigned packed[16];
            const int col = chunk * 64 + half * 32;
            if (MODE == GLU_FWD && what == 0) {
              float u[32];
              tmem_load32(v, src + col);
              tmem_load32(u, src + BN / 2 + col);
              tmem_wait_loads();
              for (int i = 0; i < 16; ++i)
                packed[i] = pack2<E>(act_value<ACT>(v[2 * i]) * u[2 * i], act_value<ACT>(v[2 * i + 1]) * u[2 * i + 1]);
            } else {
              tmem_load32(v, src + col + (what == 2 ? BN / 2 : 0));
              tmem_wait_loads();
              for (int i = 0; i < 16; ++i) packed[i] = pack2<E>(v[2 * i], v[2 * i + 1]);
            }
            stage32(buf, lane, half, packed);
          }
          send(a, MODE == GLU_DW ? t.z : what, x, row0, buf, lane);
          ++sent;
        }
      } else if (row0 < a.M) {
        const bool mine = row0 + lane < a.M;
        if constexpr (MODE == GLU_FWD) {
          for (int col = 0; col < kColumns; col += 32) {
            float v[32], u[32];
            unsigned packed[16];
            tmem_load32(v, src + col);
            tmem_load32(u, src + BN / 2 + col);
            tmem_wait_loads();
            for (int i = 0; i < 16; ++i)
              packed[i] = pack2<E>(act_value<ACT>(v[2 * i]) * u[2 * i], act_value<ACT>(v[2 * i + 1]) * u[2 * i + 1]);
            if (mine) store_row(a, 0, n0 + col, row0 + lane, packed);
            if (a.save) {
              for (int i = 0; i < 16; ++i) packed[i] = pack2<E>(v[2 * i], v[2 * i + 1]);
              if (mine) store_row(a, 1, n0 + col, row0 + lane, packed);
              for (int i = 0; i < 16; ++i) packed[i] = pack2<E>(u[2 * i], u[2 * i + 1]);
              if (mine) store_row(a, 2, n0 + col, row0 + lane, packed);
            }
          }
        } else {
          for (int col = 0; col < kColumns; col += 32) {
            float v[32];
            unsigned packed[16];
            tmem_load32(v, src + col);
            tmem_wait_loads();
            for (int i = 0; i < 16; ++i) packed[i] = pack2<E>(v[2 * i], v[2 * i + 1]);
            if (mine) store_row(a, MODE == GLU_DW ? t.z : 0, n0 + col, row0 + lane, packed);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(smem_addr(&sh.acc_empty[acc]));
    }
    if (lane == 0) store_wait_all();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && sh.stop) record(a.status, COCODC_ERR_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    tmem_free(tmem, 2 * BN);
  }
}

// The parts of dx added in order.  Tiles are numbered as in the kernel above.
template <typename E, int BN> __global__ void __launch_bounds__(256) k_add_parts(const __grid_constant__ TcArgs a) {
  wait_for_previous();
  may_follow();
  const int per = a.m_tiles * a.n_tiles;
  const int tile = blockIdx.x / (kBM / 8), row = blockIdx.x % (kBM / 8) * 8 + threadIdx.x / 32;
  const TileAt t = tile_at<GLU_DX_PARTS>(a, tile);
  const int y = t.m * kBM + row;
  if (y >= a.M) return;
  for (int col = threadIdx.x % 32 * 2; col < BN; col += 64) {
    const int x = t.n * BN + col;
    if (x >= a.N) continue;
    float2 sum = make_float2(0.f, 0.f);
    for (int z = 0; z < a.splits; ++z) {
      const float2 v = *reinterpret_cast<const float2*>(a.parts + (((long long)z * per + tile) * kBM + row) * BN + col);
      sum.x += v.x;
      sum.y += v.y;
    }
    E* out = static_cast<E*>(a.out[0]) + y * a.ld[0] + x;
    out[0] = from_f32<E>(sum.x);
    if (x + 1 < a.N) out[1] = from_f32<E>(sum.y);
  }
}

}  // namespace cocodc_lm_impl
