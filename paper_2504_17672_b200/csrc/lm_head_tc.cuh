// Tensor-core kernel of the output head: the logits' statistics, the gradient of a piece of logits, and the two products with it.
//
// Persistent, 128 x (up to 256) tiles, k-blocks of 64, the roles of the gated block's kernel:
//   warp 0   producer: TMA copies of the operands' tiles into a ring of shared-memory stages
//   warp 1   issuer: tcgen05.mma of each stage into one of two TMEM accumulators of 256 columns
//   warps 2-9 epilogue, while the other accumulator fills; a thread has a row of the tile, two of them share it
// STATS     a tile of x W^T is reduced where it lies: each thread finds its row's largest logit and the sum of powers of two among the
//           tile's columns, and picks the target's logit; 8 bytes a row and tile leave the chip instead of 512.  The tensor cores cut the sums that
//           they accumulate instead of rounding them, always towards zero: the log-sum-exp of 2048 products came out 7.5e-7 to 9.4e-7 too small on average, 4.6e-7 at
//           1024.  So long contractions (LONG, from kLongBlocks k-blocks on) are accumulated in parts of at most kPartBlocks, which the epilogue adds in registers:
//           1.8e-7 to 2.1e-7 from 1024 on (sums rounded in fp32: 3e-8 to 8e-8), for 3 % of the time.
// DZ        the same product; the epilogue forms dz from the row's lse and factors and writes it in 16 bits, 64 staged columns at a time.
// PRODUCTS  dtable = dz^T x and dx = dz W of one piece in one launch: a tile's number tells which of the two it belongs to.  Tiles differ in
//           length, so that a block takes the next one when it is ready (a counter that DZ set back), the long ones first.  dx's sums over
//           the pieces of the vocabulary (and over parts of its contraction, where its tiles are few) stay in fp32 in an order of
//           their own, in which 32 lanes' accesses are 512 consecutive bytes.
// Measured alone (ncu), tensor pipe: 8192 x 2048 x 32000 LONG 758 us (1.42 PFLOP/s, 77 %; without parts 704 us, 83 %), DZ of 16128 columns 370-376 us
// (81 %), PRODUCTS of them 768 us (1.41 PFLOP/s, 84 %; with two and four copies for an MN-major operand's slabs 864 us, 66 %).  Back to back the power cap
// lowers the clock: 890-905 us forward, 2.74 ms backward.  dx and dtable in a launch each took 405 + 372 us, together 743.  Bringing
// tiles to L2 ahead of time made all of it slower (PRODUCTS 864 -> 925 us); what feeds the tensor cores is the way from L2, 49 KB a k-block.
// 1333 x 768 x 50257 LONG 99 us (15 rounds of tiles for 14.6; without parts 94).  One row of 2048 x 32000: 29 us, 20 of which are the table's bytes; 4 are the start and
// end of the kernel, 2 the joining one.
#pragma once

#include "lm_head.cuh"
#include "lm_mma.cuh"

namespace cocodc_lm_impl {

enum { HEAD_STATS = 0, HEAD_DZ = 1, HEAD_PRODUCTS = 2, HEAD_LONG = 3 };

struct HeadJob {             // one of the two products of HEAD_PRODUCTS
  int m_tiles, n_tiles, k_blocks, splits, tiles;
  int rows, cols;            // of the output
  unsigned a_bytes;
  Out o;
};
struct HeadTc {
  CUtensorMap a[2], b[2], c[2];   // STATS, DZ: x, table, dz; PRODUCTS: dtable's and dx's operands and outputs
  int m_tiles, n_tiles, k_blocks; // STATS, LONG, DZ
  int parts;                      // LONG: accumulations of a tile
  int width;                      // columns of a tile
  unsigned a_bytes;
  int slabs;                      // PRODUCTS: slabs of 64 columns that one copy brings: all of a tile, or one (see map_slabs)
  HeadArgs h;
  DzArgs d;
  HeadJob job[2];                 // dtable, dx
  int first;                      // which of them has the longer tiles: its come first
  int* counter;                   // tiles taken beyond one for each block; DZ sets it to 0
  long long first_row;            // of the piece, in the table
  int* status;
};

constexpr int kHeadStages = 4, kHeadEpilogue = 8, kHeadThreads = 64 + kHeadEpilogue * 32;
// Below 12 k-blocks the second accumulation costs more than 4 % (9 k-blocks: 270 -> 287 us, 12: 546 -> 562, 16: 452 -> 459 at 8192 rows) and the error is below 3e-7.
constexpr int kPartBlocks = 8, kLongBlocks = 12;
constexpr int kTileRing = 4;      // tiles that the producer may be ahead
constexpr unsigned kHeadStage = kABytes + 256 * kBK * 2, kHeadSmem = 1024 + kHeadStages * kHeadStage + kHeadEpilogue * kOutBytes;
// Tiles of consecutive rows that go through one column of tiles in turn (as in the gated block).
template <int MODE> constexpr int kHeadGroup = MODE == HEAD_PRODUCTS ? 8 : 32;

struct HeadShared {
  unsigned long long full[kHeadStages], empty[kHeadStages], acc_full[2], acc_empty[2], tile_full[kTileRing], tile_empty[kTileRing], drain;
  int tile[kTileRing];
  unsigned tmem;
  int stop;
};

struct HeadTile { int kind, z, m, n, number, kb0, kb1; };
template <int MODE> __device__ __forceinline__ HeadTile head_tile(const HeadTc& a, int tile) {
  HeadTile t{};
  int m_tiles = a.m_tiles, n_tiles = a.n_tiles;
  t.kb1 = a.k_blocks;
  if (MODE == HEAD_PRODUCTS) {
    t.kind = tile < a.job[a.first].tiles ? a.first : 1 - a.first;
    const HeadJob& j = a.job[t.kind];
    if (t.kind != a.first) tile -= a.job[a.first].tiles;
    m_tiles = j.m_tiles;
    n_tiles = j.n_tiles;
    const int per = m_tiles * n_tiles;
    t.number = tile;
    t.z = tile / per;
    tile -= t.z * per;
    t.kb0 = (int)((long long)j.k_blocks * t.z / j.splits);
    t.kb1 = (int)((long long)j.k_blocks * (t.z + 1) / j.splits);
  }
  const int group = tile / (kHeadGroup<MODE> * n_tiles), first = group * kHeadGroup<MODE>;
  const int height = min(kHeadGroup<MODE>, m_tiles - first);
  tile -= group * kHeadGroup<MODE> * n_tiles;
  t.m = first + tile % height;
  t.n = tile / height;
  return t;
}

// Adds fp32 numbers of a staged tile to a matrix.
__device__ __forceinline__ void tma_add(const CUtensorMap* map, int x, int y, unsigned src) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.bulk_group [%0, {%1, %2}], [%3];"
               ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}

// Slabs of 64 columns (from number `slab` on) of 64 rows, one behind the other.
__device__ __forceinline__ void tma_load_slabs(unsigned dst, const CUtensorMap* map, int row, int slab, unsigned bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(0), "r"(row), "r"(slab), "r"(bar) : "memory");
}

// The sums of a tile: 32 columns (col, col + 1, ...) of a thread's row
__device__ __forceinline__ float4* sums_at(const Out& o, int number, int width, int col, int row) {
  return reinterpret_cast<float4*>(o.sums) + ((long long)number * width + col) / 4 * kBM + row;
}

// 32 columns of the thread's row of an output on their way: staged (16 bits: two halves of a staged tile; fp32: one), sent when the
// staged tile is complete.  Columns and rows outside are not written; what a copy cannot write alone (the last columns, where a row's
// width is no multiple of 16 bytes) leaves by ordinary stores.
template <typename E>
__device__ __forceinline__ void emit(const Out& o, const CUtensorMap* map, int rows, int cols, int x, int y, int half, unsigned buf, int lane, float (&v)[32]) {
  if (o.type == COCODC_F32) {
    float* row = static_cast<float*>(o.out) + (long long)(y + lane) * o.ld + x;
    if (cols - x >= 32 || cols % 4 == 0) {
#pragma unroll
      for (int q = 0; q < 8; ++q)
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + ((q ^ (lane & 7)) << 4)), "f"(v[4 * q]), "f"(v[4 * q + 1]),
                     "f"(v[4 * q + 2]), "f"(v[4 * q + 3]) : "memory");
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        if (o.accumulate) tma_add(map, x, y, buf);
        else tma_store(map, x, y, buf);
      }
    } else if (y + lane < rows) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (x + i < cols) row[i] = o.accumulate ? row[i] + v[i] : v[i];
    }
    if (lane == 0) store_commit();
    return;
  }
  E* row = static_cast<E*>(o.out) + (long long)(y + lane) * o.ld + x;
  const int x0 = x - 32 * half;                       // of the staged tile
  const bool by_copy = !o.accumulate && (cols - x0 >= 64 || cols % 8 == 0);
  if (by_copy) {
    unsigned packed[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) packed[i] = pack2<E>(v[2 * i], v[2 * i + 1]);
    stage32(buf, lane, half, packed);
    if (half == 1) {
      fence_async_smem();
      __syncwarp();
      if (lane == 0) tma_store(map, x0, y, buf);
    }
  } else if (y + lane < rows) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (x + i < cols) row[i] = from_f32<E>(o.accumulate ? to_f32(row[i]) + v[i] : v[i]);
  }
  if (half == 1 && lane == 0) store_commit();
}

template <typename E, int MODE>
__global__ void __launch_bounds__(kHeadThreads, 1) k_head_tc(const __grid_constant__ HeadTc a) {
  extern __shared__ unsigned char dyn[];
  __shared__ HeadShared sh;
  const unsigned base = (smem_addr(dyn) + 1023u) & ~1023u;
  const unsigned staging = base + kHeadStages * kHeadStage;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int tiles = MODE == HEAD_PRODUCTS ? a.job[0].tiles + a.job[1].tiles : a.m_tiles * a.n_tiles;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kHeadStages; ++s) {
      bar_init(smem_addr(&sh.full[s]), 1);
      bar_init(smem_addr(&sh.empty[s]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(smem_addr(&sh.acc_full[i]), 1);
      bar_init(smem_addr(&sh.acc_empty[i]), kHeadEpilogue);
    }
    for (int i = 0; i < kTileRing; ++i) {
      bar_init(smem_addr(&sh.tile_full[i]), 1);
      bar_init(smem_addr(&sh.tile_empty[i]), 1 + kHeadEpilogue);
    }
    bar_init(smem_addr(&sh.drain), 1);
    sh.stop = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  wait_for_previous();                                // before TMEM is taken, and the next kernel's blocks come only after
  if (warp == 1) tmem_alloc(smem_addr(&sh.tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  may_follow();
  const unsigned tmem = sh.tmem;
  volatile int* stop = &sh.stop;
  if (MODE == HEAD_DZ && blockIdx.x == 0 && threadIdx.x == 0) *a.counter = 0;

  // The block's n-th tile: -1 behind the last, -2 when a wait gave up.  PRODUCTS: as the producer published it; who has read it gives its place back.
  const auto nth_tile = [&](int n) -> int {
    if (MODE != HEAD_PRODUCTS) {
      const long long tile = blockIdx.x + (long long)n * gridDim.x;
      return tile < tiles ? (int)tile : -1;
    }
    const int slot = n % kTileRing;
    if (!bar_wait(smem_addr(&sh.tile_full[slot]), (unsigned)(n / kTileRing) & 1, stop)) return -2;
    return *reinterpret_cast<volatile int*>(&sh.tile[slot]);
  };
  const auto tile_read = [&](int n) {
    if (MODE == HEAD_PRODUCTS) bar_arrive(smem_addr(&sh.tile_empty[n % kTileRing]));
  };

  if (warp == 0) {
    if (lane == 0) {
      long long it = 0;
      bool ok = true;
      const int slabs = a.width / 64;
      int next = blockIdx.x;
      for (int n = 0; ok; ++n) {
        int tile = next;
        if (MODE == HEAD_PRODUCTS) {
          const int slot = n % kTileRing;
          if (tile >= tiles) tile = -1;
          else next = gridDim.x + atomicAdd(a.counter, 1);            // comes while this tile is fetched
          ok = bar_wait(smem_addr(&sh.tile_empty[slot]), ((unsigned)(n / kTileRing) & 1) ^ 1, stop);
          if (!ok) break;
          *reinterpret_cast<volatile int*>(&sh.tile[slot]) = tile;
          bar_arrive(smem_addr(&sh.tile_full[slot]));
        } else {
          tile = nth_tile(n);
        }
        if (tile < 0) break;
        const HeadTile t = head_tile<MODE>(a, tile);
        const int m0 = t.m * kBM, n0 = t.n * a.width;
        const unsigned bytes = MODE == HEAD_PRODUCTS ? a.job[t.kind].a_bytes + slabs * kSlab : a.a_bytes + a.width * kBK * 2;
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const int s = (int)(it % kHeadStages), k0 = kb * kBK;
          ok = bar_wait(smem_addr(&sh.empty[s]), (unsigned)((it / kHeadStages) & 1) ^ 1, stop);
          if (!ok) break;
          const unsigned full = smem_addr(&sh.full[s]), sa = base + s * kHeadStage, sb = sa + kABytes;
          bar_expect(full, bytes);
          if (MODE != HEAD_PRODUCTS) {
            tma_load(sa, &a.a[0], k0, m0, full);
            tma_load(sb, &a.b[0], k0, (int)a.first_row + n0, full);
          } else {
            if (t.kind == 0) tma_load_slabs(sa, &a.a[0], k0, m0 / 64, full);
            else tma_load(sa, &a.a[1], k0, m0, full);
            const int row = t.kind == 0 ? k0 : (int)a.first_row + k0;
            if (a.slabs > 1) tma_load_slabs(sb, &a.b[t.kind], row, n0 / 64, full);
            else
              for (int i = 0; i < slabs; ++i) tma_load(sb + i * kSlab, &a.b[t.kind], n0 + i * 64, row, full);
          }
        }
      }
      // the issuer's last arrivals come before the CTA leaves
      for (long long i = it > kHeadStages ? it - kHeadStages : 0; ok && i < it; ++i)
        ok = bar_wait(smem_addr(&sh.empty[i % kHeadStages]), (unsigned)((i / kHeadStages) & 1), stop);
      // given up: the copies in flight land before the CTA leaves its shared memory
      if (!ok)
        for (long long i = it > kHeadStages ? it - kHeadStages : 0; i < it; ++i)
          bar_drain(smem_addr(&sh.full[i % kHeadStages]), (unsigned)((i / kHeadStages) & 1));
    }
  } else if (warp == 1) {
    if (lane == 0) {
      long long it = 0;
      int sum = 0;                                     // accumulations so far
      const int parts = MODE == HEAD_LONG ? a.parts : 1, each = a.k_blocks / parts, rest = a.k_blocks % parts;
      bool ok = true;
      for (int turn = 0; ok; ++turn) {
        const int tile = nth_tile(turn);
        tile_read(turn);
        if (tile < 0) {
          ok = tile == -1;
          break;
        }
        const HeadTile t = head_tile<MODE>(a, tile);
        const bool a_mn = MODE == HEAD_PRODUCTS && t.kind == 0;
        constexpr bool b_mn = MODE == HEAD_PRODUCTS;
        const unsigned idesc = instr_desc<E>(kBM, a.width, a_mn, b_mn);
        int last = t.kb0, over = 0;                     // LONG: part q ends at k-block floor(k_blocks (q + 1) / parts)
        for (int q = 0; ok && q < parts; ++q, ++sum) {
          const int acc = sum & 1, first = last;
          last = t.kb1;
          if (MODE == HEAD_LONG) {
            over += rest;
            last = first + each + (over >= parts);
            if (over >= parts) over -= parts;
          }
          ok = bar_wait(smem_addr(&sh.acc_empty[acc]), (unsigned)((sum >> 1) & 1) ^ 1, stop);
          tc_fence_after();
          for (int kb = first; ok && kb < last; ++kb, ++it) {
            const int s = (int)(it % kHeadStages);
            ok = bar_wait(smem_addr(&sh.full[s]), (unsigned)((it / kHeadStages) & 1), stop);
            if (!ok) break;
            tc_fence_after();
            const unsigned sa = base + s * kHeadStage, sb = sa + kABytes;
            const unsigned long long da = tile_desc(sa, a_mn ? kSlab : 16), db = tile_desc(sb, b_mn ? kSlab : 16);
            const unsigned ka = a_mn ? 2048 >> 4 : 32 >> 4;   // 16 k: 32 bytes along a K-major row, 16 rows of an MN-major tile
            constexpr unsigned kb16 = b_mn ? 2048 >> 4 : 32 >> 4;
            for (int k = 0; k < kBK / 16; ++k) tc_mma(tmem + acc * 256, da + k * ka, db + k * kb16, idesc, kb > first || k > 0);
            tc_commit(smem_addr(&sh.empty[s]));
          }
          if (ok) tc_commit(smem_addr(&sh.acc_full[acc]));
        }
      }
      if (!ok) {
        tc_commit(smem_addr(&sh.drain));
        bar_drain(smem_addr(&sh.drain), 0);
      }
    }
  } else {
    // a warp reaches the 32 TMEM lanes of its number modulo 4; of two such warps one takes the even, one the odd pieces of the columns
    const int quarter = warp & 3, part = (warp - 2) / 4;
    const unsigned buf = staging + (warp - 2) * kOutBytes;
    int sum = 0;
    for (int turn = 0;; ++turn) {
      const int tile = nth_tile(turn);
      if (!__all_sync(~0u, tile >= 0)) break;          // every lane has read it
      if (lane == 0) tile_read(turn);
      const HeadTile t = head_tile<MODE>(a, tile);
      const int row0 = t.m * kBM + quarter * 32, n0 = t.n * a.width;
      const long long row = row0 + lane;
      // what the row needs is on its way while the tile's products run
      long long target = -1;
      RowOf r{};
      if ((MODE == HEAD_STATS || MODE == HEAD_LONG) && a.h.targets && row < a.h.T) target = raw_target(a.h.targets, a.h.targets64, row);
      if (MODE == HEAD_DZ && row < a.d.T) {
        r = row_of(a.d, row);
        target = r.y;
      }
      if constexpr (MODE == HEAD_STATS || MODE == HEAD_LONG) {
        const int cols = (int)min((long long)a.width, a.h.V - n0);
        const int hit = target >= n0 && target < n0 + cols ? (int)(target - n0) : -1;
        float m = -INFINITY, s = 0.f;
        const auto reduce = [&](float (&v)[32], int col) {
          if (cols - col < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (i >= cols - col) v[i] = -INFINITY;
          }
          float most[4] = {v[0], v[1], v[2], v[3]}, sums[4] = {0.f, 0.f, 0.f, 0.f};       // four chains: one waits for itself
#pragma unroll
          for (int i = 4; i < 32; ++i) most[i % 4] = fmaxf(most[i % 4], v[i]);
          const float now = fmaxf(m, fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]))), shift = shift_of(now) * a.h.scale2;
          s *= fast_exp2(fmaf(m, a.h.scale2, -shift));
          m = now;
#pragma unroll
          for (int i = 0; i < 32; ++i) sums[i % 4] += fast_exp2(fmaf(v[i], a.h.scale2, -shift));
          s += (sums[0] + sums[1]) + (sums[2] + sums[3]);
          const int at = hit - col;
          if (__any_sync(~0u, at >= 0 && at < 32)) {
            float picked = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (i == at) picked = v[i];
            if (at >= 0 && at < 32 && row < a.h.T) a.h.picked[row] = picked * a.h.scale2;
          }
        };
        float z[MODE == HEAD_LONG ? 4 : 1][32];         // LONG: sums of the parts; the thread's columns are the pieces part, part + 2, ... of 32
        const int parts = MODE == HEAD_LONG ? a.parts : 1;
        bool ok = true;
        for (int q = 0; ok && q < parts; ++q, ++sum) {
          const int acc = sum & 1;
          ok = __all_sync(~0u, bar_wait(smem_addr(&sh.acc_full[acc]), (unsigned)((sum >> 1) & 1), stop));
          if (!ok) break;
          tc_fence_after();
          const unsigned src = tmem + acc * 256 + ((unsigned)(quarter * 32) << 16);
          if constexpr (MODE == HEAD_LONG) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              const int col = (2 * p + part) * 32;
              if (col >= cols) continue;
              if (q == 0) {
                tmem_load32(z[p], src + col);
                tmem_wait_loads();
              } else {
                float v[32];
                tmem_load32(v, src + col);
                tmem_wait_loads();
#pragma unroll
                for (int i = 0; i < 32; ++i) z[p][i] += v[i];
              }
            }
          } else {
            for (int col = part * 32; col < cols; col += 64) {
              tmem_load32(z[0], src + col);
              tmem_wait_loads();
              reduce(z[0], col);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(smem_addr(&sh.acc_empty[acc]));
        }
        if (!ok) break;
        if constexpr (MODE == HEAD_LONG) {
#pragma unroll
          for (int p = 0; p < 4; ++p)
            if ((2 * p + part) * 32 < cols) reduce(z[p], (2 * p + part) * 32);
        }
        if (row < a.h.T) a.h.stats[(2ll * t.n + part) * a.h.T + row] = make_float2(m * a.h.scale2, s);
        continue;
      }
      const int acc = turn & 1;
      const unsigned src = tmem + acc * 256 + ((unsigned)(quarter * 32) << 16);
      if (!__all_sync(~0u, bar_wait(smem_addr(&sh.acc_full[acc]), (unsigned)((turn >> 1) & 1), stop))) break;
      tc_fence_after();
      if constexpr (MODE == HEAD_DZ) {
        const int cols = (int)min((long long)a.width, a.d.v1 - a.d.v0 - n0);
        const bool nothing = r.lse2 == INFINITY;
        const long long hit = target < 0 ? -1 : target - a.d.v0 - n0;
        Out o{};
        o.out = a.d.dz;
        o.type = COCODC_BF16;
        o.ld = a.d.pitch;
        if (row0 < a.d.T)
          for (int x0 = part * 64; x0 < cols; x0 += 128) {
            if (lane == 0) store_wait_read<0>();
            __syncwarp();
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const int col = x0 + half * 32;
              float v[32];
              tmem_load32(v, src + col);
              tmem_wait_loads();
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = fast_exp2(fmaf(v[i], a.d.scale2, -r.lse2)) * r.slope;
              if (__any_sync(~0u, hit >= col && hit < col + 32)) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] += i == (int)(hit - col) ? r.hit : 0.f;
              }
              if (nothing) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = 0.f;
              }
              emit<E>(o, &a.c[0], (int)a.d.T, (int)(a.d.v1 - a.d.v0), n0 + col, row0, half, buf, lane, v);
            }
          }
      } else {
        const HeadJob& j = a.job[t.kind];
        const Out& o = j.o;
        const Back back(o);
        const bool keep = o.sums && !o.last, whole = o.type == COCODC_F32;   // 32 columns of fp32 are a staged tile of their own
        // the last piece of the vocabulary can have fewer k-blocks than dx has parts: no product ran for such a part, and the accumulator holds an older tile's
        const bool empty = t.kb0 == t.kb1;
        if (row0 < j.rows)
          for (int x0 = part * 64; x0 < a.width && n0 + x0 < j.cols; x0 += 128) {
            for (int half = 0; half < 2; ++half) {
              const int col = x0 + half * 32, x = n0 + col;
              if (whole && x >= j.cols) break;
              float v[32];
              tmem_load32(v, src + col);
              tmem_wait_loads();
              if (empty) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = 0.f;
              }
              float4* sums = sums_at(o, t.number, a.width, col, quarter * 32 + lane);
              if (o.sums && o.add) {
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                  const float4 u = sums[q * kBM];
                  v[4 * q] += u.x;
                  v[4 * q + 1] += u.y;
                  v[4 * q + 2] += u.z;
                  v[4 * q + 3] += u.w;
                }
              }
              if (keep) {
#pragma unroll
                for (int q = 0; q < 8; ++q) sums[q * kBM] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                continue;
              }
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = back(v[i]);
              if (whole || half == 0) {
                if (lane == 0) store_wait_read<0>();
                __syncwarp();
              }
              emit<E>(o, &a.c[t.kind], j.rows, j.cols, x, row0, half, buf, lane, v);
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
    tmem_free(tmem, 512);
  }
}

// The parts of dx's sums added in order, and out: a block takes eight rows and 128 columns of a tile.
template <typename E> __global__ void __launch_bounds__(256) k_head_add(const __grid_constant__ HeadTc a) {
  wait_for_previous();
  may_follow();
  const HeadJob& j = a.job[1];
  const int per = j.m_tiles * j.n_tiles, tile = blockIdx.x / (kBM / 8), row = blockIdx.x % (kBM / 8) * 8 + threadIdx.x % 8;
  const HeadTile t = head_tile<HEAD_PRODUCTS>(a, (a.first == 1 ? 0 : a.job[0].tiles) + tile);
  const int y = t.m * kBM + row, col = blockIdx.y * 128 + threadIdx.x / 8 * 4, x = t.n * a.width + col;
  if (y >= j.rows || col >= a.width || x >= j.cols) return;
  const Back back(j.o);
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int z = 0; z < j.splits; z += 4) {
    float4 u[4];                                                      // together on their way
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = z + k < j.splits ? *sums_at(j.o, (z + k) * per + tile, a.width, col, row) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[0] += u[k].x;
      v[1] += u[k].y;
      v[2] += u[k].z;
      v[3] += u[k].w;
    }
  }
  E* out = static_cast<E*>(j.o.out) + y * j.o.ld + x;
  for (int i = 0; i < 4; ++i)
    if (x + i < j.cols) out[i] = from_f32<E>(back(v[i]));
}

}  // namespace cocodc_lm_impl
