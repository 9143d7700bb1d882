// A persistent bf16 matrix product on CTA pairs: tiles of D = A B^T, 256 columns wide and 256 or 512 rows high, fp32 sums in
// tensor memory, the epilogue supplied by the caller.
//
// Two CTAs of a cluster (two SMs) work on one tile.  Each holds half of A's rows and half of B's: 16 KiB for each 256 rows
// of the tile and 16 KiB of B a stage of 64 columns of K, brought by TMA (128-byte swizzle) into a ring of stages.  One thread
// of the even CTA issues the matrix instructions of both (M 256, N 256, K 16); each CTA's tensor memory receives its 128 rows
// of each 256, in one of two accumulators of 256 columns.
//
//   kHigh = 1  256 rows: the accumulators alternate, the epilogue of one runs beside the products into the other
//   kHigh = 2  512 rows: both accumulators belong to one tile and share its B, which takes 48 KiB from L2 where two lower
//              tiles take 64.  A long product runs at the card's power limit, and bytes moved from L2 are what is left to
//              save there; the epilogues of its halves run beside kMmaLead stages of products of the other half
//
// Operands need not be stored with K innermost: `kMn` operands have the tile's own dimension innermost (a row of the matrix
// in memory per K index), as P and x in dW = P^T x; TMA brings 64 x 64 boxes either way and the descriptor says which.
//
// Warps: 0 TMA, 1 matrix instructions (even CTA), 2 tensor memory, 4..11 epilogue: quarter w % 4 of the rows, columns
// [0, 128) for 4..7 and [128, 256) for 8..11.
//
// Every wait is bounded (mma_wait_limit).  A role that gives up stops issuing; before the pair leaves, the loads
// and products under way are waited for once more, bounded again, and the tensor memory is freed.
#pragma once
#include <cuda.h>

#include "bulk_copy.cuh"
#include "operators.cuh"

namespace ft {

constexpr uint32_t kMmaTile = 256;    // rows of an accumulator over the pair, columns of a tile
constexpr uint32_t kMmaK = 64;        // K a stage: 128 bytes of bf16
constexpr uint32_t kMmaBox = 64 * kMmaK * 2;         // one TMA box, 8 KiB
constexpr uint32_t kMmaOperand = 2 * kMmaBox;        // a CTA's half of 256 rows of an operand, a stage
// Stages by which a high tile's rows 0..255 run ahead of the others at its beginning and its end: the epilogue of one half then
// runs beside products of the other on both sides.  2460 rows x 32768 x 1024: 128 us, 135 without it; 4, the whole ring, is no better.
constexpr uint32_t kMmaLead = 3;
template <int kHigh>
constexpr int kMmaStages = kHigh == 1 ? 6 : 4;
constexpr int kMmaThreads = 384;
constexpr int kMmaEpilogueWarps = 8;
constexpr size_t kMmaRing = 6 * 2 * kMmaOperand;     // the stages of either height: 192 KiB
constexpr uint32_t kMmaOut = 32 * 128;                // an epilogue warp's staging: its 32 rows, 128 bytes each
constexpr size_t kMmaSmem = kMmaRing + kMmaEpilogueWarps * kMmaOut + 1024 + 256;  // on a 1 KiB boundary; last the barriers

struct MmaBarriers {
  uint64_t full[6], empty[6], acc_full[2], acc_empty[2], drain;
  uint32_t tmem, lost;
};
static_assert(sizeof(MmaBarriers) <= 256 && kMmaStages<2> * 3 * kMmaOperand <= kMmaRing, "kMmaSmem");

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address of the same shared-memory object in the pair's even CTA
__device__ __forceinline__ uint32_t in_even_cta(const void* p) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(p)));
  return r;
}
__device__ __forceinline__ bool mbar_try_wait_cluster(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
  return ok != 0;
}
// false: the barrier's phase did not complete within the limit
__device__ __forceinline__ bool mbar_wait_bounded(uint64_t* b, uint32_t parity, uint64_t limit_ns) {
  if (mbar_try_wait_cluster(b, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  uint32_t spins = 0;
  while (!mbar_try_wait_cluster(b, parity))
    if ((++spins & 1023u) == 0 && global_timer_ns() - t0 > limit_ns) return false;
  return true;
}
// Relaxed: what it stands for is a read of tensor memory that tcgen05.wait::ld has seen complete and tcgen05.fence orders.  With
// release it also waits for the stores that the thread has under way, 1300 cycles a time.
__device__ __forceinline__ void mbar_arrive_at(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// one 64 x 64 box to this CTA, its bytes counted on the even CTA's barrier
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
// arrives on the barrier of both CTAs once the products issued so far are done
__device__ __forceinline__ void mma_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(smem_u32(b)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void mma_issue(uint32_t tmem, uint64_t da, uint64_t db, uint32_t idesc, bool add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
               "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(tmem), "l"(da), "l"(db), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// Columns of the warp's 32 rows, 32 a load; the whole warp takes part.  The values are there behind tmem_wait().
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32]) {
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// An epilogue warp's way out: 32 rows of 128 bytes (64 bf16 or 32 fp32 columns) are written into its staging in the 128-byte
// swizzle, and one TMA store takes them to the matrix, clipped at its extents.  Direct stores put a warp's 32 rows into 32 lines
// an instruction and cost more cycles than the rest of the epilogue (see k_dw).
struct MmaOut {
  uint32_t stage;  // shared-memory address of the warp's staging
  __device__ __forceinline__ MmaOut() {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t ring = (smem_u32(smem_raw) + 1023) & ~1023u;
    stage = ring + (uint32_t)kMmaRing + ((threadIdx.x >> 5) & 7) * kMmaOut;  // warps 4..11
  }
  // the lane's row: value v(j) gives 16 bytes of it, j = 0..7.  kAdd: the fp32 values are added to what the matrix holds
  template <bool kAdd, class F>
  __device__ __forceinline__ void put(const CUtensorMap* map, int32_t x, int32_t y, F&& v) const {
    const uint32_t lane = threadIdx.x & 31;
    if (lane == 0) bulk_wait_read<0>();  // the staging's last store has read it
    __syncwarp();
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      const uint4 w = v(j);
      store_shared16(stage + lane * 128 + ((j ^ (lane & 7)) << 4), w);
    }
    fence_async_smem();
    __syncwarp();
    if (lane == 0) {
      if constexpr (kAdd)
        asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(stage), "r"(x), "r"(y) : "memory");
      else
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(stage), "r"(x), "r"(y) : "memory");
      bulk_commit();
    }
  }
  // all stores of the warp have reached memory
  __device__ __forceinline__ void done() const {
    if ((threadIdx.x & 31) == 0) bulk_wait_all<0>();
    __syncwarp();
  }
};

// Shared-memory descriptor (PTX ISA, "matrix descriptor"): bits 0-13 address / 16, 16-29 leading offset / 16, 32-45 stride
// offset / 16, 46-47 = 1, 61-63 = 2 for the 128-byte swizzle.
//   K innermost: rows of 128 bytes, groups of eight rows 1 KiB apart (stride offset); the leading offset is not used
//   tile dimension innermost: 64 elements of it a row of 128 bytes, eight K indices in 1 KiB (stride offset), the next 64
//   elements one box further (leading offset)
template <bool kMn>
__device__ __forceinline__ uint64_t mma_desc(uint32_t addr) {
  constexpr uint64_t kLead = kMn ? kMmaBox >> 4 : 1, kStride = 1024 >> 4;
  return (uint64_t)((addr & 0x3FFFF) >> 4) | kLead << 16 | kStride << 32 | 1ull << 46 | 2ull << 61;
}
// 16 further along K: 32 bytes of a row, or 16 rows
template <bool kMn>
constexpr uint32_t kMmaStep = kMn ? 2048 : 32;

// fp32 sums of bf16 x bf16, M 256, N 256; bits 15 and 16: A, B with the tile dimension innermost
template <bool kAMn, bool kBMn>
constexpr uint32_t kMmaInstr = 1u << 4 | 1u << 7 | 1u << 10 | (kAMn ? 1u << 15 : 0) | (kBMn ? 1u << 16 : 0) | (256 >> 3) << 17 | (256 >> 4) << 24;

// One tile of work: rows from m (256 times `high` of them; none: nothing to do), columns from n, K blocks [k0, k1).  From block
// `again` on, A begins once more at its first block.
struct MmaTile {
  uint32_t m, n, k0, k1, high, again = kNone;
};

// Bound of a wait inside a tile: the pool's limit, which is meant for one load, but never less than what the tile's products may take.
// A block of K of 512 rows takes a pair 0.52 us at the card's highest clock (1024 cycles), 0.8 at its power limit; 4 leave room for a
// device that others use too, the millisecond for an epilogue behind other traffic.  The test hook's waits are to run out: the limit itself.
__device__ __forceinline__ uint64_t mma_wait_limit(const PoolView& v, uint32_t k_blocks) {
  return v.bulk_tx_slack ? v.bulk_wait_ns : max(v.bulk_wait_ns, (uint64_t)1000000 + (uint64_t)k_blocks * 4000);
}

// Runs the tiles pair, pair + pairs, ... below `n_tiles`.  tile_at(i) -> MmaTile; every epilogue warp calls
// epilogue(tile, i, tmem, row, col0, release) for each 256 rows: tensor memory from `tmem` on holds 128 columns of its 32 rows, lane
// l the row `row` + l of the tile, columns col0 .. col0 + 127.  It may call release() as soon as it has read them.  A tile
// without K blocks has tmem = kNone: all sums are zero.  before(tile, row) is called ahead of the wait for the products, for
// what the epilogue reads from memory.
template <bool kAMn, bool kBMn, int kHigh, class TileAt, class Before, class Epilogue>
__device__ __forceinline__ void mma_pair_tiles(const CUtensorMap& map_a, const CUtensorMap& map_b, uint32_t n_tiles, const PoolView& v, bool* lost_out,
                                               TileAt tile_at, Before before, Epilogue epilogue) {
  extern __shared__ uint8_t smem_raw[];
  constexpr uint32_t kStages = kMmaStages<kHigh>, kStageBytes = (kHigh + 1) * kMmaOperand;
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  MmaBarriers* bar = reinterpret_cast<MmaBarriers*>(stages + kMmaRing + kMmaEpilogueWarps * kMmaOut);
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = cluster_rank();
  const uint32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < kStages; ++s) { mbar_init(&bar->full[s], 1); mbar_init(&bar->empty[s], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&bar->acc_full[i], 1); mbar_init(&bar->acc_empty[i], 2 * kMmaEpilogueWarps); }
    mbar_init(&bar->drain, 1);
    bar->lost = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bar->tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = bar->tmem, base = smem_u32(stages);
  bool lost = false;
  uint32_t it = 0;            // stages used so far
  uint32_t used[2] = {0, 0};  // times each accumulator was used so far
  uint32_t turn = 0;          // kHigh = 1: the accumulator that is next
  const uint64_t last_limit_ns = mma_wait_limit(v, 0);  // behind the last tile
  if (warp < 4) {
    if (warp == 0 && lane == 0) {
      for (uint32_t i = pair; i < n_tiles && !lost; i += pairs) {
        const MmaTile t = tile_at(i);
        if (t.high == 0) continue;
        const uint64_t limit_ns = mma_wait_limit(v, t.k1 - t.k0);
        const int32_t a0 = (int32_t)(t.m + rank * 128), b0 = (int32_t)(t.n + rank * 128);
        for (uint32_t k = t.k0; k < t.k1; ++k, ++it) {
          const uint32_t s = it % kStages;
          if (!mbar_wait_bounded(&bar->empty[s], ((it / kStages) & 1) ^ 1, limit_ns)) { lost = true; break; }
          if (rank == 0) mbar_expect_tx(&bar->full[s], 2 * (t.high + 1) * kMmaOperand + v.bulk_tx_slack);  // the slack: a test hook, 0
          const uint32_t full = in_even_cta(&bar->full[s]), sb = base + s * kStageBytes;
          const int32_t kk = (int32_t)(k * kMmaK), ka = (int32_t)((k < t.again ? k : k - t.again) * kMmaK);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (kBMn) tma_box(sb + h * kMmaBox, &map_b, b0 + 64 * h, kk, full);
            else tma_box(sb + h * kMmaBox, &map_b, kk, b0 + 64 * h, full);
          }
#pragma unroll
          for (int h = 0; h < 2 * kHigh; ++h) {
            if (h >= 2 && t.high < 2) break;
            const int32_t row = a0 + 64 * (h & 1) + (int32_t)kMmaTile * (h >> 1);
            if (kAMn) tma_box(sb + kMmaOperand + h * kMmaBox, &map_a, row, ka, full);
            else tma_box(sb + kMmaOperand + h * kMmaBox, &map_a, ka, row, full);
          }
        }
      }
      // what still arrives in this CTA's shared memory: the loads of the last stages (both CTAs' bytes are counted in the
      // even one), and the even CTA's signals that it is done with them
      const uint32_t j0 = it > kStages ? it - kStages : 0;
      if (lost && rank == 0)
        for (uint32_t j = j0; j < it; ++j) mbar_wait_bounded(&bar->full[j % kStages], (j / kStages) & 1, last_limit_ns);
      for (uint32_t j = j0; j < it && !lost; ++j) lost = !mbar_wait_bounded(&bar->empty[j % kStages], (j / kStages) & 1, last_limit_ns);
    } else if (warp == 1 && lane == 0 && rank == 0) {
      uint64_t limit_ns = 0;
      const auto take = [&](uint32_t acc) {  // waits until the accumulator's last user has read it
        if (!mbar_wait_bounded(&bar->acc_empty[acc], (used[acc]++ & 1) ^ 1, limit_ns)) lost = true;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      };
      for (uint32_t i = pair; i < n_tiles && !lost; i += pairs) {
        const MmaTile t = tile_at(i);
        if (t.high == 0 || t.k0 == t.k1) continue;
        const uint32_t acc0 = kHigh == 1 ? turn : 0;
        turn ^= 1;
        limit_ns = mma_wait_limit(v, t.k1 - t.k0);
        take(acc0);
        const auto arrived = [&](uint32_t i) {  // the stage's operands are in both CTAs
          if (!mbar_wait_bounded(&bar->full[i % kStages], (i / kStages) & 1, limit_ns)) lost = true;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          return !lost;
        };
        const auto products = [&](uint32_t h, uint32_t i, bool add) {
          const uint32_t sb = base + i % kStages * kStageBytes, sa = sb + (1 + h) * kMmaOperand;
#pragma unroll
          for (uint32_t j = 0; j < kMmaK / 16; ++j)
            mma_issue(tmem + (acc0 + h) * 256, mma_desc<kAMn>(sa + j * kMmaStep<kAMn>), mma_desc<kBMn>(sb + j * kMmaStep<kBMn>),
                      kMmaInstr<kAMn, kBMn>, add || j > 0);
        };
        const uint32_t ks = t.k1 - t.k0;
        uint32_t k = 0;  // K blocks whose products have been issued
        const auto ahead = [&](uint32_t blocks) {
          for (uint32_t g = 0; g < blocks && arrived(it + g); ++g) products(0, it + g, k + g > 0);
          if (lost) return;
          if (k + blocks == ks) mma_commit(&bar->acc_full[0]);
          if (k == 0) take(1);
          if (lost) return;
          for (uint32_t g = 0; g < blocks; ++g) {
            products(1, it + g, k + g > 0);
            mma_commit(&bar->empty[(it + g) % kStages]);
          }
          if (k + blocks == ks) mma_commit(&bar->acc_full[1]);
          it += blocks;
          k += blocks;
        };
        const bool two = kHigh == 2 && t.high == 2;
        if (two) ahead(min(kMmaLead, ks));
        const uint32_t last = two ? min(kMmaLead, ks - k) : 0;
        for (; k + last < ks && !lost; ++k, ++it) {
          if (!arrived(it)) break;
          products(0, it, k > 0);
          if (two) products(1, it, true);
          mma_commit(&bar->empty[it % kStages]);
        }
        if (lost) break;
        if (!two) mma_commit(&bar->acc_full[acc0]);
        else if (last) ahead(last);
      }
      if (lost) {  // products under way still read shared memory and write tensor memory
        mma_commit(&bar->drain);
        mbar_wait_bounded(&bar->drain, 0, last_limit_ns);
      }
    }
  } else {
    const uint32_t quarter = warp & 3, half = (warp - 4) >> 2, col0 = half * 128;
    uint32_t acc = 0;
    bool held = false;
    const auto release = [&] {
      if (!held) return;
      held = false;
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive_at(in_even_cta(&bar->acc_empty[acc]));
    };
    for (uint32_t i = pair; i < n_tiles && !lost; i += pairs) {
      const MmaTile t = tile_at(i);
      const uint64_t limit_ns = mma_wait_limit(v, t.k1 - t.k0);
      for (uint32_t h = 0; h < t.high && !lost; ++h) {
        uint32_t at = kNone;
        const uint32_t row = h * kMmaTile + rank * 128 + quarter * 32;
        before(t, row);
        if (t.k0 < t.k1) {
          acc = kHigh == 1 ? turn : h;
          turn ^= 1;
          lost = !__all_sync(0xFFFFFFFFu, mbar_wait_bounded(&bar->acc_full[acc], used[acc]++ & 1, limit_ns));
          if (lost) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          at = tmem + acc * 256 + col0 + (quarter << 21);
        }
        held = at != kNone;
        epilogue(t, i, at, row, col0, release);
        release();
      }
    }
    MmaOut().done();
  }
  if (lost) bar->lost = 1;
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  *lost_out = bar->lost != 0;
}

__device__ __forceinline__ void give_up(const PoolView& v, uint64_t call_seq, bool lost) {
  if (lost && threadIdx.x == 0) note_error(v, call_seq, FT_ERR_TIMEOUT, blockIdx.x);
}

// A matrix of bf16 rows, brought in 64 x 64 boxes; reads beyond its extents give zeros.  With box_rows = 32 the map of a store,
// whose values may be fp32 (32 columns a box).
inline CUresult mma_map(CUtensorMap* map, const void* base, uint64_t inner, uint64_t rows, uint64_t ld, uint32_t box_rows = 64, bool fp32 = false) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
    return reinterpret_cast<Encode>(f);
  }();
  if (!encode) return CUDA_ERROR_NOT_FOUND;
  const cuuint64_t dims[2] = {inner, rows}, strides[1] = {ld * (fp32 ? 4 : 2)};
  const cuuint32_t box[2] = {fp32 ? 32u : 64u, box_rows}, step[2] = {1, 1};
  return encode(map, fp32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

}  // namespace ft
