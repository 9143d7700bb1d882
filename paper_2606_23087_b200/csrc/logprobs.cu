// Log probabilities of given tokens, entropies and the likeliest alternatives of rows against a vocabulary, without a matrix of logits
// where no alternatives are asked for.
//
//   z = x W^T, u = (z - max) scale log2(e), S = sum(2^u), U = sum(u 2^u)
//   logprob = (z_token - max) scale - ln S,  entropy = ln S - ln 2 U / S
//
//   k_score_pick  takes the rows that count out of a piece of the rows: a dense copy of their x, their tokens, row numbers and tokens' logits
//   k_score       z by tiles; a row of a tile gives max, S and U of 128 columns (a segment), the token's left out, each about the segment's own
//                 maximum: every term of U is negative, so nothing cancels in an entropy; and with alternatives z itself in fp32, where it
//                 may be needed: a row's segments are dealt out to as many classes as there are alternatives, the largest logit seen so far
//                 of each class is kept, and a segment whose maximum is below all of these holds none of the alternatives
//   k_score_few   the same for up to 256 rows, which are a matter of W's bytes: W's rows lie across the tensor memory's lanes and the rows
//                 of x in its columns, so that no product is spent on rows that are not there; segments of 32 columns
//   k_score_join  joins a row's segments.  Alternatives: the `top` segments with the largest maxima (equal ones: the first) hold the `top`
//                 largest logits, so only those are read again.  The logits that a caller gets to see, the token's and the alternatives', it
//                 takes once more as x . W[id] by fp32 FMAs, corrects the sums by them, and orders the list by them: the tensor cores
//                 truncate at every addition, all one way, and in a logit that stands alone that does not average out (log probabilities of
//                 likely tokens, about -1, K = 4104 in parts of 1024: off by 4.7e-6 of their size on average without this, 0.6e-6 with it;
//                 in one piece 1.2e-5 and 1.5e-6.  Tokens at random, about -8: 1.2e-7 and 1.1e-7, 4.6e-7 and 3.8e-7)
//   k_score_list  the same for long calls with alternatives, behind the join
//
// Bound by the tensor cores, long calls by the card's power limit: 10813 rows that count of 16384 x 3584, vocabulary 32768, 8 alternatives 1.72 to
// 1.97 ms (1.29 to 1.48 PFLOP/s; k_score alone 1.56 ms, k_score_list 91 us).  Few rows by W's bytes: 24 x 1024, 32768 23 us (18 of them
// k_score_few, whose first and last 5 us read nothing, 10 alone the join), 24 x 4096, 131072 168 us (6.4 TB/s).
#include <algorithm>
#include <cmath>
#include <limits>

#include "mma_pair.cuh"

namespace ft {

constexpr uint32_t kSegCols = 128;     // columns of a segment: an epilogue warp's
constexpr uint32_t kFewCols = 32;      // the same where the rows are few
constexpr uint32_t kFewRows = 256;     // rows that count as few, where the workspace has room (ScoreWork)
// The tensor cores truncate at every addition of 16 products, all one way: few rows and tiles of 256 rows are summed in parts of kScorePart blocks
// of K, the parts joined in registers.  Tiles of 512 rows have no registers for that: they are for rows beyond 256 and K up to kScoreHigh blocks.
constexpr uint32_t kScorePart = 16, kScoreHigh = 66;
constexpr uint32_t kScoreRowsMost = 65536;  // of a piece
constexpr float kScoreLog2e = 1.4426950408889634f, kScoreLn2 = 0.6931471805599453f;
constexpr float kLeastExponent = -300.f;    // 2^-300 is zero; finite, so that its product with zero is one

struct ScorePiece {
  uint32_t rows, hidden, vocab, segs, padded, pairs, top, ld_z;  // padded: rows of xc
  uint32_t few;              // few rows: all of them are there, counted or not, and a row's segments lie side by side
  uint32_t held;             // the join keeps its rows' maxima in shared memory
  uint64_t row0, ldx;
  uint64_t ldw;
  const __nv_bfloat16 *x, *w;
  const int32_t* tokens;
  float scale, to_log2;     // to_log2: scale log2(e), or fp32's largest number where that is beyond it
  float *logprob, *entropy, *top_logprobs;
  int32_t* top_ids;
  uint64_t call_seq;
  // workspace
  uint32_t* count;          // rows of the piece that count
  int32_t *row_of, *token;  // [count] row in the piece, token
  float* target;            // [count] the token's logit, by FMAs
  float *most, *sum, *moment;  // max, S, U of a row's segment: [segs][rows], few rows [rows][segs]
  __nv_bfloat16* xc;        // [padded][hidden]
  uint32_t classes;         // of a row's segments: `top`, rounded up to fours
  float4* joined;           // [count] a row's maximum, S and U
  uint64_t* listed;         // [count][top] its alternatives but the token, as order_key of the logit that the sums give; 0: none
  uint32_t* seen;           // [rows][classes] the largest maximum so far of a class's segments, as ordered_bits
  float* z;                 // [rows][ld_z]
};

// Whole numbers in the order of the values; a NaN counts as -inf, -0 as 0.  None of them is zero.
__device__ __forceinline__ uint32_t ordered_bits(float z) {
  const uint32_t b = __float_as_uint(fmaxf(z, -INFINITY) + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A lane's share of x . w by fp32 FMAs: of every 32 pieces of 8 elements the one at its place.  The order depends on K alone, so that equal rows of W
// give equal logits wherever they are taken.
struct RowDot {
  F2 acc[2] = {F2{0}, F2{0}};
  __device__ __forceinline__ void add(uint4 x, uint4 w) {
    F2 f[4], g[4];
    Pack<__nv_bfloat16>::widen(x, f);
    Pack<__nv_bfloat16>::widen(w, g);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j & 1] = fma(f[j], g[j], acc[j & 1]);
  }
  __device__ __forceinline__ float total() const { return warp_sum(sum(acc[0] + acc[1])); }  // the whole warp
};
// x . w[i] by a warp, four pieces of each row a lane on their way at a time
template <uint32_t kRowsOfW>
__device__ __forceinline__ void row_dots(const __nv_bfloat16* x_row, const uint4* const (&w)[kRowsOfW], uint32_t hidden, float (&z)[kRowsOfW]) {
  constexpr uint32_t kAhead = kRowsOfW == 1 ? 8 : 4;
  const uint32_t vecs = hidden / 8;
  const uint4* x = reinterpret_cast<const uint4*>(x_row);
  RowDot dot[kRowsOfW];
  for (uint32_t c0 = threadIdx.x & 31; c0 < vecs; c0 += 32 * kAhead) {
    uint4 xv[kAhead], wv[kRowsOfW][kAhead];
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) {
      const uint32_t c = c0 + 32 * i;
      const bool there = c < vecs;
      xv[i] = there ? x[c] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (uint32_t r = 0; r < kRowsOfW; ++r) wv[r][i] = there ? w[r][c] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i)
#pragma unroll
      for (uint32_t r = 0; r < kRowsOfW; ++r) dot[r].add(xv[i], wv[r][i]);
  }
#pragma unroll
  for (uint32_t r = 0; r < kRowsOfW; ++r) z[r] = dot[r].total();
}
__device__ __forceinline__ float row_dot(const __nv_bfloat16* x_row, const uint4* w, uint32_t hidden) {
  const uint4* const rows[1] = {w};
  float z[1];
  row_dots<1>(x_row, rows, hidden, z);
  return z[0];
}
__device__ __forceinline__ const uint4* row_of_w(const ScorePiece& a, uint32_t id) { return reinterpret_cast<const uint4*>(a.w + id * a.ldw); }

// A CTA takes kRows rows (up to 32), its warps a row at a time; where they go it learns by counting the tokens before them itself, so nothing has to
// wait for another CTA.  Those counts read the square of the rows, so long pieces take more rows a CTA: with 8, 16, 32 rows 8192 x 3584 (66 %
// count) takes 24, 25, 40 us, 16384 x 3584 38, 33, 44, 65536 x 1024 (90 %) 76, 53, 50.
constexpr uint32_t kScorePickRows = 8, kScorePickMany = 16, kScorePickManyFrom = 16384;
template <uint32_t kRows>
__global__ void __launch_bounds__(256) k_score_pick(PoolView v, ScorePiece a) {
  __shared__ uint32_t warp_count[8];
  __shared__ int32_t dest[32];
  let_next_start();
  after_previous();
  const uint32_t r0 = blockIdx.x * kRows, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = r0 + lane;
  const int32_t* tokens = a.tokens + a.row0;
  const uint32_t mine = __reduce_add_sync(0xFFFFFFFFu, count_labels(tokens, r0, a.vocab));
  if (lane == 0) warp_count[warp] = mine;
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) before += warp_count[w];
  const int32_t t = lane < kRows && r < a.rows ? tokens[r] : kNoLabel;
  const bool counts = has_label(t, a.vocab);
  const uint32_t mask = __ballot_sync(0xFFFFFFFFu, counts), pos = before + __popc(mask & ((1u << lane) - 1));
  if (warp == 0) {
    dest[lane] = counts ? (int32_t)pos : -1;
    if (counts) {
      a.row_of[pos] = (int32_t)r;
      a.token[pos] = t;
    } else if (lane < kRows && r < a.rows) {
      const uint64_t row = a.row0 + r;
      a.logprob[row] = 0.f;
      if (a.entropy) a.entropy[row] = 0.f;
      for (uint32_t i = 0; i < a.top; ++i) { a.top_ids[row * a.top + i] = -1; a.top_logprobs[row * a.top + i] = 0.f; }
      if (t != kNoLabel) note_error(v, a.call_seq, FT_ERR_BAD_TOKEN_ID, (uint32_t)row);
    }
    if (blockIdx.x == gridDim.x - 1 && lane == 0) *a.count = before + __popc(mask);
  }
  __syncthreads();
  const uint32_t vecs = a.hidden / 8, rows = min(kRows, a.rows - r0);
  for (uint32_t i = threadIdx.x; i < rows * a.classes; i += blockDim.x) a.seen[(uint64_t)r0 * a.classes + i] = 0;
  for (uint32_t k = warp; k < rows; k += 8) {
    if (dest[k] < 0) continue;
    const uint4* src = reinterpret_cast<const uint4*>(a.x + (a.row0 + r0 + k) * a.ldx);
    const uint4* w = row_of_w(a, (uint32_t)tokens[r0 + k]);
    uint4* __restrict__ dst = reinterpret_cast<uint4*>(a.xc + (uint64_t)dest[k] * a.hidden);
    RowDot dot;
#pragma unroll 4
    for (uint32_t c = lane; c < vecs; c += 32) {
      const uint4 x = src[c];
      dot.add(x, w[c]);
      dst[c] = x;
    }
    const float target = dot.total();
    if (lane == 0) a.target[dest[k]] = target;
  }
}

// What k_score_pick clears, where every row counts
__global__ void __launch_bounds__(256) k_score_clear(ScorePiece a) {
  let_next_start();
  after_previous();
  const uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < (uint64_t)a.rows * a.classes) a.seen[i] = 0;
}

// max, S and U of a lane's segment, about its maximum
struct SegStats {
  float most, sum, moment;
};
template <uint32_t kCols, class Z>
__device__ __forceinline__ SegStats segment_stats(Z&& z, float to_log2) {
  float most = -INFINITY;
#pragma unroll
  for (uint32_t j = 0; j < kCols; j += 2) most = fmaxf(most, fmaxf(z(j), z(j + 1)));
  F2 sums = f2(0.f), moments = f2(0.f);
  const F2 less = f2(most == -INFINITY ? 0.f : -most), by = f2(to_log2);
#pragma unroll
  for (uint32_t j = 0; j < kCols; j += 2) {
    const float2 t = parts((f2(z(j), z(j + 1)) + less) * by);
    const float u0 = max_with_nan(t.x, kLeastExponent), u1 = max_with_nan(t.y, kLeastExponent);
    const F2 e = f2(exp2_fast(u0), exp2_fast(u1));
    sums = sums + e;
    moments = fma(e, f2(u0, u1), moments);
  }
  return SegStats{most, sum(sums), sum(moments)};
}

// z by tiles; a lane owns a row's segment
template <bool kKeep, int kHigh>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMmaThreads, 1)
k_score(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ PoolView v,
        const __grid_constant__ ScorePiece a) {
  let_next_start();
  after_previous();
  const uint32_t n = a.tokens ? *a.count : a.rows, n_tiles = (a.vocab + kMmaTile - 1) / kMmaTile, k_blocks = (a.hidden + kMmaK - 1) / kMmaK;
  const uint32_t blocks = (n + kMmaTile - 1) / kMmaTile, m_tiles = (blocks + kHigh - 1) / kHigh, tiles = m_tiles * n_tiles;
  constexpr uint32_t kPart = kHigh == 1 ? kScorePart : 0xFFFFFFu;
  const uint32_t k_parts = (k_blocks + kPart - 1) / kPart;
  bool lost;
  uint32_t z[kSegCols / 32][32];
  int32_t token = kNoLabel;
  [[maybe_unused]] uint32_t bound = 0;  // no alternative of the lane's row lies in a segment whose maximum is below it
  mma_pair_tiles<false, false, kHigh>(map_x, map_w, (tiles + a.pairs - 1) / a.pairs * a.pairs * k_parts, v, &lost,
    [&](uint32_t item) {  // a pair takes the parts of a tile's K one after the other
      const uint32_t round = item / a.pairs, i = item % a.pairs + round / k_parts * a.pairs, part = round % k_parts;
      if (i >= tiles) return MmaTile{0, 0, 0, 0, 0};
      // bands of 2048 rows, all columns of a band before the next: a band's x stays in L2
      constexpr uint32_t kBand = 8 / kHigh;
      const uint32_t band = i / (kBand * n_tiles), in = i - band * kBand * n_tiles, rows = min(kBand, m_tiles - band * kBand);
      // the row tiles' order shifts from column to column: else a pair might meet the same ones again and again, and never the short last one
      const uint32_t m = band * kBand + (in + in / rows) % rows;
      return MmaTile{m * kHigh * kMmaTile, in / rows * kMmaTile, part * kPart, min((part + 1) * kPart, k_blocks), min((uint32_t)kHigh, blocks - m * kHigh)};
    },
    [&](const MmaTile& t, uint32_t row) {
      const uint32_t m = t.m + row + (threadIdx.x & 31);
      token = a.tokens && m < n ? a.token[m] : kNoLabel;
      if constexpr (kKeep) {  // (others raise it meanwhile: an older, lower one keeps more)
        bound = 0xFFFFFFFFu;
        for (uint32_t i = 0; m < n && i < a.classes; i += 4) {
          const uint4 q = __ldcg(reinterpret_cast<const uint4*>(a.seen + (uint64_t)m * a.classes + i));
          bound = min(bound, min(min(q.x, q.y), min(q.z, q.w)));
        }
      }
    },
    [&](const MmaTile& t, uint32_t, uint32_t tmem, uint32_t row, uint32_t col0, auto&& release) {
      const uint32_t c0 = t.n + col0;
      if (c0 >= a.vocab) return;
      if (kHigh == 2 || t.k0 == 0) {
#pragma unroll
        for (uint32_t c = 0; c < kSegCols / 32; ++c) tmem_load32(tmem + 32 * c, z[c]);
        tmem_wait();
      } else {
#pragma unroll
        for (uint32_t c = 0; c < kSegCols / 32; ++c) {
          uint32_t part[32];
          tmem_load32(tmem + 32 * c, part);
          tmem_wait();
#pragma unroll
          for (uint32_t j = 0; j < 32; ++j) z[c][j] = __float_as_uint(__uint_as_float(z[c][j]) + __uint_as_float(part[j]));
        }
      }
      release();  // the products go on while the exponentials are taken
      if (kHigh == 1 && t.k1 < k_blocks) return;
      const uint32_t m = t.m + row + (threadIdx.x & 31), cols = min(kSegCols, a.vocab - c0), token_at = (uint32_t)token - c0;
      if (token_at < kSegCols) {  // the join adds it
#pragma unroll
        for (uint32_t j = 0; j < kSegCols; ++j)
          if (j == token_at) z[j / 32][j % 32] = 0xFF800000u;
      }
      if (cols < kSegCols) {  // beyond the vocabulary
#pragma unroll
        for (uint32_t j = 0; j < kSegCols; ++j)
          if (j >= cols) z[j / 32][j % 32] = 0xFF800000u;
      }
      const SegStats g = segment_stats<kSegCols>([&](uint32_t j) { return __uint_as_float(z[j / 32][j % 32]); }, a.to_log2);
      if (m < n) {
        const uint64_t at = (uint64_t)(c0 / kSegCols) * a.rows + m;
        a.most[at] = g.most;
        a.sum[at] = g.sum;
        a.moment[at] = g.moment;
        if constexpr (kKeep) {
          const uint32_t most = ordered_bits(g.most), seg = c0 / kSegCols;
          if (most >= bound) {
            float* to = a.z + (uint64_t)m * a.ld_z + c0;
#pragma unroll
            for (uint32_t c = 0; c < kSegCols; c += 8) store32(to + c, &z[c / 32][c % 32]);
            atomicMax(a.seen + (uint64_t)m * a.classes + seg % a.classes, most);  // any order: what is kept differs, not what is found
          }
        }
      }
    });
  give_up(v, a.call_seq, lost);
}

// ---- few rows -------------------------------------------------------------------------------------------------------

// A CTA takes a contiguous run of W's rows, 128 of them (four segments) a tile: D = W x^T, a vocabulary entry a lane of the tensor
// memory, a row of x a column.  K goes in parts of up to kScorePart blocks, into the halves of the tensor memory in turn; the epilogue adds the
// parts in its registers, so that a logit carries the truncation of 1024 of K whatever the rows and K.
//
// More than 64 rows read x from L2 as often as W from memory, or twice as often, and still take 70 us for 100 x 4096 and 77 for 200 x 3584, vocabulary
// 32768, 8 alternatives (6 of them for the alternatives' logits by FMAs).
//
// Warps: 0 TMA, 1 matrix instructions, 2 tensor memory, 3 the tokens' logits, from 4 on the epilogue, a group of four warps for each 128 rows of x.
// Waits are bounded as in mma_pair_tiles, and given up the same way.
template <uint32_t kN>
constexpr uint32_t kFewGroups = kN > 128 ? 2 : 1;
template <uint32_t kN>
constexpr int kFewThreads = 128 + 128 * kFewGroups<kN>;
constexpr uint32_t kFewTile = 128;                       // W's rows of a tile
constexpr uint32_t kFewBox = kFewCols * kMmaK * 2;       // bytes of a box of W: a segment's rows, 64 columns of K
// Blocks of K of a stage.  Two: a row's 256 bytes are asked for together; one where x takes most of a stage.
template <uint32_t kN>
constexpr uint32_t kFewSub = kN > 128 ? 1 : 2;
template <uint32_t kN>
constexpr uint32_t kFewBlock = kFewTile * kMmaK * 2 + kN * kMmaK * 2;  // bytes of a block of K: W's, then x's
template <uint32_t kN>
constexpr uint32_t kFewStage = kFewSub<kN> * kFewBlock<kN>;
template <uint32_t kN>
constexpr uint32_t kFewStages = (kN == 32 ? 10 : kN == 64 ? 8 : kN == 128 ? 6 : 4) / kFewSub<kN>;
constexpr uint32_t kFewTurn = 32 * 33 * 4;               // bytes of a warp's 32 x 32 logits, turned over
template <uint32_t kN>
constexpr size_t kFewSmem = kFewStages<kN> * (size_t)kFewStage<kN> + 4 * kFewGroups<kN> * kFewTurn + 1024 + 256;

struct FewBarriers {
  uint64_t full[10], empty[10], acc_full[2], acc_empty[2], drain;
  uint32_t tmem, lost;
};
static_assert(sizeof(FewBarriers) <= 256 && kFewSmem<32> <= 227 * 1024 && kFewSmem<64> <= 227 * 1024 && kFewSmem<128> <= 227 * 1024 && kFewSmem<256> <= 227 * 1024, "kFewSmem");

// `policy`: of the L2 cache.  W passes through it once: lines that leave first make way for themselves, not for what others have there
// (24 rows x 4096, vocabulary 131072: 192 us without, 185 with).  The same for x, although every CTA reads it again: with
// L2::evict_last it is as fast from 1 to 256 rows, with L2::evict_normal slower (200 x 3584 74 us, not 62).
__device__ __forceinline__ uint64_t leave_first() { uint64_t p; asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p)); return p; }
__device__ __forceinline__ void few_box(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint64_t* bar, uint64_t policy) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4}], [%2], %5;"
               ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "l"(policy) : "memory");
}
__device__ __forceinline__ void few_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void few_product(uint32_t tmem, uint64_t da, uint64_t db, uint32_t idesc, bool add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(tmem), "l"(da), "l"(db), "r"(idesc), "r"((uint32_t)add) : "memory");
}

// 16 columns of the warp's 32 rows, as tmem_load32
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
  __syncwarp();
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
                 "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(addr) : "memory");
}

template <uint32_t kN, bool kKeep>
__global__ void __launch_bounds__(kFewThreads<kN>, 1)
k_score_few(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_tile,
            const __grid_constant__ PoolView v, const __grid_constant__ ScorePiece a) {
  extern __shared__ uint8_t smem_raw[];
  constexpr uint32_t kStages = kFewStages<kN>, kStage = kFewStage<kN>, kSub = kFewSub<kN>, kGroups = kFewGroups<kN>;
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* turned = reinterpret_cast<float*>(stages + kStages * kStage);
  FewBarriers* bar = reinterpret_cast<FewBarriers*>(stages + kStages * kStage + 4 * kGroups * kFewTurn);
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  let_next_start();
  if (threadIdx.x == 32)
    for (const CUtensorMap* map : {&map_x, &map_w, &map_tile}) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < kStages; ++s) { mbar_init(&bar->full[s], 1); mbar_init(&bar->empty[s], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&bar->acc_full[i], 1); mbar_init(&bar->acc_empty[i], 4 * kGroups); }
    mbar_init(&bar->drain, 1);
    bar->lost = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bar->tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  after_previous();
  const uint32_t tmem = bar->tmem, base = smem_u32(stages);
  const uint32_t k_blocks = (a.hidden + kMmaK - 1) / kMmaK;
  const uint32_t parts = (k_blocks + kScorePart - 1) / kScorePart, each = ((k_blocks + parts - 1) / parts + 1) & ~1u;  // blocks of a part: whole stages
  const uint32_t seg0 = (uint32_t)((uint64_t)a.segs * blockIdx.x / gridDim.x), seg1 = (uint32_t)((uint64_t)a.segs * (blockIdx.x + 1) / gridDim.x);
  const uint64_t limit_ns = mma_wait_limit(v, k_blocks);
  bool lost = false;
  if (warp == 0 && lane == 0) {
    const uint64_t once = leave_first();
    uint32_t it = 0;
    for (uint32_t seg = seg0; seg < seg1 && !lost; seg += 4) {
      const uint32_t boxes = min(4u, seg1 - seg);
      for (uint32_t k = 0; k < k_blocks; k += kSub, ++it) {
        const uint32_t s = it % kStages, at = base + s * kStage, subs = min(kSub, k_blocks - k);
        if (!mbar_wait_bounded(&bar->empty[s], ((it / kStages) & 1) ^ 1, limit_ns)) { lost = true; break; }
        mbar_expect_tx(&bar->full[s], subs * (boxes * kFewBox + kN * kMmaK * 2) + v.bulk_tx_slack);  // the slack: a test hook, 0
        for (uint32_t i = 0; i < subs; ++i) {
          if (boxes == 4) {  // one box: four of a quarter each take 6 % longer
            few_box(at + i * kFewBlock<kN>, &map_tile, (int32_t)((k + i) * kMmaK), (int32_t)(seg * kFewCols), &bar->full[s], once);
            continue;
          }
          for (uint32_t b = 0; b < boxes; ++b)
            few_box(at + i * kFewBlock<kN> + b * kFewBox, &map_w, (int32_t)((k + i) * kMmaK), (int32_t)((seg + b) * kFewCols), &bar->full[s], once);
        }
        for (uint32_t i = 0; i < subs; ++i)
          few_box(at + i * kFewBlock<kN> + kFewTile * kMmaK * 2, &map_x, (int32_t)((k + i) * kMmaK), 0, &bar->full[s], once);
      }
    }
    // what still arrives in shared memory: the loads of the last stages, and the signals that their products are done
    const uint32_t j0 = it > kStages ? it - kStages : 0;
    if (lost)
      for (uint32_t j = j0; j < it; ++j) mbar_wait_bounded(&bar->full[j % kStages], (j / kStages) & 1, limit_ns);
    for (uint32_t j = j0; j < it && !lost; ++j) lost = !mbar_wait_bounded(&bar->empty[j % kStages], (j / kStages) & 1, limit_ns);
  } else if (warp == 1 && lane == 0) {
    constexpr uint32_t kInstr = 1u << 4 | 1u << 7 | 1u << 10 | (kN >> 3) << 17 | (kFewTile >> 4) << 24;  // fp32 sums of bf16 x bf16
    uint32_t it = 0, n = 0;  // stages and parts so far
    for (uint32_t seg = seg0; seg < seg1 && !lost; seg += 4) {
      for (uint32_t k0 = 0; k0 < k_blocks && !lost; k0 += each, ++n) {
        const uint32_t acc = n & 1, k1 = min(k0 + each, k_blocks);
        if (!mbar_wait_bounded(&bar->acc_empty[acc], ((n >> 1) & 1) ^ 1, limit_ns)) { lost = true; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (uint32_t k = k0; k < k1; k += kSub, ++it) {
          const uint32_t s = it % kStages;
          if (!mbar_wait_bounded(&bar->full[s], (it / kStages) & 1, limit_ns)) { lost = true; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          for (uint32_t i = 0; i < min(kSub, k1 - k); ++i) {
            const uint32_t sa = base + s * kStage + i * kFewBlock<kN>, sb = sa + kFewTile * kMmaK * 2;
#pragma unroll
            for (uint32_t j = 0; j < kMmaK / 16; ++j)
              few_product(tmem + acc * 256, mma_desc<false>(sa + j * kMmaStep<false>), mma_desc<false>(sb + j * kMmaStep<false>), kInstr, k + i > k0 || j > 0);
          }
          few_commit(&bar->empty[s]);
        }
        if (!lost) few_commit(&bar->acc_full[acc]);
      }
    }
    if (lost) {  // products under way still read shared memory and write tensor memory
      few_commit(&bar->drain);
      mbar_wait_bounded(&bar->drain, 0, limit_ns);
    }
  } else if (warp == 3) {  // the tokens' logits
    for (uint32_t m = blockIdx.x; a.tokens && m < a.rows; m += gridDim.x) {
      const int32_t token = a.tokens[a.row0 + m];
      if (!has_label(token, a.vocab)) continue;
      const float target = row_dot(a.x + (a.row0 + m) * a.ldx, row_of_w(a, (uint32_t)token), a.hidden);
      if (lane == 0) a.target[m] = target;
    }
  } else if (warp >= 4) {
    constexpr uint32_t kRows = kN / kGroups;  // of x, a warp's columns
    const uint32_t quarter = warp & 3, r0 = (warp - 4) / 4 * kRows;
    float* mine = turned + (warp - 4) * (kFewTurn / 4);
    uint32_t n = 0;
    for (uint32_t s0 = seg0; s0 < seg1 && !lost; s0 += 4) {
      const uint32_t seg = s0 + quarter, id = seg * kFewCols + lane;
      uint32_t z[kRows / 32][32];
      for (uint32_t k0 = 0; k0 < k_blocks; k0 += each, ++n) {
        const uint32_t acc = n & 1, at = tmem + acc * 256 + r0 + (quarter << 21);
        lost = !__all_sync(0xFFFFFFFFu, mbar_wait_bounded(&bar->acc_full[acc], (n >> 1) & 1, limit_ns));
        if (lost) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (uint32_t g = 0; g < kRows / 32; ++g) {
          if (r0 + 32 * g >= a.rows || seg >= seg1) continue;
          if (k0 == 0) {
            tmem_load32(at + 32 * g, z[g]);
            continue;
          }
#pragma unroll
          for (uint32_t h = 0; h < 32; h += 16) {
            uint32_t more[16];
            tmem_load16(at + 32 * g + h, more);
            tmem_wait();
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j) z[g][h + j] = __float_as_uint(__uint_as_float(z[g][h + j]) + __uint_as_float(more[j]));
          }
        }
        tmem_wait();
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive_at(smem_u32(&bar->acc_empty[acc]));
      }
      if (lost) break;
      // 32 rows of x at a time, those in front moved up behind them: unrolled, this much code takes 10 us to arrive where a call finds the caches cold
#pragma unroll 1
      for (uint32_t m0 = r0; m0 < min(r0 + kRows, a.rows) && seg < seg1; m0 += 32) {
        const uint32_t m = m0 + lane;
        __syncwarp();
#pragma unroll
        for (uint32_t j = 0; j < 32; ++j) {
          const float x = id < a.vocab ? __uint_as_float(z[0][j]) : -INFINITY;
          if (kKeep && m0 + j < a.rows) a.z[(uint64_t)(m0 + j) * a.ld_z + id] = x;
          mine[j * 33 + lane] = x;
        }
        __syncwarp();
        if (m < a.rows) {
          const uint32_t token_at = (uint32_t)(a.tokens ? a.tokens[a.row0 + m] : kNoLabel) - seg * kFewCols;
          if (token_at < kFewCols) mine[lane * 33 + token_at] = -INFINITY;  // the join adds it
          const SegStats t = segment_stats<kFewCols>([&](uint32_t j) { return mine[lane * 33 + j]; }, a.to_log2);
          const uint64_t to = (uint64_t)m * a.segs + seg;
          a.most[to] = t.most;
          a.sum[to] = t.sum;
          a.moment[to] = t.moment;
        }
#pragma unroll
        for (uint32_t g = 0; g + 1 < kRows / 32; ++g)
#pragma unroll
          for (uint32_t j = 0; j < 32; ++j) z[g][j] = z[g + 1][j];
      }
    }
  }
  if (lost) bar->lost = 1;
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  give_up(v, a.call_seq, bar->lost != 0);
}

// ---- joining the segments of a row ----------------------------------------------------------------------------------

// An order of (value, place): larger values first, equal ones by place.  No key is zero.
__device__ __forceinline__ uint64_t order_key(float z, uint32_t place) { return (uint64_t)ordered_bits(z) << 32 | (uint32_t)~place; }
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b & 0x80000000u ? b & 0x7FFFFFFFu : ~b);
}
__device__ __forceinline__ uint32_t key_place(uint64_t key) { return ~(uint32_t)key; }
__device__ __forceinline__ uint64_t warp_max(uint64_t key) {
  const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(key >> 32));
  const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(key >> 32) == hi ? (uint32_t)key : 0u);
  return (uint64_t)hi << 32 | lo;
}

template <uint32_t kWarps>
__device__ __forceinline__ void row_sync() {  // of the warps that share a row
  if constexpr (kWarps == 1) __syncwarp();
  else __syncthreads();
}

// The `top` first of many keys, by the warps of a row: each(f) calls f(key) for every key of a thread, the lanes of a warp as often
// (0: no key); put(rank, key) is called for each of the first.  `least`: a key that none of them is below, or 0.  Without one, or
// where it leaves too many, it is the `top`-th largest of a warp's lanes' own first keys, or the smallest of what each warp's first keys
// give for its share of `top`.  What it leaves (of 1024 segments some 20 for 8, 60 for 32) is ranked by counting.
constexpr uint32_t kFewPicks = 128;  // keys that the room holds
template <uint32_t kWarps>
struct KeyRoom {
  uint64_t key[kFewPicks], first[kWarps][32], least[kWarps], share[kWarps];
  uint32_t found;
};
template <uint32_t kWarps, class Each, class Put>
__device__ __forceinline__ void first_keys(uint32_t top, uint64_t least, KeyRoom<kWarps>& room, Each&& each, Put&& put) {
  const uint32_t lane = threadIdx.x & 31, warp = kWarps == 1 ? 0 : threadIdx.x >> 5, t = kWarps == 1 ? lane : threadIdx.x;
  uint32_t found = kFewPicks + 1;
  const auto collect = [&] {
    found = 0;
    if (kWarps > 1 && t == 0) room.found = 0;
    row_sync<kWarps>();
    each([&](uint64_t key) {
      const bool take = key >= least && key;
      const uint32_t mask = __ballot_sync(0xFFFFFFFFu, take);
      if (mask == 0) return;
      uint32_t at = found;
      if constexpr (kWarps == 1) {
        found += __popc(mask);
      } else {
        if (lane == 0) at = atomicAdd(&room.found, __popc(mask));  // any order: what is ranked is a set
        at = __shfl_sync(0xFFFFFFFFu, at, 0);
      }
      at += __popc(mask & ((1u << lane) - 1));
      if (take && at < kFewPicks) room.key[at] = key;
    });
    row_sync<kWarps>();
    if constexpr (kWarps > 1) found = room.found;
  };
  if (least) collect();
  if (found > kFewPicks) {
    uint64_t first = 0;
    each([&](uint64_t key) { first = max(first, key); });
    room.first[warp][lane] = first;
    __syncwarp();
    uint32_t rank = 0;
#pragma unroll 8
    for (uint32_t i = 0; i < 32; ++i) {
      const uint64_t other = room.first[warp][i];
      rank += other > first || (other == first && i < lane);
    }
    uint64_t bound = __shfl_sync(0xFFFFFFFFu, first, __ffs(__ballot_sync(0xFFFFFFFFu, rank == top - 1)) - 1);
    if constexpr (kWarps > 1) {
      const uint64_t share = __shfl_sync(0xFFFFFFFFu, first, __ffs(__ballot_sync(0xFFFFFFFFu, rank == (top + kWarps - 1) / kWarps - 1)) - 1);
      if (lane == 0) { room.least[warp] = bound; room.share[warp] = share; }
      __syncthreads();
      uint64_t all = ~0ull;
#pragma unroll
      for (uint32_t w = 0; w < kWarps; ++w) { bound = max(bound, room.least[w]); all = min(all, room.share[w]); }
      bound = max(bound, all);
    }
    least = max(least, bound);
    collect();
  }
  if (found <= kFewPicks) {
    for (uint32_t i = t; i < found; i += 32 * kWarps) {
      const uint64_t key = room.key[i];
      uint32_t rank = 0;
      for (uint32_t j = 0; j < found; ++j) rank += room.key[j] > key;
      if (rank < top) put(rank, key);
    }
    row_sync<kWarps>();
    return;
  }
  uint64_t last = ~0ull;  // very many equal ones: one after the other
  for (uint32_t j = 0; j < top; ++j) {
    uint64_t best = 0;
    each([&](uint64_t key) {
      if (key < last) best = max(best, key);
    });
    best = warp_max(best);
    if constexpr (kWarps > 1) {
      if (lane == 0) room.least[warp] = best;
      __syncthreads();
#pragma unroll
      for (uint32_t w = 0; w < kWarps; ++w) best = max(best, room.least[w]);
      __syncthreads();
    }
    last = best;
    if (last == 0) break;
    if (t == 0) put(j, last);
  }
  row_sync<kWarps>();
}

// A segment's numbers, or those of several, taken into numbers about `about`.
struct Joined {
  float sum = 0.f, moment = 0.f;
  __device__ __forceinline__ void add(float most, float part, float part_moment, float about, float to_log2) {
    if (most == -INFINITY && part == 0.f) return;  // nothing in it (a sum of NaN stays)
    const float u = max_with_nan(((most == -INFINITY ? 0.f : most) - about) * to_log2, kLeastExponent), e = exp2f(u);
    sum = fmaf(part, e, sum);
    moment = fmaf(e, fmaf(part, u, part_moment), moment);
  }
};
__device__ __forceinline__ float finite_about(float most) { return most == -INFINITY ? 0.f : most; }

// The room of a row, or of a warp's
template <uint32_t kWarps>
struct RowRoom {
  KeyRoom<kWarps> keys;
  uint32_t seg_of[FT_LOGPROBS_MAX_TOP];
};

// A row's alternatives but the token, into listed (zeros before), by the warps of the row.  most_of(s): the maximum of segment s.
template <uint32_t kSeg, uint32_t kWarps, class MostOf>
__device__ __forceinline__ void row_list(const ScorePiece& a, uint32_t m, int32_t token, uint64_t* listed, RowRoom<kWarps>& room, MostOf&& most_of) {
  const uint32_t lane = threadIdx.x & 31, warp = kWarps == 1 ? 0 : threadIdx.x >> 5, t = kWarps == 1 ? lane : threadIdx.x;
  const uint32_t segs = min(a.top, a.segs);
  uint64_t least = 0;
  row_sync<kWarps>();
  if (t < a.top) listed[t] = 0;
  if (a.segs > a.top) {
    first_keys<kWarps>(a.top, 0, room.keys,
      [&](auto&& f) {
#pragma unroll 4
        for (uint32_t s0 = 0; s0 < a.segs; s0 += 32 * kWarps) {
          const uint32_t s = s0 + t;
          f(s < a.segs ? order_key(most_of(s), s) : 0);
        }
      },
      [&](uint32_t rank, uint64_t key) { room.seg_of[rank] = key_place(key); });
    // no logit below the last segment's maximum is among the first
    least = order_key(most_of(room.seg_of[a.top - 1]), 0xFFFFFFFFu);
  } else {
    if (t < a.segs) room.seg_of[t] = t;
    row_sync<kWarps>();
  }
  const float* z = a.z + (uint64_t)m * a.ld_z;
  first_keys<kWarps>(a.top, least, room.keys,
    [&](auto&& f) {
      constexpr uint32_t kEach = kSeg / 32, kAtOnce = 4;  // logits of a lane in a segment; segments whose loads go out together
      for (uint32_t j0 = warp; j0 < segs; j0 += kAtOnce * kWarps) {
        float v[kAtOnce][kEach];
        uint32_t c[kAtOnce];
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) {
          const uint32_t j = j0 + i * kWarps;
          c[i] = room.seg_of[j < segs ? j : j0] * kSeg + lane * kEach;
          if constexpr (kEach == 4) {
            const float4 q = *reinterpret_cast<const float4*>(z + c[i]);
            v[i][0] = q.x; v[i][1] = q.y; v[i][2] = q.z; v[i][3] = q.w;
          } else {
            v[i][0] = z[c[i]];
          }
        }
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) {
          if (j0 + i * kWarps >= segs) break;
#pragma unroll
          for (uint32_t e = 0; e < kEach; ++e) f(order_key((int32_t)(c[i] + e) == token ? -INFINITY : v[i][e], c[i] + e));
        }
      }
    },
    [&](uint32_t rank, uint64_t key) {
      if (key_place(key) < a.vocab && (int32_t)key_place(key) != token) listed[rank] = key;
    });
}

// A row's results, by a warp, from its joined numbers, which leave the token out: the largest logit, the sum and moment about it (about 0 where it is
// -inf).  A lane has an alternative: its order_key by the sums (0: none), and its logit by FMAs.
__device__ __forceinline__ void row_results(const ScorePiece& a, uint64_t row, int32_t token, float target, float most, float sum, float moment, uint64_t key,
                                            float listed_logit) {
  const uint32_t lane = threadIdx.x & 31;
  const bool given = a.tokens != nullptr;
  const float by_sums = key_value(key), logit = key ? listed_logit : -INFINITY;
  const auto largest = [](float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
    return v;
  };
  const float to_log2 = a.to_log2;
  float about = finite_about(fmaxf(fmaxf(most, target), largest(logit)));
  const auto power = [&](float z) { return max_with_nan((z - about) * to_log2, kLeastExponent); };
  Joined others, all;
  others.add(most, sum, moment, about, to_log2);
  if (a.top) {  // the alternatives' terms by FMAs in the place of those that the sums hold
    const bool there = key && logit != -INFINITY;
    float more = 0.f, more_moment = 0.f;
    bool apart = false;
    if (there && logit != by_sums) {
      const float u = power(logit), u0 = power(by_sums), e = exp2f(u), e0 = exp2f(u0), d = (logit - by_sums) * a.scale;
      apart = fabsf(d) >= 1.f && fmaxf(e, e0) > 0x1p-12f;
      more = fabsf(d) < 1.f ? e0 * expm1f(d) : e - e0;
      more_moment = u * e - u0 * e0;
    }
    if (__any_sync(0xFFFFFFFFu, apart)) {
      // A scale at which the sums' roundings are worth powers of e, in logits that count: beside terms by FMAs the sums mean nothing
      about = finite_about(fmaxf(target, largest(logit)));
      const float u = power(logit), e = there ? exp2f(u) : 0.f;
      others.sum = warp_sum(e);
      others.moment = warp_sum(there ? u * e : 0.f);
    } else {
      others.sum += warp_sum(more);
      others.moment += warp_sum(more_moment);
    }
  }
  all = others;
  if (target != -INFINITY) all.add(target, given ? 1.f : 0.f, 0.f, about, to_log2);
  // where the token is the likeliest, from what the others have: nothing is lost to the one
  const float log_sum = given && target == about && all.sum < INFINITY ? log1pf(others.sum) : logf(all.sum);
  const auto number = [&](float z) { return (z - about) * a.scale - log_sum; };
  if (lane == 0) {
    if (given) a.logprob[row] = number(target);
    if (a.entropy) a.entropy[row] = log_sum - kScoreLn2 * all.moment / all.sum;
  }
  if (a.top == 0) return;
  const uint64_t mine = key ? order_key(logit, key_place(key)) : 0, own = given ? order_key(target, (uint32_t)token) : 0;
  uint32_t rank = own > mine;
  for (uint32_t i = 0; i < a.top; ++i) rank += __shfl_sync(0xFFFFFFFFu, mine, i) > mine;
  const uint32_t before = __popc(__ballot_sync(0xFFFFFFFFu, mine > own));
  int32_t* ids = a.top_ids + row * a.top;
  float* numbers = a.top_logprobs + row * a.top;
  if (key && rank < a.top) { ids[rank] = (int32_t)key_place(key); numbers[rank] = number(logit); }
  if (given && lane == 0 && before < a.top) { ids[before] = token; numbers[before] = number(target); }
  if (lane >= a.vocab && lane < a.top) { ids[lane] = -1; numbers[lane] = -INFINITY; }
}

constexpr uint32_t kJoinHeldMost = 132 * 1024;  // bytes of maxima in shared memory

// kRows rows a CTA, and as many warps: as the segments' numbers lie, the threads go through them rows first, whole sectors at a time; a
// warp then finishes a row, with the maxima in shared memory where they fit.  (A warp a row from the start read a sector for every
// number: 61 us for 10813 rows x 256 segments.)
template <uint32_t kRows>
__global__ void __launch_bounds__(32 * kRows) k_score_join(const __grid_constant__ ScorePiece a) {
  constexpr uint32_t kGroups = 32;
  extern __shared__ float s_held[];  // [kRows][segs, made odd]
  __shared__ float s_part[3][kGroups][kRows + 1];
  __shared__ RowRoom<1> s_room[kRows];
  after_previous();
  const uint32_t n = a.tokens ? *a.count : a.rows, m0 = blockIdx.x * kRows;
  if (m0 >= n) return;
  const uint32_t r = threadIdx.x % kRows, g = threadIdx.x / kRows, held_ld = a.segs | 1;
  const float to_log2 = a.to_log2;
  if (m0 + r < n) {
    float most = -INFINITY;
#pragma unroll 4
    for (uint32_t s = g; s < a.segs; s += kGroups) {
      const float x = a.most[(uint64_t)s * a.rows + m0 + r];
      if (a.held) s_held[r * held_ld + s] = x;
      most = fmaxf(most, x);
    }
    Joined mine;
#pragma unroll 4
    for (uint32_t s = g; s < a.segs; s += kGroups) {
      const uint64_t at = (uint64_t)s * a.rows + m0 + r;
      mine.add(a.held ? s_held[r * held_ld + s] : a.most[at], a.sum[at], a.moment[at], finite_about(most), to_log2);
    }
    s_part[0][g][r] = most;
    s_part[1][g][r] = mine.sum;
    s_part[2][g][r] = mine.moment;
  }
  __syncthreads();
  const uint32_t lane = threadIdx.x & 31, q = threadIdx.x >> 5, m = m0 + q;
  if (m >= n) return;
  float most = s_part[0][lane][q];
#pragma unroll
  for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
  Joined all;
  all.add(s_part[0][lane][q], s_part[1][lane][q], s_part[2][lane][q], finite_about(most), to_log2);
  const int32_t token = a.tokens ? a.token[m] : kNoLabel;
  const float sum = warp_sum(all.sum), moment = warp_sum(all.moment);
  if (a.top == 0) {
    row_results(a, a.row0 + (a.tokens ? (uint32_t)a.row_of[m] : m), token, a.tokens ? a.target[m] : -INFINITY, most, sum, moment, 0, 0.f);
    return;
  }
  if (lane == 0) a.joined[m] = make_float4(most, sum, moment, 0.f);
  row_list<kSegCols, 1>(a, m, token, a.listed + (uint64_t)m * a.top, s_room[q],
                        [&](uint32_t s) { return a.held ? s_held[q * held_ld + s] : a.most[(uint64_t)s * a.rows + m]; });
}

// The alternatives' logits by FMAs, two of them a warp at a time, and the results of the rows.  Bound by the rows of W that it gathers and, where K
// is small, by its chain of latencies, which several rows a CTA share: with 1, 2, 4, 8 rows a CTA 4096 rows x 1024, 8 alternatives 29, 20, 17, 16 us (67 MB
// of W's rows), 32 alternatives 49, 43, 41, 43 us (268 MB), 1599 x 4104, 20 alternatives 56, 54, 46, 69 us (262 MB).  One where four would leave SMs
// with less than two CTAs.
constexpr uint32_t kListWarps = 8, kListRows = 4;
__global__ void __launch_bounds__(32 * kListWarps, 4) k_score_list(const __grid_constant__ ScorePiece a, uint32_t rows_each) {
  __shared__ float s_logit[kListRows * FT_LOGPROBS_MAX_TOP];
  let_next_start();
  after_previous();
  const uint32_t n = a.tokens ? *a.count : a.rows, m0 = blockIdx.x * rows_each, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (m0 >= n) return;
  const uint32_t rows = min(rows_each, n - m0);
  const auto x_of = [&](uint32_t m) { return a.tokens ? a.xc + (uint64_t)m * a.hidden : a.x + (a.row0 + m) * a.ldx; };
  const uint32_t each = (a.top + 1) / 2;  // pairs of a row
  for (uint32_t i = warp; i < rows * each; i += kListWarps) {
    const uint32_t r = i / each, first = (i - r * each) * 2, second = min(first + 1, a.top - 1);
    const uint64_t* listed = a.listed + (uint64_t)(m0 + r) * a.top;
    const uint64_t k0 = listed[first], k1 = listed[second];
    const uint4* const w[2] = {row_of_w(a, k0 ? key_place(k0) : 0), row_of_w(a, k1 ? key_place(k1) : 0)};
    float z[2];
    row_dots<2>(x_of(m0 + r), w, a.hidden, z);
    if (lane == 0) {
      s_logit[r * a.top + first] = z[0];
      s_logit[r * a.top + second] = z[1];
    }
  }
  __syncthreads();
  if (warp >= rows) return;
  const uint32_t m = m0 + warp;
  const float4 j = a.joined[m];
  const bool has = lane < a.top;
  row_results(a, a.row0 + (a.tokens ? (uint32_t)a.row_of[m] : m), a.tokens ? a.token[m] : kNoLabel, a.tokens ? a.target[m] : -INFINITY, j.x, j.y, j.z,
              has ? a.listed[(uint64_t)m * a.top + lane] : 0, has ? s_logit[warp * a.top + lane] : 0.f);
}

// Few rows: a CTA a row.
constexpr uint32_t kFewWarps = 8;
__global__ void __launch_bounds__(32 * kFewWarps, 2) k_score_join_few(const __grid_constant__ PoolView v, const __grid_constant__ ScorePiece a) {
  extern __shared__ float s_held[];  // [segs]
  __shared__ RowRoom<kFewWarps> s_room;
  __shared__ uint64_t s_listed[FT_LOGPROBS_MAX_TOP];
  __shared__ float s_logit[FT_LOGPROBS_MAX_TOP];
  __shared__ float s_part[3][kFewWarps];
  after_previous();
  const uint32_t m = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const uint64_t row = a.row0 + m, first = (uint64_t)m * a.segs;
  if (a.tokens && !has_label(a.tokens[row], a.vocab)) {
    if (t == 0) {
      a.logprob[row] = 0.f;
      if (a.entropy) a.entropy[row] = 0.f;
      if (a.tokens[row] != kNoLabel) note_error(v, a.call_seq, FT_ERR_BAD_TOKEN_ID, (uint32_t)row);
    }
    if (t < a.top) { a.top_ids[row * a.top + t] = -1; a.top_logprobs[row * a.top + t] = 0.f; }
    return;
  }
  // a thread's first numbers are asked for at once
  constexpr uint32_t kAhead = 4, kStep = 32 * kFewWarps;
  float ahead[3][kAhead], most = -INFINITY;
#pragma unroll
  for (uint32_t i = 0; i < kAhead; ++i) {
    const uint32_t s = t + i * kStep;
    ahead[0][i] = s < a.segs ? a.most[first + s] : -INFINITY;
    ahead[1][i] = s < a.segs ? a.sum[first + s] : 0.f;
    ahead[2][i] = s < a.segs ? a.moment[first + s] : 0.f;
  }
#pragma unroll
  for (uint32_t i = 0; i < kAhead; ++i) {
    if (a.held && t + i * kStep < a.segs) s_held[t + i * kStep] = ahead[0][i];
    most = fmaxf(most, ahead[0][i]);
  }
#pragma unroll 4
  for (uint32_t s = t + kAhead * kStep; s < a.segs; s += kStep) {
    const float x = a.most[first + s];
    if (a.held) s_held[s] = x;
    most = fmaxf(most, x);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
  if (lane == 0) s_part[0][warp] = most;
  __syncthreads();
#pragma unroll
  for (uint32_t w = 0; w < kFewWarps; ++w) most = fmaxf(most, s_part[0][w]);
  const float about = finite_about(most), to_log2 = a.to_log2;
  Joined mine;
#pragma unroll
  for (uint32_t i = 0; i < kAhead; ++i) mine.add(ahead[0][i], ahead[1][i], ahead[2][i], about, to_log2);
#pragma unroll 4
  for (uint32_t s = t + kAhead * kStep; s < a.segs; s += kStep) mine.add(a.held ? s_held[s] : a.most[first + s], a.sum[first + s], a.moment[first + s], about, to_log2);
  float sum = warp_sum(mine.sum), moment = warp_sum(mine.moment);
  if (lane == 0) { s_part[1][warp] = sum; s_part[2][warp] = moment; }
  __syncthreads();
  sum = moment = 0.f;
#pragma unroll
  for (uint32_t w = 0; w < kFewWarps; ++w) { sum += s_part[1][w]; moment += s_part[2][w]; }
  const int32_t token = a.tokens ? a.tokens[row] : kNoLabel;
  if (a.top) {
    row_list<kFewCols, kFewWarps>(a, m, token, s_listed, s_room, [&](uint32_t s) { return a.held ? s_held[s] : a.most[first + s]; });
    for (uint32_t i = warp; i < a.top; i += kFewWarps) {
      const uint64_t key = s_listed[i];
      if (key == 0) continue;
      const float z = row_dot(a.x + row * a.ldx, row_of_w(a, key_place(key)), a.hidden);
      if (lane == 0) s_logit[i] = z;
    }
    __syncthreads();
  }
  if (warp) return;
  const bool has = lane < a.top;
  row_results(a, row, token, a.tokens ? a.target[m] : -INFINITY, most, sum, moment, has ? s_listed[lane] : 0, has ? s_logit[lane] : 0.f);
}

// ---- workspace ----------------------------------------------------------------------------------------------------

// columns of tensor memory that so many rows take in k_score_few
static uint32_t few_columns(uint32_t rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }

// Carves the workspace for pieces of `rows` rows; returns its bytes.  `few`: the call's rows are few, and one piece.
static uint64_t score_carve(ScorePiece* a, uint8_t* base, uint32_t rows, uint32_t hidden, uint32_t vocab, uint32_t top, bool few) {
  uint64_t off = 0;
  auto take = [&](uint64_t bytes) { const uint64_t o = off; off += align_up_sz(bytes, 256); return base + o; };
  a->few = few;
  const uint64_t padded = a->few ? rows : align_up_sz(rows, kMmaTile);
  const uint32_t cols = a->few ? kFewCols : kSegCols;
  a->rows = rows;
  a->padded = (uint32_t)padded;
  a->segs = (vocab + cols - 1) / cols;
  a->ld_z = a->segs * cols;
  a->count = reinterpret_cast<uint32_t*>(take(4));
  a->row_of = reinterpret_cast<int32_t*>(take(4ull * rows));
  a->token = reinterpret_cast<int32_t*>(take(4ull * rows));
  a->target = reinterpret_cast<float*>(take(4ull * rows));
  a->most = reinterpret_cast<float*>(take(4ull * rows * a->segs));
  a->sum = reinterpret_cast<float*>(take(4ull * rows * a->segs));
  a->moment = reinterpret_cast<float*>(take(4ull * rows * a->segs));
  a->xc = reinterpret_cast<__nv_bfloat16*>(take(a->few ? 0 : 2ull * padded * hidden));
  a->classes = a->few ? 0 : (top + 3) / 4 * 4;
  a->joined = reinterpret_cast<float4*>(take(a->few || top == 0 ? 0 : 16ull * rows));
  a->listed = reinterpret_cast<uint64_t*>(take(a->few ? 0 : 8ull * rows * top));
  a->seen = reinterpret_cast<uint32_t*>(take(4ull * rows * a->classes));
  a->z = reinterpret_cast<float*>(take(top ? 4ull * rows * a->ld_z : 0));
  return off;
}

// Up to kFewRows rows go the way of few rows where its layout fits, and else by tiles: segments of 32 columns take more room than those of 128,
// and a workspace that serves many rows has to serve the last, smaller call of a loop too.
struct ScoreWork {
  uint32_t hidden, vocab, top;
  uint64_t rows;
  uint64_t tile_bytes(uint32_t piece) const {
    ScorePiece a;
    return score_carve(&a, nullptr, piece, hidden, vocab, top, false);
  }
  uint64_t few_bytes() const {
    ScorePiece a;
    return rows <= kFewRows ? score_carve(&a, nullptr, (uint32_t)rows, hidden, vocab, top, true) : ~0ull;
  }
  uint32_t least_rows() const { return (uint32_t)std::min<uint64_t>(rows, kMmaTile); }
  uint32_t best_rows() const {  // with alternatives, pieces whose logits take 4 GiB
    const uint64_t most = top ? std::max<uint64_t>(kMmaTile, (4ull << 30) / (4ull * vocab) / kMmaTile * kMmaTile) : kScoreRowsMost;
    return (uint32_t)std::min<uint64_t>(rows, std::min<uint64_t>(most, kScoreRowsMost));
  }
  uint64_t least() const { return std::min(few_bytes(), tile_bytes(least_rows())); }
  uint64_t best() const { return rows <= kFewRows ? few_bytes() : tile_bytes(best_rows()); }
  bool few_in(uint64_t have) const { return few_bytes() <= have; }
  // by tiles, the largest piece that fits: all rows, or a multiple of 256
  uint32_t piece_for(uint64_t have) const {
    if (tile_bytes(best_rows()) <= have) return best_rows();
    uint32_t lo = 1, hi = (best_rows() + kMmaTile - 1) / kMmaTile;  // in units of 256 rows
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (tile_bytes(mid * kMmaTile) <= have) lo = mid; else hi = mid;
    }
    return std::min(lo * kMmaTile, best_rows());
  }
};

static int32_t token_logprobs(ft_pool* p, ScorePiece a, uint64_t rows, void* workspace, uint64_t workspace_bytes, cudaStream_t st) {
  const ScoreWork work{a.hidden, a.vocab, a.top, rows};
  if (!workspace || !aligned_to(workspace, 256)) return FT_ERR_INVALID_ARG;
  if (workspace_bytes < work.least()) return FT_ERR_CAPACITY;
  const bool few = work.few_in(workspace_bytes);
  const uint32_t piece = few ? (uint32_t)rows : work.piece_for(workspace_bytes);
  score_carve(&a, static_cast<uint8_t*>(workspace), piece, a.hidden, a.vocab, a.top, few);
  a.call_seq = status_seq(p);
  a.pairs = (uint32_t)p->sm_count / 2;
  // the join's rows a CTA: 8 where 16 would leave SMs without work, or would not have their maxima in shared memory
  const auto held_bytes = [&](uint64_t n) { return n * (a.segs | 1) * sizeof(float); };
  const uint32_t join_rows = a.few ? 1 : piece >= 32u * (uint32_t)p->sm_count && held_bytes(16) <= kJoinHeldMost ? 16 : 8;
  a.held = held_bytes(join_rows) <= kJoinHeldMost;
  const size_t join_smem = a.held ? (size_t)held_bytes(join_rows) : 0;
  const auto join = join_rows == 16 ? k_score_join<16> : k_score_join<8>;
  CUtensorMap map_x, map_w;
  if (mma_map(&map_w, a.w, a.hidden, a.vocab, a.ldw, a.few ? kFewCols : 64) != CUDA_SUCCESS) return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
  if (!p->score_attr_set) {  // once per pool, hence once per device the pool lives on
    for (auto k : {k_score<false, 1>, k_score<false, 2>, k_score<true, 1>, k_score<true, 2>})
      FT_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMmaSmem));
    for (auto k : {k_score_few<32, false>, k_score_few<32, true>})
      FT_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem<32>));
    for (auto k : {k_score_few<64, false>, k_score_few<64, true>})
      FT_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem<64>));
    for (auto k : {k_score_few<128, false>, k_score_few<128, true>})
      FT_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem<128>));
    for (auto k : {k_score_few<256, false>, k_score_few<256, true>})
      FT_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem<256>));
    for (auto k : {k_score_join<16>, k_score_join<8>})
      FT_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kJoinHeldMost));
    FT_CUDA(cudaFuncSetAttribute(k_score_join_few, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kJoinHeldMost));
    p->score_attr_set = true;
  }
  if (a.few) {
    const uint32_t n = few_columns(a.rows), grid = std::min<uint32_t>((uint32_t)p->sm_count, a.segs);
    CUtensorMap map_tile;
    if (mma_map(&map_x, a.x, a.hidden, a.rows, a.ldx, n) != CUDA_SUCCESS || mma_map(&map_tile, a.w, a.hidden, a.vocab, a.ldw, kFewTile) != CUDA_SUCCESS) return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    const auto kernel = n == 32   ? (a.top ? k_score_few<32, true> : k_score_few<32, false>)
                        : n == 64 ? (a.top ? k_score_few<64, true> : k_score_few<64, false>)
                        : n == 128 ? (a.top ? k_score_few<128, true> : k_score_few<128, false>)
                                   : (a.top ? k_score_few<256, true> : k_score_few<256, false>);
    const int threads = n == 256 ? kFewThreads<256> : kFewThreads<128>;
    const size_t smem = n == 32 ? kFewSmem<32> : n == 64 ? kFewSmem<64> : n == 128 ? kFewSmem<128> : kFewSmem<256>;
    FT_CUDA(launch_chained(kernel, grid, threads, smem, st, map_x, map_w, map_tile, p->view, a));
    FT_CUDA(launch_chained(k_score_join_few, a.rows, 32 * kFewWarps, join_smem, st, p->view, a));
    p->gpu_launches += 2;
    return FT_OK;
  }
  for (uint64_t r0 = 0; r0 < rows; r0 += piece) {
    a.row0 = r0;
    a.rows = (uint32_t)std::min<uint64_t>(piece, rows - r0);
    if ((a.tokens ? mma_map(&map_x, a.xc, a.hidden, a.padded, a.hidden) : mma_map(&map_x, a.x + r0 * a.ldx, a.hidden, a.rows, a.ldx)) != CUDA_SUCCESS)
      return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    if (a.tokens) {
      const uint32_t each = a.rows >= kScorePickManyFrom ? kScorePickMany : kScorePickRows;
      FT_CUDA(launch_chained(each == kScorePickMany ? k_score_pick<kScorePickMany> : k_score_pick<kScorePickRows>, dim3((a.rows + each - 1) / each), 256, 0, st, p->view, a));
      p->gpu_launches += 1;
    } else if (a.top) {
      FT_CUDA(launch_chained(k_score_clear, dim3((unsigned)(((uint64_t)a.rows * a.classes + 255) / 256)), 256, 0, st, a));
      p->gpu_launches += 1;
    }
    // tiles of 512 rows, unless they would leave pairs without one
    const uint64_t high_tiles = (uint64_t)((a.rows + 2 * kMmaTile - 1) / (2 * kMmaTile)) * ((a.vocab + kMmaTile - 1) / kMmaTile);
    const bool high = a.rows > kMmaTile && a.hidden <= kScoreHigh * kMmaK && high_tiles > a.pairs;
    const auto kernel = a.top ? (high ? k_score<true, 2> : k_score<true, 1>) : (high ? k_score<false, 2> : k_score<false, 1>);
    FT_CUDA(launch_chained(kernel, 2 * a.pairs, kMmaThreads, kMmaSmem, st, map_x, map_w, p->view, a));
    FT_CUDA(launch_chained(join, dim3((a.rows + join_rows - 1) / join_rows), 32 * join_rows, join_smem, st, a));
    p->gpu_launches += 2;
    if (a.top) {
      const uint32_t each = a.rows >= 2 * kListRows * (uint32_t)p->sm_count ? kListRows : 1;
      FT_CUDA(launch_chained(k_score_list, dim3((a.rows + each - 1) / each), 32 * kListWarps, 0, st, a, each));
      p->gpu_launches += 1;
    }
  }
  return FT_OK;
}

}  // namespace ft

using namespace ft;

FT_EXPORT int32_t pool_token_logprobs_workspace(ft_pool* p, uint64_t rows, uint32_t hidden, uint32_t vocab, uint32_t top, uint64_t* least, uint64_t* best) {
  if (!p || hidden == 0 || hidden % 8 || vocab == 0 || !least || !best) return FT_ERR_INVALID_ARG;
  if (rows >> 31 || vocab >> 31 || top > FT_LOGPROBS_MAX_TOP) return FT_ERR_CAPACITY;
  const ScoreWork work{hidden, vocab, top, rows};
  *least = rows ? work.least() : 0;
  *best = rows ? work.best() : 0;
  return FT_OK;
}

FT_EXPORT int32_t pool_token_logprobs(ft_pool* p, uint64_t rows, uint32_t hidden, uint32_t vocab, const void* x, uint64_t ldx, const void* w,
                                      uint64_t ldw, const int32_t* tokens, float logit_scale, float* logprob, float* entropy, uint32_t top,
                                      int32_t* top_ids, float* top_logprobs, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  if (hidden == 0 || hidden % 8 || vocab == 0) return FT_ERR_INVALID_ARG;
  if (rows >> 31 || vocab >> 31) return FT_ERR_CAPACITY;
  if (rows == 0) return FT_OK;
  if (!x || !aligned_to(x, 16) || ldx < hidden || ldx % 8 || !w || !aligned_to(w, 16) || ldw < hidden || ldw % 8) return FT_ERR_INVALID_ARG;
  if (!aligned_to(tokens, 4) || !(logit_scale > 0.f) || std::isinf(logit_scale) || !tokens != !logprob || !aligned_to(logprob, 4) || !aligned_to(entropy, 4))
    return FT_ERR_INVALID_ARG;
  if (top > FT_LOGPROBS_MAX_TOP) return FT_ERR_CAPACITY;
  if ((top && (!top_ids || !top_logprobs)) || !aligned_to(top_ids, 4) || !aligned_to(top_logprobs, 4)) return FT_ERR_INVALID_ARG;
  ScorePiece a = {};
  a.hidden = hidden; a.vocab = vocab; a.ldx = ldx; a.x = static_cast<const __nv_bfloat16*>(x); a.ldw = ldw; a.w = static_cast<const __nv_bfloat16*>(w); a.tokens = tokens; a.scale = logit_scale;
  a.to_log2 = std::min(logit_scale * kScoreLog2e, std::numeric_limits<float>::max());
  a.logprob = logprob; a.entropy = entropy; a.top = top; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
  return token_logprobs(p, a, rows, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}
