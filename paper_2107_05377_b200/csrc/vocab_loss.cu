// Softmax cross entropy over a large vocabulary without keeping the logits, and its gradient.
//
//   z = x W^T + b                                   x [rows, hidden], W [vocab, hidden], bf16; sums in fp32
//   lse = log sum_v exp z_v,  loss = lse - z_label
//   g = dloss (exp(z - lse) - onehot(label))        rounded to bf16, the operand of the two products below
//   dx = g W,  dW = g^T x,  db = sum over rows of g (from g before rounding)
//
// The forward pass is one product whose epilogue keeps, for every row and tile of columns, the largest logit and the sum of
// exponentials relative to it; a second kernel puts a row's tiles together.  The backward pass makes the logits again, a piece of the
// vocabulary at a time, and keeps g of two pieces at most: launch j computes g of piece j and, among the same tiles, the two products
// of piece j - 1, so that the tiles of all three fill the machine together and a piece costs one launch.
//
// All products are tiles of 256 x 256 of CTA pairs (tcgen05 cta_group::2, fp32 accumulators in tensor memory, two of them so that the
// epilogue of a tile overlaps the next one's products):
//   kind 0   z or g   M = rows, N = vocab,  K = hidden   both operands along K
//   kind 1   dx       M = rows, N = hidden, K = vocab    g along K, W with its rows along K (MN-major)
//   kind 2   dW       M = vocab, N = hidden, K = rows    g and x with their rows along K
// so neither g nor any input is ever transposed in memory.  Rows without a label take no part: where there are some, the rows that have
// one are gathered first (their places stay on the device; the grids are sized for all rows and bound their tiles by the count).
//
// dx is a sum over all pieces: kept in fp32 in the workspace, added to by reductions in L2 (one tile per element and launch, so the
// order is that of the launches), where a launch has few tiles of it in several ranges of the vocabulary with a place each; a last
// kernel adds the ranges in order and rounds once.
//
// What bounds it: the tensor cores from some hundred rows on, below that the bytes of W (read twice) and dW.

#include <cstring>

#include "cluster_ptx.cuh"

namespace mt {
namespace {

constexpr int kTile = 256;                 // rows and (at most) columns of a pair's tile
constexpr int kHalf = 128;                 // rows of a CTA
constexpr int kStageA = kHalf * 128;       // bytes: 128 rows of 64 elements, or two boxes of 64 x 64
constexpr int kStageB = kHalf * 128;
// What a launch of the pair kernel is for: the forward pass, the gradient (all kinds of tiles), or the two products of few rows, whose g is
// there.  The first two have twelve epilogue warps, in three groups that share the columns, and keep the logits of a tile (up to 96 a thread) in
// registers; the tiles of the third are so short (two k-blocks) that their epilogue is what they take, and sixteen warps share it.  (With eight
// warps of 128 logits a thread: forward, 8192 rows x 30522 x 1024 385 us against 371, 4096 x 768 172 against 161; gradient 4096 x 768 588 against 575.)
enum Mode { kForward, kGradient, kProducts };
__host__ __device__ constexpr int epilogue_warps(Mode mode) { return mode == kProducts ? 16 : 12; }
__host__ __device__ constexpr int first_epilogue_warp(Mode mode) { return mode == kProducts ? 2 : 4; }
__host__ __device__ constexpr int threads(Mode mode) { return 32 * (first_epilogue_warp(mode) + epilogue_warps(mode)); }
__host__ __device__ constexpr int groups(Mode mode) { return epilogue_warps(mode) / 4; }   // of the same rows: they share the columns
__host__ __device__ constexpr int blocks(Mode mode) { return (8 + groups(mode) - 1) / groups(mode); }   // of 32 columns of a tile, for a thread
// Registers of a thread: of the 128 that each of 512 threads of the first two starts with, the warpgroup of the producer and the MMA issuer
// gives up, and the epilogue's take (a share that is not there would be waited for without end: launch_pairs looks at what the kernel has).
constexpr int kPairRegs = 128, kIssueRegs = 56, kEpilogueRegs = 152;
__host__ __device__ constexpr int registers_needed(Mode mode) {
  return mode == kProducts ? 0 : 32 * (first_epilogue_warp(mode) * kIssueRegs + epilogue_warps(mode) * kEpilogueRegs);
}
static_assert(registers_needed(kForward) <= kPairRegs * threads(kForward) && registers_needed(kGradient) <= kPairRegs * threads(kGradient), "shares");
constexpr int kBook = 1024;
constexpr int kSlots = 4;                  // tiles announced ahead
constexpr uint32_t kTmemCols = 512;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxRanges = 32;             // of the vocabulary, for dx
constexpr float kFloor = -3.402823466e38f;  // the lowest finite number: below every logit that counts, and -inf minus it is no NaN

// All of shared memory is the ring: what a pair computes is bound by how many bytes are on their way (32 KB per k-block and CTA, of the 64
// per clock that an SM takes in), so results leave straight from registers instead of through staging buffers.  (A single cold launch, 8192 rows
// x 30522 x 1024: forward 311 us, 1.65 PFLOP/s; g of 7680 columns 140 us; with the products of 7680 others 296 us, 1.3 PFLOP/s.)
constexpr int kStages = 7;
constexpr int kSmemBytes = kStages * (kStageA + kStageB) + kBook + 1024;

// Shared-memory descriptor of a tile whose 128-byte rows (64 elements of M or N, 128-byte swizzle) run along K: eight of them make an
// atom, the next eight along K follow 1024 bytes on, the next 64 elements of M or N 8192 bytes on (boxes of 64 rows).
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t smem_addr) {
  uint64_t d = static_cast<uint64_t>((smem_addr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(8192 >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
constexpr uint32_t kAlongMnA = 1u << 15, kAlongMnB = 1u << 16;   // instruction descriptor: the operand's rows run along K

// Four lanes that hold four 16-byte pieces of a row each: afterwards piece i of a lane is piece (lane & 3) of the row of the i-th of them,
// so that a store covers 64 bytes of eight rows instead of 16 bytes of thirty-two.
__device__ __forceinline__ void exchange_pieces(uint4 (&v)[4], int lane) {
#pragma unroll
  for (int k = 1; k <= 2; k <<= 1) {
    const bool upper = (lane & k) != 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i & k) continue;
      uint4 give = upper ? v[i] : v[i | k];
      give.x = __shfl_xor_sync(0xffffffffu, give.x, k);
      give.y = __shfl_xor_sync(0xffffffffu, give.y, k);
      give.z = __shfl_xor_sync(0xffffffffu, give.z, k);
      give.w = __shfl_xor_sync(0xffffffffu, give.w, k);
      if (upper) v[i] = give; else v[i | k] = give;
    }
  }
}
__device__ __forceinline__ void red_add_v4(float* p, const uint4& v) {
  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(__uint_as_float(v.x)), "f"(__uint_as_float(v.y)),
               "f"(__uint_as_float(v.z)), "f"(__uint_as_float(v.w)) : "memory");
}
// An arrival on a barrier of either CTA of the pair, ordered behind this thread's own accesses in shared and tensor memory only.  (Released
// at cluster scope it would wait for the thread's stores to global memory as well: some 2000 clocks per tile.)
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Four words into the shared memory of a CTA of the pair, counted on a barrier there that this announces them to: whoever waits for the
// barrier sees them, without fences at cluster scope on either side.
__device__ __forceinline__ void send_words(uint32_t cluster_addr, int a, int b, int c, int d, uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], 16;" ::"r"(cluster_bar) : "memory");
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.s32 [%0], {%1, %2, %3, %4}, [%5];"
               ::"r"(cluster_addr), "r"(a), "r"(b), "r"(c), "r"(d), "r"(cluster_bar)
               : "memory");
}

// What a launch works on: the forward pass and few rows from the arguments, otherwise as the rows' kernel has left it (without a division
// here: every clock before the first copy counts in a short launch).
template <Mode MODE>
__device__ __forceinline__ VocabWork load_work(const VocabLossParams& p) {
  VocabWork w;
  if (MODE == kGradient) {
    const int4* src = reinterpret_cast<const int4*>(p.work);
    int4* dst = reinterpret_cast<int4*>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = __ldcg(src + i);
    return w;
  }
  w = VocabWork{};
  w.rows = MODE == kForward && p.count != nullptr ? min(p.rows, __ldcg(p.count)) : p.rows;
  w.row_tiles = (w.rows + kTile - 1) / kTile;
  if (MODE == kForward) {
    w.cols = p.vocab;
    w.n0 = w.row_tiles * p.n_tiles;
  } else {
    w.prev_cols = p.vocab;
    w.ranges = p.ranges;
    w.row_pitch = p.row_pitch;
    w.n1 = p.want_x ? p.n_tiles * p.ranges : 0;             // (one tile of rows)
    w.n2 = p.want_w ? (p.vocab + kTile - 1) / kTile * p.n_tiles : 0;
    w.k1 = p.range_blocks;
    w.k2 = (w.rows + 63) / 64;
  }
  return w;
}

// i / d by a reciprocal of d.
__device__ __forceinline__ int divide(int i, int d, float rcp) {
  if (i >= 1 << 22) return i / d;
  int q = static_cast<int>(static_cast<float>(i) * rcp);
  const int r = i - q * d;
  if (r < 0) --q;
  if (r >= d) ++q;
  return q;
}

// Few rows with a label, among however many: g in two bf16 terms, for the same reason as with few rows altogether (below).  The second
// one has its place behind the first in the buffer of g, in the unused half of the only tile of rows.  (Error of dW 2.3e-3 to 2.7e-3 -> 1.7e-3,
// 120 of 1000 rows x 30522 x 768 67 -> 72 us.  With more rows with a label the error is 2.2e-3 to 2.4e-3 and the products over rows get longer.)
__host__ __device__ constexpr int terms_of_g(int rows) { return rows <= kHalf ? 2 : 1; }

struct Tile {
  int kind, m, n, range, k_blocks, k_begin;
};
// The tiles of a launch in the order in which they are handed out, long ones first.  n_tiles: of the columns of a matrix product (forward:
// the vocabulary; backward, kinds 1 and 2: the hidden size).
template <bool GRAD>
__device__ __forceinline__ Tile find_tile(const VocabWork& w, int n_tiles, int k0, const int32_t* two_terms, int i) {
  Tile t;
  t.range = 0;
  t.k_begin = 0;
  if (GRAD && i < w.n1 + w.n2) {
    const bool first1 = w.k1 > w.k2;
    const bool is1 = first1 ? i < w.n1 : i >= w.n2;
    const float rcp_n = __frcp_rn(static_cast<float>(n_tiles));
    if (is1) {
      if (!first1) i -= w.n2;
      t.kind = 1;
      const int q = divide(i, w.row_tiles, __frcp_rn(static_cast<float>(w.row_tiles)));
      t.m = i - q * w.row_tiles;
      t.range = divide(q, n_tiles, rcp_n);
      t.n = q - t.range * n_tiles;
      t.k_begin = t.range * w.k1;
      const int all = (w.prev_cols + 63) / 64;
      t.k_blocks = max(0, min(w.k1, all - t.k_begin));
    } else {
      if (first1) i -= w.n1;
      t.kind = 2;
      const int m_tiles = (w.prev_cols + kTile - 1) / kTile;
      t.n = divide(i, m_tiles, __frcp_rn(static_cast<float>(m_tiles)));
      t.m = i - t.n * m_tiles;
      t.k_blocks = w.k2;
      // (few rows: g in two terms, one behind the other along K, where one of the words is a label)
      if (two_terms != nullptr && i < w.n2 && __ldcg(two_terms + t.m) != 0) t.k_blocks = 2 * w.k2;
    }
    return t;
  }
  i -= w.n1 + w.n2;
  t.kind = 0;
  t.n = divide(i, w.row_tiles, __frcp_rn(static_cast<float>(w.row_tiles)));
  t.m = i - t.n * w.row_tiles;
  t.k_blocks = k0;
  return t;
}

// Logits.  The tensor cores cut partial sums off towards zero, once per instruction of 16 terms, so that a logit of dense operands that is
// summed in one go is too small by some 0.27 * 2^-24 of itself for every 16 terms (measured on 64 to 16384 terms).  Sums are therefore made of
// at most this many k-blocks, each in an accumulator of its own, and joined in fp32, rounding to nearest, by the epilogue: what is cut off
// is that of a logit of 256 (forward, up to 768 wide) or 384 terms whatever the width, and a sum that fp32 holds exactly comes out exactly.
// Each further sum costs its tile a change of accumulators and a pass over one of them, some 1300 clocks, of which a wide tile hides most.
// (Against one sum per tile: forward, 8192 rows x 30522 x 1024 in three sums 363 -> 370 us, 4096 x 768 in three 150 -> 161; gradient, 8192 x 1024 in
// three 1316 -> 1370, 4096 x 768 in two 560 -> 575.  Sums of four k-blocks at a width of 1024: forward 437, gradient 1417, both with eight warps.)
__host__ __device__ constexpr int sum_blocks(bool grad, int k_blocks) { return !grad && k_blocks <= 12 ? 4 : 6; }

// A sum of 32 columns from its accumulator, and one added to what is there.
__device__ __forceinline__ void take_sum(float (&z)[32], uint32_t taddr) {
  uint32_t v[32];
  tmem_ld_32x32(taddr, v);
  tmem_ld_wait();
#pragma unroll
  for (int j = 0; j < 32; ++j) z[j] = __uint_as_float(v[j]);
}
__device__ __forceinline__ void join_sum(float (&z)[32], uint32_t taddr) {
  uint32_t v[32];
  tmem_ld_32x32(taddr, v);
  tmem_ld_wait();
#pragma unroll
  for (int j = 0; j < 32; ++j) z[j] += __uint_as_float(v[j]);
}
// The same for blocks of 32 columns from taddr + begin on, `step` columns apart, those below `end`.
template <int BLOCKS>
__device__ __forceinline__ void join_sums(float (&z)[BLOCKS][32], uint32_t taddr, int begin, int step, int end) {
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) if (begin + i * step < end) join_sum(z[i], taddr + begin + i * step);   // (the same for the whole warp)
}
// The logits to where the last of their sums was, as if all terms had been summed there.
template <int BLOCKS>
__device__ __forceinline__ void put_sums(const float (&sum)[BLOCKS][32], uint32_t taddr, int begin, int step, int end) {
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) {
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
      const int c = begin + i * step + h;
      if (c >= end) continue;
      uint32_t v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(sum[i][h + j]);
      tmem_st_32x16(taddr + c, v);
    }
  }
  tmem_st_wait();
}

// Something read for nothing but to be near: a tile's bias, which its threads take when the sums are joined (gradient of 4096 rows x 30522 x 768
// 505 -> 498 us against taking it, all at once, before them).
__device__ __forceinline__ void touch(const bf16* p) { asm volatile("{\n\t.reg .b16 t;\n\tld.global.nc.b16 t, [%0];\n\t}" ::"l"(p)); }

// The bias of a thread's words, blocks of 32 from `col` on, `step` apart, added to their logits.  At the vocabulary's end a lane reads that of
// one word per block, -inf behind the last word.
template <int BLOCKS>
__device__ __forceinline__ void add_bias(const bf16* bias, int col, int step, int vocab, int lane, float (&z)[BLOCKS][32]) {
  if (col + (BLOCKS - 1) * step + 32 > vocab) {
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      const int word = col + i * step + lane;
      const float b = word >= vocab ? -INFINITY : (bias != nullptr ? __bfloat162float(bias[word]) : 0.f);
#pragma unroll
      for (int j = 0; j < 32; ++j) z[i][j] += __shfl_sync(0xffffffffu, b, j);
    }
  } else if (bias != nullptr) {
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(bias + col + i * step) + q);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          z[i][q * 8 + 2 * j] += bf16_lo(w[j]);
          z[i][q * 8 + 2 * j + 1] += bf16_hi(w[j]);
        }
      }
    }
  }
}

// Sums over the 32 rows of a warp of 32 columns each, column `lane` in the result: halves of the columns are exchanged for halves of the
// rows five times over (31 additions per lane instead of 160).
__device__ __forceinline__ float column_sums(float (&c)[32], int lane) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const bool upper = (lane & o) != 0;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float give = upper ? c[i] : c[i + o];
      const float keep = upper ? c[i + o] : c[i];
      c[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  return c[0];
}

// exp(z - lse).  (z - lse first: what is rounded is the size of the exponent and not of its terms, in an error of its own for every entry; and
// both may be at the lowest number.)  The row's weight is a factor: its logarithm within the exponent would be rounded at a size of its own,
// 1e-6 of the weight at a weight of 1e-12.
__device__ __forceinline__ float probability(float z, float lse) { return ex2_approx((z - lse) * kLog2e); }

template <Mode MODE>
__global__ void __maxnreg__(MODE == kProducts ? 96 : kPairRegs) vocab_loss_pair_tcgen05(const __grid_constant__ VocabLossParams p) {
  constexpr bool GRAD = MODE != kForward;
  constexpr int STAGES = kStages;
  constexpr int EPILOGUE_WARPS = epilogue_warps(MODE), GROUPS = groups(MODE);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sA = smem_u32(smem);
  const uint32_t sB = sA + STAGES * kStageA;
  uint8_t* book = smem + STAGES * (kStageA + kStageB);
  const uint32_t bar_full = smem_u32(book);
  const uint32_t bar_empty = bar_full + 8 * STAGES;
  const uint32_t bar_acc_full = bar_empty + 8 * STAGES;
  const uint32_t bar_acc_empty = bar_acc_full + 16;
  const uint32_t bar_slot_full = bar_acc_empty + 16;
  const uint32_t bar_slot_empty = bar_slot_full + 8 * kSlots;      // (of rank 0)
  static_assert((2 * STAGES + 4 + 2 * kSlots) % 2 == 0, "tiles are sent in 16 bytes");
  volatile int4* slot_tile = reinterpret_cast<volatile int4*>(book + 8 * (2 * STAGES + 4 + 2 * kSlots));   // kind, m, n + 65536 range, k-blocks
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(book + 8 * (2 * STAGES + 4 + 2 * kSlots) + 16 * kSlots);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_cta_rank();
  const int worker = static_cast<int>(blockIdx.x >> 1);
  const int n_workers = static_cast<int>(gridDim.x >> 1);

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(bar_acc_full + 8 * a, 1);
      mbar_init(bar_acc_empty + 8 * a, 2 * EPILOGUE_WARPS);
    }
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(bar_slot_full + 8 * s, 1);
      mbar_init(bar_slot_empty + 8 * s, 2 * EPILOGUE_WARPS + 2);   // all epilogue warps, the MMA warp, rank 1's producer
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) tmem_alloc_pair(smem_u32(tmem_slot), kTmemCols);
  tc_fence_before();
  __syncwarp();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t bar_full_count = map_to_cta(bar_full, 0);
  const uint32_t bar_slot_empty_0 = map_to_cta(bar_slot_empty, 0);
  if (warp == 0 && lane == 0) {
    prefetch_tensormap(&p.x_k[0]);
    prefetch_tensormap(&p.w_k);
    if (GRAD) {
      prefetch_tensormap(&p.w_mn);
      prefetch_tensormap(&p.g_k[0]);
      prefetch_tensormap(&p.g_mn[0]);
      prefetch_tensormap(&p.x_mn[0]);
    }
  }
  // What the arguments alone decide is computed before the wait (a first look at each line of them costs some hundred clocks).
  const bool given = MODE == kProducts || (MODE == kForward && p.count == nullptr);
  VocabWork work = {};
  if (given) work = load_work<MODE>(p);
  asm volatile("" ::"r"(p.rows), "r"(p.block_n), "r"(p.block_h), "r"(p.n_tiles), "r"(p.want_w), "l"(p.labels), "l"(p.counter));
  grid_dependency_wait();
  grid_launch_dependents();
  if (!given) work = load_work<MODE>(p);
  const int rows = work.rows, g_pitch = p.piece << work.shift;
  const int gathered = rows == p.rows ? 0 : 1;      // which x: the caller's, or the rows with a label
  const int total = work.n0 + work.n1 + work.n2;
  const int k0 = (p.hidden + 63) / 64;
  const int first_term = (rows + 63) / 64;          // k-blocks of the first term of g in kind 2
  const bool two_terms = MODE == kGradient && p.want_w && terms_of_g(rows) == 2;

  // Tiles.  Forward: worker, worker + n_workers, ... (all tiles cost the same).  Backward: the first one likewise, then the next of the
  // list, whoever is free first; rank 0's producer takes them from a counter in memory and announces them to all roles of both CTAs.
  // (Which pair computes a tile has no influence on it.)
  int slot = 0;
  uint32_t slot_phase = 0;
  Tile t = find_tile<GRAD>(work, p.n_tiles, k0, p.two_terms, worker);
  // Forward: m and n of the next tile of this worker without a division per tile.
  const int step_m = n_workers % max(work.row_tiles, 1), step_n = n_workers / max(work.row_tiles, 1);
  int at_tile = worker;
  auto next_static = [&](bool first) -> bool {
    if (!first) {
      at_tile += n_workers;
      t.m += step_m;
      t.n += step_n;
      if (t.m >= work.row_tiles) { t.m -= work.row_tiles; ++t.n; }
    }
    return at_tile < total;
  };
  // Backward, the roles other than rank 0's producer: the next tile; false at the end and when the CTA is giving up.
  auto next_announced = [&](bool first) -> bool {
    if (first) return worker < total;
    if (!__all_sync(0xffffffffu, mbar_wait(bar_slot_full + 8 * slot, slot_phase, abort_flag))) return false;
    t.kind = slot_tile[slot].x;
    t.m = slot_tile[slot].y;
    const int n_range = slot_tile[slot].z;
    t.k_blocks = slot_tile[slot].w;
    t.n = n_range & 0xFFFF;
    t.range = n_range >> 16;
    t.k_begin = t.range * work.k1;
    __syncwarp();
    if (lane == 0) mbar_arrive_remote(bar_slot_empty_0 + 8 * slot);
    if (++slot == kSlots) { slot = 0; slot_phase ^= 1u; }
    return t.kind >= 0;
  };

  if (warp < first_epilogue_warp(MODE)) {
    if constexpr (MODE != kProducts) setmaxnreg_dec<kIssueRegs>();
    if (warp == 0) {
      // ------------------------------ TMA producer ------------------------------
      const bool leader = elect_one();
      int stage = 0;
      uint32_t phase = 0;
      long long issued = 0;
      bool ok = true;
      // (backward, rank 0) The tile after the one whose copies are under way is asked for when its turn begins and announced some k-blocks
      // later, so that neither the trip to the counter nor that to the other CTA holds up a copy.
      int asked = 0;
      if (GRAD && rank == 0 && lane == 0) asked = static_cast<int>(atomicAdd(p.counter, 1u));
      Tile ahead = t;
      if (worker >= total) ahead.kind = -1;
      auto announce = [&](int i) -> bool {
        if (i < total) ahead = find_tile<GRAD>(work, p.n_tiles, k0, p.two_terms, i); else ahead.kind = -1;
        if (!__all_sync(0xffffffffu, mbar_wait(bar_slot_empty + 8 * slot, slot_phase ^ 1u, abort_flag))) return false;
        if (lane < 2)
          send_words(map_to_cta(smem_u32(const_cast<int4*>(slot_tile) + slot), lane), ahead.kind, ahead.m, ahead.n | (ahead.range << 16), ahead.k_blocks,
                     map_to_cta(bar_slot_full + 8 * slot, lane));
        __syncwarp();
        if (++slot == kSlots) { slot = 0; slot_phase ^= 1u; }
        if (ahead.kind >= 0 && lane == 0) asked = static_cast<int>(atomicAdd(p.counter, 1u));
        return true;
      };
      for (bool first = true; ok; first = false) {
        if (!GRAD) {
          if (!next_static(first)) break;
        } else if (rank != 0) {
          if (!next_announced(first)) break;
        } else {
          t = ahead;
          if (t.kind < 0) break;
        }
        const int half_n = (t.kind == 0 ? p.block_n : p.block_h) / 2;
        const uint32_t bytes = 2 * (kStageA + half_n * 128);
        const int m0 = t.m * kTile + static_cast<int>(rank) * kHalf;
        const int n0 = t.n * (2 * half_n) + static_cast<int>(rank) * half_n;
        for (int kb = 0; kb < t.k_blocks; ++kb) {
          if (!__all_sync(0xffffffffu, mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag))) { ok = false; break; }
          if (leader) {
            const uint32_t a = sA + stage * kStageA, b = sB + stage * kStageB, bar = bar_full_count + 8 * stage;
            const int k = (t.k_begin + kb) * 64;
            if (rank == 0) mbar_expect_tx(bar_full + 8 * stage, bytes);
            if (MODE == kForward || (MODE == kGradient && t.kind == 0)) {
              tma_load_2d_pair(a, &p.x_k[gathered], k, m0, bar);
              tma_load_2d_pair(b, &p.w_k, k, work.col0 + n0, bar);
            } else if (t.kind == 1) {
              if (MODE == kProducts) {
                tma_load_2d_pair(a, &p.g_mn[work.shift], m0, work.prev_col0 + k, bar);
                tma_load_2d_pair(a + 8192, &p.g_mn[work.shift], m0 + 64, work.prev_col0 + k, bar);
              } else {
                tma_load_2d_pair(a, &p.g_k[work.shift], k, work.prev_g_row0 + m0, bar);
              }
              tma_load_2d_pair(b, &p.w_mn, n0, work.prev_col0 + k, bar);
              if (half_n > 64) tma_load_2d_pair(b + 8192, &p.w_mn, n0 + 64, work.prev_col0 + k, bar);
            } else {
              if (MODE == kProducts) {
                tma_load_2d_pair(a, &p.g_k[work.shift], k, work.prev_col0 + m0, bar);
              } else {
                const int kg = work.prev_g_row0 + (kb < first_term ? k : k - first_term * 64 + kHalf);
                tma_load_2d_pair(a, &p.g_mn[work.shift], m0, kg, bar);
                tma_load_2d_pair(a + 8192, &p.g_mn[work.shift], m0 + 64, kg, bar);
              }
              const int kx = kb < first_term ? k : k - first_term * 64;   // (both terms meet the same rows of x)
              tma_load_2d_pair(b, &p.x_mn[gathered], n0, kx, bar);
              if (half_n > 64) tma_load_2d_pair(b + 8192, &p.x_mn[gathered], n0 + 64, kx, bar);
            }
          }
          ++issued;
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          if (GRAD && rank == 0 && kb == min(3, t.k_blocks - 1) && !announce(n_workers + __shfl_sync(0xffffffffu, asked, 0))) { ok = false; break; }
        }
        if (GRAD && rank == 0 && ok && t.k_blocks == 0) ok = announce(n_workers + __shfl_sync(0xffffffffu, asked, 0));
      }
      if (!ok && rank == 0 && leader) {
        // giving up: what is still in flight gets the same limit to land
        const int pending = issued < STAGES ? static_cast<int>(issued) : STAGES;
        for (int i = 0; i < pending; ++i) {
          if (stage == 0) { stage = STAGES; phase ^= 1u; }
          --stage;
          mbar_drain(bar_full + 8 * stage, phase);
        }
      }
    } else if (warp == 1) {
      // ------------------------------ MMA issuer --------------------------------
      const bool leader = elect_one();
      if (rank == 0) {
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        bool ok = true;
        for (bool first = true; ok; first = false) {
          if (GRAD ? !next_announced(first) : !next_static(first)) break;
          const bool mn_a = GRAD && t.kind == (MODE == kProducts ? 1 : 2), mn_b = GRAD && t.kind != 0;
          const uint32_t idesc = umma_idesc_bf16(kTile, t.kind == 0 ? p.block_n : p.block_h) | (mn_a ? kAlongMnA : 0u) | (mn_b ? kAlongMnB : 0u);
          // 16 elements of K on: 32 bytes inside a row, or 16 rows
          const uint64_t step_a = mn_a ? 2048 >> 4 : 2, step_b = mn_b ? 2048 >> 4 : 2;
          const int most = MODE != kProducts && t.kind == 0 ? sum_blocks(GRAD, k0) : max(t.k_blocks, 1);
          int kb = 0;
          do {                                            // (once where there is nothing to sum)
            if (!__all_sync(0xffffffffu, mbar_wait(bar_acc_empty + 8 * acc, acc_phase ^ 1u, abort_flag))) { ok = false; break; }
            tc_fence_after();
            const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * kTile);
            const int begin = kb, end = min(kb + most, t.k_blocks);
            for (; kb < end; ++kb) {
              if (!__all_sync(0xffffffffu, mbar_wait(bar_full + 8 * stage, phase, abort_flag))) { ok = false; break; }
              tc_fence_after();
              if (leader) {
                const uint64_t da = mn_a ? smem_desc_mn(sA + stage * kStageA) : smem_desc_sw128(sA + stage * kStageA);
                const uint64_t db = mn_b ? smem_desc_mn(sB + stage * kStageB) : smem_desc_sw128(sB + stage * kStageB);
#pragma unroll
                for (int k = 0; k < 4; ++k) umma_bf16_pair(d_tmem, da + step_a * k, db + step_b * k, idesc, (kb - begin) | k ? 1u : 0u);
                umma_commit_pair(bar_empty + 8 * stage);
              }
              if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
            if (!ok) break;
            if (leader) umma_commit_pair(bar_acc_full + 8 * acc);
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
          } while (kb < t.k_blocks);
        }
      }
    }
  } else {
    // ------------------------------ epilogue ----------------------------------
    if constexpr (MODE != kProducts) setmaxnreg_inc<kEpilogueRegs>();
    const int e = warp - first_epilogue_warp(MODE);
    const int quarter = warp & 3;
    const int group = e >> 2;
    const uint32_t bar_acc_empty_0 = map_to_cta(bar_acc_empty, 0);
    const int sums = (k0 + sum_blocks(GRAD, k0) - 1) / sum_blocks(GRAD, k0);
    int acc = 0;
    uint32_t acc_phase = 0;
    const uint32_t my_tmem = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    auto wait_sum = [&] { return __all_sync(0xffffffffu, mbar_wait(bar_acc_full + 8 * acc, acc_phase, abort_flag)); };
    auto leave_sum = [&] {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(bar_acc_empty_0 + 8 * acc);
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    };
    if constexpr (MODE == kForward) {
      constexpr int BLOCKS = blocks(MODE);
      float z[BLOCKS][32];
      bool taken = false;                               // the first sum of the tile's logits is there already
      auto take = [&](int i, int end) {
        const int c = group * 32 + 32 * GROUPS * i;
        if (c < end) take_sum(z[i], my_tmem + static_cast<uint32_t>(acc * kTile + c));
      };
      // A tile's labels, and its bias on the way to L1, while the tile before is worked on.
      int next_label = -1;
      auto next_tile = [&](bool first) -> bool {
        if (!next_static(first)) return false;
        const int row = t.m * kTile + static_cast<int>(rank) * kHalf + quarter * 32 + lane, col = t.n * p.block_n + lane * 16;
        next_label = row < rows ? p.labels[row] : -1;
        if (p.bias != nullptr && lane < 16 && col < p.vocab)
          touch(p.bias + col);
        return true;
      };
      for (bool more = next_tile(true); more;) {
        const int m0 = t.m * kTile + static_cast<int>(rank) * kHalf + quarter * 32;   // of this warp
        const int row = m0 + lane, n0 = t.n * p.block_n;
        const int end = m0 < rows ? min(p.block_n, p.vocab - n0) : 0;
        const int label = next_label;
        float2* part = p.parts + static_cast<int64_t>(row) * p.part_pitch + GROUPS * t.n + group;
        if (!taken) {
          if (!wait_sum()) break;
          tc_fence_after();
#pragma unroll
          for (int i = 0; i < BLOCKS; ++i) take(i, end);
          leave_sum();
        }
        add_bias(p.bias, n0 + group * 32, 32 * GROUPS, p.vocab, lane, z);
        bool ok = true;
        for (int i = 1; i < sums; ++i) {
          if (!(ok = wait_sum())) break;
          tc_fence_after();
          join_sums(z, my_tmem + static_cast<uint32_t>(acc * kTile), group * 32, 32 * GROUPS, end);
          leave_sum();
        }
        if (!ok) break;
        if (__any_sync(0xffffffffu, label >= n0 && label < n0 + end)) {
          float mine = 0.f;
          bool here = false;
#pragma unroll
          for (int i = 0; i < BLOCKS; ++i) {
            const int at = label - (n0 + group * 32 + 32 * GROUPS * i);
            here |= at >= 0 && at < 32 && label < n0 + end;
#pragma unroll
            for (int j = 0; j < 32; ++j) if (j == at) mine = z[i][j];
          }
          if (here) p.label_logit[row] = mine;
        }
        float top = kFloor, s[4] = {0.f, 0.f, 0.f, 0.f};   // largest logit, sum of exp(z - top)
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
          if (group * 32 + 32 * GROUPS * i >= end) continue;
          float m[4] = {z[i][0], z[i][1], z[i][2], z[i][3]};
#pragma unroll
          for (int j = 4; j < 32; ++j) m[j & 3] = fmaxf(m[j & 3], z[i][j]);
          top = fmaxf(top, fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
        }
        // The exponentials keep the special-function units busy for 2048 clocks.  Half way through, the first sum of the next tile is there and
        // takes the place of the logits that are done with: otherwise the MMAs, which are two sums ahead, would wait for it.
        more = next_tile(false);
        taken = more && sums > 1;
        const int next_end = taken && t.m * kTile + static_cast<int>(rank) * kHalf + quarter * 32 < rows ? min(p.block_n, p.vocab - t.n * p.block_n) : 0;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
          if (group * 32 + 32 * GROUPS * i < end) {
#pragma unroll
            for (int j = 0; j < 32; ++j) s[j & 3] += ex2_approx((z[i][j] - top) * kLog2e);   // (differences first: logits may be at the lowest number)
          }
          if (i == BLOCKS / 2) {
            if (taken && !(ok = wait_sum())) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < i; ++k) take(k, next_end);
          }
          if (i >= BLOCKS / 2) take(i, next_end);
        }
        if (!ok) break;
        if (taken) leave_sum();
        if (row < rows) *part = make_float2(top, (s[0] + s[1]) + (s[2] + s[3]));
      }
    } else {
      for (bool first = true; next_announced(first); first = false) {
        const int m0 = t.m * kTile + static_cast<int>(rank) * kHalf + quarter * 32;   // of this warp
        const int row = m0 + lane;
        const bool row_counts = row < rows;
        if (MODE != kProducts && t.kind == 0) {
          const int label = row_counts ? p.labels[row] : -1;
          const float2 shift = row_counts ? p.row_shift[row] : make_float2(0.f, 0.f);   // lse, weight
          // The logits of this warp's rows and columns, in registers: the last of their accumulators is free before anything is done with them.
          const int n0 = t.n * p.block_n;                 // in the piece
          // (what anything below looks at: in whole k-blocks of the products that sum over columns and over rows)
          const int columns = m0 >= (rows + 63) / 64 * 64 ? 0 : min(p.block_n, (work.cols - n0 + 63) / 64 * 64);
          float z[blocks(MODE)][32] = {};
          if (p.bias != nullptr && lane < 16 && work.col0 + n0 + lane * 16 < p.vocab) touch(p.bias + work.col0 + n0 + lane * 16);
          bool ok = true;
          for (int i = 0; ok && i < sums; ++i) {
            if (!(ok = wait_sum())) break;
            tc_fence_after();
            join_sums(z, my_tmem + static_cast<uint32_t>(acc * kTile), group * 32, 32 * GROUPS, columns);
            leave_sum();
          }
          if (!ok) break;
          add_bias(p.bias, work.col0 + n0 + group * 32, 32 * GROUPS, p.vocab, lane, z);
          const bool whole = __all_sync(0xffffffffu, row_counts);
          bf16* g_out = p.g + static_cast<int64_t>(work.g_row0 + m0 + (lane & ~3)) * g_pitch + (lane & 3) * 8;
#pragma unroll
          for (int i = 0; i < blocks(MODE); ++i) {
            const int c = group * 32 + 32 * GROUPS * i;
            if (c >= columns) break;
            const int local = n0 + c;
            const int col = work.col0 + local;
            float (&g)[32] = z[i];
#pragma unroll
            for (int j = 0; j < 32; ++j) g[j] = shift.y * probability(g[j], shift.x);
            const int at = label - col;
            if (__any_sync(0xffffffffu, at >= 0 && at < 32)) {
              float mine = 0.f;
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                if (j == at) {
                  g[j] -= shift.y;
                  mine = g[j];
                }
              }
              // what rounding takes from the label's entry
              if (at >= 0 && at < 32) p.row_residual[row] = mine - __bfloat162float(__float2bfloat16_rn(mine));
            }
            if (!whole) {                               // (behind the last row lies anything)
#pragma unroll
              for (int j = 0; j < 32; ++j) g[j] = row_counts ? g[j] : 0.f;
            }
            uint4 out[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
              out[q] = make_uint4(pack_bf16(g[q * 8], g[q * 8 + 1]), pack_bf16(g[q * 8 + 2], g[q * 8 + 3]), pack_bf16(g[q * 8 + 4], g[q * 8 + 5]),
                                  pack_bf16(g[q * 8 + 6], g[q * 8 + 7]));
            exchange_pieces(out, lane);
#pragma unroll
            for (int q = 0; q < 4; ++q) *reinterpret_cast<uint4*>(g_out + static_cast<int64_t>(q) * g_pitch + local) = out[q];
            if (two_terms) {
              auto rest = [&](int j) { return g[j] - __bfloat162float(__float2bfloat16_rn(g[j])); };
#pragma unroll
              for (int q = 0; q < 4; ++q)
                out[q] = make_uint4(pack_bf16(rest(q * 8), rest(q * 8 + 1)), pack_bf16(rest(q * 8 + 2), rest(q * 8 + 3)),
                                    pack_bf16(rest(q * 8 + 4), rest(q * 8 + 5)), pack_bf16(rest(q * 8 + 6), rest(q * 8 + 7)));
              exchange_pieces(out, lane);
#pragma unroll
              for (int q = 0; q < 4; ++q) *reinterpret_cast<uint4*>(g_out + static_cast<int64_t>(kHalf + q) * g_pitch + local) = out[q];
            }
            if (p.bias_parts != nullptr && m0 < rows) {
              const float s = column_sums(g, lane);
              if (local + lane < work.cols) p.bias_parts[static_cast<int64_t>(m0 / 32) * p.bias_pitch + col + lane] = s;
            }
          }
          continue;
        }
        if (!wait_sum()) break;
        tc_fence_after();
        const uint32_t taddr0 = my_tmem + static_cast<uint32_t>(acc * kTile);
        if (t.kind == 1) {
          const int n0 = t.n * p.block_h;
          float* sums = p.dx_sums + (static_cast<int64_t>(t.range) * work.row_pitch + m0 + (lane & ~3)) * p.hidden + (lane & 3) * 4;
#pragma unroll 1
          for (int c = group * 32; c < p.block_h; c += 32 * GROUPS) {
            if (n0 + c >= p.hidden || m0 >= rows) break;
            uint32_t v[32];
            if (t.k_blocks > 0) {
              tmem_ld_32x32(taddr0 + c, v);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] = 0u;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint4 out[4];
#pragma unroll
              for (int q = 0; q < 4; ++q)
                out[q] = make_uint4(v[half * 16 + q * 4], v[half * 16 + q * 4 + 1], v[half * 16 + q * 4 + 2], v[half * 16 + q * 4 + 3]);
              exchange_pieces(out, lane);
              const int col = n0 + c + half * 16;
              if (col + (lane & 3) * 4 >= p.hidden) continue;
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                float* to = sums + static_cast<int64_t>(q) * p.hidden + col;
                if (work.prev_col0 == 0) *reinterpret_cast<uint4*>(to) = out[q]; else red_add_v4(to, out[q]);
              }
            }
          }
        } else {
          const int n0 = t.n * p.block_h;
          const int word = work.prev_col0 + m0 + (lane & ~3);   // row of dW of this lane's first piece
          bf16* dw = p.dw + static_cast<int64_t>(word) * p.dw_stride + (lane & 3) * 8;
#pragma unroll 1
          for (int c = group * 32; c < p.block_h; c += 32 * GROUPS) {
            const int col = n0 + c;
            if (col >= p.hidden || work.prev_col0 + m0 >= p.vocab) break;
            uint32_t v[32];
            if (t.k_blocks > 0) {
              tmem_ld_32x32(taddr0 + c, v);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] = 0u;
            }
            if (p.accumulate) {
              const int mine = work.prev_col0 + row;
              const bf16* old = p.dw + static_cast<int64_t>(mine) * p.dw_stride + col;
#pragma unroll
              for (int q = 0; q < 4; ++q) {               // (hidden is a multiple of eight)
                if (mine >= p.vocab || col + q * 8 >= p.hidden) continue;
                const uint4 b = *reinterpret_cast<const uint4*>(old + q * 8);
                const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  v[q * 8 + 2 * j] = __float_as_uint(__uint_as_float(v[q * 8 + 2 * j]) + bf16_lo(w[j]));
                  v[q * 8 + 2 * j + 1] = __float_as_uint(__uint_as_float(v[q * 8 + 2 * j + 1]) + bf16_hi(w[j]));
                }
              }
              __syncwarp();                               // (all of the warp has read before any of it writes)
            }
            uint4 out[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t o[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) o[j] = pack_bf16(__uint_as_float(v[q * 8 + 2 * j]), __uint_as_float(v[q * 8 + 2 * j + 1]));
              out[q] = make_uint4(o[0], o[1], o[2], o[3]);
            }
            exchange_pieces(out, lane);
            if (col + (lane & 3) * 8 >= p.hidden) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (word + q < p.vocab) *reinterpret_cast<uint4*>(dw + static_cast<int64_t>(q) * p.dw_stride + col) = out[q];
          }
        }
        leave_sum();
      }
    }
  }

  tc_fence_before();
  __syncwarp();
  cluster_sync_all();
  if (threadIdx.x == 0 && *abort_flag && p.status != nullptr) atomicOr(p.status, kFlagWaitTimeout);
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

// ---- few rows ------------------------------------------------------------------------------------

// Up to 128 rows the products are taken turned: 128 words are the rows (lanes) of an accumulator and the rows of x, rounded up to sixteen,
// its columns, so that a tile costs what its rows cost and the kernel streams W: 16 KB of it per k-block and stage, up to twelve stages.
// (20 rows x 30522 x 768 on tiles of 256 rows: 20 us, of which the tensor cores worked on empty rows for 6.)  An epilogue thread has one
// word and all rows.
//   forward   largest logit and sum of exponentials of a row over the 32 words of a warp: halves of the rows are exchanged for halves of the
//             words (as column_sums), running over the CTA's tiles; the four warps are put together at the end
//   Logits wider than four k-blocks are made in sums (see sum_blocks) that go through registers back to the last one's accumulator.
//   backward  g by words, [vocab][64 or 128 rows], zeros in rows without a label and behind the last: as it is the operand along K for dW and
//             the MN-major one for dx; db is a thread's own sum.  A row of dW whose word is a label is little else than that entry of g
//             times a row of x, and with so few rows such entries are most of dW: where one of 256 words is a label, g of all of them is
//             kept in two bf16 terms, which the product for dW takes one behind the other along K.  The hidden states are copied once with zeros in the rows without a label,
//             for the product that sums over rows.
constexpr int kFewRows = 128;
constexpr int kFewWarps = 8;             // of the epilogue: two per quarter of the words, which share the blocks of 32 rows
constexpr int kFewThreads = (2 + kFewWarps) * 32;
constexpr int kFewMaxStages = 12;
constexpr int kFewStageA = 128 * 128;
constexpr int kFewBook = 8192;
constexpr int kFewRing = 227 * 1024 - 1024 - kFewBook;
constexpr int kFewAccs = 4;              // accumulators, of a sum of a tile's logits each
constexpr uint32_t kFewTmemCols = kFewAccs * kFewRows;

// Largest over the 32 lanes of a warp of 32 columns each, column `lane` in the result (see column_sums).
__device__ __forceinline__ float column_max(const float (&z)[32], int lane) {
  float c[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const bool upper = (lane & 16) != 0;
    const float give = upper ? z[i] : z[i + 16], keep = upper ? z[i + 16] : z[i];
    c[i] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, 16));
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    const bool upper = (lane & o) != 0;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float give = upper ? c[i] : c[i + o], keep = upper ? c[i + o] : c[i];
      c[i] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, o));
    }
  }
  return c[0];
}

template <bool GRAD, int STAGE_BLOCKS>
__global__ void __launch_bounds__(kFewThreads, 1) vocab_few_tcgen05(const __grid_constant__ VocabFewParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t ring = smem_u32(smem);
  uint8_t* book = smem + kFewRing;
  const uint32_t bar_full = smem_u32(book);
  const uint32_t bar_empty = bar_full + 8 * kFewMaxStages;
  const uint32_t bar_acc_full = bar_empty + 8 * kFewMaxStages;
  const uint32_t bar_acc_empty = bar_acc_full + 8 * kFewAccs;
  const uint32_t bar_db = bar_acc_empty + 8 * kFewAccs;  // (backward) [accumulator][quarter]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(book + 8 * (2 * kFewMaxStages + 6 * kFewAccs));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_label = reinterpret_cast<int*>(book + 512);                    // of every row; -1 where it takes no part
  float2* s_row = reinterpret_cast<float2*>(book + 512 + 512);          // (backward) lse, weight
  float2* s_part = reinterpret_cast<float2*>(book + 512 + 512 + 1024);  // (forward) [quarter][row]
  float* s_db = reinterpret_cast<float*>(s_part);                       // (backward) [accumulator][quarter][word]
  static_assert(8 * (2 * kFewMaxStages + 6 * kFewAccs) + 8 <= 512 && 512 + 512 + 1024 + 4 * kFewRows * 8 <= kFewBook, "bookkeeping");
  static_assert(kFewAccs * 4 * 32 * 4 <= 4 * kFewRows * 8, "sums of db");

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int stages = p.stages, stage_bytes = p.stage_bytes;
  const int k_blocks = (p.hidden + 63) / 64;
  constexpr int SUM_BLOCKS = 4 / STAGE_BLOCKS * STAGE_BLOCKS;   // k-blocks of a sum, in whole stages
  const int sums = (k_blocks + SUM_BLOCKS - 1) / SUM_BLOCKS;
  constexpr uint32_t STAGE_A = STAGE_BLOCKS * kFewStageA;
  const int tiles = (p.vocab + 127) / 128;
  if (tid == 0) {
    for (int s = 0; s < kFewMaxStages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 1);
    }
    for (int a = 0; a < kFewAccs; ++a) {
      mbar_init(bar_acc_full + 8 * a, 1);
      mbar_init(bar_acc_empty + 8 * a, kFewWarps);
    }
    for (int i = 0; i < 4 * kFewAccs; ++i) mbar_init(bar_db + 8 * i, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
    prefetch_tensormap(&p.x_k);
    prefetch_tensormap(&p.w_k);
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), kFewTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  grid_dependency_wait();
  grid_launch_dependents();

  if (warp == 0) {
    // ------------------------------ TMA producer ------------------------------
    const bool leader = elect_one();
    int stage = 0;
    uint32_t phase = 0;
    long long issued = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      for (int kb = 0; kb < k_blocks; kb += STAGE_BLOCKS) {
        if (!__all_sync(0xffffffffu, mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag))) { ok = false; break; }
        if (leader) {
          const uint32_t a = ring + stage * stage_bytes;
          mbar_expect_tx(bar_full + 8 * stage, stage_bytes);
          if (STAGE_BLOCKS > 1) {
            tma_load_3d(a, &p.w_k, 0, tile * 128, kb, bar_full + 8 * stage);
            tma_load_3d(a + STAGE_A, &p.x_k, 0, 0, kb, bar_full + 8 * stage);
          } else {
            tma_load_2d(a, &p.w_k, kb * 64, tile * 128, bar_full + 8 * stage);
            tma_load_2d(a + STAGE_A, &p.x_k, kb * 64, 0, bar_full + 8 * stage);
          }
        }
        ++issued;
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok && leader) {
      const int pending = issued < stages ? static_cast<int>(issued) : stages;
      for (int i = 0; i < pending; ++i) {
        if (stage == 0) { stage = stages; phase ^= 1u; }
        --stage;
        mbar_drain(bar_full + 8 * stage, phase);
      }
    }
  } else if (warp == 1) {
    // ------------------------------ MMA issuer --------------------------------
    const bool leader = elect_one();
    const uint32_t idesc = umma_idesc_bf16(128, p.columns);
    int stage = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      for (int begin = 0; begin < k_blocks && ok; begin += SUM_BLOCKS) {
        if (!__all_sync(0xffffffffu, mbar_wait(bar_acc_empty + 8 * acc, acc_phase ^ 1u, abort_flag))) { ok = false; break; }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * kFewRows);
        const int end = min(begin + SUM_BLOCKS, k_blocks);
        for (int kb = begin; kb < end; kb += STAGE_BLOCKS) {
          if (!__all_sync(0xffffffffu, mbar_wait(bar_full + 8 * stage, phase, abort_flag))) { ok = false; break; }
          tc_fence_after();
          if (leader) {
#pragma unroll
            for (int j = 0; j < STAGE_BLOCKS; ++j) {
              const uint64_t da = smem_desc_sw128(ring + stage * stage_bytes + j * kFewStageA);
              const uint64_t db = smem_desc_sw128(ring + stage * stage_bytes + STAGE_A + j * p.columns * 128);
#pragma unroll
              for (int k = 0; k < 4; ++k) umma_bf16(d_tmem, da + 2 * k, db + 2 * k, idesc, (kb - begin) | j | k ? 1u : 0u);
            }
            umma_commit(bar_empty + 8 * stage);
          }
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if (leader) umma_commit(bar_acc_full + 8 * acc);
        if (++acc == kFewAccs) { acc = 0; acc_phase ^= 1u; }
      }
    }
  } else {
    // ------------------------------ epilogue ----------------------------------
    const int quarter = warp & 3;
    const int half = (warp - 2) >> 2;                               // of the two warps of the quarter
    const int first = tid - 64;
    if (first < kFewRows) {
      int label = first < p.rows ? p.labels[first] : -1;
      if (GRAD && label >= p.vocab && blockIdx.x == 0 && p.status != nullptr) atomicOr(p.status, kFlagBadToken);
      if (label >= p.vocab) label = -1;
      s_label[first] = label;
      if (GRAD)
        s_row[first] = label >= 0 ? make_float2(p.lse[first], p.grad_loss != nullptr ? p.grad_loss[first] : 1.f) : make_float2(0.f, 0.f);
    }
    // (the epilogue warps; nothing that can give up comes before it)
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kFewWarps) : "memory");
    if (GRAD && p.x_clean != nullptr) {
      // (rows of hidden states, those without a part as zeros, in whole k-blocks of the product over rows)
      const int vectors = p.hidden / 8;
      for (int r = blockIdx.x; r < p.g_pitch; r += gridDim.x) {
        const bool there = s_label[r] >= 0;
        for (int c = first; c < vectors; c += 32 * kFewWarps)
          reinterpret_cast<uint4*>(p.x_clean + static_cast<int64_t>(r) * p.hidden)[c] =
              there ? __ldg(reinterpret_cast<const uint4*>(p.x + static_cast<int64_t>(r) * p.x_stride) + c) : make_uint4(0, 0, 0, 0);
      }
    }
    if (GRAD && blockIdx.x == 0 && first == 0) *p.counter = 0;
    float2* my_part = s_part + quarter * kFewRows + lane;           // (forward) largest logit and sum of row 32 * i + lane
    if (!GRAD) {
      for (int i = half; i < 4; i += 2) my_part[i * 32] = make_float2(kFloor, 0.f);
    }
    int acc = 0;
    uint32_t acc_phase = 0, db_phases = 0;                          // (a bit per accumulator)
    auto wait_sum = [&] { return __all_sync(0xffffffffu, mbar_wait(bar_acc_full + 8 * acc, acc_phase, abort_flag)); };
    auto leave_sum = [&] {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_acc_empty + 8 * acc);
      if (++acc == kFewAccs) { acc = 0; acc_phase ^= 1u; }
    };
    const int chunks = ((GRAD ? p.g_pitch : p.rows) + 31) / 32;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
      const int word0 = tile * 128 + quarter * 32, word = word0 + lane;
      const bool is_word = word < p.vocab;
      const float bias = p.bias != nullptr && is_word ? __bfloat162float(p.bias[word]) : 0.f;
      const uint32_t my_tmem = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
      if (sums > 1) {
        float sum[kFewRows / 64][32] = {};
        bool ok = true;
        for (int i = 0;; ++i) {
          if (!(ok = wait_sum())) break;
          tc_fence_after();
          join_sums(sum, my_tmem + static_cast<uint32_t>(acc * kFewRows), half * 32, 64, chunks * 32);
          if (i + 1 == sums) break;
          leave_sum();
        }
        if (!ok) break;
        put_sums(sum, my_tmem + static_cast<uint32_t>(acc * kFewRows), half * 32, 64, chunks * 32);
      } else {
        if (!wait_sum()) break;
        tc_fence_after();
      }
      const uint32_t taddr0 = my_tmem + static_cast<uint32_t>(acc * kFewRows);
      float db = 0.f;
      bool two_terms = false;                                       // one of the 256 words that a tile of dW has is a label
      if (GRAD) {
        bool mine = false;
#pragma unroll
        for (int i = 0; i < kFewRows / 32; ++i) {
          const int l = s_label[i * 32 + lane];
          mine |= l >= 0 && (l >> 8) == (tile >> 1);
        }
        two_terms = __any_sync(0xffffffffu, mine);
        if ((tile & 1) == 0 && quarter == 0 && half == 0 && lane == 0) p.two_terms[tile >> 1] = two_terms ? 1 : 0;
      }
      // (not unrolled: four copies of the body are more than the instruction cache holds; the first tile took 13 k clocks with them)
#pragma unroll 1
      for (int i = half; i < chunks; i += 2) {
        uint32_t v[32];
        tmem_ld_32x32(taddr0 + i * 32, v);
        tmem_ld_wait();
        float z[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) z[j] = __uint_as_float(v[j]) + bias;
        const int my_label = s_label[i * 32 + lane];                // of row i * 32 + lane
        // rows whose label is one of this warp's words
        uint32_t hits = __ballot_sync(0xffffffffu, my_label >= word0 && my_label < word0 + 32);
        if (!GRAD) {
          if (hits != 0) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if ((hits >> j) & 1u) {
                if (s_label[i * 32 + j] == word) p.label_logit[i * 32 + j] = z[j];
              }
            }
          }
          if (!is_word) {
#pragma unroll
            for (int j = 0; j < 32; ++j) z[j] = -INFINITY;
          }
          const float2 part = my_part[i * 32];
          const float next = fmaxf(part.x, column_max(z, lane));
#pragma unroll
          for (int j = 0; j < 32; ++j) z[j] = ex2_approx((z[j] - __shfl_sync(0xffffffffu, next, j)) * kLog2e);
          my_part[i * 32] = make_float2(next, part.y * ex2_approx((part.x - next) * kLog2e) + column_sums(z, lane));
        } else {
          const uint32_t counts = __ballot_sync(0xffffffffu, my_label >= 0);
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const float2 shift = s_row[i * 32 + j];
            z[j] = shift.y * probability(z[j], shift.x);
          }
          if (hits != 0) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if (((hits >> j) & 1u) && s_label[i * 32 + j] == word) {
                z[j] -= s_row[i * 32 + j].y;
                p.row_residual[i * 32 + j] = z[j] - __bfloat162float(__float2bfloat16_rn(z[j]));   // what rounding takes from the label's entry
              }
            }
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) z[j] = ((counts >> j) & 1u) && is_word ? z[j] : 0.f;
          float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 32; ++j) s[j & 3] += z[j];
          db += (s[0] + s[1]) + (s[2] + s[3]);
          uint4 out[4];
#pragma unroll
          for (int q = 0; q < 4; ++q)
            out[q] = make_uint4(pack_bf16(z[q * 8], z[q * 8 + 1]), pack_bf16(z[q * 8 + 2], z[q * 8 + 3]), pack_bf16(z[q * 8 + 4], z[q * 8 + 5]),
                                pack_bf16(z[q * 8 + 6], z[q * 8 + 7]));
          exchange_pieces(out, lane);
          bf16* g = p.g + static_cast<int64_t>(word0 + (lane & ~3)) * (2 * p.g_pitch) + i * 32 + (lane & 3) * 8;
#pragma unroll
          for (int q = 0; q < 4; ++q) *reinterpret_cast<uint4*>(g + q * 2 * p.g_pitch) = out[q];
          if (two_terms) {
#pragma unroll
            for (int j = 0; j < 32; ++j) z[j] -= __bfloat162float(__float2bfloat16_rn(z[j]));
#pragma unroll
            for (int q = 0; q < 4; ++q)
              out[q] = make_uint4(pack_bf16(z[q * 8], z[q * 8 + 1]), pack_bf16(z[q * 8 + 2], z[q * 8 + 3]), pack_bf16(z[q * 8 + 4], z[q * 8 + 5]),
                                  pack_bf16(z[q * 8 + 6], z[q * 8 + 7]));
            exchange_pieces(out, lane);
#pragma unroll
            for (int q = 0; q < 4; ++q) *reinterpret_cast<uint4*>(g + p.g_pitch + q * 2 * p.g_pitch) = out[q];
          }
        }
      }
      if (GRAD && p.db != nullptr && chunks > 1) {                 // the sums of the other warp's rows
        float* other = s_db + (acc * 4 + quarter) * 32 + lane;
        const uint32_t bar = bar_db + 8 * (acc * 4 + quarter);
        if (half == 1) {
          *other = db;
          __syncwarp();
          if (lane == 0) mbar_arrive(bar);
        } else {
          if (!__all_sync(0xffffffffu, mbar_wait(bar, (db_phases >> acc) & 1u, abort_flag))) break;
          db += *other;
        }
        db_phases ^= 1u << acc;
      }
      if (GRAD && p.db != nullptr && half == 0 && is_word) p.db[word] = p.accumulate ? p.db[word] + db : db;
      leave_sum();
    }
  }

  tc_fence_before();
  __syncthreads();
  if (!GRAD && tid < p.rows) {
    float top = kFloor, sum = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) top = fmaxf(top, s_part[q * kFewRows + tid].x);
#pragma unroll
    for (int q = 0; q < 4; ++q) sum += s_part[q * kFewRows + tid].y * ex2_approx((s_part[q * kFewRows + tid].x - top) * kLog2e);
    p.parts[tid * p.part_pitch + blockIdx.x] = make_float2(top, sum);
  }
  if (tid == 0 && *abort_flag && p.status != nullptr) atomicOr(p.status, kFlagWaitTimeout);
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem_base, kFewTmemCols);
  }
}

// ---- rows with a label ---------------------------------------------------------------------------

constexpr int kRowsThreads = 256;

// Ranges of the vocabulary that dx of a piece is summed over in: a tile of it should be no longer than half of what a pair has to do
// in the launch (a tile counts as at least six k-blocks: its epilogue).
__host__ __device__ inline int choose_ranges(int rows, int piece, int pieces, int hidden, int block_h) {
  const int64_t m = (rows + kTile - 1) / kTile, h = (hidden + block_h - 1) / block_h, v = (piece + kTile - 1) / kTile;
  const int k1 = (piece + 63) / 64, k2 = (rows + 63) / 64, k0 = (hidden + 63) / 64;
  const int64_t all = m * h * k1 + v * h * (k2 > 6 ? k2 : 6) + (pieces > 1 ? m * v * (k0 > 6 ? k0 : 6) : 0);
  int64_t longest = all / 74 / 2;
  if (longest < 8) longest = 8;
  const int64_t ranges = (k1 + longest - 1) / longest;
  return ranges < kMaxRanges ? static_cast<int>(ranges) : kMaxRanges;
}

// The cut for `rows` rows: pieces as wide as the buffers hold for so many, as few ranges as keep the pairs busy.  One thread per launch.
__device__ inline void make_work(const VocabRowsParams& p, int rows, int index) {
  VocabWork w = {};
  w.rows = rows;
  w.row_tiles = (rows + kTile - 1) / kTile;
  w.row_pitch = max(1, w.row_tiles) * kTile;
  while (w.shift < p.max_shift && (p.buffer_rows >> (w.shift + 1)) >= w.row_pitch) ++w.shift;
  const int piece = p.piece << w.shift, pieces = (p.vocab + piece - 1) / piece, hidden_tiles = (p.hidden + p.block_h - 1) / p.block_h;
  w.ranges = min(choose_ranges(rows, min(piece, p.vocab), pieces, p.hidden, p.block_h), p.dx_rows / w.row_pitch);
  if (index < pieces) {
    w.col0 = index * piece;
    w.cols = min(piece, p.vocab - w.col0);
    w.g_row0 = (index & (p.buffers - 1)) * (p.buffer_rows >> w.shift);
    w.n0 = w.row_tiles * ((w.cols + kTile - 1) / kTile);
  }
  if (index > 0 && index <= pieces) {
    w.prev_col0 = (index - 1) * piece;
    w.prev_cols = min(piece, p.vocab - w.prev_col0);
    w.prev_g_row0 = ((index - 1) & (p.buffers - 1)) * (p.buffer_rows >> w.shift);
    w.n1 = p.want_x ? w.row_tiles * hidden_tiles * w.ranges : 0;
    w.n2 = p.want_w ? (w.prev_cols + kTile - 1) / kTile * hidden_tiles : 0;
    w.k1 = ((w.prev_cols + 63) / 64 + w.ranges - 1) / w.ranges;
    w.k2 = terms_of_g(rows) * ((rows + 63) / 64);
  }
  p.work[index] = w;
}

// A CTA per `rows_per_cta` rows counts the labels before them and all of them (a few KB that stay in L2), and gives every row with a
// label its place.  Unless all rows have one, their hidden states are gathered, with zeros up to the next k-block of the products that
// sum over rows.
__global__ void __launch_bounds__(kRowsThreads) vocab_rows_kernel(const __grid_constant__ VocabRowsParams p) {
  __shared__ int s_before, s_all;
  __shared__ int s_warp[kRowsThreads / 32];
  __shared__ int s_place[kRowsThreads];
  grid_dependency_wait();
  grid_launch_dependents();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int first = blockIdx.x * p.rows_per_cta;
  const int last = min(first + p.rows_per_cta, p.rows);
  auto has_label = [&](int r) { const int l = p.labels[r]; return l >= 0 && l < p.vocab; };
  if (tid == 0) s_before = s_all = 0;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll 8
  for (int r = tid; r < p.rows; r += kRowsThreads) {
    const int has = has_label(r) ? 1 : 0;
    all += has;
    if (r < first) before += has;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    before += __shfl_xor_sync(0xffffffffu, before, o);
    all += __shfl_xor_sync(0xffffffffu, all, o);
  }
  if (lane == 0) {
    atomicAdd(&s_before, before);          // (whole numbers: any order)
    atomicAdd(&s_all, all);
  }
  __syncthreads();
  all = s_all;
  if (blockIdx.x == 0) {
    if (tid == 0) *p.count = all;
    for (int i = tid; i < p.n_counters; i += kRowsThreads) {
      p.counters[i] = 0;
      make_work(p, all, i);
    }
  }
  const int vectors = p.hidden / 8;
  for (int r0 = first; r0 < last; r0 += kRowsThreads) {
    // places of up to 256 rows, then their copies, a warp per row
    const int r = r0 + tid;
    const bool has = r < last && has_label(r);
    const uint32_t mask = __ballot_sync(0xffffffffu, has);
    if (lane == 0) s_warp[warp] = __popc(mask);
    __syncthreads();
    int place = s_before + __popc(mask & ((1u << lane) - 1));
    for (int w = 0; w < warp; ++w) place += s_warp[w];
    s_place[tid] = has ? place : -1;
    if (r < last) {
      if (p.labels[r] >= p.vocab && p.status != nullptr) atomicOr(p.status, kFlagBadToken);
      if (has) {
        p.row_of[place] = r;
        p.row_label[place] = p.labels[r];
        if (p.row_shift != nullptr) p.row_shift[place] = make_float2(p.lse[r], p.grad_loss != nullptr ? p.grad_loss[r] : 1.f);
      } else if (p.loss_out != nullptr) {
        p.loss_out[r] = 0.f;
        p.lse_out[r] = 0.f;
      }
    }
    __syncthreads();
    if (all != p.rows) {
      const int end = min(kRowsThreads, last - r0);
      for (int i = warp; i < end; i += kRowsThreads / 32) {
        const int to = s_place[i];
        if (to < 0) {
          if (p.dx != nullptr) {
            uint4* zeros = reinterpret_cast<uint4*>(p.dx + static_cast<int64_t>(r0 + i) * p.dx_stride);
            for (int c = lane; c < vectors; c += 32) zeros[c] = make_uint4(0, 0, 0, 0);
          }
          continue;
        }
        const uint4* src = reinterpret_cast<const uint4*>(p.x + static_cast<int64_t>(r0 + i) * p.x_stride);
        uint4* dst = reinterpret_cast<uint4*>(p.gathered + static_cast<int64_t>(to) * p.hidden);
#pragma unroll 4
        for (int c = lane; c < vectors; c += 32) dst[c] = __ldg(src + c);
      }
    }
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < kRowsThreads / 32; ++w) s_before += s_warp[w];
    }
    __syncthreads();
  }
  if (all != p.rows && blockIdx.x == 0) {
    const int64_t from = static_cast<int64_t>(all) * vectors, to = static_cast<int64_t>((all + 63) / 64 * 64) * vectors;
    for (int64_t i = from + tid; i < to; i += kRowsThreads) reinterpret_cast<uint4*>(p.gathered)[i] = make_uint4(0, 0, 0, 0);
  }
}

// ---- a row's tiles put together ------------------------------------------------------------------

constexpr int kJoinThreads = 128;
constexpr int kSharedUnits = 1024;

// A warp per row: log-sum-exp and loss from (largest logit, sum) of every half tile.
__global__ void __launch_bounds__(kJoinThreads) vocab_loss_join_kernel(const __grid_constant__ VocabJoinParams p) {
  const int lane = threadIdx.x & 31;
  const int step = gridDim.x * (kJoinThreads / 32);
  int row = blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5);
  // The kernel before this one (the product) has waited for all before it and lets this one start after that: labels, places and the count
  // are complete when this kernel begins.
  const int rows = p.count != nullptr ? min(p.rows, __ldcg(p.count)) : p.rows;
  int label = row < rows ? __ldcg(p.labels + row) : 0, to = row;
  if (p.row_of != nullptr && row < rows) to = __ldcg(p.row_of + row);
  grid_dependency_wait();
  grid_launch_dependents();
  for (bool first = true; row < rows; row += step, first = false) {
    if (!first) {
      label = p.labels[row];
      to = p.row_of != nullptr ? p.row_of[row] : row;
    }
    if (label < 0 || label >= p.vocab) {             // (only where the rows were not gathered)
      if (lane == 0) {
        if (label >= p.vocab && p.status != nullptr) atomicOr(p.status, kFlagBadToken);
        p.loss[to] = 0.f;
        p.lse[to] = 0.f;
      }
      continue;
    }
    const float2* parts = p.parts + static_cast<int64_t>(row) * p.part_pitch;
    float top = kFloor;
    for (int i = lane; i < p.n_parts; i += 32) top = fmaxf(top, parts[i].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float sum = 0.f;
    for (int i = lane; i < p.n_parts; i += 32) {
      const float2 part = parts[i];
      sum += part.y * exp2f((part.x - top) * kLog2e);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) {
      const float log_sum = logf(sum);
      p.lse[to] = top + log_sum;
      p.loss[to] = (top - p.label_logit[row]) + log_sum;
    }
  }
}

// The last launch of a gradient.
// dx: the ranges of a row added up in order, and what rounding took from the label's entry of g times the label's row of W (that one entry
// is most of a row of g: without this a row of dx would be off by its rounding); rounded once, to the caller's row.  A warp per row in use and
// 256 columns.  (Rows without a label: zeros, from the rows' kernel, or here where the rows are in place.)
// db (the first db_ctas CTAs): the sums of all blocks of 32 rows, in order; a CTA per 32 columns, every warp each fourth block.
__global__ void __launch_bounds__(kJoinThreads) vocab_finish_kernel(const __grid_constant__ VocabFinishParams p) {
  __shared__ float s_sum[kJoinThreads / 32][32];
  __shared__ float s_acc[kJoinThreads / 32][8][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (static_cast<int>(blockIdx.x) < p.db_ctas) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int blocks = (__ldcg(&p.work->rows) + 31) / 32;
    const int col = blockIdx.x * 32 + lane;
    float sum = 0.f;
    if (col < p.vocab) {
#pragma unroll 8
      for (int b = warp; b < blocks; b += kJoinThreads / 32) sum += p.bias_parts[static_cast<int64_t>(b) * p.vocab + col];
    }
    s_sum[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || col >= p.vocab) return;
    for (int w = 1; w < kJoinThreads / 32; ++w) sum += s_sum[w][lane];
    p.db[col] = p.accumulate ? p.db[col] + sum : sum;
    return;
  }
  const int blocks = (p.hidden + 255) / 256;
  const int ranges = p.work != nullptr ? __ldcg(&p.work->ranges) : p.ranges;
  const int64_t row_pitch = p.work != nullptr ? __ldcg(&p.work->row_pitch) : p.row_pitch;
  // With many ranges the four warps of a CTA share a unit, every fourth range each, if there are so few units that all of them run at
  // once (77 rows x 768 in 18 ranges 7.6 -> 5.1 us; 4096 x 768, 614 of them in 9 ranges, 11 -> 17).
  const int rows = p.work != nullptr ? __ldcg(&p.work->rows) : p.rows;
  const int64_t units = static_cast<int64_t>(rows) * blocks;
  const bool shared = ranges >= 2 * kJoinThreads / 32 && units <= kSharedUnits;
  const int share = shared ? kJoinThreads / 32 : 1;
  const int64_t step = static_cast<int64_t>(gridDim.x - p.db_ctas) * (shared ? 1 : kJoinThreads / 32);
  const int64_t cta = blockIdx.x - p.db_ctas;
  // Only the sums come from the kernel before this one, which has waited for all before it: the rest of a first unit is fetched before the
  // wait.
  bool waited = false;
  for (int64_t u = shared ? cta : cta * (kJoinThreads / 32) + warp; u < units; u += step) {
    const int place = static_cast<int>(u / blocks), c = static_cast<int>(u % blocks) * 256 + lane * 8;
    const bool inside = c < p.hidden;
    const int label = __ldcg(p.labels + place);
    const int row = p.row_of != nullptr ? __ldcg(p.row_of + place) : place;
    const bool counts = label >= 0 && label < p.vocab;
    uint4 word = make_uint4(0, 0, 0, 0);
    float residual = 0.f;
    if (counts && inside) {
      word = __ldcg(reinterpret_cast<const uint4*>(p.w + static_cast<int64_t>(label) * p.w_stride + c));
      residual = __ldcg(p.row_residual + place);
    }
    if (!waited) {
      grid_dependency_wait();
      grid_launch_dependents();
      waited = true;
    }
    bf16* out = p.dx + static_cast<int64_t>(row) * p.dx_stride + c;
    if (!counts) {                                        // (the same for all who share a unit)
      if (inside && (!shared || warp == 0)) *reinterpret_cast<uint4*>(out) = make_uint4(0, 0, 0, 0);
      continue;
    }
    float acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    if (inside) {
      const float* src = p.sums + static_cast<int64_t>(place) * p.hidden + c;
#pragma unroll 4
      for (int s = shared ? warp : 0; s < ranges; s += share) {
        const float4* f = reinterpret_cast<const float4*>(src + s * row_pitch * p.hidden);
        const float4 x = f[0], y = f[1];
        acc[0] += x.x; acc[1] += x.y; acc[2] += x.z; acc[3] += x.w;
        acc[4] += y.x; acc[5] += y.y; acc[6] += y.z; acc[7] += y.w;
      }
      if (!shared || warp == 0) {
        const uint32_t w[4] = {word.x, word.y, word.z, word.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          acc[2 * j] = fmaf(residual, bf16_lo(w[j]), acc[2 * j]);
          acc[2 * j + 1] = fmaf(residual, bf16_hi(w[j]), acc[2 * j + 1]);
        }
      }
    }
    if (shared) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s_acc[warp][j][lane] = acc[j];
      __syncthreads();
      if (warp == 0) {
        for (int w = 1; w < kJoinThreads / 32; ++w) {
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] += s_acc[w][j][lane];
        }
      }
      __syncthreads();
      if (warp != 0) continue;
    }
    if (inside)
      *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3]), pack_bf16(acc[4], acc[5]), pack_bf16(acc[6], acc[7]));
  }
  // (with no row in use nobody has waited: this kernel must not end before the one in front of it, whose dW the next one may read)
  if (!waited) grid_dependency_wait();
}

template <bool GRAD, int STAGE_BLOCKS>
cudaError_t launch_few_blocks(VocabFewParams p, int sm_count, int* ctas, cudaStream_t stream) {
  auto kernel = vocab_few_tcgen05<GRAD, STAGE_BLOCKS>;
  static PerDeviceOnce once;
  cudaError_t err = per_device_once(once, [&](int) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewRing + kFewBook + 1024);
  });
  if (err != cudaSuccess) return err;
  p.columns = (p.rows + 15) / 16 * 16;
  p.stage_bytes = STAGE_BLOCKS * (kFewStageA + p.columns * 128);
  p.stages = kFewRing / p.stage_bytes < kFewMaxStages ? kFewRing / p.stage_bytes : kFewMaxStages;
  const int tiles = (p.vocab + 127) / 128;
  *ctas = tiles < sm_count ? tiles : (sm_count > 0 ? sm_count : 1);
  if (!GRAD) p.part_pitch = *ctas;
  return launch_kernel(kernel, dim3(*ctas), dim3(kFewThreads), kFewRing + kFewBook + 1024, stream, p);
}
// k-blocks of a stage: a copy takes its warp some 180 clocks to issue whatever its size, and rows of W come in longer pieces.  One where the
// width is no multiple of 64 (a map in whole blocks would reach into the next row); else three, or two with more than 32 rows, whose
// stages of three would be too few.  (30522 x 768 with one, two, three k-blocks: 20 rows 13.9, 13.3, 12.7 us; gradient of 77 rows 45.7, 45.7, 46.5.)
int few_stage_blocks(int rows, int hidden) { return hidden % 64 != 0 ? 1 : (rows <= 32 ? 3 : 2); }
template <bool GRAD>
cudaError_t launch_few(const VocabFewParams& p, int sm_count, int* ctas, cudaStream_t stream) {
  switch (few_stage_blocks(p.rows, p.hidden)) {
    case 3: return launch_few_blocks<GRAD, 3>(p, sm_count, ctas, stream);
    case 2: return launch_few_blocks<GRAD, 2>(p, sm_count, ctas, stream);
    default: return launch_few_blocks<GRAD, 1>(p, sm_count, ctas, stream);
  }
}

template <Mode MODE>
cudaError_t launch_pairs(const VocabLossParams& p, int tiles, int sm_count, cudaStream_t stream) {
  auto kernel = vocab_loss_pair_tcgen05<MODE>;
  static PerDeviceOnce once;
  cudaError_t err = per_device_once(once, [&](int) {
    cudaFuncAttributes has;
    cudaError_t e = cudaFuncGetAttributes(&has, kernel);
    if (e != cudaSuccess) return e;
    if (has.numRegs * threads(MODE) < registers_needed(MODE)) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  });
  if (err != cudaSuccess) return err;
  const int most = sm_count / 2 > 0 ? sm_count / 2 : 1;
  const int workers = tiles < most ? (tiles > 0 ? tiles : 1) : most;
  return launch_kernel(kernel, dim3(2 * workers), dim3(threads(MODE)), kSmemBytes, stream, p, 2u);
}

int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }
size_t whole_lines(size_t bytes) { return (bytes + 255) / 256 * 256; }

// ---- plans -----------------------------------------------------------------------------------------

constexpr int kGatherRows = kTile;       // up to one tile of rows costs the same however few of them count
constexpr int kFewPartCtas = 256;        // place for the CTAs of the kernel for few rows
constexpr int64_t kPieceElements = 64 << 20;   // of g of one piece: 128 MB, unless its narrowest
constexpr int kMinPiece = 2048;

struct ForwardPlan {
  int block_n, tiles_n, part_pitch;
  int64_t row_pitch;                     // rows in whole tiles
  bool gather;
  size_t count, row_of, row_label, label_logit, parts, gathered, bytes;
};
ForwardPlan forward_plan(int rows, int vocab, int hidden, int sm_count) {
  ForwardPlan f;
  f.row_pitch = static_cast<int64_t>(ceil_div(rows, kTile)) * kTile;
  f.gather = rows > kGatherRows;
  // Width of the tiles: the last round of pairs is as full as can be.  With many tiles the widest (fewest bytes staged per product);
  // with one tile of rows the pairs' columns decide, e.g. 30522 of them on 74 pairs: two rounds of 224 instead of two of 256.
  const int pairs = sm_count / 2 > 0 ? sm_count / 2 : 1;
  const int m = static_cast<int>(f.row_pitch / kTile);
  int64_t best = -1;
  f.block_n = kTile;
  for (int bn = kTile; bn >= kHalf; bn -= 32) {
    const int64_t tiles = static_cast<int64_t>(m < 1 ? 1 : m) * ceil_div(vocab, bn);
    const int64_t cost = (tiles + pairs - 1) / pairs * (bn + 16);
    if (best < 0 || cost < best) { best = cost; f.block_n = bn; }
  }
  f.tiles_n = ceil_div(vocab, f.block_n);
  f.part_pitch = groups(kForward) * f.tiles_n;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += whole_lines(bytes); return here; };
  f.count = take(256);
  f.row_of = take(f.row_pitch * 4);
  f.row_label = take(f.row_pitch * 4);
  f.label_logit = take(f.row_pitch * 4);
  const size_t parts_of_row = rows <= kFewRows ? kFewPartCtas : static_cast<size_t>(ceil_div(vocab, kHalf)) * groups(kForward);   // (for the narrowest tiles)
  f.parts = take(static_cast<size_t>(f.row_pitch) * parts_of_row * sizeof(float2));
  f.gathered = take(f.gather ? static_cast<size_t>(f.row_pitch) * hidden * 2 : 0);
  f.bytes = at;
  return f;
}

struct GradPlan {
  int piece, pieces, buffers, block_h, ranges, g_pitch, max_shift;
  bool few;
  int64_t row_pitch, dx_rows;
  size_t count, work, counters, row_of, row_label, row_shift, row_residual, gathered, g, two_terms, dx, bias_parts, bytes;
};
GradPlan grad_plan(int rows, int vocab, int hidden) {
  GradPlan f;
  f.row_pitch = static_cast<int64_t>(ceil_div(rows, kTile)) * kTile;
  const int64_t all = static_cast<int64_t>(ceil_div(vocab, kTile)) * kTile;
  f.few = rows <= kFewRows;
  f.g_pitch = (rows + 63) / 64 * 64;       // (few rows: g is kept by words)
  int64_t piece = kPieceElements / (f.row_pitch > 0 ? f.row_pitch : 1) / kTile * kTile;
  if (piece < kMinPiece) piece = kMinPiece;
  if (f.few) piece = all;
  f.pieces = ceil_div(all, piece);
  f.piece = static_cast<int>(ceil_div(all / kTile, f.pieces)) * kTile;      // (pieces of the same size)
  f.pieces = ceil_div(all, f.piece);
  f.buffers = f.pieces > 1 ? 2 : 1;
  f.block_h = hidden > kHalf ? kTile : kHalf;
  f.max_shift = 0;
  while (!f.few && f.max_shift + 1 < kVocabShifts && (static_cast<int64_t>(f.piece) << f.max_shift) < all && (f.row_pitch >> (f.max_shift + 1)) >= kTile)
    ++f.max_shift;
  f.ranges = choose_ranges(rows, f.piece, f.pieces, hidden, f.block_h);
  f.dx_rows = f.row_pitch * (f.max_shift > 0 && f.ranges < 2 ? 2 : f.ranges);   // (fewer rows with a label: more ranges)
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += whole_lines(bytes); return here; };
  f.count = take(256);
  f.work = take((static_cast<size_t>(f.pieces) + 1) * sizeof(VocabWork));
  f.counters = take((static_cast<size_t>(f.pieces) + 1) * 4);
  f.row_of = take(f.row_pitch * 4);
  f.row_label = take(f.row_pitch * 4);
  f.row_shift = take(f.row_pitch * 8);
  f.row_residual = take(f.row_pitch * 4);
  f.gathered = take(static_cast<size_t>(f.row_pitch) * hidden * 2);
  f.g = take(static_cast<size_t>(f.buffers) * (f.few ? 2 * f.g_pitch : f.row_pitch) * f.piece * 2);
  f.two_terms = take(f.few ? static_cast<size_t>(f.piece / kTile) * 4 : 0);
  f.dx = take(static_cast<size_t>(f.dx_rows) * hidden * 4);
  f.bias_parts = take(f.few ? 0 : static_cast<size_t>(f.row_pitch / 32) * vocab * 4);
  f.bytes = at;
  return f;
}

void launch_rows_setup(VocabRowsParams* r, int* ctas) {
  // a row per warp and CTA (the copies of a warp come one after the other), but at most 1024 CTAs, each of which reads all labels
  r->rows_per_cta = ceil_div(r->rows, 1024) > 8 ? ceil_div(r->rows, 1024) : 8;
  *ctas = ceil_div(r->rows, r->rows_per_cta);
}
template <typename T>
T* at(void* base, size_t offset) { return reinterpret_cast<T*>(static_cast<uint8_t*>(base) + offset); }

}  // namespace

// The operands of the kernel for few rows.
static cudaError_t few_maps(const VocabLossCall& c, VocabFewParams* w) {
  const int columns = ceil_div(c.rows, 16) * 16, blocks = few_stage_blocks(c.rows, c.hidden);
  cudaError_t e;
  if (blocks > 1) {
    e = encode_block_map(&w->x_k, c.x, c.rows, c.hidden, c.x_stride * 2, columns, blocks);
    return e != cudaSuccess ? e : encode_block_map(&w->w_k, c.w, c.vocab, c.hidden, c.w_stride * 2, 128, blocks);
  }
  e = encode_matrix_map(&w->x_k, c.x, c.rows, c.hidden, c.x_stride * 2, columns, 64, false);
  return e != cudaSuccess ? e : encode_matrix_map(&w->w_k, c.w, c.vocab, c.hidden, c.w_stride * 2, 128, 64, false);
}

size_t vocab_loss_workspace(int rows, int vocab, int hidden) { return forward_plan(rows, vocab, hidden, 148).bytes; }
size_t vocab_loss_grad_workspace(int rows, int vocab, int hidden) { return grad_plan(rows, vocab, hidden).bytes; }

cudaError_t launch_vocab_loss(const VocabLossCall& c, int sm_count, cudaStream_t stream) {
  const ForwardPlan f = forward_plan(c.rows, c.vocab, c.hidden, sm_count);
  void* ws = c.workspace;
  cudaError_t e;
  if (c.rows <= kFewRows) {
    VocabFewParams w;
    memset(&w, 0, sizeof(w));
    w.rows = c.rows; w.vocab = c.vocab; w.hidden = c.hidden; w.bias = c.bias; w.labels = c.labels; w.status = c.status;
    w.label_logit = at<float>(ws, f.label_logit); w.parts = at<float2>(ws, f.parts);
    if ((e = few_maps(c, &w)) != cudaSuccess) return e;
    VocabJoinParams j;
    memset(&j, 0, sizeof(j));
    if ((e = launch_few<false>(w, sm_count < kFewPartCtas ? sm_count : kFewPartCtas, &j.n_parts, stream)) != cudaSuccess) return e;
    j.part_pitch = j.n_parts; j.labels = c.labels; j.parts = w.parts; j.label_logit = w.label_logit; j.loss = c.loss; j.lse = c.lse_out;
    j.rows = c.rows; j.vocab = c.vocab; j.status = c.status;
    return launch_kernel(vocab_loss_join_kernel, dim3(ceil_div(c.rows, kJoinThreads / 32)), dim3(kJoinThreads), 0, stream, j);
  }
  if (f.gather) {
    VocabRowsParams r;
    memset(&r, 0, sizeof(r));
    r.labels = c.labels; r.x = c.x; r.x_stride = c.x_stride; r.rows = c.rows; r.vocab = c.vocab; r.hidden = c.hidden;
    r.count = at<int32_t>(ws, f.count); r.row_of = at<int32_t>(ws, f.row_of); r.row_label = at<int32_t>(ws, f.row_label);
    r.gathered = at<bf16>(ws, f.gathered); r.loss_out = c.loss; r.lse_out = c.lse_out; r.status = c.status;
    int ctas = 0;
    launch_rows_setup(&r, &ctas);
    if ((e = launch_kernel(vocab_rows_kernel, dim3(ctas), dim3(kRowsThreads), 0, stream, r)) != cudaSuccess) return e;
  }
  VocabLossParams p;
  memset(&p, 0, sizeof(p));
  p.rows = c.rows; p.vocab = c.vocab; p.hidden = c.hidden; p.block_n = f.block_n; p.block_h = kTile; p.bias = c.bias;
  p.labels = f.gather ? at<int32_t>(ws, f.row_label) : c.labels;
  p.count = f.gather ? at<int32_t>(ws, f.count) : nullptr;
  p.n_tiles = f.tiles_n;
  p.label_logit = at<float>(ws, f.label_logit); p.parts = at<float2>(ws, f.parts); p.part_pitch = f.part_pitch; p.status = c.status;
  if ((e = encode_matrix_map(&p.x_k[0], c.x, c.rows, c.hidden, c.x_stride * 2, kHalf, 64, false)) != cudaSuccess) return e;
  p.x_k[1] = p.x_k[0];
  if (f.gather &&
      (e = encode_matrix_map(&p.x_k[1], at<bf16>(ws, f.gathered), f.row_pitch, c.hidden, static_cast<int64_t>(c.hidden) * 2, kHalf, 64, false)) != cudaSuccess)
    return e;
  if ((e = encode_matrix_map(&p.w_k, c.w, c.vocab, c.hidden, c.w_stride * 2, f.block_n / 2, 64, false)) != cudaSuccess) return e;
  if ((e = launch_pairs<kForward>(p, static_cast<int>(f.row_pitch / kTile) * f.tiles_n, sm_count, stream)) != cudaSuccess) return e;
  VocabJoinParams j;
  memset(&j, 0, sizeof(j));
  j.labels = p.labels; j.count = p.count; j.row_of = f.gather ? at<int32_t>(ws, f.row_of) : nullptr; j.parts = p.parts;
  j.part_pitch = f.part_pitch; j.n_parts = f.part_pitch; j.label_logit = p.label_logit; j.loss = c.loss; j.lse = c.lse_out;
  j.rows = c.rows; j.vocab = c.vocab; j.status = c.status;
  const int ctas = ceil_div(c.rows, kJoinThreads / 32);
  return launch_kernel(vocab_loss_join_kernel, dim3(ctas < 16 * sm_count ? ctas : 16 * sm_count), dim3(kJoinThreads), 0, stream, j);
}

cudaError_t launch_vocab_loss_grad(const VocabLossCall& c, int sm_count, cudaStream_t stream) {
  const GradPlan f = grad_plan(c.rows, c.vocab, c.hidden);
  void* ws = c.workspace;
  cudaError_t e;
  VocabFinishParams d;
  memset(&d, 0, sizeof(d));
  d.sums = at<float>(ws, f.dx); d.labels = c.labels; d.row_residual = at<float>(ws, f.row_residual); d.w = c.w; d.w_stride = c.w_stride;
  d.dx = c.dx; d.dx_stride = c.dx_stride; d.rows = c.rows; d.vocab = c.vocab; d.hidden = c.hidden; d.row_pitch = f.row_pitch; d.ranges = f.ranges;
  d.db = c.db; d.accumulate = c.accumulate;
  unsigned dx_ctas = 0;
  if (c.dx != nullptr) {
    // a CTA per unit where its warps may share one, otherwise a warp
    const int64_t units = static_cast<int64_t>(c.rows) * ceil_div(c.hidden, 256);
    const int64_t ctas = units <= kSharedUnits ? units : (units + kJoinThreads / 32 - 1) / (kJoinThreads / 32);
    dx_ctas = static_cast<unsigned>(ctas < 64 * sm_count ? ctas : 64 * sm_count);
  }
  bf16* gathered = at<bf16>(ws, f.gathered);
  bf16* g = at<bf16>(ws, f.g);
  const int64_t h_stride = static_cast<int64_t>(c.hidden) * 2;
  const bool products = c.dx != nullptr || c.dw != nullptr;
  VocabLossParams p;
  memset(&p, 0, sizeof(p));
  p.rows = c.rows; p.vocab = c.vocab; p.hidden = c.hidden; p.block_n = kTile; p.block_h = f.block_h; p.bias = c.bias; p.status = c.status;
  p.dx_sums = at<float>(ws, f.dx);
  p.want_x = c.dx != nullptr ? 1 : 0; p.want_w = c.dw != nullptr ? 1 : 0; p.accumulate = c.accumulate; p.n_tiles = ceil_div(c.hidden, f.block_h);
  p.dw = c.dw; p.dw_stride = c.dw_stride;
  if ((e = encode_matrix_map(&p.w_mn, c.w, c.vocab, c.hidden, c.w_stride * 2, 64, 64, false)) != cudaSuccess) return e;

  if (f.few) {
    VocabFewParams w;
    memset(&w, 0, sizeof(w));
    w.rows = c.rows; w.vocab = c.vocab; w.hidden = c.hidden; w.bias = c.bias; w.labels = c.labels; w.status = c.status;
    w.lse = c.lse; w.grad_loss = c.grad_loss; w.x = c.x; w.x_stride = c.x_stride; w.x_clean = c.dw != nullptr ? gathered : nullptr;
    w.g = g; w.g_pitch = f.g_pitch; w.db = c.db; w.accumulate = c.accumulate; w.row_residual = at<float>(ws, f.row_residual);
    w.counter = at<uint32_t>(ws, f.counters); w.two_terms = at<int32_t>(ws, f.two_terms);
    if ((e = few_maps(c, &w)) != cudaSuccess) return e;
    int ctas = 0;
    if ((e = launch_few<true>(w, sm_count, &ctas, stream)) != cudaSuccess || !products) return e;
    const int words = ceil_div(c.vocab, 128) * 128;
    // (two terms to a row: the product for dx sees the first only)
    if ((e = encode_matrix_map(&p.g_k[0], g, words, 2 * f.g_pitch, f.g_pitch * 4, kHalf, 64, false)) != cudaSuccess ||
        (e = encode_matrix_map(&p.g_mn[0], g, words, f.g_pitch, f.g_pitch * 4, 64, 64, false)) != cudaSuccess ||
        (e = encode_matrix_map(&p.x_mn[0], gathered, f.g_pitch, c.hidden, h_stride, 64, 64, false)) != cudaSuccess)
      return e;
    p.x_mn[1] = p.x_mn[0];
    p.x_k[0] = p.w_k = p.w_mn;      // (of kind 0, which has no tiles here)
    p.two_terms = w.two_terms; p.row_pitch = static_cast<int>(f.row_pitch); p.ranges = f.ranges; p.counter = w.counter;
    p.range_blocks = ceil_div(ceil_div(c.vocab, 64), f.ranges);
    const int tiles = p.n_tiles * (f.ranges + ceil_div(c.vocab, kTile));
    if ((e = launch_pairs<kProducts>(p, tiles, sm_count, stream)) != cudaSuccess || c.dx == nullptr) return e;
    return launch_kernel(vocab_finish_kernel, dim3(dx_ctas), dim3(kJoinThreads), 0, stream, d);
  }

  VocabRowsParams r;
  memset(&r, 0, sizeof(r));
  r.labels = c.labels; r.x = c.x; r.x_stride = c.x_stride; r.rows = c.rows; r.vocab = c.vocab; r.hidden = c.hidden;
  r.count = at<int32_t>(ws, f.count); r.row_of = at<int32_t>(ws, f.row_of); r.row_label = at<int32_t>(ws, f.row_label);
  r.row_shift = at<float2>(ws, f.row_shift); r.dx = c.dx; r.dx_stride = c.dx_stride;
  r.lse = c.lse; r.grad_loss = c.grad_loss; r.gathered = at<bf16>(ws, f.gathered);
  r.counters = at<uint32_t>(ws, f.counters); r.n_counters = f.pieces + 1; r.status = c.status;
  r.work = at<VocabWork>(ws, f.work); r.piece = f.piece; r.max_shift = f.max_shift; r.buffers = f.buffers; r.buffer_rows = static_cast<int>(f.row_pitch);
  r.dx_rows = static_cast<int>(f.dx_rows); r.block_h = f.block_h; r.want_x = c.dx != nullptr ? 1 : 0; r.want_w = c.dw != nullptr ? 1 : 0;
  int ctas = 0;
  launch_rows_setup(&r, &ctas);
  if ((e = launch_kernel(vocab_rows_kernel, dim3(ctas), dim3(kRowsThreads), 0, stream, r)) != cudaSuccess) return e;

  p.labels = r.row_label; p.row_shift = r.row_shift; p.row_residual = at<float>(ws, f.row_residual);
  p.bias_parts = c.db != nullptr ? at<float>(ws, f.bias_parts) : nullptr; p.bias_pitch = c.vocab;
  p.g = g; p.piece = f.piece;
  if ((e = encode_matrix_map(&p.x_k[0], c.x, c.rows, c.hidden, c.x_stride * 2, kHalf, 64, false)) != cudaSuccess ||
      (e = encode_matrix_map(&p.x_k[1], gathered, f.row_pitch, c.hidden, h_stride, kHalf, 64, false)) != cudaSuccess ||
      (e = encode_matrix_map(&p.x_mn[0], c.x, c.rows, c.hidden, c.x_stride * 2, 64, 64, false)) != cudaSuccess ||
      (e = encode_matrix_map(&p.x_mn[1], gathered, f.row_pitch, c.hidden, h_stride, 64, 64, false)) != cudaSuccess ||
      (e = encode_matrix_map(&p.w_k, c.w, c.vocab, c.hidden, c.w_stride * 2, kHalf, 64, false)) != cudaSuccess)
    return e;
  for (int k = 0; k <= f.max_shift; ++k) {
    const int64_t g_rows = f.buffers * f.row_pitch >> k, g_cols = static_cast<int64_t>(f.piece) << k;
    if ((e = encode_matrix_map(&p.g_k[k], g, g_rows, g_cols, g_cols * 2, kHalf, 64, false)) != cudaSuccess ||
        (e = encode_matrix_map(&p.g_mn[k], g, g_rows, g_cols, g_cols * 2, 64, 64, false)) != cudaSuccess)
      return e;
  }
  // (sized for all rows; with fewer, the pieces are wider and the last launches find nothing to do)
  for (int j = 0; j <= f.pieces && (j < f.pieces || products); ++j) {
    p.work = r.work + j;
    p.counter = r.counters + j;
    if ((e = launch_pairs<kGradient>(p, sm_count, sm_count, stream)) != cudaSuccess) return e;
  }
  if (c.dx == nullptr && c.db == nullptr) return cudaSuccess;
  d.row_of = r.row_of; d.labels = r.row_label; d.work = r.work; d.bias_parts = p.bias_parts; d.db_ctas = c.db != nullptr ? ceil_div(c.vocab, 32) : 0;
  return launch_kernel(vocab_finish_kernel, dim3(dx_ctas + d.db_ctas), dim3(kJoinThreads), 0, stream, d);
}

}  // namespace mt
