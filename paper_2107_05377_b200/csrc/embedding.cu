// Rows of a table by token id, and the gradient of the table.
//
//   lookup:    out[t, :]   = scale * table[id_t, :]
//   gradient:  d_table[v, :] (+)= scale * sum over t with id_t = v of d_out[t, :]
//
// Both move bytes and compute next to nothing.  The lookup is one pass: a warp per token, 16-byte accesses.  The gradient adds up rows in an order that depends on the ids alone, so that equal calls give equal bits: the
// tokens are sorted by id (stably), every run of equal ids is summed in order of the tokens in fp32, and rounded once.
//
// Up to 1024 tokens one launch does it all (embedding_grad_few_kernel).  More:
//   sort   one cluster sorts (id, token) by least significant digits; every step between its CTAs goes through distributed shared
//          memory, so that all passes are one launch.  The other CTAs of the launch write the zeros of the rows without a token
//          meanwhile (all rows: which ones have none is not known yet).
//   sum    a CTA per chunk of the sorted list, a thread per eight columns: runs that lie inside a chunk go straight to the table, what a
//          chunk has of a run that crosses its border goes to the workspace (a run of a sixteenth of all tokens - a mask token, a full
//          stop - is thereby spread over many CTAs)
//   join   the parts of each run that crosses a border, in order

#include "tc_ptx.cuh"

namespace mt {
namespace {

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortDigitBits = 9;                     // at most
constexpr int kSortBins = 1 << kSortDigitBits;
constexpr int kSortMaxCluster = 16;                   // (more than the portable eight)
constexpr int kSortUnroll = 8;                        // rounds of a warp whose entries are in registers at a time
constexpr int kSortAlone = 2048;                      // tokens that one CTA sorts alone, in shared memory
// counters of every warp, totals of this CTA (two passes in turn), first places of the digits, warp sums of a scan
constexpr int kSortCountBytes = (kSortWarps * kSortBins + 2 * kSortBins + kSortBins + kSortWarps) * 4;
constexpr int kSortSmemBytes = kSortCountBytes + kSortAlone * 8;
constexpr int kSumColumns = 8;                        // columns of a thread
constexpr int kSumUnroll = 8;                         // rows asked for at a time
constexpr int kJoinGroups = 8;                        // warps of a CTA of the join
constexpr int kFewTokens = 1024;                      // that one launch takes without a sort
constexpr int kFewRows = 64;                          // of the table, that a CTA marks at a time

// ---- eight consecutive elements ----------------------------------------------------------------
// VEC: both addresses are 16-byte aligned and all eight exist; otherwise n of them, one by one.
template <bool VEC>
__device__ __forceinline__ void load8(const bf16* p, int n, float (&f)[8]) {
  if (VEC) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? __bfloat162float(p[i]) : 0.f;
  }
}
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, int n, float (&f)[8]) {
  if (VEC) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? p[i] : 0.f;
  }
}
template <bool VEC>
__device__ __forceinline__ void store8(bf16* p, int n, const float (&f)[8]) {
  if (VEC) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < n) p[i] = __float2bfloat16_rn(f[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void store8(float* p, int n, const float (&f)[8]) {
  if (VEC) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < n) p[i] = f[i];
  }
}
// what is there now, read past the read-only cache (accumulation into the table)
template <bool VEC, typename T>
__device__ __forceinline__ void add_present8(const T* p, int n, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) if (VEC || i < n) f[i] += static_cast<float>(p[i]);
}

// ---- lookup --------------------------------------------------------------------------------------

constexpr int kLookupThreads = 128;
constexpr int kLookupUnroll = 2;
constexpr int64_t kLookupMaxCtas = 1 << 24;

template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(kLookupThreads) embedding_lookup_kernel(const __grid_constant__ LookupParams p) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int units = (p.hidden + 7) / 8;
  const int stride = gridDim.x * (kLookupThreads / 32);
  for (int t = blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5); t < p.tokens; t += stride) {
    const int id = p.ids[t];
    const bool there = id >= 0 && id < p.vocab;
    if (id >= p.vocab && lane == 0 && p.status != nullptr) atomicOr(p.status, kFlagBadToken);
    const T* row = static_cast<const T*>(p.table) + static_cast<int64_t>(there ? id : 0) * p.table_stride;
    O* out = static_cast<O*>(p.out) + static_cast<int64_t>(t) * p.out_stride;
    for (int u0 = lane; u0 < units; u0 += 32 * kLookupUnroll) {
      float f[kLookupUnroll][8];
#pragma unroll
      for (int i = 0; i < kLookupUnroll; ++i) {
        const int u = u0 + 32 * i;
        if (there && u < units) load8<VEC>(row + u * 8, p.hidden - u * 8, f[i]);
      }
#pragma unroll
      for (int i = 0; i < kLookupUnroll; ++i) {
        const int u = u0 + 32 * i;
        if (u >= units) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[i][j] = there ? f[i][j] * p.scale : 0.f;
        store8<VEC>(out + u * 8, p.hidden - u * 8, f[i]);
      }
    }
  }
}

// ---- sort ----------------------------------------------------------------------------------------

// Lanes of `active` that hold the same digit: one vote per bit.  (match.any takes some 240 clocks of the warp here.)
__device__ __forceinline__ uint32_t same_digit(uint32_t active, uint32_t digit, int bits) {
  uint32_t same = active;
#pragma unroll
  for (int b = 0; b < kSortDigitBits; ++b) {
    if (b < bits) {                                     // (all 32 lanes vote, converged: a vote of some of them costs a warp barrier)
      const bool one = (digit >> b) & 1u;
      const uint32_t ones = __ballot_sync(0xffffffffu, one);
      same &= one ? ones : ~ones;
    }
  }
  return same;
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t cluster_addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
  return v;
}

// One cluster (cluster 0 of the grid) sorts; the other CTAs write zeros to the table.  The list is cut into one piece per warp of the
// cluster, in order; a pass counts every warp's digits, adds the counts up over digits, CTAs and warps in this order, and puts every
// element behind the equal digits before it: stable, so that after the last pass equal ids are in order of their tokens.
// `vocab` stands for what is no token (or the row without a gradient): it sorts to the end.
template <typename O>
__global__ void __launch_bounds__(kSortThreads, 1) token_sort_kernel(const __grid_constant__ EmbeddingGradParams p) {
  extern __shared__ uint32_t sort_smem[];
  uint32_t* counts = sort_smem;                                    // [warp][digit]
  uint32_t* totals = counts + kSortWarps * kSortBins;              // [pass & 1][digit]
  uint32_t* first = totals + 2 * kSortBins;                        // [digit]
  uint32_t* warp_sums = first + kSortBins;                         // [warp]
  uint2* kept = reinterpret_cast<uint2*>(warp_sums + kSortWarps);  // the list, of one CTA alone
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_ctas = p.sort_ctas;
  grid_dependency_wait();
  grid_launch_dependents();

  if (static_cast<int>(blockIdx.x) >= n_ctas) {                    // (whole clusters: none of their CTAs enters the barriers below)
    O* table = static_cast<O*>(p.grad_table);
    const int fill = blockIdx.x - n_ctas, n_fill = gridDim.x - n_ctas;
    if (p.vectors && p.table_stride == p.hidden) {
      uint4* flat = reinterpret_cast<uint4*>(table);
      const int64_t n = static_cast<int64_t>(p.vocab) * p.hidden * sizeof(O) / 16;
#pragma unroll 4
      for (int64_t i = static_cast<int64_t>(fill) * kSortThreads + tid; i < n; i += static_cast<int64_t>(n_fill) * kSortThreads)
        flat[i] = make_uint4(0, 0, 0, 0);
    } else {
      // (in 64 bits: the last step of a table of nearly 2^31 rows goes beyond them)
      for (int64_t v = fill * kSortWarps + warp; v < p.vocab; v += n_fill * kSortWarps)
        for (int c = lane; c < p.hidden; c += 32) table[v * p.table_stride + c] = O(0.f);
    }
    return;
  }

  const int rank = blockIdx.x;
  const int n = p.tokens;
  const int pieces = n_ctas * kSortWarps;
  const int piece = ((n + pieces - 1) / pieces + 31) / 32 * 32;
  const int64_t begin64 = static_cast<int64_t>(rank * kSortWarps + warp) * piece;
  const int begin = begin64 < n ? static_cast<int>(begin64) : n;
  const int end = n - begin < piece ? n : begin + piece;
  const int bins = 1 << p.digit_bits;
  uint32_t* my_counts = counts + warp * kSortBins;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.digit_bits;
    // one CTA alone keeps the list in shared memory until the last pass
    const bool alone = n_ctas == 1;
    const uint2* src = p.list[(pass + 1) & 1];
    uint2* dst = alone && pass + 1 < p.passes ? kept : p.list[pass & 1];
    // (id, token) at place i of the list as it is before this pass
    auto entry = [&](int i) -> uint2 {
      if (pass != 0) return alone ? kept[i] : __ldcg(src + i);     // (written by the other CTAs of the cluster: not through L1)
      const int id = p.ids[i];
      return make_uint2(id < 0 || id >= p.vocab || id == p.padding_id ? static_cast<uint32_t>(p.vocab) : static_cast<uint32_t>(id),
                        static_cast<uint32_t>(i));
    };
    for (int b = lane; b < bins; b += 32) my_counts[b] = 0;
    __syncwarp();
    // up to 32 * kSortUnroll entries of a warp stay in registers from the count to their places
    uint2 e[kSortUnroll];
    auto fetch = [&](int i0) {
#pragma unroll
      for (int u = 0; u < kSortUnroll; ++u) {
        const int i = i0 + 32 * u + lane;
        e[u] = i < end ? entry(i) : make_uint2(0, 0);
      }
    };
    for (int i0 = begin; i0 < end; i0 += 32 * kSortUnroll) {
      fetch(i0);
#pragma unroll
      for (int u = 0; u < kSortUnroll; ++u) {
        const int i = i0 + 32 * u + lane;
        if (i >= end) continue;
        if (pass == 0 && p.status != nullptr && p.ids[i] >= p.vocab) atomicOr(p.status, kFlagBadToken);
        atomicAdd(&my_counts[(e[u].x >> shift) & (bins - 1)], 1u);   // (of this warp: whole numbers, any order)
      }
    }
    __syncthreads();
    // counts -> places before this warp's among the CTA's; totals of the CTA
    uint32_t* my_totals = totals + (pass & 1) * kSortBins;
    uint32_t total = 0, before = 0, all = 0;
    if (tid < bins) {
#pragma unroll
      for (int w0 = 0; w0 < kSortWarps; w0 += 8) {
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = counts[(w0 + j) * kSortBins + tid];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          counts[(w0 + j) * kSortBins + tid] = total;
          total += c[j];
        }
      }
      my_totals[tid] = total;
    }
    __syncwarp();
    if (alone) all = total; else cluster_sync_all();
    if (tid < bins && !alone) {
      uint32_t c[kSortMaxCluster];                    // (all asked for before the first is used)
#pragma unroll
      for (int r = 0; r < kSortMaxCluster; ++r) c[r] = r < n_ctas ? ld_cluster_u32(map_to_cta(smem_u32(my_totals + tid), r)) : 0u;
#pragma unroll
      for (int r = 0; r < kSortMaxCluster; ++r) {
        all += c[r];
        if (r < rank) before += c[r];
      }
    }
    // places of the digits before this one, over the whole list
    uint32_t scan = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t other = __shfl_up_sync(0xffffffffu, scan, o);
      if (lane >= o) scan += other;
    }
    if (lane == 31) warp_sums[warp] = scan;
    __syncthreads();
    if (tid < bins) {
      uint32_t lower = 0;
      for (int w = 0; w < warp; ++w) lower += warp_sums[w];
      first[tid] = lower + scan - all + before;
    }
    __syncthreads();
    for (int i0 = begin; i0 < end; i0 += 32 * kSortUnroll) {
      if (end - begin > 32 * kSortUnroll) fetch(i0);
#pragma unroll
      for (int u = 0; u < kSortUnroll; ++u) {
        if (i0 + 32 * u >= end) break;                    // (the same for all lanes)
        const bool there = i0 + 32 * u + lane < end;
        const uint32_t digit = (e[u].x >> shift) & (bins - 1);
        const uint32_t same = same_digit(__ballot_sync(0xffffffffu, there), digit, p.digit_bits);
        const uint32_t place = first[digit] + my_counts[digit] + __popc(same & ((1u << lane) - 1));
        __syncwarp();
        if (there && lane == __ffs(same) - 1) my_counts[digit] += __popc(same);
        if (there) dst[place] = e[u];
        __syncwarp();
      }
    }
    // the next pass reads what the other CTAs have written (and no CTA leaves while another reads its totals)
    __syncwarp();
    if (alone) __syncthreads(); else cluster_sync_all();
  }
}

// ---- sum -----------------------------------------------------------------------------------------

// Eight columns of a row as they lie in memory.
template <typename T> struct Raw;
template <> struct Raw<bf16> { uint4 a; };
template <> struct Raw<float> { uint4 a, b; };
template <bool VEC>
__device__ __forceinline__ void load_raw(const bf16* p, int n, Raw<bf16>& r) {
  if (VEC) {
    r.a = __ldg(reinterpret_cast<const uint4*>(p));
  } else {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = i < n ? __bfloat16_as_ushort(p[i]) : 0u;
    r.a = make_uint4(w[0] | (w[1] << 16), w[2] | (w[3] << 16), w[4] | (w[5] << 16), w[6] | (w[7] << 16));
  }
}
template <bool VEC>
__device__ __forceinline__ void load_raw(const float* p, int n, Raw<float>& r) {
  if (VEC) {
    r.a = __ldg(reinterpret_cast<const uint4*>(p));
    r.b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
  } else {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = i < n ? __float_as_uint(p[i]) : 0u;
    r.a = make_uint4(w[0], w[1], w[2], w[3]);
    r.b = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
__device__ __forceinline__ void add_raw(const Raw<bf16>& r, float (&f)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] += bf16_lo(w[i]); f[2 * i + 1] += bf16_hi(w[i]); }
}
__device__ __forceinline__ void add_raw(const Raw<float>& r, float (&f)[8]) {
  const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] += __uint_as_float(w[i]);
}

// scale * sum (+ what is there) to eight columns of the table's gradient.
template <bool VEC, typename O>
__device__ __forceinline__ void finish8(const EmbeddingGradParams& p, int64_t row, int col, float (&acc)[8]) {
  O* out = static_cast<O*>(p.grad_table) + row * p.table_stride + col;
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] *= p.scale;
  if (p.accumulate) add_present8<VEC>(out, p.hidden - col, acc);
  store8<VEC>(out, p.hidden - col, acc);
}

template <typename G, typename O, bool VEC>
__global__ void __launch_bounds__(128) embedding_grad_sum_kernel(const __grid_constant__ EmbeddingGradParams p) {
  __shared__ uint32_t s_key[kEmbeddingMaxChunk + 2];     // one before the chunk, the chunk, one behind it
  __shared__ uint32_t s_token[kEmbeddingMaxChunk];
  __shared__ int s_count;
  grid_dependency_wait();
  grid_launch_dependents();
  const int n = p.tokens, len = p.chunk;
  const int e0 = blockIdx.x * len;
  const int listed = min(len, n - e0);
  const uint2* list = p.list[(p.passes - 1) & 1];
  constexpr uint32_t kNone = 0xffffffffu;                // (no id)
  const uint32_t none = static_cast<uint32_t>(p.vocab);  // (tokens without a part, at the end of the list)
  if (threadIdx.x == 0) s_count = 0;
  __syncthreads();
  int mine = 0;
  for (int i = threadIdx.x; i < listed + 2; i += blockDim.x) {
    const int e = e0 - 1 + i;
    const uint2 at = e < 0 || e >= n ? make_uint2(kNone, 0) : list[e];
    s_key[i] = at.x;
    if (i >= 1 && i <= listed) {
      s_token[i - 1] = at.y;
      mine += at.x != none ? 1 : 0;
    }
  }
  if (mine != 0) atomicAdd(&s_count, mine);
  __syncthreads();
  const int count = s_count;
  const int col = (blockIdx.y * blockDim.x + threadIdx.x) * kSumColumns;
  if (col >= p.hidden || count == 0) return;
  const int left = p.hidden - col;
  const G* grad = static_cast<const G*>(p.grad_out) + col;
  float acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  bool began_here = s_key[0] != s_key[1];
  for (int i0 = 0; i0 < count; i0 += kSumUnroll) {
    Raw<G> row[kSumUnroll];
#pragma unroll
    for (int u = 0; u < kSumUnroll; ++u) {
      // (behind the last one: it once more, unused)
      const int i = min(i0 + u, count - 1);
      load_raw<VEC>(grad + static_cast<int64_t>(s_token[i]) * p.grad_stride, left, row[u]);
    }
#pragma unroll
    for (int u = 0; u < kSumUnroll; ++u) {
      const int i = i0 + u;
      if (i >= count) break;
      add_raw(row[u], acc);
      const uint32_t key = s_key[i + 1];
      const bool ends = s_key[i + 2] != key;
      if (!ends && i + 1 < count) continue;
      if (began_here && ends) {
        finish8<VEC, O>(p, key, col, acc);
      } else {
        // (slot 0: of a run that began before this chunk; slot 1: of one that begins here and goes on)
        float* part = p.parts + (static_cast<int64_t>(blockIdx.x) * 2 + (began_here ? 1 : 0)) * p.part_stride + col;
        store8<true>(part, 8, acc);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = 0.f;
      began_here = true;
    }
  }
}

// The parts of every run that crosses a border, in order.  A warp per chunk looks whether a run begins there and goes on behind it, and
// how far (the chunks' first ids are sorted: 32 of them are tried at a time).  Of few parts the warp takes the sum alone; of more, the
// CTA's eight warps take every eighth part each, and their sums are added in order.  256 columns to a CTA.
template <typename O, bool VEC>
__global__ void __launch_bounds__(32 * kJoinGroups) embedding_grad_join_kernel(const __grid_constant__ EmbeddingGradParams p) {
  __shared__ float s_acc[kJoinGroups][32][9];
  __shared__ int s_behind[kJoinGroups];
  __shared__ uint32_t s_key[kJoinGroups];
  grid_dependency_wait();
  grid_launch_dependents();
  const int n = p.tokens, len = p.chunk;
  const int chunks = (n + len - 1) / len;
  const uint2* list = p.list[(p.passes - 1) & 1];
  const int group = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunk = blockIdx.x * kJoinGroups + group;
  const int64_t e0 = static_cast<int64_t>(chunk) * len, e1 = e0 + len;
  int behind = 0;                                         // chunks behind this one that the run reaches
  uint32_t key = 0;
  if (e1 < n) {                                           // (behind the last chunk nothing goes on)
    // lane 0: the entry before the chunk; 1: its last; 2 and on: the first of each of the next thirty
    const int64_t at = lane == 0 ? e0 - 1 : (lane == 1 ? e1 - 1 : e1 + static_cast<int64_t>(lane - 2) * len);
    const uint32_t seen = at >= 0 && at < n ? list[at].x : 0xffffffffu;
    key = __shfl_sync(0xffffffffu, seen, 1);
    const uint32_t same = __ballot_sync(0xffffffffu, seen == key);
    if (key != static_cast<uint32_t>(p.vocab) && (same & 1u) == 0) {
      behind = __popc(same >> 2);
      if (behind == 30) {
        // chunks [low, high) behind: the first id of low - 1 is the run's, that of high is not (or there is none)
        int low = chunk + 31, high = chunks;
        while (low < high) {
          const int step = (high - low + 31) / 32;
          const int64_t c = low + static_cast<int64_t>(lane) * step;
          const uint32_t hits = __ballot_sync(0xffffffffu, c < high && list[c * len].x == key);
          const int n_hits = __popc(hits);
          if (n_hits < 32 && low + static_cast<int64_t>(n_hits) * step < high) high = low + n_hits * step;
          if (n_hits > 0) low += (n_hits - 1) * step + 1;
        }
        behind = low - 1 - chunk;
      }
    }
  }
  if (lane == 0) {
    s_behind[group] = behind;
    s_key[group] = key;
  }
  const int col = (blockIdx.y * 32 + lane) * kSumColumns;
  const bool in_row = col < p.hidden;
  float acc[8];
  // part 0: slot 1 of the chunk; part i: slot 0 of the i-th behind it
  auto add_part = [&](int c, int i) {
    float f[8];
    load8<true>(p.parts + (static_cast<int64_t>(c + i) * 2 + (i == 0 ? 1 : 0)) * p.part_stride + col, 8, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += f[j];
  };
  if (behind > 0 && behind < 2 * kJoinGroups && in_row) {
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
#pragma unroll 8
    for (int i = 0; i <= behind; ++i) add_part(chunk, i);
    finish8<VEC, O>(p, key, col, acc);
  }
  __syncthreads();
  for (int g = 0; g < kJoinGroups; ++g) {
    const int far = s_behind[g];
    if (far < 2 * kJoinGroups) continue;                  // (the same for all threads)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    if (in_row) {
#pragma unroll 8
      for (int i = group; i <= far; i += kJoinGroups) add_part(blockIdx.x * kJoinGroups + g, i);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) s_acc[group][lane][j] = acc[j];
    __syncthreads();
    if (group == 0 && in_row) {
      for (int w = 1; w < kJoinGroups; ++w) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += s_acc[w][lane][j];
      }
      finish8<VEC, O>(p, s_key[g], col, acc);
    }
    __syncthreads();
  }
}

// ---- few tokens ------------------------------------------------------------------------------------

// Up to kFewTokens tokens in one launch, without a sort: every CTA keeps all ids in shared memory.  CTA t < tokens lists the tokens that have
// token t's id, in order.  The rows of k tokens are summed by the CTAs of the first of them, as many as there are blocks of 256 columns:
// each takes its share of the blocks, a block by an equal number of its eight warps, of which each takes its share of the tokens; what the
// warps of a block have is added in order.  (1000 tokens of 768, bf16: one id 55 -> 19 us, an eighth of them a mask token 10.2 -> 5.9, against one
// CTA per id.)  A token whose id no other has takes a warp per block.  The CTAs behind write the zeros of the rows that no id names, a range of rows each.
template <typename G, typename O, bool VEC>
__global__ void __launch_bounds__(32 * kJoinGroups) embedding_grad_few_kernel(const __grid_constant__ EmbeddingGradParams p) {
  constexpr int THREADS = 32 * kJoinGroups, PER = kFewTokens / THREADS;
  constexpr int UNROLL = sizeof(G) == 4 ? 4 : 8;        // rows asked for at a time
  static_assert(kFewTokens % THREADS == 0, "every thread looks at the same number of ids");
  __shared__ int s_id[kFewTokens];
  __shared__ int s_list[kFewTokens];
  __shared__ int s_warp[kJoinGroups];
  __shared__ uint32_t s_named[kFewRows / 32];
  __shared__ float s_acc[kJoinGroups][8][32];
  __shared__ int s_helper;                              // how many tokens of the id come before this one
  grid_dependency_wait();
  grid_launch_dependents();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n = p.tokens;
  for (int i = tid; i < kFewTokens; i += THREADS) {
    const int id = i < n ? p.ids[i] : -1;
    if (blockIdx.x == 0 && id >= p.vocab && p.status != nullptr) atomicOr(p.status, kFlagBadToken);
    s_id[i] = id < 0 || id >= p.vocab || id == p.padding_id ? -1 : id;
  }
  __syncthreads();
  if (static_cast<int>(blockIdx.x) >= n) {
    // zeros: kFewRows rows at a time, those that are named marked first
    O* table = static_cast<O*>(p.grad_table);
    const int fill = blockIdx.x - n, n_fill = gridDim.x - n;
    for (int64_t v0 = static_cast<int64_t>(fill) * kFewRows; v0 < p.vocab; v0 += static_cast<int64_t>(n_fill) * kFewRows) {
      for (int i = tid; i < kFewRows / 32; i += THREADS) s_named[i] = 0;
      __syncthreads();
      for (int i = tid; i < n; i += THREADS) {
        const int64_t at = s_id[i] - v0;
        if (s_id[i] >= 0 && at >= 0 && at < kFewRows) atomicOr(&s_named[at >> 5], 1u << (at & 31));
      }
      __syncthreads();
      for (int r = warp; r < kFewRows && v0 + r < p.vocab; r += kJoinGroups) {
        if ((s_named[r >> 5] >> (r & 31)) & 1u) continue;
        O* row = table + (v0 + r) * p.table_stride;
        if (VEC) {
          for (int c = lane; c < p.hidden * static_cast<int>(sizeof(O)) / 16; c += 32) reinterpret_cast<uint4*>(row)[c] = make_uint4(0, 0, 0, 0);
        } else {
          for (int c = lane; c < p.hidden; c += 32) row[c] = O(0.f);
        }
      }
      __syncthreads();
    }
    return;
  }
  const int token = blockIdx.x;
  const int id = s_id[token];
  if (id < 0) return;
  // ids [tid * PER, ...): how many are this one
  int hits = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) hits += s_id[tid * PER + k] == id ? 1 : 0;
  const G* grad = static_cast<const G*>(p.grad_out);
  const int blocks = (p.hidden + 255) / 256;
  float acc[8];
  if (!__syncthreads_or(hits - (token / PER == tid ? 1 : 0))) {          // the only one: a warp per block
    for (int b = warp; b < blocks; b += kJoinGroups) {
      const int col = b * 256 + lane * 8;
      if (col >= p.hidden) continue;
      Raw<G> r;
      load_raw<VEC>(grad + token * p.grad_stride + col, p.hidden - col, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = 0.f;
      add_raw(r, acc);
      finish8<VEC, O>(p, id, col, acc);
    }
    return;
  }
  int places = hits;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int other = __shfl_up_sync(0xffffffffu, places, o);
    if (lane >= o) places += other;
  }
  if (lane == 31) s_warp[warp] = places;
  __syncthreads();
  int count = 0;
  places -= hits;
  for (int w = 0; w < kJoinGroups; ++w) {
    if (w < warp) places += s_warp[w];
    count += s_warp[w];
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = tid * PER + k;
    if (s_id[i] == id) {
      if (i == token) s_helper = places;
      s_list[places++] = i;
    }
  }
  __syncthreads();
  const int helper = s_helper, helpers = min(count, blocks);
  if (helper >= helpers) return;
  // blocks helper, helper + helpers, ...: up to eight of them at a time
  const int mine = (blocks - helper + helpers - 1) / helpers;
  int at_a_time = 1;
  while (at_a_time < mine && at_a_time < kJoinGroups) at_a_time *= 2;
  const int share = kJoinGroups / at_a_time, part = warp % share;
  for (int b0 = 0; b0 < mine; b0 += at_a_time) {
    const int block = b0 + warp / share;
    const int col = (helper + block * helpers) * 256 + lane * 8;
    const bool in_row = block < mine && col < p.hidden;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    if (in_row) {
      for (int i = part; i < count; i += share * UNROLL) {
        Raw<G> r[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
          if (i + u * share < count) load_raw<VEC>(grad + s_list[i + u * share] * p.grad_stride + col, p.hidden - col, r[u]);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
          if (i + u * share < count) add_raw(r[u], acc);
      }
    }
    const int parts = min(share, count);
    if (parts > 1) {                                      // (the same for all threads)
#pragma unroll
      for (int j = 0; j < 8; ++j) s_acc[warp][j][lane] = acc[j];
      __syncthreads();
      if (part == 0) {
        for (int w = 1; w < parts; ++w) {
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] += s_acc[warp + w][j][lane];
        }
      }
      __syncthreads();
    }
    if (part == 0 && in_row) finish8<VEC, O>(p, id, col, acc);
  }
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

template <typename T, typename O>
cudaError_t launch_lookup_types(const LookupParams& p, bool vec, cudaStream_t stream) {
  // A warp per row and no loop over rows: 130304 rows of 1024 from an fp32 table onto bf16 58.5 us; eight CTAs per SM that loop 65.6.
  const int64_t ctas = (static_cast<int64_t>(p.tokens) + kLookupThreads / 32 - 1) / (kLookupThreads / 32);
  const int grid = static_cast<int>(ctas < kLookupMaxCtas ? ctas : kLookupMaxCtas);
  return launch_kernel(vec ? embedding_lookup_kernel<T, O, true> : embedding_lookup_kernel<T, O, false>, dim3(grid), dim3(kLookupThreads), 0, stream, p);
}

template <typename G, typename O>
cudaError_t launch_sum_join(const EmbeddingGradParams& p, bool vec, cudaStream_t stream) {
  const int chunks = (p.tokens + p.chunk - 1) / p.chunk;
  const int units = (p.hidden + 7) / 8;
  const int threads = units >= 128 ? 128 : (units + 31) / 32 * 32;
  cudaError_t e = launch_kernel(vec ? embedding_grad_sum_kernel<G, O, true> : embedding_grad_sum_kernel<G, O, false>,
                                dim3(chunks, (units + threads - 1) / threads), dim3(threads), 0, stream, p);
  if (e != cudaSuccess || chunks < 2) return e;
  return launch_kernel(vec ? embedding_grad_join_kernel<O, true> : embedding_grad_join_kernel<O, false>,
                       dim3((chunks + kJoinGroups - 1) / kJoinGroups, (units + 31) / 32), dim3(32 * kJoinGroups), 0, stream, p);
}

template <typename G, typename O>
cudaError_t launch_few(const EmbeddingGradParams& p, bool vec, int sm_count, cudaStream_t stream) {
  int64_t fill = 0;
  if (!p.accumulate) fill = (static_cast<int64_t>(p.vocab) + kFewRows - 1) / kFewRows;
  if (fill > 4 * sm_count) fill = 4 * sm_count;
  if (p.tokens + fill == 0) return cudaSuccess;
  return launch_kernel(vec ? embedding_grad_few_kernel<G, O, true> : embedding_grad_few_kernel<G, O, false>,
                       dim3(static_cast<unsigned>(p.tokens + fill)), dim3(32 * kJoinGroups), 0, stream, p);
}

template <typename O>
cudaError_t launch_sort(EmbeddingGradParams* p, int sm_count, cudaStream_t stream) {
  auto kernel = token_sort_kernel<O>;
  static PerDeviceOnce once;   // per instantiation
  static int most_ctas[kMaxDevices];
  int device = 0;
  cudaError_t err = per_device_once(once, [&](int dev) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortSmemBytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kSortMaxCluster);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = kSortSmemBytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kSortMaxCluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
    most_ctas[dev] = e == cudaSuccess && clusters > 0 ? kSortMaxCluster : 8;
    if (e != cudaSuccess) (void)cudaGetLastError();
    return cudaSuccess;
  }, &device);
  if (err != cudaSuccess) return err;
  // Up to 2048 tokens one CTA: no trip between CTAs nor to L2 between the passes (2048 tokens 10 us against 12 with two CTAs; 4096 14 against
  // 12).  Beyond, a CTA of the cluster per round of all its warps, as far as sixteen of them (where so many fit; else eight): what a pass
  // costs then is the issue of the votes and of stores to 32 places per warp.  131072 tokens: 76 us with match.any, ids and tokens stored
  // apart and eight CTAs; 57 with votes; 26 with one store for both, sixteen CTAs, entries kept in registers and all lanes voting.
  int ctas = 1;
  while (p->tokens > kSortAlone && ctas < most_ctas[device] && static_cast<int64_t>(ctas) * kSortThreads < p->tokens) ctas *= 2;
  p->sort_ctas = ctas;
  int fill = 0;
  if (!p->accumulate) {
    // zeros: of the SMs that the sort leaves, as many as have 64 KB each to write
    const int64_t bytes = static_cast<int64_t>(p->vocab) * p->hidden * sizeof(O);
    const int64_t wanted = (bytes + 65535) / 65536;
    const int64_t most = sm_count > 2 * ctas ? sm_count - 2 * ctas : 1;
    fill = static_cast<int>((wanted < most ? wanted : most) + ctas - 1) / ctas * ctas;
  }
  return launch_kernel(kernel, dim3(ctas + fill), dim3(kSortThreads), kSortSmemBytes, stream, *p, static_cast<unsigned>(ctas));
}

}  // namespace

cudaError_t launch_embedding_lookup(const LookupParams& p, bool table_f32, bool out_f32, cudaStream_t stream) {
  const bool vec = p.hidden % 8 == 0 && p.table_stride % 8 == 0 && p.out_stride % 8 == 0 && aligned16(p.table) && aligned16(p.out);
  if (table_f32) return out_f32 ? launch_lookup_types<float, float>(p, vec, stream) : launch_lookup_types<float, bf16>(p, vec, stream);
  return out_f32 ? launch_lookup_types<bf16, float>(p, vec, stream) : launch_lookup_types<bf16, bf16>(p, vec, stream);
}

// Entries of a chunk: at least one round of loads; more where the list is long, so that 16 CTAs for each of 148 SMs have one chunk
// each (up to what a CTA keeps of the list in shared memory).
int embedding_grad_chunk(int tokens) {
  const int64_t most = 16 * 148;
  int64_t len = ((static_cast<int64_t>(tokens) + most - 1) / most + kSumUnroll - 1) / kSumUnroll * kSumUnroll;
  if (len < kSumUnroll) len = kSumUnroll;
  return static_cast<int>(len < kEmbeddingMaxChunk ? len : kEmbeddingMaxChunk);
}

cudaError_t launch_embedding_grad(EmbeddingGradParams p, bool grad_f32, bool out_f32, int sm_count, cudaStream_t stream) {
  const bool vec = p.hidden % 8 == 0 && p.table_stride % 8 == 0 && p.grad_stride % 8 == 0 && aligned16(p.grad_out) && aligned16(p.grad_table);
  p.vectors = vec ? 1 : 0;
  if (p.tokens <= kFewTokens) {
    if (grad_f32) return out_f32 ? launch_few<float, float>(p, vec, sm_count, stream) : launch_few<float, bf16>(p, vec, sm_count, stream);
    return out_f32 ? launch_few<bf16, float>(p, vec, sm_count, stream) : launch_few<bf16, bf16>(p, vec, sm_count, stream);
  }
  int bits = 1;                              // of the largest key, which is `vocab`
  while (bits < 31 && (p.vocab >> bits) != 0) ++bits;
  p.passes = (bits + kSortDigitBits - 1) / kSortDigitBits;
  p.digit_bits = (bits + p.passes - 1) / p.passes;
  cudaError_t e = out_f32 ? launch_sort<float>(&p, sm_count, stream) : launch_sort<bf16>(&p, sm_count, stream);
  if (e != cudaSuccess) return e;
  if (grad_f32) return out_f32 ? launch_sum_join<float, float>(p, vec, stream) : launch_sum_join<float, bf16>(p, vec, stream);
  return out_f32 ? launch_sum_join<bf16, float>(p, vec, stream) : launch_sum_join<bf16, bf16>(p, vec, stream);
}

}  // namespace mt
