// Rows of a table by token id, and the gradient of the table.
//
//   lookup:    out[t, :]   = scale * table[id_t, :]
//   gradient:  d_table[v, :] (+)= scale * sum over t with id_t = v of d_out[t, :]
//
// Both move bytes and compute next to nothing.  The lookup is one pass: a warp per token, 16-byte accesses, up to four of them in
// flight per lane.  The gradient adds up rows in an order that depends on the ids alone, so that equal calls give equal bits: the
// tokens are sorted by id (stably), every run of equal ids is summed in order of the tokens in fp32, and rounded once.
//
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
constexpr int kSortMaxCluster = 8;
// counters of every warp, totals of this CTA (two passes in turn), first places of the digits, warp sums of a scan
constexpr int kSortSmemBytes = (kSortWarps * kSortBins + 2 * kSortBins + kSortBins + kSortWarps) * 4;
constexpr int kSumColumns = 8;                        // columns of a thread
constexpr int kSumUnroll = 8;                         // rows asked for at a time
constexpr int kJoinGroups = 8;                        // row groups of a CTA of the join, 32 threads each

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

constexpr int kLookupThreads = 256;
constexpr int kLookupUnroll = 4;

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

// Lanes of the warp that hold the same digit (of those in `active`).
__device__ __forceinline__ uint32_t same_digit(uint32_t active, uint32_t digit) { return __match_any_sync(active, digit); }

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
      for (int64_t i = static_cast<int64_t>(fill) * kSortThreads + tid; i < n; i += static_cast<int64_t>(n_fill) * kSortThreads)
        flat[i] = make_uint4(0, 0, 0, 0);
    } else {
      for (int v = fill * kSortWarps + warp; v < p.vocab; v += n_fill * kSortWarps)
        for (int c = lane; c < p.hidden; c += 32) table[static_cast<int64_t>(v) * p.table_stride + c] = O(0.f);
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
    const uint32_t* src_key = p.keys[(pass + 1) & 1];
    const uint32_t* src_token = p.order[(pass + 1) & 1];
    uint32_t* dst_key = p.keys[pass & 1];
    uint32_t* dst_token = p.order[pass & 1];
    auto key_at = [&](int i) -> uint32_t {
      if (pass != 0) return __ldcg(src_key + i);                   // (written by the other CTAs of the cluster: not through L1)
      const int id = p.ids[i];
      return id < 0 || id >= p.vocab || id == p.padding_id ? static_cast<uint32_t>(p.vocab) : static_cast<uint32_t>(id);
    };
    for (int b = lane; b < bins; b += 32) my_counts[b] = 0;
    __syncwarp();
    for (int i0 = begin; i0 < end; i0 += 32) {
      const int i = i0 + lane;
      const uint32_t active = __ballot_sync(0xffffffffu, i < end);
      if (i < end) {
        if (pass == 0 && p.status != nullptr && p.ids[i] >= p.vocab) atomicOr(p.status, kFlagBadToken);
        const uint32_t digit = (key_at(i) >> shift) & (bins - 1);
        const uint32_t same = same_digit(active, digit);
        if (lane == __ffs(same) - 1) my_counts[digit] += __popc(same);
      }
      __syncwarp();
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
    cluster_sync_all();
    if (tid < bins) {
      for (int r = 0; r < n_ctas; ++r) {
        const uint32_t c = ld_cluster_u32(map_to_cta(smem_u32(my_totals + tid), r));
        all += c;
        if (r < rank) before += c;
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
    for (int i0 = begin; i0 < end; i0 += 32) {
      const int i = i0 + lane;
      const uint32_t active = __ballot_sync(0xffffffffu, i < end);
      if (i < end) {
        const uint32_t key = key_at(i);
        const uint32_t token = pass == 0 ? static_cast<uint32_t>(i) : __ldcg(src_token + i);
        const uint32_t digit = (key >> shift) & (bins - 1);
        const uint32_t same = same_digit(active, digit);
        const uint32_t place = first[digit] + my_counts[digit] + __popc(same & ((1u << lane) - 1));
        __syncwarp(active);
        if (lane == __ffs(same) - 1) my_counts[digit] += __popc(same);
        dst_key[place] = key;
        dst_token[place] = token;
      }
      __syncwarp();
    }
    // the next pass reads what the other CTAs have written (and no CTA leaves while another reads its totals)
    __syncwarp();
    cluster_sync_all();
  }
}

// ---- sum -----------------------------------------------------------------------------------------

template <typename G, typename O, bool VEC>
__global__ void __launch_bounds__(128) embedding_grad_sum_kernel(const __grid_constant__ EmbeddingGradParams p) {
  __shared__ uint32_t s_key[kEmbeddingMaxChunk + 2];     // one before the chunk, the chunk, one behind it
  __shared__ uint32_t s_token[kEmbeddingMaxChunk];
  grid_dependency_wait();
  grid_launch_dependents();
  const int n = p.tokens, len = p.chunk;
  const int e0 = blockIdx.x * len;
  const int count = min(len, n - e0);
  const uint32_t* keys = p.keys[(p.passes - 1) & 1];
  const uint32_t* order = p.order[(p.passes - 1) & 1];
  constexpr uint32_t kNone = 0xffffffffu;                // (no id)
  for (int i = threadIdx.x; i < count + 2; i += blockDim.x) {
    const int e = e0 - 1 + i;
    s_key[i] = e < 0 || e >= n ? kNone : keys[e];
  }
  for (int i = threadIdx.x; i < count; i += blockDim.x) s_token[i] = order[e0 + i];
  __syncthreads();
  const int col = (blockIdx.y * blockDim.x + threadIdx.x) * kSumColumns;
  if (col >= p.hidden) return;
  const int left = p.hidden - col;
  const G* grad = static_cast<const G*>(p.grad_out) + col;
  float acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  bool began_here = s_key[0] != s_key[1];
  const uint32_t none = static_cast<uint32_t>(p.vocab);
  for (int i0 = 0; i0 < count && s_key[i0 + 1] != none; i0 += kSumUnroll) {
    float f[kSumUnroll][8];
#pragma unroll
    for (int u = 0; u < kSumUnroll; ++u) {
      const int i = i0 + u;
      if (i < count && s_key[i + 1] != none) load8<VEC>(grad + static_cast<int64_t>(s_token[i]) * p.grad_stride, left, f[u]);
    }
#pragma unroll
    for (int u = 0; u < kSumUnroll; ++u) {
      const int i = i0 + u;
      if (i >= count || s_key[i + 1] == none) break;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += f[u][j];
      const uint32_t key = s_key[i + 1];
      const bool ends = s_key[i + 2] != key;
      if (!ends && i + 1 < count) continue;
      if (began_here && ends) {
        O* out = static_cast<O*>(p.grad_table) + static_cast<int64_t>(key) * p.table_stride + col;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] *= p.scale;
        if (p.accumulate) add_present8<VEC>(out, left, acc);
        store8<VEC>(out, left, acc);
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

// A CTA per chunk (and 256 columns): if a run begins in this chunk and goes on behind it, adds up its parts.  Eight groups of threads
// take every eighth part each, then their sums are added in order.
template <typename O, bool VEC>
__global__ void __launch_bounds__(32 * kJoinGroups) embedding_grad_join_kernel(const __grid_constant__ EmbeddingGradParams p) {
  __shared__ float s_acc[kJoinGroups][32][9];
  grid_dependency_wait();
  grid_launch_dependents();
  const int n = p.tokens, len = p.chunk;
  const int e0 = blockIdx.x * len, e1 = e0 + len;
  if (e1 >= n) return;                                    // (the last chunk: nothing goes on behind it)
  const uint32_t* keys = p.keys[(p.passes - 1) & 1];
  const uint32_t key = keys[e1 - 1];
  if (key == static_cast<uint32_t>(p.vocab) || keys[e1] != key || (e0 > 0 && keys[e0 - 1] == key)) return;
  // chunks behind this one that the run reaches: those that begin with its id (the ids are sorted)
  int behind = 0;
  for (int64_t c0 = blockIdx.x + 1; ; c0 += blockDim.x) {
    const int64_t e = (c0 + threadIdx.x) * len;
    const int got = __syncthreads_count(e < n && keys[e] == key);
    behind += got;
    if (got < static_cast<int>(blockDim.x)) break;
  }
  const int group = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int col = (blockIdx.y * 32 + lane) * kSumColumns;
  float acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  if (col < p.hidden) {
    const float* parts = p.parts + static_cast<int64_t>(blockIdx.x) * 2 * p.part_stride + col;
#pragma unroll 4
    for (int i = group; i <= behind; i += kJoinGroups) {  // part 0: slot 1 of this chunk; part i: slot 0 of the i-th behind it
      float f[8];
      load8<true>(parts + (i == 0 ? p.part_stride : static_cast<int64_t>(i) * 2 * p.part_stride), 8, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += f[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) s_acc[group][lane][j] = acc[j];
  __syncthreads();
  if (group != 0 || col >= p.hidden) return;
  for (int g = 1; g < kJoinGroups; ++g) {
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += s_acc[g][lane][j];
  }
  O* out = static_cast<O*>(p.grad_table) + static_cast<int64_t>(key) * p.table_stride + col;
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] *= p.scale;
  if (p.accumulate) add_present8<VEC>(out, p.hidden - col, acc);
  store8<VEC>(out, p.hidden - col, acc);
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

template <typename T, typename O>
cudaError_t launch_lookup_types(const LookupParams& p, bool vec, int sm_count, cudaStream_t stream) {
  const int64_t ctas = (static_cast<int64_t>(p.tokens) + kLookupThreads / 32 - 1) / (kLookupThreads / 32);
  const int grid = static_cast<int>(ctas < 8 * sm_count ? ctas : 8 * sm_count);
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
                       dim3(chunks, (units + 31) / 32), dim3(32 * kJoinGroups), 0, stream, p);
}

template <typename O>
cudaError_t launch_sort(EmbeddingGradParams* p, int sm_count, cudaStream_t stream) {
  auto kernel = token_sort_kernel<O>;
  static PerDeviceOnce once;   // per instantiation
  cudaError_t err = per_device_once(once, [&](int) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortSmemBytes);
  });
  if (err != cudaSuccess) return err;
  // a CTA of the cluster per two rounds of all its warps, as far as eight of them
  int ctas = 1;
  while (ctas < kSortMaxCluster && static_cast<int64_t>(ctas) * 2 * kSortThreads < p->tokens) ctas *= 2;
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

cudaError_t launch_embedding_lookup(const LookupParams& p, bool table_f32, bool out_f32, int sm_count, cudaStream_t stream) {
  const bool vec = p.hidden % 8 == 0 && p.table_stride % 8 == 0 && p.out_stride % 8 == 0 && aligned16(p.table) && aligned16(p.out);
  if (table_f32) return out_f32 ? launch_lookup_types<float, float>(p, vec, sm_count, stream) : launch_lookup_types<float, bf16>(p, vec, sm_count, stream);
  return out_f32 ? launch_lookup_types<bf16, float>(p, vec, sm_count, stream) : launch_lookup_types<bf16, bf16>(p, vec, sm_count, stream);
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
  int bits = 1;                              // of the largest key, which is `vocab`
  while (bits < 31 && (p.vocab >> bits) != 0) ++bits;
  p.passes = (bits + kSortDigitBits - 1) / kSortDigitBits;
  p.digit_bits = (bits + p.passes - 1) / p.passes;
  cudaError_t e = out_f32 ? launch_sort<float>(&p, sm_count, stream) : launch_sort<bf16>(&p, sm_count, stream);
  if (e != cudaSuccess || p.tokens == 0) return e;
  if (grad_f32) return out_f32 ? launch_sum_join<float, float>(p, vec, stream) : launch_sum_join<float, bf16>(p, vec, stream);
  return out_f32 ? launch_sum_join<bf16, float>(p, vec, stream) : launch_sum_join<bf16, bf16>(p, vec, stream);
}

}  // namespace mt
