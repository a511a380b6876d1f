// Dropout whose mask is never stored:  y = residual + x * keep / (1 - p).
//
// Whether element (row, column) stays is decided by 16 bits of Philox4x32-10 (J. K. Salmon, M. A. Moraes, R. O. Dror, D. E. Shaw:
// "Parallel random numbers: as easy as 1, 2, 3", SC 2011), a block cipher of a counter: the key is the caller's seed, the counter is
// (column / 8, row, the caller's 64-bit number of the call).  The gradient is the same map of the incoming gradient, so that the
// backward pass makes the mask again instead of reading it.
//
// Why 16 bits and not 32: the kernel reads and writes 4 to 12 bytes per element, and at this card's bandwidth that leaves some twenty
// integer instructions for it; a block of ten rounds is about a hundred, for eight elements with 16 bits each and for four with 32.
// The probability is thereby a multiple of 2^-16 (0.1 becomes 0.100006); the factor is that of the probability used, so the
// expectation of y is exact.

#include "tc_ptx.cuh"

namespace mt {
namespace {

constexpr int kDropoutThreads = 256;
constexpr int64_t kDropoutMaxCtas = 1 << 24;   // (beyond, a CTA takes several)

__device__ __forceinline__ uint4 philox10(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u;
    const uint64_t b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
    c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
    c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
    c1 = static_cast<uint32_t>(b);
    c3 = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

template <bool VEC>
__device__ __forceinline__ void load_group(const bf16* p, int n, float (&f)[8]) {
  if (VEC) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? __bfloat162float(p[i]) : 0.f;
  }
}
template <bool VEC>
__device__ __forceinline__ void load_group(const float* p, int n, float (&f)[8]) {
  if (VEC) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? p[i] : 0.f;
  }
}
template <bool VEC>
__device__ __forceinline__ void store_group(bf16* p, int n, const float (&f)[8]) {
  if (VEC) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < n) p[i] = __float2bfloat16_rn(f[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void store_group(float* p, int n, const float (&f)[8]) {
  if (VEC) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < n) p[i] = f[i];
  }
}

// A thread per group of eight columns of a row (one block of the generator), and a CTA per 256 of them: as CTAs end and others begin, some
// load while others compute, and the accesses stay in the order of the memory.  (32768 x 1024, bf16 onto an fp32 residual: 50.1 us, 6.7
// TB/s; as a grid-stride loop of eight CTAs per SM 62.6, with two groups in flight 59.2, with four 65.9.)  y may be x or the residual: every
// element is read before it is written, by the thread that writes it.
template <typename X, typename Y, bool RESIDUAL, bool VEC>
__global__ void __launch_bounds__(kDropoutThreads) dropout_kernel(const __grid_constant__ DropoutParams p) {
  grid_dependency_wait();
  grid_launch_dependents();
  uint64_t counter = p.counter;
  if (p.counter_dev != nullptr) counter += *p.counter_dev;
  const uint32_t groups = static_cast<uint32_t>((p.cols + 7) / 8);
  const int64_t total = static_cast<int64_t>(p.rows) * groups;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kDropoutThreads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kDropoutThreads + threadIdx.x; i < total; i += step) {
    const uint32_t row = total >> 32 == 0 ? static_cast<uint32_t>(i) / groups : static_cast<uint32_t>(i / groups);
    const uint32_t group = static_cast<uint32_t>(i - static_cast<int64_t>(row) * groups);
    const int col = group * 8, left = p.cols - col;
    float f[8], r[8];
    load_group<VEC>(static_cast<const X*>(p.x) + row * p.x_stride + col, left, f);
    if (RESIDUAL) load_group<VEC>(static_cast<const Y*>(p.residual) + row * p.residual_stride + col, left, r);
    const uint4 bits = philox10(group, row, static_cast<uint32_t>(counter), static_cast<uint32_t>(counter >> 32),
                                static_cast<uint32_t>(p.seed), static_cast<uint32_t>(p.seed >> 32));
    const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t draw = (j & 1) ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu;
      // (a choice, not a product: what is dropped may be infinite or not a number)
      const float kept = draw >= p.threshold ? f[j] * p.factor : 0.f;
      f[j] = RESIDUAL ? r[j] + kept : kept;
    }
    store_group<VEC>(static_cast<Y*>(p.y) + row * p.y_stride + col, left, f);
  }
}

template <typename X, typename Y>
cudaError_t launch_types(const DropoutParams& p, cudaStream_t stream) {
  auto aligned = [](const void* q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
  const bool vec = p.cols % 8 == 0 && p.x_stride % 8 == 0 && p.y_stride % 8 == 0 && (p.residual == nullptr || p.residual_stride % 8 == 0) &&
                   aligned(p.x) && aligned(p.y) && aligned(p.residual);
  const int64_t groups = static_cast<int64_t>(p.rows) * ((p.cols + 7) / 8);
  const int64_t ctas = (groups + kDropoutThreads - 1) / kDropoutThreads;
  const int grid = static_cast<int>(ctas < kDropoutMaxCtas ? ctas : kDropoutMaxCtas);
  auto kernel = p.residual != nullptr ? (vec ? dropout_kernel<X, Y, true, true> : dropout_kernel<X, Y, true, false>)
                                      : (vec ? dropout_kernel<X, Y, false, true> : dropout_kernel<X, Y, false, false>);
  return launch_kernel(kernel, dim3(grid), dim3(kDropoutThreads), 0, stream, p);
}

}  // namespace

cudaError_t launch_dropout(const DropoutParams& p, bool x_f32, bool y_f32, cudaStream_t stream) {
  if (x_f32) return y_f32 ? launch_types<float, float>(p, stream) : launch_types<float, bf16>(p, stream);
  return y_f32 ? launch_types<bf16, float>(p, stream) : launch_types<bf16, bf16>(p, stream);
}

}  // namespace mt
