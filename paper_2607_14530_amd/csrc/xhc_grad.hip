// Global norm of many gradient tensors, and their clip by it.
//
//   norm = sqrt(sum_i sum_e g_i[e]^2),  c = min(1, max_norm / (norm + 1e-6)),  out_i = c g_i
//
// Bound by HBM: every element is read once for the norm, and read and written
// once for the clip.  Squares and sums are fp64: exact for bf16 and to 2^-53
// for fp32, no overflow or underflow at any fp32 value, at a few of the
// operations that the bytes leave time for.  The tensors are cut into chunks,
// one workgroup each; a workgroup finds its tensor by a search in a table that
// the launch carries in its arguments, so that nothing is copied to the device
// and a captured launch keeps its table.  The chunks' sums are added in a fixed
// order: the norm does not depend on timing.
#include <math.h>

#include "xhc_device.h"
#include "xhc_grad_launches.h"

namespace xhc {

namespace {

constexpr int kGradThreads = 256;
constexpr int kGradVecs = 8;         // vectors of 8 elements that a thread has on the way

struct GradChunk {
  int i;
  int64_t at, n;   // elements before it in its tensor, and its own
  bool f32;
};
__device__ __forceinline__ GradChunk find_chunk(const GradBatch& b, int block) {
  int lo = 0, hi = b.n;             // first[lo] <= block < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (b.first[mid] <= block) lo = mid; else hi = mid;
  }
  GradChunk c;
  c.i = lo;
  c.at = (int64_t)(block - b.first[lo]) * b.chunk;
  const int64_t left = b.count[lo] - c.at;
  c.n = left < b.chunk ? left : b.chunk;
  c.f32 = (b.f32[lo / 64] >> (lo % 64)) & 1;
  return c;
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}
template <int THREADS>
__device__ __forceinline__ double block_sum_f64(double v, double* red) {
  v = wave_sum_f64(v);
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  double s = red[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) s += red[w];
  return s;
}

template <typename TS> __device__ __forceinline__ float elem(const TS* p, int64_t i);
template <> __device__ __forceinline__ float elem<uint16_t>(const uint16_t* p, int64_t i) {
  return __uint_as_float((uint32_t)p[i] << 16);
}
template <> __device__ __forceinline__ float elem<float>(const float* p, int64_t i) { return p[i]; }

__device__ __forceinline__ bool aligned16_dev(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <typename TS>
__device__ __forceinline__ double chunk_squares(const TS* __restrict__ p, int64_t n) {
  using R8 = Raw8<TS>;
  double s[4] = {0., 0., 0., 0.};
  int64_t i = 0;
  if (aligned16_dev(p)) {
    const int64_t n8 = n / 8;
    for (int64_t b = threadIdx.x; b < n8; b += kGradVecs * kGradThreads) {
      typename R8::raw r[kGradVecs];
#pragma unroll
      for (int u = 0; u < kGradVecs; ++u)
        if (b + u * kGradThreads < n8) r[u] = R8::load(p + (b + u * kGradThreads) * 8);
#pragma unroll
      for (int u = 0; u < kGradVecs; ++u)
        if (b + u * kGradThreads < n8) {
          float f[8];
          R8::unpack(r[u], f);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[e % 4] = fma((double)f[e], (double)f[e], s[e % 4]);
        }
    }
    i = n8 * 8;
  }
  for (int64_t b = i + threadIdx.x; b < n; b += 8 * kGradThreads) {
    float f[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) f[u] = b + u * kGradThreads < n ? elem<TS>(p, b + u * kGradThreads) : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) s[u % 4] = fma((double)f[u], (double)f[u], s[u % 4]);
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

__global__ __launch_bounds__(kGradThreads) void k_grad_squares(const GradBatch b, double* __restrict__ part) {
  __shared__ double red[kGradThreads / 64];
  const GradChunk c = find_chunk(b, (int)blockIdx.x);
  const double s = c.f32 ? chunk_squares(reinterpret_cast<const float*>(b.src[c.i]) + c.at, c.n)
                         : chunk_squares(reinterpret_cast<const uint16_t*>(b.src[c.i]) + c.at, c.n);
  const double t = block_sum_f64<kGradThreads>(s, red);
  if (threadIdx.x == 0) part[b.part_at + blockIdx.x] = t;
}

// c of the reported (fp32) norm; 1 where that is not finite, so that the
// gradients are left as they are
__device__ __forceinline__ float clip_factor(double norm, float max_norm) {
  const float n32 = (float)norm;
  if (!(n32 <= 3.402823466e38f)) return 1.0f;
  const double c = (double)max_norm / (norm + 1e-6);
  return c < 1.0 ? (float)c : 1.0f;
}

constexpr int kNormThreads = 1024;
__global__ __launch_bounds__(kNormThreads) void k_grad_norm(const double* __restrict__ part, int64_t chunks,
                                                            float max_norm, float* __restrict__ norm,
                                                            float* __restrict__ factor) {
  __shared__ double red[kNormThreads / 64];
  double p[4] = {0., 0., 0., 0.};
  for (int64_t i = threadIdx.x; i < chunks; i += 4 * kNormThreads)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u * kNormThreads < chunks) p[u] += part[i + u * kNormThreads];
  double s = (p[0] + p[1]) + (p[2] + p[3]);
  s = sqrt(block_sum_f64<kNormThreads>(s, red));
  if (threadIdx.x == 0) {
    *norm = (float)s;
    if (factor) *factor = clip_factor(s, max_norm);
  }
}

template <typename TS> __device__ __forceinline__ void put(TS* p, int64_t i, float v);
template <> __device__ __forceinline__ void put<uint16_t>(uint16_t* p, int64_t i, float v) { p[i] = (uint16_t)f2bf(v); }
template <> __device__ __forceinline__ void put<float>(float* p, int64_t i, float v) { p[i] = v; }

// src and dst may be the same
template <typename TS>
__device__ __forceinline__ void chunk_scale(const TS* src, TS* dst, int64_t n, float c) {
  using R8 = Raw8<TS>;
  int64_t i = 0;
  if (aligned16_dev(src) && aligned16_dev(dst)) {
    const int64_t n8 = n / 8;
    for (int64_t b = threadIdx.x; b < n8; b += kGradVecs * kGradThreads) {
      typename R8::raw r[kGradVecs];
#pragma unroll
      for (int u = 0; u < kGradVecs; ++u)
        if (b + u * kGradThreads < n8) r[u] = R8::load(src + (b + u * kGradThreads) * 8);
#pragma unroll
      for (int u = 0; u < kGradVecs; ++u)
        if (b + u * kGradThreads < n8) {
          float f[8];
          R8::unpack(r[u], f);
          if (c != 1.0f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= c;
            Vec8<TS>::store(dst + (b + u * kGradThreads) * 8, f);
          } else {
            R8::store(dst + (b + u * kGradThreads) * 8, r[u]);   // as it is, a NaN's bits too
          }
        }
    }
    i = n8 * 8;
  }
  for (int64_t b = i + threadIdx.x; b < n; b += kGradThreads) {
    if (c != 1.0f)
      put<TS>(dst, b, elem<TS>(src, b) * c);
    else
      dst[b] = src[b];
  }
}

// The workgroups take the chunks from the last to the first: what the pass
// before read last is still in the caches then (617 MB of eight sublayers 4 %
// faster than from the first on).  part: the chunks' sums to add here, else null.
__global__ __launch_bounds__(kGradThreads) void k_grad_scale(const GradBatch b, const float* __restrict__ factor,
                                                             const double* __restrict__ part, int chunks,
                                                             float max_norm, float* __restrict__ norm) {
  float c;
  if (part) {
    __shared__ double red[kGradThreads / 64];
    double s = 0.;
    for (int i = threadIdx.x; i < chunks; i += kGradThreads) s += part[i];
    s = sqrt(block_sum_f64<kGradThreads>(s, red));
    c = clip_factor(s, max_norm);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)s;
  } else {
    c = *factor;
  }
  const GradChunk k = find_chunk(b, (int)(gridDim.x - 1 - blockIdx.x));
  const uint64_t src = b.src[k.i], dst = b.dst[k.i];
  if (c == 1.0f && src == dst) return;
  if (k.f32)
    chunk_scale(reinterpret_cast<const float*>(src) + k.at, reinterpret_cast<float*>(dst) + k.at, k.n, c);
  else
    chunk_scale(reinterpret_cast<const uint16_t*>(src) + k.at, reinterpret_cast<uint16_t*>(dst) + k.at, k.n, c);
}

// the launches themselves, on a stream
struct GradStream {
  double* part;
  float *factor, *norm_out;
  float max_norm;
  hipStream_t s;
  hipError_t squares(const GradBatch& b) {
    k_grad_squares<<<dim3((unsigned)b.first[b.n]), dim3(kGradThreads), 0, s>>>(b, part);
    return hipGetLastError();
  }
  hipError_t norm(int64_t chunks, bool clip) {
    k_grad_norm<<<dim3(1), dim3(kNormThreads), 0, s>>>(part, chunks, max_norm, norm_out, clip ? factor : nullptr);
    return hipGetLastError();
  }
  hipError_t scale(const GradBatch& b, bool own, int64_t chunks) {
    k_grad_scale<<<dim3((unsigned)b.first[b.n]), dim3(kGradThreads), 0, s>>>(b, factor, own ? part : nullptr,
                                                                             (int)chunks, max_norm, norm_out);
    return hipGetLastError();
  }
};

}  // namespace

size_t grad_ws_bytes(int n) { return 16 + grad_places(n) * sizeof(double); }

hipError_t launch_grad_clip(int n, const void* const* grads, const int64_t* counts, const int32_t* dtypes,
                            float max_norm, void* const* outs, float* norm, void* ws, hipStream_t s) {
  GradStream launch{reinterpret_cast<double*>(reinterpret_cast<char*>(ws) + 16), reinterpret_cast<float*>(ws), norm,
                    max_norm, s};
  return grad_launches(launch, n, grads, counts, dtypes, outs);
}

}  // namespace xhc
