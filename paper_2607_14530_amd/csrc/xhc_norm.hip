// RMSNorm of token rows with a gain, forward and backward.
//
//   r_t = 1 / sqrt(mean_c x[t,c]^2 + eps),  y = x r w
//   dx  = r v - x r^3 mean_c(v x),  v = dy w;   dw[c] = sum_t dy[t,c] x[t,c] r_t
//
// Bound by HBM: 2 T C elements forward, 3 T C backward.  Forward a wave takes
// a row and holds all of it in registers (C <= 4096: up to eight 8-element
// vectors per lane), so that each element is read once and there is no barrier;
// backward up to C = 1024, and up to 4096 a workgroup takes four rows.  Wider
// rows take a workgroup each, which reads them a second time (from the caches).
// All sums are fp32; y and dx are rounded once.
//
// The gain's gradient: every lane keeps the sums of its columns over its rows,
// a workgroup adds its waves' sums, and a second kernel adds the workgroups' in
// order, so that the result does not depend on timing.
#include "xhc_device.h"

namespace xhc {

namespace {

constexpr int kNormWaves = 4;            // rows of a workgroup at a time
constexpr int kNormRegC = 4096;          // widest row that a wave holds

template <int V> __device__ __forceinline__ bool in_row(int v, int lane, int C) { return (v * 64 + lane) * 8 < C; }

template <typename TS, int V>
__global__ __launch_bounds__(64 * kNormWaves) void k_rmsnorm(const TS* __restrict__ x, const float* __restrict__ gain,
                                                             int64_t T, int C, float eps, TS* __restrict__ y,
                                                             float* __restrict__ rstd) {
  using R8 = Raw8<TS>;
  const int lane = threadIdx.x % 64;
  const int64_t t = (int64_t)blockIdx.x * kNormWaves + threadIdx.x / 64;
  if (t >= T) return;
  typename R8::raw raw[V];
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (in_row<V>(v, lane, C)) raw[v] = R8::load(x + t * C + (v * 64 + lane) * 8);
  float s = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (in_row<V>(v, lane, C)) {
      float f[8];
      R8::unpack(raw[v], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(f[e], f[e], s);
    }
  const float r = 1.0f / sqrtf(wave_sum(s) / (float)C + eps);
  if (rstd && lane == 0) rstd[t] = r;
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (in_row<V>(v, lane, C)) {
      float f[8], w[8];
      R8::unpack(raw[v], f);
      Vec8<float>::load(gain + (v * 64 + lane) * 8, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = f[e] * r * w[e];
      Vec8<TS>::store(y + t * C + (v * 64 + lane) * 8, f);
    }
}

__device__ __forceinline__ float block_sum256(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}

// one workgroup per row, any width
template <typename TS>
__global__ __launch_bounds__(256) void k_rmsnorm_wide(const TS* __restrict__ x, const float* __restrict__ gain,
                                                      int C, float eps, TS* __restrict__ y,
                                                      float* __restrict__ rstd) {
  __shared__ float red[4];
  const int64_t t = blockIdx.x;
  float s = 0.f;
  for (int c = threadIdx.x * 8; c < C; c += 2048) {
    float f[8];
    Vec8<TS>::load(x + t * C + c, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(f[e], f[e], s);
  }
  const float r = 1.0f / sqrtf(block_sum256(s, red) / (float)C + eps);
  if (rstd && threadIdx.x == 0) rstd[t] = r;
  for (int c = threadIdx.x * 8; c < C; c += 2048) {
    float f[8], w[8];
    Vec8<TS>::load(x + t * C + c, f);
    Vec8<float>::load(gain + c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = f[e] * r * w[e];
    Vec8<TS>::store(y + t * C + c, f);
  }
}

// dx of a wave's rows, and its columns' part of dw.  Rows t = first, first +
// stride, ...: the waves of the launch take turns.
template <typename TS, int V>
__global__ __launch_bounds__(64 * kNormWaves) void k_rmsnorm_bwd(const TS* __restrict__ x,
                                                                 const float* __restrict__ gain,
                                                                 const float* __restrict__ rstd,
                                                                 const TS* __restrict__ dy, int64_t T, int C,
                                                                 TS* __restrict__ dx, float* __restrict__ part) {
  using R8 = Raw8<TS>;
  __shared__ float red[64 * 8 * V];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  float acc[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[v][e] = 0.f;
  const int64_t stride = (int64_t)gridDim.x * kNormWaves;
  for (int64_t t = (int64_t)blockIdx.x * kNormWaves + wave; t < T; t += stride) {
    typename R8::raw rx[V], rd[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (in_row<V>(v, lane, C)) {
        rx[v] = R8::load(x + t * C + (v * 64 + lane) * 8);
        rd[v] = R8::load(dy + t * C + (v * 64 + lane) * 8);
      }
    const float r = rstd[t];
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (in_row<V>(v, lane, C)) {
        float fx[8], fd[8], w[8];
        R8::unpack(rx[v], fx);
        R8::unpack(rd[v], fd);
        Vec8<float>::load(gain + (v * 64 + lane) * 8, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s = fmaf(fd[e] * w[e], fx[e], s);
          acc[v][e] = fmaf(fd[e], fx[e] * r, acc[v][e]);
        }
      }
    const float m = wave_sum(s) / (float)C * r * r;   // dx = r (v - x r^2 mean(v x))
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (in_row<V>(v, lane, C)) {
        float fx[8], fd[8], w[8];
        R8::unpack(rx[v], fx);
        R8::unpack(rd[v], fd);
        Vec8<float>::load(gain + (v * 64 + lane) * 8, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) fd[e] = r * (fd[e] * w[e] - fx[e] * m);
        Vec8<TS>::store(dx + t * C + (v * 64 + lane) * 8, fd);
      }
  }
  // the waves add to the workgroup's sums one after another
  for (int w = 0; w < kNormWaves; ++w) {
    if (w == wave) {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float* p = red + (v * 8 + e) * 64 + lane;
          *p = w == 0 ? acc[v][e] : *p + acc[v][e];
        }
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < 64 * 8 * V; i += 64 * kNormWaves) {
    const int c = ((i / 512) * 64 + i % 64) * 8 + (i / 64) % 8;
    if (c < C) part[(int64_t)blockIdx.x * C + c] = red[i];
  }
}

// The same for wider rows: the workgroup's threads take the columns of four
// rows at a time, so that a thread has few columns: their sums and their gain
// stay in registers, with eight vectors on the way (T = 16384, C = 4096 with a
// wave a row, its gain read twice from the cache: 108 us).
constexpr int kNormRows = 4;
template <typename TS, int V>
__global__ __launch_bounds__(256) void k_rmsnorm_bwd_cols(const TS* __restrict__ x, const float* __restrict__ gain,
                                                          const float* __restrict__ rstd,
                                                          const TS* __restrict__ dy, int64_t T, int C,
                                                          TS* __restrict__ dx, float* __restrict__ part) {
  using R8 = Raw8<TS>;
  __shared__ float red[2][kNormRows][4];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  float acc[V][8], w[V][8];
  bool in[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    in[v] = (v * 256 + tid) * 8 < C;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[v][e] = w[v][e] = 0.f;
    if (in[v]) Vec8<float>::load(gain + (v * 256 + tid) * 8, w[v]);
  }
  int flip = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * kNormRows; t0 < T; t0 += (int64_t)gridDim.x * kNormRows, flip ^= 1) {
    typename R8::raw rx[kNormRows][V], rd[kNormRows][V];
    float r[kNormRows];
#pragma unroll
    for (int i = 0; i < kNormRows; ++i) {
      if (t0 + i >= T) continue;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (in[v]) {
          rx[i][v] = R8::load(x + (t0 + i) * C + (v * 256 + tid) * 8);
          rd[i][v] = R8::load(dy + (t0 + i) * C + (v * 256 + tid) * 8);
        }
      r[i] = rstd[t0 + i];
    }
#pragma unroll
    for (int i = 0; i < kNormRows; ++i) {
      float s = 0.f;
      if (t0 + i < T) {
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (in[v]) {
            float fx[8], fd[8];
            R8::unpack(rx[i][v], fx);
            R8::unpack(rd[i][v], fd);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              s = fmaf(fd[e] * w[v][e], fx[e], s);
              acc[v][e] = fmaf(fd[e], fx[e] * r[i], acc[v][e]);
            }
          }
      }
      s = wave_sum(s);
      if (lane == 0) red[flip][i][wave] = s;
    }
    __syncthreads();   // one a turn: the next turn's sums go to the other half
#pragma unroll
    for (int i = 0; i < kNormRows; ++i) {
      if (t0 + i >= T) continue;
      const float* q = red[flip][i];
      const float m = (q[0] + q[1] + q[2] + q[3]) / (float)C * r[i] * r[i];
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (in[v]) {
          float fx[8], fd[8];
          R8::unpack(rx[i][v], fx);
          R8::unpack(rd[i][v], fd);
#pragma unroll
          for (int e = 0; e < 8; ++e) fd[e] = r[i] * (fd[e] * w[v][e] - fx[e] * m);
          Vec8<TS>::store(dx + (t0 + i) * C + (v * 256 + tid) * 8, fd);
        }
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (in[v]) Vec8<float>::store(part + (int64_t)blockIdx.x * C + (v * 256 + tid) * 8, acc[v]);
}

// dx of any width, one workgroup per row
template <typename TS>
__global__ __launch_bounds__(256) void k_rmsnorm_bwd_wide(const TS* __restrict__ x, const float* __restrict__ gain,
                                                          const float* __restrict__ rstd,
                                                          const TS* __restrict__ dy, int C, TS* __restrict__ dx) {
  __shared__ float red[4];
  const int64_t t = blockIdx.x;
  const float r = rstd[t];
  float s = 0.f;
  for (int c = threadIdx.x * 8; c < C; c += 2048) {
    float fx[8], fd[8], w[8];
    Vec8<TS>::load(x + t * C + c, fx);
    Vec8<TS>::load(dy + t * C + c, fd);
    Vec8<float>::load(gain + c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(fd[e] * w[e], fx[e], s);
  }
  const float m = block_sum256(s, red) / (float)C * r * r;
  for (int c = threadIdx.x * 8; c < C; c += 2048) {
    float fx[8], fd[8], w[8];
    Vec8<TS>::load(x + t * C + c, fx);
    Vec8<TS>::load(dy + t * C + c, fd);
    Vec8<float>::load(gain + c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) fd[e] = r * (fd[e] * w[e] - fx[e] * m);
    Vec8<TS>::store(dx + t * C + c, fd);
  }
}
// its part of dw: a workgroup takes 512 columns of a run of rows
template <typename TS>
__global__ __launch_bounds__(64) void k_rmsnorm_dw_wide(const TS* __restrict__ x, const float* __restrict__ rstd,
                                                        const TS* __restrict__ dy, int64_t T, int C, int64_t run,
                                                        float* __restrict__ part) {
  const int c = ((int)blockIdx.x * 64 + (int)threadIdx.x) * 8;
  if (c >= C) return;
  const int64_t t0 = blockIdx.y * run, t1 = t0 + run < T ? t0 + run : T;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int64_t t = t0; t < t1; ++t) {
    float fx[8], fd[8];
    Vec8<TS>::load(x + t * C + c, fx);
    Vec8<TS>::load(dy + t * C + c, fd);
    const float r = rstd[t];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = fmaf(fd[e], fx[e] * r, acc[e]);
  }
  Vec8<float>::store(part + (int64_t)blockIdx.y * C + c, acc);
}

// dw[c] = sum over the rows of part, in order: 16 threads take every 16th row
// of a column, kDwRows on the way, then their sums are added in order (512 rows
// of C = 4096: 4.8 us, 9.7 with a row at a time)
constexpr int kDwRows = 16;
__global__ __launch_bounds__(256) void k_rmsnorm_dw(const float* __restrict__ part, int rows, int C,
                                                    float* __restrict__ dw) {
  __shared__ float red[16][16];
  const int cl = threadIdx.x % 16, g = threadIdx.x / 16;
  const int c = (int)blockIdx.x * 16 + cl;
  float s = 0.f;
  if (c < C)
    for (int i = g; i < rows; i += 16 * kDwRows) {
      float f[kDwRows];
#pragma unroll
      for (int u = 0; u < kDwRows; ++u) f[u] = i + 16 * u < rows ? part[(int64_t)(i + 16 * u) * C + c] : 0.f;
#pragma unroll
      for (int u = 0; u < kDwRows; ++u) s += f[u];
    }
  red[g][cl] = s;
  __syncthreads();
  if (g == 0 && c < C) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += red[i][cl];
    dw[c] = s;
  }
}

// workgroups of the backward: two per CU, each wave a row at least
int64_t norm_bwd_blocks(int64_t T) {
  const int64_t b = (T + kNormWaves - 1) / kNormWaves;
  return b < 512 ? b : 512;
}

template <typename TS>
hipError_t rmsnorm(const TS* x, const float* gain, int64_t T, int C, float eps, TS* y, float* rstd, hipStream_t s) {
  const dim3 grid((unsigned)((T + kNormWaves - 1) / kNormWaves)), block(64 * kNormWaves);
  const int v = (C / 8 + 63) / 64;
  if (C > kNormRegC)
    k_rmsnorm_wide<TS><<<dim3((unsigned)T), dim3(256), 0, s>>>(x, gain, C, eps, y, rstd);
  else if (v <= 1)
    k_rmsnorm<TS, 1><<<grid, block, 0, s>>>(x, gain, T, C, eps, y, rstd);
  else if (v <= 2)
    k_rmsnorm<TS, 2><<<grid, block, 0, s>>>(x, gain, T, C, eps, y, rstd);
  else if (v <= 4)
    k_rmsnorm<TS, 4><<<grid, block, 0, s>>>(x, gain, T, C, eps, y, rstd);
  else
    k_rmsnorm<TS, 8><<<grid, block, 0, s>>>(x, gain, T, C, eps, y, rstd);
  return hipGetLastError();
}

template <typename TS>
hipError_t rmsnorm_bwd(const TS* x, const float* gain, const float* rstd, const TS* dy, int64_t T, int C, TS* dx,
                       float* dgain, float* part, hipStream_t s) {
  const int64_t blocks = norm_bwd_blocks(T);
  const dim3 grid((unsigned)blocks), block(64 * kNormWaves);
  int64_t rows = blocks;
  if (T == 0) {
    // no rows: dgain is zero
  } else if (C <= 512) {
    k_rmsnorm_bwd<TS, 1><<<grid, block, 0, s>>>(x, gain, rstd, dy, T, C, dx, part);
  } else if (C <= 1024) {
    k_rmsnorm_bwd<TS, 2><<<grid, block, 0, s>>>(x, gain, rstd, dy, T, C, dx, part);
  } else if (C <= 2048) {
    k_rmsnorm_bwd_cols<TS, 1><<<grid, block, 0, s>>>(x, gain, rstd, dy, T, C, dx, part);
  } else if (C <= 4096) {
    k_rmsnorm_bwd_cols<TS, 2><<<grid, block, 0, s>>>(x, gain, rstd, dy, T, C, dx, part);
  } else {
    const int64_t run = (T + blocks - 1) / blocks;
    rows = (T + run - 1) / run;
    k_rmsnorm_bwd_wide<TS><<<dim3((unsigned)T), dim3(256), 0, s>>>(x, gain, rstd, dy, C, dx);
    k_rmsnorm_dw_wide<TS><<<dim3((unsigned)((C / 8 + 63) / 64), (unsigned)rows), dim3(64), 0, s>>>(x, rstd, dy, T, C,
                                                                                                   run, part);
  }
  k_rmsnorm_dw<<<dim3((unsigned)((C + 15) / 16)), dim3(256), 0, s>>>(part, (int)rows, C, dgain);
  return hipGetLastError();
}

}  // namespace

size_t rmsnorm_bwd_ws_bytes(int64_t T, int C) { return (size_t)norm_bwd_blocks(T) * C * sizeof(float); }

hipError_t launch_rmsnorm(int state_dtype, const void* x, const float* gain, int64_t T, int C, float eps, void* y,
                          float* rstd, hipStream_t s) {
  if (state_dtype == XHC_BF16)
    return rmsnorm<uint16_t>(reinterpret_cast<const uint16_t*>(x), gain, T, C, eps, reinterpret_cast<uint16_t*>(y),
                             rstd, s);
  return rmsnorm<float>(reinterpret_cast<const float*>(x), gain, T, C, eps, reinterpret_cast<float*>(y), rstd, s);
}

hipError_t launch_rmsnorm_bwd(int state_dtype, const void* x, const float* gain, const float* rstd, const void* dy,
                              int64_t T, int C, void* dx, float* dgain, float* part, hipStream_t s) {
  if (state_dtype == XHC_BF16)
    return rmsnorm_bwd<uint16_t>(reinterpret_cast<const uint16_t*>(x), gain, rstd,
                                 reinterpret_cast<const uint16_t*>(dy), T, C, reinterpret_cast<uint16_t*>(dx), dgain,
                                 part, s);
  return rmsnorm_bwd<float>(reinterpret_cast<const float*>(x), gain, rstd, reinterpret_cast<const float*>(dy), T, C,
                            reinterpret_cast<float*>(dx), dgain, part, s);
}

}  // namespace xhc
