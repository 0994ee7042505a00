// Gated feed-forward block, forward and backward.
//
//   h = act(g) u,  g = x W_gate,  u = x W_up;   F = h W_down
//   dh = dF W_down^T,  du = dh act(g),  dg = dh u act'(g)
//   dx = dg W_gate^T + du W_up^T,  dW_gate = x^T dg,  dW_up = x^T du,  dW_down = h^T dF
//
// Five launches' worth of products: [g|u] with the activation and the product
// in its epilogue, F; backward dh with the gate's reverse in its epilogue, dx
// (one product over k = 2 H), [dW_gate | dW_up] and dW_down.  Weights enter as
// bf16 (packed once a step), sums are fp32.  bf16 state: h, dg and du are
// rounded to bf16, as operands of the next product, and so are the saved g and
// u: each rounding (2^-9 of the value) is of the size of the one that F, dx
// and the weight gradients get as outputs.  fp32 state: activations are
// multiplied as three bf16 parts that add up to them exactly, so that nothing
// is rounded below fp32 (three passes over k; six for the weight gradients).
#include "xhc_ffn.h"

#include <algorithm>

namespace xhc {

namespace {

__host__ __device__ constexpr int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline int64_t pad_k(int64_t n) { return round_up(n, kBK); }

// ---------------------------------------------------------------- packing
// Fragment (nb, kb) of a packed matrix: lane l holds B[n(nb, l % 16)][32 kb + 8 (l / 16) + e].
// Two blocks of 16 make up 32 n: row p of block a is n = 32 j + 8 (p / 4) + 4 a
// + p % 4, so that a lane's sums of the two blocks are eight consecutive n.
// The up projection's blocks come gate, up, gate, up for each 32 columns of h.
__device__ __forceinline__ int perm_n(int a, int p) { return 8 * (p / 4) + 4 * a + p % 4; }

struct PackArgs {
  const float* W;      // [R, Q]
  int64_t R, Q;
  // n = column, k = row: blocks of 32 columns are nmul blocks of 16 apart, nadd + step * a within
  uint4* kr;
  int64_t kr_ld;       // k blocks
  int nmul, nadd, step;
  // n = row, k = koff + column (NULL: not wanted)
  uint4* kc;
  int64_t kc_ld, koff;
  int64_t nr, nc;      // n up to where blocks exist (of 32; values past the matrix are zero)
};

__device__ __forceinline__ uint32_t pair(uint16_t a, uint16_t b) { return (uint32_t)a | (uint32_t)b << 16; }

// one 64 x 64 tile: read once, written in both orders
__global__ __launch_bounds__(256) void k_ffn_pack(const PackArgs a) {
  constexpr int LD = 72;
  __shared__ __align__(16) uint16_t s[64][LD];
  const int64_t r0 = (int64_t)blockIdx.y * 64, q0 = (int64_t)blockIdx.x * 64;
  for (int i = threadIdx.x; i < 64 * 64; i += 256) {
    const int64_t r = r0 + i / 64, q = q0 + i % 64;
    s[i / 64][i % 64] = r < a.R && q < a.Q ? (uint16_t)f2bf(a.W[r * a.Q + q]) : (uint16_t)0;
  }
  __syncthreads();
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, p = lane % 16, g = lane / 16;
  // k = row: n blocks of the columns (two 32s of two blocks) x two k blocks
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    const int id = wave * 2 + f, j = id / 4, blk = id / 2 % 2, kb = id % 2;
    const int n = 32 * j + perm_n(blk, p), k = 32 * kb + 8 * g;
    if (q0 + 32 * j < a.nr) {
      const uint4 v = make_uint4(pair(s[k][n], s[k + 1][n]), pair(s[k + 2][n], s[k + 3][n]),
                                 pair(s[k + 4][n], s[k + 5][n]), pair(s[k + 6][n], s[k + 7][n]));
      const int64_t nb = (q0 / 32 + j) * a.nmul + a.nadd + blk * a.step;
      a.kr[(nb * a.kr_ld + r0 / 32 + kb) * 64 + lane] = v;
    }
  }
  if (!a.kc) return;
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    const int id = wave * 2 + f, j = id / 4, blk = id / 2 % 2, kb = id % 2;
    const int n = 32 * j + perm_n(blk, p), k = 32 * kb + 8 * g;
    if (r0 + 32 * j < a.nc) {
      const uint4 v = *reinterpret_cast<const uint4*>(&s[n][k]);
      const int64_t nb = (r0 / 32 + j) * 2 + blk;
      a.kc[(nb * a.kc_ld + (a.koff + q0) / 32 + kb) * 64 + lane] = v;
    }
  }
}

// the packed buffer's parts, in bytes
struct Packed {
  int64_t Cp, Hp, n32C, n32H;   // n32: blocks of 32 n
  size_t up, down, dh, dx, total_fwd, total;
  Packed(int64_t C, int64_t H) {
    Cp = pad_k(C);
    Hp = pad_k(H);
    n32C = (C + 31) / 32;
    n32H = Hp / 32;
    up = 0;
    down = up + (size_t)n32H * 4 * (Cp / 32) * 1024;
    dh = total_fwd = down + (size_t)n32C * 2 * (Hp / 32) * 1024;
    dx = dh + (size_t)n32H * 2 * (Cp / 32) * 1024;
    total = dx + (size_t)n32C * 2 * (2 * Hp / 32) * 1024;
  }
};

// ---------------------------------------------------------------- activations

// act(g) and, with D, act'(g)
template <bool D>
__device__ __forceinline__ float act_of(int act, float g, float& d) {
  if (act == XHC_ACT_SILU) {
    const float e = __builtin_amdgcn_rcpf(1.0f + __expf(-g));
    if (D) d = e * (1.0f + g * (1.0f - e));
    return g * e;
  }
  const float e = 0.5f * (1.0f + erff(g * 0.70710678118654752f));
  if (D) d = e + g * __expf(-0.5f * g * g) * 0.39894228040143268f;
  return g * e;
}

// x as three bf16 parts that add up to it: the top 8 bits of what is left, each
// time.  An Inf or NaN is its first part alone.
__device__ __forceinline__ void split3(float x, float (&p)[3]) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7f800000u) == 0x7f800000u) {
    p[0] = __uint_as_float((u & 0x007fffffu) ? (u | 0x00400000u) & 0xffff0000u : u);
    p[1] = p[2] = 0.f;
    return;
  }
  p[0] = __uint_as_float(u & 0xffff0000u);
  const float r = x - p[0];
  p[1] = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
  p[2] = r - p[1];
}

// eight values as the operand of a later product: bf16, or the three parts
template <typename TS> __device__ __forceinline__ void store_operand(uint16_t* p, int64_t plane, const float (&f)[8]);
template <>
__device__ __forceinline__ void store_operand<uint16_t>(uint16_t* p, int64_t, const float (&f)[8]) {
  Vec8<uint16_t>::store(p, f);
}
template <>
__device__ __forceinline__ void store_operand<float>(uint16_t* p, int64_t plane, const float (&f)[8]) {
  float v[3][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float q[3];
    split3(f[e], q);
    v[0][e] = q[0];
    v[1][e] = q[1];
    v[2][e] = q[2];
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) Vec8<uint16_t>::store(p + i * plane, v[i]);
}

__global__ __launch_bounds__(256) void k_ffn_split(const float* __restrict__ x, int64_t n8, uint16_t* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n8) return;
  float f[8];
  Vec8<float>::load(x + i * 8, f);
  store_operand<float>(out + i * 8, n8 * 8, f);
}

// ---------------------------------------------------------------- epilogues

// h from g and u (eight columns of one token); g and u saved where wanted
template <typename TS>
struct EpiUp {
  static constexpr bool kTwo = true;
  int64_t T;
  int H, cols;         // cols: Hp
  int act;
  uint16_t* h;
  int64_t h_plane;
  TS* saved;           // [2, T, Hp]: g, u
  __device__ __forceinline__ void finish(int64_t t, int64_t c, const float (&g)[8], const float (&u)[8]) const {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float d;
      f[e] = c + e < H ? act_of<false>(act, g[e], d) * u[e] : 0.f;
    }
    store_operand<TS>(h + t * cols + c, h_plane, f);
    if (saved) {
      Vec8<TS>::store(saved + t * cols + c, g);
      Vec8<TS>::store(saved + (T + t) * cols + c, u);
    }
  }
};

// F or dx
template <typename TS>
struct EpiOut {
  static constexpr bool kTwo = false;
  int64_t T;
  int cols;
  TS* out;
  __device__ __forceinline__ void finish(int64_t t, int64_t c, const float (&v)[8], const float (&)[8]) const {
    Vec8<TS>::store(out + t * cols + c, v);
  }
};

// dg, du and h again from dh and the saved g and u
template <typename TS>
struct EpiGate {
  static constexpr bool kTwo = false;
  int64_t T;
  int H, cols;         // cols: Hp
  int act;
  const TS* saved;
  uint16_t *dgu, *h;   // [T, 2 Hp], [T, Hp]
  int64_t dgu_plane, h_plane;
  __device__ __forceinline__ void finish(int64_t t, int64_t c, const float (&dh)[8], const float (&)[8]) const {
    float g[8], u[8], f[8], dg[8], du[8];
    Vec8<TS>::load(saved + t * cols + c, g);
    Vec8<TS>::load(saved + (T + t) * cols + c, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float d;
      const float a = act_of<true>(act, g[e], d);
      const bool in = c + e < H;
      f[e] = in ? a * u[e] : 0.f;
      dg[e] = in ? dh[e] * u[e] * d : 0.f;
      du[e] = in ? dh[e] * a : 0.f;
    }
    store_operand<TS>(dgu + t * 2 * cols + c, dgu_plane, dg);
    store_operand<TS>(dgu + t * 2 * cols + cols + c, dgu_plane, du);
    store_operand<TS>(h + t * cols + c, h_plane, f);
  }
};

// weight gradients: row m, columns n of out[n / nsplit]
template <typename TS>
struct EpiWeight {
  int64_t M, N;        // rows, columns of the product
  int64_t ncols;       // columns of one output
  int64_t nsplit;      // product columns of the first
  TS *out0, *out1;
  __device__ __forceinline__ void finish(int64_t m, int64_t n, const float (&v)[4]) const {
    TS* o = out0;
    if (n >= nsplit) {
      n -= nsplit;
      o = out1;
    }
    o += m * ncols + n;
    if (ncols % 4 == 0) {          // n too: whole groups of four, aligned
      if (n < ncols) put4(o, v);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < ncols) put1(o + e, v[e]);
    }
  }
  static __device__ __forceinline__ void put4(uint16_t* p, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]));
  }
  static __device__ __forceinline__ void put4(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
  static __device__ __forceinline__ void put1(uint16_t* p, float v) { *p = (uint16_t)f2bf(v); }
  static __device__ __forceinline__ void put1(float* p, float v) { *p = v; }
};

// ---------------------------------------------------------------- products

// activations [t, k] times packed weights; part: the sums of a part of k, [part][T][cols (x 2)]
template <int FN, int FT, int WN, int WT, class Epi>
__global__ __launch_bounds__(64 * WN * WT) void k_ffn_rows(const GemmArgs a, const Epi e, float* __restrict__ part) {
  __shared__ __align__(1024) unsigned char lds[2 * 128 * 16 * (FN * WN + FT * WT)];
  gemm_tile<FragTile, RowTile, FN, FT, WN, WT>(a, lds, [&](f32x4 (&acc)[FN][FT], int64_t n0, int64_t t0, int lane) {
    constexpr int PER = Epi::kTwo ? 4 : 2;       // blocks of 16 that give eight columns
    static_assert(FN % PER == 0, "whole groups");
    const int q = lane / 16;
#pragma unroll
    for (int j = 0; j < FT; ++j) {
      const int64_t t = t0 + j * 16 + lane % 16;
#pragma unroll
      for (int i = 0; i < FN / PER; ++i) {
        const int64_t c = (Epi::kTwo ? n0 / 2 : n0) + i * 32 + q * 8;
        if (t >= e.T || c >= e.cols) continue;
        float v[8], w[8];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (Epi::kTwo) {
            v[x] = acc[4 * i][j][x];
            w[x] = acc[4 * i + 1][j][x];
            v[4 + x] = acc[4 * i + 2][j][x];
            w[4 + x] = acc[4 * i + 3][j][x];
          } else {
            v[x] = acc[2 * i][j][x];
            v[4 + x] = acc[2 * i + 1][j][x];
          }
        }
        if (gridDim.y > 1) {
          float* p = part + ((int64_t)blockIdx.y * e.T + t) * e.cols * (Epi::kTwo ? 2 : 1) + c;
          Vec8<float>::store(p, v);
          if (Epi::kTwo) Vec8<float>::store(p + e.cols, w);
        } else {
          e.finish(t, c, v, w);
        }
      }
    }
  });
}

// the parts of k added in order, then the epilogue
template <class Epi>
__global__ __launch_bounds__(256) void k_ffn_rows_join(const Epi e, const float* __restrict__ part, int parts) {
  const int64_t g = e.cols / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t t = i / g, c = i % g * 8, ld = (int64_t)e.cols * (Epi::kTwo ? 2 : 1);
  if (t >= e.T) return;
  float v[8] = {}, w[8] = {};
  for (int p = 0; p < parts; ++p) {
    const float* s = part + ((int64_t)p * e.T + t) * ld + c;
    float f[8];
    Vec8<float>::load(s, f);
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] += f[x];
    if (Epi::kTwo) {
      Vec8<float>::load(s + e.cols, f);
#pragma unroll
      for (int x = 0; x < 8; ++x) w[x] += f[x];
    }
  }
  e.finish(t, c, v, w);
}

// weight gradients: k is the token on both sides; part: [part][M][N]
template <int FN, int FT, int WN, int WT, class Epi>
__global__ __launch_bounds__(64 * WN * WT) void k_ffn_cols(const GemmArgs a, const Epi e, float* __restrict__ part) {
  __shared__ __align__(1024) unsigned char lds[2 * 128 * 16 * (FN * WN + FT * WT)];
  gemm_tile<ColTile, ColTile, FN, FT, WN, WT>(a, lds, [&](f32x4 (&acc)[FN][FT], int64_t n0, int64_t t0, int lane) {
#pragma unroll
    for (int j = 0; j < FT; ++j) {
      const int64_t m = t0 + j * 16 + lane % 16;
#pragma unroll
      for (int i = 0; i < FN; ++i) {
        const int64_t n = n0 + i * 16 + lane / 16 * 4;
        if (m >= e.M || n >= e.N) continue;
        const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        if (gridDim.y > 1)
          *reinterpret_cast<float4*>(part + ((int64_t)blockIdx.y * e.M + m) * e.N + n) =
              make_float4(v[0], v[1], v[2], v[3]);
        else
          e.finish(m, n, v);
      }
    }
  });
}

template <class Epi>
__global__ __launch_bounds__(256) void k_ffn_cols_join(const Epi e, const float* __restrict__ part, int parts) {
  const int64_t g = e.N / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t m = i / g, n = i % g * 4;
  if (m >= e.M) return;
  float v[4] = {};
  for (int p = 0; p < parts; ++p) {
    const float4 f = *reinterpret_cast<const float4*>(part + ((int64_t)p * e.M + m) * e.N + n);
    v[0] += f.x;
    v[1] += f.y;
    v[2] += f.z;
    v[3] += f.w;
  }
  e.finish(m, n, v);
}

// ---------------------------------------------------------------- host side

// How a product runs: its tile and the parts that k is cut into.
struct Plan {
  int bn, bt;
  int64_t gn, gt, ksteps, per;   // per: stages of a part
  int nseg, parts;
};
Plan plan_product(int64_t n, int64_t t, int64_t k, int nseg) {
  Plan p{};
  p.bn = p.bt = 128;
  p.gn = (n + p.bn - 1) / p.bn;
  p.gt = (t + p.bt - 1) / p.bt;
  p.ksteps = std::max<int64_t>(1, (k + kBK - 1) / kBK);   // no tokens: one stage of zeros
  p.nseg = nseg;
  p.parts = 1;
  p.per = p.ksteps * nseg;
  return p;
}
size_t part_floats(const Plan& p, int64_t t, int64_t cols) { return p.parts > 1 ? (size_t)p.parts * t * cols : 0; }

GemmArgs args_of(const Plan& p, const Operand& n, const Operand& t, const Segments& seg) {
  return GemmArgs{n, t, seg, (int)p.ksteps, p.per, p.gn, p.gt};
}

template <class Epi>
hipError_t rows(const Plan& p, const GemmArgs& a, const Epi& e, float* part, hipStream_t s) {
  k_ffn_rows<4, 4, 2, 2, Epi><<<dim3((unsigned)(p.gn * p.gt), (unsigned)p.parts), dim3(256), 0, s>>>(a, e, part);
  if (p.parts > 1) {
    const int64_t n = e.T * (e.cols / 8);
    k_ffn_rows_join<Epi><<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(e, part, p.parts);
  }
  return hipGetLastError();
}
template <class Epi>
hipError_t cols(const Plan& p, const GemmArgs& a, const Epi& e, float* part, hipStream_t s) {
  k_ffn_cols<4, 4, 2, 2, Epi><<<dim3((unsigned)(p.gn * p.gt), (unsigned)p.parts), dim3(256), 0, s>>>(a, e, part);
  if (p.parts > 1) {
    const int64_t n = e.M * (e.N / 4);
    k_ffn_cols_join<Epi><<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(e, part, p.parts);
  }
  return hipGetLastError();
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// the workspace: the fp32 state's parts of x (and dF), h, [dg|du], parts of k
struct Ws {
  Plan up, down, dh, dx, dwgu, dwd;
  size_t x, dF, h, dgu, part, total;
  Ws(int state_dtype, int64_t T, int64_t C, int64_t H, bool bwd) {
    const Packed pk(C, H);
    const bool f32 = state_dtype == XHC_F32;
    const int P = f32 ? 3 : 1, ns = f32 ? 3 : 1, nw = f32 ? 6 : 1;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
      const size_t o = at;
      at += align256(bytes);
      return o;
    };
    x = take(f32 ? (size_t)P * T * C * 2 : 0);
    dF = take(f32 && bwd ? (size_t)P * T * C * 2 : 0);
    h = take((size_t)P * T * pk.Hp * 2);
    dgu = take(bwd ? (size_t)P * T * pk.Hp * 4 : 0);
    size_t most = 0;
    if (bwd) {
      dh = plan_product(pk.Hp, T, C, ns);
      dx = plan_product(C, T, 2 * pk.Hp, ns);
      dwgu = plan_product(2 * pk.Hp, C, T, nw);
      dwd = plan_product(C, H, T, nw);
      most = std::max({part_floats(dh, T, pk.Hp), part_floats(dx, T, C), part_floats(dwgu, C, 2 * pk.Hp),
                       part_floats(dwd, H, C)});
    } else {
      up = plan_product(2 * pk.Hp, T, C, ns);
      down = plan_product(C, T, pk.Hp, ns);
      most = std::max(part_floats(up, T, 2 * pk.Hp), part_floats(down, T, C));
    }
    part = take(most * sizeof(float));
    total = at;
  }
};

hipError_t split_planes(const float* x, int64_t n, void* out, hipStream_t s) {
  if (n == 0) return hipSuccess;
  k_ffn_split<<<dim3((unsigned)((n / 8 + 255) / 256)), dim3(256), 0, s>>>(x, n / 8, reinterpret_cast<uint16_t*>(out));
  return hipGetLastError();
}

template <typename TS>
hipError_t ffn(int state_dtype, int64_t T, int64_t C, int64_t H, int act, const void* input, const void* packed,
               void* F, void* saved, void* workspace, hipStream_t s) {
  const Packed pk(C, H);
  const Ws w(state_dtype, T, C, H, false);
  const bool f32 = state_dtype == XHC_F32;
  char* ws = reinterpret_cast<char*>(workspace);
  const char* pw = reinterpret_cast<const char*>(packed);
  const Segments seg = f32 ? segs_weights() : segs_bf16();
  float* part = reinterpret_cast<float*>(ws + w.part);
  uint16_t* h = reinterpret_cast<uint16_t*>(ws + w.h);
  const void* x = input;
  hipError_t e = hipSuccess;
  if (f32) {
    x = ws + w.x;
    e = split_planes(reinterpret_cast<const float*>(input), T * C, ws + w.x, s);
  }
  if (e == hipSuccess)
    e = rows(w.up, args_of(w.up, Operand{pw + pk.up, 0, pk.Cp / 32, pk.n32H * 4, 0},
                           Operand{x, T * C * 2, C, T, (int)C}, seg),
             EpiUp<TS>{T, (int)H, (int)pk.Hp, act, h, T * pk.Hp, reinterpret_cast<TS*>(saved)}, part, s);
  if (e == hipSuccess)
    e = rows(w.down, args_of(w.down, Operand{pw + pk.down, 0, pk.Hp / 32, pk.n32C * 2, 0},
                             Operand{h, T * pk.Hp * 2, pk.Hp, T, (int)pk.Hp}, seg),
             EpiOut<TS>{T, (int)C, reinterpret_cast<TS*>(F)}, part, s);
  return e;
}

template <typename TS>
hipError_t ffn_bwd(int state_dtype, int64_t T, int64_t C, int64_t H, int act, const void* input, const void* packed,
                   const void* saved, const void* dF, void* d_input, void* dW_gate, void* dW_up, void* dW_down,
                   void* workspace, hipStream_t s) {
  const Packed pk(C, H);
  const Ws w(state_dtype, T, C, H, true);
  const bool f32 = state_dtype == XHC_F32;
  char* ws = reinterpret_cast<char*>(workspace);
  const char* pw = reinterpret_cast<const char*>(packed);
  const Segments sw = f32 ? segs_weights() : segs_bf16(), sa = f32 ? segs_f32() : segs_bf16();
  float* part = reinterpret_cast<float*>(ws + w.part);
  uint16_t *h = reinterpret_cast<uint16_t*>(ws + w.h), *dgu = reinterpret_cast<uint16_t*>(ws + w.dgu);
  const void *x = input, *df = dF;
  hipError_t e = hipSuccess;
  if (f32) {
    x = ws + w.x;
    df = ws + w.dF;
    e = split_planes(reinterpret_cast<const float*>(input), T * C, ws + w.x, s);
    if (e == hipSuccess) e = split_planes(reinterpret_cast<const float*>(dF), T * C, ws + w.dF, s);
  }
  const Operand ox{x, T * C * 2, C, T, (int)C}, odf{df, T * C * 2, C, T, (int)C};
  const Operand oh{h, T * pk.Hp * 2, pk.Hp, T, (int)pk.Hp};
  const Operand odgu{dgu, T * pk.Hp * 4, 2 * pk.Hp, T, (int)(2 * pk.Hp)};
  if (e == hipSuccess && T > 0)
    e = rows(w.dh, args_of(w.dh, Operand{pw + pk.dh, 0, pk.Cp / 32, pk.n32H * 2, 0}, odf, sw),
             EpiGate<TS>{T, (int)H, (int)pk.Hp, act, reinterpret_cast<const TS*>(saved), dgu, h, T * 2 * pk.Hp,
                         T * pk.Hp},
             part, s);
  if (e == hipSuccess && T > 0)
    e = rows(w.dx, args_of(w.dx, Operand{pw + pk.dx, 0, 2 * pk.Hp / 32, pk.n32C * 2, 0}, odgu, sw),
             EpiOut<TS>{T, (int)C, reinterpret_cast<TS*>(d_input)}, part, s);
  if (e == hipSuccess)
    e = cols(w.dwgu, args_of(w.dwgu, odgu, ox, sa),
             EpiWeight<TS>{C, 2 * pk.Hp, H, pk.Hp, reinterpret_cast<TS*>(dW_gate), reinterpret_cast<TS*>(dW_up)},
             part, s);
  if (e == hipSuccess)
    e = cols(w.dwd, args_of(w.dwd, odf, oh, sa),
             EpiWeight<TS>{H, C, C, C, reinterpret_cast<TS*>(dW_down), nullptr}, part, s);
  return e;
}

}  // namespace

size_t ffn_packed_bytes(int64_t C, int64_t H, bool with_bwd) {
  const Packed p(C, H);
  return with_bwd ? p.total : p.total_fwd;
}
size_t ffn_saved_bytes(int state_dtype, int64_t T, int64_t H) {
  return (size_t)2 * T * pad_k(H) * (state_dtype == XHC_F32 ? 4 : 2);
}
size_t ffn_ws_bytes(int state_dtype, int64_t T, int64_t C, int64_t H, bool bwd) {
  return Ws(state_dtype, T, C, H, bwd).total;
}

hipError_t launch_ffn_pack(int64_t C, int64_t H, const float* W_gate, const float* W_up, const float* W_down,
                           bool with_bwd, void* packed, hipStream_t s) {
  const Packed p(C, H);
  char* b = reinterpret_cast<char*>(packed);
  const auto at = [&](size_t o) { return reinterpret_cast<uint4*>(b + o); };
  const unsigned tc = (unsigned)(p.Cp / 64), th = (unsigned)(p.Hp / 64);
  for (int i = 0; i < 2; ++i)
    k_ffn_pack<<<dim3(th, tc), dim3(256), 0, s>>>(PackArgs{i ? W_up : W_gate, C, H, at(p.up), p.Cp / 32, 4, i, 2,
                                                           with_bwd ? at(p.dx) : nullptr, 2 * p.Hp / 32, i * p.Hp,
                                                           p.Hp, C});
  k_ffn_pack<<<dim3(tc, th), dim3(256), 0, s>>>(PackArgs{W_down, H, C, at(p.down), p.Hp / 32, 2, 0, 1,
                                                         with_bwd ? at(p.dh) : nullptr, p.Cp / 32, 0, C, p.Hp});
  return hipGetLastError();
}

hipError_t launch_ffn(int state_dtype, int64_t T, int64_t C, int64_t H, int act, const void* input,
                      const void* packed, void* F, void* saved, void* workspace, hipStream_t s) {
  return state_dtype == XHC_BF16
             ? ffn<uint16_t>(state_dtype, T, C, H, act, input, packed, F, saved, workspace, s)
             : ffn<float>(state_dtype, T, C, H, act, input, packed, F, saved, workspace, s);
}

hipError_t launch_ffn_bwd(int state_dtype, int64_t T, int64_t C, int64_t H, int act, const void* input,
                          const void* packed, const void* saved, const void* dF, void* d_input, void* dW_gate,
                          void* dW_up, void* dW_down, void* workspace, hipStream_t s) {
  return state_dtype == XHC_BF16 ? ffn_bwd<uint16_t>(state_dtype, T, C, H, act, input, packed, saved, dF, d_input,
                                                     dW_gate, dW_up, dW_down, workspace, s)
                                 : ffn_bwd<float>(state_dtype, T, C, H, act, input, packed, saved, dF, d_input,
                                                  dW_gate, dW_up, dW_down, workspace, s);
}

}  // namespace xhc
