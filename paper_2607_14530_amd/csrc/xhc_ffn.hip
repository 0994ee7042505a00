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
// rounded to bf16, as operands of the next product: a rounding of the size of
// the one that F, dx and the weight gradients get as outputs.  fp32 state:
// activations are multiplied as three bf16 parts that add up to them exactly,
// so that nothing is rounded below fp32 (three passes over k; six for the
// weight gradients).
#include "xhc_ffn.h"

#include <algorithm>

namespace xhc {

namespace {

__host__ __device__ constexpr int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline int64_t pad_k(int64_t n) { return round_up(n, 64); }   // whole stages

// ---------------------------------------------------------------- packing
// The weights' rows (n) are permuted within blocks of 16 (perm_n).  The up
// projection's blocks come gate, up, gate, up.
struct PackArgs {
  const float* W;      // [R, Q]
  int64_t R, Q;
  // n = column, k = row: block b of 16 columns is block nmul b + nadd
  uint4* kr;
  int64_t kr_kb;       // k blocks
  int nmul, nadd;
  // n = row, k = koff + column (NULL: not wanted)
  uint4* kc;
  int64_t kc_kb, koff;
  int64_t nr, nc;      // n up to where blocks exist (values past the matrix are zero)
};

__device__ __forceinline__ uint32_t pair(uint16_t a, uint16_t b) { return (uint32_t)a | (uint32_t)b << 16; }

// one 64 x 64 tile of one matrix (blockIdx.z; the last has columns and rows the
// other way round): read once, written in both orders
struct PackAll { PackArgs m[3]; };
__global__ __launch_bounds__(256) void k_ffn_pack(const PackAll all) {
  constexpr int LD = 72;
  __shared__ __align__(16) uint16_t s[64][LD];
  const PackArgs a = all.m[blockIdx.z];
  const int64_t r0 = (int64_t)(blockIdx.z == 2 ? blockIdx.x : blockIdx.y) * 64;
  const int64_t q0 = (int64_t)(blockIdx.z == 2 ? blockIdx.y : blockIdx.x) * 64;
  for (int i = threadIdx.x; i < 64 * 64; i += 256) {
    const int64_t r = r0 + i / 64, q = q0 + i % 64;
    s[i / 64][i % 64] = r < a.R && q < a.Q ? (uint16_t)f2bf(a.W[r * a.Q + q]) : (uint16_t)0;
  }
  __syncthreads();
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, p = lane % 16, g = lane / 16;
  // four blocks of 16 n x two of 32 k, each way
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    const int blk = wave, kb = f, n = 16 * blk + perm_n(p), k = 32 * kb + 8 * g;
    if (q0 + 16 * blk < a.nr) {
      const uint4 v = make_uint4(pair(s[k][n], s[k + 1][n]), pair(s[k + 2][n], s[k + 3][n]),
                                 pair(s[k + 4][n], s[k + 5][n]), pair(s[k + 6][n], s[k + 7][n]));
      a.kr[(((q0 / 16 + blk) * a.nmul + a.nadd) * a.kr_kb + r0 / 32 + kb) * 64 + lane] = v;
    }
    if (a.kc && r0 + 16 * blk < a.nc)
      a.kc[((r0 / 16 + blk) * a.kc_kb + (a.koff + q0) / 32 + kb) * 64 + lane] =
          *reinterpret_cast<const uint4*>(&s[n][k]);
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

// act(g) and, with D, act'(g).  The distribution function of GELU: for an fp32
// state half of the complementary error function at -g / sqrt 2, which keeps its
// relative accuracy in the lower tail; for a bf16 state formula 7.1.26 of
// Abramowitz and Stegun, Handbook of Mathematical Functions:
//   1 - erf(x) = (a1 t + .. + a5 t^5) exp(-x^2),  t = 1 / (1 + p x),  x >= 0,
// to 1.5e-7, with x = |g| / sqrt 2: evaluated in fp32 the distribution is within
// 2^-21 (of 1: 6e-5 of the value at g = -3, 1.7e-3 at -5), below the rounding
// of h where a sum of them counts, in a dozen instructions that share the
// exponential with the density (erff is about eighty, and an epilogue has nothing
// to hide them behind: T = 8192, C = 4096, H = 11008 forward 1827 us with it,
// 1788 so).
template <bool D, typename TS>
__device__ __forceinline__ float act_of(int act, float g, float& d) {
  if (act == XHC_ACT_SILU) {
    const float e = __builtin_amdgcn_rcpf(1.0f + __expf(-g)), a = g * e;
    if (D) d = fmaf(a, 1.0f - e, e);
    return a;
  }
  float e, x;
  if (sizeof(TS) == 4) {
    e = 0.5f * erfcf(-0.70710678118654752f * g);
    if (D) x = __expf(-0.5f * g * g);
  } else {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752f, fabsf(g), 1.0f));
    x = __expf(-0.5f * g * g);
    float q = fmaf(t, 1.061405429f, -1.453152027f);
    q = fmaf(t, q, 1.421413741f);
    q = fmaf(t, q, -0.284496736f);
    q = fmaf(t, q, 0.254829592f);
    q *= 0.5f * t * x;
    e = g < 0.f ? q : 1.0f - q;
  }
  if (D) d = fmaf(g * x, 0.39894228040143268f, e);
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

// W = 4 or 8 consecutive values of the state dtype
template <int W>
__device__ __forceinline__ void store_vec(uint16_t* p, const float (&f)[W]) {
  if constexpr (W == 8)
    Vec8<uint16_t>::store(p, f);
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2bf(f[0], f[1]), pack2bf(f[2], f[3]));
}
template <int W>
__device__ __forceinline__ void store_vec(float* p, const float (&f)[W]) {
#pragma unroll
  for (int i = 0; i < W; i += 4)
    *reinterpret_cast<float4*>(p + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
}
template <int W>
__device__ __forceinline__ void load_vec(const uint16_t* p, float (&f)[W]) {
  if constexpr (W == 8) {
    Vec8<uint16_t>::load(p, f);
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    f[0] = bf_lo(v.x), f[1] = bf_hi(v.x), f[2] = bf_lo(v.y), f[3] = bf_hi(v.y);
  }
}
template <int W>
__device__ __forceinline__ void load_vec(const float* p, float (&f)[W]) {
#pragma unroll
  for (int i = 0; i < W; i += 4) {
    const float4 v = *reinterpret_cast<const float4*>(p + i);
    f[i] = v.x, f[i + 1] = v.y, f[i + 2] = v.z, f[i + 3] = v.w;
  }
}

// values as the operand of a later product: bf16, or the three parts
template <typename TS, int W>
__device__ __forceinline__ void store_operand(uint16_t* p, int64_t plane, const float (&f)[W]) {
  if constexpr (sizeof(TS) == 2) {
    store_vec<W>(p, f);
  } else {
    float v[3][W];
#pragma unroll
    for (int e = 0; e < W; ++e) {
      float q[3];
      split3(f[e], q);
      v[0][e] = q[0], v[1][e] = q[1], v[2][e] = q[2];
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) store_vec<W>(p + i * plane, v[i]);
  }
}

// g and u as they are saved.  fp32 state: fp32.  bf16 state: 24 bits, the upper
// 16 of the fp32 value in one plane and the next 8 in another, the rest cut off
// (less than 2^-15 of the value; in bf16 alone their rounding would double the
// error of dx and of the weight gradients, which is otherwise that of rounding
// dg and du and of their own).
template <typename TS> struct Saved;
template <> struct Saved<float> {
  float* p;
  int64_t n;           // elements of g, in fragments
  template <int W> struct Raw { float f[W]; };
  template <int W> __device__ __forceinline__ void store(int which, int64_t i, const float (&f)[W]) const {
    store_vec<W>(p + which * n + i, f);
  }
  template <int W> __device__ __forceinline__ void load(int which, int64_t i, Raw<W>& r) const {
    load_vec<W>(p + which * n + i, r.f);
  }
  template <int W> static __device__ __forceinline__ void unpack(const Raw<W>& r, float (&f)[W]) {
#pragma unroll
    for (int e = 0; e < W; ++e) f[e] = r.f[e];
  }
};
template <> struct Saved<uint16_t> {
  uint16_t* p;         // upper halves of g and u, then bytes of both
  int64_t n;
  template <int W> struct Raw { uint32_t hi[W / 2], lo[W / 4]; };
  template <int W> __device__ __forceinline__ void store(int which, int64_t i, const float (&f)[W]) const {
    uint32_t hi[W / 2], lo[W / 4];
#pragma unroll
    for (int e = 0; e < W; e += 4) {
      uint32_t u[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) u[x] = __float_as_uint(f[e + x]);
      hi[e / 2] = __builtin_amdgcn_perm(u[1], u[0], 0x07060302);
      hi[e / 2 + 1] = __builtin_amdgcn_perm(u[3], u[2], 0x07060302);
      const uint32_t a = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0501), b = __builtin_amdgcn_perm(u[3], u[2], 0x05010c0c);
      lo[e / 4] = a | b;
    }
    uint16_t* ph = p + which * n + i;
    uint8_t* pl = reinterpret_cast<uint8_t*>(p + 2 * n) + which * n + i;
    if constexpr (W == 8) {
      *reinterpret_cast<uint4*>(ph) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint2*>(pl) = make_uint2(lo[0], lo[1]);
    } else {
      *reinterpret_cast<uint2*>(ph) = make_uint2(hi[0], hi[1]);
      *reinterpret_cast<uint32_t*>(pl) = lo[0];
    }
  }
  template <int W> __device__ __forceinline__ void load(int which, int64_t i, Raw<W>& r) const {
    const uint16_t* ph = p + which * n + i;
    const uint8_t* pl = reinterpret_cast<const uint8_t*>(p + 2 * n) + which * n + i;
    if constexpr (W == 8) {
      const uint4 a = *reinterpret_cast<const uint4*>(ph);
      const uint2 b = *reinterpret_cast<const uint2*>(pl);
      r.hi[0] = a.x, r.hi[1] = a.y, r.hi[2] = a.z, r.hi[3] = a.w, r.lo[0] = b.x, r.lo[1] = b.y;
    } else {
      const uint2 a = *reinterpret_cast<const uint2*>(ph);
      r.hi[0] = a.x, r.hi[1] = a.y, r.lo[0] = *reinterpret_cast<const uint32_t*>(pl);
    }
  }
  template <int W> static __device__ __forceinline__ void unpack(const Raw<W>& r, float (&f)[W]) {
#pragma unroll
    for (int e = 0; e < W; ++e)     // bytes 0, lo, hi, hi
      f[e] = __uint_as_float(__builtin_amdgcn_perm(r.hi[e / 2], r.lo[e / 4],
                                                   (e % 2 ? 0x0706000cu : 0x0504000cu) + (uint32_t)(e % 4) * 0x100u));
  }
};

// Rows [T, C] into fragments, one wave a fragment; rows up to a whole block and
// columns up to 64 are zero.  Bound by HBM:
// each element read once, written once.
template <typename TS>
__global__ __launch_bounds__(256) void k_ffn_arrange(const TS* __restrict__ x, const TS* __restrict__ x2, int64_t T,
                                                     int C, int64_t kb, int64_t frags, uint16_t* __restrict__ out,
                                                     uint16_t* __restrict__ out2) {
  if (blockIdx.y) {
    x = x2;
    out = out2;
  }
  const int64_t f = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  const int lane = threadIdx.x % 64;
  if (f >= frags) return;
  const int64_t t = f / kb * 16 + lane % 16;
  const int c = (int)(f % kb) * 32 + lane / 16 * 8;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (t < T && c < C) Vec8<TS>::load(x + t * C + c, v);
  store_operand<TS, 8>(out + f * 512 + lane * 8, frags * 512, v);
}

// ---------------------------------------------------------------- epilogues

// sums of a token past the last: zero, whatever the weights hold
template <int W>
__device__ __forceinline__ void clear(float (&v)[W], float (&w)[W]) {
#pragma unroll
  for (int x = 0; x < W; ++x) v[x] = w[x] = 0.f;
}

// finish is called for the tokens t < rows (whole blocks of 16) and columns c <
// cols (whole blocks of 64); past T the sums are zero.  What it reads comes
// through fetch, some calls ahead.  Where the values lie in fragments is given
// as an offset (at), which the caller has without a division: between two calls
// it grows by constants.  Without that and the byte permutes, 128 values of
// dg, du and h per lane cost 35 us a tile of 256 x 256, a third of its products.
struct Nothing {};
struct Place {
  int64_t t, c;
  int64_t at;          // frag_at(t, c, cols / 32)
};
__device__ __forceinline__ Place place_of(int64_t t, int64_t c, int64_t cols) {
  return Place{t, c, frag_at(t, c, cols / 32)};
}

// h from g and u (W columns of one token); g and u saved where wanted
template <typename TS>
struct EpiUp {
  static constexpr bool kTwo = true;
  static constexpr int kParts = sizeof(TS) == 2 ? 1 : 3;   // of an activation as an operand
  int64_t T, rows;
  int H, cols;           // cols: Hp
  int act;
  uint16_t* h;
  Saved<TS> saved;     // p null: not wanted
  template <int W> using Pre = Nothing;
  template <int W> __device__ __forceinline__ Nothing fetch(const Place&) const { return Nothing{}; }
  template <int W>
  __device__ __forceinline__ void finish(const Place& p, const float (&g)[W], const float (&u)[W],
                                         const Nothing&) const {
    float f[W];
#pragma unroll
    for (int e = 0; e < W; ++e) {
      float d;
      f[e] = act_of<false, TS>(act, g[e], d) * u[e];
    }
    if (p.c + W > H) {
#pragma unroll
      for (int e = 0; e < W; ++e) f[e] = p.c + e < H ? f[e] : 0.f;
    }
    store_operand<TS, W>(h + p.at, rows * cols, f);
    if (saved.p) {
      saved.template store<W>(0, p.at, g);
      saved.template store<W>(1, p.at, u);
    }
  }
};

// F or dx
template <typename TS>
struct EpiOut {
  static constexpr bool kTwo = false;
  static constexpr int kParts = sizeof(TS) == 2 ? 1 : 3;
  int64_t T, rows;
  int cols;
  TS* out;
  template <int W> using Pre = Nothing;
  template <int W> __device__ __forceinline__ Nothing fetch(const Place&) const { return Nothing{}; }
  template <int W>
  __device__ __forceinline__ void finish(const Place& p, const float (&v)[W], const float (&)[W],
                                         const Nothing&) const {
    if (p.t < T) store_vec<W>(out + p.t * cols + p.c, v);
  }
};

// dg, du and h again from dh and the saved g and u
template <typename TS>
struct EpiGate {
  static constexpr bool kTwo = false;
  static constexpr int kParts = sizeof(TS) == 2 ? 1 : 3;
  int64_t T, rows;
  int H, cols;           // cols: Hp
  int act;
  Saved<TS> saved;
  uint16_t *dgu, *h;   // 2 Hp and Hp columns
  template <int W> struct Pre { typename Saved<TS>::template Raw<W> g, u; };
  template <int W> __device__ __forceinline__ Pre<W> fetch(const Place& p) const {
    Pre<W> r;
    saved.template load<W>(0, p.at, r.g);
    saved.template load<W>(1, p.at, r.u);
    return r;
  }
  template <int W>
  __device__ __forceinline__ void finish(const Place& p, const float (&dh)[W], const float (&)[W],
                                         const Pre<W>& r) const {
    float g[W], u[W], f[W], dg[W], du[W];
    Saved<TS>::unpack(r.g, g);
    Saved<TS>::unpack(r.u, u);
#pragma unroll
    for (int e = 0; e < W; ++e) {
      float d;
      const float a = act_of<true, TS>(act, g[e], d);
      f[e] = a * u[e];
      dg[e] = dh[e] * u[e] * d;
      du[e] = dh[e] * a;
    }
    if (p.c + W > H) {
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (p.c + e >= H) f[e] = dg[e] = du[e] = 0.f;
    }
    // a row block of dg and du is twice as long: its blocks before this one's, again
    const int64_t at = p.at + (p.t & ~(int64_t)15) * cols;
    store_operand<TS, W>(dgu + at, rows * 2 * cols, dg);
    store_operand<TS, W>(dgu + at + 16 * cols, rows * 2 * cols, du);
    store_operand<TS, W>(h + p.at, rows * cols, f);
  }
};

// weight gradients: row m, columns n of out[n / nsplit]
template <typename TS>
struct EpiWeight {
  int64_t M, N;        // rows, columns of the product
  int64_t ncols;       // columns of one output
  int64_t nsplit;      // product columns of the first
  TS *out0, *out1;
  __device__ __forceinline__ void finish(int64_t m, int64_t n, const float (&v)[8]) const {
    TS* o = out0;
    if (n >= nsplit) {
      n -= nsplit;
      o = out1;
    }
    o += m * ncols + n;
    if (ncols % 8 == 0) {          // n too: whole groups of eight, aligned
      if (n < ncols) store_vec<8>(o, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (n + e < ncols) put1(o + e, v[e]);
    }
  }
  static __device__ __forceinline__ void put1(uint16_t* p, float v) { *p = (uint16_t)f2bf(v); }
  static __device__ __forceinline__ void put1(float* p, float v) { *p = v; }
};

// ---------------------------------------------------------------- products

// activations [t, k] times packed weights; part: the sums of a part of k, [part][rows][cols (x 2)]
template <class S, class Epi>
__global__ __launch_bounds__(64 * S::NW) void k_ffn_rows(const GemmArgs a, const Epi e, float* __restrict__ part) {
  __shared__ __align__(1024) unsigned char lds[S::kLds];
  gemm_tile<FragTile, FragTile, S>(a, lds, [&](f32x16 (&acc)[S::FN][S::FT], int64_t n0, int64_t t0, int lane) {
    // 32 tokens by 16 columns at a time, fetched some ahead
    constexpr int NB = S::FN * (Epi::kTwo ? 1 : 2), ALL = S::FT * NB, AHEAD = Epi::kParts == 1 ? 4 : 2;
    const bool whole = gridDim.y == 1;
    const Place p0 = place_of(t0 + lane % 32, (Epi::kTwo ? n0 / 2 : n0) + lane / 32 * 8, e.cols);
    const int64_t step = e.cols * 32;             // 32 tokens on, in fragments
    const auto place = [&](int q) {               // columns start at a block of 32
      return Place{p0.t + q / NB * 32, p0.c + q % NB * 16, p0.at + q / NB * step + (q % NB / 2 * 512 + q % 2 * 256)};
    };
    typename Epi::template Pre<8> pre[AHEAD];
    const auto inside = [&](const Place& p) { return p.t < e.rows && p.c < e.cols; };
    const auto fetch = [&](int q) {
      if (whole && inside(place(q))) pre[q % AHEAD] = e.template fetch<8>(place(q));
    };
#pragma unroll
    for (int q = 0; q < AHEAD - 1; ++q) fetch(q);
    // unrolled by hand: with EpiGate<float> it is more than the compiler unrolls, and
    // sums indexed in a loop lie in scratch memory (T = 2048, C = 2560, H = 6912 dh
    // 3990 us, 268 so)
    unroll<ALL>([&](auto qc) {
      constexpr int q = qc.value, j = q / NB, i = q % NB;
      if constexpr (q + AHEAD - 1 < ALL) fetch(q + AHEAD - 1);
      const Place p = place(q);
      if (!inside(p)) return;
      float v[8], w[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        if constexpr (Epi::kTwo) {
          v[x] = acc[i][j][x];
          w[x] = acc[i][j][8 + x];
        } else {
          v[x] = acc[i / 2][j][i % 2 * 8 + x];
          w[x] = 0.f;
        }
      }
      if (p.t >= e.T) clear<8>(v, w);
      if (whole) {
        e.template finish<8>(p, v, w, pre[q % AHEAD]);
      } else {
        float* to = part + ((int64_t)blockIdx.y * e.rows + p.t) * e.cols * (Epi::kTwo ? 2 : 1) + p.c;
        Vec8<float>::store(to, v);
        if (Epi::kTwo) Vec8<float>::store(to + e.cols, w);
      }
    });
  });
}

// eight columns of the parts of k added in order, four parts on the way (eleven
// one after another, T = 96, C = 256: 5.6 us, 4.0 so)
__device__ __forceinline__ void add_parts(const float* p, int64_t stride, int parts, float (&v)[8]) {
  constexpr int AHEAD = 4;
  for (int i = 0; i < parts; i += AHEAD, p += AHEAD * stride) {
    float f[AHEAD][8];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (i + u < parts) Vec8<float>::load(p + u * stride, f[u]);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (i + u < parts) {
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] += f[u][x];
      }
  }
}

// the parts joined, then the epilogue
template <class Epi>
__global__ __launch_bounds__(256) void k_ffn_rows_join(const Epi e, const float* __restrict__ part, int parts) {
  const int64_t g = e.cols / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t t = i / g, c = i % g * 8, ld = (int64_t)e.cols * (Epi::kTwo ? 2 : 1);
  if (t >= e.rows) return;
  const Place at = place_of(t, c, e.cols);
  const auto pre = e.template fetch<8>(at);
  float v[8] = {}, w[8] = {};
  add_parts(part + t * ld + c, e.rows * ld, parts, v);
  if (Epi::kTwo) add_parts(part + t * ld + c + e.cols, e.rows * ld, parts, w);
  e.template finish<8>(at, v, w, pre);
}

// Few tokens (up to 16 for each of MB blocks): bound by the weights' bytes, which
// go from memory straight to registers, a fragment (1 KiB) a load.  A workgroup
// takes FR blocks of 16 n, its waves a part of k each, and keeps two sets of U k
// blocks per wave in flight, one under way while the other is multiplied: 128
// KiB of weights up to 16 tokens (64 with three-part activations), 32 to 128
// beyond, where the activations take registers.  The waves' sums are added
// through LDS in order.  Tokens past the last read it again.
struct FewArgs {
  const uint4* w;      // packed
  int64_t wkb;         // its k blocks
  int kb;              // k blocks of the activations
  const uint16_t* x;   // rows [T, ldx] (ldx > 0) or fragments; one or three planes
  int64_t ldx, plane;  // elements
  int T;
};
template <int FR, int MB, int NW, int U, class Epi>
__global__ __launch_bounds__(64 * NW) void k_ffn_few(const FewArgs a, const Epi e) {
  constexpr int P = Epi::kParts, PER = Epi::kTwo ? 2 : 1;
  static_assert(FR % PER == 0, "gate and up together");
  __shared__ f32x4 red[NW][FR * MB][64];
  // wave from a scalar register: a matrix instruction heeds no lane mask, so
  // what it runs under has to be a real branch
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint4* w = a.w + (int64_t)blockIdx.x * FR * a.wkb * 64 + lane;
  const uint16_t* x[MB];
  const int xk = a.ldx ? 32 : 512;       // elements between k blocks
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    const int t = m * 16 + lane % 16 < a.T ? m * 16 + lane % 16 : a.T - 1;
    x[m] = a.x + (a.ldx ? t * a.ldx + lane / 16 * 8 : frag_at(t, lane / 16 * 8, a.kb));
  }
  f32x4 acc[FR][MB];
#pragma unroll
  for (int f = 0; f < FR; ++f)
#pragma unroll
    for (int m = 0; m < MB; ++m) acc[f][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int k0 = (int)((int64_t)a.kb * wave / NW), k1 = (int)((int64_t)a.kb * (wave + 1) / NW);
  uint4 wr[2][U][FR], xr[2][U][MB][P];
  // past the part's end the last block again, whose products are left out
  auto load = [&](int b, int k) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kk = k + u < k1 ? k + u : k1 - 1;
#pragma unroll
      for (int f = 0; f < FR; ++f) wr[b][u][f] = w[(f * a.wkb + kk) * 64];
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int p = 0; p < P; ++p)
          xr[b][u][m][p] = *reinterpret_cast<const uint4*>(x[m] + p * a.plane + (int64_t)kk * xk);
    }
  };
  auto multiply = [&](int b, int k) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k + u < k1) {
#pragma unroll
        for (int p = P - 1; p >= 0; --p)
#pragma unroll
          for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int f = 0; f < FR; ++f) acc[f][m] = mfma_16x16x32(wr[b][u][f], xr[b][u][m][p], acc[f][m]);
      }
    }
  };
  if (k0 < k1) {
    load(0, k0);
    for (int k = k0; k < k1; k += 2 * U) {
      if (k + U < k1) load(1, k + U);
      multiply(0, k);
      if (k + U < k1) {
        if (k + 2 * U < k1) load(0, k + 2 * U);
        multiply(1, k + U);
      }
    }
  }
#pragma unroll
  for (int f = 0; f < FR; ++f)
#pragma unroll
    for (int m = 0; m < MB; ++m) red[wave][f * MB + m][lane] = acc[f][m];
  __syncthreads();
  // a wave finishes every NW-th of the (block, 16 tokens) pairs
  for (int i = wave; i < FR / PER * MB; i += NW) {
    const int f = i / MB * PER, m = i % MB, t = m * 16 + lane % 16;
    float v[4], u[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = u[c] = 0.f;
    for (int n = 0; n < NW; ++n) {
      const f32x4 r = red[n][f * MB + m][lane];
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] += r[c];
      if (Epi::kTwo) {
        const f32x4 s = red[n][(f + 1) * MB + m][lane];
#pragma unroll
        for (int c = 0; c < 4; ++c) u[c] += s[c];
      }
    }
    const int q = lane / 16;                               // rows 4 q .. + 4 of the block
    const int64_t c = ((int64_t)blockIdx.x * FR + f) / PER * 16 + perm_n(4 * q);
    if (t >= a.T) clear<4>(v, u);
    if (t < e.rows && c < e.cols) {
      const Place p = place_of(t, c, e.cols);
      e.template finish<4>(p, v, u, e.template fetch<4>(p));
    }
  }
}

// weight gradients: k is the token on both sides; part: [part][M][N]
template <class S, class Epi>
__global__ __launch_bounds__(64 * S::NW) void k_ffn_cols(const GemmArgs a, const Epi e, float* __restrict__ part) {
  __shared__ __align__(1024) unsigned char lds[S::kLds];
  gemm_tile<ColTilePerm, ColTile, S>(a, lds, [&](f32x16 (&acc)[S::FN][S::FT], int64_t n0, int64_t t0, int lane) {
#pragma unroll
    for (int j = 0; j < S::FT; ++j) {
      const int64_t m = t0 + j * 32 + lane % 32;
      if (m >= e.M) continue;
#pragma unroll
      for (int i = 0; i < S::FN * 2; ++i) {
        const int64_t n = n0 + i * 16 + lane / 32 * 8;
        if (n >= e.N) continue;
        float v[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] = acc[i / 2][j][i % 2 * 8 + x];
        if (gridDim.y > 1)
          Vec8<float>::store(part + ((int64_t)blockIdx.y * e.M + m) * e.N + n, v);
        else
          e.finish(m, n, v);
      }
    }
  });
}

template <class Epi>
__global__ __launch_bounds__(256) void k_ffn_cols_join(const Epi e, const float* __restrict__ part, int parts) {
  const int64_t g = e.N / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t m = i / g, n = i % g * 8;
  if (m >= e.M) return;
  float v[8] = {};
  add_parts(part + m * e.N + n, e.M * e.N, parts, v);
  e.finish(m, n, v);
}

// ---------------------------------------------------------------- host side

// Rings of 128 KiB in LDS, or 80 and 64 where two workgroups share a CU.  (In us,
// T = 8192, C = 4096, H = 11008: four stages of 32 k or two of 64 in a large
// tile up 1252 or 1293, dW_gate and dW_up 1249 or 1309; T = 512, C = 2560, H =
// 6912: five of 32 or two of 64 in a small one dx 120 or 176, dW_gate and dW_up
// 63 or 58.)
using Large = Shape<2, 4, 4, 2, 1, 4>;
using SmallRows = Shape<2, 2, 2, 2, 1, 5>;
using SmallCols = Shape<2, 2, 2, 2, 2, 2>;
// 128 n by 64 tokens
using Narrow = Shape<2, 1, 2, 2, 1, 6>;
constexpr int64_t kNarrow = 64;
// 64 by 64: four times the workgroups and a quarter of the epilogue's values per
// lane, which count where a product is short (T = 96, C = 256, H = 683 forward
// and backward 82 us without these tiles, 62 with them)
using TinyRows = Shape<1, 1, 2, 2, 1, 6>;
using TinyCols = Shape<1, 1, 2, 2, 2, 3>;
constexpr int64_t kTiny = 32;          // their mark in a plan

// How a product runs: its tile and the parts that k is cut into.
struct Plan {
  int64_t tile, gn, gt, ksteps, per;   // tile 0: k_ffn_few; per: stages of a part
  int64_t rest;                        // large tiles computed as four small ones each, at the end
  int64_t rest_ksteps;                 // their stages
  int nseg, parts;
};
// Tiles of 256 x 256 (a workgroup per CU), 128 x 128 (two) or 64 x 64 (three),
// with k in parts where there are few of them; by an estimate of the time in us.
// Measured per 32 k and round: a large tile 0.8 on a full chip, below half of it
// 0.6 (power); small ones 0.57, 0.5 where not every CU has two, 0.3 where none
// has; tiny ones 0.35, 0.25 and 0.2 with three, two and one.  Parts cost a write and a read of fp32 sums and a launch: T = 512, C =
// 2560, H = 6912 dx (80 small tiles of 432 steps) 242 us with large tiles, 120
// with small ones, 66 in 4 parts; T = 2048 (80 large tiles of 432) backward 527
// without parts of large tiles, 487 with them.  A rest of small tiles: T = 4096,
// C = 2560, H = 6912 forward 450 -> 437, backward 977 -> 926.  An fp32 state's
// epilogue taken as long as others: T = 1024, C = 1024, H = 2816 backward 260,
// 248 so.  Tiny ones: C =
// 1024, H = 2816 T = 200 43 -> 34 and 61 -> 51, T = 1500 69 -> 65 and 111 -> 110.
// `narrow` takes 128 x 64 alone: it is reached with large weights, whose tiny
// tiles read the tokens twice as often (T = 64, C = 4096, H = 11008 forward 120,
// 112 so).
Plan plan_product(int64_t n, int64_t t, int64_t k, int nseg, int stage128, int64_t out, bool narrow = false) {
  const auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  Plan best{};
  double least = 0;
  // large tiles, with a rest of small ones, small ones, tiny ones
  for (int kind = narrow ? 2 : 0; kind < (narrow ? 3 : 4); ++kind) {
    Plan p{};
    const int64_t tile = p.tile = kind < 2 ? 256 : kind == 3 ? kTiny : narrow ? kNarrow : 128;
    p.gn = up(n, kind == 3 ? 64 : std::max<int64_t>(tile, 128));
    p.gt = up(t, kind == 3 ? 64 : tile);
    p.nseg = nseg;
    const int stage = tile == 256 ? 32 : stage128;
    p.ksteps = std::max<int64_t>(1, up(k, stage));   // no tokens: one stage of zeros
    p.rest_ksteps = std::max<int64_t>(1, up(k, stage128));
    const int64_t steps = p.ksteps * nseg, tiles = p.gn * p.gt;
    for (int parts = 1; parts <= (kind == 1 ? 1 : kind == 0 ? 8 : 32); ++parts) {
      p.per = up(steps, parts);
      p.parts = (int)up(steps, p.per);
      if (p.parts != parts) continue;
      const int64_t w = tiles * parts;
      double rounds;
      if (tile == 256) {
        // a last round of few large tiles as small ones, in a launch of its own
        p.rest = kind == 1 && w > 256 && w % 256 <= 128 ? w % 256 : 0;
        if (kind == 1 && p.rest == 0) continue;
        rounds = w <= 128 ? 0.6 : 0.8 * up(w - p.rest, 256) + (p.rest == 0 ? 0 : p.rest <= 64 ? 0.3 : 0.57);
      } else if (kind == 3) {
        const int64_t rest = w % 768;
        rounds = 0.35 * (w / 768) + (rest == 0 ? 0 : rest <= 256 ? 0.2 : rest <= 512 ? 0.25 : 0.35);
      } else {
        const int64_t rest = w % 512;
        rounds = 0.57 * (w / 512) + (rest == 0 ? 0 : rest <= 256 ? 0.3 : 0.5);
      }
      const double epilogue = nseg == 3 ? 8 : 3;   // three-part activations: many values to write
      double us = rounds * p.per * (stage / 32) + (kind == 3 ? epilogue / 4 * up(w, 768) : epilogue);
      if (p.rest) us += 8;
      if (parts > 1) us += 4 + (double)parts * out * 8 / 3.5e6;
      if (least == 0 || us < least) {
        least = us;
        best = p;
      }
    }
  }
  return best;
}
size_t part_floats(const Plan& p, int64_t t, int64_t cols) { return p.parts > 1 ? (size_t)p.parts * t * cols : 0; }

GemmArgs args_of(const Plan& p, const Operand& n, const Operand& t, const Segments& seg) {
  return GemmArgs{n, t, seg, (int)p.ksteps, p.per, p.gn, p.gt, 0, 0};
}
// the launch of the rest
GemmArgs rest_of(const Plan& p, GemmArgs a) {
  a.ksteps = (int)p.rest_ksteps;
  a.steps_per_split = p.rest_ksteps * p.nseg;
  a.from = p.gn * p.gt - p.rest;
  a.quarters = 1;
  return a;
}
dim3 grid_of(const Plan& p) { return dim3((unsigned)(p.gn * p.gt - p.rest), (unsigned)p.parts); }

// Whether k_ffn_few runs (and reads an input of bf16 rows as it lies): up to 16
// tokens, up to 64 where the block is small.  Its workgroups read all activations
// again for every block or two of n, the tiles for every eight; but the tiles take
// two launches more, and three passes over the weights for an fp32 state.  us,
// forward, here and in tiles: C = 1024, H = 2816 T = 64 15 and 25, C = 2560, H =
// 6912 T = 32 33 and 39, T = 64 46 and 42; C = 4096, H = 11008 T = 32 81 and 72.
// fp32 state: C = 4096, H = 11008 T = 48 127 and 139, T = 64 153 and 145.
constexpr int64_t kFewMost = 64;
bool few_tokens(bool f32, int64_t T, int64_t C, int64_t H) {
  return T <= 16 || (T <= kFewMost && T * (C * H) <= (int64_t)5 << (f32 ? 29 : 27));
}
// all n blocks of the packed matrix a.n; ldx: elements between rows of the activations, 0 for fragments
template <class Epi>
hipError_t few(const GemmArgs& a, int64_t ldx, const Epi& e, hipStream_t s) {
  const FewArgs f{reinterpret_cast<const uint4*>(a.n.p), a.n.kb, (int)a.t.kb,
                  reinterpret_cast<const uint16_t*>(a.t.p), ldx, a.t.plane / 2, (int)e.T};
  // Blocks of 16 n per workgroup: one (with its gate's: two) up to 16 tokens and
  // where twice as many would leave more than half of the CUs idle; else twice as
  // many, as the activations' bytes count, too (us, forward, one and two: C =
  // 1024, H = 2816 T = 24 10.4 and 12.8, T = 64 15 and 17, C = 2560, H = 6528 T =
  // 48 46 and, gate and up in twos, 41).  Waves: 16, for the most loads in flight
  // where there are few blocks; fewer where their sums would not fit LDS (gate and
  // up), their fragments the registers that 16 waves have (three-part
  // activations), or where the parts of k would be short.
  constexpr bool two = Epi::kTwo, f32 = Epi::kParts == 3;
  constexpr int PER = two ? 2 : 1;
  const unsigned g1 = (unsigned)(a.n.rows / PER), g2 = g1 / 2;
  if (e.T <= 16) {
    constexpr int NW = two ? 8 : 16;
    k_ffn_few<PER, 1, NW, f32 ? 2 : 4, Epi><<<dim3(g1), dim3(64 * NW), 0, s>>>(f, e);
  } else if (g2 >= 128) {
    constexpr int NW32 = two ? 8 : 16, NW = two ? 4 : f32 ? 8 : 16, U = two && !f32 ? 2 : 1;
    if (e.T <= 32)
      k_ffn_few<2 * PER, 2, NW32, f32 ? 1 : 2, Epi><<<dim3(g2), dim3(64 * NW32), 0, s>>>(f, e);
    else if (e.T <= 48)
      k_ffn_few<2 * PER, 3, NW, U, Epi><<<dim3(g2), dim3(64 * NW), 0, s>>>(f, e);
    else
      k_ffn_few<2 * PER, 4, NW, U, Epi><<<dim3(g2), dim3(64 * NW), 0, s>>>(f, e);
  } else {
    constexpr int NW = two ? 4 : 8, U = f32 ? 1 : two ? 4 : 2;
    if (e.T <= 32)
      k_ffn_few<PER, 2, NW, f32 ? 2 : U, Epi><<<dim3(g1), dim3(64 * NW), 0, s>>>(f, e);
    else if (e.T <= 48)
      k_ffn_few<PER, 3, NW, U, Epi><<<dim3(g1), dim3(64 * NW), 0, s>>>(f, e);
    else
      k_ffn_few<PER, 4, NW, U, Epi><<<dim3(g1), dim3(64 * NW), 0, s>>>(f, e);
  }
  return hipGetLastError();
}

template <class Epi>
hipError_t rows(const Plan& p, const GemmArgs& a, const Epi& e, float* part, hipStream_t s, int64_t ldx = 0) {
  if (p.tile == 0) return few(a, ldx, e, s);
  if (p.tile == 256) {
    k_ffn_rows<Large, Epi><<<grid_of(p), dim3(64 * Large::NW), 0, s>>>(a, e, part);
    if (p.rest)
      k_ffn_rows<SmallRows, Epi>
          <<<dim3((unsigned)(4 * p.rest)), dim3(64 * SmallRows::NW), 0, s>>>(rest_of(p, a), e, part);
  } else if (p.tile == kTiny) {
    k_ffn_rows<TinyRows, Epi><<<grid_of(p), dim3(64 * TinyRows::NW), 0, s>>>(a, e, part);
  } else if (p.tile == kNarrow) {
    k_ffn_rows<Narrow, Epi><<<grid_of(p), dim3(64 * Narrow::NW), 0, s>>>(a, e, part);
  } else {
    k_ffn_rows<SmallRows, Epi><<<grid_of(p), dim3(64 * SmallRows::NW), 0, s>>>(a, e, part);
  }
  if (p.parts > 1) {
    const int64_t n = e.rows * (e.cols / 8);
    k_ffn_rows_join<Epi><<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(e, part, p.parts);
  }
  return hipGetLastError();
}
template <class Epi>
hipError_t cols(const Plan& p, const GemmArgs& a, const Epi& e, float* part, hipStream_t s) {
  if (p.tile == 256) {
    k_ffn_cols<Large, Epi><<<grid_of(p), dim3(64 * Large::NW), 0, s>>>(a, e, part);
    if (p.rest)
      k_ffn_cols<SmallCols, Epi>
          <<<dim3((unsigned)(4 * p.rest)), dim3(64 * SmallCols::NW), 0, s>>>(rest_of(p, a), e, part);
  } else if (p.tile == kTiny) {
    k_ffn_cols<TinyCols, Epi><<<grid_of(p), dim3(64 * TinyCols::NW), 0, s>>>(a, e, part);
  } else {
    k_ffn_cols<SmallCols, Epi><<<grid_of(p), dim3(64 * SmallCols::NW), 0, s>>>(a, e, part);
  }
  if (p.parts > 1) {
    const int64_t n = e.M * (e.N / 8);
    k_ffn_cols_join<Epi><<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(e, part, p.parts);
  }
  return hipGetLastError();
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// the workspace: x and dF in fragments, h, [dg|du], parts of k
struct Ws {
  Plan up, down, dh, dx, dwgu, dwd;
  int64_t rows;                  // tokens in whole blocks
  size_t x, dF, h, dgu, part, total;
  Ws(int state_dtype, int64_t T, int64_t C, int64_t H, bool bwd) {
    const Packed pk(C, H);
    const bool f32 = state_dtype == XHC_F32;
    const int P = f32 ? 3 : 1, ns = f32 ? 3 : 1, nw = f32 ? 6 : 1;
    rows = round_up(T, 16);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
      const size_t o = at;
      at += align256(bytes);
      return o;
    };
    x = take((size_t)P * rows * pk.Cp * 2);
    dF = take(bwd ? (size_t)P * rows * pk.Cp * 2 : 0);
    h = take((size_t)P * rows * pk.Hp * 2);
    dgu = take(bwd ? (size_t)P * rows * pk.Hp * 4 : 0);
    size_t most = 0;
    const auto product = [&](int64_t n, int64_t k) {       // of the tokens by packed weights
      if (few_tokens(f32, T, C, H)) return Plan{};
      const Plan p = plan_product(n, T, k, ns, 32, rows * n, T <= kNarrow);
      most = std::max(most, part_floats(p, rows, n));
      return p;
    };
    const auto weights = [&](int64_t n, int64_t m) {       // their gradients
      const Plan p = plan_product(n, m, T, nw, 64, n * m);
      most = std::max(most, part_floats(p, m, n));
      return p;
    };
    if (bwd) {
      dh = product(pk.Hp, pk.Cp);
      dx = product(C, 2 * pk.Hp);
      dwgu = weights(2 * pk.Hp, C);
      dwd = weights(C, H);
    } else {
      up = product(2 * pk.Hp, pk.Cp);
      down = product(C, pk.Hp);
    }
    part = take(most * sizeof(float));
    total = at;
  }
};

Operand weight(const void* p, int64_t nb, int64_t kb) { return Operand{p, 0, nb, kb}; }
Operand activation(const void* p, int64_t kb, int64_t tb) { return Operand{p, tb * kb * 1024, tb, kb}; }

// rows in fragments; x2: another tensor like x, or null
template <typename TS>
hipError_t arrange(const void* x, const void* x2, int64_t T, int64_t C, int64_t kb, void* out, void* out2,
                   hipStream_t s) {
  const int64_t frags = (T + 15) / 16 * kb;
  if (frags == 0) return hipSuccess;
  k_ffn_arrange<TS><<<dim3((unsigned)((frags + 3) / 4), x2 ? 2 : 1), dim3(256), 0, s>>>(
      reinterpret_cast<const TS*>(x), reinterpret_cast<const TS*>(x2), T, (int)C, kb, frags,
      reinterpret_cast<uint16_t*>(out), reinterpret_cast<uint16_t*>(out2));
  return hipGetLastError();
}

template <typename TS>
hipError_t ffn(int state_dtype, int64_t T, int64_t C, int64_t H, int act, const void* input, const void* packed,
               void* F, void* saved, void* workspace, hipStream_t s) {
  const Packed pk(C, H);
  const Ws w(state_dtype, T, C, H, false);
  const bool f32 = state_dtype == XHC_F32, direct = !f32 && few_tokens(f32, T, C, H);
  char* ws = reinterpret_cast<char*>(workspace);
  const char* pw = reinterpret_cast<const char*>(packed);
  const Segments seg = f32 ? segs_weights() : segs_bf16();
  const int64_t tb = w.rows / 16, kc = pk.Cp / 32, kh = pk.Hp / 32;
  float* part = reinterpret_cast<float*>(ws + w.part);
  uint16_t* h = reinterpret_cast<uint16_t*>(ws + w.h);
  hipError_t e = direct ? hipSuccess : arrange<TS>(input, nullptr, T, C, kc, ws + w.x, nullptr, s);
  const Operand ox = direct ? Operand{input, 0, tb, C / 32} : activation(ws + w.x, kc, tb);
  if (e == hipSuccess)
    e = rows(w.up, args_of(w.up, weight(pw + pk.up, pk.n32H * 4, kc), ox, seg),
             EpiUp<TS>{T, w.rows, (int)H, (int)pk.Hp, act, h,
                       Saved<TS>{reinterpret_cast<TS*>(saved), w.rows * pk.Hp}},
             part, s, direct ? C : 0);
  if (e == hipSuccess)
    e = rows(w.down, args_of(w.down, weight(pw + pk.down, pk.n32C * 2, kh), activation(h, kh, tb), seg),
             EpiOut<TS>{T, w.rows, (int)C, reinterpret_cast<TS*>(F)}, part, s);
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
  const int64_t tb = w.rows / 16, kc = pk.Cp / 32, kh = pk.Hp / 32;
  float* part = reinterpret_cast<float*>(ws + w.part);
  uint16_t *h = reinterpret_cast<uint16_t*>(ws + w.h), *dgu = reinterpret_cast<uint16_t*>(ws + w.dgu);
  hipError_t e = arrange<TS>(input, dF, T, C, kc, ws + w.x, ws + w.dF, s);
  const Operand ox = activation(ws + w.x, kc, tb), odf = activation(ws + w.dF, kc, tb);
  const Operand oh = activation(h, kh, tb), odgu = activation(dgu, 2 * kh, tb);
  if (e == hipSuccess && T > 0)
    e = rows(w.dh, args_of(w.dh, weight(pw + pk.dh, pk.n32H * 2, kc), odf, sw),
             EpiGate<TS>{T, w.rows, (int)H, (int)pk.Hp, act,
                         Saved<TS>{const_cast<TS*>(reinterpret_cast<const TS*>(saved)), w.rows * pk.Hp}, dgu, h},
             part, s);
  if (e == hipSuccess && T > 0)
    e = rows(w.dx, args_of(w.dx, weight(pw + pk.dx, pk.n32C * 2, 2 * kh), odgu, sw),
             EpiOut<TS>{T, w.rows, (int)C, reinterpret_cast<TS*>(d_input)}, part, s);
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
  return (size_t)2 * round_up(T, 16) * pad_k(H) * (state_dtype == XHC_F32 ? 4 : 3);
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
  PackAll all;
  for (int i = 0; i < 2; ++i)
    all.m[i] = PackArgs{i ? W_up : W_gate, C, H, at(p.up), p.Cp / 32, 2, i, with_bwd ? at(p.dx) : nullptr,
                        2 * p.Hp / 32, i * p.Hp, p.Hp, C};
  all.m[2] = PackArgs{W_down, H, C, at(p.down), p.Hp / 32, 1, 0, with_bwd ? at(p.dh) : nullptr, p.Cp / 32, 0, C, p.Hp};
  k_ffn_pack<<<dim3(th, tc, 3), dim3(256), 0, s>>>(all);
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
