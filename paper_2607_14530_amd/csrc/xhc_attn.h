// Building blocks of the attention kernels (gfx950).
//
// Every product is one of 32x32 blocks on matrix instructions with fp32 sums.
// A wave owns 32 columns (queries forward and for dq, keys for dk and dv), a
// lane one of them, l % 32; the other side comes from LDS tiles of 64 rows that
// the workgroup's waves share.  The order of an instruction's inner index is
// free as long as both operands agree on it, and that is used throughout:
//
//   row_frag   eight consecutive channels of one row: the operand whose rows the
//              block's rows are, of the products over channels
//   col_frag   eight rows of one channel, in the order in which a lane holds the
//              sums of such a product (rows 16 s + 8 (j / 4) + 4 (l / 32) + j % 4),
//              so that those, rounded, are the other operand as they lie: the
//              probabilities never leave their lane's registers
//
// With a bf16 state probabilities and the gradients of scores are rounded to bf16
// there, as the instructions take operands of one type: held in two halves each
// product of theirs would be two.  Outputs and gradients are then off by 0.0024 of
// their norm; their own rounding alone makes 0.0017.
//
// fp32 tensors use the 32x32x2 instruction eight times on the same eight
// elements, which takes their products in full at a sixteenth of the rate.
#pragma once

#include "xhc_ffn.h"

namespace xhc {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kTile = 64;                     // rows of an LDS tile
constexpr int kAttnWaves = 4;

struct Frag32 {
  float v[8];
};
template <typename TS> struct FragOf;
template <> struct FragOf<uint16_t> { using type = uint4; };
template <> struct FragOf<float> { using type = Frag32; };
template <typename TS> using Frag = typename FragOf<TS>::type;

__device__ __forceinline__ f32x16 mfma32(const uint4& a, const uint4& b, f32x16 c) { return mfma_32x32x16(a, b, c); }
__device__ __forceinline__ f32x16 mfma32(const Frag32& a, const Frag32& b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
  return c;
}

// sums 8 s .. 8 s + 7 of a block, as the operand that col_frag goes with
__device__ __forceinline__ void sums_frag(const f32x16& x, int s, uint4& f) {
  f = make_uint4(pack2bf(x[8 * s], x[8 * s + 1]), pack2bf(x[8 * s + 2], x[8 * s + 3]),
                 pack2bf(x[8 * s + 4], x[8 * s + 5]), pack2bf(x[8 * s + 6], x[8 * s + 7]));
}
__device__ __forceinline__ void sums_frag(const f32x16& x, int s, Frag32& f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) f.v[j] = x[8 * s + j];
}
// l and the sum of a fragment's elements, as they are in it
__device__ __forceinline__ float add_frag(const uint4& f, float l) {
  const bf16x2 one = __builtin_bit_cast(bf16x2, 0x3f803f80u);
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, f.x), one, l, false);
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, f.y), one, l, false);
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, f.z), one, l, false);
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, f.w), one, l, false);
}
__device__ __forceinline__ float add_frag(const Frag32& f, float l) {
#pragma unroll
  for (int j = 0; j < 8; ++j) l += f.v[j];
  return l;
}

__device__ __forceinline__ void load_frag(const uint16_t* p, uint4& f) { f = *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void load_frag(const float* p, Frag32& f) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f = Frag32{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}

// whether one of a 16-byte piece's elements is an infinity or NaN
template <typename TS> __device__ __forceinline__ bool not_finite(const uint4& w);
template <> __device__ __forceinline__ bool not_finite<uint16_t>(const uint4& w) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
    bad |= (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u;
  }
  return bad;
}
template <> __device__ __forceinline__ bool not_finite<float>(const uint4& w) {
  constexpr uint32_t e = 0x7f800000u;
  return (w.x & e) == e || (w.y & e) == e || (w.z & e) == e || (w.w & e) == e;
}

// lds_dma16 from a scalar base and an offset for each lane
__device__ __forceinline__ void lds_dma16_at(const void* base, uint32_t off, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(lds_addr)
               : "memory", "m0");
}

// A tile of kTile rows of D elements in LDS, in 16-byte pieces.  Piece c of row
// r lies at place c ^ turn(r), so that sixteen rows' pieces of one number, which
// row_frag reads at a time, and four rows' fours of pieces, which the transposing
// read takes, meet all 64 banks (turned for eight rows and pairs only, half of
// the LDS cycles were conflicts).  The copy leaves a run of 1 KiB where it
// puts it, so the pieces are turned on the way: each lane reads the piece that
// belongs to its place.
template <typename TS, int D, int NW = kAttnWaves>
struct Tile {
  static constexpr int kPieces = D * (int)sizeof(TS) / 16, kRowBytes = kPieces * 16, kBytes = kTile * kRowBytes;
  static constexpr int kCopies = kTile * kPieces / 64 / NW;
  static_assert(kTile * kPieces % (64 * NW) == 0 && kPieces % NW == 0, "whole copies, and rows, for every wave");
  static __device__ __forceinline__ int turn(int r) {
    if (kPieces % 16 == 0) return 4 * (r % 4) + r / 4 % 4;
    if (kPieces % 8 == 0) return 4 * (r / 2 % 2) + r / 4 % 4;
    return r / 4 % 4;
  }
  // Rows row0 .. of a tensor whose rows lie `stride` bytes apart, those behind
  // `last` as copies of it (what becomes of them is masked).  A copy's rows and
  // pieces follow from the wave's first copy's: by whole rows, which are added
  // to the scalar base, and by the turn, which changes with the row's number.
  static __device__ __forceinline__ void copy(const unsigned char* base, uint32_t stride, int row0, int last,
                                              uint32_t to, int wave, int lane) {
    if (row0 + kTile - 1 <= last) {
      base += (uint64_t)(uint32_t)row0 * stride;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const int at = (wave * kCopies + i) * 64;
        if constexpr (64 % kPieces == 0 && 16 % (64 / kPieces) == 0) {
          constexpr int R = 64 / kPieces;        // rows of a copy
          const int r = at / kPieces, x = lane / kPieces;        // (r: a multiple of R)
          const int c = lane % kPieces ^ turn(x) ^ turn(r % 16);
          static_assert(R <= 16, "turn(r + x) = turn(r) ^ turn(x) for x below R, r a multiple of it");
          lds_dma16_at(base + (uint64_t)(uint32_t)r * stride, (uint32_t)x * stride + c * 16, to + at * 16);
        } else {
          const int r = (at + lane) / kPieces, c = (at + lane) % kPieces ^ turn(r);
          lds_dma16_at(base, (uint32_t)r * stride + c * 16, to + at * 16);
        }
      }
      return;
    }
#pragma unroll 1
    for (int i = 0; i < kCopies; ++i) {
      const int at = (wave * kCopies + i) * 64 + lane, r = at / kPieces, c = at % kPieces ^ turn(r);
      const int t = row0 + r < last ? row0 + r : last;
      lds_dma16(base + ((uint64_t)(uint32_t)t * stride + c * 16),
                (uint32_t)__builtin_amdgcn_readfirstlane((int)to) + (wave * kCopies + i) * 1024);
    }
  }
  static __device__ __forceinline__ uint4& piece(unsigned char* s, int r, int c) {
    return *reinterpret_cast<uint4*>(s + r * kRowBytes + (c ^ turn(r)) * 16);
  }
  // channels 16 ks + 8 (lane / 32) .. of row 32 rb + lane % 32
  static __device__ __forceinline__ void row_frag(const unsigned char* s, int rb, int ks, int lane, uint4& f) {
    const int r = lane % 32;
    f = *reinterpret_cast<const uint4*>(s + (rb * 32 + r) * kRowBytes + ((2 * ks + lane / 32) ^ turn(r)) * 16);
  }
  static __device__ __forceinline__ void row_frag(const unsigned char* s, int rb, int ks, int lane, Frag32& f) {
    const int r = lane % 32, c = 4 * ks + 2 * (lane / 32);
    const unsigned char* p = s + (rb * 32 + r) * kRowBytes;
    const float4 a = *reinterpret_cast<const float4*>(p + (c ^ turn(r)) * 16);
    const float4 b = *reinterpret_cast<const float4*>(p + ((c + 1) ^ turn(r)) * 16);
    f = Frag32{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
  }
  // rows 16 s + 8 (j / 4) + 4 (lane / 32) + j % 4 of channel 32 f + lane % 32, j = 0 .. 7
  static __device__ __forceinline__ void col_frag(const unsigned char* s, int f, int st, int lane, uint4& out) {
    const int r = 4 * (lane / 32) + lane % 16 / 4, q = lane % 4;   // of this lane's read: a row, four channels
    const int c = 4 * f + 2 * (lane / 16 % 2) + q / 2;
    const unsigned char* p = s + (16 * st + r) * kRowBytes + q % 2 * 8;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (c ^ turn(r)) * 16));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * kRowBytes + (c ^ turn(r + 8)) * 16));
    const uint2 ua = __builtin_bit_cast(uint2, a), ub = __builtin_bit_cast(uint2, b);
    out = make_uint4(ua.x, ua.y, ub.x, ub.y);
  }
  static __device__ __forceinline__ void col_frag(const unsigned char* s, int f, int st, int lane, Frag32& out) {
    const int c = 8 * f + lane % 32 / 4;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 8 * (j / 4) + 4 * (lane / 32) + j % 4;
      out.v[j] = *reinterpret_cast<const float*>(s + (16 * st + r) * kRowBytes + (c ^ turn(r)) * 16 + lane % 4 * 4);
    }
  }
  // Rows that hold an infinity or NaN become zeros; they are the bits' ones.
  // A product over rows adds 0 times what lies in a row that its column does not
  // see, which has to be finite: so tiles that a mask cuts are looked over, and
  // for the columns that do see such a row the caller puts a NaN in the row's
  // place.  Called by all waves, each for the rows that its own copies brought:
  // so before the barrier that shows the tile to the others, and the bits with
  // it (a barrier of its own for them cost the forward of 8190 tokens in
  // documents, Hq = 16, D = 64, 1.2 of 49.8 us).
  static __device__ __forceinline__ void clean(unsigned char* s, uint64_t* bits, int wave, int lane) {
    constexpr int RW = kTile / NW;               // rows of a wave, NW lanes each
    const int r = wave * RW + lane / NW;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kPieces / NW; ++i) bad |= not_finite<TS>(piece(s, r, lane % NW + NW * i));
    const uint64_t all = __ballot(bad);
    constexpr uint64_t lanes = (1u << NW) - 1;
    uint32_t rows = 0;
    if (all) {
      for (int i = 0; i < RW; ++i) rows |= (uint32_t)((all >> (NW * i) & lanes) != 0) << i;
      if (rows >> (lane / NW) & 1) {
#pragma unroll
        for (int i = 0; i < kPieces / NW; ++i) piece(s, r, lane % NW + NW * i) = make_uint4(0, 0, 0, 0);
      }
    }
    if (lane == 0) {
      if constexpr (RW == 16)
        reinterpret_cast<uint16_t*>(bits)[wave] = (uint16_t)rows;
      else
        reinterpret_cast<uint8_t*>(bits)[wave] = (uint8_t)rows;
    }
  }
};

// The same lane, which the compiler does not know to be: what follows from it is
// formed where it is used, and not kept in registers over a loop.
__device__ __forceinline__ int again(int lane) {
  asm volatile("" : "+v"(lane));
  return lane & 63;
}

// Waits for all copies and loads of this wave.  (By the builtin: the compiler
// then knows that what it has loaded itself is there.  Not knowing, it waited
// in every turn of a loop for fragments loaded before it, and so for the copies
// that had just been sent.)
__device__ __forceinline__ void wait_loads() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt = 0, expcnt = 7, lgkmcnt = 15 (no wait)
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// Stands in a branch that the compiler is not to turn into selections.
__device__ __forceinline__ void branch_only() { __builtin_amdgcn_sched_barrier(0); }

// N products: use(i, fragment i), with the fragments of the next AHEAD on their
// way from LDS (its latency is that of some three products).  In this order,
// which the compiler is kept from changing, and before what other waves do.
template <int N, int AHEAD, typename F, class Read, class Use>
__device__ __forceinline__ void feed(Read&& read, Use&& use) {
  F f[AHEAD + 1];
  __builtin_amdgcn_s_setprio(1);
  __builtin_amdgcn_sched_barrier(0);
  unroll<(AHEAD < N ? AHEAD : N)>([&](auto i) { read(i, f[i.value]); });
  unroll<N>([&](auto i) {
    if constexpr (i.value + AHEAD < N) read(Int<i.value + AHEAD>{}, f[(i.value + AHEAD) % (AHEAD + 1)]);
    use(i, f[i.value % (AHEAD + 1)]);
    __builtin_amdgcn_sched_barrier(0);
  });
  __builtin_amdgcn_s_setprio(0);
}

// Step i's share of N pieces of work among STEPS steps.
template <int N, int STEPS, class I, class F> __device__ __forceinline__ void share(I, F&& f) {
  constexpr int each = (N + STEPS - 1) / STEPS, from = I::value * each;
  unroll<each>([&](auto x) {
    if constexpr (from + x.value < N) f(Int<from + x.value>{});
  });
}

// What an attention call is about, as its kernels take it.
struct AttnArgs {
  const void* qkv;          // [T][Hq + 2 Hkv][D]
  const int2* span;         // [T]: the first key that a token sees, and one behind the last; null: causal
  const float* slopes;      // [Hq] or null
  void* out;                // [T][Hq][D]
  float* lse;               // [Hq][Tp] or null: base-2 logarithms of the rows' sums
  uint16_t* low;            // [T][Hq][D], bf16 state: what out's rounding left, where lse is not null
  const void* dout;
  void* dqkv;
  const float* delta;       // [Hq][Tp]: of a backward
  const int* lo;            // [Tp], [Tp]: spans, cut to 0 .. T, 0 .. 0 for rows behind the last
  const int* hi;
  const int4* range;        // [Tp / kTile]: of a tile's rows that see keys, min lo, max hi; of all, max lo, min hi
  float* part;              // dk, dv of parts of a group's heads
  int64_t T, S, Tp;
  int Hq, Hkv, window;
  int parts, slices;        // of dk and dv: shares of a group's heads times slices of the queries
  int qslices;              // of dq: slices of the keys
  float scale, cap;
};

// keys that token t sees
__device__ __forceinline__ int2 span_of(const AttnArgs& a, int t) {
  if (t >= a.T) return make_int2(0, 0);
  if (a.span) {
    const int2 s = a.span[t];
    const int T = (int)a.T;
    return make_int2(min(max(s.x, 0), T), min(max(s.y, 0), T));
  }
  int lo = t - (int)((uint32_t)t % (uint32_t)a.S);       // (S <= T where there are tokens)
  if (a.window > 0 && t - a.window + 1 > lo) lo = t - a.window + 1;
  return make_int2(lo, t + 1);
}

// a value that all lanes have, in a scalar register
__device__ __forceinline__ float scalar(float x) {
  return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x)));
}

// A row's reference is a product that has been rounded.  A fused x mul - ref
// leaves of the row's largest score what that rounding took, up to 2^-24 of it:
// exp2 makes a weight of 15 of that at scores of 2^24, and an infinity at 2^32.
// Where a row's scores are far, above this (in units of log2 e; below, 2^-10 is
// left at most), its products are therefore rounded before the difference, which
// then is 0 for the largest.  The forward, its form over the cache and dq do so in
// a branch that a wave takes if one of its rows asks for it (and for those rows
// only: what a row gives does not depend on its neighbours); dk and dv, and the
// cache's tiles of 32 rows, whose registers leave no room for a branch, always.
// (T = 16384 in two sequences, Hq = 32, Hkv = 8, D = 128: forward 1105 -> 1112 us,
// backward 3750 -> 3757; always rounded, the forward took 4 % more.  8192 tokens in
// sequences of 512, Hq = 16, Hkv = 4, D = 64: forward 27.8 -> 28.0, backward 112 -> 114.7.)
constexpr float kFar = 16384.f;
__device__ __forceinline__ float rounded_diff(float x, float mul, float y) {
#pragma clang fp contract(off)
  const float p = x * mul;
  return p - y;
}

// Scores in units of log2 e (their softmax then takes exp2), of raw products x:
// (cap tanh(scale x / cap) - slope |i - j|) log2 e, or scale x log2 e for the first.
template <typename TS> struct Score {
  float mul, cap, slope;    // without a cap mul is scale log2 e; with one what tanh_of takes x with
  __device__ __forceinline__ void init(const AttnArgs& a, int head) {
    cap = scalar(a.cap * kLog2e);
    mul = scalar(a.cap > 0.f ? a.scale / a.cap * (sizeof(TS) == 2 ? 2.f * kLog2e : 1.f) : a.scale * kLog2e);
    slope = a.slopes ? scalar(a.slopes[head] * kLog2e) : 0.f;
  }
  // 1 / (1 + exp 2z), z = scale x / cap: tanh z = 1 - 2 of it.  Off by some 2^-23
  // of 1, where a bf16 product's factors are off by 2^-9 of it.
  __device__ __forceinline__ float share_of(float x) const {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * mul));
  }
  __device__ __forceinline__ float tanh_of(float x) const {
    if constexpr (sizeof(TS) == 2)
      return fmaf(-2.f, share_of(x), 1.f);
    else
      return tanhf(x * mul);
  }
  // tanh z and its derivative 1 - tanh^2 z = 4 e / (1 + e)^2, e = exp(-2 |z|), or
  // 4 r (1 - r) with r = 1 / (1 + exp 2 |z|).  Relative to itself either is as exact
  // next to the cap as elsewhere; 1 less the square of a rounded tanh is off by a
  // third of it at z = 8.5, and 0 from 9 on.  (Backward of T = 8192 in one
  // sequence, Hq = 32, Hkv = 8, D = 128, bf16, cap 30: 2490 us, 2460 with that
  // square; T = 777, Hq = 6, Hkv = 2, D = 96, fp32: 113 and 106.)
  __device__ __forceinline__ float tanh_of(float x, float& der) const {
    if constexpr (sizeof(TS) == 2) {
      const float r = share_of(fabsf(x));
      der = 4.f * fmaf(-r, r, r);
      return copysignf(fmaf(-2.f, r, 1.f), x);
    } else {
      const float e = expf(-2.f * fabsf(x * mul));
      der = 4.f * e / ((1.f + e) * (1.f + e));
      return tanhf(x * mul);
    }
  }
};

__device__ __forceinline__ float max_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// the row of sum r of a block, less 4 (lane / 32)
__host__ __device__ __forceinline__ constexpr int sum_row(int r) { return 8 * (r / 4) + r % 4; }

// NC of k_attn and k_attn_dq: two where there is less than a workgroup a CU
// (T = 777, Hq = 6, D = 96, fp32: 94 -> 68 us forward; at 512 workgroups, T =
// 2048, Hq = 32, D = 128, the extra copies cost more, 90 -> 95).
inline int attn_parts(int64_t T, int Hq) { return (T + 127) / 128 * Hq <= 256 ? 2 : 1; }

// least of the 32 lanes of a half wave, in all of them
__device__ __forceinline__ int half_min(int v) {
  v = min(v, __builtin_amdgcn_update_dpp(v, v, 0xB1, 0xF, 0xF, false));    // quad_perm 1,0,3,2
  v = min(v, __builtin_amdgcn_update_dpp(v, v, 0x4E, 0xF, 0xF, false));    // quad_perm 2,3,0,1
  v = min(v, __builtin_amdgcn_update_dpp(v, v, 0x141, 0xF, 0xF, false));   // row_half_mirror
  v = min(v, __builtin_amdgcn_update_dpp(v, v, 0x140, 0xF, 0xF, false));   // row_mirror
  const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  return min((int)r[0], (int)r[1]);
}

// The extremes of the spans of the workgroup's rows t0 .. t0 + rows - 1 (a
// lane's own: s, of row t0 + 32 RW ..): x min lo, y max hi of the rows that see
// keys (x >= y where none does), z max lo, w min hi of all.  Rows behind the
// last are left out.  own: x and y of the wave's rows, from row w0 on.
// Causal spans ascend, so that the first and the last row have all four.
__device__ __forceinline__ int4 attn_extremes(const AttnArgs& a, int t0, int rows, int w0, int2 s, bool row, int4* red,
                                              int wave, int lane, int2& own) {
  if (!a.span) {
    const int T1 = (int)a.T - 1, t1 = min(t0 + rows - 1, T1), w1 = min(w0 + 31, T1);
    const int2 first = span_of(a, t0), last = span_of(a, t1);
    own = w0 <= T1 ? make_int2(span_of(a, w0).x, w1 + 1) : make_int2(INT32_MAX, 0);
    return make_int4(first.x, last.y, last.x, first.y);
  }
  const bool some = row && s.x < s.y;
  const int x = half_min(some ? s.x : INT32_MAX), y = -half_min(some ? -s.y : 0),
            z = -half_min(row ? (some ? -s.x : -INT32_MAX) : 0), w = half_min(row ? (some ? s.y : 0) : INT32_MAX);
  own = make_int2(__builtin_amdgcn_readfirstlane(x), __builtin_amdgcn_readfirstlane(y));
  if (lane == 0) red[wave] = make_int4(x, y, z, w);
  __syncthreads();
  int4 e = red[0];
#pragma unroll
  for (int i = 1; i < kAttnWaves; ++i) {
    e.x = min(e.x, red[i].x);
    e.y = max(e.y, red[i].y);
    e.z = max(e.z, red[i].z);
    e.w = min(e.w, red[i].w);
  }
  return make_int4(__builtin_amdgcn_readfirstlane(e.x), __builtin_amdgcn_readfirstlane(e.y),
                   __builtin_amdgcn_readfirstlane(e.z), __builtin_amdgcn_readfirstlane(e.w));
}

// Sums of one 32-channel block of 32 tokens (a lane: token lane % 32, channels
// 8 i + 4 (lane / 32) + 0 .. 3) times m, to row p of the lane's token: the two
// halves exchange fours of channels, so that each writes runs of eight.  low:
// null, or where what the rounding leaves goes.
template <typename TS>
__device__ __forceinline__ void store_sums(const f32x16& x, float m, TS* p, bool row, int lane, TS* low = nullptr) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float f[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[8 * i + e] * m),
                                                      __float_as_uint(x[8 * i + 4 + e] * m), false, false);
      f[e] = __uint_as_float(r[0]);
      f[4 + e] = __uint_as_float(r[1]);
    }
    // the lower half now has channels 16 i + 0 .. 7, the upper 16 i + 8 .. 15
    const int at = 16 * i + 8 * (lane / 32);
    if (row) Vec8<TS>::store(p + at, f);
    if (sizeof(TS) == 2 && row && low) {
      float g[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = f[e];
      Vec8<TS>::round(g);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] -= g[e];
      Vec8<TS>::store(low + at, f);
    }
  }
}

// The rotation: pairs (a, b) -> (a c - b s, b c + a s), products and sums
// rounded one by one (no fused ones), so that the result is the formula's to
// the bit in fp32 whatever compiles it.
template <int N>
__device__ __forceinline__ void turn(float (&a)[N], float (&b)[N], const float* cs, float sign) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float c = cs[2 * i], s = cs[2 * i + 1] * sign;
    const float x = a[i] * c - b[i] * s, y = b[i] * c + a[i] * s;
    a[i] = x;
    b[i] = y;
  }
}

// Workgroup b's head and tile of rows, of `tiles` tiles and `heads` heads: an
// XCD (b % 8) takes heads of its own where they divide among the eight, so that
// its L2 keeps their keys and values, and later tiles, which see more, go first.
__device__ __forceinline__ void attn_place(int heads, int tiles, int& head, int& tile) {
  const uint32_t b = blockIdx.x;
  if (heads % 8 == 0) {
    const uint32_t mine = heads / 8, l = b / 8;
    head = (int)(b % 8 * mine + l % mine);
    tile = tiles - 1 - (int)(l / mine);
  } else {
    head = (int)(b % heads);
    tile = tiles - 1 - (int)(b / heads);
  }
}

}  // namespace xhc
