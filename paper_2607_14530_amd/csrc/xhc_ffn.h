// Building blocks of the gated feed-forward block's matrix products (gfx950).
//
// Every product is out[t, n] = sum_k A[t, k] B[n, k] on 16x16x32 bf16 MFMA with
// fp32 sums, the n side as the first operand: a lane then holds four
// consecutive n of one t.  A workgroup keeps two stages of 64 k of its tile's
// operands in LDS, filled by copies that go from global memory to LDS without
// passing through registers.  Three operand layouts:
//
//   FragTile  packed weights, [n block of 16][k block of 32] fragments of 1 KiB
//             in the MFMA's own lane order: copied and read linearly
//   RowTile   rows with k contiguous (activations, [t][k]): 128 bytes of each
//             row, its 16-byte pieces at (piece ^ row % 8), so that the 16 rows
//             of a fragment read meet different banks
//   ColTile   rows along k (the same activations as the operands of a weight
//             gradient, whose k is the token): 8 x 128-byte pieces, read by the
//             transposing LDS load; 32-byte pieces at (piece ^ swz(k)), so that
//             the 8 rows of a half wave meet different banks
//
// Copies go through buffer descriptors that end with the tensor: what lies
// behind its last row is read as zero, and k past the last column is sent
// behind that end, so that no length needs a padded tensor.
#pragma once

#include "xhc_device.h"

namespace xhc {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kBK = 64;                           // k of a stage
constexpr uint32_t kNowhere = 0x80000000u;        // an offset behind every descriptor's end

// descriptor of `bytes` bytes at p (below 2 GiB of them; none where bytes <= 0)
__device__ __forceinline__ i32x4 make_srd(const void* p, int64_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  const int64_t n = bytes < 0 ? 0 : bytes > 0x7ffffff0 ? 0x7ffffff0 : bytes;
  return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
               __builtin_amdgcn_readfirstlane((int)((a >> 32) & 0xffff)),
               __builtin_amdgcn_readfirstlane((int)n), 0x00020000};
}

// 16 bytes per lane into LDS at lds_addr + 16 lane; lds_addr is the same in
// every lane.  Inline assembly, waited for by the caller, as lds_dma16.
__device__ __forceinline__ void buf_dma16(const i32x4& srd, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %1\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds"
               :
               : "v"(voff), "s"(lds_addr), "s"(srd)
               : "memory", "m0");
}

__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// an operand: its planes lie `plane` bytes apart (one for bf16, three for fp32:
// x = plane 0 + plane 1 + plane 2 exactly)
struct Operand {
  const void* p;
  int64_t plane;
  int64_t ld;     // elements between rows (FragTile: k blocks of 32)
  int64_t rows;   // rows of the tensor (FragTile: n blocks)
  int klim;       // columns that exist (RowTile)
};

template <int ROWS, int NW>
struct FragTile {
  static constexpr int kBytes = ROWS * 128, NI = ROWS / 8 / NW;
  static_assert(ROWS % (8 * NW) == 0, "whole copies for every wave");
  i32x4 srd;
  uint32_t voff, nstride;
  int wave;
  const Operand* op;
  int64_t row0;
  __device__ __forceinline__ void init(const Operand& o, int64_t r0, int w, int lane) {
    op = &o;
    row0 = r0;
    wave = w;
    nstride = (uint32_t)o.ld * 1024;
    voff = lane * 16;
    const int64_t at = r0 / 16 * o.ld * 1024;
    srd = make_srd(reinterpret_cast<const char*>(o.p) + at, o.rows * o.ld * 1024 - at);
  }
  __device__ __forceinline__ void plane(int) {}      // weights have one
  __device__ __forceinline__ void issue(uint32_t lds, int ks) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int f = wave * NI + i;
      buf_dma16(srd, voff + (uint32_t)(f / 2) * nstride + (uint32_t)(ks * 2 + f % 2) * 1024,
                __builtin_amdgcn_readfirstlane(lds + f * 1024));
    }
  }
  static __device__ __forceinline__ uint4 frag(const unsigned char* s, int f16, int kk, int lane) {
    return *reinterpret_cast<const uint4*>(s + (f16 * 2 + kk) * 1024 + lane * 16);
  }
};

template <int ROWS, int NW>
struct RowTile {
  static constexpr int kBytes = ROWS * 128, NI = ROWS / 8 / NW;
  static_assert(ROWS % (8 * NW) == 0, "whole copies for every wave");
  i32x4 srd;
  uint32_t voff, rstride;
  int wave, kcol;
  const Operand* op;
  int64_t row0;
  __device__ __forceinline__ void init(const Operand& o, int64_t r0, int w, int lane) {
    op = &o;
    row0 = r0;
    wave = w;
    const int chunk = (lane % 8) ^ (lane / 8);
    kcol = chunk * 8;
    rstride = (uint32_t)o.ld * 16;                   // 8 rows
    voff = (uint32_t)(w * NI) * rstride + (uint32_t)(lane / 8) * (uint32_t)o.ld * 2 + chunk * 16;
    plane(0);
  }
  __device__ __forceinline__ void plane(int p) {
    srd = make_srd(reinterpret_cast<const char*>(op->p) + p * op->plane + row0 * op->ld * 2,
                   (op->rows - row0) * op->ld * 2);
  }
  __device__ __forceinline__ void issue(uint32_t lds, int ks) {
    const uint32_t at = ks * kBK + kcol < op->klim ? voff + (uint32_t)ks * (kBK * 2) : kNowhere;
#pragma unroll
    for (int i = 0; i < NI; ++i)
      buf_dma16(srd, at == kNowhere ? kNowhere : at + i * rstride,
                __builtin_amdgcn_readfirstlane(lds + (wave * NI + i) * 1024));
  }
  static __device__ __forceinline__ uint4 frag(const unsigned char* s, int f16, int kk, int lane) {
    return *reinterpret_cast<const uint4*>(s + (f16 * 16 + lane % 16) * 128 +
                                           (((kk * 4 + lane / 16) ^ (lane & 7)) << 4));
  }
};

// COLS columns of 64 rows along k
template <int COLS, int NW>
struct ColTile {
  static constexpr int kBytes = COLS * 128, NI = COLS / 8 / NW;
  static_assert(COLS % 64 == 0 && (COLS / 8) % NW == 0, "whole copies for every wave");
  i32x4 srd;
  uint32_t voff;
  int wave, cur = 0;
  const Operand* op;
  int64_t col0;
  __device__ __forceinline__ static int swz(int k) { return (k & 3) ^ ((k >> 2) & 1); }
  __device__ __forceinline__ void init(const Operand& o, int64_t c0, int w, int lane) {
    op = &o;
    col0 = c0;
    wave = w;
    const int k = lane / 8, chunk = (lane % 8) ^ (2 * swz(k));
    voff = (uint32_t)k * (uint32_t)o.ld * 2 + chunk * 16;
  }
  __device__ __forceinline__ void plane(int p) { cur = p; }
  __device__ __forceinline__ void issue(uint32_t lds, int ks) {
    const int64_t at = ((int64_t)ks * kBK * op->ld + col0) * 2;
    srd = make_srd(reinterpret_cast<const char*>(op->p) + cur * op->plane + at, op->rows * op->ld * 2 - at);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int f = wave * NI + i;
      buf_dma16(srd, voff + (uint32_t)(f % 8) * (uint32_t)op->ld * 16 + (uint32_t)(f / 8) * 128,
                __builtin_amdgcn_readfirstlane(lds + f * 1024));
    }
  }
  // k = 32 kk + 16 j + 4 (lane / 16) + r for element 4 j + r, on both sides alike
  static __device__ __forceinline__ uint4 frag(const unsigned char* s, int f16, int kk, int lane) {
    const int g = lane / 16, r = (lane % 16) / 4, q = lane % 4;
    const unsigned char* p = s + (f16 / 4 * 8 + kk * 4 + g / 2) * 1024 + (4 * (g & 1) + r) * 128 +
                             (((f16 % 4) ^ r ^ (g & 1)) << 5) + q * 8;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 2048));
    const uint2 ua = __builtin_bit_cast(uint2, a), ub = __builtin_bit_cast(uint2, b);
    return make_uint4(ua.x, ua.y, ub.x, ub.y);
  }
};

// The pairs of planes that a product of two fp32 activations takes: those of
// 2^-16 and more, the small ones first.  (What is left out is below 2^-23 of
// the product.)
struct Segments {
  int n;
  uint8_t a[6], b[6];
};
inline Segments segs_bf16() { return Segments{1, {0}, {0}}; }
inline Segments segs_weights() { return Segments{3, {0, 0, 0}, {2, 1, 0}}; }   // bf16 weights, fp32 activations
inline Segments segs_f32() { return Segments{6, {2, 0, 1, 1, 0, 0}, {0, 2, 1, 0, 1, 0}}; }

struct GemmArgs {
  Operand n, t;
  Segments seg;
  int ksteps;               // stages of one segment
  int64_t steps_per_split;  // of all ksteps * seg.n stages, in blockIdx.y parts
  int64_t gn, gt;           // tiles
};

// Workgroup b's tile: each XCD (b % 8) takes a run of consecutive tiles, and
// tiles go in groups of 8 rows of t, so that the workgroups that an XCD runs
// at a time share their operands in its L2.
__device__ __forceinline__ void tile_of(int64_t gn, int64_t gt, int64_t& tn, int64_t& tt) {
  const int64_t total = gn * gt, b = blockIdx.x, x = b % 8, q = total / 8, r = total % 8;
  const int64_t t = x * q + (x < r ? x : r) + b / 8;
  constexpr int64_t G = 8;
  const int64_t grp = t / (G * gn), first = grp * G, rows = gt - first < G ? gt - first : G;
  const int64_t l = t - grp * G * gn;
  tt = first + l % rows;
  tn = l / rows;
}

// One tile's product.  FN x FT fragments per wave, WN x WT waves; epi is
// called once per wave with its sums.
template <template <int, int> class TN, template <int, int> class TT, int FN, int FT, int WN, int WT, class Epi>
__device__ __forceinline__ void gemm_tile(const GemmArgs& a, unsigned char* lds, Epi&& epi) {
  constexpr int NW = WN * WT, BN = WN * FN * 16, BT = WT * FT * 16;
  using LN = TN<BN, NW>;
  using LT = TT<BT, NW>;
  constexpr int STAGE = LN::kBytes + LT::kBytes;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wn = wave % WN, wt = wave / WN;
  int64_t tn, tt;
  tile_of(a.gn, a.gt, tn, tt);
  LN ln;
  LT lt;
  ln.init(a.n, tn * BN, wave, lane);
  lt.init(a.t, tt * BT, wave, lane);
  const uint32_t base = lds_offset(lds);

  const int64_t first = blockIdx.y * a.steps_per_split, all = (int64_t)a.ksteps * a.seg.n;
  const int64_t left = all - first;
  const int steps = (int)(left < a.steps_per_split ? left : a.steps_per_split);
  int seg = (int)(first / a.ksteps), ks = (int)(first % a.ksteps);
  ln.plane(a.seg.a[seg]);
  lt.plane(a.seg.b[seg]);
  auto issue = [&](int buf) {
    ln.issue(base + buf * STAGE, ks);
    lt.issue(base + buf * STAGE + LN::kBytes, ks);
    if (++ks == a.ksteps && seg + 1 < a.seg.n) {
      ks = 0;
      ++seg;
      ln.plane(a.seg.a[seg]);
      lt.plane(a.seg.b[seg]);
    }
  };
  f32x4 acc[FN][FT];
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  issue(0);
  for (int it = 0; it < steps; ++it) {
    // this wave's copies of the stage have landed; after the barrier everyone's,
    // and nobody reads the other stage any more
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();
    if (it + 1 < steps) issue((it + 1) & 1);
    const unsigned char* sn = lds + (it & 1) * STAGE;
    const unsigned char* st = sn + LN::kBytes;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      uint4 fn[FN], ft[FT];
#pragma unroll
      for (int i = 0; i < FN; ++i) fn[i] = LN::frag(sn, wn * FN + i, kk, lane);
#pragma unroll
      for (int j = 0; j < FT; ++j) ft[j] = LT::frag(st, wt * FT + j, kk, lane);
#pragma unroll
      for (int j = 0; j < FT; ++j)
#pragma unroll
        for (int i = 0; i < FN; ++i) acc[i][j] = mfma_16x16x32(fn[i], ft[j], acc[i][j]);
    }
  }
  epi(acc, tn * BN + wn * FN * 16, tt * BT + wt * FT * 16, lane);
}

}  // namespace xhc
