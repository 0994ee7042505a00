// Building blocks of the gated feed-forward block's matrix products (gfx950).
//
// Every product is out[t, n] = sum_k A[t, k] B[n, k] on bf16 MFMA with fp32
// sums, the n side as the first operand: a lane then holds consecutive n of
// one t.  Tiles use 32x32x16 (each operand register feeds twice the products
// of 16x16x32, which counts where the clock is held down by power), the few
// tokens of a decoding step 16x16x32.
//
// All operands lie in fragments: 16 rows x 32 columns in 1 KiB, [piece][row][8],
// piece = columns 8 piece .. + 8 (the lane order of a 16x16x32 operand), in the
// order [row block][column block].  A workgroup keeps a ring of stages of its
// tile's operands in LDS, filled by copies that go from global memory to LDS
// without passing through registers, 1 KiB run each: a stage of 64 KiB comes
// in 1.05 us so, in 1.45 from rows as torch has them (runs of 128 bytes), which
// is what its products take.  So x and dF are brought into fragments first,
// and the epilogues write h, dg and du so.
//
//   FragTile  k is the column: a fragment is an operand as it lies
//   ColTile   k is the row (a weight gradient's token): the transposing LDS
//             load takes it from the same fragments
//
// Either is read without bank conflicts: 16 lanes read a run of 256 bytes, or
// (ColTile) a half wave reads pieces that the copy has put into different banks.
// Copies go through buffer descriptors that end with the tensor: what lies
// behind is read as zero.
#pragma once

#include "xhc_device.h"

namespace xhc {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// v_mfma_f32_32x32x16_bf16: D[32x32] += A[32x16] * B[16x32].  Lane l holds
// A[l%32][8*(l/32) .. +8], B[8*(l/32) .. +8][l%32] and
// D[8*(v/4) + 4*(l/32) + v%4][l%32], v = 0..15.
__device__ __forceinline__ f32x16 mfma_32x32x16(uint4 a, uint4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                 0, 0);
}
// Row p of a block of 16 n holds n = 8 (p / 4 % 2) + 4 (p / 8) + p % 4 of it, so
// that a lane's eight sums of the block (rows 8 i + 4 (l / 32) + 0 .. 3, i = 0, 1)
// are eight consecutive n.
__host__ __device__ __forceinline__ constexpr int perm_n(int p) { return 8 * (p / 4 % 2) + 4 * (p / 8) + p % 4; }

// descriptor of `bytes` bytes at p (below 2 GiB of them; none where bytes <= 0)
__device__ __forceinline__ i32x4 make_srd(uint64_t a, int64_t bytes) {
  const int64_t n = bytes < 0 ? 0 : bytes > 0x7ffffff0 ? 0x7ffffff0 : bytes;
  return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
               __builtin_amdgcn_readfirstlane((int)((a >> 32) & 0xffff)),
               __builtin_amdgcn_readfirstlane((int)n), 0x00020000};
}

// 16 bytes per lane from voff + soff into LDS at lds_addr + AT + 16 lane;
// lds_addr and soff are the same in every lane.  soff stays within a row of
// fragments, and the descriptor holds whole rows, at least one: soff is below
// its length, and does not reach past its end where voff does not.  Inline
// assembly, waited for by the caller, as lds_dma16 (the wait state after the
// write of m0 too).  The five wait states between a vector write of a scalar
// register (make_srd's readfirstlane) and its read here are in the code around
// it, which a test checks in the built library (within the statement, or where
// a descriptor is made, they cost: T = 8192, C = 4096, H = 11008 forward 1748
// us, 1780 with either).
template <int AT>
__device__ __forceinline__ void buf_dma16(const i32x4& srd, uint32_t voff, uint32_t soff, uint32_t lds_addr) {
  asm volatile("s_add_u32 m0, %1, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %2, %3 offen lds"
               :
               : "v"(voff), "s"(lds_addr), "s"(srd), "s"(soff), "n"(AT)
               : "memory", "m0", "scc");
}

__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// where element (t, c) lies in fragments with kb column blocks
__host__ __device__ __forceinline__ int64_t frag_at(int64_t t, int64_t c, int64_t kb) {
  return (t / 16 * kb + c / 32) * 512 + ((c / 8 % 4) * 16 + t % 16) * 8 + c % 8;
}

// an operand in fragments: its planes lie `plane` bytes apart (one for bf16,
// three for fp32: x = plane 0 + plane 1 + plane 2 exactly)
struct Operand {
  const void* p;
  int64_t plane;
  int64_t rows, kb;   // row blocks of 16, column blocks of 32
};

// Tiles of ROWS rows (COLS columns) by KH blocks of 32 k, copied by NW waves of
// kCopies instructions each.  A tile's rows past the last read what follows:
// they only reach sums that nobody writes.
template <int ROWS, int KH, int NW>
struct FragTile {
  static constexpr int kBytes = ROWS * 64 * KH, kCopies = ROWS * KH / 16 / NW;
  static_assert(ROWS * KH % (16 * NW) == 0, "whole copies for every wave");
  i32x4 srd;
  uint32_t voff[kCopies], soff, lds;
  const Operand* op;
  int64_t at;
  static __device__ __forceinline__ int64_t extent(const Operand& o) { return o.rows * 16; }
  __device__ __forceinline__ void init(const Operand& o, int64_t row0, int wave, int lane) {
    op = &o;
    lds = wave * kCopies * 1024;
    at = row0 / 16 * o.kb * 1024;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int f = wave * kCopies + i;
      voff[i] = lane * 16 + (uint32_t)(f / KH) * (uint32_t)o.kb * 1024 + (uint32_t)(f % KH) * 1024;
    }
  }
  // from stage ks of a plane on
  __device__ __forceinline__ void start(int plane, int64_t ks) {
    srd = make_srd((uint64_t)(uintptr_t)op->p + plane * op->plane + at, op->rows * op->kb * 1024 - at);
    soff = (uint32_t)ks * (KH * 1024);
  }
  __device__ __forceinline__ void next() { soff += KH * 1024; }
  // nothing more: copies read no memory and leave zeros
  __device__ __forceinline__ void end() {
    srd.z = 0;
    soff = 0;
  }
  template <int I> __device__ __forceinline__ void copy(uint32_t to) const {
    buf_dma16<I * 1024>(srd, voff[I], soff, to + lds);
  }
  // rows 32 f .., k = 32 kk + 16 m + 8 (lane / 32) + e
  static __device__ __forceinline__ uint4 frag(const unsigned char* s, int f, int kk, int m, int lane) {
    return *reinterpret_cast<const uint4*>(s + ((f * 2 + lane % 32 / 16) * KH + kk) * 1024 +
                                           (2 * m + lane / 32) * 256 + lane % 16 * 16);
  }
};

// The rows (k) of a piece lie at (row ^ 4 piece), so that the four pieces of a
// fragment's 32 columns meet different banks.  PERM: columns as perm_n has them.
template <int COLS, int KH, int NW, bool PERM>
struct ColTileOf {
  static constexpr int kBytes = COLS * 64 * KH, kCopies = COLS * KH / 16 / NW;
  static_assert(COLS % 32 == 0 && COLS * KH % (16 * NW) == 0, "whole copies for every wave");
  static constexpr int kBlocks = COLS / 32;          // fragments side by side
  uint64_t base;
  int64_t left, step;
  i32x4 srd;
  uint32_t voff[kCopies], lds;
  const Operand* op;
  int64_t col0;
  static __device__ __forceinline__ int64_t extent(const Operand& o) { return o.kb * 32; }
  __device__ __forceinline__ void init(const Operand& o, int64_t c0, int wave, int lane) {
    op = &o;
    col0 = c0;
    lds = wave * kCopies * 1024;
    step = o.kb * (2 * KH * 1024);
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int f = wave * kCopies + i;
      voff[i] = (lane ^ (4 * (lane / 16))) * 16 +
                ((uint32_t)(f / kBlocks) * (uint32_t)o.kb + (uint32_t)(f % kBlocks)) * 1024;
    }
  }
  __device__ __forceinline__ void start(int plane, int64_t ks) {
    const int64_t at = ks * step + col0 / 32 * 1024;
    base = (uint64_t)(uintptr_t)op->p + plane * op->plane + at;
    left = op->rows * op->kb * 1024 - at;
    srd = make_srd(base, left);
  }
  __device__ __forceinline__ void next() {
    base += step;
    left -= step;
    srd = make_srd(base, left);
  }
  __device__ __forceinline__ void end() { srd.z = 0; }
  template <int I> __device__ __forceinline__ void copy(uint32_t to) const {
    buf_dma16<I * 1024>(srd, voff[I], 0, to + lds);
  }
  // columns 32 f .., k = 32 kk + 16 m + 8 (lane / 32) + e
  static __device__ __forceinline__ uint4 frag(const unsigned char* s, int f, int kk, int m, int lane) {
    const int r = lane % 16 / 4, q = PERM ? 2 * (lane % 2) + lane % 4 / 2 : lane % 4;   // a row, four columns
    const int piece = 2 * (lane / 16 % 2) + q / 2;
    const unsigned char* p = s + ((kk * 2 + m) * kBlocks + f) * 1024 + piece * 256 + q % 2 * 8;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int k = 8 * (lane / 32) + r;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (k ^ 4 * piece) * 16));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + ((k + 4) ^ 4 * piece) * 16));
    const uint2 ua = __builtin_bit_cast(uint2, a), ub = __builtin_bit_cast(uint2, b);
    return make_uint4(ua.x, ua.y, ub.x, ub.y);
  }
};
template <int COLS, int KH, int NW> using ColTile = ColTileOf<COLS, KH, NW, false>;
template <int COLS, int KH, int NW> using ColTilePerm = ColTileOf<COLS, KH, NW, true>;

// The pairs of planes that a product of two fp32 activations takes: those of
// 2^-16 and more, the small ones first.  (What is left out is below 2^-21 of
// the product, 2^-24 in the mean: the second part is below 2^-7 of the value,
// the third below 2^-15.)
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
  int64_t gn, gt;           // tiles (where `quarters`, of twice the size)
  int64_t from;             // the launch's first of them
  int quarters;             // four workgroups share a tile of twice the size
};

// Workgroup b's tile: each XCD (b % 8) takes a run of consecutive tiles, and
// tiles go in groups of 8 rows of t, so that the workgroups that an XCD runs
// at a time share their operands in its L2.
__device__ __forceinline__ void tile_of(const GemmArgs& a, int64_t& tn, int64_t& tt) {
  const int64_t total = gridDim.x, b = blockIdx.x, x = b % 8, q = total / 8, r = total % 8;
  const int64_t mine = x * q + (x < r ? x : r) + b / 8;
  const int64_t t = a.from + (a.quarters ? mine / 4 : mine);
  constexpr int64_t G = 8;
  const int64_t grp = t / (G * a.gn), first = grp * G, rows = a.gt - first < G ? a.gt - first : G;
  const int64_t l = t - grp * G * a.gn;
  tt = first + l % rows;
  tn = l / rows;
  if (a.quarters) {
    tt = tt * 2 + mine % 4 / 2;
    tn = tn * 2 + mine % 2;
  }
}

template <int V> struct Int { static constexpr int value = V; };
template <int N, class F, int I = 0>
__device__ __forceinline__ void unroll(F&& f) {
  if constexpr (I < N) {
    f(Int<I>{});
    unroll<N, F, I + 1>(static_cast<F&&>(f));
  }
}
template <int N> __device__ __forceinline__ void wait_vm() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }

// How a tile is computed: FN x FT blocks of 32 x 32 per wave, WN x WT waves,
// a ring of R stages of KH blocks of 32 k.
template <int FN_, int FT_, int WN_, int WT_, int KH_, int R_>
struct Shape {
  static constexpr int FN = FN_, FT = FT_, WN = WN_, WT = WT_, KH = KH_, R = R_;
  static constexpr int NW = WN * WT, BN = WN * FN * 32, BT = WT * FT * 32;
  static constexpr int kLds = (BN + BT) * 64 * KH * R;
};

// One tile's product; epi is called once per wave with its sums.
//
// The fragments of 16 k are read into registers while those before them are
// multiplied.  The barrier of a stage stands before its last 16 k's products:
// by then all its fragments are in registers, so its place in the ring takes
// the stage R further on, and the next stage, R - 1 stages' products on the
// way, has landed.  Copies and reads are issued between products, one at a
// time: in front of them they kept the matrix cores waiting (a weight gradient
// at T = 8192, C = 4096, H = 11008 1.64 ms).
template <template <int, int, int> class TN, template <int, int, int> class TT, class S, class Epi>
__device__ __forceinline__ void gemm_tile(const GemmArgs& a, unsigned char* lds, Epi&& epi) {
  constexpr int FN = S::FN, FT = S::FT, KH = S::KH, R = S::R;
  using LN = TN<S::BN, KH, S::NW>;
  using LT = TT<S::BT, KH, S::NW>;
  constexpr int STAGE = LN::kBytes + LT::kBytes, COPIES = LN::kCopies + LT::kCopies;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wn = wave % S::WN, wt = wave / S::WN;
  int64_t tn, tt;
  tile_of(a, tn, tt);
  // a quarter tile past the edge (a FragTile's descriptor would be empty there
  // and its check, of voff against its length less soff, could wrap)
  if (a.quarters && (tn * S::BN >= LN::extent(a.n) || tt * S::BT >= LT::extent(a.t))) return;
  LN ln;
  LT lt;
  ln.init(a.n, tn * S::BN, wave, lane);
  lt.init(a.t, tt * S::BT, wave, lane);
  const uint32_t base = lds_offset(lds);

  const int64_t first = blockIdx.y * a.steps_per_split, all = (int64_t)a.ksteps * a.seg.n;
  const int64_t left = all - first;
  const int steps = (int)(left < a.steps_per_split ? left : a.steps_per_split);
  int seg = (int)(first / a.ksteps), ks = (int)(first % a.ksteps);
  ln.start(a.seg.a[seg], ks);
  lt.start(a.seg.b[seg], ks);
  // copy c of the stage that is next in order, to `to`; after the last of them
  // the one after is next
  auto copy = [&](auto c, uint32_t to) {
    if constexpr (c.value < LN::kCopies)
      ln.template copy<c.value>(to);
    else if constexpr (c.value < COPIES)
      lt.template copy<c.value - LN::kCopies>(to + LN::kBytes);
  };
  int ahead = 0;                  // stages copied or on the way
  auto next = [&] {
    if (++ahead >= steps) {
      ln.end();
      lt.end();
    } else if (++ks == a.ksteps) {
      ks = 0;
      ++seg;
      ln.start(a.seg.a[seg], 0);
      lt.start(a.seg.b[seg], 0);
    } else {
      ln.next();
      lt.next();
    }
  };
  f32x16 acc[FN][FT];
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FT; ++j) acc[i][j] = f32x16{};
  // fragments of 16 k, in two sets: one is read while the other is multiplied
  uint4 frag[2][FN + FT];
  auto read = [&](int set, const unsigned char* s, int unit, int i) {
    frag[set][i] = i < FN ? LN::frag(s, wn * FN + i, unit / 2, unit % 2, lane)
                          : LT::frag(s + LN::kBytes, wt * FT + i - FN, unit / 2, unit % 2, lane);
  };
  constexpr int READS = FN + FT, PRODUCTS = FN * FT, UNITS = 2 * KH;
  constexpr int READ = (READS + PRODUCTS - 1) / PRODUCTS, COPY = (COPIES + PRODUCTS - 1) / PRODUCTS;
  // The products of one set.  Between them the reads of the other (16 k number
  // `unit` of the stage at s) and, with `copied`, the copies of the next stage
  // to `to`: in this order, which the compiler is kept from changing.
  auto multiply = [&](auto copied, auto set, const unsigned char* s, auto unit, uint32_t to) {
    __builtin_amdgcn_sched_barrier(0);
    unroll<PRODUCTS>([&](auto p) {
      unroll<READ>([&](auto r) {
        constexpr int i = p.value * READ + r.value;
        if constexpr (i < READS) read(set.value ^ 1, s, unit.value, i);
      });
      constexpr int j = p.value / FN, i = p.value % FN;
      acc[i][j] = mfma_32x32x16(frag[set.value][i], frag[set.value][FN + j], acc[i][j]);
      if constexpr (copied.value) unroll<COPY>([&](auto c) { copy(Int<p.value * COPY + c.value>{}, to); });
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (copied.value) next();
  };
  for (int i = 0; i < R; ++i) {
    unroll<COPIES>([&](auto c) { copy(c, base + i * STAGE); });
    next();
  }
  wait_vm<(R - 1) * COPIES>();
  lds_barrier();
#pragma unroll
  for (int i = 0; i < READS; ++i) read(0, lds, 0, i);
  int at = 0;                     // of the current stage in the ring
  for (int it = 0; it < steps; ++it) {
    unroll<UNITS - 1>([&](auto u) {
      multiply(Int<0>{}, Int<u.value % 2>{}, lds + at * STAGE, Int<u.value + 1>{}, 0);
    });
    wait_vm<(R - 2) * COPIES>();
    lds_barrier();
    const uint32_t to = base + at * STAGE;
    at = at + 1 == R ? 0 : at + 1;
    // past the last stage the fragments are those of an old one, and unused
    multiply(Int<1>{}, Int<(UNITS - 1) % 2>{}, lds + at * STAGE, Int<0>{}, to);
  }
  wait_vm<0>();                   // nothing may still come when the LDS is another workgroup's
  epi(acc, tn * S::BN + wn * FN * 32, tt * S::BT + wt * FT * 32, lane);
}

}  // namespace xhc
