// A paged cache of keys and values in 4 bits, and attention over it.
//
// A page holds, for each key and value head, blocks of 32 tokens, and a block
// the four operands of its products as the matrix instructions take them, so
// that attention reads runs and unpacks in place:
//
//   keys    [half of 16 tokens][lane][D / 32 words]: lane l has channels 32 g +
//           8 (l / 16) + 0 .. 7 of token l % 16 in word g, an operand of scores^T
//           = K Q^T over the 32 channels of group g
//   values  [lane][D / 16 words] in pieces of four words: lane l has channel 16 n
//           + l % 16 of tokens 16 (j / 4) + 4 (l / 16) + j % 4, j = 0 .. 7, in word
//           n: the order in which a lane holds the probabilities of its query
//   scales  of keys, of values: [l / 16][half][group][4 tokens] bf16: lane l
//           loads a word of its row of 16 lanes, which takes it from there (a DPP
//           broadcast within the row, part of the instruction that multiplies)
//
// A group's scale is a factor of its share of a score, and of a probability
// before it is rounded (bf16 state) as an operand of the product with the values.
// The row's sum is of the unrounded ones: a rounded one goes with its group's scale.
//
// Measured at Hq = 32, Hkv = 8, D = 128, bf16: a token's attention over 131072
// keys 34 us (151 MB, 4.4 TB/s) and the join 8; over 64 sequences of 2048 to
// 8192 80 us with its join (350 MB); appending 8192 tokens 38 us (177 MB, 4.6
// TB/s), reading them 16.
#include "xhc_attn.h"

namespace xhc {

namespace {

constexpr int kBlock = 32;                       // tokens of a block

struct CacheArgs {
  const void* qkv;        // append: [T][Hq + 2 Hkv][D]
  const float* table;
  const int *starts, *lens, *pages;
  unsigned char* pool;
  void *q, *k, *v;        // append's q, read's k and v; attend: q in, out in k
  const float* slopes;
  int64_t T;
  int Hq, Hkv, R, pairs, window, page, npages, B, per_seq;
  int rows;               // append: tokens that a workgroup looks after
  int tokens;             // append: of which a workgroup behind those rotates the queries
  unsigned blocks;        // append: workgroups that look after keys and values
  float scale, cap;
  // attend
  float* part;            // [2 grid][16 RT][D]
  float2* ml;             // [2 grid][16 RT]: maximum and sum
  int64_t* where;         // [B][2]: first unit of a sequence, units of its segments; [2 B]: units of a workgroup
};

template <int D> struct Block {
  static constexpr int G = D / 32, W = D / 16;
  static constexpr int kCodes = 16 * D, kScales = 2 * D, kBytes = 2 * kCodes + 2 * kScales;
  static constexpr int kKeys = 0, kValues = kCodes, kKeyScales = 2 * kCodes, kValueScales = 2 * kCodes + kScales;
  // byte of the word of channels 8 c .. 8 c + 7 of a token's key
  static __device__ __forceinline__ int key_word(int tok, int c) {
    return kKeys + ((tok / 16 * 64 + c % 4 * 16 + tok % 16) * G + c / 4) * 4;
  }
  // byte of word n of a lane's values
  static __device__ __forceinline__ int value_word(int lane, int n) {
    const int at = n / 4 * 4, wide = W - at < 4 ? W - at : 4;
    return kValues + (at * 64 + lane * wide + n % 4) * 4;
  }
  static __device__ __forceinline__ int value_lane(int tok, int ch) { return tok % 16 / 4 * 16 + ch % 16; }
  static __device__ __forceinline__ int value_slot(int tok) { return tok / 16 * 4 + tok % 4; }
  // byte of a token's scale of group g, from the first of the keys' or values'
  static __device__ __forceinline__ int scale_at(int tok, int g) {
    return ((tok % 16 / 4 * 2 + tok / 16) * G + g) * 8 + tok % 4 * 2;
  }
};

template <int D> __device__ __forceinline__ unsigned char* block_at(const CacheArgs& a, int page, int head, int tok) {
  return a.pool + (((int64_t)page * a.Hkv + head) * (a.page / kBlock) + tok / kBlock) * Block<D>::kBytes;
}

// The sequence that token t of a call belongs to: the last b with starts[b] <=
// t, or -1.  All lanes of the wave ask for the same t; a step looks at 64 places.
__device__ __forceinline__ int sequence_of(const int* starts, int B, int64_t t, int lane) {
  int first = 0, n = B;
  do {
    const int step = (n + 63) / 64, i = lane * step;
    const int c = __popcll(__ballot(i < n && starts[first + i] <= t));
    if (c == 0) return -1;
    first += (c - 1) * step;
    n = n - (c - 1) * step < step ? n - (c - 1) * step : step;
  } while (n > 1);
  return __builtin_amdgcn_readfirstlane(first);
}

// four pairs of neighbours by w (cosine, sine of each)
__device__ __forceinline__ void turn_pairs(float (&x)[8], const float* w) {
  float a[4], b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = x[2 * i], b[i] = x[2 * i + 1];
  turn<4>(a, b, w, 1.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = a[i], x[2 * i + 1] = b[i];
}

// Eight consecutive channels from channel c of a head, rotated at the position
// whose table row is cs.
template <typename TS>
__device__ __forceinline__ void rotated8(const TS* head, int c, const float* cs, int R, int pairs, float (&x)[8]) {
  Vec8<TS>::load(head + c, x);
  if (c >= R) return;
  if (pairs) {
    float w[8];
    Vec8<float>::load(cs + c, w);
    turn_pairs(x, w);
  } else {
    const bool low = c < R / 2;
    float w[16], y[8];
    Vec8<float>::load(cs + 2 * (low ? c : c - R / 2), *reinterpret_cast<float(*)[8]>(w));
    Vec8<float>::load(cs + 2 * (low ? c : c - R / 2) + 8, *reinterpret_cast<float(*)[8]>(w + 8));
    Vec8<TS>::load(head + (low ? c + R / 2 : c - R / 2), y);
    if (low) {
      turn<8>(x, y, w, 1.f);
    } else {
      turn<8>(y, x, w, 1.f);
    }
  }
}

// Codes of eight channels of a group that four neighbouring lanes share, and
// its scale (bf16 bits): the largest magnitude / 6, rounded; divisions rounded
// to the nearest, so that the codes are the definition's to the bit.  The
// quotients by one scale share its reciprocal r: with r rounded to the nearest
// and q within one step of x / s, q + (x - q s) r in fused products is x / s
// rounded to the nearest (Markstein's theorem); x r may be two steps off, so
// the correction is made twice.  Nothing underflows where it matters: s is
// 2^-103 or more, and quotients far below 1/4 may have any last bits.  (IEEE
// divisions and seven comparisons an element, and a thread's loads one after
// another, took 55 us instead of 45 for 8192 tokens of Hq = 32, Hkv = 8, D = 128.)
__device__ __forceinline__ uint32_t hold8(const float (&x)[8], uint32_t& bits) {
  uint32_t top = 0;                              // magnitudes order as their bits do, NaN above all
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  bits = top >= 0x7f800000u              ? 0x7fc0u
         : top < (27u << 23)             ? 0u               // below 2^-100
                                         : f2bf(__uint_as_float(top) / 6.f);
  const float s = __uint_as_float(bits << 16);
  uint32_t w = 0;
  if (bits != 0 && bits != 0x7fc0u) {
    const float r = 1.f / s;
    float m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = x[i] * r;
      m[i] = fmaf(fmaf(-m[i], s, x[i]), r, m[i]);
      m[i] = copysignf(fmaf(fmaf(-m[i], s, x[i]), r, m[i]), x[i]);         // (-0 keeps its sign)
    }
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, m[0], m[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, m[2], m[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, m[4], m[5], 1.f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, m[6], m[7], 1.f, 3);
  }
  return w;
}

// Some workgroups rotate the queries, a few tokens each.  Each of the `blocks`
// others, which wait for more and move less, looks after `rows` tokens for one
// head: it stores the block of each token that is the call's first in its block,
// which may go on behind them; so no two workgroups write to a block.  Tokens
// that were there before keep their bits.
template <typename TS, int D>
__global__ __launch_bounds__(256) void k_cache_append(CacheArgs a) {
  using BL = Block<D>;
  constexpr int P = D / 8;                       // threads of a head
  __shared__ uint8_t codes[kBlock][D + 4];
  __shared__ int64_t pos[256];
  const int tid = threadIdx.x, lane = tid % 64, H = a.Hq + 2 * a.Hkv;
  const int64_t cap = (int64_t)a.per_seq * a.page;
  const TS* qkv = static_cast<const TS*>(a.qkv);
  // eights of both kinds in turn, which go to the eight XCDs, then what is left of one
  const unsigned eights = (a.blocks < gridDim.x - a.blocks ? a.blocks : gridDim.x - a.blocks) / 8;
  const bool turns = blockIdx.x < 16 * eights;
  const unsigned left = a.blocks - 8 * eights;
  const bool queries = turns ? blockIdx.x % 16 >= 8 : blockIdx.x - 16 * eights >= left;
  const unsigned mine = turns ? blockIdx.x / 16 * 8 + blockIdx.x % 8 : blockIdx.x - 8 * eights - (queries ? left : 0);
  if (queries) {
    const int64_t t0 = (int64_t)mine * a.tokens;
    for (int i = tid / 64; i < a.tokens; i += 4) {
      const int64_t t = t0 + i;
      const int b = t < a.T ? sequence_of(a.starts, a.B, t, lane) : -1;
      int64_t p = -1;
      if (b >= 0 && t < a.starts[b + 1]) p = a.lens[b] - (a.starts[b + 1] - t);
      if (lane == 0) pos[i] = p < cap ? p : -1;
    }
    __syncthreads();
    // a thread has 16 channels (rotated ones with their partners) of some heads
    // of a token, which share a table's row; two heads' loads first
    constexpr int per = D / 16, slots = 256 / per;
    const int heads = min(a.Hq, max(1, slots / a.tokens)), n = slots / heads, j = tid % per, slot = tid / per;
    if (slot >= n * heads) return;
    for (int i = slot / heads; i < a.tokens; i += n) {
      const int64_t p = pos[i];
      if (p < 0) continue;
      const bool turned = 16 * j < a.R, split = turned && !a.pairs;
      float cs[16];
      if (turned) {
        Vec8<float>::load(a.table + p * a.R + 16 * j, *reinterpret_cast<float(*)[8]>(cs));
        Vec8<float>::load(a.table + p * a.R + 16 * j + 8, *reinterpret_cast<float(*)[8]>(cs + 8));
      }
      const int ca = split ? 8 * j : 16 * j, cb = split ? 8 * j + a.R / 2 : 16 * j + 8;
      const TS* src = qkv + (t0 + i) * H * D;
      TS* q = static_cast<TS*>(a.q) + (t0 + i) * a.Hq * D;
      for (int h0 = slot % heads; h0 < a.Hq; h0 += 2 * heads) {
        float x[2][8], y[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int h = min(h0 + k * heads, a.Hq - 1);
          Vec8<TS>::load(src + h * D + ca, x[k]);
          Vec8<TS>::load(src + h * D + cb, y[k]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int h = h0 + k * heads;
          if (h >= a.Hq) break;
          if (split) {
            turn<8>(x[k], y[k], cs, 1.f);
          } else if (turned) {
            turn_pairs(x[k], cs);
            turn_pairs(y[k], cs + 8);
          }
          Vec8<TS>::store(q + h * D + ca, x[k]);
          Vec8<TS>::store(q + h * D + cb, y[k]);
        }
      }
    }
    return;
  }
  const int head = mine % a.Hkv;
  int64_t t = (int64_t)(mine / a.Hkv) * a.rows;
  const int64_t behind = t + a.rows < a.T ? t + a.rows : a.T;
  while (t < behind) {
    const int b = sequence_of(a.starts, a.B, t, lane);
    if (b < 0) {                                 // in front of the first sequence
      const int64_t s = a.starts[0];
      if (s >= behind) return;
      t = s;
      continue;
    }
    const int64_t first = a.starts[b] > 0 ? a.starts[b] : 0, after = a.starts[b + 1], end = after < a.T ? after : a.T;
    if (t >= end) return;                        // behind the last (starts ascend)
    const int64_t p = a.lens[b] - (after - t);
    if (p < 0 || p >= cap) {
      t = p < 0 && t - p < end ? t - p : end;
      continue;
    }
    const int64_t next = t + kBlock - p % kBlock < end ? t + kBlock - p % kBlock : end;
    const int idx = a.pages[(int64_t)b * a.per_seq + p / a.page];
    // the block's first token of this call: where it begins, or where the call's tokens of the sequence do
    if ((p % kBlock == 0 || t == first) && idx >= 0 && idx < a.npages) {
      unsigned char* to = block_at<D>(a, idx, head, (int)(p % a.page));
      const int at = (int)(p % kBlock), n = (int)(next - t);     // tokens at .. at + n - 1 of the block are new
      // all loads of a thread's two tokens before the first use
      for (int u0 = tid; u0 < n * P; u0 += 512) {
        float x[2][8], y[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int u = min(u0 + 256 * k, n * P - 1), c = u % P, i = u / P;
          const TS* src = qkv + ((t + i) * H + a.Hq + head) * D;
          Vec8<TS>::load(src + (int64_t)a.Hkv * D + 8 * c, y[k]);
          rotated8<TS>(src, 8 * c, a.table + (p + i) * a.R, a.R, a.pairs, x[k]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int u = u0 + 256 * k, c = u % P, tok = at + u / P;
          if (u >= n * P) break;
          uint32_t bits, vbits;
          const uint32_t w = hold8(x[k], bits), v = hold8(y[k], vbits);
          if (c % 4 == 0) {
            *reinterpret_cast<uint16_t*>(to + BL::kKeyScales + BL::scale_at(tok, c / 4)) = (uint16_t)bits;
            *reinterpret_cast<uint16_t*>(to + BL::kValueScales + BL::scale_at(tok, c / 4)) = (uint16_t)vbits;
          }
          *reinterpret_cast<uint32_t*>(to + BL::key_word(tok, c)) = w;
#pragma unroll
          for (int e = 0; e < 8; ++e) codes[tok][8 * c + e] = (uint8_t)(v >> (4 * e) & 15);
        }
      }
      __syncthreads();
      for (int u = tid; u < 64 * BL::W; u += 256) {
        const int l = u % 64, word = u / 64, ch = 16 * word + l % 16;
        uint32_t w = 0, keep = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int tok = 16 * (j / 4) + 4 * (l / 16) + j % 4;
          if (tok >= at && tok < at + n)
            w |= (uint32_t)codes[tok][ch] << (4 * j);
          else
            keep |= 15u << (4 * j);
        }
        if (keep == 0xffffffffu) continue;
        uint32_t* p32 = reinterpret_cast<uint32_t*>(to + BL::value_word(l, word));
        *p32 = keep ? (*p32 & keep) | w : w;
      }
      __syncthreads();
    }
    t = next;
  }
}

__device__ __forceinline__ float held_value(uint32_t code) {
  const float m = (float)(0xc8643210u >> (4 * (code & 7)) & 15) * 0.5f;
  return code & 8 ? -m : m;
}

// A few tokens a workgroup, as with the queries above: their places first, which
// three loads one after another find.  Bound by its loads: a token's value codes
// are a nibble in each of eight words (8192 tokens of Hkv = 8, D = 128: 16 us
// for 42 MB).
template <typename TS, int D>
__global__ __launch_bounds__(256) void k_cache_read(CacheArgs a) {
  using BL = Block<D>;
  constexpr int P = D / 8;
  __shared__ int2 place[256];                    // a token's page (-1: none) and place in it
  const int tid = threadIdx.x, lane = tid % 64;
  const int64_t t0 = (int64_t)blockIdx.x * a.tokens, cap = (int64_t)a.per_seq * a.page;
  for (int i = tid / 64; i < a.tokens; i += 4) {
    const int64_t t = t0 + i;
    const int b = t < a.T ? sequence_of(a.starts, a.B, t, lane) : -1;
    int2 at = make_int2(-1, 0);
    if (b >= 0 && t < a.starts[b + 1]) {
      const int64_t p = a.lens[b] - (a.starts[b + 1] - t);
      if (p >= 0 && p < cap) at = make_int2(a.pages[(int64_t)b * a.per_seq + p / a.page], (int)(p % a.page));
    }
    if (lane == 0) place[i] = at;
  }
  __syncthreads();
  const int all = a.tokens * a.Hkv * P;
  for (int u = tid; u < all; u += 256) {
    const int c = u % P, head = u / P % a.Hkv, i = u / P / a.Hkv;
    const int2 at = place[i];
    if (at.x < 0 || at.x >= a.npages) continue;
    const unsigned char* from = block_at<D>(a, at.x, head, at.y);
    const int tok = at.y % kBlock;
    const uint32_t ks = *reinterpret_cast<const uint16_t*>(from + BL::kKeyScales + BL::scale_at(tok, c / 4));
    const uint32_t vs = *reinterpret_cast<const uint16_t*>(from + BL::kValueScales + BL::scale_at(tok, c / 4));
    const uint32_t k = *reinterpret_cast<const uint32_t*>(from + BL::key_word(tok, c));
    uint32_t v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int ch = 8 * c + e;
      const uint32_t word = *reinterpret_cast<const uint32_t*>(from + BL::value_word(BL::value_lane(tok, ch), ch / 16));
      v |= (word >> (4 * BL::value_slot(tok)) & 15) << (4 * e);
    }
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = held_value(k >> (4 * e) & 15) * __uint_as_float(ks << 16);
      y[e] = held_value(v >> (4 * e) & 15) * __uint_as_float(vs << 16);
    }
    const int64_t to = ((t0 + i) * a.Hkv + head) * D + 8 * c;
    Vec8<TS>::store(static_cast<TS*>(a.k) + to, x);
    Vec8<TS>::store(static_cast<TS*>(a.v) + to, y);
  }
}

// ---------------------------------------------------------------- attention over the cache

__device__ __forceinline__ f32x4 mfma16(const uint4& a, const uint4& b, f32x4 c) { return mfma_16x16x32(a, b, c); }
__device__ __forceinline__ f32x4 mfma16(const Frag32& a, const Frag32& b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
  return c;
}
// a word's eight codes, exact in either type
__device__ __forceinline__ void unpack_codes(uint32_t w, uint4& f) {
  f.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 0));
  f.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 1));
  f.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 2));
  f.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 3));
}
__device__ __forceinline__ void unpack_codes(uint32_t w, Frag32& f) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1),
              c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
  f = Frag32{{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y}};
}
__device__ __forceinline__ void pack_frag(const float (&x)[8], uint4& f) { f = pack8(x); }
__device__ __forceinline__ void pack_frag(const float (&x)[8], Frag32& f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) f.v[j] = x[j];
}
// lane i's value, in scalar registers
__device__ __forceinline__ int64_t scalar64(int64_t x, int i) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, i);
  return (int64_t)__builtin_amdgcn_readlane((int)(x >> 32), i) << 32 | lo;
}
// lane K of this lane's row of 16
template <int K> __device__ __forceinline__ float row_lane(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x150 + K, 0xF, 0xF, true));
}
__device__ __forceinline__ float max_quarters(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// A block of keys and values of one head, on its way.
template <int D> struct Raw {
  uint32_t k[2][D / 32], v[D / 16], ks, vs;
  template <int N> static __device__ __forceinline__ void words(const unsigned char* p, uint32_t* w) {
    if constexpr (N == 4) {
      const uint4 x = *reinterpret_cast<const uint4*>(p);
      w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    } else if constexpr (N == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[0] = x.x, w[1] = x.y;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
    }
  }
  __device__ __forceinline__ void load(const unsigned char* p, uint32_t lane) {
    using BL = Block<D>;
#pragma unroll
    for (int h = 0; h < 2; ++h) words<BL::G>(p + BL::kKeys + (h * 64 + lane) * BL::G * 4, k[h]);
#pragma unroll
    for (int at = 0; at < BL::W; at += 4) {
      if (BL::W - at >= 4)
        words<4>(p + BL::kValues + (at * 64 + lane * 4) * 4, v + at);
      else
        words<2>(p + BL::kValues + (at * 64 + lane * 2) * 4, v + at);
    }
    // of a row of 16 lanes the first 4 G have a word each
    const uint32_t s = (lane / 16 * 4 * BL::G + (lane % 16 < 4 * BL::G ? lane % 16 : 0)) * 4;
    ks = *reinterpret_cast<const uint32_t*>(p + BL::kKeyScales + s);
    vs = *reinterpret_cast<const uint32_t*>(p + BL::kValueScales + s);
  }
};

struct Sequence {
  int64_t first, end, after;   // its tokens of the call (within 0 .. T), and starts[b + 1]
  int64_t len, upto;           // its tokens, and those that its row of the table has room for
  int blocks, block0;          // of 32 keys that its tokens see, the first of them
  int tiles;                   // of its rows
};
__device__ __forceinline__ Sequence sequence(const CacheArgs& a, int b, int rows) {
  Sequence s;
  s.first = a.starts[b] > 0 ? a.starts[b] : 0;
  s.after = a.starts[b + 1];
  s.end = s.after < a.T ? s.after : a.T;
  s.len = a.lens[b];
  const int64_t cap = (int64_t)a.per_seq * a.page;
  s.upto = s.len < cap ? s.len : cap;
  const int64_t p = s.len - (s.after - s.first);
  const int64_t lo = a.window > 0 && p - a.window + 1 > 0 ? p - a.window + 1 : 0;
  const bool some = s.end > s.first && s.upto > lo;
  s.block0 = (int)(some ? lo / kBlock : 0);
  s.blocks = some ? (int)((s.upto + kBlock - 1) / kBlock) - s.block0 : 0;
  s.tiles = some ? (int)(((s.end - s.first) * (a.Hq / a.Hkv) + rows - 1) / rows) : 0;
  return s;
}

// The work in units of one block of one head and tile of rows, in the order
// sequence, tile, head, block, is cut into equal runs, one for each workgroup:
// lengths need not be alike, nor known to the host.  A run takes the end of a
// segment (a sequence's tile and head), whole segments, and the beginning of
// another; what it has of a segment that it does not have whole goes to one of
// its two places, and k_cache_join adds those up in order.
//
// Within a run a segment's blocks go around the four waves, each with the
// running maximum and sum of its rows; a block's loads are under way while the
// one before is worked on.  16 RT rows (tokens times the query heads of the
// group) are the columns of 16x16x32 products.
constexpr int attend_wgs(bool f32, int rows) { return rows == 16 ? (f32 ? 2 : 3) : (f32 ? 1 : 2); }   // of a CU

template <typename TS, int D, int RT, bool EX>
__global__ __launch_bounds__(256, attend_wgs(sizeof(TS) == 4, 16 * RT)) void k_cache_attend(CacheArgs a) {
  using BL = Block<D>;
  constexpr int G = BL::G, W = BL::W, ROWS = 16 * RT, LD = D + 4;
  constexpr bool ROUND = RT == 2;                // scores always rounded before their difference (see kFar)
  __shared__ __align__(16) float sums[4][16][LD];
  __shared__ float2 mls[4][16];
  __shared__ int64_t scan[256];
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = a.Hq / a.Hkv;

  // The run's first unit's sequence b, and the units in front of that.
  int b;
  int64_t u0, u1, before;
  auto runs = [&](int64_t all) {
    // at least four blocks a workgroup, one for each wave
    int64_t run = (all + gridDim.x - 1) / gridDim.x;
    if (run < 4) run = 4;
    if (blockIdx.x == 0 && tid == 0) a.where[2 * (int64_t)a.B] = run;
    u0 = (int64_t)blockIdx.x * run;
    u1 = u0 + run < all ? u0 + run : all;
  };
  auto units = [&](int i) {
    const Sequence s = sequence(a, i, ROWS);
    return (int64_t)s.tiles * a.Hkv * s.blocks;
  };
  auto note = [&](int i, int64_t at) {
    a.where[2 * i] = at;
    a.where[2 * i + 1] = sequence(a, i, ROWS).blocks;
  };
  if (a.B <= 64) {                               // each wave by itself, a lane a sequence
    const int64_t mine = lane < a.B ? units(lane) : 0;
    int64_t sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t x = __shfl_up((long long)sum, d);
      if (lane >= d) sum += x;
    }
    runs(scalar64(sum, 63));
    if (blockIdx.x == 0 && wave == 0 && lane < a.B) note(lane, sum - mine);
    if (u0 >= u1) return;
    b = __popcll(__ballot(sum <= u0));
    before = b > 0 ? scalar64(sum, b - 1) : 0;
  } else {
    // the workgroup's threads have a share of the sequences each
    const int share = (a.B + 255) / 256, b0 = tid * share, b1 = min(a.B, b0 + share);
    int64_t mine = 0;
    for (int i = b0; i < b1; ++i) mine += units(i);
    scan[tid] = mine;
    __syncthreads();
    for (int d = 1; d < 256; d *= 2) {
      const int64_t x = tid >= d ? scan[tid - d] : 0;
      __syncthreads();
      scan[tid] += x;
      __syncthreads();
    }
    runs(scan[255]);
    if (blockIdx.x == 0) {
      int64_t at = scan[tid] - mine;
      for (int i = b0; i < b1; ++i) {
        note(i, at);
        at += units(i);
      }
    }
    if (u0 >= u1) return;
    int owner = 0;                               // the first thread whose share ends behind u0
    for (int upto = 255; owner < upto;) {
      const int c = (owner + upto) / 2;
      if (scan[c] > u0)
        upto = c;
      else
        owner = c + 1;
    }
    before = owner > 0 ? scan[owner - 1] : 0;
    for (b = owner * share;; ++b) {
      const int64_t n = units(b);
      if (before + n > u0) break;
      before += n;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    before = scalar64(before, 0);
  }
  u0 = scalar64(u0, 0);
  u1 = scalar64(u1, 0);
  Sequence sq = sequence(a, b, ROWS);

  for (int64_t u = u0; u < u1;) {
    while (u >= before + (int64_t)sq.tiles * a.Hkv * sq.blocks) {
      before += (int64_t)sq.tiles * a.Hkv * sq.blocks;
      sq = sequence(a, ++b, ROWS);
    }
    const int64_t seg = (u - before) / sq.blocks, seg0 = before + seg * sq.blocks;
    int heads = a.Hkv;
    const float* slopes = a.slopes;
    asm volatile("" : "+s"(heads), "+s"(slopes));      // (what follows from them is not kept in registers over the loop)
    const int head = (int)(seg % heads), tile = (int)(seg / heads);
    const int from = (int)(u - seg0);
    const int64_t last = u1 < seg0 + sq.blocks ? u1 : seg0 + sq.blocks;
    const int upto = (int)(last - seg0);         // blocks from .. upto - 1 of the segment are taken here

    const int r16 = again(lane) % 16, quarter = again(lane) / 16;
    // this lane's rows: row r16 of each of the RT tiles
    Frag<TS> q[RT][G];
    int see[RT], low[RT];                        // the row sees low .. see - 1
    float m[RT], l[RT], slope[RT];
    f32x4 o[RT][W];
    int least = INT32_MAX, most = 0;             // every row sees most .. least - 1
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int64_t row = (int64_t)tile * ROWS + rt * 16 + r16, i = row / g;
      const int64_t t = sq.first + i, p = sq.len - (sq.after - t);
      const bool is = t < sq.end && p >= 0 && p < (int64_t)a.per_seq * a.page;
      const int qh = head * g + (int)(row % g);
      see[rt] = is ? (int)p + 1 : 0;
      low[rt] = is && a.window > 0 && p - a.window + 1 > 0 ? (int)(p - a.window + 1) : 0;
      slope[rt] = slopes ? slopes[qh] * kLog2e : 0.f;
      if (is) {                                  // (what the other rows give is not used)
        least = min(least, see[rt]);
        most = max(most, low[rt]);
      }
      const TS* qp = static_cast<const TS*>(a.q) + ((is ? t : sq.first) * a.Hq + qh) * D + 8 * quarter;
#pragma unroll
      for (int k = 0; k < G; ++k) load_frag(qp + 32 * k, q[rt][k]);
      m[rt] = -__builtin_huge_valf();
      l[rt] = 0.f;
#pragma unroll
      for (int n = 0; n < W; ++n) o[rt][n] = f32x4{};
    }
    least = __builtin_amdgcn_readfirstlane(half_min(least));
    most = -__builtin_amdgcn_readfirstlane(half_min(-most));
    Score<TS> sc;
    sc.mul = a.cap > 0.f ? a.scale / a.cap * (sizeof(TS) == 2 ? 2.f * kLog2e : 1.f) : a.scale * kLog2e;
    sc.cap = a.cap * kLog2e;
    bool far = false;                            // some row's m is above kFar

    const int count = (upto - from - wave + 3) / 4;          // this wave's blocks: from + wave + 4 i
    const int* pages = a.pages + (int64_t)b * a.per_seq;
    auto token0 = [&](int i) { return (sq.block0 + from + wave + 4 * i) * kBlock; };
    for (int i0 = 0; i0 < count; i0 += 64) {
      const int n = min(64, count - i0);
      // a lane finds a block's place: its number in the pool
      int64_t place = 0;
      bool there = false;
      int page = a.page;
      asm volatile("" : "+s"(page));             // (nor the reciprocal for the division by it)
      if (lane < n) {
        const uint32_t tok = (uint32_t)token0(i0 + lane);
        const int pg = pages[tok / (uint32_t)page];
        there = pg >= 0 && pg < a.npages;
        place = ((int64_t)pg * a.Hkv + head) * (page / kBlock) + tok % (uint32_t)page / kBlock;
      }
      // the blocks that are there, one bit each
      uint64_t left = __ballot(there);
      // three of them on their way or worked on, where the registers hold them
      // (one ahead of the present one does not cover the way from memory)
      constexpr int RING = RT == 1 && !(EX && D == 128) ? 3 : 2;
      Raw<D> ring[RING];
      int in[RING];
      const unsigned char* from_at = a.pool;
      auto fetch = [&](Raw<D>& r, int& i) {
        i = -1;
        if (left) {
          i = __builtin_ctzll(left);
          left &= left - 1;
          from_at = a.pool + scalar64(place, i) * Block<D>::kBytes;
        }
        // (behind the last block the same once more: with loads that are always
        // sent the compiler knows how many of them may be on their way)
        r.load(from_at, (uint32_t)again(lane));
      };
      auto work = [&](const Raw<D>& raw, int i) __attribute__((always_inline)) {
        const int j0 = token0(i0 + i);
        const bool cut = j0 + kBlock > least || j0 < most;   // some row does not see all of the block
        f32x4 s[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][0] = s[rt][1] = f32x4{};
        __builtin_amdgcn_sched_barrier(0);
        const float kl = bf_lo(raw.ks), kh = bf_hi(raw.ks), vl = bf_lo(raw.vs), vh = bf_hi(raw.vs);
        unroll<2 * G>([&](auto hg) {
          constexpr int h = hg.value / G, k = hg.value % G;
          Frag<TS> x;
          unpack_codes(raw.k[h][k], x);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const f32x4 part = mfma16(x, q[rt][k], f32x4{});
            constexpr int W0 = (h * G + k) * 2;  // words of the row of lanes: tokens 0, 1 and 2, 3 of the four
            s[rt][h][0] = fmaf(row_lane<W0>(kl), part[0], s[rt][h][0]);
            s[rt][h][1] = fmaf(row_lane<W0>(kh), part[1], s[rt][h][1]);
            s[rt][h][2] = fmaf(row_lane<W0 + 1>(kl), part[2], s[rt][h][2]);
            s[rt][h][3] = fmaf(row_lane<W0 + 1>(kh), part[3], s[rt][h][3]);
          }
          if constexpr (hg.value % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        });
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          __builtin_amdgcn_sched_barrier(0);
          const int first = j0 + 4 * (again(lane) / 16);     // this lane's tokens: first + 16 (e / 4) + e % 4
          if constexpr (EX) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float x = s[rt][e / 4][e % 4];
              x = a.cap > 0.f ? sc.cap * sc.tanh_of(x) : x * sc.mul;
              s[rt][e / 4][e % 4] = fmaf(-slope[rt], (float)(see[rt] - 1 - first - 16 * (e / 4) - e % 4), x);
            }
          }
          if (cut) {
            branch_only();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int j = first + 16 * (e / 4) + e % 4;
              if (!(j < see[rt] && j >= low[rt])) s[rt][e / 4][e % 4] = -__builtin_huge_valf();
            }
          }
          float top = s[rt][0][0];
#pragma unroll
          for (int e = 1; e < 8; ++e) top = fmaxf(top, s[rt][e / 4][e % 4]);
          if constexpr (!EX) top *= sc.mul;        // (the raw products so far; exp takes the factor with it)
          top = max_quarters(top);
          // (reference and far scores as in the attention of token rows)
          float mul = sc.mul;
          const bool rise = __any(top > m[rt] + 8.f);
          if (rise || far) {
            if (rise) {
              const float to = top > m[rt] + 8.f ? top : m[rt];
              const float c = m[rt] == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(m[rt] - to);
              m[rt] = to;
              l[rt] *= c;
#pragma unroll
              for (int n2 = 0; n2 < W; ++n2)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[rt][n2][e] *= c;
              if (!EX && !ROUND) far = __any(m[rt] != -__builtin_huge_valf() && fabsf(m[rt]) > kFar);
            }
            if (far) {
              const float ref = m[rt] == -__builtin_huge_valf() ? 0.f : m[rt];
              const bool mine = fabsf(ref) > kFar;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float y = s[rt][e / 4][e % 4];
                s[rt][e / 4][e % 4] = mine ? rounded_diff(y, sc.mul, ref) : fmaf(y, sc.mul, -ref);
              }
              mul = scalar(1.f);
            }
          }
          const float ref = far || m[rt] == -__builtin_huge_valf() ? 0.f : m[rt];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float y = s[rt][e / 4][e % 4];
            const float x = __builtin_amdgcn_exp2f(EX      ? y - ref
                                                   : ROUND ? rounded_diff(y, sc.mul, ref)
                                                           : fmaf(y, mul, -ref));
            s[rt][e / 4][e % 4] = x;
            l[rt] += x;
          }
        }
        unroll<G>([&](auto kk) {
          constexpr int k = kk.value;
          Frag<TS> x0, x1;
          unpack_codes(raw.v[2 * k], x0);
          unpack_codes(raw.v[2 * k + 1], x1);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            float p[8];
            unroll<2>([&](auto hh) {
              constexpr int h = hh.value, W0 = (h * G + k) * 2;
              p[4 * h] = row_lane<W0>(vl) * s[rt][h][0];
              p[4 * h + 1] = row_lane<W0>(vh) * s[rt][h][1];
              p[4 * h + 2] = row_lane<W0 + 1>(vl) * s[rt][h][2];
              p[4 * h + 3] = row_lane<W0 + 1>(vh) * s[rt][h][3];
            });
            if (cut) {                           // what is not seen may have any scale, NaN too
              branch_only();
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (s[rt][e / 4][e % 4] == 0.f) p[e] = 0.f;
            }
            Frag<TS> pf;
            pack_frag(p, pf);
            o[rt][2 * k] = mfma16(x0, pf, o[rt][2 * k]);
            o[rt][2 * k + 1] = mfma16(x1, pf, o[rt][2 * k + 1]);
          }
          __builtin_amdgcn_sched_barrier(0);
        });
      };
      if (!left) continue;
      unroll<RING>([&](auto k) { fetch(ring[k.value], in[k.value]); });
      for (;;) {
        work(ring[0], in[0]);
        fetch(ring[0], in[0]);
        if (in[1] < 0) break;
        work(ring[1], in[1]);
        fetch(ring[1], in[1]);
        if constexpr (RING == 3) {
          if (in[2] < 0) break;
          work(ring[2], in[2]);
          fetch(ring[2], in[2]);
        }
        if (in[0] < 0) break;
      }
    }

    // the waves' sums of each 16 rows, added in order
    const bool whole = from == 0 && upto == sq.blocks;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (from == 0 ? 1 : 0);
    const int ln = again(lane), me = wave * 64 + ln;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const auto s16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(l[rt]), __float_as_uint(l[rt]), false, false);
      float ls = __uint_as_float(s16[0]) + __uint_as_float(s16[1]);
      ls = swap32_add(ls);
      __syncthreads();
      if (ln < 16) mls[wave][ln] = make_float2(m[rt], ls);
#pragma unroll
      for (int n = 0; n < W; ++n)
        *reinterpret_cast<f32x4*>(&sums[wave][ln % 16][16 * n + 4 * (ln / 16)]) = o[rt][n];
      __syncthreads();
      for (int i = me; i < 16 * (D / 8); i += 256) {
        const int row = i / (D / 8), c = i % (D / 8) * 8;
        const int64_t ri = (int64_t)tile * ROWS + rt * 16 + row, t = sq.first + ri / g, p = sq.len - (sq.after - t);
        if (t >= sq.end || p < 0 || p >= (int64_t)a.per_seq * a.page) continue;
        float top = mls[0][row].x;
#pragma unroll
        for (int w = 1; w < 4; ++w) top = fmaxf(top, mls[w][row].x);
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, sum = 0.f;
        const float ref = top == -__builtin_huge_valf() ? 0.f : top;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float2 ml = mls[w][row];
          const float c2 = __builtin_amdgcn_exp2f(ml.x - ref);
          sum = fmaf(c2, ml.y, sum);
          float y[8];
          Vec8<float>::load(&sums[w][row][c], y);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = fmaf(c2, y[e], x[e]);
        }
        if (whole) {
          const float inv = top == -__builtin_huge_valf() && sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= inv;
          Vec8<TS>::store(static_cast<TS*>(a.k) + (t * a.Hq + head * g + ri % g) * D + c, x);
        } else {
          const int64_t to = slot * ROWS + rt * 16 + row;
          Vec8<float>::store(a.part + to * D + c, x);
          if (c == 0) a.ml[to] = make_float2(top, sum);
        }
      }
    }
    u = last;
  }
}

// Rows of the output from the places of their segments' runs, where there are
// several: a lane has eight channels of one, and its workgroup's W waves share
// the runs.
template <typename TS, int D, int W>
__global__ __launch_bounds__(64 * W) void k_cache_join(CacheArgs a, int ROWS, int64_t wgs) {
  constexpr int P = D / 8;
  __shared__ float red[W][10][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, g = a.Hq / a.Hkv;
  const int64_t t = blockIdx.x;
  const int b = sequence_of(a.starts, a.B, t, lane);
  // (t in front of the start: only where starts do not ascend; its row would lie in front of the places)
  if (b < 0 || t < a.starts[b] || t >= a.starts[b + 1]) return;
  const int64_t first = a.starts[b] > 0 ? a.starts[b] : 0;
  const int64_t p = a.lens[b] - (a.starts[b + 1] - t);
  if (p < 0 || p >= (int64_t)a.per_seq * a.page) return;
  const int64_t before = a.where[2 * b], blocks = a.where[2 * b + 1], run = a.where[2 * (int64_t)a.B];
  const int u = blockIdx.y * 64 + lane, qh = u / P, c = u % P * 8;
  const int64_t row = (t - first) * g + qh % g, tile = row / ROWS;
  const int64_t seg0 = before + (tile * a.Hkv + qh / g) * blocks;
  const int64_t w0 = seg0 / run, w1 = (seg0 + blocks - 1) / run;
  const bool is = u < a.Hq * P && w0 < w1 && w1 < wgs;       // (w1 >= wgs: only where starts do not ascend)
  auto place = [&](int64_t w) { return (2 * w + (w == w0 ? 1 : 0)) * ROWS + row % ROWS; };
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, top = -__builtin_huge_valf(), sum = 0.f;
  // adds (m, l, y) to what there is: the larger maximum is the reference
  auto add = [&](float m, float l, const float (&y)[8]) {
    const float to = fmaxf(top, m), ref = to == -__builtin_huge_valf() ? 0.f : to;
    const float c0 = __builtin_amdgcn_exp2f(top - ref), c1 = __builtin_amdgcn_exp2f(m - ref);
    sum = sum * c0 + l * c1;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] * c0 + y[e] * c1;
    top = to;
  };
  if (is) {
#pragma unroll 4
    for (int64_t w = w0 + wave; w <= w1; w += W) {
      const float2 ml = a.ml[place(w)];
      float y[8];
      Vec8<float>::load(a.part + place(w) * D + c, y);
      add(ml.x, ml.y, y);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) red[wave][e][lane] = x[e];
  red[wave][8][lane] = top;
  red[wave][9][lane] = sum;
  __syncthreads();
  if (wave != 0 || !is) return;
  for (int w = 1; w < W; ++w) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = red[w][e][lane];
    add(red[w][8][lane], red[w][9][lane], y);
  }
  const float inv = top == -__builtin_huge_valf() && sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= inv;
  Vec8<TS>::store(static_cast<TS*>(a.k) + (t * a.Hq + qh) * D + c, x);
}

CacheArgs args_of(const xhc_dims* d, const xhc_heads* h, const xhc_cache* c, const int32_t* starts,
                  const int32_t* lens, const int32_t* pages, const void* pool) {
  CacheArgs a{};
  a.starts = starts, a.lens = lens, a.pages = pages;
  a.pool = static_cast<unsigned char*>(const_cast<void*>(pool));
  a.T = d->T;
  a.Hq = h->Hq, a.Hkv = h->Hkv, a.R = h->R, a.pairs = h->pairs, a.window = h->window;
  a.page = c->page, a.npages = c->npages, a.B = c->B, a.per_seq = c->per_seq;
  a.scale = h->scale, a.cap = h->cap;
  return a;
}

template <class F> void with_width(int D, F&& f) {
  switch (D) {
    case 32: return f(Int<32>{});
    case 64: return f(Int<64>{});
    case 96: return f(Int<96>{});
    default: return f(Int<128>{});
  }
}

// tokens of a workgroup that has `per` threads' work with each: all its threads
// work, and where there are many tokens it has enough of them that finding
// their places is a small part
int tokens_of(int64_t T, int per) {
  int n = per >= 256 ? 1 : 256 / per;
  while (n < 64 && T > 2048 * (int64_t)n) n *= 2;
  return n;
}

// rows of a tile: 32 where the sequences have more than 16 on average
int tile_rows(int64_t T, int B, int g) { return T * g > 16 * (int64_t)B ? 32 : 16; }

// Workgroups: what the chip holds at a time, or one for each four blocks there can be.
int64_t attend_grid(const xhc_dims* d, const xhc_heads* h, const xhc_cache* c) {
  const int rows = tile_rows(d->T, c->B, h->Hq / h->Hkv);
  const int64_t tiles = d->T * (h->Hq / h->Hkv) / rows + (c->B < d->T ? c->B : d->T);
  const int64_t blocks = (int64_t)c->per_seq * c->page / kBlock;
  const int64_t full = 256 * attend_wgs(d->state_dtype == XHC_F32, rows);
  const int64_t units = tiles * h->Hkv;
  if (units >= 4 * full || blocks >= 4 * full) return full;
  const int64_t need = (units * blocks + 3) / 4;
  return need < full ? need : full;
}

constexpr size_t up(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t cache_bytes(const xhc_heads* h, const xhc_cache* c) {
  return (size_t)c->npages * h->Hkv * (c->page / kBlock) * (36 * h->D);
}

size_t cache_attend_ws_bytes(const xhc_dims* d, const xhc_heads* h, const xhc_cache* c) {
  const size_t slots = 2 * (size_t)attend_grid(d, h, c) * tile_rows(d->T, c->B, h->Hq / h->Hkv);
  return up(slots * h->D * 4) + up(slots * 8) + up((2 * (size_t)c->B + 1) * 8);
}

hipError_t launch_cache_append(const xhc_dims* d, const xhc_heads* h, const xhc_cache* c, const void* qkv,
                               const float* table, const int32_t* starts, const int32_t* lens, const int32_t* pages,
                               void* pool, void* q, hipStream_t s) {
  CacheArgs a = args_of(d, h, c, starts, lens, pages, pool);
  a.qkv = qkv, a.table = table, a.q = q;
  const int64_t mean = d->T / c->B;
  a.rows = (int)(mean < 1 ? 1 : mean > kBlock ? kBlock : mean);
  while ((d->T + a.rows - 1) / a.rows * h->Hkv > (1 << 22)) a.rows *= 2;   // (a launch's threads stay below 2^32)
  a.tokens = tokens_of(d->T, h->Hq * (h->D / 8));
  a.blocks = (unsigned)((d->T + a.rows - 1) / a.rows * h->Hkv);
  const dim3 grid(a.blocks + (q ? (unsigned)((d->T + a.tokens - 1) / a.tokens) : 0)), block(256);
  with_width(h->D, [&](auto D) {
    if (d->state_dtype == XHC_BF16)
      k_cache_append<uint16_t, D.value><<<grid, block, 0, s>>>(a);
    else
      k_cache_append<float, D.value><<<grid, block, 0, s>>>(a);
  });
  return hipGetLastError();
}

hipError_t launch_cache_read(const xhc_dims* d, const xhc_heads* h, const xhc_cache* c, const int32_t* starts,
                             const int32_t* lens, const int32_t* pages, const void* pool, void* k, void* v,
                             hipStream_t s) {
  CacheArgs a = args_of(d, h, c, starts, lens, pages, pool);
  a.k = k, a.v = v;
  a.tokens = tokens_of(d->T, h->Hkv * (h->D / 8));
  const dim3 grid((unsigned)((d->T + a.tokens - 1) / a.tokens)), block(256);
  with_width(h->D, [&](auto D) {
    if (d->state_dtype == XHC_BF16)
      k_cache_read<uint16_t, D.value><<<grid, block, 0, s>>>(a);
    else
      k_cache_read<float, D.value><<<grid, block, 0, s>>>(a);
  });
  return hipGetLastError();
}

hipError_t launch_cache_attend(const xhc_dims* d, const xhc_heads* h, const xhc_cache* c, const void* q,
                               const float* slopes, const int32_t* starts, const int32_t* lens, const int32_t* pages,
                               const void* pool, void* out, void* ws, hipStream_t s) {
  CacheArgs a = args_of(d, h, c, starts, lens, pages, pool);
  a.q = const_cast<void*>(q), a.k = out, a.slopes = slopes;
  const int rows = tile_rows(d->T, c->B, h->Hq / h->Hkv);
  const int64_t wgs = attend_grid(d, h, c);
  const size_t slots = 2 * (size_t)wgs * rows;
  char* p = static_cast<char*>(ws);
  a.part = reinterpret_cast<float*>(p);
  a.ml = reinterpret_cast<float2*>(p + up(slots * h->D * 4));
  a.where = reinterpret_cast<int64_t*>(p + up(slots * h->D * 4) + up(slots * 8));
  const dim3 grid((unsigned)wgs), block(256), tokens((unsigned)d->T, (unsigned)((h->Hq * (h->D / 8) + 63) / 64));
  with_width(h->D, [&](auto D) {
    auto run = [&](auto type, auto rt, auto ex) {
      k_cache_attend<decltype(type), D.value, rt.value, ex.value != 0><<<grid, block, 0, s>>>(a);
    };
    auto of = [&](auto type) {
      const bool ex = a.cap > 0.f || slopes;
      if (rows == 16)
        ex ? run(type, Int<1>{}, Int<1>{}) : run(type, Int<1>{}, Int<0>{});
      else
        ex ? run(type, Int<2>{}, Int<1>{}) : run(type, Int<2>{}, Int<0>{});
      // (few tokens have many runs each: 16 waves take 5 us where four take 13, at one token of 131072)
      if (d->T <= 16)
        k_cache_join<decltype(type), D.value, 16><<<tokens, dim3(1024), 0, s>>>(a, rows, wgs);
      else
        k_cache_join<decltype(type), D.value, 4><<<tokens, block, 0, s>>>(a, rows, wgs);
    };
    d->state_dtype == XHC_BF16 ? of(uint16_t{}) : of(float{});
  });
  return hipGetLastError();
}

}  // namespace xhc
