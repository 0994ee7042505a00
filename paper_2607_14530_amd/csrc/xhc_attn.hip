// Attention of token rows, its spans and its rotation:
//
//   s_ij = cap tanh(scale q_i k_j / cap) - slope |i - j|,  lo_i <= j < hi_i
//   p_i = softmax_j s_ij,  o_i = sum_j p_ij v_j,  lse_i = log2 sum_j exp s_ij
//
// Forward (k_attn): a workgroup takes 128 queries of a head, a wave 32 of them,
// and goes once over the keys that its rows see, 64 at a time, with the running
// maximum and sum of each row.  T = 16384 in two sequences, Hq = 32, Hkv = 8,
// D = 128, bf16: 1.11 to 1.17 ms, 0.94 to 0.99 PFLOP/s of the pairs that are seen,
// with the matrix cores busy for 47 % of the cycles, the vector ones for 63 %, at a
// clock that power holds near 1.9 GHz; no bank conflicts.  8190 tokens in 23
// documents, Hq = 16, D = 64: 44 us, where the matrix cores are busy for 9 % and
// a workgroup's start, with its first copies, and the longest documents count.
#include <float.h>

#include "xhc_attn.h"
#include "xhc_spans.h"

namespace xhc {

namespace {

constexpr float kNoKey = -__builtin_huge_valf();

// With NC = 2 a workgroup takes 64 queries, and two waves share 32 of them: each
// has one block of 32 keys of every tile, and their sums are joined at the end.
// That halves the way through the longest rows' keys, which counts where the
// chip holds all workgroups at once.
// MODE: 0 products times a factor, 1 capped, 2 with a bias or (fp32) capped
template <typename TS, int D, int MODE, int NC>
__global__ __launch_bounds__(64 * kAttnWaves, sizeof(TS) == 2 ? 2 : 1) void k_attn(AttnArgs a) {
  using TL = Tile<TS, D>;
  constexpr int KS = D / 16, F = D / 32, AHEAD = sizeof(TS) == 2 ? 4 : 2;
  constexpr int ROWS = 128 / NC, RW = kAttnWaves / NC, NB = 2 / NC;   // blocks of keys of a wave
  __shared__ __align__(1024) unsigned char lds[4 * TL::kBytes];
  __shared__ int4 red[kAttnWaves];
  __shared__ uint64_t bits[2];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  int head, tile;
  attn_place(a.Hq, (int)((a.T + ROWS - 1) / ROWS), head, tile);
  const int kc = NC == 1 ? 0 : wave / RW;        // which of the keys' blocks
  const int kvh = head / (a.Hq / a.Hkv), H = a.Hq + 2 * a.Hkv;
  const int t = tile * ROWS + wave % RW * 32 + lane % 32, T1 = (int)a.T - 1;
  const bool row = t <= T1;
  const int2 see = span_of(a, t);
  int2 own;
  const int4 ex = attn_extremes(a, tile * ROWS, ROWS, tile * ROWS + wave % RW * 32, see, row, red, wave, lane, own);
  const uint32_t stride = (uint32_t)H * D * sizeof(TS);
  const unsigned char* base = reinterpret_cast<const unsigned char*>(a.qkv);
  const unsigned char* kb = base + (size_t)(a.Hq + kvh) * D * sizeof(TS);
  const unsigned char* vb = kb + (size_t)a.Hkv * D * sizeof(TS);
  const uint32_t at = lds_offset(lds);

  f32x16 o[F];
#pragma unroll
  for (int f = 0; f < F; ++f) o[f] = f32x16{};
  float m = kNoKey, l = 0.f;
  const int first = ex.x / kTile, end = (ex.y + kTile - 1) / kTile;
  if (ex.x < ex.y) {
    Score<TS> sc;
    sc.init(a, head);
    bool far = false;                            // some row's m is above kFar
    Frag<TS> q[KS];
    const TS* qp = reinterpret_cast<const TS*>(base) + (int64_t)(row ? t : T1) * H * D + head * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) load_frag(qp + 16 * ks + 8 * (lane / 32), q[ks]);
    TL::copy(kb, stride, first * kTile, T1, at, wave, lane);
    TL::copy(vb, stride, first * kTile, T1, at + TL::kBytes, wave, lane);
    for (int kt = first; kt < end; ++kt) {
      const uint32_t off = (kt - first) % 2 * 2 * TL::kBytes, next = 2 * TL::kBytes - off;
      unsigned char *K = lds + off, *V = K + TL::kBytes;
      const int j0 = kt * kTile;
      const bool cut = j0 < ex.z || j0 + kTile > ex.w;      // some row does not see all of the tile
      wait_loads();
      if (cut) TL::clean(V, bits + (kt - first) % 2, wave, again(lane));
      lds_barrier();
      if (kt + 1 < end) {
        const int ln = again(lane);
        TL::copy(kb, stride, (kt + 1) * kTile, T1, at + next, wave, ln);
        TL::copy(vb, stride, (kt + 1) * kTile, T1, at + next + TL::kBytes, wave, ln);
      }
      const uint64_t bad = cut ? bits[(kt - first) % 2] : 0;
      if (j0 >= own.y || j0 + kTile <= own.x) continue;     // no row of this wave sees a key of the tile
      f32x16 s[NB];
#pragma unroll
      for (int rb = 0; rb < NB; ++rb) s[rb] = f32x16{};
      int ln = again(lane);
      feed<NB * KS, AHEAD, Frag<TS>>(
          [&](auto i, Frag<TS>& k) { TL::row_frag(K, kc + i.value / KS, i.value % KS, ln, k); },
          [&](auto i, Frag<TS>& k) { s[i.value / KS] = mfma32(k, q[i.value % KS], s[i.value / KS]); });
      const int j1 = j0 + 32 * kc + 4 * (lane / 32);          // a lane's keys: j1 + 32 rb + sum_row(r)
      if constexpr (MODE == 2) {
        const float d0 = (float)(t - j1);
#pragma unroll
        for (int rb = 0; rb < NB; ++rb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float x = a.cap > 0.f ? sc.cap * sc.tanh_of(s[rb][r]) : s[rb][r] * sc.mul;
            s[rb][r] = fmaf(-sc.slope, fabsf(d0 - (float)(32 * rb + sum_row(r))), x);
          }
      }
      if (cut) {
        branch_only();
        const int lo = see.x - j1, hi = see.y - j1;
#pragma unroll
        for (int rb = 0; rb < NB; ++rb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int j = 32 * rb + sum_row(r);
            if (MODE == 1 && s[rb][r] == kNoKey) s[rb][r] = -FLT_MAX;      // seen, with a score of -cap
            if (!(j >= lo && j < hi)) s[rb][r] = kNoKey;
          }
        if (bad) {
#pragma unroll
          for (int rb = 0; rb < NB; ++rb) {
            const uint32_t keys = (uint32_t)(bad >> (32 * (kc + rb))) >> (4 * (lane / 32));
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if ((keys >> sum_row(r) & 1) && s[rb][r] != kNoKey) s[rb][r] = __builtin_nanf("");
          }
        }
      }
      float top = s[0][0];
#pragma unroll
      for (int rb = 0; rb < NB; ++rb)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[rb][r]);
      top = max_halves(top);
      // (s: still the raw products where the scores rise with them)
      if (MODE == 0) top *= sc.mul;
      if (MODE == 1 && (!cut || top != kNoKey)) top = fmaf(-2.f * sc.cap, sc.share_of(top), sc.cap);
      // The row's reference only follows its maximum when that is 2^8 above it:
      // probabilities up to 256 are as exact, and sums are rarely rescaled.
      // Far scores: the exponents are formed in the branch, and 1 times them less 0
      // is what exp2 then takes (so that the way of all others stays as it is).
      float ref = m == kNoKey ? 0.f : m, mul = sc.mul;      // (a row that has seen nothing: exp2(-inf) = 0)
      const bool rise = __any(top > m + 8.f);
      if (rise || (MODE == 0 && far)) {
        if (rise) {
          const float to = top > m + 8.f ? top : m;           // (from -inf: the first maximum)
          const float c = m == kNoKey ? 0.f : __builtin_amdgcn_exp2f(m - to);
          m = to;
          l *= c;
#pragma unroll
          for (int f = 0; f < F; ++f)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[f][r] *= c;
          if (MODE == 0) far = __any(m != kNoKey && fabsf(m) > kFar);
        }
        ref = m == kNoKey ? 0.f : m;
        if (MODE == 0 && far) {
          const bool mine = fabsf(m) > kFar;
#pragma unroll
          for (int rb = 0; rb < NB; ++rb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              s[rb][r] = mine ? rounded_diff(s[rb][r], sc.mul, ref) : fmaf(s[rb][r], sc.mul, -ref);
          mul = scalar(1.f);
          ref = 0.f;
        }
      }
#pragma unroll
      for (int rb = 0; rb < NB; ++rb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = s[rb][r];
          s[rb][r] = __builtin_amdgcn_exp2f(MODE == 2   ? x - ref
                                            : MODE == 0 ? fmaf(x, mul, -ref)
                                                        : fmaf(-2.f * sc.cap, sc.share_of(x), sc.cap - ref));
          if (MODE == 1 && cut && x == kNoKey) s[rb][r] = 0.f;           // (the cap has its say there too)
        }
      ln = again(lane);
      Frag<TS> p;
      feed<2 * NB * F, AHEAD, Frag<TS>>(
          [&](auto i, Frag<TS>& v) { TL::col_frag(V, i.value % F, 2 * kc + i.value / F, ln, v); },
          [&](auto i, Frag<TS>& v) {
            constexpr int st = i.value / F, f = i.value % F;
            if constexpr (f == 0) {
              sums_frag(s[st / 2], st % 2, p);
              l = add_frag(p, l);                // (the sum of what the values are multiplied with)
            }
            o[f] = mfma32(v, p, o[f]);
          });
    }
  }
  if constexpr (NC == 2) {
    __syncthreads();
    float* part = reinterpret_cast<float*>(lds) + wave % RW * (F * 16 + 2) * 64 + lane;
    if (kc == 1) {
      part[0] = m;
      part[64] = l;
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) part[(2 + 16 * f + r) * 64] = o[f][r];
    }
    __syncthreads();
    if (kc == 1) return;
    const float m1 = part[0], to = fmaxf(m, m1), ref = to == kNoKey ? 0.f : to;
    const float c0 = __builtin_amdgcn_exp2f(m - ref), c1 = __builtin_amdgcn_exp2f(m1 - ref);
    m = to;
    l = l * c0 + part[64] * c1;
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[f][r] = o[f][r] * c0 + part[(2 + 16 * f + r) * 64] * c1;
  }
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const float inv = see.x < see.y ? 1.f / l : 0.f;
  TS* op = reinterpret_cast<TS*>(a.out) + ((int64_t)t * a.Hq + head) * D;
#pragma unroll
  for (int f = 0; f < F; ++f)
    store_sums<TS>(o[f], inv, op + 32 * f, row, lane,
                   a.low ? reinterpret_cast<TS*>(a.low) + ((int64_t)t * a.Hq + head) * D + 32 * f : nullptr);
  if (a.lse && row && lane < 32)
    a.lse[(int64_t)head * a.Tp + t] = see.x < see.y ? m + __builtin_amdgcn_logf(l) : kNoKey;
}

// The spans of documents, by one thread each token.  Document i holds the
// tokens starts[i] .. starts[i + 1] - 1; its first prefix[i] see one another.
__global__ __launch_bounds__(256) void k_attn_spans(int64_t T, int64_t S, int window, int n, const int* starts,
                                                    const int* prefix, int2* span) {
  const int64_t t64 = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t64 >= T) return;
  const int t = (int)t64;
  int from = t - (int)(t % S), hi = t + 1;
  if (starts) {
    const int a = last_start(starts, n, t);
    if (starts[0] > t || a == n) {
      span[t] = make_int2(0, 0);
      return;
    }
    const int64_t s0 = starts[a], s1 = starts[a + 1] < T ? starts[a + 1] : T;
    from = s0 > 0 ? (int)s0 : 0;
    if (prefix) {
      const int64_t p = s0 + prefix[a] < s1 ? s0 + prefix[a] : s1;
      if (p > hi) hi = (int)p;
    }
  }
  if (window > 0 && t - window + 1 > from) from = t - window + 1;
  span[t] = make_int2(from, hi);
}

// A thread takes 16 channels of a head: eight pairs, or sixteen behind the
// rotated ones; eight or fewer threads a head, the heads of a token (or of
// several) side by side, so that a workgroup reads runs.  Bound by HBM: 68 us
// for 2 x 201 MB (T = 16384, Hq = 32, Hkv = 8, D = 128, bf16), 5.9 TB/s.
template <typename TS>
__global__ __launch_bounds__(256) void k_rotate(int64_t T, int64_t S, int H, int Hrot, int D, int R, int pairs,
                                                const TS* src, const int* pos, const float* table, int64_t positions,
                                                float sign, TS* dst, int heads, int tokens) {
  const int per = D / 16, j = threadIdx.x % per, slot = threadIdx.x / per;
  const int64_t t = (int64_t)blockIdx.x * tokens + slot / heads;
  if (slot / heads >= tokens || t >= T) return;
  const int64_t p = pos ? pos[t] : t % S;
  const bool turned = 16 * j < R && p >= 0 && p < positions;
  float cs[16];
  if (turned) {
    Vec8<float>::load(table + p * R + 16 * j, *reinterpret_cast<float(*)[8]>(cs));
    Vec8<float>::load(table + p * R + 16 * j + 8, *reinterpret_cast<float(*)[8]>(cs + 8));
  }
  for (int h = slot % heads; h < H; h += heads) {
    const bool now = turned && h < Hrot;
    if (!now && src == dst) continue;
    const int64_t at = (t * H + h) * D;
    const bool split = now && !pairs;        // halves: channels 8 j .. + 8 with R / 2 + 8 j .. + 8
    const int xa = split ? 8 * j : 16 * j, xb = split ? 8 * j + R / 2 : 16 * j + 8;
    float a[8], b[8];
    Vec8<TS>::load(src + at + xa, a);
    Vec8<TS>::load(src + at + xb, b);
    if (split) {
      turn<8>(a, b, cs, sign);
    } else if (now) {                        // neighbours: a and b hold four pairs each
      float x[8], y[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = a[2 * i], y[i] = a[2 * i + 1];
        x[4 + i] = b[2 * i], y[4 + i] = b[2 * i + 1];
      }
      turn<8>(x, y, cs, sign);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[2 * i] = x[i], a[2 * i + 1] = y[i];
        b[2 * i] = x[4 + i], b[2 * i + 1] = y[4 + i];
      }
    }
    Vec8<TS>::store(dst + at + xa, a);
    Vec8<TS>::store(dst + at + xb, b);
  }
}

template <typename TS, int D> hipError_t run_attn(const AttnArgs& a, hipStream_t s) {
  const int nc = attn_parts(a.T, a.Hq);
  const dim3 grid((unsigned)((a.T + 128 / nc - 1) / (128 / nc) * a.Hq)), block(64 * kAttnWaves);
  const int mode = a.slopes || (a.cap > 0.f && sizeof(TS) == 4) ? 2 : a.cap > 0.f ? 1 : 0;
  auto run = [&](auto m, auto n) { k_attn<TS, D, m.value, n.value><<<grid, block, 0, s>>>(a); };
  auto of = [&](auto n) {
    if (mode == 2) return run(Int<2>{}, n);
    if constexpr (sizeof(TS) == 2)
      if (mode == 1) return run(Int<1>{}, n);
    run(Int<0>{}, n);
  };
  nc == 1 ? of(Int<1>{}) : of(Int<2>{});
  return hipGetLastError();
}

template <typename TS> hipError_t run_attn_of(int D, const AttnArgs& a, hipStream_t s) {
  switch (D) {
    case 32: return run_attn<TS, 32>(a, s);
    case 64: return run_attn<TS, 64>(a, s);
    case 96: return run_attn<TS, 96>(a, s);
    default: return run_attn<TS, 128>(a, s);
  }
}

constexpr int64_t padded(int64_t T) { return (T + kTile - 1) / kTile * kTile; }

}  // namespace

size_t attn_lse_bytes(int64_t T, int Hq) { return ((size_t)padded(T) * Hq * 4 + 255) / 256 * 256; }
size_t attn_saved_bytes(int state_dtype, int64_t T, int Hq, int D) {
  return attn_lse_bytes(T, Hq) + (state_dtype == XHC_BF16 ? (size_t)T * Hq * D * 2 : 0);
}

hipError_t launch_attn(const xhc_dims* d, const xhc_heads* h, const void* qkv, const int32_t* span,
                       const float* slopes, void* out, void* saved, hipStream_t s) {
  AttnArgs a{};
  a.qkv = qkv;
  a.span = reinterpret_cast<const int2*>(span);
  a.slopes = slopes;
  a.out = out;
  a.T = d->T, a.S = d->S, a.Tp = padded(d->T);
  if (saved) {
    a.lse = static_cast<float*>(saved);
    if (d->state_dtype == XHC_BF16)
      a.low = reinterpret_cast<uint16_t*>(static_cast<char*>(saved) + attn_lse_bytes(d->T, h->Hq));
  }
  a.Hq = h->Hq, a.Hkv = h->Hkv, a.window = h->window;
  a.scale = h->scale, a.cap = h->cap;
  return d->state_dtype == XHC_BF16 ? run_attn_of<uint16_t>(h->D, a, s) : run_attn_of<float>(h->D, a, s);
}

hipError_t launch_attn_spans(int64_t T, int64_t S, int window, int n, const int32_t* starts, const int32_t* prefix,
                             int32_t* span, hipStream_t s) {
  k_attn_spans<<<dim3((unsigned)((T + 255) / 256)), dim3(256), 0, s>>>(T, S, window, n, starts, prefix,
                                                                      reinterpret_cast<int2*>(span));
  return hipGetLastError();
}

hipError_t launch_rotate(const xhc_dims* d, const xhc_heads* h, const void* src, const int32_t* pos,
                         const float* table, int64_t positions, bool inverse, void* dst, hipStream_t s) {
  const int H = h->Hq + 2 * h->Hkv, slots = 256 / (h->D / 16);
  const int heads = H < slots ? H : slots, tokens = slots / heads;
  const dim3 grid((unsigned)((d->T + tokens - 1) / tokens)), block(256);
  const float sign = inverse ? -1.f : 1.f;
  if (d->state_dtype == XHC_BF16)
    k_rotate<uint16_t><<<grid, block, 0, s>>>(d->T, d->S, H, h->Hq + h->Hkv, h->D, h->R, h->pairs,
                                              static_cast<const uint16_t*>(src), pos, table, positions, sign,
                                              static_cast<uint16_t*>(dst), heads, tokens);
  else
    k_rotate<float><<<grid, block, 0, s>>>(d->T, d->S, H, h->Hq + h->Hkv, h->D, h->R, h->pairs,
                                           static_cast<const float*>(src), pos, table, positions, sign,
                                           static_cast<float*>(dst), heads, tokens);
  return hipGetLastError();
}

}  // namespace xhc
