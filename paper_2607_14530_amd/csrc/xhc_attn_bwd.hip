// Reverse of the attention of token rows, given do:
//
//   p_ij = exp2(s_ij - lse_i),  delta_i = sum_c do_ic o_ic,  dP_ij = do_i v_j
//   dS_ij = p_ij (dP_ij - delta_i) d s_ij / d (scale q_i k_j)
//   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i p_ij do_i
//
// Two kernels form the probabilities again, each with the sums that it owns in
// registers: k_attn_dq as the forward goes, k_attn_dkv with a wave's 32 keys
// fixed and the queries of all heads of the group passing by.  That is seven
// products in place of five, but no sum is shared between workgroups: no
// atomics, no fp32 copy of dq, and an order that only the sizes fix.  T = 16384
// in two sequences, Hq = 32, Hkv = 8, D = 128, bf16: k_attn_prep 73 us (5.5
// TB/s), k_attn_dkv 2.2 ms and k_attn_dq 1.5 ms (1.0 PFLOP/s of their products,
// the matrix cores busy for 45 and 55 % of the cycles; the clock as forward).
#include <float.h>

#include "xhc_attn.h"

namespace xhc {

namespace {

// Tile blockIdx.x of 64 rows: for head blockIdx.y < Hq the rows' delta; in the
// last of them the spans and what they have in common.  A bf16 out is taken
// with what its rounding left, which the forward has saved: rounded, it raised
// the error of dq and dk by a twentieth of theirs.
template <typename TS, int D>
__global__ __launch_bounds__(256) void k_attn_prep(AttnArgs a, float* delta, int* lo, int* hi, int4* range) {
  constexpr int LP = D == 96 ? 16 : D / 8;       // lanes of a row
  const int tile = blockIdx.x, head = blockIdx.y, t0 = tile * kTile;
  if (head == a.Hq) {
    if (threadIdx.x >= 64) return;
    const int t = t0 + threadIdx.x;
    const int2 s = span_of(a, t);
    const bool some = s.x < s.y;
    lo[t] = s.x;
    hi[t] = s.y;
    int4 e = make_int4(some ? s.x : INT32_MAX, some ? s.y : 0, some ? s.x : INT32_MAX, some ? s.y : 0);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      e.x = min(e.x, __shfl_xor(e.x, d));
      e.y = max(e.y, __shfl_xor(e.y, d));
      e.z = max(e.z, __shfl_xor(e.z, d));
      e.w = min(e.w, __shfl_xor(e.w, d));
    }
    if (threadIdx.x == 0) range[tile] = e;
    return;
  }
  const int c = threadIdx.x % LP * 8;
#pragma unroll
  for (int r = threadIdx.x / LP; r < kTile; r += 256 / LP) {
    const int t = t0 + r;
    float sum = 0.f;
    if (t < a.T && c < D) {
      const int64_t at = ((int64_t)t * a.Hq + head) * D + c;
      float x[8], y[8];
      Vec8<TS>::load(reinterpret_cast<const TS*>(a.out) + at, x);
      Vec8<TS>::load(reinterpret_cast<const TS*>(a.dout) + at, y);
      if (sizeof(TS) == 2) {
        float z[8];
        Vec8<uint16_t>::load(a.low + at, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += z[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(x[i], y[i], sum);
    }
#pragma unroll
    for (int d = 1; d < LP; d *= 2) sum += __shfl_xor(sum, d);
    if (threadIdx.x % LP == 0) delta[(int64_t)head * a.Tp + t] = sum;
  }
}

// p and dS of N pairs from the raw products and dP; dist, lse, delta: of pair r.
// The score is rounded as the forward rounds it (and a far one's largest is then lse).
// A cap is asked for once for them all: asked for with each pair, its two ways
// kept more than the registers hold, and at D = 128 k_attn_dkv went through
// scratch memory (backward of T = 8192, Hq = 32, Hkv = 8, cap 30: 2960 us instead
// of 2490; with a bias at D = 64, Hq = 16, Hkv = 4: 970 instead of 664).
template <typename TS, int N, class I, class L, class E>
__device__ __forceinline__ void reverse_scores(float* x, float* dp, const Score<TS>& sc, bool capped, I&& dist, L&& lse,
                                               E&& delta) {
  if (capped) {
    branch_only();
#pragma unroll
    for (int r = 0; r < N; ++r) {
      float der;
      x[r] = sc.cap * sc.tanh_of(x[r], der);
      dp[r] = (dp[r] - delta(r)) * der;
    }
  } else {
    branch_only();
#pragma unroll
    for (int r = 0; r < N; ++r) {
      x[r] *= sc.mul;
      dp[r] -= delta(r);
    }
  }
#pragma unroll
  for (int r = 0; r < N; ++r) {
    x[r] = __builtin_amdgcn_exp2f(fmaf(-sc.slope, dist(r), x[r]) - lse(r));
    dp[r] *= x[r];
  }
}

// (NC as in k_attn)
template <typename TS, int D, bool EX, int NC>
__global__ __launch_bounds__(64 * kAttnWaves, sizeof(TS) == 2 ? 2 : 1) void k_attn_dq(AttnArgs a) {
  using TL = Tile<TS, D>;
  constexpr int KS = D / 16, F = D / 32, AHEAD = sizeof(TS) == 2 ? 4 : 2;
  constexpr int ROWS = 128 / NC, RW = kAttnWaves / NC, NB = 2 / NC;
  __shared__ __align__(1024) unsigned char lds[4 * TL::kBytes];
  __shared__ int4 red[kAttnWaves];
  __shared__ uint64_t bits[2];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  int head, tile;
  attn_place(a.Hq * a.qslices, (int)((a.T + ROWS - 1) / ROWS), head, tile);
  const int slice = head % a.qslices;
  head /= a.qslices;
  const int kc = NC == 1 ? 0 : wave / RW;
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

  f32x16 dq[F];
#pragma unroll
  for (int f = 0; f < F; ++f) dq[f] = f32x16{};
  int first = ex.x / kTile, end = (ex.y + kTile - 1) / kTile;
  if (a.qslices > 1) {                           // the keys of this slice
    const int n = end - first, of = first;
    first = of + n * slice / a.qslices;
    end = of + n * (slice + 1) / a.qslices;
  }
  if (ex.x < ex.y && first < end) {
    Score<TS> sc;
    sc.init(a, head);
    const int64_t tc = row ? t : T1;
    float lse = a.lse[(int64_t)head * a.Tp + tc];
    const float delta = a.delta[(int64_t)head * a.Tp + tc];
    // where scores are far: the exponents are formed in a branch, and 1 times them
    // less 0 is what exp2 then takes
    const bool far = !EX && __any(fabsf(lse) > kFar && fabsf(lse) <= FLT_MAX);
    const float mul = scalar(far ? 1.f : sc.mul);
    if (far) lse = 0.f;
    Frag<TS> q[KS], go[KS];
    const TS* qp = reinterpret_cast<const TS*>(base) + tc * H * D + head * D;
    const TS* gp = reinterpret_cast<const TS*>(a.dout) + (tc * a.Hq + head) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      load_frag(qp + 16 * ks + 8 * (lane / 32), q[ks]);
      load_frag(gp + 16 * ks + 8 * (lane / 32), go[ks]);
    }
    TL::copy(kb, stride, first * kTile, T1, at, wave, lane);
    TL::copy(vb, stride, first * kTile, T1, at + TL::kBytes, wave, lane);
    for (int kt = first; kt < end; ++kt) {
      const uint32_t off = (kt - first) % 2 * 2 * TL::kBytes, next = 2 * TL::kBytes - off;
      unsigned char *K = lds + off, *V = K + TL::kBytes;
      const int j0 = kt * kTile;
      const bool cut = j0 < ex.z || j0 + kTile > ex.w;
      wait_loads();
      if (cut) TL::clean(K, bits + (kt - first) % 2, wave, again(lane));
      lds_barrier();
      if (kt + 1 < end) {
        const int ln = again(lane);
        TL::copy(kb, stride, (kt + 1) * kTile, T1, at + next, wave, ln);
        TL::copy(vb, stride, (kt + 1) * kTile, T1, at + next + TL::kBytes, wave, ln);
      }
      const uint64_t bad = cut ? bits[(kt - first) % 2] : 0;
      const bool none = j0 >= own.y || j0 + kTile <= own.x;   // no row of this wave sees a key of the tile
#pragma unroll 1
      for (int rb = none ? 2 : kc; rb < kc + NB; ++rb) {
        const int ln = again(lane);
        f32x16 s = f32x16{}, dp = f32x16{};
        feed<2 * KS, AHEAD, Frag<TS>>(
            [&](auto i, Frag<TS>& k) { TL::row_frag(i.value < KS ? K : V, rb, i.value % KS, ln, k); },
            [&](auto i, Frag<TS>& k) {
              if constexpr (i.value < KS)
                s = mfma32(k, q[i.value], s);
              else
                dp = mfma32(k, go[i.value - KS], dp);
            });
        const int j1 = j0 + 32 * rb + 4 * (ln / 32);         // this lane's keys: j1 + sum_row(r)
        if constexpr (EX) {
          const float d0 = (float)(t - j1);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x[4], y[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = s[4 * i + r], y[r] = dp[4 * i + r];
            reverse_scores<TS, 4>(x, y, sc, a.cap > 0.f,
                                  [&](int r) { return fabsf(d0 - (float)sum_row(4 * i + r)); },
                                  [&](int) { return lse; }, [&](int) { return delta; });
#pragma unroll
            for (int r = 0; r < 4; ++r) dp[4 * i + r] = y[r];
          }
        } else {
          if (far) {
            branch_only();
            const float of = a.lse[(int64_t)head * a.Tp + (row ? t : T1)];
            const bool mine = fabsf(of) > kFar;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = mine ? rounded_diff(s[r], sc.mul, of) : fmaf(s[r], sc.mul, -of);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r)
            dp[r] = __builtin_amdgcn_exp2f(fmaf(s[r], mul, -lse)) * (dp[r] - delta);
        }
        if (bad) {
          branch_only();
          const uint32_t keys = (uint32_t)(bad >> (32 * rb)) >> (4 * (ln / 32));
#pragma unroll
          for (int r = 0; r < 16; ++r) dp[r] += keys >> sum_row(r) & 1 ? __builtin_nanf("") : 0.f;
        }
        if (cut) {
          branch_only();
          const int lo = see.x - j1, hi = see.y - j1;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (!(sum_row(r) >= lo && sum_row(r) < hi)) dp[r] = 0.f;
        }
        Frag<TS> ds;
        feed<2 * F, AHEAD, Frag<TS>>(
            [&](auto i, Frag<TS>& k) { TL::col_frag(K, i.value % F, 2 * rb + i.value / F, ln, k); },
            [&](auto i, Frag<TS>& k) {
              if constexpr (i.value % F == 0) sums_frag(dp, i.value / F, ds);
              dq[i.value % F] = mfma32(k, ds, dq[i.value % F]);
            });
      }
    }
  }
  if constexpr (NC == 2) {
    __syncthreads();
    float* part = reinterpret_cast<float*>(lds) + wave % RW * F * 16 * 64 + lane;
    if (kc == 1) {
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) part[(16 * f + r) * 64] = dq[f][r];
    }
    __syncthreads();
    if (kc == 1) return;
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[f][r] += part[(16 * f + r) * 64];
  }
  if (a.qslices > 1) {
    float* p = a.part + (((int64_t)slice * a.T + t) * a.Hq + head) * D;
#pragma unroll
    for (int f = 0; f < F; ++f) store_sums<float>(dq[f], a.scale, p + 32 * f, row, lane);
    return;
  }
  TS* p = reinterpret_cast<TS*>(a.dqkv) + (int64_t)t * H * D + head * D;
#pragma unroll
  for (int f = 0; f < F; ++f) store_sums<TS>(dq[f], a.scale, p + 32 * f, row, lane);
}

// A stage of k_attn_dkv: a tile of queries and of do, and lse, delta, lo and hi
// of their rows.
template <typename TL> struct QStage {
  static constexpr int kRows = 2 * TL::kBytes, kBytes = kRows + 1024;
};

// Waves of a workgroup of k_attn_dkv.  At D = 128, bf16, a wave's sums and the
// fragments that it keeps do not fit the 256 registers that two waves a SIMD
// leave it: the values' last PARKED fragments lie in LDS, which one workgroup
// of eight waves a CU has room for (two of four waves, three parked: 2.33 ms at
// T = 16384, Hq = 32, Hkv = 8 with its instructions one after another, which
// those registers asked for).
constexpr int dkv_waves(bool f32, int D) { return !f32 && D == 128 ? 8 : 4; }

template <typename TS, int D, bool EX>
__global__ __launch_bounds__(64 * dkv_waves(sizeof(TS) == 4, D), sizeof(TS) == 2 ? 2 : 1) void k_attn_dkv(AttnArgs a) {
  constexpr int NW = dkv_waves(sizeof(TS) == 4, D), KEYS = 32 * NW;
  using TL = Tile<TS, D, NW>;
  using ST = QStage<TL>;
  constexpr int KS = D / 16, F = D / 32, AHEAD = 2, PARKED = NW == 8 ? 7 : 0;
  __shared__ __align__(1024) unsigned char lds[2 * ST::kBytes + PARKED * NW * 1024];
  __shared__ uint64_t bits[2];
  __shared__ int reach[2];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int g = a.Hq / a.Hkv, shares = a.parts / a.slices, mine = g / shares, H = a.Hq + 2 * a.Hkv;
  const int tiles = (int)((a.T + KEYS - 1) / KEYS), qtiles = (int)(a.Tp / kTile);
  int which, tile;
  attn_place(a.Hkv * a.parts, tiles, which, tile);
  tile = tiles - 1 - tile;                       // the first keys are seen by most queries
  const int kvh = which / a.parts, part = which % a.parts;
  const int head0 = kvh * g + part % shares * mine, slice = part / shares;
  const int j0 = tile * KEYS, T1 = (int)a.T - 1;
  const int key = j0 + wave * 32 + lane % 32;
  const bool row = key <= T1;
  const unsigned char* qb = reinterpret_cast<const unsigned char*>(a.qkv);
  const unsigned char* gb = reinterpret_cast<const unsigned char*>(a.dout);
  const uint32_t qstride = (uint32_t)H * D * sizeof(TS), gstride = (uint32_t)a.Hq * D * sizeof(TS);
  const uint32_t at = lds_offset(lds);

  // The first and last tile of queries of which some row sees one of these keys.
  // Each workgroup reads the ranges of all tiles, out of its XCD's L2 (in sequences
  // of 512, Hq = 16, Hkv = 4, D = 64, where the work itself grows with T alone, a backward
  // takes 168 us for 16384 of T = 2^17 tokens and 164 for as many of 2^19).
  if (threadIdx.x < 2) reach[threadIdx.x] = threadIdx.x ? -1 : INT32_MAX;
  __syncthreads();
  auto sees = [&](const int4& e) { return e.x < j0 + KEYS && e.y > j0 && e.x < e.y; };
  int from = INT32_MAX, upto = -1;
  for (int i = threadIdx.x; i < qtiles; i += 64 * NW)
    if (sees(a.range[i])) {
      from = min(from, i);
      upto = max(upto, i);
    }
  if (upto >= 0) {
    atomicMin(&reach[0], from);
    atomicMax(&reach[1], upto);
  }
  __syncthreads();
  from = __builtin_amdgcn_readfirstlane(reach[0]);
  upto = __builtin_amdgcn_readfirstlane(reach[1]);
  if (a.slices > 1 && from <= upto) {            // the queries of this slice
    const int n = upto - from + 1, of = from;
    from = of + n * slice / a.slices;
    upto = of + n * (slice + 1) / a.slices - 1;
  }

  f32x16 dk[F], dv[F];
#pragma unroll
  for (int f = 0; f < F; ++f) dk[f] = dv[f] = f32x16{};
  if (from <= upto) {
    Frag<TS> kf[KS], vf[KS];
    const TS* kp = reinterpret_cast<const TS*>(qb) + ((int64_t)(row ? key : T1) * H + a.Hq + kvh) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      load_frag(kp + 16 * ks + 8 * (lane / 32), kf[ks]);
      load_frag(kp + (int64_t)a.Hkv * D + 16 * ks + 8 * (lane / 32), vf[ks]);
    }
    Frag<TS>* parked = reinterpret_cast<Frag<TS>*>(lds + 2 * ST::kBytes) + wave * PARKED * 64;
#pragma unroll
    for (int i = 0; i < PARKED; ++i) parked[i * 64 + lane] = vf[KS - PARKED + i];
    auto copy = [&](int head, int qt, uint32_t to) {
      const int ln = again(lane);
      TL::copy(qb + (size_t)head * D * sizeof(TS), qstride, qt * kTile, T1, to, wave, ln);
      TL::copy(gb + (size_t)head * D * sizeof(TS), gstride, qt * kTile, T1, to + TL::kBytes, wave, ln);
      const int64_t r = (int64_t)qt * kTile + ln;
      if (wave >= 4) return;
      const void* p = wave == 0   ? (const void*)(a.lse + (int64_t)head * a.Tp + r)
                      : wave == 1 ? (const void*)(a.delta + (int64_t)head * a.Tp + r)
                      : wave == 2 ? (const void*)(a.lo + r)
                                  : (const void*)(a.hi + r);
      lds_dma4(p, to + ST::kRows + wave * 256);
    };
    // a tile's range, on its way in one register: four lanes have a part each
    auto range_at = [&](int i) { return reinterpret_cast<const int*>(a.range + i)[lane % 4]; };
    auto scalars = [](int x) {
      return make_int4(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 1),
                       __builtin_amdgcn_readlane(x, 2), __builtin_amdgcn_readlane(x, 3));
    };
    // the tile behind (head, qt); head == head0 + mine: none
    auto behind = [&](int& head, int& qt) {
      if (++qt > upto) {
        qt = from;
        ++head;
      }
    };
    // What is known of the tile behind the one being copied is loaded with it,
    // and waited for with it: by itself it kept each turn waiting.
    int head = head0, qt = from, stage = 0;
    int4 e = scalars(range_at(qt));
    copy(head, qt, at);
    int nhead = head, nqt = qt;
    behind(nhead, nqt);
    int ahead = range_at(nqt);
    while (head < head0 + mine) {
      Score<TS> sc;
      sc.init(a, head);
      wait_loads();
      lds_barrier();
      unsigned char* Q = lds + stage * ST::kBytes;
      unsigned char* G = Q + TL::kBytes;
      stage ^= 1;
      int4 ne = scalars(ahead);
      while (nhead < head0 + mine && !sees(ne)) {
        behind(nhead, nqt);
        ne = scalars(range_at(nqt));
      }
      const int head1 = nhead, qt1 = nqt;
      if (nhead < head0 + mine) {
        copy(nhead, nqt, at + stage * ST::kBytes);
        behind(nhead, nqt);
        ahead = range_at(nqt);
      }
      const bool cut = e.z > j0 || e.w < j0 + KEYS;
      uint64_t bad = 0;
      if (cut) {
        // rows whose lse or delta is not finite count as such (rows that see nothing are among them);
        // all others are finite: an infinity or NaN of a query makes its lse one, unless a cap
        // bounds the scores, and one of do its delta (0 times it is NaN)
        float* r = reinterpret_cast<float*>(Q + ST::kRows);
        const uint64_t more = __ballot(!(fabsf(r[lane]) <= FLT_MAX && fabsf(r[64 + lane]) <= FLT_MAX));
        if (more || (EX && a.cap > 0.f)) {
          TL::clean(Q, bits, wave, again(lane));
          TL::clean(G, bits + 1, wave, again(lane));
          lds_barrier();
          bad = more | bits[0] | bits[1];
          if (wave == 0 && (more >> lane & 1)) r[lane] = r[64 + lane] = 0.f;
          lds_barrier();
        }
      }
      const bool none = e.x >= j0 + 32 * wave + 32 || e.y <= j0 + 32 * wave;     // no row sees a key of this wave
#pragma unroll 1
      for (int rb = none ? 2 : 0; rb < 2; ++rb) {
        const int ln = again(lane);
        const float* rows = reinterpret_cast<const float*>(Q + ST::kRows) + 32 * rb + 4 * (ln / 32);
        f32x16 s = f32x16{}, dp = f32x16{};
        // the scores, then dP with the scores' probabilities beside it
        feed<KS, AHEAD, Frag<TS>>([&](auto i, Frag<TS>& q) { TL::row_frag(Q, rb, i.value, ln, q); },
                                  [&](auto i, Frag<TS>& q) { s = mfma32(q, kf[i.value], s); });
        Frag<TS> v;
        float4 four;
        feed<KS, AHEAD, Frag<TS>>(
            [&](auto i, Frag<TS>& q) { TL::row_frag(G, rb, i.value, ln, q); },
            [&](auto i, Frag<TS>& q) {
              if constexpr (i.value < KS - PARKED) v = vf[i.value];
              dp = mfma32(q, v, dp);
              if constexpr (i.value + 1 >= KS - PARKED && i.value + 1 < KS)
                v = parked[(i.value + 1 - KS + PARKED) * 64 + ln];
              if constexpr (!EX)
                share<16, KS>(i, [&](auto e) {
                  if constexpr (e.value % 4 == 0) four = *reinterpret_cast<const float4*>(rows + 2 * e.value);
                  s[e.value] = __builtin_amdgcn_exp2f(rounded_diff(s[e.value], sc.mul, (&four.x)[e.value % 4]));
                });
            });
        if constexpr (EX) {
          const float d0 = (float)(qt * kTile + 32 * rb + 4 * (ln / 32) - key);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 lse = *reinterpret_cast<const float4*>(rows + 8 * i);
            const float4 del = *reinterpret_cast<const float4*>(rows + 64 + 8 * i);
            float x[4], y[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = s[4 * i + r], y[r] = dp[4 * i + r];
            reverse_scores<TS, 4>(x, y, sc, a.cap > 0.f,
                                  [&](int r) { return fabsf(d0 + (float)sum_row(4 * i + r)); },
                                  [&](int r) { return (&lse.x)[r]; }, [&](int r) { return (&del.x)[r]; });
#pragma unroll
            for (int r = 0; r < 4; ++r) s[4 * i + r] = x[r], dp[4 * i + r] = y[r];
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (cut) {
          branch_only();
          const uint32_t rows32 = (uint32_t)(bad >> (32 * rb)) >> (4 * (ln / 32));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int4 lo = *reinterpret_cast<const int4*>(rows + 128 + 8 * i);
            const int4 hi = *reinterpret_cast<const int4*>(rows + 192 + 8 * i);
            const float4 del = *reinterpret_cast<const float4*>(rows + 64 + 8 * i);
#pragma unroll
            for (int r = 4 * i; r < 4 * i + 4; ++r) {
              const bool seen = key >= (&lo.x)[r % 4] && key < (&hi.x)[r % 4];
              if (rows32 >> sum_row(r) & 1) s[r] = dp[r] = __builtin_nanf("");
              if (!seen) {
                s[r] = 0.f;
                dp[r] = EX ? 0.f : (&del.x)[r % 4];          // p (dP - delta) = 0 below
              }
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        // dv, with dS = p (dP - delta) beside it, then dk
        Frag<TS> p;
        feed<2 * F, AHEAD, Frag<TS>>(
            [&](auto i, Frag<TS>& x) { TL::col_frag(G, i.value % F, 2 * rb + i.value / F, ln, x); },
            [&](auto i, Frag<TS>& x) {
              if constexpr (i.value % F == 0) sums_frag(s, i.value / F, p);
              dv[i.value % F] = mfma32(x, p, dv[i.value % F]);
              if constexpr (!EX)
                share<16, 2 * F>(i, [&](auto e) {
                  if constexpr (e.value % 4 == 0) four = *reinterpret_cast<const float4*>(rows + 64 + 2 * e.value);
                  dp[e.value] = s[e.value] * (dp[e.value] - (&four.x)[e.value % 4]);
                });
            });
        feed<2 * F, AHEAD, Frag<TS>>(
            [&](auto i, Frag<TS>& x) { TL::col_frag(Q, i.value % F, 2 * rb + i.value / F, ln, x); },
            [&](auto i, Frag<TS>& x) {
              if constexpr (i.value % F == 0) sums_frag(dp, i.value / F, p);
              dk[i.value % F] = mfma32(x, p, dk[i.value % F]);
            });
      }
      head = head1;
      qt = qt1;
      e = ne;
    }
  }
  if (a.parts == 1) {
    TS* p = reinterpret_cast<TS*>(a.dqkv) + ((int64_t)key * H + a.Hq + kvh) * D;
#pragma unroll
    for (int f = 0; f < F; ++f) {
      store_sums<TS>(dk[f], a.scale, p + 32 * f, row, lane);
      store_sums<TS>(dv[f], 1.f, p + (int64_t)a.Hkv * D + 32 * f, row, lane);
    }
  } else {
    float* p = a.part + (((int64_t)part * a.T + key) * 2 * a.Hkv + kvh) * D;
#pragma unroll
    for (int f = 0; f < F; ++f) {
      store_sums<float>(dk[f], a.scale, p + 32 * f, row, lane);
      store_sums<float>(dv[f], 1.f, p + (int64_t)a.Hkv * D + 32 * f, row, lane);
    }
  }
}

// Sums of a token's `row` elements from their parts, added in order: dk and dv,
// or dq (Hq = 0: what lies in front of them)
template <typename TS>
__global__ __launch_bounds__(256) void k_attn_join(int64_t T, int row, int parts, const float* part, int H, int Hq, int D,
                                                   TS* dqkv) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= T * row) return;
  const int64_t t = i / row;
  float s[8];
  Vec8<float>::load(part + i, s);
  for (int p = 1; p < parts; ++p) {
    float x[8];
    Vec8<float>::load(part + (int64_t)p * T * row + i, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += x[e];
  }
  Vec8<TS>::store(dqkv + (t * H + Hq) * D + (i - t * row), s);
}

constexpr size_t up(size_t n) { return (n + 255) / 256 * 256; }

// Parts of the sums of dk and dv, which are added afterwards: the chip holds
// 512 workgroups of four waves, of unlike lengths where masks cut; with less
// than twice as many, a group's heads are divided among several (8190 tokens in
// documents, Hq = 16, Hkv = 4, D = 64: backward 157 us in four parts, 189 in
// two).  Where those leave room, so are the tiles of queries that see a
// workgroup's keys, in up to eight slices (backward of T = 815, Hq = 14, Hkv =
// 2, D = 128: 122 us without slices, 95 with a workgroup of four waves for each
// CU, 86 with two; T = 777, Hq = 6, Hkv = 2, D = 96, fp32: 209, 128, 121).
struct Parts {
  int parts, slices;                             // parts = shares of a group's heads times slices of the queries
};
Parts parts_of(int64_t T, int Hq, int Hkv, int keys) {
  const int64_t wg = (T + keys - 1) / keys * Hkv, tiles = (T + kTile - 1) / kTile;
  const int g = Hq / Hkv;
  if (T == 0) return {1, 1};
  for (int p = 1; p < g; ++p)
    if (g % p == 0 && wg * p * keys >= 1024 * 128) return {p, 1};
  int64_t n = 512 * 128 / (wg * g * keys);
  n = n < 1 ? 1 : n < 8 ? n : 8;
  n = n < tiles ? n : tiles;
  return {g * (int)n, (int)n};
}

// Slices of the keys for dq, added afterwards, where the rows are few and the keys
// many: until the chip has two workgroups a CU (fp32: one), with four tiles each
// (backward of T = 777, Hq = 6, Hkv = 2, D = 96, fp32: 121 -> 85 us in three; T =
// 763, Hq = 4, Hkv = 4, D = 64, bf16: 45 -> 43 in three).
int dq_slices(bool f32, int64_t T, int Hq) {
  if (T == 0 || attn_parts(T, Hq) == 1) return 1;
  const int64_t wg = (T + 63) / 64 * Hq, tiles = (T + kTile - 1) / kTile;
  int64_t n = (f32 ? 256 : 512) / wg;
  n = n < tiles / 4 ? n : tiles / 4;
  return n < 1 ? 1 : n < 4 ? (int)n : 4;
}

template <typename TS, int D, bool EX> hipError_t run_bwd(AttnArgs a, char* ws, hipStream_t s) {
  const size_t heads = up((size_t)a.Tp * a.Hq * 4), rows = up((size_t)a.Tp * 4);
  float* delta = reinterpret_cast<float*>(ws);
  int* lo = reinterpret_cast<int*>(ws + heads);
  int* hi = reinterpret_cast<int*>(ws + heads + rows);
  int4* range = reinterpret_cast<int4*>(ws + heads + 2 * rows);
  a.part = reinterpret_cast<float*>(ws + heads + 2 * rows + up((size_t)a.Tp / kTile * 16));
  k_attn_prep<TS, D><<<dim3((unsigned)(a.Tp / kTile), a.Hq + 1), dim3(256), 0, s>>>(a, delta, lo, hi, range);
  a.delta = delta, a.lo = lo, a.hi = hi, a.range = range;
  constexpr int NW = dkv_waves(sizeof(TS) == 4, D);
  const unsigned ktiles = (unsigned)((a.T + 32 * NW - 1) / (32 * NW));
  k_attn_dkv<TS, D, EX><<<dim3(ktiles * a.Hkv * a.parts), dim3(64 * NW), 0, s>>>(a);
  if (a.parts > 1) {
    const int row = 2 * a.Hkv * D;
    k_attn_join<TS><<<dim3((unsigned)((a.T * row / 8 + 255) / 256)), dim3(256), 0, s>>>(
        a.T, row, a.parts, a.part, a.Hq + 2 * a.Hkv, a.Hq, D, static_cast<TS*>(a.dqkv));
  }
  if (attn_parts(a.T, a.Hq) == 1)
    k_attn_dq<TS, D, EX, 1><<<dim3((unsigned)((a.T + 127) / 128) * a.Hq), dim3(64 * kAttnWaves), 0, s>>>(a);
  else
    k_attn_dq<TS, D, EX, 2><<<dim3((unsigned)((a.T + 63) / 64) * a.Hq * a.qslices), dim3(64 * kAttnWaves), 0, s>>>(a);
  if (a.qslices > 1) {
    const int row = a.Hq * D;
    k_attn_join<TS><<<dim3((unsigned)((a.T * row / 8 + 255) / 256)), dim3(256), 0, s>>>(
        a.T, row, a.qslices, a.part, a.Hq + 2 * a.Hkv, 0, D, static_cast<TS*>(a.dqkv));
  }
  return hipGetLastError();
}

template <typename TS> hipError_t run_bwd_of(int D, const AttnArgs& a, char* ws, hipStream_t s) {
  const bool ex = a.cap > 0.f || a.slopes;
  switch (D) {
    case 32: return ex ? run_bwd<TS, 32, true>(a, ws, s) : run_bwd<TS, 32, false>(a, ws, s);
    case 64: return ex ? run_bwd<TS, 64, true>(a, ws, s) : run_bwd<TS, 64, false>(a, ws, s);
    case 96: return ex ? run_bwd<TS, 96, true>(a, ws, s) : run_bwd<TS, 96, false>(a, ws, s);
    default: return ex ? run_bwd<TS, 128, true>(a, ws, s) : run_bwd<TS, 128, false>(a, ws, s);
  }
}

}  // namespace

size_t attn_bwd_ws_bytes(int state_dtype, int64_t T, int Hq, int Hkv, int D) {
  const int64_t Tp = (T + kTile - 1) / kTile * kTile;
  const int parts = parts_of(T, Hq, Hkv, 32 * dkv_waves(state_dtype == XHC_F32, D)).parts;
  const int slices = dq_slices(state_dtype == XHC_F32, T, Hq);
  const size_t kv = parts > 1 ? (size_t)parts * T * 2 * Hkv * D * 4 : 0, q = slices > 1 ? (size_t)slices * T * Hq * D * 4 : 0;
  // (the parts of dk and dv are added before dq begins: one place for both)
  return up((size_t)Tp * Hq * 4) + 2 * up((size_t)Tp * 4) + up((size_t)Tp / kTile * 16) + (kv > q ? kv : q);
}

hipError_t launch_attn_bwd(const xhc_dims* d, const xhc_heads* h, const void* qkv, const int32_t* span,
                           const float* slopes, const void* out, const void* saved, const void* dout, void* dqkv,
                           void* ws, hipStream_t s) {
  AttnArgs a{};
  a.qkv = qkv;
  a.span = reinterpret_cast<const int2*>(span);
  a.slopes = slopes;
  a.out = const_cast<void*>(out);
  a.lse = static_cast<float*>(const_cast<void*>(saved));
  a.low = reinterpret_cast<uint16_t*>(reinterpret_cast<char*>(a.lse) + attn_lse_bytes(d->T, h->Hq));
  a.dout = dout;
  a.dqkv = dqkv;
  a.T = d->T, a.S = d->S, a.Tp = (d->T + kTile - 1) / kTile * kTile;
  a.Hq = h->Hq, a.Hkv = h->Hkv, a.window = h->window;
  const Parts parts = parts_of(d->T, h->Hq, h->Hkv, 32 * dkv_waves(d->state_dtype == XHC_F32, h->D));
  a.parts = parts.parts, a.slices = parts.slices;
  a.qslices = dq_slices(d->state_dtype == XHC_F32, d->T, h->Hq);
  a.scale = h->scale, a.cap = h->cap;
  return d->state_dtype == XHC_BF16 ? run_bwd_of<uint16_t>(h->D, a, static_cast<char*>(ws), s)
                                    : run_bwd_of<float>(h->D, a, static_cast<char*>(ws), s);
}

}  // namespace xhc
