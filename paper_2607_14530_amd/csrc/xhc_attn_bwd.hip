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
// atomics, no fp32 copy of dq, and an order that only the sizes fix.
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

// p and dS of one pair from the raw product and dP
template <typename TS>
__device__ __forceinline__ void reverse_score(float& x, float& dp, const Score& sc, bool capped, float bias, float lse,
                                              float delta) {
  float der = 1.f;
  if (capped) {
    const float t = tanh_of<TS>(x * sc.mul);
    x = sc.cap * t;
    der = 1.f - t * t;
  } else {
    x *= sc.mul;
  }
  x = __builtin_amdgcn_exp2f(x + bias - lse);
  dp = x * (dp - delta) * der;
}

template <typename TS, int D, bool EX>
__global__ __launch_bounds__(64 * kAttnWaves, sizeof(TS) == 2 ? 2 : 1) void k_attn_dq(AttnArgs a) {
  using TL = Tile<TS, D>;
  constexpr int KS = D / 16, F = D / 32;
  __shared__ __align__(1024) unsigned char lds[4 * TL::kBytes];
  __shared__ int4 red[kAttnWaves];
  __shared__ __align__(8) uint16_t bits[4];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  int head, tile;
  attn_place(a.Hq, (int)((a.T + 127) / 128), head, tile);
  const int kvh = head / (a.Hq / a.Hkv), H = a.Hq + 2 * a.Hkv;
  const int t = tile * 128 + wave * 32 + lane % 32, T1 = (int)a.T - 1;
  const bool row = t <= T1;
  const int2 see = span_of(a, t);
  const int4 ex = attn_extremes(see, row, red, wave, lane);
  const uint32_t stride = (uint32_t)H * D * sizeof(TS);
  const unsigned char* base = reinterpret_cast<const unsigned char*>(a.qkv);
  const unsigned char* kb = base + (size_t)(a.Hq + kvh) * D * sizeof(TS);
  const unsigned char* vb = kb + (size_t)a.Hkv * D * sizeof(TS);
  const uint32_t at = lds_offset(lds);

  f32x16 dq[F];
#pragma unroll
  for (int f = 0; f < F; ++f) dq[f] = f32x16{};
  const int first = ex.x / kTile, end = (ex.y + kTile - 1) / kTile;
  if (ex.x < ex.y) {
    Score sc;
    sc.init(a, head);
    const int64_t tc = row ? t : T1;
    const float lse = a.lse[(int64_t)head * a.Tp + tc], delta = a.delta[(int64_t)head * a.Tp + tc];
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
      wait_loads();
      lds_barrier();
      if (kt + 1 < end) {
        const int ln = again(lane);
        TL::copy(kb, stride, (kt + 1) * kTile, T1, at + next, wave, ln);
        TL::copy(vb, stride, (kt + 1) * kTile, T1, at + next + TL::kBytes, wave, ln);
      }
      unsigned char *K = lds + off, *V = K + TL::kBytes;
      const int j0 = kt * kTile;
      const bool cut = j0 < ex.z || j0 + kTile > ex.w;
      uint64_t bad = 0;
      if (cut) bad = TL::clean(K, bits, wave, again(lane));
#pragma unroll 1
      for (int rb = 0; rb < 2; ++rb) {
        const int ln = again(lane);
        f32x16 s = f32x16{}, dp = f32x16{};
        Frag<TS> k[2];
        TL::row_frag(K, rb, 0, ln, k[0]);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {       // a fragment is read while the one before is multiplied
          if (i + 1 < 2 * KS) TL::row_frag(i + 1 < KS ? K : V, rb, (i + 1) % KS, ln, k[(i + 1) % 2]);
          if (i < KS)
            s = mfma32(k[i % 2], q[i % KS], s);
          else
            dp = mfma32(k[i % 2], go[i % KS], dp);
          __builtin_amdgcn_sched_barrier(0);
        }
        const int j1 = j0 + 32 * rb + 4 * (ln / 32);         // this lane's keys: j1 + sum_row(r)
        if constexpr (EX) {
          const float d0 = (float)(t - j1);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float x = s[r], y = dp[r];
            reverse_score<TS>(x, y, sc, a.cap > 0.f, -sc.slope * fabsf(d0 - (float)sum_row(r)), lse, delta);
            dp[r] = y;
          }
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            dp[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sc.mul, -lse)) * (dp[r] - delta);
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
        __builtin_amdgcn_sched_barrier(0);
        Frag<TS> x[2], ds;
        TL::col_frag(K, 0, 2 * rb, ln, x[0]);
#pragma unroll
        for (int i = 0; i < 2 * F; ++i) {
          const int st = i / F, f = i % F;
          if (f == 0) sums_frag(dp, st, ds);
          if (i + 1 < 2 * F) TL::col_frag(K, (i + 1) % F, 2 * rb + (i + 1) / F, ln, x[(i + 1) % 2]);
          dq[f] = mfma32(x[i % 2], ds, dq[f]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
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

template <typename TS, int D, bool EX>
__global__ __launch_bounds__(64 * kAttnWaves, sizeof(TS) == 2 ? 2 : 1) void k_attn_dkv(AttnArgs a) {
  using TL = Tile<TS, D>;
  using ST = QStage<TL>;
  constexpr int KS = D / 16, F = D / 32;
  // Of the fragments that a wave keeps, the values' last ones lie in LDS where
  // the registers do not hold all (D = 128, bf16): two workgroups a CU have 256
  // registers a lane and 80 KiB each.
  constexpr int PARKED = sizeof(TS) == 2 && D == 128 ? 3 : 0;
  __shared__ __align__(1024) unsigned char lds[2 * ST::kBytes + PARKED * kAttnWaves * 1024];
  __shared__ __align__(8) uint16_t bits[8];
  __shared__ int reach[2];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int g = a.Hq / a.Hkv, mine = g / a.parts, H = a.Hq + 2 * a.Hkv;
  const int tiles = (int)((a.T + 127) / 128), qtiles = (int)(a.Tp / kTile);
  int which, tile;
  attn_place(a.Hkv * a.parts, tiles, which, tile);
  tile = tiles - 1 - tile;                       // the first keys are seen by most queries
  const int kvh = which / a.parts, part = which % a.parts;
  const int head0 = kvh * g + part * mine;
  const int j0 = tile * 128, T1 = (int)a.T - 1;
  const int key = j0 + wave * 32 + lane % 32;
  const bool row = key <= T1;
  const unsigned char* qb = reinterpret_cast<const unsigned char*>(a.qkv);
  const unsigned char* gb = reinterpret_cast<const unsigned char*>(a.dout);
  const uint32_t qstride = (uint32_t)H * D * sizeof(TS), gstride = (uint32_t)a.Hq * D * sizeof(TS);
  const uint32_t at = lds_offset(lds);

  // the first and last tile of queries of which some row sees one of these keys
  if (threadIdx.x < 2) reach[threadIdx.x] = threadIdx.x ? -1 : INT32_MAX;
  __syncthreads();
  auto sees = [&](const int4& e) { return e.x < j0 + 128 && e.y > j0 && e.x < e.y; };
  int from = INT32_MAX, upto = -1;
  for (int i = threadIdx.x; i < qtiles; i += 64 * kAttnWaves)
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
      const void* p = wave == 0   ? (const void*)(a.lse + (int64_t)head * a.Tp + r)
                      : wave == 1 ? (const void*)(a.delta + (int64_t)head * a.Tp + r)
                      : wave == 2 ? (const void*)(a.lo + r)
                                  : (const void*)(a.hi + r);
      lds_dma4(p, to + ST::kRows + wave * 256);
    };
    auto range_of = [&](int i) {                 // (into scalar registers)
      const int4 x = a.range[i];
      return make_int4(__builtin_amdgcn_readfirstlane(x.x), __builtin_amdgcn_readfirstlane(x.y),
                       __builtin_amdgcn_readfirstlane(x.z), __builtin_amdgcn_readfirstlane(x.w));
    };
    // the tile behind (head, qt) that is to be taken; head == head0 + mine: none
    auto advance = [&](int& head, int& qt, int4& e) {
      do {
        if (++qt > upto) {
          qt = from;
          ++head;
        }
        e = range_of(qt);
      } while (head < head0 + mine && !sees(e));
    };
    int head = head0, qt = from, stage = 0;
    int4 e = range_of(qt);
    copy(head, qt, at);
    while (head < head0 + mine) {
      int nhead = head, nqt = qt;
      int4 ne;
      advance(nhead, nqt, ne);      // (loads of its own stand before the copies, which a wait for them would wait for)
      Score sc;
      sc.init(a, head);
      wait_loads();
      lds_barrier();
      unsigned char* Q = lds + stage * ST::kBytes;
      unsigned char* G = Q + TL::kBytes;
      stage ^= 1;
      if (nhead < head0 + mine) copy(nhead, nqt, at + stage * ST::kBytes);
      const bool cut = e.z > j0 || e.w < j0 + 128;
      uint64_t bad = 0;
      if (cut) bad = TL::clean(Q, bits, wave, again(lane)) | TL::clean(G, bits + 4, wave, again(lane));
#pragma unroll 1
      for (int rb = 0; rb < 2; ++rb) {
        const int ln = again(lane);
        const float* rows = reinterpret_cast<const float*>(Q + ST::kRows) + 4 * (ln / 32);
        const float d0 = (float)(qt * kTile + 4 * (ln / 32) - key);
        f32x16 s = f32x16{}, dp = f32x16{};
        // (one product after the other: few registers are left beside the sums and the keys' and values' fragments)
        Frag<TS> q[2], v;
        TL::row_frag(Q, rb, 0, ln, q[0]);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
          if (i + 1 < 2 * KS) TL::row_frag(i + 1 < KS ? Q : G, rb, (i + 1) % KS, ln, q[(i + 1) % 2]);
          if (i < KS) {
            s = mfma32(q[i % 2], kf[i % KS], s);
          } else {
            if (i - KS < KS - PARKED) v = vf[i - KS];
            dp = mfma32(q[i % 2], v, dp);
          }
          if (i + 1 >= 2 * KS - PARKED && i + 1 < 2 * KS) v = parked[(i + 1 - 2 * KS + PARKED) * 64 + ln];
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 lse = *reinterpret_cast<const float4*>(rows + 32 * rb + 8 * i);
          const float4 del = *reinterpret_cast<const float4*>(rows + 64 + 32 * rb + 8 * i);
          const float L[4] = {lse.x, lse.y, lse.z, lse.w}, E[4] = {del.x, del.y, del.z, del.w};
#pragma unroll
          for (int e4 = 0; e4 < 4; ++e4) {
            const int r = 4 * i + e4;
            if constexpr (EX) {
              float x = s[r], y = dp[r];
              reverse_score<TS>(x, y, sc, a.cap > 0.f, -sc.slope * fabsf(d0 + (float)(32 * rb + sum_row(r))), L[e4],
                                E[e4]);
              s[r] = x;
              dp[r] = y;
            } else {
              s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sc.mul, -L[e4]));
              dp[r] = s[r] * (dp[r] - E[e4]);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (bad) {
          branch_only();
          const uint32_t rows32 = (uint32_t)(bad >> (32 * rb)) >> (4 * (ln / 32));
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float nan = rows32 >> sum_row(r) & 1 ? __builtin_nanf("") : 0.f;
            s[r] += nan;
            dp[r] += nan;
          }
        }
        if (cut) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            branch_only();
            const int4 lo = *reinterpret_cast<const int4*>(rows + 128 + 32 * rb + 8 * i);
            const int4 hi = *reinterpret_cast<const int4*>(rows + 192 + 32 * rb + 8 * i);
            const int L[4] = {lo.x, lo.y, lo.z, lo.w}, U[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
              const int r = 4 * i + e4;
              const bool seen = key >= L[e4] && key < U[e4];
              if (!seen) s[r] = dp[r] = 0.f;
            }
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        Frag<TS> x[2], y[2], p, ds;
        TL::col_frag(G, 0, 2 * rb, ln, x[0]);
        TL::col_frag(Q, 0, 2 * rb, ln, y[0]);
#pragma unroll
        for (int i = 0; i < 2 * F; ++i) {
          const int st = i / F, f = i % F;
          if (f == 0) {
            sums_frag(s, st, p);
            sums_frag(dp, st, ds);
          }
          if (i + 1 < 2 * F) {
            TL::col_frag(G, (i + 1) % F, 2 * rb + (i + 1) / F, ln, x[(i + 1) % 2]);
            TL::col_frag(Q, (i + 1) % F, 2 * rb + (i + 1) / F, ln, y[(i + 1) % 2]);
          }
          dv[f] = mfma32(x[i % 2], p, dv[f]);
          dk[f] = mfma32(y[i % 2], ds, dk[f]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      head = nhead;
      qt = nqt;
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

// dk and dv from the parts, added in order; `row` = 2 Hkv D elements a token
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

// Parts of a group's heads for dk and dv: 512 workgroups fill the chip's 256 CUs
// twice over; with fewer, a group's heads are divided among several, whose sums
// are then added.
int parts_of(int64_t T, int Hq, int Hkv) {
  const int64_t wg = (T + 127) / 128 * Hkv;
  const int g = Hq / Hkv;
  for (int p = 1; p < g; ++p)
    if (g % p == 0 && wg * p >= 512) return p;
  return g;
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
  const unsigned tiles = (unsigned)((a.T + 127) / 128);
  k_attn_dkv<TS, D, EX><<<dim3(tiles * a.Hkv * a.parts), dim3(64 * kAttnWaves), 0, s>>>(a);
  if (a.parts > 1) {
    const int row = 2 * a.Hkv * D;
    k_attn_join<TS><<<dim3((unsigned)((a.T * row / 8 + 255) / 256)), dim3(256), 0, s>>>(
        a.T, row, a.parts, a.part, a.Hq + 2 * a.Hkv, a.Hq, D, static_cast<TS*>(a.dqkv));
  }
  k_attn_dq<TS, D, EX><<<dim3(tiles * a.Hq), dim3(64 * kAttnWaves), 0, s>>>(a);
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

size_t attn_bwd_ws_bytes(int64_t T, int Hq, int Hkv, int D) {
  const int64_t Tp = (T + kTile - 1) / kTile * kTile;
  const int parts = parts_of(T, Hq, Hkv);
  return up((size_t)Tp * Hq * 4) + 2 * up((size_t)Tp * 4) + up((size_t)Tp / kTile * 16) +
         (parts > 1 ? (size_t)parts * T * 2 * Hkv * D * 4 : 0);
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
  a.parts = parts_of(d->T, h->Hq, h->Hkv);
  a.scale = h->scale, a.cap = h->cap;
  return d->state_dtype == XHC_BF16 ? run_bwd_of<uint16_t>(h->D, a, static_cast<char*>(ws), s)
                                    : run_bwd_of<float>(h->D, a, static_cast<char*>(ws), s);
}

}  // namespace xhc
