// The gradient of attention over the caller's rows.  Probabilities are computed again from the scores and the logarithms of their
// sums that the forward pass left, p = exp(s - lse); e = p (dp - delta) with dp = dout v and delta = dout out.  No atomics: every
// result has one wavefront that sums it, in one order.
//
// Half precision: p enters its product times 2^12 (p <= 1, so it fits), which keeps the small probabilities of long rows out of the
// type's subnormal numbers; dp and delta are taken times 2^-12 in exchange, where float32 loses nothing, so that e is what it is.
#include "attention_mx.h"

namespace ff {
namespace {

template <typename T> constexpr float kLift = 0.f;
template <> constexpr float kLift<f16_t> = 12.f;
template <typename T> constexpr float kLower = 1.f;
template <> constexpr float kLower<f16_t> = 1.f / 4096.f;

// What a row's scores and its dp start from: minus the logarithm of the row's sum (-infinity, every p zero, where the row has no key)
// and minus delta.  With 16 bits the products of the scores begin at it, in units of the scores.  In float32 every step of a product
// that carried it would round at its size, so it comes in behind them, s scale - lse rounded once and then taken to base 2: the error
// is half a step of the exponent, which is small where p is large.
// Half precision, whose dp is scaled first: minus delta 2^-12.
template <typename T> constexpr bool kBehind = sizeof(T) == 4;
template <typename T> __device__ __forceinline__ float score_factor(const Attn& a) {
  return kBehind<T> ? score_scale(a) : exponent_factor(a);
}
template <typename T> __device__ __forceinline__ float score_start(float lse, float c) {
  return lse == -INFINITY ? -INFINITY : kBehind<T> ? -lse : -lse * kLog2e / c;
}
// p and e, in the places of scores and dp that began so; shift: what is left to add to the exponents
template <typename T> __device__ __forceinline__ void p_and_e(f32x4& s, f32x4& dp, float c, f32x4 shift, f32x4 minus_delta) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float x = fmaf(s[r], c, shift[r]);
    s[r] = exp2_fast(kBehind<T> ? x * kLog2e : x);
    dp[r] = s[r] * (kLift<T> > 0.f ? fmaf(dp[r], kLower<T>, minus_delta[r]) : dp[r]);
  }
}
template <typename T> __device__ __forceinline__ f32x4 s_start(f32x4 start) { return kBehind<T> ? all4(0.f) : start; }
template <typename T> __device__ __forceinline__ f32x4 s_shift(f32x4 start) { return kBehind<T> ? start : all4(kLift<T>); }
template <typename T> __device__ __forceinline__ f32x4 dp_start(f32x4 minus_delta) { return kLift<T> > 0.f ? all4(0.f) : minus_delta; }

template <typename T> __device__ __forceinline__ float dot_pieces(const Piece& a, const Piece& b) {
  float s = 0.f;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) s = fmaf(a.f[j], b.f[j], s);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      T x, y;
      x.bits = (uint16_t)(a.q[j / 2] >> (16 * (j % 2)));
      y.bits = (uint16_t)(b.q[j / 2] >> (16 * (j % 2)));
      s = fmaf(Elem<T>::load(&x), Elem<T>::load(&y), s);
    }
  }
  return s;
}

// ---- short groups: a wavefront holds all keys, values and their gradients of a group and key head ---------------
// Scores with the queries down and the keys across (Q K^T): a lane holds scores of one key, and p and e are the right operands of
// (dv)^T = dout^T p and (dk)^T = q^T e as they lie in the registers.  For (dq)^T = K^T e^T e goes through LDS once, which turns it.
// All rows come and go through LDS, for the workgroup's heads together.  Region A: keys, then e, then dk; B: values, then queries (and dq
// in their places) and dout by CH rows, then dv.  delta is summed where the rows of dout and out come in.
// Registers decide how many wavefronts a SIMD takes: three for 64 keys of 16 elements (30,000 rows of 8 heads: 21.4 us, with two 23.5, with
// four and some registers in scratch memory 30.7), two as long as that leaves next to none in scratch memory (80 keys in three: 30.1 for 29.7,
// 96 keys: 43 for 32), else one.  Large launches are near the memory's rate (240,000 rows, groups of 69, 8 heads of 32 elements of 16
// bits: 224 us, 4.4 TB/s).
template <typename T, int DP, int KT, int HW, bool WHOLE>
__global__ __launch_bounds__(64 * HW, KT * DP <= 64 && DP * sizeof(T) <= 64 ? 3 : KT * DP <= (sizeof(T) == 4 ? (DP == 16 ? 128 : 96) : 192) ? 2 : 1)
void k_attention_backward_group(Attn a, Items items) {
  constexpr int KF = Mx<T>::KF, E = Mx<T>::E, TILES = Mx<T>::TILES, NF = (DP + KF - 1) / KF, DT = DP / 16, NT = 64 * HW;
  constexpr int CH = DP * (int)sizeof(T) <= 32 ? 32 : 16;  // (one piece of each array a thread, two of rows of 128 bytes)
  constexpr int KP = (KT + TILES - 1) / TILES, RK = KP * TILES * 16, PAD = 16 / (int)sizeof(T), LD = DP + PAD, LDE = 16 + PAD;
  constexpr int PITCH_A = RK * (LD > LDE ? LD : LDE);
  constexpr bool ONE = HW * (PITCH_A + KT * 16 * LD) * sizeof(T) > 78 * 1024;  // two workgroups would not fit: values and dv by A too
  constexpr int PITCH_B = (!ONE && KT * 16 > 2 * CH ? KT * 16 : 2 * CH) * LD;
  typedef KeyPieces<T, DP, HW, KT * 16> KeyP;
  typedef QueryPieces<T, DP, HW, CH> QueryP;
  constexpr int PER = QueryP::H::PER, UQ = QueryP::H::U;
  __shared__ __attribute__((aligned(16))) T region_a[HW * PITCH_A], region_b[HW * PITCH_B];
  __shared__ __attribute__((aligned(16))) float bias[KT * 16], offs_all[HW][CH], deltas_all[HW][CH];
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, i = lane & 15, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  touch_arguments(a);
  const uint32_t group = quotient(blockIdx.x, items.sets);
  const int kh0 = (blockIdx.x - group * items.sets.by) * HW, h0 = kh0 * (int)a.share.by;
  const Span sq = span_of(a.ql, group), sk = span_of(a.kl, group);
  if ((int32_t)group >= groups_of(a)) return;
  const int32_t PC = quotient(CH, a.share), last = sq.len;

  KeyP kp;
  QueryP qp;
  Piece kr[KeyP::H::U], vr[KeyP::H::U], qr[UQ], gr[UQ], yr[UQ];
  float lse[UQ];
  kp.place(tid);
  kp.ask(a, sk);
  qp.place(a, tid);
  int32_t end = PC < last ? PC : last;
  auto fetch = [&](int32_t p0) {
    qp.look(a, sq, p0, end);
    qp.template fetch<WHOLE>(qr, a.q, h0, a.D);
    qp.template fetch<WHOLE>(gr, a.dout, h0, a.D);
    qp.template fetch<WHOLE>(yr, a.out, h0, a.D);
#pragma unroll
    for (int u = 0; u < UQ; ++u) lse[u] = qp.row[u] >= 0 ? a.lse[stat_at(a, qp.row[u], h0 + qp.h[u])] : -INFINITY;
    if (p0 + PC < last) qp.ask(a, sq, p0 + PC);
  };
  if (last > 0) qp.ask(a, sq, 0);
  kp.look(a, sk);
  kp.template fetch<WHOLE>(kr, a.k, kh0, a.D);
  kp.template fetch<WHOLE>(vr, a.v, kh0, a.D);
  if (last > 0) fetch(0);
  T *const ta = region_a + wave * PITCH_A, *const qs = region_b + wave * PITCH_B, *const gs = qs + CH * LD;
  float *const offs = offs_all[wave], *const deltas = deltas_all[wave];
  if constexpr (KT * 16 < RK) {  // keys that make the last piece whole
    for (int x = lane; x < (RK - KT * 16) * LD / E; x += 64) *reinterpret_cast<u32x4*>(ta + KT * 16 * LD + x * E) = u32x4{0u, 0u, 0u, 0u};
  }
  kp.put(region_a, PITCH_A, LD, kr);
  if (!ONE) kp.put(region_b, PITCH_B, LD, vr);
  if (kp.head == 0 && kp.c == 0) {
#pragma unroll
    for (int u = 0; u < KeyP::H::U; ++u)
      if (kp.first + u * KeyP::H::STEP < KT * 16) bias[kp.first + u * KeyP::H::STEP] = kp.live >> u & 1 ? 0.f : -INFINITY;
  }
  __syncthreads();
  auto rows_of = [&](const T* tile, int r, int f) {
    Piece p;
    if constexpr (DP < KF) {  // zero behind the row's end
      p = row_piece(tile, LD, r, g4 * E % DP);
      if (g4 * E >= DP) p.q = u32x4{0u, 0u, 0u, 0u};
    } else {
      p = row_piece(tile, LD, r, f * KF + g4 * E);
    }
    return p;
  };
  Piece kf[KT][NF], vf[KT][NF], kc[DT][KP];
  uint32_t live = 0;  // bit t: key t of this lane is one that queries look at
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    if (bias[t * 16 + i] == 0.f) live |= 1u << t;
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      kf[t][f] = rows_of(ta, t * 16 + i, f);
      if (!ONE) vf[t][f] = rows_of(qs, t * 16 + i, f);
      if (a.scale < 0.f) kf[t][f] = negated<T>(kf[t][f]);
    }
  }
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int t = 0; t < KP; ++t) kc[d][t] = column_piece(ta, LD, t * 16 * TILES, d * 16, lane);
  if constexpr (ONE) {
    __syncthreads();
    kp.put(region_a, PITCH_A, LD, vr);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int f = 0; f < NF; ++f) vf[t][f] = rows_of(ta, t * 16 + i, f);
  }
  wave_sync();
  if constexpr (KT * 16 < RK) {  // and e of them
    for (int x = lane; x < (RK - KT * 16) * LDE / E; x += 64) *reinterpret_cast<u32x4*>(ta + KT * 16 * LDE + x * E) = u32x4{0u, 0u, 0u, 0u};
  }
  const float c = score_factor<T>(a);
  f32x4 dk[KT][DT], dv[KT][DT];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[t][d] = dv[t][d] = all4(0.f);

  for (int32_t p0 = 0; p0 < last; p0 += PC) {
    __syncthreads();  // values, or the last chunk's rows, have been read
    qp.put(region_b, PITCH_B, LD, qr);
    qp.put(region_b + CH * LD, PITCH_B, LD, gr);
#pragma unroll
    for (int u = 0; u < UQ; ++u) {
      float delta = dot_pieces<T>(gr[u], yr[u]);
#pragma unroll
      for (int d = 1; d < PER; d *= 2) delta += __shfl_xor(delta, d);
      if (qp.c == 0 && qp.v[u] < CH) {
        offs_all[qp.w[u]][qp.v[u]] = score_start<T>(lse[u], c);
        deltas_all[qp.w[u]][qp.v[u]] = delta * -kLower<T>;
      }
    }
    const QueryP now = qp;
    const int32_t rows = (end - p0) * (int32_t)a.share.by;
    if (p0 + PC < last) {
      end = p0 + 2 * PC < last ? p0 + 2 * PC : last;
      fetch(p0 + PC);
    }
    __syncthreads();
    for (int32_t r0 = 0; r0 < rows; r0 += 16) {
      const f32x4 fo = *reinterpret_cast<const f32x4*>(offs + r0 + g4 * 4), fd = *reinterpret_cast<const f32x4*>(deltas + r0 + g4 * 4);
      Piece qf[NF], gf[NF], qc[DT], gc[DT];
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        qf[f] = rows_of(qs, r0 + i, f);
        gf[f] = rows_of(gs, r0 + i, f);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        qc[d] = column_half(qs, LD, r0, d * 16, lane);
        gc[d] = column_half(gs, LD, r0, d * 16, lane);
      }
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        f32x4 s = s_start<T>(fo), dp = dp_start<T>(fd);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          s = mma<T>(qf[f], kf[t][f], s);
          dp = mma<T>(gf[f], vf[t][f], dp);
        }
        p_and_e<T>(s, dp, c, s_shift<T>(fo), fd);
        const bool here = live >> t & 1;
        if (!__all(here)) {  // keys that no query looks at
#pragma unroll
          for (int r = 0; r < 4; ++r) dp[r] = here ? dp[r] : 0.f;
        }
        const Piece p = as_half<T>(s), e = as_half<T>(dp);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          dv[t][d] = mma_half<T>(gc[d], p, dv[t][d]);
          dk[t][d] = mma_half<T>(qc[d], e, dk[t][d]);
        }
        if constexpr (sizeof(T) == 4) *reinterpret_cast<u32x4*>(ta + (t * 16 + i) * LDE + g4 * 4) = e.q;
        else                          *reinterpret_cast<s16x4*>(ta + (t * 16 + i) * LDE + g4 * 4) = e.s[0];
      }
      wave_sync();
      f32x4 dq[DT];
#pragma unroll
      for (int d = 0; d < DT; ++d) dq[d] = all4(0.f);
#pragma unroll
      for (int t = 0; t < KP; ++t) {
        const Piece e = column_piece(ta, LDE, t * 16 * TILES, 0, lane);
#pragma unroll
        for (int d = 0; d < DT; ++d) dq[d] = mma<T>(kc[d][t], e, dq[d]);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) store4<T, true>(qs + (r0 + i) * LD, d * 16 + g4 * 4, dq[d] * a.scale, DP);  // over their queries
      wave_sync();
    }
    __syncthreads();
    now.template store<WHOLE>(a.dq, h0, a.D, region_b, PITCH_B, LD);
  }
  __syncthreads();
  auto lay = [&](T* tile, const f32x4 (&x)[KT][DT], float by) {
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int d = 0; d < DT; ++d) store4<T, true>(tile + (t * 16 + i) * LD, d * 16 + g4 * 4, live >> t & 1 ? x[t][d] * by : all4(0.f), DP);
  };
  lay(ta, dk, a.scale);
  if (!ONE) lay(qs, dv, kLower<T>);
  __syncthreads();
  kp.template store<WHOLE>(a.dk, kh0, a.D, region_a, PITCH_A, LD);
  if (!ONE) {
    kp.template store<WHOLE>(a.dv, kh0, a.D, region_b, PITCH_B, LD);
  } else {
    __syncthreads();
    lay(ta, dv, kLower<T>);
    __syncthreads();
    kp.template store<WHOLE>(a.dv, kh0, a.D, region_a, PITCH_A, LD);
  }
}

// ---- any lengths -----------------------------------------------------------------------------------------
// What the products of every row and head start from: a few lanes a head, 16 bytes each
template <typename T, int DP, bool WHOLE> __global__ __launch_bounds__(256) void k_attention_stats(Attn a, Div heads) {
  constexpr int PER = DP * (int)sizeof(T) / 16;
  const uint32_t x = blockIdx.x * (256 / PER) + threadIdx.x / PER, all = (uint32_t)a.ql.n * (uint32_t)a.H;
  const int e = (threadIdx.x % PER) * Mx<T>::E;
  const uint32_t row = quotient(x, heads), h = x - row * heads.by;
  float s = 0.f, lse = 0.f;
  if (x < all) {
    lse = a.lse[x];
    s = dot_pieces<T>(load_piece<T, WHOLE>(a.dout, row, h, e, a.D), load_piece<T, WHOLE>(a.out, row, h, e, a.D));
  }
#pragma unroll
  for (int d = PER / 2; d; d >>= 1) s += __shfl_xor(s, d);
  if (x < all && threadIdx.x % PER == 0) a.stats[x] = make_float2(score_start<T>(lse, score_factor<T>(a)), s * -kLower<T>);
}

// dk and dv: NW wavefronts of KW x 16 keys each hold keys, values and the sums of their gradients; the queries that look at them and
// the gradients of their results go by in tiles of BQ rows through LDS.  splits > 1: each workgroup takes a stretch of the queries.
// Seven products in all, two of them made twice (here and for dq), are the price of sums without atomics.  4 groups of 4,096 rows, 8 heads,
// bfloat16: 540 us of 64 elements and 1140 of 128, 640 and 600 TFLOP/s counting five; registers are what bounds it (of 128 elements some
// lie in scratch memory; of 64 the matrix unit is 37 % busy, the vector unit 45 %, LDS 47 %).
template <typename T, int DP, int NW, int KW, int BQ, bool WHOLE>
__global__ __launch_bounds__(64 * NW, DP * sizeof(T) <= 128 ? 2 : 1) void k_attention_dkv(Attn a, TileGrid tg, Order order, int splits, float* part) {
  constexpr int KF = Mx<T>::KF, E = Mx<T>::E, TILES = Mx<T>::TILES, NF = (DP + KF - 1) / KF, DT = DP / 16, NT = 64 * NW, PQ = 2 / TILES;
  constexpr int W = NF * KF, LD = W + 16 / (int)sizeof(T);
  typedef Rows<T, DP, BQ, NT> R;
  constexpr int NB = NW == 1 ? 1 : 2;  // (a wavefront alone writes when it has read)
  __shared__ __attribute__((aligned(16))) T qs[NB][BQ * LD];
  __shared__ __attribute__((aligned(16))) T gs[NB][BQ * LD];
  __shared__ __attribute__((aligned(16))) float offs[NB][BQ], deltas[NB][BQ];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g4 = lane >> 4, i = lane & 15;
  touch_arguments(a);
  const uint32_t work = in_order(order);
  if (work >= order.total) return;
  const uint32_t row_of_work = work / tg.tiles;
  const int split = row_of_work / a.K, kh = row_of_work - split * a.K;
  const TileAt at = tile_at<16 * NW * KW>(a, a.kl, tg, work - row_of_work * tg.tiles, lane);
  if (at.g < 0) return;
  const Span sq = span_of(a.ql, at.g), sk = span_of(a.kl, at.g);
  const int32_t k0 = at.tile * (16 * NW * KW);
  if (at.tile > sk.len / (16 * NW * KW) || k0 >= sk.len) return;
  const int32_t all_rows = sq.len * (int32_t)a.share.by, tiles = (all_rows + BQ - 1) / BQ, per = (tiles + splits - 1) / splits;
  const int32_t t0 = split * per, t1 = t0 + per < tiles ? t0 + per : tiles;

  // As in KeyTiles: numbers two tiles ahead, looked at where their pieces are asked for
  int32_t rows[R::U], heads[R::U];
  auto number = [&](int32_t t) {
    if (t >= t1) return;
    const int32_t* const list = a.ql.perm ? a.ql.perm : &zero_number;
#pragma unroll
    for (int u = 0; u < R::U; ++u) {
      const int32_t p = quotient(t * BQ + R::row(tid, u), a.share);
      rows[u] = list[a.ql.perm ? sq.at + (p < sq.len ? p : sq.len - 1) : 0];
    }
  };
  Piece qr[R::U], gr[R::U];
  float2 st[R::U];
  auto fetch = [&](int32_t t) {
#pragma unroll
    for (int u = 0; u < R::U; ++u) {
      const int r = R::row(tid, u);
      const int32_t v = t * BQ + r, p = quotient(v, a.share);
      heads[u] = kh * a.share.by + v - p * a.share.by;
      if (!a.ql.perm) rows[u] = sq.at + p;
      if ((uint32_t)rows[u] >= (uint32_t)a.ql.n || p >= sq.len || (BQ * R::PER % NT != 0 && r >= BQ)) rows[u] = -1;
    }
    R::template fetch<WHOLE>(qr, a.q, rows, heads, tid, a.D);
    R::template fetch<WHOLE>(gr, a.dout, rows, heads, tid, a.D);
#pragma unroll
    for (int u = 0; u < R::U; ++u) {
      st[u] = make_float2(-INFINITY, 0.f);
      if (tid % R::PER == 0 && rows[u] >= 0) st[u] = a.stats[stat_at(a, rows[u], heads[u])];
    }
  };
  number(t0);
  int32_t key[KW];
  bool live[KW];
#pragma unroll
  for (int t = 0; t < KW; ++t) {
    const int32_t p = k0 + (wave * KW + t) * 16 + i;
    key[t] = p < sk.len ? row_at(a.kl, sk.at + p) : -1;
    live[t] = key[t] >= 0 && (!a.mask || a.mask[key[t]]);
  }
  if (t0 < t1) fetch(t0);
  number(t0 + 1);
  Piece kf[KW][NF], vf[KW][NF];
#pragma unroll
  for (int t = 0; t < KW; ++t)
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      kf[t][f] = load_piece<T, WHOLE>(a.k, live[t] ? key[t] : -1, kh, f * KF + g4 * E, a.D);
      vf[t][f] = load_piece<T, WHOLE>(a.v, live[t] ? key[t] : -1, kh, f * KF + g4 * E, a.D);
    }
  if constexpr (W > DP) {
    for (int x = tid; x < NB * BQ; x += NT)
#pragma unroll
      for (int e = DP; e < W; e += E) {
        *reinterpret_cast<u32x4*>(&qs[0][0] + x * LD + e) = u32x4{0u, 0u, 0u, 0u};
        *reinterpret_cast<u32x4*>(&gs[0][0] + x * LD + e) = u32x4{0u, 0u, 0u, 0u};
      }
  }
  const float c = score_factor<T>(a);
  if (a.scale < 0.f) {
#pragma unroll
    for (int t = 0; t < KW; ++t)
#pragma unroll
      for (int f = 0; f < NF; ++f) kf[t][f] = negated<T>(kf[t][f]);
  }
  f32x4 dk[KW][DT], dv[KW][DT];
#pragma unroll
  for (int t = 0; t < KW; ++t)
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[t][d] = dv[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int32_t t = t0; t < t1; ++t) {
    const int buf = NB == 1 ? 0 : (t - t0) & 1;
    if constexpr (NB == 1) wave_sync();
    R::put(qs[buf], LD, qr, tid);
    R::put(gs[buf], LD, gr, tid);
    if (tid % R::PER == 0) {
#pragma unroll
      for (int u = 0; u < R::U; ++u)
        if (BQ * R::PER % NT == 0 || R::row(tid, u) < BQ) {
          offs[buf][R::row(tid, u)] = st[u].x;
          deltas[buf][R::row(tid, u)] = st[u].y;
        }
    }
    if constexpr (NB == 1) wave_sync();
    else __syncthreads();
    if (t + 1 < t1) {
      fetch(t + 1);
      number(t + 2);
    }
#pragma unroll
    for (int half = 0; half < BQ; half += 32) {
      f32x4 s[KW][2], dp[KW][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = half + u * 16;
        const f32x4 o = *reinterpret_cast<const f32x4*>(offs[buf] + r + g4 * 4), l = *reinterpret_cast<const f32x4*>(deltas[buf] + r + g4 * 4);
#pragma unroll
        for (int k = 0; k < KW; ++k) {
          s[k][u] = s_start<T>(o);
          dp[k][u] = dp_start<T>(l);
        }
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const Piece qf = row_piece(qs[buf], LD, r + i, f * KF + g4 * E), gf = row_piece(gs[buf], LD, r + i, f * KF + g4 * E);
#pragma unroll
          for (int k = 0; k < KW; ++k) {
            s[k][u] = mma<T>(qf, kf[k][f], s[k][u]);
            dp[k][u] = mma<T>(gf, vf[k][f], dp[k][u]);
          }
        }
#pragma unroll
        for (int k = 0; k < KW; ++k) p_and_e<T>(s[k][u], dp[k][u], c, s_shift<T>(o), l);
      }
      Piece p[KW][PQ], e[KW][PQ];
#pragma unroll
      for (int k = 0; k < KW; ++k)
#pragma unroll
        for (int u = 0; u < PQ; ++u) {
          p[k][u] = as_piece<T>(s[k] + u * TILES);
          e[k][u] = as_piece<T>(dp[k] + u * TILES);
        }
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int u = 0; u < PQ; ++u) {
          const Piece gc = column_piece(gs[buf], LD, half + u * 16 * TILES, d * 16, lane), qc = column_piece(qs[buf], LD, half + u * 16 * TILES, d * 16, lane);
#pragma unroll
          for (int k = 0; k < KW; ++k) {
            dv[k][d] = mma<T>(gc, p[k][u], dv[k][d]);
            dk[k][d] = mma<T>(qc, e[k][u], dk[k][d]);
          }
        }
    }
  }
#pragma unroll
  for (int t = 0; t < KW; ++t) {
    if (key[t] < 0) continue;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    if (splits > 1) {
      const int32_t slot = slot_of(a.kl, at.g, sk) + k0 + (wave * KW + t) * 16 + i;
      const int64_t all = (int64_t)a.kl.slots * a.K;
      float* to = part + (split * all + (int64_t)slot * a.K + kh) * 2 * DP + g4 * 4;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        *reinterpret_cast<f32x4*>(to + d * 16) = live[t] ? dk[t][d] : zero;
        *reinterpret_cast<f32x4*>(to + DP + d * 16) = live[t] ? dv[t][d] : zero;
      }
      continue;
    }
    T *tk = row_of_head<T>(a.dk, key[t], kh), *tv = row_of_head<T>(a.dv, key[t], kh);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      store4<T, WHOLE>(tk, d * 16 + g4 * 4, live[t] ? dk[t][d] * a.scale : zero, a.D);
      store4<T, WHOLE>(tv, d * 16 + g4 * 4, live[t] ? dv[t][d] * kLower<T> : zero, a.D);
    }
  }
}

// dq: the forward kernel's arrangement, with keys and values by BK through LDS and scores with the keys down (K Q^T), so that e is the
// right operand of (dq)^T = K^T e^T as it lies in the registers.
template <typename T, int DP, int NW, int QT, int BK, bool WHOLE>
__global__ __launch_bounds__(64 * NW, DP * sizeof(T) <= 256 ? 2 : 1) void k_attention_dq(Attn a, TileGrid tg, Order order, int splits, float* part) {
  constexpr int KF = Mx<T>::KF, E = Mx<T>::E, TILES = Mx<T>::TILES, NF = (DP + KF - 1) / KF, DT = DP / 16, NT = 64 * NW;
  constexpr int W = NF * KF, LD = W + 16 / (int)sizeof(T), BQ = 16 * QT * NW;
  constexpr int NB = NW == 1 ? 1 : 2;  // (a wavefront alone writes when it has read)
  __shared__ __attribute__((aligned(16))) T ks[NB][BK * LD];
  __shared__ __attribute__((aligned(16))) T vs[NB][BK * LD];
  __shared__ __attribute__((aligned(16))) float bias[NB][BK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g4 = lane >> 4, i = lane & 15;
  touch_arguments(a);
  const uint32_t work = in_order(order);
  if (work >= order.total) return;
  const uint32_t row_of_work = work / tg.tiles;
  const int split = row_of_work / a.K, kh = row_of_work - split * a.K;
  const TileAt at = tile_at<BQ>(a, a.ql, tg, work - row_of_work * tg.tiles, lane);
  if (at.g < 0) return;
  const Span sq = span_of(a.ql, at.g), sk = span_of(a.kl, at.g);
  if ((int64_t)at.tile * BQ >= (int64_t)sq.len * tg.share) return;
  const int32_t tiles = (sk.len + BK - 1) / BK, per = (tiles + splits - 1) / splits;
  const int32_t t0 = split * per, t1 = t0 + per < tiles ? t0 + per : tiles;

  KeyTiles<T, DP, BK, NT> kt;
  kt.next(a, sk, t0, t1, tid);
  QueryRow q[QT];
#pragma unroll
  for (int u = 0; u < QT; ++u) q[u] = query_row(a, sq, kh, at.tile * BQ + (wave * QT + u) * 16 + i);
  if (t0 < t1) kt.template fetch<WHOLE>(a, sk, t0, kh, tid);
  kt.next(a, sk, t0 + 1, t1, tid);
  Piece qf[QT][NF], gf[QT][NF];
  f32x4 dp0[QT];
  float shift[QT];
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    float2 st = make_float2(-INFINITY, 0.f);
    if (q[u].row >= 0) st = a.stats[stat_at(a, q[u].row, q[u].h)];
    shift[u] = kBehind<T> ? st.x : st.x * exponent_factor(a) + kLift<T>;
    dp0[u] = all4(st.y);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      qf[u][f] = load_piece<T, WHOLE>(a.q, q[u].row, q[u].h, f * KF + g4 * E, a.D);
      gf[u][f] = load_piece<T, WHOLE>(a.dout, q[u].row, q[u].h, f * KF + g4 * E, a.D);
      if (a.scale < 0.f) qf[u][f] = negated<T>(qf[u][f]);
    }
  }
  if constexpr (W > DP) {
    for (int x = tid; x < NB * BK; x += NT)
#pragma unroll
      for (int e = DP; e < W; e += E) {
        *reinterpret_cast<u32x4*>(&ks[0][0] + x * LD + e) = u32x4{0u, 0u, 0u, 0u};
        *reinterpret_cast<u32x4*>(&vs[0][0] + x * LD + e) = u32x4{0u, 0u, 0u, 0u};
      }
  }
  const float c = score_factor<T>(a);
  f32x4 dq[QT][DT];
#pragma unroll
  for (int u = 0; u < QT; ++u)
#pragma unroll
    for (int d = 0; d < DT; ++d) dq[u][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int32_t t = t0; t < t1; ++t) {
    const int buf = NB == 1 ? 0 : (t - t0) & 1;
    if constexpr (NB == 1) wave_sync();
    kt.put(a, ks[buf], LD, vs[buf], LD, bias[buf], tid);
    if constexpr (NB == 1) wave_sync();
    else __syncthreads();
    if (t + 1 < t1) {
      kt.template fetch<WHOLE>(a, sk, t + 1, kh, tid);
      kt.next(a, sk, t + 2, t1, tid);
    }
#pragma unroll
    for (int k = 0; k < BK / 16 / TILES; ++k) {
      f32x4 s[QT][TILES], dp[QT][TILES];
#pragma unroll
      for (int x = 0; x < TILES; ++x) {
        const int r = (k * TILES + x) * 16;
        const f32x4 b = *reinterpret_cast<const f32x4*>(bias[buf] + r + g4 * 4);  // minus infinity for keys that are not there
#pragma unroll
        for (int u = 0; u < QT; ++u) {
          s[u][x] = b;
          dp[u][x] = dp_start<T>(dp0[u]);
        }
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const Piece kf = row_piece(ks[buf], LD, r + i, f * KF + g4 * E), vf = row_piece(vs[buf], LD, r + i, f * KF + g4 * E);
#pragma unroll
          for (int u = 0; u < QT; ++u) {
            s[u][x] = mma<T>(kf, qf[u][f], s[u][x]);
            dp[u][x] = mma<T>(vf, gf[u][f], dp[u][x]);
          }
        }
#pragma unroll
        for (int u = 0; u < QT; ++u) p_and_e<T>(s[u][x], dp[u][x], c, all4(shift[u]), dp0[u]);
      }
      Piece e[QT];
#pragma unroll
      for (int u = 0; u < QT; ++u) e[u] = as_piece<T>(dp[u]);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const Piece kc = column_piece(ks[buf], LD, k * 16 * TILES, d * 16, lane);
#pragma unroll
        for (int u = 0; u < QT; ++u) dq[u][d] = mma<T>(kc, e[u], dq[u][d]);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    if (q[u].row < 0) continue;
    if (splits > 1) {
      const int32_t slot = slot_of(a.ql, at.g, sq) + quotient(at.tile * BQ + (wave * QT + u) * 16 + i, a.share);
      const int64_t all = (int64_t)a.ql.slots * a.H;
      float* to = part + (split * all + stat_at(a, slot, q[u].h)) * DP + g4 * 4;
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(to + d * 16) = dq[u][d];
      continue;
    }
    T* to = row_of_head<T>(a.dq, q[u].row, q[u].h);
#pragma unroll
    for (int d = 0; d < DT; ++d) store4<T, WHOLE>(to, d * 16 + g4 * 4, dq[u][d] * a.scale, a.D);
  }
}

// Sums of the stretches, 64 rows of a head a workgroup, four elements a thread; N arrays of DP sums lie side by side in a part.
template <typename T, int DP, int N, bool WHOLE>
__global__ __launch_bounds__(256) void k_attention_sum(Attn a, GroupList l, TileGrid tg, int heads, int splits, const float* part, Heads to0, Heads to1,
                                                       float by0, float by1) {
  constexpr int LANES = N * DP / 4, ROWS = 64;
  const int tid = threadIdx.x, h = blockIdx.x / tg.tiles, e = tid % LANES * 4;
  const TileAt at = tile_at<ROWS>(a, l, tg, blockIdx.x - h * tg.tiles, tid & 63);
  if (at.g < 0) return;
  const Span sp = span_of(l, at.g);
  if (at.tile > sp.len / ROWS) return;
  const int32_t slot = slot_of(l, at.g, sp);
  const uint64_t all = (uint64_t)(uint32_t)l.slots * heads * (N * DP);
  for (int r = tid / LANES; r < ROWS; r += 256 / LANES) {
    const int32_t p = at.tile * ROWS + r, row = p < sp.len ? row_at(l, sp.at + p) : -1;
    if (row < 0) continue;
    const float* from = part + ((uint64_t)(uint32_t)(slot + p) * heads + h) * (N * DP) + e;
    f32x4 s = all4(0.f);
#pragma unroll 4
    for (int k = 0; k < splits; ++k) s += *reinterpret_cast<const f32x4*>(from + k * all);
    if (N == 1 || e < DP) store4<T, WHOLE>(row_of_head<T>(to0, row, h), e, s * by0, a.D);
    else                  store4<T, WHOLE>(row_of_head<T>(to1, row, h), e - DP, s * by1, a.D);
  }
}

// ---- which kernels -----------------------------------------------------------------------------------------
struct Plan {
  bool group;
  int rows, keys;  // of a workgroup of k_attention_dq: 128 or 16; of k_attention_dkv: 256, 128 or 16
  TileGrid tq, tk, sum_q, sum_k;
  int splits_q, splits_k;
  bool fits;
  size_t stats, parts_q, parts_k, bytes;  // of the workspace: stats, then the parts of dq, then those of dk and dv
};
// Stretches of the other side's rows, 256 rows each at least, so that tiles fill the chip; lists of uneven groups twice over, as the
// tiles of the long groups take longest.  Stretches are paid for with sums in the workspace (2 groups of 4,096 rows, 8 heads of 128
// elements: 560 us in one, 660 in two; 12 groups of 1 to 4,000 rows: 460 in one, 415 in three).
int stretches(const TileGrid& tg, int64_t groups, int waves, int64_t other) {
  const int wanted = tg.per_group.by ? kChipWaves : 2 * kChipWaves;
  if (groups < 1 || groups * waves >= wanted) return 1;
  const int64_t s = ceil_div(wanted, groups * waves), most = other / 256 > 0 ? other / 256 : 1;
  return (int)(s < most ? s : most);
}
// Does a wavefront have registers for the keys and values of a group, and for their gradients?
constexpr bool holds_group(int DP, int64_t G, size_t size) { return DP <= 32 && G <= 128 && (size == 2 || (G + 15) / 16 * DP <= 160); }
Plan plan(const Attn& a, size_t size) {
  Plan p{};
  const int DP = padded(a.D), share = a.H / a.K;
  const int64_t rows = (int64_t)a.ql.G * share;
  p.fits = rows <= INT32_MAX - 512;
  if (!p.fits) return p;
  p.group = holds_group(DP, a.kl.G, size) && rows <= 512 && share <= 16;
  if (p.group) {
    p.fits = one_launch((int64_t)a.max_groups * a.K, 64);
    return p;
  }
  bool f[4];
  // Few rows go to one wavefront.  Long lists of 16-bit keys of 64 and more elements go by 256 to eight wavefronts, which share what they
  // read (4,096 keys of 64 elements: 304 us instead of 336, of 128: 650 instead of 720; of groups of 64 keys: 217 instead of 130),
  // unless groups are uneven, where smaller tiles fill the chip better (30 of 1 to 4,000 keys of 64 elements: 1053 us instead of 1009).
  p.rows = rows > 32 ? 128 : 16;
  const bool even = tile_grid(a.kl.n, a.kl.G, 1, a.max_groups, 256, &f[1]).per_group.by != 0;
  p.keys = a.kl.G <= 32 ? 16 : size == 2 && DP >= 64 && a.kl.G >= 1024 && even ? 256 : 128;
  p.tq = tile_grid(a.ql.n, a.ql.G, share, a.max_groups, p.rows, &f[0]);
  p.tk = tile_grid(a.kl.n, a.kl.G, 1, a.max_groups, p.keys, &f[1]);
  p.sum_q = tile_grid(a.ql.n, a.ql.G, 1, a.max_groups, 64, &f[2]);
  p.sum_k = tile_grid(a.kl.n, a.kl.G, 1, a.max_groups, 64, &f[3]);
  const int64_t gq = (int64_t)p.tq.tiles * a.K, gk = (int64_t)p.tk.tiles * a.K;
  p.splits_q = stretches(p.tq, gq, p.rows == 16 ? 1 : 4, a.kl.G);
  p.splits_k = stretches(p.tk, gk, p.keys == 16 ? 1 : p.keys / 32, rows);
  const int64_t stats = ceil_div((int64_t)a.ql.n * a.H * (DP * (int64_t)size / 16), 256);
  p.fits = f[0] && f[1] && one_launch_in_order(gq * p.splits_q, p.rows == 16 ? 64 : 256) && (int64_t)a.ql.n * a.H <= INT32_MAX && one_launch(stats, 256) &&
           one_launch_in_order(gk * p.splits_k, p.keys == 16 ? 64 : p.keys == 128 ? 256 : 512);
  if (p.splits_q > 1) p.fits = p.fits && f[2] && one_launch((int64_t)p.sum_q.tiles * a.H, 256);
  if (p.splits_k > 1) p.fits = p.fits && f[3] && one_launch((int64_t)p.sum_k.tiles * a.K, 256);
  p.stats = align_up((size_t)a.ql.n * a.H * 8, 256);
  p.parts_q = p.splits_q > 1 ? align_up((size_t)p.splits_q * a.ql.slots * a.H * DP * 4, 256) : 0;
  p.parts_k = p.splits_k > 1 ? align_up((size_t)p.splits_k * a.kl.slots * a.K * DP * 8, 256) : 0;
  p.bytes = p.stats + p.parts_q + p.parts_k;
  return p;
}

template <typename T, int DP, int KT, bool WHOLE> int group_launch(const Attn& a, hipStream_t st) {
  const int hw = heads_together(a.K);
  const Items items = make_items(a.max_groups, a.K / hw, 1);
  if (items.total == 0) return FF_OK;
  if (hw == 4)      k_attention_backward_group<T, DP, KT, 4, WHOLE><<<items.total, 256, 0, st>>>(a, items);
  else if (hw == 2) k_attention_backward_group<T, DP, KT, 2, WHOLE><<<items.total, 128, 0, st>>>(a, items);
  else              k_attention_backward_group<T, DP, KT, 1, WHOLE><<<items.total, 64, 0, st>>>(a, items);
  return launch_status();
}
template <typename T, int DP, bool WHOLE> int run(Attn a, const Plan& p, char* ws, hipStream_t st) {
  if constexpr (DP <= 32) {
    if (p.group) {
      const int kt = (a.kl.G + 15) / 16;
      if (kt <= 2) return group_launch<T, DP, 2, WHOLE>(a, st);
      if (kt <= 4) return group_launch<T, DP, 4, WHOLE>(a, st);
      if (kt <= 5) return group_launch<T, DP, 5, WHOLE>(a, st);
      if constexpr (holds_group(DP, 128, sizeof(T))) {
        if (kt <= 6) return group_launch<T, DP, 6, WHOLE>(a, st);
        return group_launch<T, DP, 8, WHOLE>(a, st);
      }
    }
  }
  // rows of a tile of the other side: fewer barriers, or (float32) fewer registers (64 elements: 16-bit 253 us instead of 272, float32 267
  // instead of 288)
  constexpr int BK = sizeof(T) == 2 ? 64 : 32;
  a.stats = reinterpret_cast<float2*>(ws);
  float *pq = reinterpret_cast<float*>(ws + p.stats), *pk = reinterpret_cast<float*>(ws + p.stats + p.parts_q);
  if (a.ql.n > 0) {
    constexpr int PER = DP * (int)sizeof(T) / 16;
    k_attention_stats<T, DP, WHOLE><<<dim3((uint32_t)ceil_div((int64_t)a.ql.n * a.H, 256 / PER)), 256, 0, st>>>(a, make_div(a.H));
    const Order order = make_order((int64_t)p.tq.tiles * a.K * p.splits_q);
    const uint32_t grid = workgroups(order);
    if (p.rows == 128)
      k_attention_dq<T, DP, 4, 2, BK, WHOLE><<<grid, 256, 0, st>>>(a, p.tq, order, p.splits_q, pq);
    else
      k_attention_dq<T, DP, 1, 1, 32, WHOLE><<<grid, 64, 0, st>>>(a, p.tq, order, p.splits_q, pq);
    if (p.splits_q > 1)
      k_attention_sum<T, DP, 1, WHOLE><<<dim3((uint32_t)((int64_t)p.sum_q.tiles * a.H)), 256, 0, st>>>(a, a.ql, p.sum_q, a.H, p.splits_q, pq, a.dq,
                                                                                                       a.dq, a.scale, a.scale);
  }
  if (a.kl.n > 0) {
    const Order order = make_order((int64_t)p.tk.tiles * a.K * p.splits_k);
    const uint32_t grid = workgroups(order);
    if (p.keys == 16) {
      k_attention_dkv<T, DP, 1, 1, 32, WHOLE><<<grid, 64, 0, st>>>(a, p.tk, order, p.splits_k, pk);
    } else if (p.keys == 128) {
      k_attention_dkv<T, DP, 4, 2, BK, WHOLE><<<grid, 256, 0, st>>>(a, p.tk, order, p.splits_k, pk);
    } else {
      if constexpr (sizeof(T) == 2 && DP >= 64) k_attention_dkv<T, DP, 8, 2, BK, WHOLE><<<grid, 512, 0, st>>>(a, p.tk, order, p.splits_k, pk);
    }
    if (p.splits_k > 1)
      k_attention_sum<T, DP, 2, WHOLE><<<dim3((uint32_t)((int64_t)p.sum_k.tiles * a.K)), 256, 0, st>>>(a, a.kl, p.sum_k, a.K, p.splits_k, pk, a.dk,
                                                                                                       a.dv, a.scale, kLower<T>);
  }
  return launch_status();
}
template <typename T, int DP> int run_whole(const Attn& a, const Plan& p, char* ws, hipStream_t st) {
  bool whole = true;
  for (const Heads* x : {&a.q, &a.k, &a.v, &a.out, &a.dout, &a.dq, &a.dk, &a.dv}) whole = whole && whole_pieces(*x, a.D, sizeof(T));
  return whole ? run<T, DP, true>(a, p, ws, st) : run<T, DP, false>(a, p, ws, st);
}
template <typename T> int run_type(const Attn& a, const Plan& p, char* ws, hipStream_t st) {
  switch (padded(a.D)) {
    case 16: return run_whole<T, 16>(a, p, ws, st);
    case 32: return run_whole<T, 32>(a, p, ws, st);
    case 64: return run_whole<T, 64>(a, p, ws, st);
    default: return run_whole<T, 128>(a, p, ws, st);
  }
}

}  // namespace

size_t attention_backward_workspace_bytes(const Attn& a, int dtype) { return plan(a, dtype == FF_F32 ? 4 : 2).bytes; }

int attention_backward_launch(const Attn& a, int dtype, void* workspace, hipStream_t stream) {
  const Plan p = plan(a, dtype == FF_F32 ? 4 : 2);
  if (!p.fits) return FF_ERR_UNSUPPORTED;
  char* ws = reinterpret_cast<char*>(workspace);
  return dtype == FF_F32    ? run_type<float>(a, p, ws, stream)
         : dtype == FF_BF16 ? run_type<bf16_t>(a, p, ws, stream)
                            : run_type<f16_t>(a, p, ws, stream);
}

}  // namespace ff
