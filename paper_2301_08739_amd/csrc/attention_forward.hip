// Attention over the caller's rows, forward.  One pass over the keys with the running maximum and sum of the softmax, scores and
// probabilities in registers only.  Scores are computed with the keys down and the queries across (K Q^T), so that a lane holds
// scores of one query, and the probabilities are the right operand of (out)^T = V^T P^T as they lie in the registers.
#include "attention_mx.h"

namespace ff {
namespace {

// ---- short groups: a wavefront holds all keys and values of a group and head ----------------------------------
// Keys and values come through LDS into registers once (values turned there), the queries by CH rows, of which a wavefront takes 16 at
// a time; results go back the way the queries came.  Region A holds keys, then queries, then results; B values.  Of 32 elements and
// more B is A: two more barriers, and twice the wavefronts a compute unit has LDS for.
//
// Large launches are near the memory's rate (240,000 rows, groups of 69, 8 heads of 32 elements of 16 bits: 118 us, 4.2 TB/s; groups of 64,
// 16 elements: 58 us, 4.2 TB/s), small ones a chain of three trips (lists, rows, results; 30,000 rows: 12 us), float32 the matrix unit
// (80,000 rows, groups of 128, 16 elements: 72 us, 73 TFLOP/s, the unit 51 % busy).
template <typename T, int DP, int KT, int HW, bool WHOLE>
__global__ __launch_bounds__(64 * HW, KT * DP <= 256 ? 2 : 1) void k_attention_group(Attn a, Items items) {
  constexpr int KF = Mx<T>::KF, E = Mx<T>::E, TILES = Mx<T>::TILES, NF = (DP + KF - 1) / KF, DT = DP / 16, NT = 64 * HW;
  constexpr int CH = DP * (int)sizeof(T) <= 32 ? 64 : DP * (int)sizeof(T) <= 64 ? 32 : 16;  // (two pieces a thread)
  constexpr int KP = (KT + TILES - 1) / TILES, RK = KP * TILES * 16, LD = DP + 16 / (int)sizeof(T);
  constexpr bool TWO = DP * sizeof(T) <= 32;
  constexpr int PITCH = (RK > CH ? RK : CH) * LD;
  typedef KeyPieces<T, DP, HW, KT * 16> KeyP;
  typedef QueryPieces<T, DP, HW, CH> QueryP;
  __shared__ __attribute__((aligned(16))) T region[TWO ? 2 : 1][HW * PITCH];
  __shared__ __attribute__((aligned(16))) float bias[RK], lses[HW][CH];
  T *const ra = region[0], *const rb = region[TWO ? 1 : 0];
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, i = lane & 15, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  touch_arguments(a);
  const uint32_t rest = quotient(blockIdx.x, items.sets), group = quotient(rest, items.parts);
  const int kh0 = (blockIdx.x - rest * items.sets.by) * HW, h0 = kh0 * (int)a.share.by;
  const Span sq = span_of(a.ql, group), sk = span_of(a.kl, group);
  const int32_t per = (sq.len + (int32_t)items.parts.by - 1) / (int32_t)items.parts.by;
  const int32_t first = (int32_t)(rest - group * items.parts.by) * per, last = first + per < sq.len ? first + per : sq.len;
  if ((int32_t)group >= groups_of(a) || first >= last) return;
  const int32_t PC = quotient(CH, a.share);  // positions of a chunk

  KeyP kp;
  QueryP qp;
  Piece kr[KeyP::H::U], vr[KeyP::H::U], qr[QueryP::H::U];
  kp.place(tid);
  kp.ask(a, sk);
  qp.place(a, tid);
  qp.ask(a, sq, first);
  kp.look(a, sk);
  kp.template fetch<WHOLE>(kr, a.k, kh0, a.D);
  kp.template fetch<WHOLE>(vr, a.v, kh0, a.D);
  int32_t end = first + PC < last ? first + PC : last;
  qp.look(a, sq, first, end);
  qp.template fetch<WHOLE>(qr, a.q, h0, a.D);
  qp.ask(a, sq, first + PC);
  if constexpr (KT * 16 < RK) {  // values of the keys that make the last piece whole
    for (int x = tid; x < HW * (RK - KT * 16) * LD / E; x += NT) {
      const int w = x / ((RK - KT * 16) * LD / E);
      *reinterpret_cast<u32x4*>(rb + w * PITCH + KT * 16 * LD + (x - w * ((RK - KT * 16) * LD / E)) * E) = u32x4{0u, 0u, 0u, 0u};
    }
  }
  kp.put(ra, PITCH, LD, kr);
  if (TWO) kp.put(rb, PITCH, LD, vr);
  if (kp.head == 0 && kp.c == 0) {
#pragma unroll
    for (int u = 0; u < KeyP::H::U; ++u)
      if (kp.first + u * KeyP::H::STEP < KT * 16) bias[kp.first + u * KeyP::H::STEP] = kp.live >> u & 1 ? 0.f : -INFINITY;
  }
  __syncthreads();
  T *const ta = ra + wave * PITCH, *const tb = rb + wave * PITCH;
  Piece kf[KT][NF], vf[DT][KP];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      if constexpr (DP < KF) {  // zero behind the row's end
        kf[t][f] = row_piece(ta, LD, t * 16 + i, g4 * E % DP);
        if (g4 * E >= DP) kf[t][f].q = u32x4{0u, 0u, 0u, 0u};
      } else {
        kf[t][f] = row_piece(ta, LD, t * 16 + i, f * KF + g4 * E);
      }
      if (a.scale < 0.f) kf[t][f] = negated<T>(kf[t][f]);
    }
  if (!TWO) {
    __syncthreads();
    kp.put(rb, PITCH, LD, vr);
    __syncthreads();
  }
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int t = 0; t < KP; ++t) vf[d][t] = column_piece(tb, LD, t * 16 * TILES, d * 16, lane);
  const float c = exponent_factor(a);

  for (int32_t p0 = first; p0 < last; p0 += PC) {
    __syncthreads();  // keys, values and the last chunk's results have been read
    qp.put(ra, PITCH, LD, qr);
    QueryP now = qp;
    const int32_t rows = (end - p0) * (int32_t)a.share.by;
    if (p0 + PC < last) {
      end = p0 + 2 * PC < last ? p0 + 2 * PC : last;
      qp.look(a, sq, p0 + PC, end);
      qp.template fetch<WHOLE>(qr, a.q, h0, a.D);
      qp.ask(a, sq, p0 + 2 * PC);
    }
    __syncthreads();
    for (int32_t r0 = 0; r0 < rows; r0 += 16) {
      Piece qf[NF];
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        if constexpr (DP < KF) {
          qf[f] = row_piece(ta, LD, r0 + i, g4 * E % DP);
          if (g4 * E >= DP) qf[f].q = u32x4{0u, 0u, 0u, 0u};
        } else {
          qf[f] = row_piece(ta, LD, r0 + i, f * KF + g4 * E);
        }
      }
      f32x4 s[KP * TILES];
#pragma unroll
      for (int t = 0; t < KP * TILES; ++t) s[t] = t < KT ? *reinterpret_cast<const f32x4*>(bias + t * 16 + g4 * 4) : all4(0.f);
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int f = 0; f < NF; ++f) s[t] = mma<T>(kf[t][f], qf[f], s[t]);
      float top = kLowest;
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[t][r]);
      top = over_lanes16_max(top);
      top = top > kLowest ? top * c : 0.f;
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[t][r] = exp2_fast(fmaf(s[t][r], c, -top));
          sum += s[t][r];
        }
      sum = over_lanes16_sum(sum);
      f32x4 o[DT];
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] = all4(0.f);
#pragma unroll
      for (int t = 0; t < KP; ++t) {
        const Piece p = as_piece<T>(s + t * TILES);
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = mma<T>(vf[d][t], p, o[d]);
      }
      const float by = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);  // no key: zero
      wave_sync();
#pragma unroll
      for (int d = 0; d < DT; ++d) store4<T, true>(ta + (r0 + i) * LD, d * 16 + g4 * 4, o[d] * by, DP);  // over the queries they are of
      if (g4 == 0) lses[wave][r0 + i] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
    __syncthreads();
    now.template store<WHOLE>(a.out, h0, a.D, ra, PITCH, LD);
    if (a.lse && now.c == 0) {
#pragma unroll
      for (int u = 0; u < QueryP::H::U; ++u)
        if (now.row[u] >= 0 && now.v[u] < CH) a.lse[stat_at(a, now.row[u], h0 + now.h[u])] = lses[now.w[u]][now.v[u]];
    }
  }
}

// ---- any lengths: tiles of keys and values through LDS, shared by the wavefronts of a workgroup ---------------
// NW wavefronts of QT x 16 rows of queries each.  Tiles of BK keys lie twice in LDS: one is read while the next one is written, its
// rows fetched into registers a tile ahead and their numbers two.  splits > 1: each workgroup takes a stretch of a group's keys and
// leaves sums, maximum and total in the workspace; k_attention_join brings them together.
//
// The vector unit is what such a kernel waits for (an exponential takes as long as four other instructions), so little else is done a
// score.  Products start from minus infinity instead of zero for keys that are not there.  The running maximum may be too low by a
// factor of 2^8 in p (no type's range minds), so that lanes need not compare notes: only where a lane finds a score beyond that, or its
// row has met no key yet, is the maximum made good and what was summed brought down.  The sum of p is one of float32 additions: a
// product with ones would sum the rounded p, and lse would be 2^-9 off.  4 groups of 4,096 rows, 8 heads, bfloat16: 960 TFLOP/s of 128
// elements, 710 of 64, 500 of 32; 12 groups of 1 to 6,000 rows of 64: 300 us, vector unit 70 % busy, matrix unit 35 %.  One wavefront to a
// workgroup (32 rows and fewer) reads keys and values at 4.8 TB/s (one row, 32 heads on 8 of 65,537 keys, 128 elements: 56 us, join 6.5).
// A wavefront without rows, in a group's last tile, only loads (200 rows: 46.4 us instead of 47.3).
template <typename T, int DP, int NW, int QT, int BK, bool WHOLE>
__global__ __launch_bounds__(64 * NW, DP * sizeof(T) <= (NW == 1 ? 256 : 128) || (DP == 64 && NW == 4) ? 2 : 1) void k_attention_tiles(Attn a, TileGrid tg, Order order, int splits, float* part) {
  constexpr int KF = Mx<T>::KF, E = Mx<T>::E, TILES = Mx<T>::TILES, NF = (DP + KF - 1) / KF, DT = DP / 16, NT = 64 * NW;
  constexpr int KW = NF * KF, LDK = KW + 16 / (int)sizeof(T), LDV = DP + 32 / (int)sizeof(T), BQ = 16 * QT * NW;
  constexpr int NB = NW == 1 ? 1 : 2;  // (a wavefront alone writes when it has read)
  __shared__ __attribute__((aligned(16))) T ks[NB][BK * LDK];
  __shared__ __attribute__((aligned(16))) T vs[NB][BK * LDV];
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

  const bool busy = NW == 1 || at.tile * BQ + __builtin_amdgcn_readfirstlane(wave) * (QT * 16) < sq.len * tg.share;  // has this wavefront rows?

  KeyTiles<T, DP, BK, NT> kt;
  kt.next(a, sk, t0, t1, tid);
  QueryRow q[QT];
  Piece qf[QT][NF];
#pragma unroll
  for (int u = 0; u < QT; ++u) q[u] = query_row(a, sq, kh, at.tile * BQ + (wave * QT + u) * 16 + i);
  if (t0 < t1) kt.template fetch<WHOLE>(a, sk, t0, kh, tid);
  kt.next(a, sk, t0 + 1, t1, tid);
#pragma unroll
  for (int u = 0; u < QT; ++u)
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      qf[u][f] = load_piece<T, WHOLE>(a.q, q[u].row, q[u].h, f * KF + g4 * E, a.D);
      if (a.scale < 0.f) qf[u][f] = negated<T>(qf[u][f]);
    }
  if constexpr (KW > DP) {  // columns behind the rows' ends: zero in both operands
    for (int x = tid; x < NB * BK; x += NT)
#pragma unroll
      for (int e = DP; e < KW; e += E) *reinterpret_cast<u32x4*>(&ks[0][0] + x * LDK + e) = u32x4{0u, 0u, 0u, 0u};
  }
  const float c = exponent_factor(a), far = 8.f / c;
  f32x4 o[QT][DT], sum[QT];
  float most[QT], shift[QT];  // running maximum of the scores, -infinity until the row has met a key, and what it adds to the exponents
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    most[u] = -INFINITY;
    shift[u] = 0.f;
    sum[u] = all4(0.f);
#pragma unroll
    for (int d = 0; d < DT; ++d) o[u][d] = all4(0.f);
  }
  auto tile = [&](const T* kb, const T* vb, const float* bb) {
    f32x4 s[QT][BK / 16];
#pragma unroll
    for (int k = 0; k < BK / 16; ++k) {
      const f32x4 b = *reinterpret_cast<const f32x4*>(bb + k * 16 + g4 * 4);
#pragma unroll
      for (int u = 0; u < QT; ++u) s[u][k] = b;
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        const Piece kf = row_piece(kb, LDK, k * 16 + i, f * KF + g4 * E);
#pragma unroll
        for (int u = 0; u < QT; ++u) s[u][k] = mma<T>(kf, qf[u][f], s[u][k]);
      }
    }
    bool raise = false;
    float top[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      top[u] = s[u][0][0];
#pragma unroll
      for (int k = 0; k < BK / 16; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) top[u] = fmaxf(top[u], s[u][k][r]);
      raise |= top[u] > most[u] + far;
    }
    if (__any(raise)) {
#pragma unroll
      for (int u = 0; u < QT; ++u) {
        const float m = over_lanes16_max(top[u]);
        if (m > most[u]) {
          const float f = exp2_fast(c * (most[u] - m));
          sum[u] *= f;
#pragma unroll
          for (int d = 0; d < DT; ++d) o[u][d] *= f;
          most[u] = m;
          shift[u] = -c * m;
        }
      }
    }
    Piece p[QT][BK / 16 / TILES];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
#pragma unroll
      for (int k = 0; k < BK / 16; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[u][k][r] = exp2_fast(fmaf(s[u][k][r], c, shift[u]));
          sum[u][r] += s[u][k][r];
        }
#pragma unroll
      for (int k = 0; k < BK / 16 / TILES; ++k) p[u][k] = as_piece<T>(s[u] + k * TILES);
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int k = 0; k < BK / 16 / TILES; ++k) {
        const Piece vf = column_piece(vb, LDV, k * 16 * TILES, d * 16, lane);
#pragma unroll
        for (int u = 0; u < QT; ++u) o[u][d] = mma<T>(vf, p[u][k], o[u][d]);
      }
  };
  for (int32_t t = t0; t < t1; ++t) {
    const int buf = NB == 1 ? 0 : (t - t0) & 1;
    if constexpr (NB == 1) wave_sync();
    kt.put(a, ks[buf], LDK, vs[buf], LDV, bias[buf], tid);
    if constexpr (NB == 1) wave_sync();
    else __syncthreads();
    if (t + 1 < t1) {
      kt.template fetch<WHOLE>(a, sk, t + 1, kh, tid);
      kt.next(a, sk, t + 2, t1, tid);
    }
    if (busy) tile(ks[buf], vs[buf], bias[buf]);
  }
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    const float total = over_lanes16_sum((sum[u][0] + sum[u][1]) + (sum[u][2] + sum[u][3]));
    const float top = most[u] > -INFINITY ? -shift[u] : kLowest;
    if (q[u].row < 0) continue;
    const int64_t at_row = stat_at(a, q[u].row, q[u].h);
    if (splits > 1) {
      const int32_t slot = slot_of(a.ql, at.g, sq) + quotient(at.tile * BQ + (wave * QT + u) * 16 + i, a.share);
      const int64_t all = (int64_t)a.ql.slots * a.H, at_slot = stat_at(a, slot, q[u].h);
      float* ml = part + (split * all + at_slot) * 2;
      float* po = part + splits * all * 2 + (split * all + at_slot) * DP;
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(po + d * 16 + g4 * 4) = o[u][d];
      if (g4 == 0) {
        ml[0] = top;
        ml[1] = total;
      }
      continue;
    }
    const float by = total == 0.f ? 0.f : __builtin_amdgcn_rcpf(total);  // no key: zero
    T* out = row_of_head<T>(a.out, q[u].row, q[u].h);
#pragma unroll
    for (int d = 0; d < DT; ++d) store4<T, WHOLE>(out, d * 16 + g4 * 4, o[u][d] * by, a.D);
    if (a.lse && g4 == 0) a.lse[at_row] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
  }
}

constexpr int kMostSplits = 512;  // of a group's keys

// The stretches of one row and head.  A few lanes hold a stretch's sums, four elements each, so that a workgroup's loads cover many
// stretches at once; their weights are worked out first, a stretch a thread.
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attention_join(Attn a, TileGrid tg, int splits, const float* part) {
  constexpr int LANES = DP / 4, AT_ONCE = 256 / LANES;
  __shared__ float weight[kMostSplits], tops[4], sums[4];
  __shared__ __attribute__((aligned(16))) float os[AT_ONCE][DP];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kh = blockIdx.x / tg.tiles;
  const TileAt at = tile_at<1>(a, a.ql, tg, blockIdx.x - kh * tg.tiles, lane);
  if (at.g < 0) return;
  const Span sq = span_of(a.ql, at.g);
  const QueryRow q = query_row(a, sq, kh, at.tile);
  if (q.row < 0) return;
  const int64_t all = (int64_t)a.ql.slots * a.H, at_row = stat_at(a, q.row, q.h);
  const int64_t at_slot = stat_at(a, slot_of(a.ql, at.g, sq) + quotient(at.tile, a.share), q.h);
  const float2* const ml = reinterpret_cast<const float2*>(part) + at_slot;
  const float* const po = part + splits * all * 2 + at_slot * DP + tid % LANES * 4;
  constexpr int MINE = kMostSplits / 256;
  float2 mine[MINE];
  float top = kLowest;
#pragma unroll
  for (int s = 0; s < MINE; ++s) {
    mine[s] = s * 256 + tid < splits ? ml[(s * 256 + tid) * all] : make_float2(kLowest, 0.f);
    top = fmaxf(top, mine[s].x);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  float total = 0.f;
#pragma unroll
  for (int s = 0; s < MINE; ++s) {
    const float f = exp2_fast(mine[s].x - top);
    if (s * 256 + tid < splits) weight[s * 256 + tid] = f;
    total = fmaf(f, mine[s].y, total);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
  if (lane == 0) sums[wave] = total;
  __syncthreads();
  total = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = tid / LANES; s < splits; s += AT_ONCE) o += *reinterpret_cast<const f32x4*>(po + s * all * DP) * weight[s];
  *reinterpret_cast<f32x4*>(&os[tid / LANES][tid % LANES * 4]) = o;
  __syncthreads();
  if (tid < a.D) {
    float v = 0.f;
#pragma unroll 8
    for (int s = 0; s < AT_ONCE; ++s) v += os[s][tid];
    Elem<T>::store(row_of_head<T>(a.out, q.row, q.h) + tid, total == 0.f ? 0.f : v / total);
  }
  if (tid == 0 && a.lse) a.lse[at_row] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
}

// ---- which kernel ---------------------------------------------------------------------------------------
struct Plan {
  bool group;       // k_attention_group
  int parts;        // of a group's queries there
  int rows;         // of a workgroup of k_attention_tiles: 256, 128 or 16
  TileGrid tg, join;
  int splits;
  bool fits;
  size_t bytes;
};
Plan plan(const Attn& a, size_t size) {
  Plan p{};
  const int DP = padded(a.D), share = a.H / a.K;
  const int64_t rows = (int64_t)a.ql.G * share;
  p.fits = rows <= INT32_MAX - 512;
  if (!p.fits) return p;
  p.group = a.kl.G <= 128 && DP <= (size == 4 ? 32 : 64) && share <= 16;
  if (p.group) {
    const int64_t waves = (int64_t)a.max_groups * a.K, tiles = ceil_div(rows, 16);
    const int64_t want = waves ? ceil_div(kChipWaves, waves) : 1;
    p.parts = (int)(want < tiles ? want : tiles);
    p.fits = one_launch(waves * p.parts, 64);
    return p;
  }
  // 128 rows (four wavefronts of 32) unless there are fewer than a third of that.  128 elements of 16 bits, two rounds of the chip and
  // more: 256 rows, which halves what a thread keeps in flight (4 groups of 4,096 rows, 8 heads: 274 us instead of 311; but 256
  // workgroups, of 2 groups, 243 instead of 160).
  auto grid = [&](int r) {
    p.rows = r;
    p.tg = tile_grid(a.ql.n, a.ql.G, share, a.max_groups, r, &p.fits);
    return (int64_t)p.tg.tiles * a.K;
  };
  int64_t groups = grid(rows > 32 ? 128 : 16);
  if (size == 2 && DP == 128 && rows >= 1024 && groups >= 1024) groups = grid(256);
  const int64_t waves = groups * (p.rows == 16 ? 1 : 4);
  int64_t s = groups ? ceil_div(p.rows == 16 ? kChipWaves : 2 * kChipWaves, waves ? waves : 1) : 1;
  const int64_t most = a.kl.G / 256 > 0 ? a.kl.G / 256 : 1;
  if (s > most) s = most;
  if (s > kMostSplits) s = kMostSplits;
  if (waves * 2 > kChipWaves) s = 1;
  p.splits = (int)s;
  p.fits = p.fits && one_launch_in_order(groups * s, p.rows == 16 ? 64 : 2 * p.rows);
  if (s > 1) {
    bool fits;
    p.join = tile_grid(a.ql.n, a.ql.G, share, a.max_groups, 1, &fits);
    p.fits = p.fits && fits && one_launch((int64_t)p.join.tiles * a.K, 256);
    p.bytes = (size_t)s * a.ql.slots * a.H * (2 + DP) * 4;
  }
  return p;
}

template <typename T, int DP, int KT, bool WHOLE> int group_launch(const Attn& a, const Plan& p, hipStream_t st) {
  const int hw = heads_together(a.K);
  const Items items = make_items(a.max_groups, a.K / hw, p.parts);
  if (items.total == 0) return FF_OK;
  if (hw == 4)      k_attention_group<T, DP, KT, 4, WHOLE><<<items.total, 256, 0, st>>>(a, items);
  else if (hw == 2) k_attention_group<T, DP, KT, 2, WHOLE><<<items.total, 128, 0, st>>>(a, items);
  else              k_attention_group<T, DP, KT, 1, WHOLE><<<items.total, 64, 0, st>>>(a, items);
  return launch_status();
}
template <typename T, int DP, bool WHOLE> int run(const Attn& a, const Plan& p, float* ws, hipStream_t st) {
  if constexpr (DP <= (sizeof(T) == 4 ? 32 : 64)) {
    if (p.group) {
      const int kt = (a.kl.G + 15) / 16;
      if (kt <= 2) return group_launch<T, DP, 2, WHOLE>(a, p, st);
      if (kt <= 4) return group_launch<T, DP, 4, WHOLE>(a, p, st);
      if (kt <= 5) return group_launch<T, DP, 5, WHOLE>(a, p, st);
      if (kt <= 6) return group_launch<T, DP, 6, WHOLE>(a, p, st);
      return group_launch<T, DP, 8, WHOLE>(a, p, st);
    }
  }
  const Order order = make_order((int64_t)p.tg.tiles * a.K * p.splits);
  const uint32_t grid = workgroups(order);
  if (grid == 0) return FF_OK;
  if (p.rows == 16) {
    k_attention_tiles<T, DP, 1, 1, 32, WHOLE><<<grid, 64, 0, st>>>(a, p.tg, order, p.splits, ws);
  } else if (p.rows == 128) {
    k_attention_tiles<T, DP, 4, 2, 64, WHOLE><<<grid, 256, 0, st>>>(a, p.tg, order, p.splits, ws);
  } else {
    if constexpr (sizeof(T) == 2 && DP == 128) k_attention_tiles<T, DP, 8, 2, 64, WHOLE><<<grid, 512, 0, st>>>(a, p.tg, order, p.splits, ws);
  }
  if (p.splits > 1) k_attention_join<T, DP><<<dim3((uint32_t)((int64_t)p.join.tiles * a.K)), 256, 0, st>>>(a, p.join, p.splits, ws);
  return launch_status();
}
template <typename T, int DP> int run_whole(const Attn& a, const Plan& p, float* ws, hipStream_t st) {
  bool whole = true;
  for (const Heads* x : {&a.q, &a.k, &a.v, &a.out}) whole = whole && whole_pieces(*x, a.D, sizeof(T));
  return whole ? run<T, DP, true>(a, p, ws, st) : run<T, DP, false>(a, p, ws, st);
}
template <typename T> int run_type(const Attn& a, const Plan& p, float* ws, hipStream_t st) {
  switch (padded(a.D)) {
    case 16: return run_whole<T, 16>(a, p, ws, st);
    case 32: return run_whole<T, 32>(a, p, ws, st);
    case 64: return run_whole<T, 64>(a, p, ws, st);
    default: return run_whole<T, 128>(a, p, ws, st);
  }
}

}  // namespace

size_t attention_workspace_bytes(const Attn& a, int dtype) { return plan(a, dtype == FF_F32 ? 4 : 2).bytes; }

int attention_launch(const Attn& a, int dtype, void* workspace, hipStream_t stream) {
  const Plan p = plan(a, dtype == FF_F32 ? 4 : 2);
  if (!p.fits) return FF_ERR_UNSUPPORTED;
  float* ws = reinterpret_cast<float*>(workspace);
  return dtype == FF_F32    ? run_type<float>(a, p, ws, stream)
         : dtype == FF_BF16 ? run_type<bf16_t>(a, p, ws, stream)
                            : run_type<f16_t>(a, p, ws, stream);
}

}  // namespace ff
