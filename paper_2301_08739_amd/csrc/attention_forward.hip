// Attention over the caller's rows, forward.  One pass over the keys with the running maximum and sum of the softmax, scores and
// probabilities in registers only.  Scores are computed with the keys down and the queries across (K Q^T), so that a lane holds
// scores of one query, and the probabilities are the right operand of (out)^T = V^T P^T as they lie in the registers.
#include "attention_mx.h"

namespace ff {
namespace {

// ---- short groups: a wavefront holds all keys and values of a group and head ----------------------------------
// Keys and values are read once into registers (values through LDS, which turns them), the queries go by 16 at a time.
template <typename T, int DP, int KT>
__global__ __launch_bounds__(256) void k_attention_group(Attn a, int parts, bool whole, bool whole_out) {
  constexpr int KF = Mx<T>::KF, E = Mx<T>::E, TILES = Mx<T>::TILES, NF = (DP + KF - 1) / KF, DT = DP / 16;
  constexpr int KP = (KT + TILES - 1) / TILES, RK = KP * TILES * 16, LD = DP + 16 / (int)sizeof(T), PER = DP * (int)sizeof(T) / 16;
  __shared__ __attribute__((aligned(16))) T vs_all[4][RK * LD];
  __shared__ __attribute__((aligned(16))) float bias_all[4][RK];
  const int lane = threadIdx.x & 63, g4 = lane >> 4, i = lane & 15, wave = threadIdx.x >> 6;
  T* const vs = vs_all[wave];
  float* const bias = bias_all[wave];
  const int share = a.H / a.K;
  int64_t item = (int64_t)blockIdx.x * 4 + wave;
  const int kh = (int)(item % a.K);
  item /= a.K;
  const int part = (int)(item % parts);
  item /= parts;
  if (item >= groups_of(a)) return;
  const int32_t group = (int32_t)item;
  const Span sq = span_of(a.ql, group), sk = span_of(a.kl, group);
  const int32_t rows = sq.len * share;
  if (part * 16 >= rows) return;

  int32_t key[RK / 16];
#pragma unroll
  for (int t = 0; t < RK / 16; ++t) {
    const int32_t p = t * 16 + i;
    key[t] = p < sk.len ? row_at(a.kl, sk.at + p) : -1;
  }
  QueryRow q = query_row(a, sq, share, kh, part * 16 + i);
  if (a.mask) {
#pragma unroll
    for (int t = 0; t < RK / 16; ++t)
      if (key[t] >= 0 && !a.mask[key[t]]) key[t] = -1;
  }
  Piece kf[KT][NF], vr[RK / 16][(PER + 3) / 4], qf[NF];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      kf[t][f].q = u32x4{0u, 0u, 0u, 0u};
      if (key[t] >= 0) kf[t][f] = load_piece(row_of_head<const T>(a.k, key[t], kh), f * KF + g4 * E, a.D, whole);
    }
  auto fetch_q = [&]() {
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      qf[f].q = u32x4{0u, 0u, 0u, 0u};
      if (q.row >= 0) qf[f] = load_piece(row_of_head<const T>(a.q, q.row, q.h), f * KF + g4 * E, a.D, whole);
    }
  };
  fetch_q();
#pragma unroll
  for (int t = 0; t < RK / 16; ++t)
#pragma unroll
    for (int c = 0; c < (PER + 3) / 4; ++c) {
      vr[t][c].q = u32x4{0u, 0u, 0u, 0u};
      if (key[t] >= 0 && c * 4 + g4 < PER) vr[t][c] = load_piece(row_of_head<const T>(a.v, key[t], kh), (c * 4 + g4) * E, a.D, whole);
    }
#pragma unroll
  for (int t = 0; t < RK / 16; ++t) {
#pragma unroll
    for (int c = 0; c < (PER + 3) / 4; ++c)
      if (c * 4 + g4 < PER) *reinterpret_cast<u32x4*>(vs + (t * 16 + i) * LD + (c * 4 + g4) * E) = vr[t][c].q;
    if (g4 == 0) bias[t * 16 + i] = key[t] >= 0 ? 0.f : -INFINITY;
  }
  wave_sync();
  Piece vf[DT][KP];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int t = 0; t < KP; ++t) vf[d][t] = column_piece(vs, LD, t * 16 * TILES, d * 16, lane);

  const float c = a.scale * kLog2e;
  for (int32_t r0 = part * 16; r0 < rows; r0 += parts * 16) {
    const QueryRow now = q;
    f32x4 s[KP * TILES];
#pragma unroll
    for (int t = 0; t < KP * TILES; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int f = 0; f < NF; ++f) s[t] = mma<T>(kf[t][f], qf[f], s[t]);
    if (r0 + parts * 16 < rows) {
      q = query_row(a, sq, share, kh, r0 + parts * 16 + i);
      fetch_q();
    }
    float top = kLowest;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const f32x4 b = *reinterpret_cast<const f32x4*>(bias + t * 16 + g4 * 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[t][r] = fmaf(s[t][r], c, b[r]);
        top = fmaxf(top, s[t][r]);
      }
    }
    top = over_lanes16_max(top);
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[t][r] = exp2_fast(s[t][r] - top);
        sum += s[t][r];
      }
    sum = over_lanes16_sum(sum);
    f32x4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < KP; ++t) {
      const Piece p = as_piece<T>(s + t * TILES);
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] = mma<T>(vf[d][t], p, o[d]);
    }
    if (now.row < 0) continue;
    const float by = sum == 0.f ? 0.f : 1.f / sum;  // no key: zero
    T* out = row_of_head<T>(a.out, now.row, now.h);
#pragma unroll
    for (int d = 0; d < DT; ++d) store4(out, d * 16 + g4 * 4, o[d] * by, a.D, whole_out);
    if (a.lse && g4 == 0) a.lse[(int64_t)now.row * a.H + now.h] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
  }
}

// ---- any lengths: tiles of keys and values through LDS, shared by the wavefronts of a workgroup ---------------
// NW wavefronts of QT x 16 rows of queries each.  Tiles of BK keys lie twice in LDS: one is read while the next one is written, its
// rows fetched into registers a tile ahead and their numbers two.  splits > 1: each workgroup takes a stretch of a group's keys and
// leaves sums, maximum and total in the workspace; k_attention_join brings them together.
template <typename T, int DP, int NW, int QT, int BK>
__global__ __launch_bounds__(64 * NW) void k_attention_tiles(Attn a, TileGrid tg, int splits, float* part, bool whole, bool whole_out) {
  constexpr int KF = Mx<T>::KF, E = Mx<T>::E, TILES = Mx<T>::TILES, NF = (DP + KF - 1) / KF, DT = DP / 16, NT = 64 * NW;
  constexpr int KW = NF * KF, LDK = KW + 16 / (int)sizeof(T), LDV = DP + 32 / (int)sizeof(T), BQ = 16 * QT * NW;
  typedef Rows<T, DP, BK, NT> R;
  __shared__ __attribute__((aligned(16))) T ks[2][BK * LDK];
  __shared__ __attribute__((aligned(16))) T vs[2][BK * LDV];
  __shared__ __attribute__((aligned(16))) float bias[2][BK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g4 = lane >> 4, i = lane & 15;
  const int split = blockIdx.x % splits;
  const int32_t rest = blockIdx.x / splits;
  const int kh = rest / tg.tiles;
  const TileAt at = tile_at<BQ>(a, a.ql, tg, rest - kh * tg.tiles, lane);
  if (at.g < 0) return;
  const Span sq = span_of(a.ql, at.g), sk = span_of(a.kl, at.g);
  if ((int64_t)at.tile * BQ >= (int64_t)sq.len * tg.share) return;
  const int32_t tiles = (sk.len + BK - 1) / BK, per = (tiles + splits - 1) / splits;
  const int32_t t0 = split * per, t1 = t0 + per < tiles ? t0 + per : tiles;

  int32_t rows[R::U], heads[R::U];
  auto number = [&](int32_t t) {
#pragma unroll
    for (int u = 0; u < R::U; ++u) {
      const int r = R::row(tid, u);
      const int32_t p = t * BK + r;
      rows[u] = t < t1 && r < BK && p < sk.len ? row_at(a.kl, sk.at + p) : -1;
      heads[u] = kh;
      if (a.mask && rows[u] >= 0 && !a.mask[rows[u]]) rows[u] = -1;
    }
  };
  Piece kr[R::U], vr[R::U];
  float br[R::U];
  auto fetch = [&]() {
    R::fetch(kr, a.k, rows, heads, tid, a.D, whole);
    R::fetch(vr, a.v, rows, heads, tid, a.D, whole);
#pragma unroll
    for (int u = 0; u < R::U; ++u) br[u] = rows[u] >= 0 ? 0.f : -INFINITY;
  };
  number(t0);
  QueryRow q[QT];
  Piece qf[QT][NF];
#pragma unroll
  for (int u = 0; u < QT; ++u) q[u] = query_row(a, sq, tg.share, kh, at.tile * BQ + (wave * QT + u) * 16 + i);
  fetch();
  number(t0 + 1);
#pragma unroll
  for (int u = 0; u < QT; ++u)
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      qf[u][f].q = u32x4{0u, 0u, 0u, 0u};
      if (q[u].row >= 0) qf[u][f] = load_piece(row_of_head<const T>(a.q, q[u].row, q[u].h), f * KF + g4 * E, a.D, whole);
    }
  if constexpr (KW > DP) {  // columns behind the rows' ends: zero in both operands
    for (int x = tid; x < 2 * BK; x += NT)
#pragma unroll
      for (int e = DP; e < KW; e += E) *reinterpret_cast<u32x4*>(&ks[0][0] + x * LDK + e) = u32x4{0u, 0u, 0u, 0u};
  }
  const float c = a.scale * kLog2e;
  f32x4 o[QT][DT];
  float top[QT], sum[QT];
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    top[u] = kLowest;
    sum[u] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[u][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  for (int32_t t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    R::put(ks[buf], LDK, kr, tid);
    R::put(vs[buf], LDV, vr, tid);
    if (tid % R::PER == 0) {
#pragma unroll
      for (int u = 0; u < R::U; ++u)
        if (BK * R::PER % NT == 0 || R::row(tid, u) < BK) bias[buf][R::row(tid, u)] = br[u];
    }
    __syncthreads();
    if (t + 1 < t1) {
      fetch();
      number(t + 2);
    }
    f32x4 s[QT][BK / 16];
#pragma unroll
    for (int k = 0; k < BK / 16; ++k) {
#pragma unroll
      for (int u = 0; u < QT; ++u) s[u][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        const Piece kf = row_piece(ks[buf], LDK, k * 16 + i, f * KF + g4 * E);
#pragma unroll
        for (int u = 0; u < QT; ++u) s[u][k] = mma<T>(kf, qf[u][f], s[u][k]);
      }
    }
    Piece p[QT][BK / 16 / TILES];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      float m = top[u];
#pragma unroll
      for (int k = 0; k < BK / 16; ++k) {
        const f32x4 b = *reinterpret_cast<const f32x4*>(bias[buf] + k * 16 + g4 * 4);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[u][k][r] = fmaf(s[u][k][r], c, b[r]);
          m = fmaxf(m, s[u][k][r]);
        }
      }
      m = over_lanes16_max(m);
      if (__any(m > top[u])) {  // after the first tiles the maximum seldom grows
        const float f = exp2_fast(top[u] - m);
        sum[u] *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[u][d] *= f;
        top[u] = m;
      }
#pragma unroll
      for (int k = 0; k < BK / 16; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[u][k][r] = exp2_fast(s[u][k][r] - m);
          sum[u] += s[u][k][r];
        }
#pragma unroll
      for (int k = 0; k < BK / 16 / TILES; ++k) p[u][k] = as_piece<T>(s[u] + k * TILES);
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int k = 0; k < BK / 16 / TILES; ++k) {
        const Piece vf = column_piece(vs[buf], LDV, k * 16 * TILES, d * 16, lane);
#pragma unroll
        for (int u = 0; u < QT; ++u) o[u][d] = mma<T>(vf, p[u][k], o[u][d]);
      }
  }
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    const float total = over_lanes16_sum(sum[u]);
    if (q[u].row < 0) continue;
    const int64_t at_row = (int64_t)q[u].row * a.H + q[u].h;
    if (splits > 1) {
      const int64_t all = (int64_t)a.ql.n * a.H;
      float* ml = part + (split * all + at_row) * 2;
      float* po = part + splits * all * 2 + (split * all + at_row) * DP;
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(po + d * 16 + g4 * 4) = o[u][d];
      if (g4 == 0) {
        ml[0] = top[u];
        ml[1] = total;
      }
      continue;
    }
    const float by = total == 0.f ? 0.f : 1.f / total;  // no key: zero
    T* out = row_of_head<T>(a.out, q[u].row, q[u].h);
#pragma unroll
    for (int d = 0; d < DT; ++d) store4(out, d * 16 + g4 * 4, o[u][d] * by, a.D, whole_out);
    if (a.lse && g4 == 0) a.lse[at_row] = total == 0.f ? -INFINITY : (top[u] + __builtin_amdgcn_logf(total)) * kLn2;
  }
}

// One workgroup of four wavefronts a row and head: each joins every fourth stretch, then the four.
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attention_join(Attn a, TileGrid tg, int splits, const float* part) {
  __shared__ float tops[4], sums[4], os[4][DP];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kh = blockIdx.x / tg.tiles;
  const TileAt at = tile_at<1>(a, a.ql, tg, blockIdx.x - kh * tg.tiles, lane);
  if (at.g < 0) return;
  const QueryRow q = query_row(a, span_of(a.ql, at.g), tg.share, kh, at.tile);
  if (q.row < 0) return;
  const int64_t all = (int64_t)a.ql.n * a.H, at_row = (int64_t)q.row * a.H + q.h;
  const float *ml = part + at_row * 2, *po = part + splits * all * 2 + at_row * DP;
  float top = kLowest, sum = 0.f, o[(DP + 63) / 64] = {};
  for (int s = wave; s < splits; s += 4) top = fmaxf(top, ml[s * all * 2]);
  for (int s = wave; s < splits; s += 4) {
    const float f = exp2_fast(ml[s * all * 2] - top);
    sum += f * ml[s * all * 2 + 1];
#pragma unroll
    for (int e = 0; e < (DP + 63) / 64; ++e)
      if (e * 64 + lane < DP) o[e] = fmaf(f, po[s * all * DP + e * 64 + lane], o[e]);
  }
  if (lane == 0) {
    tops[wave] = top;
    sums[wave] = sum;
  }
#pragma unroll
  for (int e = 0; e < (DP + 63) / 64; ++e)
    if (e * 64 + lane < DP) os[wave][e * 64 + lane] = o[e];
  __syncthreads();
  const float m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  float f[4], total = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = exp2_fast(tops[w] - m);
    total += f[w] * sums[w];
  }
  if (tid < a.D) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) v = fmaf(f[w], os[w][tid], v);
    Elem<T>::store(row_of_head<T>(a.out, q.row, q.h) + tid, total == 0.f ? 0.f : v / total);
  }
  if (tid == 0 && a.lse) a.lse[at_row] = total == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(total)) * kLn2;
}

// ---- which kernel ---------------------------------------------------------------------------------------
struct Plan {
  bool group;       // k_attention_group
  int parts;        // of a group's queries there
  bool wide;        // k_attention_tiles: four wavefronts of 32 rows, else one of 16
  TileGrid tg, join;
  int splits;
  bool fits;
  size_t bytes;
};
Plan plan(const Attn& a, size_t size) {
  Plan p{};
  const int DP = padded(a.D), share = a.H / a.K;
  const int64_t rows = (int64_t)a.ql.G * share;
  p.fits = true;
  p.group = a.kl.G <= 128 && DP <= (size == 4 ? 32 : 64);
  if (p.group) {
    const int64_t waves = (int64_t)a.max_groups * a.K, tiles = ceil_div(rows, 16);
    const int64_t want = waves ? ceil_div(kChipWaves, waves) : 1;
    p.parts = (int)(want < tiles ? want : tiles);
    p.fits = ceil_div(waves * p.parts, 4) <= INT32_MAX;
    return p;
  }
  p.wide = rows > 32;
  const int64_t BQ = p.wide ? 128 : 16;
  p.tg = tile_grid(a.ql.n, a.ql.G, share, a.max_groups, BQ, &p.fits);
  const int64_t groups = (int64_t)p.tg.tiles * a.K, waves = groups * (p.wide ? 4 : 1);
  int64_t s = groups ? ceil_div(p.wide ? 2 * kChipWaves : kChipWaves, waves ? waves : 1) : 1;
  const int64_t most = a.kl.G / 256 > 0 ? a.kl.G / 256 : 1;
  if (s > most) s = most;
  if (waves * 2 > kChipWaves) s = 1;
  p.splits = (int)s;
  p.fits = p.fits && groups * s <= INT32_MAX;
  if (s > 1) {
    bool fits;
    p.join = tile_grid(a.ql.n, a.ql.G, share, a.max_groups, 1, &fits);
    p.fits = p.fits && fits && (int64_t)p.join.tiles * a.K <= INT32_MAX;
    p.bytes = (size_t)s * a.ql.n * a.H * (2 + DP) * 4;
  }
  return p;
}

template <typename T, int DP, int KT> int group_launch(const Attn& a, const Plan& p, bool whole, bool whole_out, hipStream_t st) {
  const int64_t waves = (int64_t)a.max_groups * a.K * p.parts;
  k_attention_group<T, DP, KT><<<dim3((uint32_t)ceil_div(waves, 4)), 256, 0, st>>>(a, p.parts, whole, whole_out);
  return launch_status();
}
template <typename T, int DP> int run(const Attn& a, const Plan& p, float* ws, hipStream_t st) {
  const bool whole = whole_pieces(a.q, a.D, sizeof(T)) && whole_pieces(a.k, a.D, sizeof(T)) && whole_pieces(a.v, a.D, sizeof(T));
  const bool whole_out = whole_pieces(a.out, a.D, sizeof(T));
  if constexpr (DP <= (sizeof(T) == 4 ? 32 : 64)) {
    if (p.group) {
      const int kt = (a.kl.G + 15) / 16;
      if (kt <= 2) return group_launch<T, DP, 2>(a, p, whole, whole_out, st);
      if (kt <= 4) return group_launch<T, DP, 4>(a, p, whole, whole_out, st);
      if (kt <= 5) return group_launch<T, DP, 5>(a, p, whole, whole_out, st);
      if (kt <= 6) return group_launch<T, DP, 6>(a, p, whole, whole_out, st);
      return group_launch<T, DP, 8>(a, p, whole, whole_out, st);
    }
  }
  const dim3 grid((uint32_t)((int64_t)p.tg.tiles * a.K * p.splits));
  if (p.wide)
    k_attention_tiles<T, DP, 4, 2, 64><<<grid, 256, 0, st>>>(a, p.tg, p.splits, ws, whole, whole_out);
  else
    k_attention_tiles<T, DP, 1, 1, 32><<<grid, 64, 0, st>>>(a, p.tg, p.splits, ws, whole, whole_out);
  if (p.splits > 1) k_attention_join<T, DP><<<dim3((uint32_t)((int64_t)p.join.tiles * a.K)), 256, 0, st>>>(a, p.join, p.splits, ws);
  return launch_status();
}
template <typename T> int run_type(const Attn& a, const Plan& p, float* ws, hipStream_t st) {
  switch (padded(a.D)) {
    case 16: return run<T, 16>(a, p, ws, st);
    case 32: return run<T, 32>(a, p, ws, st);
    case 64: return run<T, 64>(a, p, ws, st);
    default: return run<T, 128>(a, p, ws, st);
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
