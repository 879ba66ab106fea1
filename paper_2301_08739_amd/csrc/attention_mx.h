// Matrix-core pieces of the attention kernels, alike for bfloat16, half and float32.
//
// Every product is made of 16 x 16 tiles.  An operand piece holds 16 bytes a lane: lane (g, i) = (lane / 16, lane % 16) has, of row i
// of the operand (a column of the right one), the KF / 4 elements from k = g * KF / 4 on; KF is 32 for 16-bit types (one instruction)
// and 16 for float32 (four, one an element: the order of k is another one on both sides alike).  A result tile holds rows 4 g .. 4 g + 3
// of column i.  So where a product's result is next summed over its rows, it becomes the right operand of the next product as it
// lies in the registers: a piece of KF rows is KF / 16 tiles one after the other, and the left operand is read in that order of k,
// from LDS, down its columns (16 bits: the transposing read; float32: element by element).
#pragma once
#include "attention.h"

namespace ff {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr float kLowest = -3.402823466e38f;

union Piece {  // 16 bytes of an operand
  u32x4 q;
  f32x4 f;
  b16x8 b;
  h16x8 h;
  s16x4 s[2];
  b16x4 b4[2];
  h16x4 h4[2];
};

template <typename T> struct Mx {
  static constexpr int KF = 32, E = 8, TILES = 2;
};
template <> struct Mx<float> {
  static constexpr int KF = 16, E = 4, TILES = 1;
};

template <typename T> __device__ __forceinline__ f32x4 mma(const Piece& a, const Piece& b, f32x4 c);
template <> __device__ __forceinline__ f32x4 mma<bf16_t>(const Piece& a, const Piece& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 mma<f16_t>(const Piece& a, const Piece& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.h, c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 mma<float>(const Piece& a, const Piece& b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.f[j], b.f[j], c, 0, 0, 0);
  return c;
}

// TILES result tiles as the right operand of the next product, rounded to the type (to nearest even)
template <typename T> __device__ __forceinline__ Piece as_piece(const f32x4* t);
template <> __device__ __forceinline__ Piece as_piece<bf16_t>(const f32x4* t) {
  Piece p;
  p.b4[0] = __builtin_convertvector(t[0], b16x4);
  p.b4[1] = __builtin_convertvector(t[1], b16x4);
  return p;
}
template <> __device__ __forceinline__ Piece as_piece<f16_t>(const f32x4* t) {
  Piece p;
  p.h4[0] = __builtin_convertvector(t[0], h16x4);
  p.h4[1] = __builtin_convertvector(t[1], h16x4);
  return p;
}
template <> __device__ __forceinline__ Piece as_piece<float>(const f32x4* t) {
  Piece p;
  p.f = t[0];
  return p;
}

// The same for one result tile of sixteen rows, where that is all a product sums over (16 bits: half a piece, s[0])
template <typename T> __device__ __forceinline__ Piece as_half(f32x4 t) {
  const f32x4 both[2] = {t, t};
  return as_piece<T>(both);
}
template <typename T> __device__ __forceinline__ f32x4 mma_half(const Piece& a, const Piece& b, f32x4 c);
template <> __device__ __forceinline__ f32x4 mma_half<bf16_t>(const Piece& a, const Piece& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a.s[0], b.s[0], c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 mma_half<f16_t>(const Piece& a, const Piece& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x16f16(a.h4[0], b.h4[0], c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 mma_half<float>(const Piece& a, const Piece& b, f32x4 c) { return mma<float>(a, b, c); }

// Four elements side by side (one lane's part of a result tile) into memory, those from D on left out
template <typename T, bool WHOLE> __device__ __forceinline__ void store4(T* row, int e, f32x4 v, int D) {
  if constexpr (WHOLE) {
    if (e >= D) return;
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4*>(row + e) = v;
    } else {
      const f32x4 t[2] = {v, v};
      const Piece p = as_piece<T>(t);
      *reinterpret_cast<s16x4*>(row + e) = p.s[0];
    }
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (e + r < D) Elem<T>::store(row + e + r, v[r]);
  }
}

__device__ int32_t zero_number = 0;
__device__ u32x4 zero_piece = {0u, 0u, 0u, 0u};  // (never written; a constant would be of another address space, and the loads flat)

// 16 bytes of row `row` (negative: none) and head h from element e on, zero from D on.  WHOLE: rows are pieces of 16 bytes, from their
// addresses to their ends; what is not there is then read from a piece of zeros, so that a wavefront asks for all its pieces at once.
template <typename T, bool WHOLE> __device__ __forceinline__ Piece load_piece(const Heads& x, int32_t row, int32_t h, int e, int D) {
  Piece p;
  const T* at = row_of_head<const T>(x, row, h) + e;
  if constexpr (WHOLE) {
    p.q = *(row >= 0 && e < D ? reinterpret_cast<const u32x4*>(at) : &zero_piece);
  } else {
    p.q = u32x4{0u, 0u, 0u, 0u};
    if (row < 0) return p;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (e + j < D) p.f[j] = at[j];
    } else {
      const uint16_t* x16 = reinterpret_cast<const uint16_t*>(at);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (e + j < D) p.q[j / 2] |= (uint32_t)x16[j] << (16 * (j % 2));
    }
  }
  return p;
}

// The piece down column d0 + i of an LDS tile: rows r0 + 16 t + 4 g + j for tiles t < TILES, in the order of as_piece
template <typename T> __device__ __forceinline__ Piece column_piece(const T* tile, int ld, int r0, int d0, int lane) {
  Piece p;
  const int g = lane >> 4, i = lane & 15;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) p.f[j] = tile[(r0 + 4 * g + j) * ld + d0 + i];
  } else {
    // sixteen lanes read four rows of sixteen elements, 8 bytes a lane, and get a column of four each
    const T* at = tile + (r0 + 4 * g + (i >> 2)) * ld + d0 + (i & 3) * 4;
    p.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
    p.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * ld));
  }
  return p;
}
// and the half of it for sixteen rows
template <typename T> __device__ __forceinline__ Piece column_half(const T* tile, int ld, int r0, int d0, int lane) {
  if constexpr (sizeof(T) == 4) {
    return column_piece(tile, ld, r0, d0, lane);
  } else {
    Piece p;
    const int g = lane >> 4, i = lane & 15;
    p.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + (r0 + 4 * g + (i >> 2)) * ld + d0 + (i & 3) * 4));
    return p;
  }
}
template <typename T> __device__ __forceinline__ Piece row_piece(const T* tile, int ld, int r, int e) {
  Piece p;
  p.q = *reinterpret_cast<const u32x4*>(tile + r * ld + e);
  return p;
}

// What lanes of a wavefront wrote into LDS is there for its other lanes
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename T> __device__ __forceinline__ Piece negated(Piece p) {
  const uint32_t sign = sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
  p.q ^= u32x4{sign, sign, sign, sign};
  return p;
}
__device__ __forceinline__ f32x4 all4(float v) { return f32x4{v, v, v, v}; }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float over_lanes16_max(float v) {  // over the four lanes of a column
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float over_lanes16_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Scores as they come from the products, as the exponents of p grow with them: c > 0, and the queries (or keys) negated where the
// scale is negative; a scale of zero, or smaller than any score makes up for, as next to nothing.
__device__ __forceinline__ float score_scale(const Attn& a) { return fmaxf(fabsf(a.scale), 1e-30f); }
__device__ __forceinline__ float exponent_factor(const Attn& a) { return score_scale(a) * kLog2e; }

// A launch's arguments lie in a few lines of memory that no cache holds yet; asked for one by one, as they are first used, each is a
// trip.  So one word of every line is asked for at the start, all together.
__device__ __forceinline__ void touch_arguments(const Attn& a) {
  asm volatile("" ::"s"(a.q.p), "s"(a.v.p), "s"(a.dout.p), "s"(a.dk.p), "s"(a.lse), "s"(a.num_groups), "s"(a.kl.perm), "s"(a.mask));
}

// ---- which tile of which group ---------------------------------------------------------------------------
// Tiles of B rows (positions times `share` heads that have their keys in common).  Groups of about the same length: tile t is tile
// t % per_group of group t / per_group.  Else, so that long lists of mostly short groups launch few empty workgroups: group g owns
// tiles floor(offsets[g] * share / B) + g and on, which is at least as many as it has, whatever the lengths, and a wavefront finds
// the group of a tile in two or three looks at 64 offsets.
struct TileGrid {
  int32_t tiles, share;
  Div per_group;  // by 0: by offsets
};
struct TileAt {
  int32_t g, tile;  // g < 0: none
};
template <int B> __device__ __forceinline__ TileAt tile_at(const Attn& a, const GroupList& l, const TileGrid& tg, int32_t t, int lane) {
  const int32_t ng = groups_of(a);
  if (ng <= 0) return {-1, 0};
  if (tg.per_group.by) {
    const int32_t g = quotient(t, tg.per_group);
    return {g < ng ? g : -1, t - g * (int32_t)tg.per_group.by};
  }
  auto base = [&](int32_t g) { return (int32_t)((int64_t)clamp_to(l.off[g], l.n) * tg.share / B) + g; };
  int32_t lo = 0, hi = ng;
  while (hi - lo > 1) {
    const int32_t step = (hi - lo + 63) / 64, g = lo + lane * step;
    const int below = __popcll(__ballot(g < hi && base(g) <= t));
    lo += (below > 0 ? below - 1 : 0) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  const int32_t first = base(lo);
  return {first <= t ? lo : -1, t - first};
}
inline TileGrid tile_grid(int64_t n, int64_t G, int64_t share, int64_t max_groups, int64_t B, bool* fits) {
  const int64_t per = ceil_div(G * share, B), even = per * max_groups, by_offsets = n * share / B + max_groups + 1;
  const bool direct = even <= by_offsets + by_offsets / 2;
  const int64_t tiles = direct ? even : by_offsets;
  *fits = tiles <= INT32_MAX;
  return {(int32_t)(*fits ? tiles : 0), (int32_t)share, direct && *fits && per > 0 ? make_div((uint32_t)per) : Div{0, 0, 0}};
}

// Workgroups go to the eight XCDs in turn, each with an L2 of its own.  Tiles that read the same rows are neighbours in the order of
// the work; runs of `run` of them are given to one XCD, as long as that leaves the XCDs evenly filled.
struct Order {
  uint32_t total, run;  // workgroups that have work, and of a run
};
__device__ __forceinline__ uint32_t in_order(const Order& o) {
  const uint32_t xcd = blockIdx.x % 8, j = blockIdx.x / 8;
  return (j / o.run * 8 + xcd) * o.run + j % o.run;
}
inline Order make_order(int64_t total) {
  uint32_t run = 16;
  while (run > 1 && (total + 8 * run - 1) / (8 * run) * (8 * run) - total > total / 16) run /= 2;
  return {(uint32_t)total, run};
}
// A launch's threads are counted in 32 bits.
inline bool one_launch(int64_t workgroups, int threads) { return workgroups <= (int64_t)(UINT32_MAX / threads); }
inline bool one_launch_in_order(int64_t total, int threads) { return one_launch(total + total / 16 + 128, threads); }
inline uint32_t workgroups(const Order& o) { return (o.total + 8 * o.run - 1) / (8 * o.run) * (8 * o.run); }

// ---- a tile of rows into LDS ------------------------------------------------------------------------------
template <typename T, int DP, int R, int NT> struct Rows {
  static constexpr int PER = DP * (int)sizeof(T) / 16;              // pieces of a row
  static constexpr int U = (R * PER + NT - 1) / NT;                 // pieces of a thread
  static constexpr int STEP = NT / PER;                             // rows between two pieces of a thread
  static __device__ __forceinline__ int row(int tid, int u) { return tid / PER + u * STEP; }
  template <bool WHOLE>
  static __device__ __forceinline__ void fetch(Piece (&r)[U], const Heads& x, const int32_t (&rows)[U], const int32_t (&heads)[U], int tid, int D) {
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = load_piece<T, WHOLE>(x, rows[u], heads[u], (tid % PER) * Mx<T>::E, D);
  }
  static __device__ __forceinline__ void put(T* tile, int ld, const Piece (&r)[U], int tid) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (R * PER % NT == 0 || row(tid, u) < R) *reinterpret_cast<u32x4*>(tile + row(tid, u) * ld + (tid % PER) * Mx<T>::E) = r[u].q;
  }
};

// Tiles of BK keys and values on their way into LDS: numbers of rows two tiles ahead, pieces one.  Nothing here waits for what it has
// just asked for: a row's number is looked at when its piece is asked for, its mask when the piece is put down.
template <typename T, int DP, int BK, int NT> struct KeyTiles {
  typedef Rows<T, DP, BK, NT> R;
  int32_t number[R::U], heads[R::U];
  Piece k[R::U], v[R::U];
  uint32_t there;      // bit u: piece u is of a row
  uint8_t seen[R::U];  // and of one that the mask leaves

  // Tile t's numbers; end: one behind the last tile there is.  Positions behind the group's end are read as its last.
  __device__ __forceinline__ void next(const Attn& a, const Span& sk, int32_t t, int32_t end, int tid) {
    if (t >= end) return;
    const int32_t* const list = a.kl.perm ? a.kl.perm : &zero_number;
#pragma unroll
    for (int u = 0; u < R::U; ++u) {
      const int32_t p = t * BK + R::row(tid, u);
      number[u] = list[a.kl.perm ? sk.at + (p < sk.len ? p : sk.len - 1) : 0];
    }
  }
  template <bool WHOLE> __device__ __forceinline__ void fetch(const Attn& a, const Span& sk, int32_t t, int kh, int tid) {
    there = 0;
#pragma unroll
    for (int u = 0; u < R::U; ++u) {
      const int r = R::row(tid, u);
      const int32_t p = t * BK + r;
      heads[u] = kh;
      if (!a.kl.perm) number[u] = sk.at + p;
      if ((uint32_t)number[u] >= (uint32_t)a.kl.n || p >= sk.len || (BK * R::PER % NT != 0 && r >= BK)) number[u] = -1;
      there |= number[u] >= 0 ? 1u << u : 0u;
    }
    R::template fetch<WHOLE>(k, a.k, number, heads, tid, a.D);
    R::template fetch<WHOLE>(v, a.v, number, heads, tid, a.D);
    if (a.mask) {
#pragma unroll
      for (int u = 0; u < R::U; ++u) seen[u] = a.mask[number[u] < 0 ? 0 : number[u]];
    }
  }
  __device__ __forceinline__ void put(const Attn& a, T* ks, int ldk, T* vs, int ldv, float* bias, int tid) {
    if (a.mask) {
#pragma unroll
      for (int u = 0; u < R::U; ++u)
        if (!seen[u]) {
          there &= ~(1u << u);
          k[u].q = v[u].q = u32x4{0u, 0u, 0u, 0u};
        }
    }
    R::put(ks, ldk, k, tid);
    R::put(vs, ldv, v, tid);
    if (tid % R::PER == 0) {
#pragma unroll
      for (int u = 0; u < R::U; ++u)
        if (BK * R::PER % NT == 0 || R::row(tid, u) < BK) bias[R::row(tid, u)] = there >> u & 1 ? 0.f : -INFINITY;
    }
  }
};

// A row of queries among those of a group that share their keys: row v is position v / share, head v % share of the key head's
struct QueryRow {
  int32_t row, h;  // row < 0: none
};
__device__ __forceinline__ QueryRow query_row(const Attn& a, const Span& sq, int kh, int32_t v) {
  const int32_t p = quotient(v, a.share), h = kh * a.share.by + v - p * a.share.by;
  return {p < sq.len ? row_at(a.ql, sq.at + p) : -1, h};
}
__device__ __forceinline__ uint64_t stat_at(const Attn& a, int32_t row, int32_t h) { return (uint64_t)(uint32_t)row * (uint32_t)a.H + (uint32_t)h; }

// ---- rows of several heads into LDS ----------------------------------------------------------------------
// Short groups: HW wavefronts take a group, a key head each.  Their heads lie side by side in a row, so the workgroup reads and writes
// whole rows of them, a 16-byte piece a thread, and LDS is where they are dealt out to the wavefronts' own tiles (and gathered from
// them).  A wavefront by itself would touch as many lines of memory for 32 bytes of each, head after head: the address unit was busy 78 %
// of the time with that, and 3,750 groups of 64 rows, 8 heads of 16 took 65 us.
template <typename T, int DP, int HW, int RMAX> struct HeadRows {
  static constexpr int PER = DP * (int)sizeof(T) / 16, NT = 64 * HW, STEP = 64 / PER;  // STEP: rows between two pieces of a thread
  static constexpr int U = (RMAX * PER + 63) / 64;                                     // pieces of a thread
};
template <typename T, bool WHOLE> __device__ __forceinline__ void store_piece(const Heads& x, int32_t row, int32_t h, int e, int D, const Piece& p) {
  T* to = row_of_head<T>(x, row, h) + e;
  if constexpr (WHOLE) {
    if (e < D) *reinterpret_cast<u32x4*>(to) = p.q;
  } else {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (e + j < D) to[j] = p.f[j];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (e + j < D) reinterpret_cast<uint16_t*>(to)[j] = (uint16_t)(p.q[j / 2] >> (16 * (j % 2)));
    }
  }
}
// The keys of a group, R rows at most: this thread's pieces are of head `head` (of HW), element c * E on, and rows first + u * STEP.
template <typename T, int DP, int HW, int R> struct KeyPieces {
  typedef HeadRows<T, DP, HW, R> H;
  int head, c, first;
  int32_t row[H::U];  // -1: none
  uint32_t live;      // bit u: one that queries look at
  __device__ __forceinline__ void place(int tid) {
    c = tid % H::PER;
    head = tid / H::PER % HW;
    first = tid / (H::PER * HW);
  }
  __device__ __forceinline__ void ask(const Attn& a, const Span& sk) {
    const int32_t* const list = a.kl.perm ? a.kl.perm : &zero_number;
    const bool some = sk.len > 0;
#pragma unroll
    for (int u = 0; u < H::U; ++u) {
      const int32_t p = first + u * H::STEP;
      row[u] = list[a.kl.perm && some ? sk.at + (p < sk.len ? p : sk.len - 1) : 0];
    }
  }
  __device__ __forceinline__ void look(const Attn& a, const Span& sk) {
    live = 0;
#pragma unroll
    for (int u = 0; u < H::U; ++u) {
      const int32_t p = first + u * H::STEP;
      if (!a.kl.perm) row[u] = sk.at + p;
      if (p >= sk.len || p >= R || (uint32_t)row[u] >= (uint32_t)a.kl.n) row[u] = -1;
      live |= row[u] >= 0 ? 1u << u : 0u;
    }
    if (a.mask) {
      uint8_t seen[H::U];
#pragma unroll
      for (int u = 0; u < H::U; ++u) seen[u] = a.mask[row[u] < 0 ? 0 : row[u]];
#pragma unroll
      for (int u = 0; u < H::U; ++u)
        if (!seen[u]) live &= ~(1u << u);
    }
  }
  template <bool WHOLE> __device__ __forceinline__ void fetch(Piece (&x)[H::U], const Heads& from, int32_t kh0, int D) const {
#pragma unroll
    for (int u = 0; u < H::U; ++u) x[u] = load_piece<T, WHOLE>(from, live >> u & 1 ? row[u] : -1, kh0 + head, c * Mx<T>::E, D);
  }
  // tiles: `pitch` elements from one head's to the next
  __device__ __forceinline__ void put(T* tiles, int pitch, int ld, const Piece (&x)[H::U]) const {
#pragma unroll
    for (int u = 0; u < H::U; ++u)
      if (R * H::PER % 64 == 0 || first + u * H::STEP < R) *reinterpret_cast<u32x4*>(tiles + head * pitch + (first + u * H::STEP) * ld + c * Mx<T>::E) = x[u].q;
  }
  template <bool WHOLE> __device__ __forceinline__ void store(const Heads& to, int32_t kh0, int D, const T* tiles, int pitch, int ld) const {
#pragma unroll
    for (int u = 0; u < H::U; ++u) {
      if (row[u] < 0) continue;
      Piece p;
      p.q = *reinterpret_cast<const u32x4*>(tiles + head * pitch + (first + u * H::STEP) * ld + c * Mx<T>::E);
      store_piece<T, WHOLE>(to, row[u], kh0 + head, c * Mx<T>::E, D, p);
    }
  }
};
// Queries by CH rows of each key head (CH / share positions times the heads that share it): piece u of a thread is of row v[u] of key
// head w[u]'s tile.
template <typename T, int DP, int HW, int CH> struct QueryPieces {
  typedef HeadRows<T, DP, HW, CH> H;
  int c;
  int32_t raw[H::U], row[H::U], h[H::U];
  int v[H::U], w[H::U];  // v >= CH: none
  // In the order in which rows and heads lie in memory.  Where `share` does not divide CH, every tile ends in rows that no position has;
  // the pieces that are left clear them (their position is behind the chunk's end), as sums over a tile's rows run over them too.
  __device__ __forceinline__ void place(const Attn& a, int tid) {
    c = tid % H::PER;
    const int used = quotient(CH, a.share) * a.share.by, over = CH - used;
#pragma unroll
    for (int u = 0; u < H::U; ++u) {
      const int t = tid / H::PER + u * (H::NT / H::PER), s = quotient(t, a.share), p = s / HW;
      w[u] = s % HW;
      h[u] = w[u] * a.share.by + t - s * a.share.by;
      v[u] = p * a.share.by + t - s * a.share.by;
      if (t >= used * HW) {
        const int left = t - used * HW;
        w[u] = h[u] = left < over * HW ? left / over : 0;
        v[u] = left < over * HW ? used + left % over : CH;
      }
    }
  }
  __device__ __forceinline__ int position(const Attn& a, int u) const { return quotient(v[u], a.share); }
  __device__ __forceinline__ void ask(const Attn& a, const Span& sq, int32_t p0) {
    const int32_t* const list = a.ql.perm ? a.ql.perm : &zero_number;
#pragma unroll
    for (int u = 0; u < H::U; ++u) {
      const int32_t p = p0 + position(a, u);
      raw[u] = list[a.ql.perm ? sq.at + (p < sq.len ? p : sq.len - 1) : 0];
    }
  }
  // end: one behind the last position of the chunk
  __device__ __forceinline__ void look(const Attn& a, const Span& sq, int32_t p0, int32_t end) {
#pragma unroll
    for (int u = 0; u < H::U; ++u) {
      const int32_t p = p0 + position(a, u), r = a.ql.perm ? raw[u] : sq.at + p;
      row[u] = p < end && (uint32_t)r < (uint32_t)a.ql.n ? r : -1;
    }
  }
  template <bool WHOLE> __device__ __forceinline__ void fetch(Piece (&x)[H::U], const Heads& from, int32_t h0, int D) const {
#pragma unroll
    for (int u = 0; u < H::U; ++u) x[u] = load_piece<T, WHOLE>(from, row[u], h0 + h[u], c * Mx<T>::E, D);
  }
  __device__ __forceinline__ void put(T* tiles, int pitch, int ld, const Piece (&x)[H::U]) const {
#pragma unroll
    for (int u = 0; u < H::U; ++u)
      if (v[u] < CH) *reinterpret_cast<u32x4*>(tiles + w[u] * pitch + v[u] * ld + c * Mx<T>::E) = x[u].q;
  }
  template <bool WHOLE> __device__ __forceinline__ void store(const Heads& to, int32_t h0, int D, const T* tiles, int pitch, int ld) const {
#pragma unroll
    for (int u = 0; u < H::U; ++u) {
      if (row[u] < 0 || v[u] >= CH) continue;
      Piece p;
      p.q = *reinterpret_cast<const u32x4*>(tiles + w[u] * pitch + v[u] * ld + c * Mx<T>::E);
      store_piece<T, WHOLE>(to, row[u], h0 + h[u], c * Mx<T>::E, D, p);
    }
  }
};
// Which of a launch's workgroups this is: sets of heads, then parts of a group's queries, then groups
struct Items {
  uint32_t total;
  Div sets, parts;
};
inline Items make_items(int64_t groups, int sets, int parts) { return {(uint32_t)(groups * sets * parts), make_div(sets), make_div(parts)}; }
inline int heads_together(int K) { return K % 4 == 0 ? 4 : K % 2 == 0 ? 2 : 1; }

// May rows of this array be read and written in pieces of 16 bytes?
inline bool whole_pieces(const Heads& x, int D, size_t size) {
  return ((uintptr_t)x.p | (uintptr_t)x.rs | (uintptr_t)x.hs | (uintptr_t)(D * size)) % 16 == 0;
}

constexpr int kChipWaves = 2048;  // two wavefronts a SIMD

inline int padded(int D) { return D <= 16 ? 16 : D <= 32 ? 32 : D <= 64 ? 64 : 128; }

}  // namespace
}  // namespace ff
