// Rotary positions: pairs of elements of every head of a row turned by position x frequency.  Memory-bound: every element is read
// and written once.  A workgroup takes a few rows (or a part of one) of queries and keys, 1,024 pieces; it asks for all of them
// first, then works out the sines and cosines of its rows, once for all heads, into LDS, and turns the pieces as they come.  131,071 rows
// of 20 heads of 64 elements, half of each turned, float32: 244 us, 5.5 TB/s; 30,000 rows of 16 heads of 16, bfloat16: 7 us, of which a
// launch's two trips to memory are 3.
#include "attention.h"

namespace ff {
namespace {

constexpr int kPieces = 4;             // of a thread, all in flight together
constexpr int kItems = 256 * kPieces;  // of a workgroup
constexpr int kAngles = 2048;          // sines and cosines of a workgroup

struct RotaryPlan {
  int32_t rows;              // of a workgroup
  int32_t per_row, turning;  // items of a row; of a head, those that are turned
  Div row, head;             // items of a row, of a head
};

template <typename T> struct Bits;
template <> struct Bits<float> {
  typedef float type;
  static __device__ __forceinline__ float to(float x) { return x; }
  static __device__ __forceinline__ float from(float x) { return x; }
};
template <> struct Bits<bf16_t> {
  typedef __bf16 type;
  static __device__ __forceinline__ float to(__bf16 x) { return (float)x; }
  static __device__ __forceinline__ __bf16 from(float x) { return (__bf16)x; }
};
template <> struct Bits<f16_t> {
  typedef _Float16 type;
  static __device__ __forceinline__ float to(_Float16 x) { return (float)x; }
  static __device__ __forceinline__ _Float16 from(float x) { return (_Float16)x; }
};

// V elements a piece.  S > 0: the elements of a pair lie S apart in one piece (neighbours, or the halves of axes that are no longer
// than a piece).  S == 0: a piece and its partner, `pairs` elements on, are one item.  LOOSE: rows begin at any element, and what
// passes through goes element by element.
template <typename T, int V, int S, bool LOOSE = false>
__global__ __launch_bounds__(256) void k_rotary(Rotary r, RotaryPlan pl) {
  typedef typename Bits<T>::type el;
  typedef el vec __attribute__((ext_vector_type(V), aligned(LOOSE ? sizeof(el) : sizeof(el) * V)));
  __shared__ __attribute__((aligned(16))) float cs[kAngles], sn[kAngles];
  const int tid = threadIdx.x, turned = r.axes * r.pairs;
  const int64_t row0 = (int64_t)blockIdx.x * pl.rows;
  const int32_t rows = r.n - row0 < pl.rows ? (int32_t)(r.n - row0) : pl.rows;
  const uint32_t items = (uint32_t)rows * pl.per_row, item0 = blockIdx.y * kItems;
  auto axis_of = [&](int j) { return j >= 2 * r.pairs ? 2 : j >= r.pairs ? 1 : 0; };  // (three at most)

  vec a[kPieces], b[kPieces];
  el* to[kPieces];
  int32_t angle[kPieces];  // of the piece's first pair; -1: no item, -2: passes through
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    const uint32_t item = item0 + u * 256 + tid;
    angle[u] = -1;
    if (item >= items) continue;
    const uint32_t row = quotient(item, pl.row), in_row = item - row * pl.row.by, head = quotient(in_row, pl.head);
    const int c = (int)(in_row - head * pl.head.by);
    const bool key = head >= (uint32_t)r.q_heads;
    const int64_t h = key ? head - r.q_heads : head;
    const HeadsAt &from = key ? r.k : r.q, &out = key ? r.k_out : r.q_out;
    int e;
    if (c >= pl.turning) {
      e = 2 * turned + (c - pl.turning) * (LOOSE ? 1 : V);
      angle[u] = -2;
    } else if (S > 0) {
      e = c * V;
      angle[u] = (int32_t)row * turned + c * (V / 2);
    } else {
      e = c * V + axis_of(c * V) * r.pairs;
      angle[u] = (int32_t)row * turned + c * V;
    }
    const el* x = reinterpret_cast<const el*>(from.p) + (row0 + row) * from.rs + h * from.hs + e;
    to[u] = reinterpret_cast<el*>(out.p) + (row0 + row) * out.rs + h * out.hs + e;
    if (LOOSE && angle[u] == -2) {
      a[u][0] = *x;
      continue;
    }
    a[u] = *reinterpret_cast<const vec*>(x);
    if (S == 0 && angle[u] >= 0) b[u] = *reinterpret_cast<const vec*>(x + r.pairs);
  }

  for (int t = tid; t < rows * turned; t += 256) {
    const int row = t / turned, j = t - row * turned;
    double turns = (double)r.pos[(row0 + row) * r.pos_rs + axis_of(j) * r.pos_as] * (r.freqs[j] * 0.15915494309189533577);
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    sn[t] = s * (r.sign * r.amplitude);
    cs[t] = c * r.amplitude;
  }
  __syncthreads();

#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    if (angle[u] == -1) continue;
    if (angle[u] >= 0) {
#pragma unroll
      for (int p = 0; p < (S ? V / 2 : V); ++p) {
        const float c = cs[angle[u] + p], s = sn[angle[u] + p];
        if constexpr (S > 0) {
          const int first = p / S * (2 * S) + p % S, second = first + S;
          const float x = Bits<T>::to(a[u][first]), y = Bits<T>::to(a[u][second]);
          a[u][first] = Bits<T>::from(x * c - y * s);
          a[u][second] = Bits<T>::from(x * s + y * c);
        } else {
          const float x = Bits<T>::to(a[u][p]), y = Bits<T>::to(b[u][p]);
          a[u][p] = Bits<T>::from(x * c - y * s);
          b[u][p] = Bits<T>::from(x * s + y * c);
        }
      }
      if (S == 0) *reinterpret_cast<vec*>(to[u] + r.pairs) = b[u];
    }
    if (LOOSE && angle[u] == -2) *to[u] = a[u][0];
    else                         *reinterpret_cast<vec*>(to[u]) = a[u];
  }
}

template <typename T, int V, int S, bool LOOSE = false> int launch(const Rotary& r, bool copies, hipStream_t stream) {
  const int turned = r.axes * r.pairs, heads = r.q_heads + r.k_heads;
  RotaryPlan pl;
  pl.turning = S ? 2 * turned / V : turned / V;
  const int per_head = pl.turning + (copies ? (r.D - 2 * turned) / (LOOSE ? 1 : V) : 0);
  pl.per_row = per_head * heads;
  const int by_items = kItems / pl.per_row, by_angles = kAngles / turned;
  pl.rows = by_items < 1 ? 1 : by_items < by_angles ? by_items : by_angles;
  pl.row = make_div(pl.per_row);
  pl.head = make_div(per_head);
  if (ceil_div(r.n, pl.rows) > (int64_t)(UINT32_MAX / 256)) return FF_ERR_UNSUPPORTED;  // (a launch's threads are counted in 32 bits)
  const dim3 grid((uint32_t)ceil_div(r.n, pl.rows), (uint32_t)ceil_div((int64_t)pl.rows * pl.per_row, kItems));
  k_rotary<T, V, S, LOOSE><<<grid, 256, 0, stream>>>(r, pl);
  return launch_status();
}

// The widest pieces that addresses, strides, axes and the elements behind them are multiples of
template <typename T> int run(const Rotary& r, hipStream_t stream) {
  constexpr int size = (int)sizeof(T), most = 16 / size;
  const int turned = r.axes * r.pairs, rest = r.D - 2 * turned;
  auto same = [](const HeadsAt& a, const HeadsAt& b) { return a.p == b.p; };
  const bool copies = rest > 0 && !(same(r.q, r.q_out) && (r.k_heads == 0 || same(r.k, r.k_out)));
  uint64_t all = copies ? (uint64_t)rest * size : 0;
  for (const HeadsAt* x : {&r.q, &r.q_out, &r.k, &r.k_out})
    if (x->p) all |= (uintptr_t)x->p | (uint64_t)x->rs * size | (uint64_t)x->hs * size;
  auto fits = [&](int v, int64_t length) { return v <= most && all % (v * size) == 0 && length % v == 0; };
  const int apart = r.layout == FF_ROTARY_INTERLEAVED ? 1 : r.pairs;
  if (apart == 1) {
    if (fits(8, 2 * turned)) { if constexpr (most == 8) return launch<T, 8, 1>(r, copies, stream); }
    if (fits(4, 2 * turned)) return launch<T, 4, 1>(r, copies, stream);
    if (fits(2, 2 * turned)) return launch<T, 2, 1>(r, copies, stream);
  } else if (apart == 2 && fits(4, 2 * turned)) {
    if (fits(8, 2 * turned)) { if constexpr (most == 8) return launch<T, 8, 2>(r, copies, stream); }
    return launch<T, 4, 2>(r, copies, stream);
  } else if (apart == 4 && fits(8, 2 * turned)) {
    if constexpr (most == 8) return launch<T, 8, 4>(r, copies, stream);
  }
  if (r.layout == FF_ROTARY_INTERLEAVED) return launch<T, 2, 1, true>(r, copies, stream);
  if (fits(8, r.pairs)) { if constexpr (most == 8) return launch<T, 8, 0>(r, copies, stream); }
  if (fits(4, r.pairs)) return launch<T, 4, 0>(r, copies, stream);
  if (fits(2, r.pairs)) return launch<T, 2, 0>(r, copies, stream);
  return launch<T, 1, 0>(r, copies, stream);
}

}  // namespace

int rotary_launch(const Rotary& r, int dtype, hipStream_t stream) {
  return dtype == FF_F32 ? run<float>(r, stream) : dtype == FF_BF16 ? run<bf16_t>(r, stream) : run<f16_t>(r, stream);
}

}  // namespace ff
