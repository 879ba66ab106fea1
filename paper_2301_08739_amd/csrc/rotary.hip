// Rotary positions: pairs of elements of every head of a row turned by position x frequency.
#include "attention.h"

namespace ff {
namespace {

// One thread a pair of a head, or an element that passes through.
template <typename T> __global__ __launch_bounds__(256) void k_rotary(Rotary r) {
  const int turned = r.axes * r.pairs, rest = r.D - 2 * turned, items = turned + rest, heads = r.q_heads + r.k_heads;
  const int64_t total = r.n * heads * items;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int item = (int)(i % items), head = (int)(i / items % heads);
    const int64_t row = i / items / heads;
    const bool key = head >= r.q_heads;
    const Heads &from = key ? r.k : r.q, &to = key ? r.k_out : r.q_out;
    const int h = key ? head - r.q_heads : head;
    const T* x = reinterpret_cast<const T*>(from.p) + row * from.rs + h * from.hs;
    T* y = reinterpret_cast<T*>(to.p) + row * to.rs + h * to.hs;
    if (item >= turned) {
      y[turned + item] = x[turned + item];
      continue;
    }
    const int axis = item / r.pairs, j = item - axis * r.pairs, base = axis * 2 * r.pairs;
    const int ia = base + (r.layout == FF_ROTARY_HALF ? j : 2 * j), ib = r.layout == FF_ROTARY_HALF ? ia + r.pairs : ia + 1;
    double turns = (double)r.pos[row * r.pos_rs + axis * r.pos_as] * (r.freqs[item] * 0.15915494309189533577);
    turns -= rint(turns);
    float sn, cs;
    sincospif(2.f * (float)turns, &sn, &cs);
    sn *= r.sign * r.amplitude;
    cs *= r.amplitude;
    const float u = Elem<T>::load(x + ia), v = Elem<T>::load(x + ib);
    Elem<T>::store(y + ia, u * cs - v * sn);
    Elem<T>::store(y + ib, u * sn + v * cs);
  }
}

template <typename T> int launch(const Rotary& r, hipStream_t stream) {
  const int64_t total = r.n * (r.q_heads + r.k_heads) * (r.D - r.axes * r.pairs);
  const int64_t groups = ceil_div(total, 256);
  k_rotary<T><<<dim3((uint32_t)(groups < 65536 ? groups : 65536)), 256, 0, stream>>>(r);
  return launch_status();
}

}  // namespace

int rotary_launch(const Rotary& r, int dtype, hipStream_t stream) {
  return dtype == FF_F32 ? launch<float>(r, stream) : dtype == FF_BF16 ? launch<bf16_t>(r, stream) : launch<f16_t>(r, stream);
}

}  // namespace ff
