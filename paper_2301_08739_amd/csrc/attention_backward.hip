// The gradient of attention over the caller's rows: plain kernels.  A wavefront takes one query (or one key) of one head and
// goes through the rows of the other side 64 at a time: a lane a row for the scores, a lane two elements for the sums.  Right for
// every shape; bound by instruction issue and by rows that every wavefront reads again.
#include "attention.h"

namespace ff {
namespace {

// p and e of one (query, key) pair of rows
template <typename T>
__device__ __forceinline__ void pair_terms(const Attn& a, int32_t rq, int32_t rk, int h, int kh, float* p, float* e) {
  const T *q = row_of_head<T>(a.q, rq, h), *g = row_of_head<T>(a.dout, rq, h), *o = row_of_head<T>(a.out, rq, h);
  const T *k = row_of_head<T>(a.k, rk, kh), *v = row_of_head<T>(a.v, rk, kh);
  float s = 0.f, dp = 0.f, delta = 0.f;
  for (int i = 0; i < a.D; ++i) {
    const float gi = Elem<T>::load(g + i);
    s = fmaf(Elem<T>::load(q + i), Elem<T>::load(k + i), s);
    dp = fmaf(gi, Elem<T>::load(v + i), dp);
    delta = fmaf(gi, Elem<T>::load(o + i), delta);
  }
  *p = expf(a.scale * s - a.lse[(int64_t)rq * a.H + h]);
  *e = *p * (dp - delta) * a.scale;
}

template <typename T> __global__ __launch_bounds__(64) void k_attention_dq_plain(Attn a) {
  __shared__ float es[64];
  __shared__ int32_t rows[64];
  const int lane = threadIdx.x, h = blockIdx.y, kh = h / (a.H / a.K);
  const int g = blockIdx.x / a.ql.G, i = blockIdx.x % a.ql.G;
  if (g >= groups_of(a)) return;
  const Span sq = span_of(a.ql, g), sk = span_of(a.kl, g);
  if (i >= sq.len) return;
  const int32_t row = row_at(a.ql, sq.at + i);
  if (row < 0) return;
  float d0 = 0.f, d1 = 0.f;
  for (int j0 = 0; j0 < sk.len; j0 += 64) {
    const int32_t r = j0 + lane < sk.len ? row_at(a.kl, sk.at + j0 + lane) : -1;
    const bool ok = r >= 0 && (!a.mask || a.mask[r]);
    float p = 0.f, e = 0.f;
    if (ok) pair_terms<T>(a, row, r, h, kh, &p, &e);
    es[lane] = e;
    rows[lane] = ok ? r : -1;
    __syncthreads();
    for (int j = 0; j < 64; ++j) {
      if (rows[j] < 0) continue;
      const T* k = row_of_head<T>(a.k, rows[j], kh);
      if (lane < a.D) d0 = fmaf(es[j], Elem<T>::load(k + lane), d0);
      if (lane + 64 < a.D) d1 = fmaf(es[j], Elem<T>::load(k + lane + 64), d1);
    }
    __syncthreads();
  }
  T* dq = row_of_head<T>(a.dq, row, h);
  if (lane < a.D) Elem<T>::store(dq + lane, d0);
  if (lane + 64 < a.D) Elem<T>::store(dq + lane + 64, d1);
}

template <typename T> __global__ __launch_bounds__(64) void k_attention_dkv_plain(Attn a) {
  __shared__ float es[64], ps[64];
  __shared__ int32_t rows[64];
  const int lane = threadIdx.x, kh = blockIdx.y, share = a.H / a.K;
  const int g = blockIdx.x / a.kl.G, i = blockIdx.x % a.kl.G;
  if (g >= groups_of(a)) return;
  const Span sq = span_of(a.ql, g), sk = span_of(a.kl, g);
  if (i >= sk.len) return;
  const int32_t row = row_at(a.kl, sk.at + i);
  if (row < 0) return;
  const bool ok = !a.mask || a.mask[row];
  float k0 = 0.f, k1 = 0.f, v0 = 0.f, v1 = 0.f;
  for (int h = kh * share; ok && h < (kh + 1) * share; ++h)
    for (int j0 = 0; j0 < sq.len; j0 += 64) {
      const int32_t r = j0 + lane < sq.len ? row_at(a.ql, sq.at + j0 + lane) : -1;
      float p = 0.f, e = 0.f;
      if (r >= 0) pair_terms<T>(a, r, row, h, kh, &p, &e);
      es[lane] = e;
      ps[lane] = p;
      rows[lane] = r;
      __syncthreads();
      for (int j = 0; j < 64; ++j) {
        if (rows[j] < 0) continue;
        const T *q = row_of_head<T>(a.q, rows[j], h), *go = row_of_head<T>(a.dout, rows[j], h);
        if (lane < a.D) {
          k0 = fmaf(es[j], Elem<T>::load(q + lane), k0);
          v0 = fmaf(ps[j], Elem<T>::load(go + lane), v0);
        }
        if (lane + 64 < a.D) {
          k1 = fmaf(es[j], Elem<T>::load(q + lane + 64), k1);
          v1 = fmaf(ps[j], Elem<T>::load(go + lane + 64), v1);
        }
      }
      __syncthreads();
    }
  T *dk = row_of_head<T>(a.dk, row, kh), *dv = row_of_head<T>(a.dv, row, kh);
  if (lane < a.D) {
    Elem<T>::store(dk + lane, k0);
    Elem<T>::store(dv + lane, v0);
  }
  if (lane + 64 < a.D) {
    Elem<T>::store(dk + lane + 64, k1);
    Elem<T>::store(dv + lane + 64, v1);
  }
}

template <typename T> int backward(const Attn& a, hipStream_t stream) {
  const int64_t sq = (int64_t)a.max_groups * a.ql.G, sk = (int64_t)a.max_groups * a.kl.G;
  if (sq > INT32_MAX || sk > INT32_MAX || a.H > 65535) return FF_ERR_UNSUPPORTED;
  k_attention_dq_plain<T><<<dim3((uint32_t)sq, a.H), 64, 0, stream>>>(a);
  k_attention_dkv_plain<T><<<dim3((uint32_t)sk, a.K), 64, 0, stream>>>(a);
  return launch_status();
}

}  // namespace

size_t attention_backward_workspace_bytes(const Attn&, int) { return 0; }
int attention_backward_launch(const Attn& a, int dtype, void*, hipStream_t stream) {
  return dtype == FF_F32 ? backward<float>(a, stream) : dtype == FF_BF16 ? backward<bf16_t>(a, stream) : backward<f16_t>(a, stream);
}

}  // namespace ff
