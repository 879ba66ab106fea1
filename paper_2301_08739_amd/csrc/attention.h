// Attention over the caller's rows (attention_*.hip): what the entry points hand to the launches, and how kernels see rows and lists.
#pragma once
#include "common.h"

namespace ff {

struct Heads {  // head h of row r begins r * rs + h * hs bytes on
  char* p;
  uint32_t rs, hs;  // (so that an address is two multiplications and additions: strides of 4 GiB and more are refused)
};
struct GroupList {
  const int32_t* perm;  // or nullptr: position p is row p
  const int32_t* off;
  int32_t n, G;
  int32_t slots;  // positions that groups can have: n, or the groups times G where that is less (few rows out of many)
};
struct Div {  // quotients of numbers below 2^31 by a constant: a multiplication instead of a division
  uint32_t by, mul, shift;
};
inline Div make_div(uint32_t by) {
  uint32_t s = 0;
  while ((1u << s) < by) ++s;
  return {by, (uint32_t)((((uint64_t)1 << (32 + s)) + by - 1) / by), s};  // less the bit of 2^32, which the addition puts back
}
__device__ __forceinline__ uint32_t quotient(uint32_t x, const Div& d) { return (__umulhi(x, d.mul) + x) >> d.shift; }

struct Attn {
  Heads q, k, v, out, dout, dq, dk, dv;
  float* lse;         // [queries, H] or nullptr
  float2* stats;      // [queries, H], workspace of the backward pass
  int32_t H, K, D;    // query heads, key heads, elements of a head
  Div share;          // query heads of a key head
  float scale;
  const int32_t* num_groups;
  int32_t max_groups;
  GroupList ql, kl;
  const uint8_t* mask;  // or nullptr
};

size_t attention_workspace_bytes(const Attn& a, int dtype);
int attention_launch(const Attn& a, int dtype, void* workspace, hipStream_t stream);
size_t attention_backward_workspace_bytes(const Attn& a, int dtype);
int attention_backward_launch(const Attn& a, int dtype, void* workspace, hipStream_t stream);

struct HeadsAt {  // element e of head h of row r: p[r * rs + h * hs + e]
  void* p;
  int64_t rs, hs;
};
struct Rotary {
  HeadsAt q, q_out, k, k_out;
  int32_t q_heads, k_heads, D;
  int64_t n;
  const int32_t* pos;
  int64_t pos_rs, pos_as;
  const double* freqs;
  int32_t axes, pairs, layout;
  float sign, amplitude;
};
int rotary_launch(const Rotary& r, int dtype, hipStream_t stream);

// ---- on the device -------------------------------------------------------------------------------------
struct Span { int32_t at, len; };
__device__ __forceinline__ int32_t clamp_to(int32_t v, int32_t n) { return v < 0 ? 0 : v < n ? v : n; }
__device__ __forceinline__ int32_t groups_of(const Attn& a) {
  const int32_t listed = a.num_groups ? *a.num_groups : a.max_groups;
  return listed < a.max_groups ? listed : a.max_groups;
}
// Positions of group g; whatever the offsets hold, they lie in 0..n-1.
__device__ __forceinline__ Span span_of(const GroupList& l, int32_t g) {
  const int32_t from = clamp_to(l.off[g], l.n), to = clamp_to(l.off[g + 1], l.n), len = to - from;
  return {from, len < 0 ? 0 : len < l.G ? len : l.G};
}
// Where the sums of a group's first position lie in a workspace that has a place for every position of a list
__device__ __forceinline__ int32_t slot_of(const GroupList& l, int32_t g, const Span& s) { return l.slots < l.n ? g * l.G : s.at; }
// Row at position p, -1 where the list holds none of the rows.
__device__ __forceinline__ int32_t row_at(const GroupList& l, int32_t p) {
  const int32_t r = l.perm ? l.perm[p] : p;
  return (uint32_t)r < (uint32_t)l.n ? r : -1;
}
template <typename T> __device__ __forceinline__ T* row_of_head(const Heads& x, int32_t row, int32_t h) {
  return reinterpret_cast<T*>(x.p + (uint64_t)(uint32_t)h * x.hs + (uint64_t)(uint32_t)row * x.rs);
}

}  // namespace ff
