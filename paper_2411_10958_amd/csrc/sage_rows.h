// Rows of 16-bit tensors with strides of their own, as the operators on queries, keys and values take them (sage_rope.hip, sage_norm_rope.hip,
// sage_cache_append.hip): vectors of a row on the device, strides and overlaps on the host.
#pragma once
#include "sage_ops.h"

#include <algorithm>

namespace sage {

template <int VW> struct Vec;
template <> struct Vec<8> { typedef unsigned type __attribute__((ext_vector_type(4))); };
template <> struct Vec<4> { typedef unsigned type __attribute__((ext_vector_type(2))); };
template <> struct Vec<1> { typedef unsigned short type; };

template <bool BF16, int VW> __device__ __forceinline__ void unpack(const typename Vec<VW>::type& v, float (&f)[VW]) {
  if constexpr (VW == 1) {
    f[0] = load16<BF16>(v);
  } else {
#pragma unroll
    for (int i = 0; i < VW / 2; ++i) {
      f[2 * i] = load16<BF16>((unsigned short)v[i]);
      f[2 * i + 1] = load16<BF16>((unsigned short)(v[i] >> 16));
    }
  }
}
template <bool BF16, int VW> __device__ __forceinline__ typename Vec<VW>::type pack(const float (&f)[VW]) {
  typename Vec<VW>::type v;
  if constexpr (VW == 1) {
    v = (unsigned short)pack16x2<BF16>(f[0], 0.0f);
  } else {
#pragma unroll
    for (int i = 0; i < VW / 2; ++i) v[i] = pack16x2<BF16>(f[2 * i], f[2 * i + 1]);
  }
  return v;
}

// Strides of one tensor, as given or contiguous in `layout`; false if they are not usable.
inline bool tensor_strides(const long long* given, int layout, int heads, int N, int d, long long (&st)[3]) {
  if (given[0] == 0 && given[1] == 0 && given[2] == 0) {
    const TensorMap m = make_tensor_map(layout, heads, N, d);
    st[0] = m.sb; st[1] = m.sh; st[2] = m.sn;
    return true;
  }
  for (int i = 0; i < 3; ++i) {
    if (given[i] < 0) return false;
    st[i] = given[i];
  }
  return true;
}

// Whether no two rows of a tensor share a value: in the order of their strides, each extent steps over all that lies inside it.
// (Rows of an output that did would be written by several threads.)
inline bool rows_apart(const long long (&st)[3], long long B, long long heads, long long N, long long d) {
  const long long extent[3] = {B, heads, N};
  int at[3] = {0, 1, 2};
  std::sort(at, at + 3, [&](int i, int j) { return st[i] < st[j]; });
  long long span = d;
  for (int i : at) {
    if (extent[i] == 1) continue;
    if (st[i] < span) return false;
    span += st[i] * (extent[i] - 1);
  }
  return true;
}

// Whether a row of x and a row of y share a value: whether some  delta + sum of stride times index  lies within d of zero, the indices of y
// counted up and those of x down.  Strides are taken from the largest on; an index is tried where what the smaller ones can add may still
// reach zero - one or two values each for tensors in the usual orders.  (After 65536 tries the answer is no.)
struct Terms {
  int n;
  long long stride[6], lo[6], hi[6], low[7], high[7];      // low, high: the least and the most that terms i .. n - 1 add
  long long d;
  int tries;
};
inline bool reaches(Terms& t, int i, long long at) {
  if (i == t.n) return at > -t.d && at < t.d;
  const long long s = t.stride[i], least = -t.d + 1 - at - t.high[i + 1], most = t.d - 1 - at - t.low[i + 1];
  const long long from = std::max(t.lo[i], least >= 0 ? (least + s - 1) / s : -(-least / s)), to = std::min(t.hi[i], most >= 0 ? most / s : -((-most + s - 1) / s));
  for (long long v = from; v <= to; ++v)
    if (t.tries-- <= 0 || reaches(t, i + 1, at + v * s)) return t.tries > 0;
  return false;
}
inline bool rows_meet(const void* x, const long long (&sx)[3], int hx, const void* y, const long long (&sy)[3], int hy, long long B, long long N, long long d) {
  const long long ex[3] = {B, hx, N}, ey[3] = {B, hy, N};
  long long span_x = d, span_y = d;                // values from the first to the last
  for (int i = 0; i < 3; ++i) { span_x += sx[i] * (ex[i] - 1); span_y += sy[i] * (ey[i] - 1); }
  const long long delta = ((long long)(uintptr_t)y - (long long)(uintptr_t)x) / 2;
  if (delta >= span_x || -delta >= span_y) return false;
  Terms t;
  t.n = 0; t.d = d; t.tries = 65536;
  auto add = [&](long long s, long long lo, long long hi) {
    if (s == 0) return;
    int i = 0;
    while (i < t.n && t.stride[i] > s) ++i;
    if (i == t.n || t.stride[i] != s) {
      for (int j = t.n++; j > i; --j) { t.stride[j] = t.stride[j - 1]; t.lo[j] = t.lo[j - 1]; t.hi[j] = t.hi[j - 1]; }
      t.stride[i] = s; t.lo[i] = t.hi[i] = 0;
    }
    t.lo[i] += lo; t.hi[i] += hi;
  };
  for (int i = 0; i < 3; ++i) { add(sx[i], 1 - ex[i], 0); add(sy[i], 0, ey[i] - 1); }
  t.low[t.n] = t.high[t.n] = 0;
  for (int i = t.n - 1; i >= 0; --i) { t.low[i] = t.low[i + 1] + t.stride[i] * t.lo[i]; t.high[i] = t.high[i + 1] + t.stride[i] * t.hi[i]; }
  return reaches(t, 0, delta);
}

}  // namespace sage
