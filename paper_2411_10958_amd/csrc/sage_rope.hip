// Rotary positions of queries and keys (sage_rope) and their frequencies (sage_rope_frequencies).
//
// Channel pair i of the first `rot` channels is turned by the angle p f_i: (a, b) -> scale (a cos - b sin, b cos + a sin), the
// pair being channels (i, i + rot/2) or (2i, 2i + 1).  Nothing but bytes moves this: every value is read and written once, 4 bytes
// (4 x 4096 tokens of 40 heads of 128: 57 to 60 us, 5.6 to 5.9 TB/s; a copy of 2 GB 5.0).
// A thread owns one vector of VW channels of a token, or two, a pair's channels in each, works their angles out once and then walks over
// heads, so the FP64 product and the sine and cosine are shared by all of them.  Angles are taken in 64 bits (position 10^6 times the fastest
// frequency in FP32 would be off by 0.03 rad), reduced to a fraction of a turn there, and their sine and cosine in FP32.
#include "sage_attn.h"
#include "sage_ops.h"

#include <algorithm>
#include <cmath>

namespace sage {
namespace {

struct RopeTensor {
  const unsigned short* x;
  unsigned short* y;
  long long xb, xh, xn, yb, yh, yn;      // strides of batch, head and token, in elements
  int heads;
};
struct RopeParams {
  RopeTensor q, k;                       // k.heads = 0 without keys
  const double* inv_freq;
  const int* positions;                  // null: the token's index
  long long pos_sb, offset, total;       // total: units of all tokens
  int N, d, rot, units, turned, hchunk;  // units per token, the first `turned` of which are rotated, the others copied
  int lanes;                             // heads side by side in a workgroup
  float scale, sign;
};

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

// Vectors of a thread: neighbours in a pair are in one vector, halves apart in two.  (Neighbours one by one, VW = 1, are two as well.)
template <int VW, bool INTER> constexpr int vectors() { return INTER && VW > 1 ? 1 : 2; }

// The vectors of one head; INTER: elements 2i, 2i + 1 of them laid end to end are a pair, otherwise i and VW + i.
template <bool BF16, int VW, bool INTER, int NV>
__device__ __forceinline__ void turn(typename Vec<VW>::type (&v)[NV], const float (&c)[NV * VW / 2], const float (&s)[NV * VW / 2]) {
  float x[NV * VW], f[VW];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    unpack<BF16, VW>(v[k], f);
#pragma unroll
    for (int i = 0; i < VW; ++i) x[k * VW + i] = f[i];
  }
#pragma unroll
  for (int i = 0; i < NV * VW / 2; ++i) {
    const int at = INTER ? 2 * i : i, to = INTER ? 2 * i + 1 : VW + i;
    const float a = x[at], b = x[to];
    x[at] = __fmaf_rn(a, c[i], -__fmul_rn(b, s[i]));
    x[to] = __fmaf_rn(b, c[i], __fmul_rn(a, s[i]));
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int i = 0; i < VW; ++i) f[i] = x[k * VW + i];
    v[k] = pack<BF16, VW>(f);
  }
}

// Grid: (units of all tokens / 256, pieces of the heads, what of the first does not fit a dimension).  PAST: reads and writes pass the caches by.
template <bool BF16, int VW, bool INTER, bool PAST>
__global__ void __launch_bounds__(256) k_rope(const RopeParams p) {
  constexpr int NV = vectors<VW, INTER>(), NP = NV * VW / 2;       // vectors and pairs of a thread
  const long long id = ((long long)blockIdx.z * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  if (id >= p.total) return;
  const long long th = id / p.units, tok = th / p.lanes;
  const int unit = (int)(id - th * p.units), hl = (int)(th - tok * p.lanes);
  const long long b = tok / p.N;
  const int n = (int)(tok - b * p.N);
  const bool turned = unit < p.turned;
  float c[NP], s[NP];
  int at[NV];                        // first channel of each vector; what is not turned is split like what is
  at[0] = (turned ? 0 : p.rot) + (INTER ? NV : 1) * VW * (turned ? unit : unit - p.turned);
  if constexpr (NV == 2) at[1] = at[0] + (INTER ? VW : (turned ? p.rot : p.d - p.rot) / 2);
  if (turned) {
    const double pos = (double)((p.positions ? (long long)p.positions[b * p.pos_sb + n] : (long long)n) + p.offset);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const double turns = pos * p.inv_freq[NP * unit + i] * 0.15915494309189533577;      // 1 / (2 pi)
      const float x = 2.0f * (float)(turns - rint(turns));
      float si, co;
      sincospif(x, &si, &co);
      c[i] = __fmul_rn(co, p.scale);
      s[i] = __fmul_rn(si, p.sign);
    }
  }
  const int h0 = blockIdx.y * p.hchunk, h1 = min(h0 + p.hchunk, p.q.heads + p.k.heads);
  typedef typename Vec<VW>::type V;
  constexpr int HU = 8 / NV;         // heads whose loads are in flight together
  auto run = [&](const RopeTensor& t, int ha, int hb) {
    const unsigned short* x = t.x + b * t.xb + (long long)n * t.xn;
    unsigned short* y = t.y + b * t.yb + (long long)n * t.yn;
    for (int h = ha + hl; h < hb; h += HU * p.lanes) {
      V v[HU][NV];
#pragma unroll
      for (int i = 0; i < HU; ++i) {
        const unsigned short* r = x + (long long)min(h + i * p.lanes, hb - 1) * t.xh;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const V* from = reinterpret_cast<const V*>(r + at[k]);
          v[i][k] = PAST ? __builtin_nontemporal_load(from) : *from;
        }
      }
#pragma unroll
      for (int i = 0; i < HU; ++i) {
        if (h + i * p.lanes >= hb) break;
        if (turned) turn<BF16, VW, INTER, NV>(v[i], c, s);
        unsigned short* r = y + (long long)(h + i * p.lanes) * t.yh;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          V* to = reinterpret_cast<V*>(r + at[k]);
          if (PAST) __builtin_nontemporal_store(v[i][k], to);
          else *to = v[i][k];
        }
      }
    }
  };
  if (h0 < p.q.heads) run(p.q, h0, min(h1, p.q.heads));
  if (h1 > p.q.heads) run(p.k, max(h0 - p.q.heads, 0), h1 - p.q.heads);
}

// Strides of one tensor, as given or contiguous in `layout`; false if they are not usable.
bool tensor_strides(const long long* given, int layout, int heads, int N, int d, long long (&st)[3]) {
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
bool rows_apart(const long long (&st)[3], long long B, long long heads, long long N, long long d) {
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
bool reaches(Terms& t, int i, long long at) {
  if (i == t.n) return at > -t.d && at < t.d;
  const long long s = t.stride[i], least = -t.d + 1 - at - t.high[i + 1], most = t.d - 1 - at - t.low[i + 1];
  const long long from = std::max(t.lo[i], least >= 0 ? (least + s - 1) / s : -(-least / s)), to = std::min(t.hi[i], most >= 0 ? most / s : -((-most + s - 1) / s));
  for (long long v = from; v <= to; ++v)
    if (t.tries-- <= 0 || reaches(t, i + 1, at + v * s)) return t.tries > 0;
  return false;
}
bool rows_meet(const void* x, const long long (&sx)[3], int hx, const void* y, const long long (&sy)[3], int hy, long long B, long long N, long long d) {
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

template <bool BF16, int VW>
void launch(const RopeParams& p, bool inter, bool past, dim3 grid, hipStream_t s) {
  if constexpr (VW == 8) {
    if (past && inter) return k_rope<BF16, VW, true, true><<<grid, 256, 0, s>>>(p);
    if (past) return k_rope<BF16, VW, false, true><<<grid, 256, 0, s>>>(p);
  }
  if (inter) k_rope<BF16, VW, true, false><<<grid, 256, 0, s>>>(p);
  else k_rope<BF16, VW, false, false><<<grid, 256, 0, s>>>(p);
}

}  // namespace
}  // namespace sage

using namespace sage;

extern "C" int sage_rope(const sage_rope_args* a) {
  if (!a) return SAGE_ERR_INVALID_ARG;
  const bool keys = a->k != nullptr;
  if (a->B <= 0 || a->H <= 0 || a->N <= 0 || a->rot_dim <= 0 || (keys ? a->H_kv <= 0 : a->k_out != nullptr)) return SAGE_ERR_INVALID_ARG;
  if (!a->q || !a->q_out || (keys && !a->k_out) || !a->inv_freq) return SAGE_ERR_INVALID_ARG;
  if (a->d != 64 && a->d != 128 && a->d != 256) return SAGE_ERR_UNSUPPORTED;
  if (a->rot_dim % 2 != 0 || a->rot_dim > a->d) return SAGE_ERR_UNSUPPORTED;
  if (a->dtype != SAGE_DT_FP16 && a->dtype != SAGE_DT_BF16) return SAGE_ERR_UNSUPPORTED;
  if (a->layout != SAGE_LAYOUT_HND && a->layout != SAGE_LAYOUT_NHD) return SAGE_ERR_UNSUPPORTED;
  if (a->N > MAX_TOKENS || a->B > 65535 || a->H > 65535 || a->H_kv > 65535) return SAGE_ERR_UNSUPPORTED;
  if ((a->interleaved & ~1) != 0 || (a->inverse & ~1) != 0) return SAGE_ERR_UNSUPPORTED;
  if ((((uintptr_t)a->q | (uintptr_t)a->k | (uintptr_t)a->q_out | (uintptr_t)a->k_out) & 1u) != 0) return SAGE_ERR_INVALID_ARG;
  if (((uintptr_t)a->inv_freq & 7u) != 0 || ((uintptr_t)a->positions & 3u) != 0 || a->positions_stride < 0) return SAGE_ERR_INVALID_ARG;
  if (!std::isfinite(a->scale) || a->offset > 1LL << 52 || a->offset < -(1LL << 52)) return SAGE_ERR_INVALID_ARG;        // (positions stay whole numbers in FP64)

  RopeParams p;
  long long st[4][3];
  const long long* given[4] = {a->q_strides, a->k_strides, a->q_out_strides, a->k_out_strides};
  for (int i = 0; i < 4; ++i) {
    const int heads = (i & 1) ? a->H_kv : a->H;
    if ((i & 1) && !keys) { st[i][0] = st[i][1] = st[i][2] = 0; continue; }
    if (!tensor_strides(given[i], a->layout, heads, a->N, a->d, st[i])) return SAGE_ERR_INVALID_ARG;
    const int extent[3] = {a->B, heads, a->N};
    for (int x = 0; x < 3; ++x) {
      if (extent[x] == 1) st[i][x] = 0;        // (no step is taken: whatever it is, it does not count)
      else if (st[i][x] > (1LL << 50) / (extent[x] - 1)) return SAGE_ERR_INVALID_ARG;        // (past any memory, and sums stay within 64 bits)
    }
    if (i >= 2 && !rows_apart(st[i], a->B, heads, a->N, a->d)) return SAGE_ERR_INVALID_ARG;
  }
  // Each output against all that is there before it: in place the same rows, or a thread would overwrite what another has still to read.
  const void* at[4] = {a->q, a->k, a->q_out, a->k_out};
  const int heads_of[4] = {a->H, a->H_kv, a->H, a->H_kv};
  for (int y = 2; y < (keys ? 4 : 3); ++y)
    for (int x = 0; x < y; ++x) {
      if (x == 1 && !keys) continue;
      if (x == y - 2 && at[x] == at[y]) {
        if (st[x][0] != st[y][0] || st[x][1] != st[y][1] || st[x][2] != st[y][2]) return SAGE_ERR_INVALID_ARG;
      } else if (rows_meet(at[x], st[x], heads_of[x], at[y], st[y], heads_of[y], a->B, a->N, a->d)) {
        return SAGE_ERR_INVALID_ARG;
      }
    }
  auto tensor = [&](const void* x, void* y, int i, int heads) {
    RopeTensor t;
    t.x = (const unsigned short*)x; t.y = (unsigned short*)y;
    t.xb = st[i][0]; t.xh = st[i][1]; t.xn = st[i][2];
    t.yb = st[i + 2][0]; t.yh = st[i + 2][1]; t.yn = st[i + 2][2];
    t.heads = heads;
    return t;
  };
  p.q = tensor(a->q, a->q_out, 0, a->H);
  p.k = tensor(a->k, a->k_out, 1, keys ? a->H_kv : 0);
  p.inv_freq = a->inv_freq; p.positions = a->positions; p.pos_sb = a->positions_stride; p.offset = a->offset;
  p.N = a->N; p.d = a->d; p.rot = a->rot_dim;
  p.scale = a->scale == 0.0f ? 1.0f : a->scale;
  p.sign = a->inverse ? -p.scale : p.scale;

  // Widest access that every row allows: both halves of a pair's vectors start at a multiple of it.
  unsigned long long rows = (uintptr_t)a->q / 2 | (uintptr_t)a->q_out / 2 | (uintptr_t)a->k / 2 | (uintptr_t)a->k_out / 2;
  for (auto& s : st) rows |= (unsigned long long)(s[0] | s[1] | s[2]);
  const unsigned long long bits = rows | (unsigned long long)(a->rot_dim / 2);
  const int vw = (bits & 7) == 0 ? 8 : (bits & 3) == 0 ? 4 : 1;
  const bool inter = a->interleaved != 0;
  const int unit = inter && vw > 1 ? vw : 2 * vw;       // channels of a thread
  p.turned = a->rot_dim / unit;
  // (in place, what is not turned stays where it is)
  const bool in_place = a->q == a->q_out && (!keys || a->k == a->k_out);
  const int rest = in_place ? 0 : a->d - a->rot_dim;
  p.units = p.turned + rest / unit;
  // Reads and writes pass the caches by where every access of a wavefront is whole lines of 128 bytes - pieces of lines would be slower that way:
  // 30000 tokens of 64 heads of 64 in halves of 64 bytes 107 us, not 95 - and where what is read and written does not fit the
  // 256 MB of the memory-side cache.  Below that what comes next, which reads these rows, finds them there: 2 x 1024 tokens of 40 heads of 128 and
  // their attention 59.2 us, 60.6 past the caches.  From there on 2 x 17776 tokens of 96 heads of 64 165 kept / 155 past, 4 x 4096 of
  // 40 heads of 128 65 / 60, with the statistics of the keys after it 76.8 / 76.8.
  const bool whole_lines = vw == 8 && (rows & 63) == 0 && (inter ? (a->rot_dim + rest) % 64 == 0 : a->rot_dim % 128 == 0 && rest % 128 == 0);
  const bool past = whole_lines && 4LL * a->B * a->N * (p.q.heads + p.k.heads) * (a->rot_dim + rest) > 256LL << 20;
  // Token-major rows: neighbouring threads take neighbouring heads of a token, which are one stretch of memory; with a token each they
  // would read pieces of 256 bytes, a token's row apart (4 x 4096 tokens of 40 heads of 128: 80 us, so 60).
  p.lanes = 1;
  if (st[0][1] < st[0][2] && a->N > 1) while (p.lanes * 2 * p.units <= 64 && p.lanes * 2 <= a->H) p.lanes *= 2;
  p.total = (long long)a->B * a->N * p.units * p.lanes;
  const long long blocks = (p.total + 255) / 256;
  const long long wide = std::min(blocks, 1LL << 22), deep = (blocks + wide - 1) / wide;
  if (deep > 65535) return SAGE_ERR_UNSUPPORTED;
  // Heads are divided over workgroups only until there are sixteen of these per CU: each pays for the angles again.  (Eight: 2 x 17776
  // tokens of 96 heads of 64 163 us, sixteen 155.)  Heads that lie side by side in one stay together.
  const int heads = p.q.heads + p.k.heads;
  const long long pieces = std::max(1LL, std::min((4096 + blocks - 1) / blocks, (long long)heads / p.lanes));
  p.hchunk = (int)((heads + pieces - 1) / pieces);
  const dim3 grid((unsigned)wide, (unsigned)((heads + p.hchunk - 1) / p.hchunk), (unsigned)deep);
  const hipStream_t s = (hipStream_t)a->stream;
  if (a->dtype == SAGE_DT_BF16) {
    if (vw == 8) launch<true, 8>(p, inter, past, grid, s); else if (vw == 4) launch<true, 4>(p, inter, false, grid, s); else launch<true, 1>(p, inter, false, grid, s);
  } else {
    if (vw == 8) launch<false, 8>(p, inter, past, grid, s); else if (vw == 4) launch<false, 4>(p, inter, false, grid, s); else launch<false, 1>(p, inter, false, grid, s);
  }
  return op_status(hipGetLastError());
}

extern "C" int sage_rope_frequencies(int rot_dim, double base, int scaling, double factor, double original_length, double low, double high,
                                     double* inv_freq) {
  if (!inv_freq || rot_dim <= 0 || rot_dim % 2 != 0 || !(base > 1.0) || !std::isfinite(base)) return SAGE_ERR_INVALID_ARG;
  if (scaling < SAGE_ROPE_PLAIN || scaling > SAGE_ROPE_PARTS) return SAGE_ERR_UNSUPPORTED;
  if (scaling != SAGE_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return SAGE_ERR_INVALID_ARG;
  if (scaling == SAGE_ROPE_PARTS && (!(original_length > 0.0) || !std::isfinite(original_length) || !(low < high) || !std::isfinite(low) || !std::isfinite(high)))
    return SAGE_ERR_INVALID_ARG;
  if (scaling == SAGE_ROPE_BASE && rot_dim == 2) return SAGE_ERR_UNSUPPORTED;      // (one frequency, which no base moves)
  if (scaling == SAGE_ROPE_BASE) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
  if (!std::isfinite(base)) return SAGE_ERR_INVALID_ARG;                            // (the raised one)
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == SAGE_ROPE_LINEAR) f /= factor;
    if (scaling == SAGE_ROPE_PARTS) {
      const double turns = original_length * f / 6.283185307179586477;
      const double keep = std::fmin(std::fmax((turns - low) / (high - low), 0.0), 1.0);
      f *= keep + (1.0 - keep) / factor;
    }
    inv_freq[i] = f;
  }
  return SAGE_OK;
}
