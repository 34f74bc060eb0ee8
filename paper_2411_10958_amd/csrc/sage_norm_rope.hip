// Norms of every head's queries and keys with their rotation (sage_qk_norm_rope), and the gradient (sage_qk_norm_rope_bwd).
//
// y = R(x r w), r = 1 / sqrt(mean(x^2) + eps), R the rotation of sage_rope.hip.  With g = R^T dy:  dw = sum over rows of g x r  and, since
// x r has a norm of its own that no step along x changes,  dx = r (g w - x r^2 mean(g w x)).  Both sums of a row, x^2 and g w x, are taken
// in one go, so every value is read once.
// A row is d / 16 neighbouring threads, each with 8 pairs of channels in registers; a thread works the angles and weights of its channels out once and then walks over
// the heads of its token.  Only bytes bound it: 4 a value forward, 6 backward.
#include "sage_attn.h"
#include "sage_quant.h"
#include "sage_rows.h"

#include <algorithm>
#include <cmath>

namespace sage {
namespace {

struct NormTensor {
  const unsigned short *x, *dy;          // dy: the gradient that comes in (backward)
  unsigned short* y;                     // the result, or dx
  const void* w;
  float* part;                           // of the weight's gradient, [workgroup][2 d]; null: not wanted
  long long xs[3], gs[3], ys[3];         // strides of batch, head and token of x, dy, y
  int heads;
};
struct NormParams {
  NormTensor q, k;                       // k.heads = 0 without keys
  const double* inv_freq;
  const int* positions;                  // null: the token's index
  long long pos_sb, offset, total;       // total: threads of all tokens
  int N, d, rot, units, hchunk, lanes;   // threads of a row; heads of a workgroup, and those side by side in it
  int weight_same;
  float eps, scale;
};

// Sum over the `units` neighbouring threads of a row, in all of them.
__device__ __forceinline__ float row_sum(float x, int units) {
  x += __uint_as_float(butterfly<1>(__float_as_uint(x)));
  x += __uint_as_float(butterfly<2>(__float_as_uint(x)));
  if (units >= 8) x += __uint_as_float(butterfly<4>(__float_as_uint(x)));
  if (units >= 16) x += __uint_as_float(butterfly<8>(__float_as_uint(x)));
  return x;
}

// The 16 channels of a thread of a row, in vectors of VW: pairs 8 u .. 8 u + 7, of which the first rot / 2 of the row are turned.  Neighbours (INTER) are
// channels 16 u .. 16 u + 15 in order; otherwise the first VW * NV / 2 are the pairs' first channels and the others their second ones, and what
// is not turned is split like what is.
template <int VW, bool INTER> struct Channels {
  static constexpr int NV = 16 / VW;
  int at[NV];
  __device__ __forceinline__ Channels(int u, int rot, int d) {
#pragma unroll
    for (int s = 0; s < NV; ++s) {
      if (INTER) {
        at[s] = 16 * u + VW * s;
      } else {
        const int pair = 8 * u + VW * (s % (NV / 2));
        const bool turned = pair < rot / 2, second = s >= NV / 2;
        at[s] = pair + (second ? (turned ? rot / 2 : d / 2) : (turned ? 0 : rot / 2));
      }
    }
  }
};
// Where pair i of a thread is among its 16 channels.
template <bool INTER> __device__ __forceinline__ constexpr int first_of(int i) { return INTER ? 2 * i : i; }
template <bool INTER> __device__ __forceinline__ constexpr int second_of(int i) { return INTER ? 2 * i + 1 : 8 + i; }

template <bool BF16, int VW> __device__ __forceinline__ void unpack16(const typename Vec<VW>::type (&v)[16 / VW], float (&x)[16]) {
#pragma unroll
  for (int s = 0; s < 16 / VW; ++s) {
    float f[VW];
    unpack<BF16, VW>(v[s], f);
#pragma unroll
    for (int i = 0; i < VW; ++i) x[VW * s + i] = f[i];
  }
}
template <int VW, bool PAST> __device__ __forceinline__ void load_row(typename Vec<VW>::type (&v)[16 / VW], const unsigned short* row, const int (&at)[16 / VW]) {
  typedef typename Vec<VW>::type V;
#pragma unroll
  for (int s = 0; s < 16 / VW; ++s) {
    const V* from = reinterpret_cast<const V*>(row + at[s]);
    v[s] = PAST ? __builtin_nontemporal_load(from) : *from;
  }
}
template <bool BF16, int VW, bool PAST> __device__ __forceinline__ void store_row(const float (&x)[16], unsigned short* row, const int (&at)[16 / VW]) {
  typedef typename Vec<VW>::type V;
#pragma unroll
  for (int s = 0; s < 16 / VW; ++s) {
    float f[VW];
#pragma unroll
    for (int i = 0; i < VW; ++i) f[i] = x[VW * s + i];
    const V v = pack<BF16, VW>(f);
    V* to = reinterpret_cast<V*>(row + at[s]);
    if (PAST) __builtin_nontemporal_store(v, to);
    else *to = v;
  }
}
template <bool BF16, int VW> __device__ __forceinline__ void load_weight(float (&w)[16], const void* from, int same, const int (&at)[16 / VW]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int c = at[i / VW] + i % VW;
    w[i] = !from ? 1.0f : same ? load16<BF16>(reinterpret_cast<const unsigned short*>(from)[c]) : reinterpret_cast<const float*>(from)[c];
  }
}

// Which token, head and channels a thread has, and the angles of its pairs; angles are taken as in sage_rope.hip.
struct Place { long long b; int n, unit, hl; };
__device__ __forceinline__ Place place_of(const NormParams& p, long long id) {
  Place a;
  const long long th = id / p.units, tok = th / p.lanes;
  a.unit = (int)(id - th * p.units);
  a.hl = (int)(th - tok * p.lanes);
  a.b = tok / p.N;
  a.n = (int)(tok - a.b * p.N);
  return a;
}
__device__ __forceinline__ void angles(const NormParams& p, const Place& a, float (&c)[8], float (&s)[8]) {
  if (16 * a.unit >= p.rot) return;
  const double pos = (double)((p.positions ? (long long)p.positions[a.b * p.pos_sb + a.n] : (long long)a.n) + p.offset);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double turns = 8 * a.unit + i < p.rot / 2 ? pos * p.inv_freq[8 * a.unit + i] * 0.15915494309189533577 : 0.0;      // 1 / (2 pi)
    float si, co;
    sincospif(2.0f * (float)(turns - rint(turns)), &si, &co);
    c[i] = __fmul_rn(co, p.scale);
    s[i] = __fmul_rn(si, p.scale);
  }
}

// Grid: (threads of all tokens / 256, pieces of the heads, what of the first does not fit a dimension).  PAST: reads and writes pass the caches by.
template <bool BF16, int VW, bool INTER, bool PAST>
__global__ void __launch_bounds__(256) k_norm_rope(const NormParams p) {
  const long long id = ((long long)blockIdx.z * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  if (id >= p.total) return;             // (whole rows)
  const Place a = place_of(p, id);
  const Channels<VW, INTER> ch(a.unit, p.rot, p.d);
  const int pairs = p.rot / 2 - 8 * a.unit;       // pairs of mine that are turned: the first
  float c[8], s[8];
  angles(p, a, c, s);
  const float inv_d = 1.0f / (float)p.d;
  auto run = [&](const NormTensor& t, int ha, int hb) {
    float w[16];
    load_weight<BF16, VW>(w, t.w, p.weight_same, ch.at);
    const unsigned short* x0 = t.x + a.b * t.xs[0] + (long long)a.n * t.xs[2];
    unsigned short* y0 = t.y + a.b * t.ys[0] + (long long)a.n * t.ys[2];
    for (int h = ha + a.hl; h < hb; h += p.lanes) {
      typename Vec<VW>::type v[16 / VW];
      load_row<VW, PAST>(v, x0 + (long long)h * t.xs[1], ch.at);
      float x[16];
      unpack16<BF16, VW>(v, x);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum = __fmaf_rn(x[i], x[i], sum);
      const float r = rsqrtf(__fmaf_rn(row_sum(sum, p.units), inv_d, p.eps));
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = x[i] * r * w[i];
      if (pairs > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float f = x[first_of<INTER>(i)], g = x[second_of<INTER>(i)];
          x[first_of<INTER>(i)] = i < pairs ? __fmaf_rn(f, c[i], -__fmul_rn(g, s[i])) : f;
          x[second_of<INTER>(i)] = i < pairs ? __fmaf_rn(g, c[i], __fmul_rn(f, s[i])) : g;
        }
      }
      store_row<BF16, VW, PAST>(x, y0 + (long long)h * t.ys[1], ch.at);
    }
  };
  const int h0 = blockIdx.y * p.hchunk, h1 = min(h0 + p.hchunk, p.q.heads + p.k.heads);
  if (h0 < p.q.heads) run(p.q, h0, min(h1, p.q.heads));
  if (h1 > p.q.heads) run(p.k, max(h0 - p.q.heads, 0), h1 - p.q.heads);
}

// A workgroup walks over every gridDim.x-th 256 threads of all tokens, and leaves its sums for the weights' gradients.
constexpr int BWD_GROUPS = 1024;         // workgroups at most
template <bool BF16, int VW, bool INTER, bool PAST>
__global__ void __launch_bounds__(256) k_norm_rope_bwd(const NormParams p) {
  __shared__ float s_dw[4][512];         // [wavefront][q, k][channel]
  float dw[2][16];
#pragma unroll
  for (int i = 0; i < 16; ++i) dw[0][i] = dw[1][i] = 0.0f;
  const float inv_d = 1.0f / (float)p.d;
  const int h0 = blockIdx.y * p.hchunk, h1 = min(h0 + p.hchunk, p.q.heads + p.k.heads);
  const Channels<VW, INTER> ch((int)(threadIdx.x % p.units), p.rot, p.d);      // (256 is a multiple of the units: the same for all tokens)
  for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < p.total; id += (long long)gridDim.x * 256) {
    const Place a = place_of(p, id);
    const int pairs = p.rot / 2 - 8 * a.unit;
    float c[8], s[8];
    angles(p, a, c, s);
    auto run = [&](const NormTensor& t, int ha, int hb, float (&acc)[16]) {
      float w[16];
      load_weight<BF16, VW>(w, t.w, p.weight_same, ch.at);
      const unsigned short* x0 = t.x + a.b * t.xs[0] + (long long)a.n * t.xs[2];
      const unsigned short* g0 = t.dy + a.b * t.gs[0] + (long long)a.n * t.gs[2];
      unsigned short* y0 = t.y + a.b * t.ys[0] + (long long)a.n * t.ys[2];
      for (int h = ha + a.hl; h < hb; h += p.lanes) {
        typename Vec<VW>::type v[16 / VW], u[16 / VW];
        load_row<VW, PAST>(v, x0 + (long long)h * t.xs[1], ch.at);
        load_row<VW, PAST>(u, g0 + (long long)h * t.gs[1], ch.at);
        float x[16], g[16];
        unpack16<BF16, VW>(v, x);
        unpack16<BF16, VW>(u, g);
        if (pairs > 0) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float f = g[first_of<INTER>(i)], e = g[second_of<INTER>(i)];
            g[first_of<INTER>(i)] = i < pairs ? __fmaf_rn(f, c[i], __fmul_rn(e, s[i])) : f;
            g[second_of<INTER>(i)] = i < pairs ? __fmaf_rn(e, c[i], -__fmul_rn(f, s[i])) : e;
          }
        }
        float squares = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          squares = __fmaf_rn(x[i], x[i], squares);
          dot = __fmaf_rn(g[i] * w[i], x[i], dot);
        }
        const float r = rsqrtf(__fmaf_rn(row_sum(squares, p.units), inv_d, p.eps));
        const float m = row_sum(dot, p.units) * inv_d * r * r;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          acc[i] = __fmaf_rn(g[i], x[i] * r, acc[i]);
          x[i] = r * __fmaf_rn(-x[i], m, g[i] * w[i]);
        }
        store_row<BF16, VW, PAST>(x, y0 + (long long)h * t.ys[1], ch.at);
      }
    };
    if (h0 < p.q.heads) run(p.q, h0, min(h1, p.q.heads), dw[0]);
    if (h1 > p.q.heads) run(p.k, max(h0 - p.q.heads, 0), h1 - p.q.heads, dw[1]);
  }
  if (!p.q.part && !p.k.part) return;
  // Threads of the same channels: those of a wavefront by shuffles, then the four wavefronts'
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x = dw[k][i];
      for (int o = p.units; o < 64; o <<= 1) x += __shfl_xor(x, o);
      if (lane < p.units) s_dw[wave][k * p.d + ch.at[i / VW] + i % VW] = x;
    }
  __syncthreads();
  float* part = p.q.part ? p.q.part : p.k.part;
  const size_t group = (size_t)blockIdx.y * gridDim.x + blockIdx.x;
  for (int i = threadIdx.x; i < 2 * p.d; i += 256) part[group * 2 * p.d + i] = (s_dw[0][i] + s_dw[1][i]) + (s_dw[2][i] + s_dw[3][i]);
}

// The weights' gradients from the workgroups' sums: 32 channels a workgroup, every 32nd workgroup's sum a thread.
__global__ void __launch_bounds__(1024) k_weight_grad(const float* part, int groups, int d, float* dqw, float* dkw) {
  __shared__ double s_sum[32][33];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5, at = blockIdx.x * 32 + c;
  double sum = 0.0;
#pragma unroll 8
  for (int i = g; i < groups; i += 32) sum += (double)part[(size_t)i * 2 * d + at];
  s_sum[g][c] = sum;
  __syncthreads();
  if (g != 0) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) sum += s_sum[i][c];
  float* to = at < d ? dqw : dkw;
  if (to) to[at < d ? at : at - d] = (float)sum;
}

// What the two calls' structures have in common, checked.
struct NormShape {
  int B, H, Hkv, N, d, rot, dtype, layout, weight_type, interleaved;
  float eps, scale;
  const double* inv_freq;
  const int* positions;
  long long pos_sb, offset;
  const void *q_weight, *k_weight;
  bool keys;
};
template <typename A> NormShape shape_of(const A* a) {
  return {a->B, a->H, a->H_kv, a->N, a->d, a->rot_dim, a->dtype, a->layout, a->weight_type, a->interleaved, a->eps, a->scale, a->inv_freq, a->positions,
          a->positions_stride, a->offset, a->q_weight, a->k_weight, a->k != nullptr};
}
int check_shape(const NormShape& a) {
  if (a.B <= 0 || a.H <= 0 || a.N <= 0 || a.rot < 0 || (a.keys && a.Hkv <= 0) || (!a.keys && a.k_weight)) return SAGE_ERR_INVALID_ARG;
  if (a.d != 64 && a.d != 128 && a.d != 256) return SAGE_ERR_UNSUPPORTED;
  if (a.rot % 2 != 0 || a.rot > a.d) return SAGE_ERR_UNSUPPORTED;
  if (a.dtype != SAGE_DT_FP16 && a.dtype != SAGE_DT_BF16) return SAGE_ERR_UNSUPPORTED;
  if (a.layout != SAGE_LAYOUT_HND && a.layout != SAGE_LAYOUT_NHD) return SAGE_ERR_UNSUPPORTED;
  if (a.weight_type != SAGE_WEIGHT_FP32 && a.weight_type != SAGE_WEIGHT_SAME) return SAGE_ERR_UNSUPPORTED;
  if (a.N > MAX_TOKENS || a.B > 65535 || a.H > 65535 || (a.keys && a.Hkv > 65535)) return SAGE_ERR_UNSUPPORTED;
  if ((a.interleaved & ~1) != 0) return SAGE_ERR_UNSUPPORTED;
  return SAGE_OK;
}
int check_values(const NormShape& a) {
  if (a.rot > 0 && !a.inv_freq) return SAGE_ERR_INVALID_ARG;
  if (((uintptr_t)a.inv_freq & 7u) != 0 || ((uintptr_t)a.positions & 3u) != 0 || a.pos_sb < 0) return SAGE_ERR_INVALID_ARG;
  if ((((uintptr_t)a.q_weight | (uintptr_t)a.k_weight) & (a.weight_type == SAGE_WEIGHT_FP32 ? 3u : 1u)) != 0) return SAGE_ERR_INVALID_ARG;
  if (!(a.eps >= 0.0f) || !std::isfinite(a.eps) || !std::isfinite(a.scale) || a.offset > 1LL << 52 || a.offset < -(1LL << 52)) return SAGE_ERR_INVALID_ARG;
  return SAGE_OK;
}

// One strided tensor of a call: where, its strides, and whether it is written.
struct NormView { const void* at; const long long* given; int heads; bool out; int in_place; long long st[3]; };      // in_place: which view it may be, or -1
// Strides, and each output against all that is there before it and all that is read besides: in place the same rows.
int check_views(NormView* v, int count, const NormShape& a, const Span* read, int reads) {
  for (int i = 0; i < count; ++i) {
    if (!v[i].at) { v[i].st[0] = v[i].st[1] = v[i].st[2] = 0; continue; }
    if (((uintptr_t)v[i].at & 1u) != 0 || !tensor_strides(v[i].given, a.layout, v[i].heads, a.N, a.d, v[i].st)) return SAGE_ERR_INVALID_ARG;
    const int extent[3] = {a.B, v[i].heads, a.N};
    long long span = a.d;
    for (int x = 0; x < 3; ++x) {
      if (extent[x] == 1) v[i].st[x] = 0;      // (no step is taken: whatever it is, it does not count)
      else if (v[i].st[x] > (1LL << 50) / (extent[x] - 1)) return SAGE_ERR_INVALID_ARG;      // (past any memory, and sums stay within 64 bits)
      span += v[i].st[x] * (extent[x] - 1);
    }
    if (!v[i].out) continue;
    if (!rows_apart(v[i].st, a.B, v[i].heads, a.N, a.d)) return SAGE_ERR_INVALID_ARG;
    for (int r = 0; r < reads; ++r) if (overlap({v[i].at, (size_t)span * 2}, read[r])) return SAGE_ERR_INVALID_ARG;
  }
  for (int y = 0; y < count; ++y) {
    if (!v[y].out || !v[y].at) continue;
    for (int x = 0; x < count; ++x) {
      if (x == y || !v[x].at || (v[x].out && x > y)) continue;
      if (x == v[y].in_place && v[x].at == v[y].at) {
        for (int i = 0; i < 3; ++i) if (v[x].st[i] != v[y].st[i]) return SAGE_ERR_INVALID_ARG;
      } else if (rows_meet(v[x].at, v[x].st, v[x].heads, v[y].at, v[y].st, v[y].heads, a.B, a.N, a.d)) {
        return SAGE_ERR_INVALID_ARG;
      }
    }
  }
  return SAGE_OK;
}

// What the kernels take, but for the tensors' pointers; the widest access that every row allows, and the grid.
struct NormLaunch { dim3 grid; int vw; bool inter, past; };
void plan(NormParams* p, NormLaunch* l, const NormShape& a, const NormView* v, int count, int most, int bytes) {
  unsigned long long rows = 0;
  for (int i = 0; i < count; ++i) if (v[i].at) rows |= (uintptr_t)v[i].at / 2 | (unsigned long long)(v[i].st[0] | v[i].st[1] | v[i].st[2]);
  l->inter = a.interleaved != 0;
  const unsigned long long bits = rows | (l->inter ? 0ull : (unsigned long long)(a.rot / 2));
  l->vw = (bits & 7) == 0 ? 8 : (bits & 3) == 0 ? 4 : 1;
  l->past = false;
  (void)bytes;
  p->inv_freq = a.inv_freq; p->positions = a.positions; p->pos_sb = a.pos_sb; p->offset = a.offset;
  p->N = a.N; p->d = a.d; p->rot = a.rot; p->units = a.d / 16;
  p->weight_same = a.weight_type == SAGE_WEIGHT_SAME;
  p->eps = a.eps; p->scale = a.scale == 0.0f ? 1.0f : a.scale;
  // Token-major rows: neighbouring threads take neighbouring heads of a token, which are one stretch of memory.
  p->lanes = 1;
  if (v[0].st[1] < v[0].st[2] && a.N > 1) while (p->lanes * 2 * p->units <= 64 && p->lanes * 2 <= a.H) p->lanes *= 2;
  p->total = (long long)a.B * a.N * p->units * p->lanes;
  const long long blocks = (p->total + 255) / 256;
  const int heads = a.H + (a.keys ? a.Hkv : 0);
  const long long wide = std::min(blocks, most > 0 ? (long long)most : 1LL << 22), deep = most > 0 ? 1 : (blocks + wide - 1) / wide;
  const long long want = most > 0 ? most / wide : (4096 + blocks - 1) / blocks;
  const long long pieces = std::max(1LL, std::min(want, (long long)heads / p->lanes));
  p->hchunk = (int)((heads + pieces - 1) / pieces);
  l->grid = dim3((unsigned)wide, (unsigned)((heads + p->hchunk - 1) / p->hchunk), (unsigned)deep);
}

template <bool BF16, int VW> void launch(const NormParams& p, const NormLaunch& l, hipStream_t s) {
  if constexpr (VW == 8) {
    if (l.past && l.inter) return k_norm_rope<BF16, VW, true, true><<<l.grid, 256, 0, s>>>(p);
    if (l.past) return k_norm_rope<BF16, VW, false, true><<<l.grid, 256, 0, s>>>(p);
  }
  if (l.inter) k_norm_rope<BF16, VW, true, false><<<l.grid, 256, 0, s>>>(p);
  else k_norm_rope<BF16, VW, false, false><<<l.grid, 256, 0, s>>>(p);
}
template <bool BF16, int VW> void launch_bwd(const NormParams& p, const NormLaunch& l, hipStream_t s) {
  if constexpr (VW == 8) {
    if (l.past && l.inter) return k_norm_rope_bwd<BF16, VW, true, true><<<l.grid, 256, 0, s>>>(p);
    if (l.past) return k_norm_rope_bwd<BF16, VW, false, true><<<l.grid, 256, 0, s>>>(p);
  }
  if (l.inter) k_norm_rope_bwd<BF16, VW, true, false><<<l.grid, 256, 0, s>>>(p);
  else k_norm_rope_bwd<BF16, VW, false, false><<<l.grid, 256, 0, s>>>(p);
}

NormTensor tensor(const NormView* x, const NormView* dy, const NormView& y, const void* w) {
  NormTensor t = {};
  t.x = (const unsigned short*)x->at; t.y = (unsigned short*)const_cast<void*>(y.at); t.w = w; t.heads = x->at ? x->heads : 0;
  if (dy) t.dy = (const unsigned short*)dy->at;
  for (int i = 0; i < 3; ++i) { t.xs[i] = x->st[i]; t.ys[i] = y.st[i]; if (dy) t.gs[i] = dy->st[i]; }
  return t;
}
size_t weight_bytes(const NormShape& a) { return (size_t)a.d * (a.weight_type == SAGE_WEIGHT_FP32 ? 4 : 2); }
size_t positions_bytes(const NormShape& a) { return a.positions ? ((size_t)a.pos_sb * (a.B - 1) + a.N) * 4 : 0; }
// Workgroups never outnumber the rows of all heads, nor BWD_GROUPS.
size_t bwd_bytes(const sage_qk_norm_rope_bwd_args* a) {
  if (!a->dq_weight && !a->dk_weight) return 0;
  const long long rows = (long long)a->B * a->N * (a->H + (a->k ? a->H_kv : 0));
  return align256((size_t)std::min(rows, (long long)BWD_GROUPS) * 2 * a->d * sizeof(float));
}

}  // namespace
}  // namespace sage

using namespace sage;

extern "C" int sage_qk_norm_rope(const sage_qk_norm_rope_args* a) {
  if (!a) return SAGE_ERR_INVALID_ARG;
  const NormShape sh = shape_of(a);
  if (!a->q || !a->q_out || (a->k != nullptr) != (a->k_out != nullptr)) return SAGE_ERR_INVALID_ARG;
  int st = check_shape(sh);
  if (st == SAGE_OK) st = check_values(sh);
  if (st != SAGE_OK) return st;
  NormView v[4] = {{a->q, a->q_strides, a->H, false, -1, {}}, {a->k, a->k_strides, a->H_kv, false, -1, {}},
                   {a->q_out, a->q_out_strides, a->H, true, 0, {}}, {a->k_out, a->k_out_strides, a->H_kv, true, 1, {}}};
  const Span read[4] = {{a->q_weight, weight_bytes(sh)}, {a->k_weight, weight_bytes(sh)}, {a->rot_dim > 0 ? a->inv_freq : nullptr, (size_t)a->rot_dim * 4},
                        {a->positions, positions_bytes(sh)}};
  st = check_views(v, 4, sh, read, 4);
  if (st != SAGE_OK) return st;
  NormParams p = {};
  NormLaunch l;
  plan(&p, &l, sh, v, 4, 0, 4);
  if (l.grid.z > 65535) return SAGE_ERR_UNSUPPORTED;
  p.q = tensor(&v[0], nullptr, v[2], a->q_weight);
  p.k = tensor(&v[1], nullptr, v[3], a->k_weight);
  const hipStream_t s = (hipStream_t)a->stream;
  if (a->dtype == SAGE_DT_BF16) {
    if (l.vw == 8) launch<true, 8>(p, l, s); else if (l.vw == 4) launch<true, 4>(p, l, s); else launch<true, 1>(p, l, s);
  } else {
    if (l.vw == 8) launch<false, 8>(p, l, s); else if (l.vw == 4) launch<false, 4>(p, l, s); else launch<false, 1>(p, l, s);
  }
  return op_status(hipGetLastError());
}

extern "C" size_t sage_qk_norm_rope_bwd_workspace_bytes(const sage_qk_norm_rope_bwd_args* a) {
  if (!a || check_shape(shape_of(a)) != SAGE_OK) return 0;
  return bwd_bytes(a);
}

extern "C" int sage_qk_norm_rope_bwd(const sage_qk_norm_rope_bwd_args* a) {
  if (!a) return SAGE_ERR_INVALID_ARG;
  const NormShape sh = shape_of(a);
  if (!a->q || !a->dq_out || !a->dq || (a->k != nullptr) != (a->dk_out != nullptr) || (a->k != nullptr) != (a->dk != nullptr)) return SAGE_ERR_INVALID_ARG;
  if (!a->k && a->dk_weight) return SAGE_ERR_INVALID_ARG;
  int st = check_shape(sh);
  if (st == SAGE_OK) st = check_values(sh);
  if (st != SAGE_OK) return st;
  if ((((uintptr_t)a->dq_weight | (uintptr_t)a->dk_weight) & 3u) != 0) return SAGE_ERR_INVALID_ARG;
  const size_t need = bwd_bytes(a);
  if (need > 0 && (!a->workspace || a->workspace_bytes < need || ((uintptr_t)a->workspace & 255u) != 0)) return SAGE_ERR_WORKSPACE;
  NormView v[6] = {{a->q, a->q_strides, a->H, false, -1, {}}, {a->k, a->k_strides, a->H_kv, false, -1, {}},
                   {a->dq_out, a->dq_out_strides, a->H, false, -1, {}}, {a->dk_out, a->dk_out_strides, a->H_kv, false, -1, {}},
                   {a->dq, a->dq_strides, a->H, true, 2, {}}, {a->dk, a->dk_strides, a->H_kv, true, 3, {}}};
  // What is read besides the rows, and then what is written besides them
  const Span other[7] = {{a->q_weight, weight_bytes(sh)}, {a->k_weight, weight_bytes(sh)}, {a->rot_dim > 0 ? a->inv_freq : nullptr, (size_t)a->rot_dim * 4},
                         {a->positions, positions_bytes(sh)}, {a->dq_weight, (size_t)a->d * 4}, {a->dk_weight, (size_t)a->d * 4}, {need > 0 ? a->workspace : nullptr, need}};
  st = check_views(v, 6, sh, other, 7);
  if (st != SAGE_OK) return st;
  for (int i = 4; i < 7; ++i) {
    for (int j = 0; j < i; ++j) if (overlap(other[i], other[j])) return SAGE_ERR_INVALID_ARG;
    for (int j = 0; j < 4; ++j) {
      size_t span = (size_t)a->d;
      const int extent[3] = {a->B, v[j].heads, a->N};
      for (int x = 0; x < 3; ++x) span += (size_t)v[j].st[x] * (extent[x] - 1);
      if (v[j].at && overlap(other[i], {v[j].at, span * 2})) return SAGE_ERR_INVALID_ARG;
    }
  }
  NormParams p = {};
  NormLaunch l;
  plan(&p, &l, sh, v, 6, BWD_GROUPS, 6);
  p.q = tensor(&v[0], &v[2], v[4], a->q_weight);
  p.k = tensor(&v[1], &v[3], v[5], a->k_weight);
  if (need > 0) p.q.part = (float*)a->workspace;
  const hipStream_t s = (hipStream_t)a->stream;
  if (a->dtype == SAGE_DT_BF16) {
    if (l.vw == 8) launch_bwd<true, 8>(p, l, s); else if (l.vw == 4) launch_bwd<true, 4>(p, l, s); else launch_bwd<true, 1>(p, l, s);
  } else {
    if (l.vw == 8) launch_bwd<false, 8>(p, l, s); else if (l.vw == 4) launch_bwd<false, 4>(p, l, s); else launch_bwd<false, 1>(p, l, s);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && need > 0) {
    k_weight_grad<<<2 * a->d / 32, 1024, 0, s>>>((const float*)a->workspace, (int)(l.grid.x * l.grid.y), a->d, a->dq_weight, a->dk_weight);
    e = hipGetLastError();
  }
  return op_status(e);
}
