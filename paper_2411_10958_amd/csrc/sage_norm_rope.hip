// Norms of every head's queries and keys with their rotation (sage_qk_norm_rope), and the gradient (sage_qk_norm_rope_bwd).
//
// y = R(x r w), r = 1 / sqrt(mean(x^2) + eps), R the rotation of sage_rope.hip.  With g = R^T dy:  dw = sum over rows of g x r  and, since
// x r has a norm of its own that no step along x changes,  dx = r (g w - x r^2 mean(g w x)).  Both sums of a row, x^2 and g w x, are taken
// in one go, so every value is read once.
// A row is d / 16 neighbouring threads, each with 8 pairs of channels in registers.  A workgroup takes the heads of a few tokens: it works their angles out
// once, an angle a thread, and leaves them and the weights in LDS (each thread with its own angles, and one row in flight: 77 and 115 us where this takes 62 and 53).  Only bytes bound
// it, 4 a value forward and 6 backward: 4 x 4096 tokens of 40 heads of 128 62 us (5.4 TB/s), the gradient of 2 x 4096 54 us (4.9 TB/s in its first kernel).
#include "sage_attn.h"
#include "sage_quant.h"
#include "sage_rows.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

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
  long long pos_sb, offset;
  unsigned tokens;                       // B N
  int d, rot, units, hchunk;             // threads of a row; heads of a workgroup
  int lanes, at_once, heads_first;       // of a workgroup: heads side by side, tokens; which of them neighbouring threads are
  int weight_same;
  float eps, scale;
  FastDiv by_n, by_pairs, by_lanes, by_at_once;      // N, rot / 2
};

// Sum over the `units` neighbouring threads of a row, in all of them.
__device__ __forceinline__ float row_sum(float x, int units) {
  x += __uint_as_float(butterfly<1>(__float_as_uint(x)));
  x += __uint_as_float(butterfly<2>(__float_as_uint(x)));
  if (units >= 8) x += __uint_as_float(butterfly<4>(__float_as_uint(x)));
  if (units >= 16) x += __uint_as_float(butterfly<8>(__float_as_uint(x)));
  return x;
}

// The 16 channels of a thread of a row, in vectors of VW, eight here and eight there so that a row's threads read stretches of d bytes.  Channels i and rot / 2 + i are a pair: pairs
// 8 u .. 8 u + 7, first channels first; what is not turned is split like what is.  Neighbours (INTER): channels 8 u .. 8 u + 7 and as many d / 2 on.
template <bool INTER> __device__ __forceinline__ int channel_of(int i, int u, int rot, int d) {      // of the thread's value i
  if (INTER) return 8 * u + (i & 7) + (i < 8 ? 0 : d / 2);
  const int pair = 8 * u + (i & 7);
  return pair + (pair < rot / 2 ? (i < 8 ? 0 : rot / 2) : (i < 8 ? rot / 2 : d / 2));
}
template <int VW, bool INTER> struct Channels {
  int at[16 / VW];                       // of each vector's first
  __device__ __forceinline__ Channels(int u, int rot, int d) {
#pragma unroll
    for (int s = 0; s < 16 / VW; ++s) at[s] = channel_of<INTER>(VW * s, u, rot, d);
  }
};
// Where pair i of a thread is among its 16 channels, and which pair of the row it is.
template <bool INTER> __device__ __forceinline__ constexpr int first_of(int i) { return INTER ? 2 * i : i; }
template <bool INTER> __device__ __forceinline__ constexpr int second_of(int i) { return INTER ? 2 * i + 1 : 8 + i; }
template <bool INTER> __device__ __forceinline__ int pair_of(int i, int u, int d) { return INTER ? 4 * u + (i & 3) + (i < 4 ? 0 : d / 4) : 8 * u + i; }

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
// What a workgroup shares: the weights, [q, k][d], and cosines and sines of its tokens' angles, [token][rot / 2], taken as in sage_rope.hip.
constexpr int MAX_AT_ONCE = 64;          // tokens of a workgroup: 256 threads, 4 a row at least
constexpr int CS_ENTRIES = 2048;         // (64 tokens of 64 channels, 32 of 128, 16 of 256)
struct NormShared {
  float w[512];
  float2 cs[CS_ENTRIES];
};
template <bool BF16> __device__ __forceinline__ void share_weights(const NormParams& p, NormShared& sh) {
  for (int i = threadIdx.x; i < 2 * p.d; i += 256) {
    const void* w = i < p.d ? p.q.w : p.k.w;
    const int c = i < p.d ? i : i - p.d;
    sh.w[i] = !w ? 1.0f : p.weight_same ? load16<BF16>(reinterpret_cast<const unsigned short*>(w)[c]) : reinterpret_cast<const float*>(w)[c];
  }
}
__device__ __forceinline__ void share_angles(const NormParams& p, NormShared& sh, unsigned tok0) {
  const int pairs = p.rot / 2;
  for (int i = threadIdx.x; i < p.at_once * pairs; i += 256) {
    unsigned pair = (unsigned)i;
    const unsigned tok = tok0 + split_by(pair, p.by_pairs);
    if (tok >= p.tokens) break;
    unsigned n = tok;
    const unsigned b = split_by(n, p.by_n);
    const double pos = (double)((p.positions ? (long long)p.positions[(long long)b * p.pos_sb + n] : (long long)n) + p.offset);
    const double turns = pos * p.inv_freq[pair] * 0.15915494309189533577;      // 1 / (2 pi)
    float si, co;
    sincospif(2.0f * (float)(turns - rint(turns)), &si, &co);
    sh.cs[i] = make_float2(__fmul_rn(co, p.scale), __fmul_rn(si, p.scale));
  }
}

// Which row of a workgroup a thread has, and its channels.
struct Place { int unit, token, lane; };
__device__ __forceinline__ Place place_of(const NormParams& p) {
  Place a;
  a.unit = (int)(threadIdx.x & (unsigned)(p.units - 1));
  unsigned row = threadIdx.x / (unsigned)p.units;
  if (p.heads_first) {
    a.token = (int)split_by(row, p.by_lanes);
    a.lane = (int)row;
  } else {
    a.lane = (int)split_by(row, p.by_at_once);
    a.token = (int)row;
  }
  return a;
}
template <int VW> __device__ __forceinline__ void weights_of(float (&w)[16], const float* from, const int (&at)[16 / VW]) {
#pragma unroll
  for (int s = 0; s < 16 / VW; ++s) {
    if constexpr (VW >= 4) {
#pragma unroll
      for (int i = 0; i < VW / 4; ++i) {
        const v4f y = *reinterpret_cast<const v4f*>(from + at[s] + 4 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[VW * s + 4 * i + e] = y[e];
      }
    } else {
      w[s] = from[at[s]];
    }
  }
}
// Cosines and sines of a thread's pairs: 1 and 0 for what is not turned.  Whether any is.
template <bool INTER> __device__ __forceinline__ bool angles_of(const NormParams& p, const NormShared& sh, const Place& a, float (&c)[8], float (&s)[8]) {
  const int pairs = p.rot / 2;
  bool any = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int pair = pair_of<INTER>(i, a.unit, p.d);
    c[i] = 1.0f;
    s[i] = 0.0f;
    if (pair < pairs) {
      const float2 y = sh.cs[a.token * pairs + pair];
      c[i] = y.x;
      s[i] = y.y;
      any = true;
    }
  }
  return any;
}
// A product that is zero where a factor is, whatever the other one; else the ordinary one, small results included.
__device__ __forceinline__ float product_or_zero(float x, float y) {
  float r;
  asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(r) : "v"(x), "v"(y));
  return r;
}
// A thread's pairs turned, or turned back.  Where nothing is turned the sine is zero, and a partner that is not finite has no part in the result.
template <bool INTER, bool BACK> __device__ __forceinline__ void turn(float (&x)[16], const float (&c)[8], const float (&s)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float f = x[first_of<INTER>(i)], g = x[second_of<INTER>(i)], fs = product_or_zero(f, s[i]), gs = product_or_zero(g, s[i]);
    x[first_of<INTER>(i)] = __fmaf_rn(f, c[i], BACK ? gs : -gs);
    x[second_of<INTER>(i)] = __fmaf_rn(g, c[i], BACK ? -fs : fs);
  }
}

// Whether nothing of a row is lost in its mean square (with eps): from 2^-60 to 2^120.  Where it is not, the row is multiplied by a power of two first, as its norm does not change by: up, so that
// squares that vanished count, or down, so that their sum fits; then the smallest bf16 numbers have squares that are normal, and those of 256 of the largest add up to 2^124.
// (fp16's squares are all within it.)  The look costs 0.3 us of the 64 of 4 x 4096 tokens of 40 heads of 128, 0.5 of the gradient's 55 of 2 x 4096.
__device__ __forceinline__ bool ordinary(float v) { return __float_as_uint(v) - 0x21800000u < 0x5a000000u; }
__device__ __forceinline__ float lift_of(float v) { return v < 1.0f ? 0x1p70f : 0x1p-70f; }
__device__ __forceinline__ float lifted_root(float (&x)[16], float lift, int units, float inv_d, float eps) {      // 1 / sqrt(mean x^2 + eps) of the row times the power
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    x[i] *= lift;
    sum = __fmaf_rn(x[i], x[i], sum);
  }
  return rsqrtf(__fmaf_rn(row_sum(sum, units), inv_d, eps * lift * lift));
}

// Grid: (groups of tokens, pieces of the heads).  PAST: reads and writes pass the caches by.
template <bool BF16, int VW, bool INTER, bool PAST>
__global__ void __launch_bounds__(256) k_norm_rope(const NormParams p) {
  __shared__ __align__(16) NormShared sh;
  typedef typename Vec<VW>::type V;
  constexpr int HU = VW == 8 ? 4 : 1;    // heads whose loads are in flight together
  const Place a = place_of(p);
  const Channels<VW, INTER> ch(a.unit, p.rot, p.d);
  const unsigned tok0 = blockIdx.x * (unsigned)p.at_once, tok = tok0 + a.token;
  const int heads = p.q.heads + p.k.heads, h0 = blockIdx.y * p.hchunk, h1 = min(h0 + p.hchunk, heads);
  const bool there = tok < p.tokens;
  unsigned n = there ? tok : p.tokens - 1;
  const unsigned b = split_by(n, p.by_n);
  const unsigned short *xq = p.q.x + b * p.q.xs[0] + n * p.q.xs[2], *xk = p.k.x + b * p.k.xs[0] + n * p.k.xs[2];
  auto row_of = [&](int h) { return h < p.q.heads ? xq + h * p.q.xs[1] : xk + (h - p.q.heads) * p.k.xs[1]; };
  V v[HU][16 / VW];
#pragma unroll
  for (int i = 0; i < HU; ++i) load_row<VW, PAST>(v[i], row_of(min(h0 + a.lane + i * p.lanes, h1 - 1)), ch.at);
  share_weights<BF16>(p, sh);
  share_angles(p, sh, tok0);
  __syncthreads();
  if (!there) return;                    // (whole rows)
  float c[8], s[8];
  const bool turned = angles_of<INTER>(p, sh, a, c, s);
  const float inv_d = 1.0f / (float)p.d;
  for (int hh = h0 + a.lane; hh < h1; hh += HU * p.lanes) {
#pragma unroll
    for (int k = 0; k < HU; ++k) {
      const int h = hh + k * p.lanes;
      if (h >= h1) break;
      float x[16], w[16];
      unpack16<BF16, VW>(v[k], x);
      weights_of<VW>(w, sh.w + (h < p.q.heads ? 0 : p.d), ch.at);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum = __fmaf_rn(x[i], x[i], sum);
      const float v2 = __fmaf_rn(row_sum(sum, p.units), inv_d, p.eps);
      float r = rsqrtf(v2);
      if (BF16 && !ordinary(v2)) r = lifted_root(x, lift_of(v2), p.units, inv_d, p.eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = x[i] * r * w[i];
      if (turned) turn<INTER, false>(x, c, s);
      unsigned short* y = h < p.q.heads ? p.q.y + b * p.q.ys[0] + n * p.q.ys[2] + h * p.q.ys[1] : p.k.y + b * p.k.ys[0] + n * p.k.ys[2] + (h - p.q.heads) * p.k.ys[1];
      store_row<BF16, VW, PAST>(x, y, ch.at);
    }
    if (hh + HU * p.lanes < h1) {
#pragma unroll
      for (int i = 0; i < HU; ++i) load_row<VW, PAST>(v[i], row_of(min(hh + (HU + i) * p.lanes, h1 - 1)), ch.at);
    }
  }
}

// A workgroup walks over every gridDim.x-th group of tokens, and leaves its sums for the weights' gradients.
constexpr int BWD_GROUPS = 512;          // workgroups at most: two on a CU, what it has registers for
template <bool BF16, int VW, bool INTER, bool PAST>
__global__ void __launch_bounds__(256) k_norm_rope_bwd(const NormParams p) {
  __shared__ __align__(16) NormShared sh;
  __shared__ float s_dw[4][512];         // [wavefront][q, k][channel]
  typedef typename Vec<VW>::type V;
  constexpr int HU = VW == 8 ? 2 : 1;    // heads whose loads are in flight together
  float dw[32];                          // of q, of k
#pragma unroll
  for (int i = 0; i < 32; ++i) dw[i] = 0.0f;
  const Place a = place_of(p);
  const Channels<VW, INTER> ch(a.unit, p.rot, p.d);
  const float inv_d = 1.0f / (float)p.d;
  const int h0 = blockIdx.y * p.hchunk, h1 = min(h0 + p.hchunk, p.q.heads + p.k.heads);
  share_weights<BF16>(p, sh);
  for (unsigned tok0 = blockIdx.x * (unsigned)p.at_once; tok0 < p.tokens; tok0 += gridDim.x * (unsigned)p.at_once) {
    const unsigned tok = tok0 + a.token;
    const bool there = tok < p.tokens;
    unsigned n = there ? tok : p.tokens - 1;
    const unsigned b = split_by(n, p.by_n);
    V v[HU][16 / VW], u[HU][16 / VW];
    auto load = [&](int hh) {
#pragma unroll
      for (int k = 0; k < HU; ++k) {
        int h = min(hh + k * p.lanes, h1 - 1);
        const NormTensor& t = h < p.q.heads ? p.q : p.k;
        h -= h < p.q.heads ? 0 : p.q.heads;
        load_row<VW, PAST>(v[k], t.x + b * t.xs[0] + n * t.xs[2] + h * t.xs[1], ch.at);
        load_row<VW, PAST>(u[k], t.dy + b * t.gs[0] + n * t.gs[2] + h * t.gs[1], ch.at);
      }
    };
    load(h0 + a.lane);
    __syncthreads();                     // (the angles of the group before have been read)
    share_angles(p, sh, tok0);
    __syncthreads();
    if (!there) continue;
    float c[8], s[8];
    const bool turned = angles_of<INTER>(p, sh, a, c, s);
    for (int hh = h0 + a.lane; hh < h1; hh += HU * p.lanes) {
#pragma unroll
      for (int k = 0; k < HU; ++k) {
        const int h = hh + k * p.lanes;
        if (h >= h1) break;
        const bool key = h >= p.q.heads;
        float x[16], g[16], w[16];
        unpack16<BF16, VW>(v[k], x);
        unpack16<BF16, VW>(u[k], g);
        weights_of<VW>(w, sh.w + (key ? p.d : 0), ch.at);
        if (turned) turn<INTER, true>(g, c, s);
        float squares = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          squares = __fmaf_rn(x[i], x[i], squares);
          dot = __fmaf_rn(g[i] * w[i], x[i], dot);
        }
        const float v2 = __fmaf_rn(row_sum(squares, p.units), inv_d, p.eps);
        float r = rsqrtf(v2), of_x = r, m = row_sum(dot, p.units) * inv_d * r * r;
        if (BF16 && !ordinary(v2)) {                       // (x becomes x r, so that its product with g w does not vanish either; the power of two is in r but for 2^10, for r to fit, which is in w)
          const float lift = lift_of(v2), some = v2 < 1.0f ? 0x1p10f : 0x1p-10f;
          r = lifted_root(x, lift, p.units, inv_d, p.eps);
          dot = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            x[i] *= r;
            dot = __fmaf_rn(g[i] * w[i], x[i], dot);
            w[i] *= some;
          }
          m = row_sum(dot, p.units) * inv_d * some;
          r *= v2 < 1.0f ? 0x1p60f : 0x1p-60f;
          of_x = 1.0f;
        }
        if (!key) {
#pragma unroll
          for (int i = 0; i < 16; ++i) dw[i] = __fmaf_rn(g[i], x[i] * of_x, dw[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) dw[16 + i] = __fmaf_rn(g[i], x[i] * of_x, dw[16 + i]);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = r * __fmaf_rn(-x[i], m, g[i] * w[i]);
        const NormTensor& t = key ? p.k : p.q;
        store_row<BF16, VW, PAST>(x, t.y + b * t.ys[0] + n * t.ys[2] + (h - (key ? p.q.heads : 0)) * t.ys[1], ch.at);
      }
      if (hh + HU * p.lanes < h1) load(hh + HU * p.lanes);
    }
  }
  if (!p.q.part) return;
  // Threads of the same channels, 64 / units of a wavefront: each step leaves half of the values in either half of them (30 exchanges, not 32 a step)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int first = 0;
  auto halve = [&](auto left, int o) {
    constexpr int H = decltype(left)::value / 2;
    if (o < p.units) return;
    const bool up = (lane & o) != 0;
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const float mine = up ? dw[H + i] : dw[i], other = up ? dw[i] : dw[H + i];
      dw[i] = mine + __shfl_xor(other, o);
    }
    first += up ? H : 0;
  };
  halve(std::integral_constant<int, 32>{}, 32);
  halve(std::integral_constant<int, 16>{}, 16);
  halve(std::integral_constant<int, 8>{}, 8);
  halve(std::integral_constant<int, 4>{}, 4);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < p.units / 2) {
      const int at = first + i;
      s_dw[wave][(at >> 4) * p.d + channel_of<INTER>(at & 15, a.unit, p.rot, p.d)] = dw[i];
    }
  __syncthreads();
  const size_t group = (size_t)blockIdx.y * gridDim.x + blockIdx.x;
  for (int i = threadIdx.x; i < 2 * p.d; i += 256) p.q.part[group * 2 * p.d + i] = (s_dw[0][i] + s_dw[1][i]) + (s_dw[2][i] + s_dw[3][i]);
}

// The weights' gradients from the workgroups' sums: 32 channels a workgroup, every 32nd workgroup's sum a thread.
__global__ void __launch_bounds__(1024) k_weight_grad(const float* part, int groups, int d, float* dqw, float* dkw) {
  __shared__ double s_sum[32][33];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5, at = blockIdx.x * 32 + c;
  double sum = 0.0;
#pragma unroll 16
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
  if (((long long)a.B * a.N + 3) / 4 * 256 > MAX_THREADS) return SAGE_ERR_UNSUPPORTED;      // (a workgroup takes four tokens at least)
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

// What the kernels take, but for the tensors' pointers; the widest access that every row allows, and the grid (of at most `most` workgroups, if that is not 0).
constexpr long long PAST_BYTES = 192LL << 20;
struct NormLaunch { dim3 grid; int vw; bool inter, past; };
void plan(NormParams* p, NormLaunch* l, const NormShape& a, const NormView* v, int count, int most) {
  unsigned long long rows = 0;
  for (int i = 0; i < count; ++i) if (v[i].at) rows |= (uintptr_t)v[i].at / 2 | (unsigned long long)(v[i].st[0] | v[i].st[1] | v[i].st[2]);
  l->inter = a.interleaved != 0;
  const unsigned long long bits = rows | (l->inter ? 0ull : (unsigned long long)(a.rot / 2));
  l->vw = (bits & 7) == 0 ? 8 : (bits & 3) == 0 ? 4 : 1;
  p->inv_freq = a.inv_freq; p->positions = a.positions; p->pos_sb = a.pos_sb; p->offset = a.offset;
  p->tokens = (unsigned)(a.B * (long long)a.N); p->d = a.d; p->rot = a.rot; p->units = a.d / 16;
  p->weight_same = a.weight_type == SAGE_WEIGHT_SAME;
  p->eps = a.eps; p->scale = a.scale == 0.0f ? 1.0f : a.scale;
  // A workgroup's 256 threads are 4 tokens, or more where there are few heads.
  const int heads = a.H + (a.keys ? a.Hkv : 0), rows_of = 256 / p->units;
  p->lanes = 1;
  while (p->lanes * 2 <= rows_of / 4 && p->lanes * 2 <= heads) p->lanes *= 2;
  // (Backward: half as many where the workgroups' last round would be near empty: 24 x 98 tokens of 60 heads of 128, 588 groups of 4 for 512 workgroups 36.6 us, 1176 of 2 33.8.)
  if (most > 0) {
    const long long groups = ((long long)p->tokens * p->lanes + rows_of - 1) / rows_of;
    if (groups > most && 4 * ((groups + most - 1) / most) * most > 5 * groups && p->lanes * 2 <= rows_of && p->lanes * 2 <= heads) p->lanes *= 2;
  }
  p->at_once = rows_of / p->lanes;
  // Reads and writes pass the caches by where every access is whole lines of 128 bytes and what is read and written is most of the 256 MB of the memory-side cache: 4 x 4096 tokens of 40 heads
  // of 128 61.8 us, through the caches 71.9; the gradient of 2 x 4096 63.9 and 68.7 when it was taken, of 3001 tokens of 32 heads of 64, in pieces of lines, 25.6 and 22.8.
  const bool whole_lines = l->vw == 8 && (rows & 63) == 0 && (l->inter ? a.d % 128 == 0 : a.rot % 128 == 0 && a.d % 128 == 0);
  l->past = whole_lines && (most > 0 ? 6LL : 4LL) * p->tokens * heads * a.d > PAST_BYTES;
  p->heads_first = v[0].st[1] < v[0].st[2];       // (token-major: a token's heads are one stretch of memory)
  const long long groups = ((long long)p->tokens + p->at_once - 1) / p->at_once;
  const long long wide = most > 0 ? std::min(groups, (long long)most) : groups;
  const long long pieces = std::max(1LL, std::min((most > 0 ? most : 1024) / wide, (long long)heads / p->lanes));
  p->hchunk = (int)((heads + pieces - 1) / pieces);
  l->grid = dim3((unsigned)wide, (unsigned)((heads + p->hchunk - 1) / p->hchunk));
  p->by_n = fast_div(a.N); p->by_pairs = fast_div(a.rot > 0 ? a.rot / 2 : 1); p->by_lanes = fast_div(p->lanes); p->by_at_once = fast_div(p->at_once);
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
  plan(&p, &l, sh, v, 4, 0);
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
  plan(&p, &l, sh, v, 6, BWD_GROUPS);
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
