// New tokens into a cache of 8 bits and pages (sage_cache_append).
//
// A block of 32 tokens of a page and KV head has one scale 2^(byte - 127), the smallest power of two with max |x| <= 448 scale: with
// max |x| = 1.m 2^E and 448 = 1.75 2^8 that is 2^(E - 8), one more where 1.m > 1.75.  x / scale is exact in FP32, so the code is x / scale
// correctly rounded, whatever computes it.
// One wavefront takes one block's new tokens (up to 32 rows, held in registers between the maximum and the codes) of K or of V: every value is read once.  Bound by memory: 2 x 8192 tokens of
// 8 heads of 128 24.7 us, 4.1 TB/s with a start of some 4 us (26.4 with each value scaled, cut and converted in FP32, as it still is where something has to be cut).
#include "sage_paged.h"
#include "sage_quant.h"
#include "sage_rows.h"

#include <algorithm>

namespace sage {
namespace {

struct AppendTensor {
  const unsigned short* x;
  long long sb, sh, sn;
};
struct AppendParams {
  AppendTensor k, v;
  PagedCache c;
  const int *lens, *news;
  int N, most, cap;              // cap: max_pages * page; most: largest scale byte
  int heads_first;               // which runs faster over the workgroups, heads or blocks
  long long items;               // B * blocks * H_kv
  FastDiv by_hkv, by_blocks;
};

// Four values (two dwords) as codes: divided by the scale, rounded to the nearest, all in one instruction for two.
template <bool BF16> __device__ __forceinline__ unsigned codes_of(unsigned a, unsigned b, float scale) {
  typedef short v2s __attribute__((ext_vector_type(2)));
  v2s r = {0, 0};
  if constexpr (BF16) {
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(v2b, a), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(v2b, b), scale, true);
  } else {
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(v2h, a), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(v2h, b), scale, true);
  }
  return __builtin_bit_cast(unsigned, r);
}

template <bool BF16, int D, bool WIDE>
__global__ void __launch_bounds__(256) k_append(const AppendParams p) {
  constexpr int L = D / 8, R = 64 / L, STEPS = BLOCK / R;      // threads of a row, rows of a step
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned item = blockIdx.x * 4 + (unsigned)wave;
  if (item >= (unsigned)p.items) return;
  unsigned h, i, b = item;
  if (p.heads_first) {
    h = b; b = split_by(h, p.by_hkv);
    i = b; b = split_by(i, p.by_blocks);
  } else {
    i = b; b = split_by(i, p.by_blocks);
    h = b; b = split_by(h, p.by_hkv);
  }
  const bool values = blockIdx.y != 0;
  const int len = p.lens ? min(max(p.lens[b], 0), p.cap) : p.cap, count = p.news ? min(max(p.news[b], 0), p.N) : p.N;
  const int first = len - count, start = max(first, 0);        // (where first < 0 the sequence has room for the last ones only)
  const int t0 = start / BLOCK * BLOCK + BLOCK * (int)i, lo = max(t0, start), hi = min(t0 + BLOCK, len);
  if (lo >= hi) return;
  const long long at = pool_block(p.c, (int)b, (int)h, t0 / BLOCK);
  if (at < 0) return;
  const AppendTensor& t = values ? p.v : p.k;
  const unsigned short* x = t.x + (long long)b * t.sb + (long long)h * t.sh + 8 * (lane % L);
  unsigned v[STEPS][4];
  unsigned most = 0;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int tok = t0 + s * R + lane / L;
    v[s][0] = v[s][1] = v[s][2] = v[s][3] = 0;
    if (tok >= lo && tok < hi) {
      const unsigned short* row = x + (long long)(tok - first) * t.sn;
      if constexpr (WIDE) {
        const uint4 u = *reinterpret_cast<const uint4*>(row);
        v[s][0] = u.x; v[s][1] = u.y; v[s][2] = u.z; v[s][3] = u.w;
      } else {
#pragma unroll
        for (int y = 0; y < 4; ++y) v[s][y] = row[2 * y] | (unsigned)row[2 * y + 1] << 16;
      }
    }
  }
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
#pragma unroll
    for (int y = 0; y < 4; ++y) most = larger_pair(most, v[s][y] & 0x7fff7fff);
  most = largest_of_all(most);
  const bool finite = most < (BF16 ? 0x7f80u : 0x7c00u);
  if (!finite) {                                   // (the same, of what is finite)
    most = 0;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int y = 0; y < 4; ++y) most = larger_pair(most, finite_pair<BF16>(v[s][y]));
    most = largest_of_all(most);
  }
  const unsigned bits = __float_as_uint(load16<BF16>((unsigned short)most));
  const int fits = max((int)(bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0), 63);
  int e = min(fits, p.most);
  unsigned char* codes = (values ? p.c.v : p.c.k) + (size_t)at * (BLOCK * D) + 8 * (lane % L);
  unsigned char* scale = (values ? p.c.vs : p.c.ks) + at;
  if (lo > t0) {                                   // the block holds earlier tokens
    const int old = *scale;
    if (e > old || old == 255) {                   // (255 is NaN: so is all that the block holds, and stays)
      const float f = old == 255 ? NAN : e - old < 127 ? __uint_as_float((unsigned)(127 - (e - old)) << 23) : 0.0f;
#pragma unroll 1
      for (int s = 0; s < STEPS; ++s) {
        const int r = s * R + lane / L;
        if (t0 + r >= lo) break;
        unsigned* c = reinterpret_cast<unsigned*>(codes + (size_t)r * D);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[y], false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[y], true);
          int u = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * f, a[1] * f, 0, false);
          c[y] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(d[0] * f, d[1] * f, u, true);
        }
      }
    }
    e = max(e, old);
  }
  if (finite && e >= fits && e < 254) {            // nothing to cut
    const float two = scale_of((unsigned)e);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int r = s * R + lane / L;
      if (t0 + r < lo || t0 + r >= hi) continue;
      *reinterpret_cast<uint2*>(codes + (size_t)r * D) = make_uint2(codes_of<BF16>(v[s][0], v[s][1], two), codes_of<BF16>(v[s][2], v[s][3], two));
    }
  } else {
    const float inv = e == 255 ? NAN : e == 254 ? 0x1p-127f : __uint_as_float((unsigned)(254 - e) << 23);
    auto scaled = [&](unsigned u) {
      const float y = load16<BF16>((unsigned short)u) * inv;
      const float cut = fminf(fmaxf(y, -E4M3_MAX), E4M3_MAX);      // (of a NaN a number)
      return (u & 0x7fff) < (BF16 ? 0x7f80u : 0x7c00u) && y == y ? cut : NAN;
    };
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int r = s * R + lane / L;
      if (t0 + r < lo || t0 + r >= hi) continue;
      int u[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        u[y] = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(v[s][2 * y] & 0xffff), scaled(v[s][2 * y] >> 16), 0, false);
        u[y] = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(v[s][2 * y + 1] & 0xffff), scaled(v[s][2 * y + 1] >> 16), u[y], true);
      }
      *reinterpret_cast<uint2*>(codes + (size_t)r * D) = make_uint2((unsigned)u[0], (unsigned)u[1]);
    }
  }
  if (lane == 0) *scale = (unsigned char)e;
}

template <bool BF16, int D> void launch(const AppendParams& p, bool wide, dim3 grid, hipStream_t s) {
  if (wide) k_append<BF16, D, true><<<grid, 256, 0, s>>>(p);
  else k_append<BF16, D, false><<<grid, 256, 0, s>>>(p);
}
template <bool BF16> void launch(const AppendParams& p, int d, bool wide, dim3 grid, hipStream_t s) {
  if (d == 64) launch<BF16, 64>(p, wide, grid, s);
  else if (d == 128) launch<BF16, 128>(p, wide, grid, s);
  else launch<BF16, 256>(p, wide, grid, s);
}

}  // namespace
}  // namespace sage

using namespace sage;

extern "C" int sage_cache_append(const sage_cache_append_args* a) {
  if (!a || a->N <= 0) return SAGE_ERR_INVALID_ARG;
  AppendParams p;
  int st = cache_shape(&p.c, a->B, a->H_kv, a->d, a->n_pages, a->page, a->max_pages);
  if (st != SAGE_OK) return st;
  if (a->dtype != SAGE_DT_FP16 && a->dtype != SAGE_DT_BF16) return SAGE_ERR_UNSUPPORTED;
  if (a->layout != SAGE_LAYOUT_HND && a->layout != SAGE_LAYOUT_NHD) return SAGE_ERR_UNSUPPORTED;
  if (a->N > MAX_TOKENS) return SAGE_ERR_UNSUPPORTED;
  st = cache_arrays(&p.c, a->k_cache, a->v_cache, a->k_scale, a->v_scale, a->page_table);
  if (st != SAGE_OK) return st;
  if (!a->k || !a->v || (((uintptr_t)a->k | (uintptr_t)a->v) & 1u) != 0 || (((uintptr_t)a->kv_lens | (uintptr_t)a->new_lens) & 3u) != 0) return SAGE_ERR_INVALID_ARG;
  long long s[2][3];
  size_t span[2];
  const long long* given[2] = {a->k_strides, a->v_strides};
  unsigned long long rows = (uintptr_t)a->k / 2 | (uintptr_t)a->v / 2;
  for (int i = 0; i < 2; ++i) {
    if (!tensor_strides(given[i], a->layout, a->H_kv, a->N, a->d, s[i])) return SAGE_ERR_INVALID_ARG;
    const int extent[3] = {a->B, a->H_kv, a->N};
    span[i] = (size_t)a->d;
    for (int x = 0; x < 3; ++x) {
      if (extent[x] == 1) s[i][x] = 0;
      else if (s[i][x] > (1LL << 50) / (extent[x] - 1)) return SAGE_ERR_INVALID_ARG;      // (past any memory, and sums stay within 64 bits)
      span[i] += (size_t)s[i][x] * (extent[x] - 1);
      rows |= (unsigned long long)s[i][x];
    }
  }
  const size_t blocks = cache_blocks(p.c), bytes = blocks * BLOCK * a->d;
  const Span out[4] = {{a->k_cache, bytes}, {a->v_cache, bytes}, {a->k_scale, blocks}, {a->v_scale, blocks}};
  const Span in[5] = {{a->k, span[0] * 2}, {a->v, span[1] * 2}, {a->page_table, (size_t)a->B * a->max_pages * 4}, {a->kv_lens, (size_t)a->B * 4}, {a->new_lens, (size_t)a->B * 4}};
  for (int i = 0; i < 4; ++i) {
    for (const Span& x : in) if (overlap(out[i], x)) return SAGE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j) if (overlap(out[i], out[j])) return SAGE_ERR_INVALID_ARG;
  }
  p.k = {(const unsigned short*)a->k, s[0][0], s[0][1], s[0][2]};
  p.v = {(const unsigned short*)a->v, s[1][0], s[1][1], s[1][2]};
  p.lens = a->kv_lens; p.news = a->new_lens;
  p.N = a->N; p.cap = a->max_pages * a->page;
  p.most = a->dtype == SAGE_DT_BF16 ? 246 : 134;       // 448 2^119 and 448 2^7 are numbers of the type; twice that is not
  p.heads_first = s[0][1] < s[0][2];
  const int touched = (std::min(a->N, p.cap) + 2 * BLOCK - 2) / BLOCK;      // blocks of N tokens that start anywhere in one
  p.items = (long long)a->B * a->H_kv * touched;
  p.by_hkv = fast_div(a->H_kv); p.by_blocks = fast_div(touched);
  const long long groups = (p.items + 3) / 4;
  if (p.items > 0x7fffffff || groups * 256 > MAX_THREADS) return SAGE_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)groups, 2);
  const bool wide = (rows & 7) == 0;
  if (a->dtype == SAGE_DT_BF16) launch<true>(p, a->d, wide, grid, (hipStream_t)a->stream);
  else launch<false>(p, a->d, wide, grid, (hipStream_t)a->stream);
  return op_status(hipGetLastError());
}
