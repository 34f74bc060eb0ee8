// Attention over a cache of 8 bits and pages (sage_attn_paged).
//
// O = softmax(kappa Q K^T) V with K = codes 2^ek, V = codes 2^ev, one exponent for each block of 32 tokens.  One wavefront per query: a block's 32
// scores at a time, half of the channels in each half of the lanes, then its 32 weights times V, a few channels in each lane.
#include "sage_paged.h"

#include <algorithm>

namespace sage {
namespace {

struct PagedParams {
  PagedCache c;
  const unsigned short* q;
  unsigned short* out;
  float* lse;
  const int *lens, *qlens;
  TensorMap qm;
  int B, H, N, G, cap;               // cap: max_pages * page
  int causal, window, sink;
  float kappa;                       // sm_scale log2(e)
};

// The tokens that query r sees: t < sink and from <= t < to.
struct Seen { int sink, from, to; };
__device__ __forceinline__ Seen seen_by(const PagedParams& p, int len, int count, int r) {
  const int pos = max(len - count, 0) + r;
  Seen s;
  s.to = p.causal ? min(len, pos + 1) : len;
  s.from = p.window > 0 ? max(pos + 1 - p.window, 0) : 0;
  s.sink = p.window > 0 ? min(p.sink, s.to) : 0;
  return s;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(64) k_paged(const PagedParams p) {
  constexpr int C = D / 64;
  __shared__ float s_q[D];
  const int lane = threadIdx.x, col = lane & 31, half = lane >> 5;
  const int r = blockIdx.x, h = blockIdx.y % p.H, b = blockIdx.y / p.H, hkv = h / p.G;
  const int len = p.lens ? min(max(p.lens[b], 0), p.cap) : p.cap, count = p.qlens ? min(max(p.qlens[b], 0), p.N) : p.N;
  if (r >= count) return;
  const Seen s = seen_by(p, len, count, r);
  const size_t row = row_offset(p.qm, head_offset_of(p.qm, b, h), r);
  for (int c = lane; c < D; c += 64) s_q[c] = load16<BF16>(p.q[row + c]);
  __syncthreads();
  float m = -INFINITY, l = 0.0f, o[C] = {};
  for (int i = 0; i * BLOCK < s.to; ++i) {
    const int t0 = i * BLOCK;
    if (t0 >= s.sink && t0 + BLOCK <= s.from) continue;
    const long long at = pool_block(p.c, b, hkv, i);
    if (at < 0) continue;
    const unsigned* kr = reinterpret_cast<const unsigned*>(p.c.k + ((size_t)at * BLOCK + col) * D + half * (D / 2));
    float x = 0.0f;
    for (int c = 0; c < D / 8; ++c) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)kr[c], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)kr[c], true);
      const float* q = s_q + half * (D / 2) + 4 * c;
      x += lo[0] * q[0] + lo[1] * q[1] + hi[0] * q[2] + hi[1] * q[3];
    }
    x = half_sum(x) * (p.kappa * scale_of(p.c.ks[at]));
    const int t = t0 + col;
    const bool see = t < s.to && (t >= s.from || t < s.sink);
    x = see ? x : -INFINITY;
    float top = x;
#pragma unroll
    for (int y = 16; y > 0; y >>= 1) top = fmaxf(top, __shfl_xor(top, y));
    const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.0f : m_new, alpha = exp2f(m - base);
    const float e = see ? exp2f(x - base) : 0.0f;
    float sum = e;
#pragma unroll
    for (int y = 16; y > 0; y >>= 1) sum += __shfl_xor(sum, y);
    l = l * alpha + sum;
    m = m_new;
    const float vs = scale_of(p.c.vs[at]);
    for (int c = 0; c < C; ++c) o[c] *= alpha;
    for (int k = 0; k < BLOCK; ++k) {
      if (!__shfl((int)see, k)) continue;
      const float w = __shfl(e, k) * vs;
      const unsigned char* v = p.c.v + ((size_t)at * BLOCK + k) * D + lane * C;
      for (int c = 0; c < C; ++c) o[c] += w * __builtin_amdgcn_cvt_f32_fp8((int)v[c], 0);
    }
  }
  const bool none = m == -INFINITY && l == 0.0f;
  const float inv = none ? 0.0f : 1.0f / l;
  for (int c = 0; c < C; ++c) p.out[row + lane * C + c] = (unsigned short)pack16x2<BF16>(o[c] * inv, 0.0f);
  if (p.lse && lane == 0) p.lse[((size_t)b * p.H + h) * p.N + r] = none ? -INFINITY : LN2 * (m + log2f(l));
}

int paged_params(const sage_attn_paged_args* a, PagedParams* p, bool need_io) {
  if (!a || a->H <= 0 || a->N <= 0) return SAGE_ERR_INVALID_ARG;
  const int st = cache_shape(&p->c, a->B, a->H_kv, a->d, a->n_pages, a->page, a->max_pages);
  if (st != SAGE_OK) return st;
  if (a->H % a->H_kv != 0 || a->window < 0 || a->sink < 0 || (a->causal & ~1) != 0 || (a->window > 0 && !a->causal)) return SAGE_ERR_INVALID_ARG;
  if (a->dtype != SAGE_DT_FP16 && a->dtype != SAGE_DT_BF16) return SAGE_ERR_UNSUPPORTED;
  if (a->layout != SAGE_LAYOUT_HND && a->layout != SAGE_LAYOUT_NHD) return SAGE_ERR_UNSUPPORTED;
  if (a->N > MAX_TOKENS || (long long)a->B * a->H > 65535 || (long long)a->B * a->H * a->N > 1LL << 24) return SAGE_ERR_UNSUPPORTED;
  if (need_io) {
    if (!a->q || !a->out || (((uintptr_t)a->q | (uintptr_t)a->out) & 15u) != 0) return SAGE_ERR_INVALID_ARG;
    if ((((uintptr_t)a->lse | (uintptr_t)a->kv_lens | (uintptr_t)a->q_lens) & 3u) != 0) return SAGE_ERR_INVALID_ARG;
    const int io = cache_arrays(&p->c, a->k_cache, a->v_cache, a->k_scale, a->v_scale, a->page_table);
    if (io != SAGE_OK) return io;
  }
  p->q = (const unsigned short*)a->q; p->out = (unsigned short*)a->out; p->lse = a->lse; p->lens = a->kv_lens; p->qlens = a->q_lens;
  p->qm = make_tensor_map(a->layout == SAGE_LAYOUT_NHD, a->H, a->N, a->d);
  p->B = a->B; p->H = a->H; p->N = a->N; p->G = a->H / a->H_kv; p->cap = a->max_pages * a->page;
  p->causal = a->causal; p->window = std::min(a->window, MAX_TOKENS * 2); p->sink = std::min(a->sink, MAX_TOKENS);
  p->kappa = (a->sm_scale > 0.0f ? a->sm_scale : (float)(1.0 / std::sqrt((double)a->d))) * LOG2E;
  return SAGE_OK;
}

template <int D> void launch(const PagedParams& p, bool bf16, hipStream_t s) {
  const dim3 grid((unsigned)p.N, (unsigned)(p.B * p.H));
  if (bf16) k_paged<D, true><<<grid, 64, 0, s>>>(p);
  else k_paged<D, false><<<grid, 64, 0, s>>>(p);
}

}  // namespace
}  // namespace sage

using namespace sage;

extern "C" size_t sage_attn_paged_workspace_bytes(const sage_attn_paged_args* a) {
  PagedParams p;
  if (paged_params(a, &p, false) != SAGE_OK) return 0;
  return 0;
}

extern "C" int sage_attn_paged(const sage_attn_paged_args* a) {
  PagedParams p;
  const int st = paged_params(a, &p, true);
  if (st != SAGE_OK) return st;
  const size_t rows = (size_t)a->B * a->H * a->N, blocks = cache_blocks(p.c), bytes = blocks * BLOCK * a->d, need = 0;
  if (need > 0 && (!a->workspace || a->workspace_bytes < need || ((uintptr_t)a->workspace & 255u) != 0)) return SAGE_ERR_WORKSPACE;
  // (a row's query is read before its output is written, by the same workgroup or a kernel before: out may be q)
  const Span in[8] = {{a->out == a->q ? nullptr : a->q, rows * a->d * 2}, {a->k_cache, bytes}, {a->v_cache, bytes}, {a->k_scale, blocks}, {a->v_scale, blocks},
                      {a->page_table, (size_t)a->B * a->max_pages * 4}, {a->kv_lens, (size_t)a->B * 4}, {a->q_lens, (size_t)a->B * 4}};
  const Span out[3] = {{a->out, rows * a->d * 2}, {a->lse, rows * 4}, {need > 0 ? a->workspace : nullptr, need}};
  for (int i = 0; i < 3; ++i) {
    for (const Span& x : in) if (overlap(out[i], x)) return SAGE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j) if (overlap(out[i], out[j])) return SAGE_ERR_INVALID_ARG;
  }
  const hipStream_t s = (hipStream_t)a->stream;
  const bool bf16 = a->dtype == SAGE_DT_BF16;
  if (a->d == 64) launch<64>(p, bf16, s);
  else if (a->d == 128) launch<128>(p, bf16, s);
  else launch<256>(p, bf16, s);
  return op_status(hipGetLastError());
}
