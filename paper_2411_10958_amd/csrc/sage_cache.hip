// Eviction from a key / value cache (sage_cache_evict).
#include "sage_attn.h"
#include "sage_ops.h"

#include <algorithm>

namespace sage {
namespace {

struct EvictParams {
  const unsigned short *k, *v;
  const float* w;
  const int* lens;
  unsigned short *k_out, *v_out;
  float* w_out;
  int *kept, *lens_out;
  int Hkv, N, keep, room, sink, recent, clear;
  int heads, d;                  // B H_kv
  TensorMap in, out;
};

// A weight as an unsigned number of the same order: NaN below everything, -0 with +0.
__device__ __forceinline__ unsigned order_of(float w) {
  const unsigned u = __float_as_uint(w + 0.0f);
  const unsigned k = (u >> 31) ? ~u : u | 0x80000000u;
  return w == w ? k : 0u;
}

constexpr int SEL_THREADS = 1024, SEL_WAVES = SEL_THREADS / 64;
constexpr int SMALL_K = 4, SMALL_ROWS = 32768;        // of the kernel that copies rows too: 64s of a wavefront, elements of K for a workgroup
constexpr int DIGIT = 11, BINS = 1 << DIGIT;      // three digits of 11, 11 and 10 bits

// Which tokens stay, one workgroup per sequence and KV head: the m-th largest weight between sink and recent, found digit by digit by
// counting, then one pass in order that keeps what is larger and the first of what equals it.  A wavefront has a stretch of
// 64 K weights in registers, in the order of unsigned numbers, so they are read and converted once; K = 0: more than that, read
// again each time, eight loads in flight.  Bound by the instructions of its five passes on one CU: 32 rows of 32768 20 us of the call's
// 107 (51 with 8-bit digits and weights read from memory in each pass; counts in four copies changed nothing).  (The first digit is sign, exponent and two bits: with 8-bit digits a wavefront's
// counts would fall on a dozen addresses.)  What a stretch has behind the last weight counts as less than any and comes after
// all, so it is never taken: n > m.
template <int K> __device__ __forceinline__ int select_tokens(const EvictParams& p) {
  __shared__ unsigned s_hist[BINS];
  __shared__ unsigned s_wave[SEL_WAVES], s_pick[2];
  __shared__ unsigned s_gt[SEL_WAVES], s_eq[SEL_WAVES];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int b = blockIdx.x / p.Hkv;
  const int len = p.lens ? min(max(p.lens[b], 0), p.N) : p.N;
  const float* w = p.w + (size_t)blockIdx.x * p.N;
  int* kept = p.kept + (size_t)blockIdx.x * p.keep;
  if (t == 0 && blockIdx.x % p.Hkv == 0) p.lens_out[b] = min(len, p.keep);
  if (len <= p.keep) {
    for (int i = t; i < len; i += SEL_THREADS) kept[i] = i;
    return len;
  }
  const int c0 = p.sink, n = len - p.recent - p.sink, m = p.keep - p.sink - p.recent;     // n > m >= 0 tokens to choose from
  constexpr int STEP = K > 0 ? K : 8;             // 64s that a wavefront has at a time
  const int seg = K > 0 ? 64 * K : ((n + SEL_WAVES - 1) / SEL_WAVES + 63) / 64 * 64;
  const int i0 = min(wave * seg, n), i1 = min(i0 + seg, n);
  unsigned u[STEP];
  auto load = [&](int from) __attribute__((always_inline)) {
    constexpr int PART = STEP < 32 ? STEP : 32;   // loads in flight (64 at once would leave no registers for the weights)
#pragma unroll
    for (int j0 = 0; j0 < STEP; j0 += PART) {
      float x[PART];
#pragma unroll
      for (int j = 0; j < PART; ++j) x[j] = from + 64 * (j0 + j) < i1 ? w[c0 + min(from + 64 * (j0 + j) + lane, i1 - 1)] : 0.0f;
#pragma unroll
      for (int j = 0; j < PART; ++j) u[j0 + j] = from + 64 * (j0 + j) + lane < i1 ? order_of(x[j]) : 0u;
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (K > 0) load(i0);
  for (int i = t; i < p.sink; i += SEL_THREADS) kept[i] = i;
  for (int i = t; i < p.recent; i += SEL_THREADS) kept[p.keep - p.recent + i] = len - p.recent + i;
  if (m == 0) return p.keep;
  // f(weights in order, first token) for the 64s of my stretch
  auto each = [&](auto f) __attribute__((always_inline)) {
    for (int i = i0; i < i1; i += 64 * STEP) {
      if (K == 0) load(i);
#pragma unroll
      for (int j = 0; j < STEP; ++j)
        if (i + 64 * j < i1) {
          unsigned v = u[j];
          // (What the compiler knows of a weight it would keep from one pass to the next, masks of 64 lanes for each and more than there are
          // registers for.  Us, with that kept / this: 32 rows of 30000 25.6 / 23.2, of 50000 44.6 / 32.9.)
          if (K > 16) asm volatile("" : "+v"(v));
          f(v, i + 64 * j);
        }
    }
  };
  unsigned prefix = 0, need = (unsigned)m;
#pragma unroll
  for (int d = 0; d < 3; ++d) {
    const int low = d == 0 ? 32 - DIGIT : d == 1 ? 32 - 2 * DIGIT : 0, bits = d < 2 ? DIGIT : 32 - 2 * DIGIT;
    for (int i = t; i < BINS; i += SEL_THREADS) s_hist[i] = 0;
    __syncthreads();
    each([&](unsigned v, int) __attribute__((always_inline)) {
      if (d == 0 || (v >> (low + bits)) == (prefix >> (low + bits))) atomicAdd(&s_hist[(v >> low) & ((1u << bits) - 1)], 1u);
    });
    __syncthreads();
    // thread t holds digits 2047 - 2t and 2046 - 2t: from the largest down
    const unsigned a0 = s_hist[BINS - 1 - 2 * t], a1 = s_hist[BINS - 2 - 2 * t];
    unsigned upto = a0 + a1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const unsigned y = __shfl_up(upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    for (int i = 0; i < wave; ++i) upto += s_wave[i];
    const unsigned before = upto - a0 - a1;
    if (before < need && upto >= need) {
      const bool second = before + a0 < need;
      s_pick[0] = (unsigned)(BINS - 1 - 2 * t) - second;
      s_pick[1] = before + (second ? a0 : 0u);
    }
    __syncthreads();
    prefix |= s_pick[0] << low;
    need -= s_pick[1];
  }
  unsigned gt = 0, eq = 0;
  each([&](unsigned v, int) __attribute__((always_inline)) {
    gt += (unsigned)__popcll(__ballot(v > prefix));
    eq += (unsigned)__popcll(__ballot(v == prefix));
  });
  if (lane == 0) { s_gt[wave] = gt; s_eq[wave] = eq; }
  __syncthreads();
  unsigned above = (unsigned)p.sink, ties = 0;
  for (int i = 0; i < wave; ++i) { above += s_gt[i]; ties += s_eq[i]; }
  // (lanes of a mask before mine, counted from c on)
  auto place = [](unsigned long long mask, unsigned c) __attribute__((always_inline)) {
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, c));
  };
  each([&](unsigned v, int i) __attribute__((always_inline)) {
    const unsigned long long bg = __ballot(v > prefix), be = __ballot(v == prefix);
    if (be == 0) {
      if (v > prefix) kept[place(bg, above + min(ties, need))] = c0 + i + lane;
    } else {
      const unsigned tie = place(be, ties);
      if (v > prefix || (v == prefix && tie < need)) kept[place(bg, above) + min(tie, need)] = c0 + i + lane;
      ties += (unsigned)__popcll(be);
    }
    above += (unsigned)__popcll(bg);
  });
  return p.keep;
}

// Place `at` behind what head bh keeps: its weight, and which token it would be.
__device__ __forceinline__ void clear_place(const EvictParams& p, unsigned bh, int at) {
  if (p.w_out) p.w_out[(size_t)bh * p.room + at] = 0.0f;
  if (at < p.keep) p.kept[(size_t)bh * p.keep + at] = 0;
}

// Zeros in the places of the outputs behind what is kept, by workgroup z of n: stretches of CLEAR values of K and as many of V.
constexpr int CLEAR = 32768;
__device__ __forceinline__ void clear_places(const EvictParams& p, unsigned z, unsigned n) {
  const int per = CLEAR / p.d, row = 31 - __builtin_clz((unsigned)p.d / 8);      // places of a stretch, log2(pieces of a row)
  const unsigned stretches = (unsigned)((p.room + per - 1) / per);
  for (unsigned long long s = z; s < (unsigned long long)stretches * p.heads; s += n) {
    const unsigned bh = (unsigned)(s / stretches);
    const int b = (int)bh / p.Hkv, len = p.lens ? min(max(p.lens[b], 0), p.N) : p.N, at = (int)(s - (unsigned long long)bh * stretches) * per;
    const int from = max(at, min(len, p.keep)), to = min(at + per, p.room);
    if (from >= to) continue;
    const size_t ho = head_offset(p.out, bh);
    for (int i = from + (int)threadIdx.x; i < to; i += SEL_THREADS) clear_place(p, bh, i);
    for (int i = (int)threadIdx.x; i < (to - from) << row; i += SEL_THREADS) {
      const size_t x = row_offset(p.out, ho, from + (i >> row)) + 8 * (i & ((1 << row) - 1));
      *reinterpret_cast<v4i*>(p.k_out + x) = v4i{0, 0, 0, 0};
      *reinterpret_cast<v4i*>(p.v_out + x) = v4i{0, 0, 0, 0};
    }
  }
}

// Workgroups: one to a row; where `clear` is set, more that write the zeros, while the rows' have the memory to themselves.  (Us, outputs of the
// caches' size filled before the call / this / zeros by the kernel that moves the rows: 32 heads of 32768 tokens of 128 cut to half 198 / 128 / 138, of
// 8192 62 / 40 / 44, 16 of 100000 cut to a fifth 270 / 227 / 291.)
template <int K> __global__ void __launch_bounds__(SEL_THREADS) k_evict_select(const EvictParams p) {
  if (blockIdx.x < (unsigned)p.heads) select_tokens<K>(p);
  else clear_places(p, blockIdx.x - (unsigned)p.heads, gridDim.x - (unsigned)p.heads);
}

// The same, and the rows too: one launch, where a row's workgroup has at most 4096 weights and 64 KB of K and as much of V (us, two launches /
// this: 4 heads cut to 256 tokens of 64 14.7 / 11.5, of 128 14.2 / 11.3; 32 heads cut to 1000 of 64, 128 KB, 15.0 / 19.5).
template <int D> __global__ void __launch_bounds__(SEL_THREADS) k_evict_small(const EvictParams p) {
  constexpr int P = D / 8, U = 4;                 // pieces of a row, those in flight
  const int there = select_tokens<SMALL_K>(p);
  __syncthreads();                                // (the indices, which this workgroup wrote, are read from memory)
  const int* kept = p.kept + (size_t)blockIdx.x * p.keep;
  const size_t hi = head_offset(p.in, blockIdx.x), ho = head_offset(p.out, blockIdx.x);
  if (p.w_out)
    for (int i = threadIdx.x; i < there; i += SEL_THREADS) p.w_out[(size_t)blockIdx.x * p.room + i] = p.w[(size_t)blockIdx.x * p.N + kept[i]];
  for (int i = threadIdx.x; i < there * P; i += SEL_THREADS * U) {
    v4i a[U], x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = min(i + u * SEL_THREADS, there * P - 1);
      const size_t from = row_offset(p.in, hi, kept[at / P]) + 8 * (at % P);
      a[u] = *reinterpret_cast<const v4i*>(p.k + from);
      x[u] = *reinterpret_cast<const v4i*>(p.v + from);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = i + u * SEL_THREADS;
      if (at >= there * P) break;
      const size_t to = row_offset(p.out, ho, at / P) + 8 * (at % P);
      *reinterpret_cast<v4i*>(p.k_out + to) = a[u];
      *reinterpret_cast<v4i*>(p.v_out + to) = x[u];
    }
  }
  if (!p.clear) return;
  for (int i = threadIdx.x; i < (p.room - there) * P; i += SEL_THREADS) {
    const int at = there + i / P;
    const size_t to = row_offset(p.out, ho, at) + 8 * (i % P);
    *reinterpret_cast<v4i*>(p.k_out + to) = v4i{0, 0, 0, 0};
    *reinterpret_cast<v4i*>(p.v_out + to) = v4i{0, 0, 0, 0};
    if (i % P == 0) clear_place(p, blockIdx.x, at);
  }
}

// The rows of the kept tokens, and their weights: a thread moves 16 bytes of K and of V of GU tokens, the first of a row also its
// weight.  Reads pass the caches by, since the old rows are not needed again; with PAST writes do too, where rows read and written do not fit
// the 256 MB of the memory-side cache (32 heads of 32768 tokens of 128 cut to half: the call, with 22 us of selection, 123 us with both kept, 120 with reads past,
// 111 with both, 5.4 TB/s; with the decode step that reads the rows after it 174 either way).  Below that the step finds rows there (32
// heads of 8000 cut to half, and the step: 54.9, 57.4 with writes past).
// Grid: (pieces of the kept tokens, heads).
constexpr int GU = 4;
template <int D, bool PAST> __global__ void __launch_bounds__(256) k_evict_rows(const EvictParams p) {
  constexpr int P = D / 8, TOK = 256 / P;
  const int b = blockIdx.y / p.Hkv;
  const int len = p.lens ? min(max(p.lens[b], 0), p.N) : p.N, there = min(len, p.keep);
  const int first = blockIdx.x * (TOK * GU) + threadIdx.x / P;
  if (first >= there) return;
  const int c = 8 * (threadIdx.x % P);
  const int* kept = p.kept + (size_t)blockIdx.y * p.keep;
  const size_t hi = head_offset(p.in, blockIdx.y) + c, ho = head_offset(p.out, blockIdx.y) + c;
  int from[GU];
#pragma unroll
  for (int i = 0; i < GU; ++i) from[i] = kept[min(first + i * TOK, there - 1)];
  v4i a[GU], x[GU];
  float wt[GU];
  const bool weigh = p.w_out && c == 0;
#pragma unroll
  for (int i = 0; i < GU; ++i) wt[i] = weigh ? p.w[(size_t)blockIdx.y * p.N + from[i]] : 0.0f;
#pragma unroll
  for (int i = 0; i < GU; ++i) {
    const size_t at = row_offset(p.in, hi, from[i]);
    a[i] = __builtin_nontemporal_load(reinterpret_cast<const v4i*>(p.k + at));
    x[i] = __builtin_nontemporal_load(reinterpret_cast<const v4i*>(p.v + at));
  }
#pragma unroll
  for (int i = 0; i < GU; ++i) {
    if (first + i * TOK < there) {
      const size_t at = row_offset(p.out, ho, first + i * TOK);
      v4i *ka = reinterpret_cast<v4i*>(p.k_out + at), *va = reinterpret_cast<v4i*>(p.v_out + at);
      if (PAST) {
        __builtin_nontemporal_store(a[i], ka);
        __builtin_nontemporal_store(x[i], va);
      } else {
        *ka = a[i];
        *va = x[i];
      }
      if (weigh) p.w_out[(size_t)blockIdx.y * p.room + first + i * TOK] = wt[i];
    }
  }
}

template <int D> void launch_rows(const EvictParams& p, bool past, dim3 grid, hipStream_t s) {
  if (past) k_evict_rows<D, true><<<grid, 256, 0, s>>>(p);
  else k_evict_rows<D, false><<<grid, 256, 0, s>>>(p);
}

}  // namespace
}  // namespace sage

using namespace sage;

extern "C" int sage_cache_evict(const sage_cache_evict_args* a) {
  if (!a || a->B <= 0 || a->H_kv <= 0 || a->N_kv <= 0 || a->N_keep <= 0 || a->sink < 0 || a->recent < 0) return SAGE_ERR_INVALID_ARG;
  if ((a->clear & ~1) != 0) return SAGE_ERR_UNSUPPORTED;
  const int room = a->N_out == 0 ? a->N_keep : a->N_out;
  if ((long long)a->sink + a->recent > a->N_keep || room < a->N_keep) return SAGE_ERR_INVALID_ARG;
  if (!a->k || !a->v || !a->weights || !a->k_out || !a->v_out || !a->kept || !a->lens_out) return SAGE_ERR_INVALID_ARG;
  if (a->d != 64 && a->d != 128 && a->d != 256) return SAGE_ERR_UNSUPPORTED;
  if (a->dtype != SAGE_DT_FP16 && a->dtype != SAGE_DT_BF16) return SAGE_ERR_UNSUPPORTED;
  if (a->layout != SAGE_LAYOUT_HND && a->layout != SAGE_LAYOUT_NHD) return SAGE_ERR_UNSUPPORTED;
  if (a->N_kv > MAX_TOKENS || room > MAX_TOKENS || (long long)a->B * a->H_kv > 65535) return SAGE_ERR_UNSUPPORTED;
  if ((((uintptr_t)a->k | (uintptr_t)a->v | (uintptr_t)a->k_out | (uintptr_t)a->v_out) & 15u) != 0) return SAGE_ERR_INVALID_ARG;
  if ((((uintptr_t)a->weights | (uintptr_t)a->weights_out | (uintptr_t)a->kept | (uintptr_t)a->lens_out | (uintptr_t)a->kv_lens) & 3u) != 0)
    return SAGE_ERR_INVALID_ARG;
  const size_t heads = (size_t)a->B * a->H_kv, rows = heads * a->N_kv, out_rows = heads * room;
  const Span in[4] = {{a->k, rows * a->d * 2}, {a->v, rows * a->d * 2}, {a->weights, rows * 4}, {a->kv_lens, (size_t)a->B * 4}};
  const Span out[5] = {{a->k_out, out_rows * a->d * 2}, {a->v_out, out_rows * a->d * 2}, {a->weights_out, out_rows * 4}, {a->kept, heads * a->N_keep * 4},
                       {a->lens_out, (size_t)a->B * 4}};
  for (int i = 0; i < 5; ++i) {
    for (const Span& s : in) if (overlap(out[i], s)) return SAGE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j) if (overlap(out[i], out[j])) return SAGE_ERR_INVALID_ARG;
  }
  EvictParams p;
  p.k = (const unsigned short*)a->k; p.v = (const unsigned short*)a->v; p.w = a->weights; p.lens = a->kv_lens;
  p.k_out = (unsigned short*)a->k_out; p.v_out = (unsigned short*)a->v_out; p.w_out = a->weights_out; p.kept = a->kept; p.lens_out = a->lens_out;
  p.Hkv = a->H_kv; p.N = a->N_kv; p.keep = a->N_keep; p.room = room; p.sink = a->sink; p.recent = a->recent; p.clear = a->clear;
  p.heads = (int)heads; p.d = a->d;
  const int nhd = a->layout == SAGE_LAYOUT_NHD;
  p.in = make_tensor_map(nhd, a->H_kv, a->N_kv, a->d);
  p.out = make_tensor_map(nhd, a->H_kv, room, a->d);
  const hipStream_t s = (hipStream_t)a->stream;
  const int most = a->N_kv - a->sink - a->recent;       // weights to choose from
  const long long moved = std::min(a->N_keep, a->N_kv), places = a->clear ? room : moved;       // tokens of a head, at most; those written
  if (most <= SMALL_K * 64 * SEL_WAVES && places * a->d <= SMALL_ROWS) {
    if (a->d == 64) k_evict_small<64><<<(unsigned)heads, SEL_THREADS, 0, s>>>(p);
    else if (a->d == 128) k_evict_small<128><<<(unsigned)heads, SEL_THREADS, 0, s>>>(p);
    else k_evict_small<256><<<(unsigned)heads, SEL_THREADS, 0, s>>>(p);
    return op_status(hipGetLastError());
  }
  const long long stretches = p.clear ? (long long)heads * ((room + CLEAR / a->d - 1) / (CLEAR / a->d)) : 0;
  const unsigned groups = (unsigned)(heads + std::min(stretches, 2048LL));
  if (most <= 4 * SEL_THREADS) k_evict_select<4><<<groups, SEL_THREADS, 0, s>>>(p);
  else if (most <= 16 * SEL_THREADS) k_evict_select<16><<<groups, SEL_THREADS, 0, s>>>(p);
  else if (most <= 32 * SEL_THREADS) k_evict_select<32><<<groups, SEL_THREADS, 0, s>>>(p);
  else if (most <= 64 * SEL_THREADS) k_evict_select<64><<<groups, SEL_THREADS, 0, s>>>(p);
  else k_evict_select<0><<<groups, SEL_THREADS, 0, s>>>(p);
  int st = op_status(hipGetLastError());
  if (st != SAGE_OK) return st;
  const int per = 256 / (a->d / 8) * GU;
  const dim3 grid((unsigned)((moved + per - 1) / per), (unsigned)heads);
  const bool past = 8LL * (long long)heads * moved * a->d > 256LL << 20;
  if (a->d == 64) launch_rows<64>(p, past, grid, s);
  else if (a->d == 128) launch_rows<128>(p, past, grid, s);
  else launch_rows<256>(p, past, grid, s);
  return op_status(hipGetLastError());
}
