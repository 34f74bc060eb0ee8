// The attention weight that each key has received (sage_attn_key_weights).
//
// w_t = sum over rows r of 2^(kappa <q_r, k_t> - lse_r log2(e)): half of attention's products, and column sums instead of a second
// one.  A wavefront keeps 64 keys in registers as the B operand and a workgroup of four walks over tiles of 64 queries that
// come through LDS; in the accumulators a lane has one key (its column), so the sum over queries stays inside the lane and
// nothing is exchanged before the end.  A key tile's queries are cut into pieces of equal length for several workgroups - under a causal mask the
// first keys meet N queries and the last ones few - whose sums a second kernel adds in order: no atomics, one result.
#include "sage_attn.h"
#include "sage_ops.h"

#include <algorithm>
#include <cmath>

namespace sage {
namespace {

constexpr int KW_KEYS = 256;     // keys of a workgroup: 64 per wavefront
constexpr int KW_ROWS = 64;      // queries of a tile

struct KwParams {
  const unsigned short *q, *k;
  const float *lse, *w_in;
  float *w, *part;               // part: [piece][batch and KV head][N_kv]
  const int* lens;
  TensorMap qm, km;
  int B, H, Hkv, G, N, Nk;
  int causal, flat;              // flat: tiles run over the G N queries of a group, else over the N of each head
  float kappa;
  int key_tiles, pieces, piece;  // most pieces of a key tile, query tiles of a piece
};

// Query tiles of the keys t0 .. t0 + 255 of a sequence with `len` keys: per head those from the first query that sees t0 on.
struct KwItems { int first, per_head, count; };
__host__ __device__ __forceinline__ KwItems kw_items(int flat, int causal, int G, int N, int len, int t0) {
  KwItems x;
  if (flat) {
    x.first = 0;
    x.per_head = x.count = (G * N + KW_ROWS - 1) / KW_ROWS;
    return x;
  }
  const int coff = len > N ? len - N : 0, r = causal && t0 > coff ? t0 - coff : 0;
  const int all = (N + KW_ROWS - 1) / KW_ROWS;
  x.first = r / KW_ROWS < all ? r / KW_ROWS : all;
  x.per_head = all - x.first;
  x.count = x.per_head * G;
  return x;
}

__device__ __forceinline__ int kw_len(const KwParams& p, int b) { return p.lens ? min(max(p.lens[b], 0), p.Nk) : p.Nk; }

template <int D> constexpr int kw_occupancy() { return D == 64 ? 4 : 2; }

template <int D, bool BF16>
__global__ void __launch_bounds__(256, kw_occupancy<D>()) k_key_weights(const KwParams p) {
  constexpr int NP = D / 8, KS = D / 16, TILE = KW_ROWS * NP;
  __shared__ v4i s_q[2][TILE];
  __shared__ __align__(16) float s_nl[2][KW_ROWS];    // -lse log2(e) of the tile's queries
  __shared__ __align__(16) int s_vis[2][KW_ROWS];     // how many keys they see
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int col = lane & 31, half = lane >> 5;
  // workgroups in order: piece, key tile, head - the first keys' (the longest) first, heads side by side on different XCDs
  int id = blockIdx.x;
  const int bh = id % (p.B * p.Hkv); id /= p.B * p.Hkv;
  const int kt = id % p.key_tiles, piece = id / p.key_tiles;
  const int b = bh / p.Hkv, hkv = bh - b * p.Hkv;
  const int len = kw_len(p, b), t0 = kt * KW_KEYS;
  if (t0 >= len) return;
  const KwItems it = kw_items(p.flat, p.causal, p.G, p.N, len, t0);
  const int i0 = min(piece * p.piece, it.count), i1 = min(i0 + p.piece, it.count);
  const bool alone = p.pieces == 1;
  if (i0 >= i1 && !alone) return;
  const int coff = max(len - p.N, 0);

  // ---- my keys: column l % 32 of two operands, channels 16 s + 8 (l / 32) + 0..7
  const int key0 = t0 + 64 * wave;
  const size_t khead = head_offset(p.km, (unsigned)bh);
  v4i kreg[2][KS];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const unsigned short* kp = p.k + row_offset(p.km, khead, min(key0 + 32 * x + col, len - 1)) + 8 * half;
#pragma unroll
    for (int s = 0; s < KS; ++s) kreg[x][s] = *reinterpret_cast<const v4i*>(kp + 16 * s);
  }

  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)&s_q[0][0];
  const int rows_all = p.flat ? p.G * p.N : p.N;       // rows of the list that a tile is cut from
  const unsigned step = (unsigned)p.qm.sn * 2;
  auto copy = [&](int i, int stage) {
    const int g = i / it.per_head, r0 = (it.first + i - g * it.per_head) * KW_ROWS, last = rows_all - 1 - r0;
    const size_t head = head_offset(p.qm, (unsigned)(b * p.H + hkv * p.G + (p.flat ? 0 : g)));
    const char* base = uniform_ptr(reinterpret_cast<const char*>(p.q + head + (p.flat ? 0 : (size_t)r0 * p.qm.sn)));
#pragma unroll
    for (int x = 0; x < TILE / 256; ++x) {
      const int pc = (x * 4 + wave) * 64 + lane, r = pc / NP, c = (pc % NP) ^ swizzle<D>(r);
      unsigned off;
      if (p.flat) {
        const unsigned at = (unsigned)(r0 + min(r, last)), gg = at / (unsigned)p.N, n = at - gg * (unsigned)p.N;
        off = gg * (unsigned)(p.qm.sh * 2) + n * step;
      } else {
        off = (unsigned)min(r, last) * step;
      }
      dma_b128(base, off + (unsigned)c * 16, lds0 + (unsigned)(stage * TILE + (x * 4 + wave) * 64) * 16);
    }
  };
  // the first wavefront's lanes look up their query's constants; written to LDS a tile later
  float nl = 0.0f;
  int vis = 0;
  auto look = [&](int i) {
    const int g = i / it.per_head, r = (it.first + i - g * it.per_head) * KW_ROWS + lane;
    vis = 0;
    nl = 0.0f;
    if (r < rows_all) {
      const int gg = p.flat ? r / p.N : g, n = p.flat ? r - gg * p.N : r;
      const float x = p.lse[((size_t)b * p.H + hkv * p.G + gg) * p.N + n];
      nl = -x * LOG2E;
      vis = x == -INFINITY ? 0 : p.causal ? min(coff + n + 1, len) : len;
    }
  };

  float sum[2] = {0.0f, 0.0f};
  if (i0 < i1) {
    copy(i0, 0);
    if (wave == 0) {
      look(i0);
      s_nl[0][lane] = nl;
      s_vis[0][lane] = vis;
    }
  }
  for (int i = i0; i < i1; ++i) {
    const int stage = (i - i0) & 1;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();                 // tile i is there, and nobody reads the other stage any more
    asm volatile("" ::: "memory");
    if (i + 1 < i1) {
      copy(i + 1, stage ^ 1);
      if (wave == 0) look(i + 1);
    }
#pragma unroll 1
    for (int hr = 0; hr < 2; ++hr) {
      v16f acc[2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[x][v] = 0.0f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const v4i a = s_q[stage][row_piece<D>(32 * hr + col, 2 * s + half)];
#pragma unroll
        for (int x = 0; x < 2; ++x) acc[x] = mfma16<BF16>(a, kreg[x][s], acc[x]);
      }
      // rows 8 g + 4 h + r of the tile half: four runs of four
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const v4f n4 = *reinterpret_cast<const v4f*>(&s_nl[stage][32 * hr + 8 * g + 4 * half]);
        const v4i v4 = *reinterpret_cast<const v4i*>(&s_vis[stage][32 * hr + 8 * g + 4 * half]);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float e = __builtin_amdgcn_exp2f(__fmaf_rn(acc[x][4 * g + r], p.kappa, n4[r]));
            sum[x] += key0 + 32 * x + col < v4[r] ? e : 0.0f;
          }
      }
    }
    if (i + 1 < i1 && wave == 0) {
      s_nl[stage ^ 1][lane] = nl;
      s_vis[stage ^ 1][lane] = vis;
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const float y = half_sum(sum[x]);
    const int key = key0 + 32 * x + col;
    if (half == x && key < len) {
      const size_t at = (size_t)bh * p.Nk + key;
      if (alone) p.w[at] = (p.w_in ? p.w_in[at] : 0.0f) + y;
      else p.part[(size_t)piece * p.B * p.Hkv * p.Nk + at] = y;
    }
  }
}

// The pieces of each key, in order.  Grid: (keys / 256, batch and KV head).
__global__ void __launch_bounds__(256) k_key_weights_sum(const KwParams p) {
  const int key = blockIdx.x * 256 + threadIdx.x, bh = blockIdx.y, b = bh / p.Hkv;
  const int len = kw_len(p, b);
  if (key >= len) return;
  const KwItems it = kw_items(p.flat, p.causal, p.G, p.N, len, blockIdx.x * KW_KEYS);
  const int n = (it.count + p.piece - 1) / p.piece;
  const size_t at = (size_t)bh * p.Nk + key, step = (size_t)p.B * p.Hkv * p.Nk;
  float y = 0.0f;
  for (int i = 0; i < n; ++i) y += p.part[i * step + at];
  p.w[at] = (p.w_in ? p.w_in[at] : 0.0f) + y;
}

int kw_params(const sage_attn_key_weights_args* a, KwParams* p, bool need_io) {
  if (!a || a->B <= 0 || a->H <= 0 || a->H_kv <= 0 || a->N <= 0 || a->N_kv <= 0 || a->H % a->H_kv != 0) return SAGE_ERR_INVALID_ARG;
  if (a->d != 64 && a->d != 128 && a->d != 256) return SAGE_ERR_UNSUPPORTED;
  if (a->dtype != SAGE_DT_FP16 && a->dtype != SAGE_DT_BF16) return SAGE_ERR_UNSUPPORTED;
  if (a->layout != SAGE_LAYOUT_HND && a->layout != SAGE_LAYOUT_NHD) return SAGE_ERR_UNSUPPORTED;
  if (a->N > MAX_TOKENS || a->N_kv > MAX_TOKENS || (long long)a->B * a->H > 65535) return SAGE_ERR_UNSUPPORTED;
  if (need_io) {
    if (!a->q || !a->k || !a->lse || !a->weights) return SAGE_ERR_INVALID_ARG;
    if ((((uintptr_t)a->q | (uintptr_t)a->k) & 15u) != 0) return SAGE_ERR_INVALID_ARG;
    if ((((uintptr_t)a->lse | (uintptr_t)a->weights_in | (uintptr_t)a->weights | (uintptr_t)a->kv_lens) & 3u) != 0) return SAGE_ERR_INVALID_ARG;
  }
  p->q = (const unsigned short*)a->q; p->k = (const unsigned short*)a->k;
  p->lse = a->lse; p->w_in = a->weights_in; p->w = a->weights; p->lens = a->kv_lens; p->part = (float*)a->workspace;
  p->B = a->B; p->H = a->H; p->Hkv = a->H_kv; p->G = a->H / a->H_kv; p->N = a->N; p->Nk = a->N_kv;
  p->causal = a->causal != 0;
  p->kappa = (a->sm_scale > 0.0f ? a->sm_scale : (float)(1.0 / std::sqrt((double)a->d))) * LOG2E;
  const int nhd = a->layout == SAGE_LAYOUT_NHD;
  p->qm = make_tensor_map(nhd, a->H, a->N, a->d);
  p->km = make_tensor_map(nhd, a->H_kv, a->N_kv, a->d);
  // Few queries per head: the group's share tiles.  (A causal mask then skips nothing, of at most one tile per head.)
  p->flat = a->N <= KW_ROWS;
  if ((long long)p->G * ((p->N + KW_ROWS - 1) / KW_ROWS) > (1LL << 30)) return SAGE_ERR_UNSUPPORTED;
  const long long heads = (long long)a->B * a->H_kv, kts = (a->N_kv + KW_KEYS - 1) / KW_KEYS;
  long long all = 0;
  int most = 1;
  for (long long kt = 0; kt < kts; ++kt) {
    const int c = kw_items(p->flat, p->causal, p->G, p->N, p->Nk, (int)(kt * KW_KEYS)).count;
    all += c;
    most = std::max(most, c);
  }
  p->key_tiles = (int)kts;
  p->piece = (int)std::min<long long>(most, std::max(16LL, (heads * all + 2047) / 2048));
  p->pieces = (most + p->piece - 1) / p->piece;
  if (heads * kts * p->pieces > 0x7fffffffLL) return SAGE_ERR_UNSUPPORTED;
  return SAGE_OK;
}

size_t kw_bytes(const KwParams& p) { return p.pieces == 1 ? 0 : align256((size_t)p.pieces * p.B * p.Hkv * p.Nk * sizeof(float)); }

}  // namespace
}  // namespace sage

using namespace sage;

extern "C" size_t sage_attn_key_weights_workspace_bytes(const sage_attn_key_weights_args* a) {
  KwParams p;
  return kw_params(a, &p, false) == SAGE_OK ? kw_bytes(p) : 0;
}

extern "C" int sage_attn_key_weights(const sage_attn_key_weights_args* a) {
  KwParams p;
  int st = kw_params(a, &p, true);
  if (st != SAGE_OK) return st;
  const size_t need = kw_bytes(p);
  if (need > 0 && (!a->workspace || a->workspace_bytes < need || ((uintptr_t)a->workspace & 255u) != 0)) return SAGE_ERR_WORKSPACE;
  const hipStream_t s = (hipStream_t)a->stream;
  const unsigned blocks = (unsigned)((long long)p.B * p.Hkv * p.key_tiles * p.pieces);
  const bool bf16 = a->dtype == SAGE_DT_BF16;
  if (a->d == 64) { if (bf16) k_key_weights<64, true><<<blocks, 256, 0, s>>>(p); else k_key_weights<64, false><<<blocks, 256, 0, s>>>(p); }
  else if (a->d == 128) { if (bf16) k_key_weights<128, true><<<blocks, 256, 0, s>>>(p); else k_key_weights<128, false><<<blocks, 256, 0, s>>>(p); }
  else { if (bf16) k_key_weights<256, true><<<blocks, 256, 0, s>>>(p); else k_key_weights<256, false><<<blocks, 256, 0, s>>>(p); }
  st = op_status(hipGetLastError());
  if (st != SAGE_OK || p.pieces == 1) return st;
  k_key_weights_sum<<<dim3((unsigned)p.key_tiles, (unsigned)(p.B * p.Hkv)), 256, 0, s>>>(p);
  return op_status(hipGetLastError());
}
