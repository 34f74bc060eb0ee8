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
#include <type_traits>

namespace sage {
namespace {

constexpr int KW_KEYS = 256;     // keys of a workgroup: 64 per wavefront
constexpr int KW_ROWS = 64;      // queries of a tile
constexpr int KW_FEW = 64;       // rows of a group that are few
constexpr int KW_PIECE = 16;     // most query tiles of a workgroup: their constants are kept in LDS

struct KwParams {
  const unsigned short *q, *k;
  const float *lse, *w_in;
  float *w, *part;               // part: [piece][batch and KV head][N_kv]
  const int* lens;
  TensorMap qm, km;
  int B, H, Hkv, G, N, Nk;
  int few;                       // k_key_weights_few takes it: `piece` is then key tiles of a wavefront, `key_tiles` workgroups per head
  int causal, flat;              // flat: tiles run over the G N queries of a group, else over the N of each head
  float kappa;                   // sm_scale log2(e), rounded ..
  float lse_hi, lse_lo;          // .. and what that makes of log2(e): kappa / sm_scale, in two parts (see nl_of)
  int key_tiles, pieces, piece;  // most pieces of a key tile, query tiles of a piece
  FastDiv by_heads, by_hkv, by_kt, by_n;      // B H_kv, H_kv, key_tiles, N
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

// The constant of a query's exponents, -lse log2(e).  Of two numbers that nearly cancel, so the same log2(e) as in kappa, in more bits than one
// FP32 number has: each rounded for itself, the difference would be a share of lse that is the same for all keys and does not average out
// (weights 4e-6 too large at lse 80).
__device__ __forceinline__ float nl_of(const KwParams& p, float lse) {
  return fabsf(lse) < INFINITY ? __fmaf_rn(-lse, p.lse_hi, -(lse * p.lse_lo)) : -lse;
}
// That of a row that is not there, a copy of the last one: finite, so that it adds zero to finite scores and no NaN to an infinite weight.
constexpr float NL_NO_ROW = -3.40282347e38f;

__device__ __forceinline__ int kw_len(const KwParams& p, int b) { return p.lens ? min(max(p.lens[b], 0), p.Nk) : p.Nk; }

constexpr long long WIDE = 1 << 22;       // workgroups in the first dimension of a grid: more are in the second

// Wavefronts per SIMD that registers and LDS are cut for.
template <int D> constexpr int kw_occupancy() { return D == 256 ? 2 : 3; }

template <int D, bool BF16>
__global__ void __launch_bounds__(256, kw_occupancy<D>()) k_key_weights(const KwParams p) {
  constexpr int NP = D / 8, KS = D / 16, TILE = KW_ROWS * NP, NST = 2;
  constexpr unsigned ROW = D * 2;
  __shared__ __align__(1024) v4i s_q[NST][TILE];
  __shared__ __align__(16) float s_nl[KW_PIECE * KW_ROWS + 32];    // -lse log2(e) of the piece's queries; -inf: adds nothing; 32 of those
  __shared__ __align__(16) int s_vis[KW_PIECE * KW_ROWS];     // how many keys they see; -1: no query
  __shared__ int s_masked[KW_PIECE];                          // whether a query of the tile does not see all of the workgroup's keys
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int col = lane & 31, half = lane >> 5;
  // workgroups in order: piece, key tile, head - the first keys' (the longest) first, heads side by side on different XCDs
  unsigned bh = blockIdx.y * gridDim.x + blockIdx.x, kt = split_by(bh, p.by_heads), hkv = bh;
  const int piece = (int)split_by(kt, p.by_kt), b = (int)split_by(hkv, p.by_hkv);
  const int len = kw_len(p, b), t0 = (int)kt * KW_KEYS;
  if (piece >= p.pieces || t0 >= len) return;
  const KwItems it = kw_items(p.flat, p.causal, p.G, p.N, len, t0);
  const int used = (it.count + p.piece - 1) / p.piece, each = used > 0 ? (it.count + used - 1) / used : 0;     // pieces of this key tile, all of a length
  const int i0 = min(piece * each, it.count), i1 = min(i0 + each, it.count);
  const bool alone = p.pieces == 1;
  if (i0 >= i1 && !alone) return;
  const int coff = max(len - p.N, 0);

  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)&s_q[0][0];
  const int rows_all = p.flat ? p.G * p.N : p.N;       // rows of the list that a tile is cut from
  const unsigned step = (unsigned)p.qm.sn * 2;
  const unsigned short* qb = p.q + head_offset_of(p.qm, b, (int)hkv * p.G);
  // The tile to copy next: row r0 of head g of the group.  What a lane adds to its first byte stays the same but for a head's last tile.
  const int g0 = i0 / it.per_head;
  int g = g0, r0 = (it.first + i0 - g0 * it.per_head) * KW_ROWS;
  unsigned offs[TILE / 256];
#pragma unroll
  for (int x = 0; x < TILE / 256; ++x) {
    const int pc = (x * 4 + wave) * 64 + lane, r = pc / NP;
    offs[x] = (unsigned)r * step + (unsigned)((pc % NP) ^ swizzle<D>(r)) * 16;
  }
  auto copy = [&](int stage) __attribute__((always_inline)) {
    const unsigned to = lds0 + (unsigned)(stage * TILE + wave * 64) * 16;
    const char* base = uniform_ptr(reinterpret_cast<const char*>(qb + (p.flat ? 0 : (size_t)g * p.qm.sh + (size_t)r0 * p.qm.sn)));
    if (!p.flat && r0 + KW_ROWS <= rows_all) {
#pragma unroll
      for (int x = 0; x < TILE / 256; ++x) dma_b128(base, offs[x], to + x * 4096);
    } else {
#pragma unroll 1
      for (int x = 0; x < TILE / 256; ++x) {
        const int pc = (x * 4 + wave) * 64 + lane, r = pc / NP, c = (pc % NP) ^ swizzle<D>(r);
        unsigned n = (unsigned)min(r0 + r, rows_all - 1);
        unsigned off;
        if (p.flat) {
          const unsigned gg = split_by(n, p.by_n);
          off = gg * (unsigned)(p.qm.sh * 2) + n * step;
        } else {
          off = (n - (unsigned)r0) * step;
        }
        dma_b128(base, off + (unsigned)c * 16, to + x * 4096);
      }
    }
    r0 += KW_ROWS;
    if (!p.flat && r0 >= rows_all) {
      r0 = it.first * KW_ROWS;
      ++g;
    }
  };
  if (i0 < i1) copy(0);

  // ---- my keys: column l % 32 of two operands, channels 16 s + 8 (l / 32) + 0..7
  const int key0 = t0 + 64 * wave;
  const size_t khead = head_offset_of(p.km, b, (int)hkv);
  v4i kreg[2][KS];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const unsigned short* kp = p.k + row_offset(p.km, khead, min(key0 + 32 * x + col, len - 1)) + 8 * half;
#pragma unroll
    for (int s = 0; s < KS; ++s) kreg[x][s] = *reinterpret_cast<const v4i*>(kp + 16 * s);
  }
  // ---- the queries' constants, a wavefront per tile, four of its loads together
  int gi = g0, qi = i0 - g0 * it.per_head + wave;
  for (int i = i0 + wave; i < i1; i += 16) {
    float lse[4];
    int seen[4];
#pragma unroll
    for (int y = 0; y < 4; ++y, qi += 4) {
      for (; qi >= it.per_head && gi < p.G; qi -= it.per_head) ++gi;
      const int r = (it.first + qi) * KW_ROWS + lane;
      // Rows behind the last repeat it, and add nothing: they see no key, since a row that adds nothing may hold anything.  They do not
      // make a tile one that needs the mask: where the row that they repeat does not either, its scores count, and theirs are as good.
      lse[y] = 0.0f;
      seen[y] = -1;
      if (i + 4 * y < i1 && r < rows_all) {
        unsigned n = (unsigned)r;
        const int gg = p.flat ? (int)split_by(n, p.by_n) : gi;
        lse[y] = p.lse[((size_t)b * p.H + (int)hkv * p.G + gg) * p.N + n];
        seen[y] = p.causal ? min(coff + (int)n + 1, len) : len;
      }
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int at = i - i0 + 4 * y;
      if (at < i1 - i0) {
        const int vis = lse[y] == -INFINITY ? 0 : seen[y];
        const int masked = __ballot(vis >= 0 && vis < min(t0 + KW_KEYS, len)) != 0;
        s_nl[at * KW_ROWS + lane] = seen[y] < 0 ? NL_NO_ROW : nl_of(p, lse[y]);
        s_vis[at * KW_ROWS + lane] = vis;
        if (lane == 0) s_masked[at] = masked;
      }
    }
  }
  if (t < 32) s_nl[KW_PIECE * KW_ROWS + t] = -INFINITY;
  // (the keys are here before the loop, or it would wait for its copies with the first use of each)
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int y = 0; y < 4; ++y) use_now(kreg[x][s][y]);

  // Scores of 32 queries and my 64 keys, and the weights of 32 others, whose scores are there: the matrix unit works on the one while
  // the vector unit takes the other.  A row's pieces are one exclusive or apart (see swizzle).
  typedef __attribute__((address_space(3))) const v4i* lds_v4i;
  const unsigned q_at = (unsigned)row_piece<D>(col, half) * 16;
  float sum[2][2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
  auto constants = [&](int row, int g) __attribute__((always_inline)) {        // rows 8 g + 4 h + 0..3
    return *reinterpret_cast<const v4f*>(&s_nl[row + 8 * g + 4 * half]);
  };
  auto weight = [&](int e, const v16f (&sc)[2], const v4f& n) __attribute__((always_inline)) {
    const int x = e & 1, v = e >> 1;
    sum[x][v & 1] += __builtin_amdgcn_exp2f(__fmaf_rn(sc[x][v], p.kappa, n[v & 3]));
  };
  auto weights = [&](const v16f (&sc)[2], int row) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const v4f n = constants(row, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) weight(8 * g + e, sc, n);
    }
  };
  auto scores = [&](unsigned at, v16f (&acc)[2], const v16f (&sc)[2], int row) __attribute__((always_inline)) {
    constexpr int AHEAD = 2;            // operands come from LDS so many steps before their products
    v4i a[KS];
    v4f n = constants(row, 0), next;
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) a[s] = *(lds_v4i)(uintptr_t)(at ^ (32 * s));
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      if (s + AHEAD < KS) a[s + AHEAD] = *(lds_v4i)(uintptr_t)(at ^ (32 * (s + AHEAD)));
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        v16f c = acc[x];
        if (s == 0) {
#pragma unroll
          for (int v = 0; v < 16; ++v) c[v] = 0.0f;
        }
        acc[x] = mfma16<BF16>(a[s], kreg[x][s], c);
        constexpr int PER = 16 / KS;    // weights after a product; eight share their constants
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int w = (2 * s + x) * PER + e;
          if (w % 8 == 0 && w < 24) next = constants(row, w / 8 + 1);
          weight(w, sc, n);
          if (w % 8 == 7) n = next;
        }
        __builtin_amdgcn_sched_barrier(0);      // (a product, then its share of the weights: not all products first)
      }
    }
  };

  v16f acc_a[2], acc_b[2];
  constexpr int NO_ROW = KW_PIECE * KW_ROWS;
  int row_b;                                      // where the constants of acc_b's queries are
  auto nothing = [&]() __attribute__((always_inline)) {       // scores whose weights are zero
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc_b[x][v] = 0.0f;
    row_b = NO_ROW;
  };
  nothing();
  int stage = 0;
  for (int i = i0; i < i1; ++i) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();                 // tile i is there, and nobody reads the other stage any more
    asm volatile("" ::: "memory");
    if (i + 1 < i1) copy(stage ^ 1);
    const unsigned at = lds0 + (unsigned)stage * (TILE * 16) + q_at;
    const int row = (i - i0) * KW_ROWS;
    if (__builtin_amdgcn_readfirstlane(s_masked[i - i0]) == 0) {
      scores(at, acc_a, acc_b, row_b);
      scores(at + 32 * ROW, acc_b, acc_a, row);
      row_b = row + 32;
    } else {
      asm volatile("" : "+s"(row_b));             // (or the weights of acc_b, common to both ways, would be taken before them)
      weights(acc_b, row_b);
#pragma unroll 1
      for (int hr = 0; hr < 2; ++hr) {
        const unsigned here = at + 32 * hr * ROW;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc_a[x][v] = 0.0f;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int x = 0; x < 2; ++x) acc_a[x] = mfma16<BF16>(*(lds_v4i)(uintptr_t)(here ^ (32 * s)), kreg[x][s], acc_a[x]);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const v4f n = constants(row + 32 * hr, g);
          const v4i v4 = *reinterpret_cast<const v4i*>(&s_vis[row + 32 * hr + 8 * g + 4 * half]);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const float e = __builtin_amdgcn_exp2f(__fmaf_rn(acc_a[x][4 * g + r], p.kappa, n[r]));
              sum[x][r & 1] += key0 + 32 * x + col < v4[r] ? e : 0.0f;
            }
        }
      }
      nothing();
    }
    stage ^= 1;
  }
  weights(acc_b, row_b);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const float y = half_sum(sum[x][0] + sum[x][1]);
    const int key = key0 + 32 * x + col;
    if (half == x && key < len) {
      const size_t at = ((size_t)b * p.Hkv + hkv) * p.Nk + key;
      if (alone) p.w[at] = (p.w_in ? p.w_in[at] : 0.0f) + y;
      else p.part[(size_t)piece * p.B * p.Hkv * p.Nk + at] = y;
    }
  }
}

// Few queries (16 RT rows of a group at most): nothing but the keys is read to speak of, and each of them once.  The queries stay in
// registers, and each wavefront walks over tiles of 16 keys that come to LDS of its own, some ahead of the one it multiplies: no
// barrier, and rows that are not there are paid for in products that nobody waits for.  Bound by reading: the copies take whole rows and pass the
// caches by (us, operands loaded to registers, which come in pieces of 64 bytes of a row / this: 16 caches of 20000 keys, 8 heads
// of 128 channels, 90 / 80, 5.5 TB/s; 8 of them token-major 53.5 / 42.8; 16 of 9000 of 64 22.8 / 19.9; copies that stay in the caches 90).
// Stages: LDS for 16 wavefronts of 64 channels or 8 of 128 or 256 per CU, three tiles in flight each or, of 256 channels, one (with
// three of these and 4 wavefronts 30.7 for 26.9 us, of 128 with two for 8 / one for 16 42 and 39.5 for 39.3).
constexpr int KF_KEYS = 16;
template <int D> constexpr int kf_stages() { return D == 256 ? 2 : 4; }
template <int D> constexpr int kf_held() { return D == 64 ? 16 : 8; }       // wavefronts of a CU
template <int D, bool BF16, int RT>
__global__ void __launch_bounds__(256, kf_held<D>() / 4) k_key_weights_few(const KwParams p) {
  constexpr int KF_STAGES = kf_stages<D>();
  constexpr int KS = D / 32, NP = D / 8, TILE = KF_KEYS * NP, COPIES = TILE / 64;
  constexpr unsigned ROW = D * 2;
  __shared__ __align__(1024) v4i s_k[4][KF_STAGES][TILE];
  __shared__ float s_w[4][KF_STAGES][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  unsigned bh = blockIdx.x;
  const int chunk = (int)split_by(bh, p.by_heads);
  unsigned hkv = bh;
  const int b = (int)split_by(hkv, p.by_hkv);
  const int len = kw_len(p, b), rows = p.G * p.N, coff = max(len - p.N, 0);
  const int tiles = (len + KF_KEYS - 1) / KF_KEYS, j0 = chunk * 4 * p.piece + wave, j1 = min(chunk * 4 * p.piece + 4 * p.piece, tiles);
  if (j0 >= j1) return;
  const size_t wb = (size_t)bh * p.Nk;

  // ---- copies of a tile: rows behind the last key repeat it
  const char* gk = uniform_ptr(reinterpret_cast<const char*>(p.k + head_offset_of(p.km, b, (int)hkv)));
  const char* gw = uniform_ptr(reinterpret_cast<const char*>(p.w_in + wb));
  const bool add = p.w_in != nullptr;
  const unsigned step = (unsigned)p.km.sn * 2;    // bytes from token to token
  const unsigned k0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)&s_k[wave][0][0];
  const unsigned w0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)&s_w[wave][0][0];
  auto copy = [&](int j, int stage) __attribute__((always_inline)) {
    const int last = len - 1 - j * KF_KEYS;
    const char* from = gk + (size_t)j * KF_KEYS * step;
#pragma unroll
    for (int x = 0; x < COPIES; ++x) {
      const int pc = x * 64 + lane, r = pc / NP;
      dma_b128_once(from, (unsigned)min(r, last) * step + (unsigned)((pc % NP) ^ swizzle<D>(r)) * 16, k0 + (unsigned)(stage * TILE + x * 64) * 16);
    }
    if (add) dma_b32(gw + (size_t)j * (KF_KEYS * 4), (unsigned)min(col, last) * 4, w0 + stage * 256);
  };
#pragma unroll
  for (int x = 0; x < KF_STAGES - 1; ++x)
    if (j0 + 4 * x < j1) copy(j0 + 4 * x, x);

  // ---- the queries: row l % 16 of RT operands, and the constants of the rows of my accumulators (4 (l / 16) + 0..3)
  v4i q[RT][KS];
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    unsigned n = (unsigned)min(16 * x + col, rows - 1);
    const int g = (int)split_by(n, p.by_n);
    const unsigned short* at = p.q + head_offset_of(p.qm, b, (int)hkv * p.G + g) + (size_t)n * p.qm.sn + 8 * quad;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[x][s] = *reinterpret_cast<const v4i*>(at + 32 * s);
  }
  float mine = 0.0f;                              // lse of row `lane`
  if (lane < rows) {
    unsigned n = (unsigned)lane;
    const int g = (int)split_by(n, p.by_n);
    mine = p.lse[((size_t)b * p.H + (int)hkv * p.G + g) * p.N + n];
  }
  // (waited for here, with the first tiles: in the loop the compiler would wait for every copy)
#pragma unroll
  for (int x = 0; x < RT; ++x)
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int y = 0; y < 4; ++y) use_now(q[x][s][y]);
  const bool blind = __ballot(mine == -INFINITY) != 0;      // (a row that saw nothing: whatever its scores, it adds nothing)
  const int sees_all = blind ? 0 : p.causal ? min(coff + 1, len) : len;
  const float my_nl = lane < rows ? nl_of(p, mine) : NL_NO_ROW;
  float nl[RT][4];
#pragma unroll
  for (int x = 0; x < RT; ++x)
#pragma unroll
    for (int v = 0; v < 4; ++v) nl[x][v] = __shfl(my_nl, 16 * x + 4 * quad + v);

  typedef __attribute__((address_space(3))) const v4i* lds_v4i;
  const unsigned k_at = k0 + (unsigned)row_piece<D>(col, quad) * 16;       // (a step of 4 pieces is an exclusive or: see swizzle)
  int stage = 0;
  for (int j = j0; j < j1; j += 4) {
    // copies are counted in order; stores, which are counted too, can only make the wait longer
    const int later = min((j1 - 1 - j) / 4, KF_STAGES - 2);
    auto wait = [&](auto per) __attribute__((always_inline)) {
      constexpr int P = decltype(per)::value;
      if (later == 0) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      else if (later == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(P) : "memory");
      else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * P) : "memory");
    };
    if (add) wait(std::integral_constant<int, COPIES + 1>{}); else wait(std::integral_constant<int, COPIES>{});
    // (the stage of the tile before, whose reads are over)
    if (j + 4 * (KF_STAGES - 1) < j1) copy(j + 4 * (KF_STAGES - 1), (stage + KF_STAGES - 1) % KF_STAGES);
    v4f acc[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) acc[x] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const unsigned at = k_at + (unsigned)stage * (TILE * 16);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const v4i k = *(lds_v4i)(uintptr_t)(at ^ (64 * s));
#pragma unroll
      for (int x = 0; x < RT; ++x) acc[x] = mfma16_small<BF16>(q[x][s], k, acc[x]);
    }
    const float was = add ? s_w[wave][stage][lane] : 0.0f;
    float sum = 0.0f;
    if (KF_KEYS * j + KF_KEYS <= sees_all) {
#pragma unroll
      for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int v = 0; v < 4; ++v) sum += __builtin_amdgcn_exp2f(__fmaf_rn(acc[x][v], p.kappa, nl[x][v]));
    } else {
#pragma unroll
      for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int r = 16 * x + 4 * quad + v;
          unsigned n = (unsigned)min(r, rows - 1);
          (void)split_by(n, p.by_n);
          const bool see = r < rows && nl[x][v] != INFINITY;      // (+inf: an lse of -inf)
          const int vis = !see ? 0 : p.causal ? min(coff + (int)n + 1, len) : len;
          const float e = __builtin_amdgcn_exp2f(__fmaf_rn(acc[x][v], p.kappa, nl[x][v]));
          sum += KF_KEYS * j + col < vis ? e : 0.0f;
        }
    }
    const unsigned u = __float_as_uint(sum);
    const auto sw = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    sum = half_sum(__uint_as_float(sw[0]) + __uint_as_float(sw[1]));
    const int key = KF_KEYS * j + lane;
    if (lane < KF_KEYS && key < len) p.w[wb + key] = was + sum;
    stage = (stage + 1) % KF_STAGES;
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
  for (int i0 = 0; i0 < n; i0 += 8) {             // eight loads in flight, added in order
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p.part[(size_t)min(i0 + i, n - 1) * step + at];
#pragma unroll
    for (int i = 0; i < 8; ++i) y += i0 + i < n ? x[i] : 0.0f;
  }
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
  const double scale = a->sm_scale > 0.0f ? (double)a->sm_scale : 1.0 / std::sqrt((double)a->d);
  p->kappa = (float)(scale * 1.4426950408889634);
  p->lse_hi = (float)(p->kappa / scale);
  p->lse_lo = (float)(p->kappa / scale - p->lse_hi);
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
  p->by_heads = fast_div((unsigned)heads); p->by_hkv = fast_div((unsigned)a->H_kv); p->by_kt = fast_div((unsigned)kts); p->by_n = fast_div((unsigned)a->N);
  // As many tiles as give 1024 workgroups, 2 to 16: what a workgroup does before its first tile costs as much as three to six, but
  // with fewer of them the last ones run alone.  Us, tiles of a workgroup: 66 k tiles (8192 causal queries, 32 heads of 128) 4 / 8 / 16 / 32
  // 339 / 306 / 296 / 293, 17 k 103 / 94 / 93 / 97, 9 k (not causal) 52 / 49 / 53 / 60, 1.2 k 24 / 28 / 46 / 64, 96 (2 / 4 / 8) 15 / 19 / 24; of 256
  // channels 8 k 73 / 69 / 73; of 64 33 k 134 / 119 / 116 / 120.
  p->piece = (int)std::min<long long>(std::min(most, KW_PIECE), std::max(2LL, (heads * all + 1023) / 1024));
  // A few are not divided, for then nothing has to be added up.  (Us, divided / not: 3 tiles on 4 heads of 64 channels 15.0 / 10.9, of 128
  // 14.7 / 13.3, of 256 17.5 / 18.5; 4 tiles 14.6 / 12.8, 15.0 / 15.8, 18.1 / 22.4.)
  if (most * (a->d + 64) <= 576) p->piece = most;
  p->pieces = (most + p->piece - 1) / p->piece;
  // Few rows; more than 32 only from 64 k keys on, because every wavefront has all of them to read first (us, tiles of queries / few rows: 48
  // rows of 128 channels on 128 caches of 16000 keys 87 / 73, on 8 of 9000 11.7 / 10.9, on 8 of 4000 9.2 / 10.6).  Its key tiles: as
  // many as make two rounds of the wavefronts that the chip holds - lengths differ, and with one round it empties early (one and a half / two / three: 32
  // caches of 32768 keys of 128 channels 47 / 39 / 42, 128 of 20000 91 / 81 / 80) - but four at least, eight for more than 16 rows (one / two
  // / four / eight: 24 rows on 32 caches of 4000 keys of 128 channels 16.3 / 12.1 / 9.6 / 9.5, 4 rows 11.8 / 11.7 / 9.1 / -).
  const long long rows = (long long)p->G * a->N, tiles = (a->N_kv + KF_KEYS - 1) / KF_KEYS;
  p->few = rows <= 32 || (rows <= KW_FEW && heads * tiles >= 4096);
  if (p->few) {
    const long long held = 256 * (a->d == 64 ? kf_held<64>() : a->d == 128 ? kf_held<128>() : kf_held<256>());
    p->pieces = 1;
    p->piece = (int)std::max(rows > 16 ? 8LL : 4LL, std::min(128LL, heads * tiles / (2 * held)));
    p->key_tiles = (int)((tiles + 4 * p->piece - 1) / (4 * p->piece));
  }
  if (heads * p->key_tiles * p->pieces > 0x7fffffffLL - WIDE || (p->few && heads * p->key_tiles > WIDE)) return SAGE_ERR_UNSUPPORTED;
  return SAGE_OK;
}

template <int D, bool BF16> hipError_t launch_kw(const KwParams& p, hipStream_t s) {
  const long long all = (long long)p.B * p.Hkv * p.key_tiles * p.pieces;
  const dim3 blocks((unsigned)std::min(all, WIDE), (unsigned)((all + WIDE - 1) / WIDE));
  if (!p.few) k_key_weights<D, BF16><<<blocks, 256, 0, s>>>(p);
  else if (p.G * p.N <= 16) k_key_weights_few<D, BF16, 1><<<blocks, 256, 0, s>>>(p);
  else if (p.G * p.N <= 32) k_key_weights_few<D, BF16, 2><<<blocks, 256, 0, s>>>(p);
  else k_key_weights_few<D, BF16, 4><<<blocks, 256, 0, s>>>(p);
  return hipGetLastError();
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
  // (workgroups add to keys in any order: weights_in is the same tensor, or another one)
  const size_t rows = (size_t)a->B * a->H * a->N, keys = (size_t)a->B * a->H_kv * a->N_kv;
  const Span w = {a->weights, keys * 4}, ws = {need > 0 ? a->workspace : nullptr, need}, in[5] = {{a->q, rows * a->d * 2}, {a->k, keys * a->d * 2}, {a->lse, rows * 4},
                       {a->kv_lens, (size_t)a->B * 4}, {a->weights_in == a->weights ? nullptr : a->weights_in, keys * 4}};
  for (const Span& x : in) if (overlap(w, x) || overlap(ws, x)) return SAGE_ERR_INVALID_ARG;
  if (overlap(w, ws)) return SAGE_ERR_INVALID_ARG;
  const hipStream_t s = (hipStream_t)a->stream;
  const bool bf16 = a->dtype == SAGE_DT_BF16;
  const hipError_t e = a->d == 64 ? (bf16 ? launch_kw<64, true>(p, s) : launch_kw<64, false>(p, s))
                     : a->d == 128 ? (bf16 ? launch_kw<128, true>(p, s) : launch_kw<128, false>(p, s))
                                   : (bf16 ? launch_kw<256, true>(p, s) : launch_kw<256, false>(p, s));
  st = op_status(e);
  if (st != SAGE_OK || p.pieces == 1) return st;
  k_key_weights_sum<<<dim3((unsigned)p.key_tiles, (unsigned)(p.B * p.Hkv)), 256, 0, s>>>(p);
  return op_status(hipGetLastError());
}
