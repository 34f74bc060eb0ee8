// 16-bit attention of a batch whose sequences share a prefix of keys and values (sage_attn_shared_prefix).
//
// O = softmax(kappa [Q Kp^T, Q Ko^T]) [Vp; Vo]: the prefix's keys are the same for every sequence, so the rows of one
// product over them are the queries of all sequences and of all query heads of a KV head (B G N rows, G = H / H_kv), and the
// prefix is read once instead of B times.  A sequence's own keys meet only its own G N rows.  The two parts, and chunks
// of their keys, are independent workgroups of one launch; each leaves (m, l, O) under its own running maximum (Sec. 2.1, Eq. 1)
// and a second kernel merges them: O = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i.  (Where there are few keys, a workgroup takes them all.)
//
// With few rows this reads the cache and nothing else bounds it, so K and V stay in the 16 bits they are kept in: quantizing them
// on the way would cost vector instructions for nothing.  P is rounded to the type of V for the second product (half a step, 2^-9
// of a weight with bf16, which averages out over the keys; the output is rounded to the same type); scores, the running
// maximum, the sum and O are FP32.  fp16 has no numbers for weights below 2^-25 of the largest, which are in the sum all the same: there m
// is kept 14 below the maximum, so that weights are up to 2^14 and vanish from 2^-39 of the largest on, too small for 2^25 keys (the most)
// to add up to half a step of the output (2^-11).
#include "sage_attn.h"
#include "sage_ops.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace sage {
namespace {

template <bool BF16> __device__ __forceinline__ bool not_finite(unsigned x) {
  constexpr unsigned EXP = BF16 ? 0x7f80 : 0x7c00;
  return (x & EXP) == EXP;
}

constexpr int SH_KEYS = 64;      // keys of a tile
// Wavefronts of a workgroup, 32 query rows each.  Two wavefronts share a SIMD where 128 rows do (one's vector work runs beside
// the other's products); 256-wide heads, whose two tiles of K and V fill the LDS of a CU, need eight in one workgroup for that.
template <int D> constexpr int shared_waves() { return D == 256 ? 8 : 4; }
constexpr int shared_rows(int d) { return d == 256 ? 256 : 128; }

struct SharedParams {
  const unsigned short *q, *kp, *vp, *ko, *vo;
  unsigned short* out;
  float* lse;
  const int* lens;
  float *part_o, *part_ml;       // [partial][row][d], [partial][row][2]: see part_row
  TensorMap qm, pm, om;          // of q and out; of the prefix; of the own caches
  int B, H, Hkv, G, N, P, Nk;
  int causal, one;               // one: no key chunks and no merge (ONE)
  float kappa;                   // sm_scale log2(e)
  int Sp, So;                    // key chunks of the prefix and of the own keys
  int rtp, rto;                  // row tiles of the prefix (of B G N rows) and of the own keys (of G N rows)
  int n_prefix;                  // workgroups of the prefix; those of the own keys follow
  int full;                      // of them, those of whole groups of 8 chunks
  FastDiv by_group, by_rtp, by_hkv, by_rto, by_b, by_gn, by_n, by_rows, by_sp, by_so;      // 8 rtp, rtp, H_kv, rto, B, G N, N, B G N, Sp, So
};

// Where partial result `s` of a row is kept: the prefix's chunks first, then the own ones.  Rows are numbered (KV head, batch, head of
// the group, query), partials of one row are a chunk apart.
__device__ __forceinline__ size_t part_row(const SharedParams& p, int s, int hkv, long long i) {
  const size_t rows = (size_t)p.B * p.G * p.N;
  return ((size_t)s * p.Hkv + hkv) * rows + i;
}

__device__ __forceinline__ int own_len(const SharedParams& p, int b) { return p.lens ? min(max(p.lens[b], 0), p.Nk) : p.Nk; }

template <int D> constexpr int shared_occupancy() { return D == 64 ? 3 : 2; }   // wavefronts per SIMD

// ONE: a workgroup walks over the whole prefix and then its sequence's own keys, and leaves the output itself (see choose_chunks).
template <int D, bool BF16, bool ONE>
__global__ void __launch_bounds__(64 * shared_waves<D>(), shared_occupancy<D>()) k_shared(const SharedParams p) {
  constexpr int NP = D / 8;                       // 16-byte pieces of a row
  constexpr int KS = D / 16;                      // contraction steps of the score product
  constexpr int CT = D / 32;                      // channel tiles of the output
  constexpr int TILE = SH_KEYS * NP;              // pieces of a K (or V) tile
  constexpr int W = shared_waves<D>(), ROWS = 32 * W;
  __shared__ __align__(1024) v4i s_kv[2][2 * TILE];     // [stage][K, V]
  __shared__ float s_ml[shared_waves<D>()][64];         // maxima and sums of the rows of each wavefront
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int col = lane & 31, half = lane >> 5;

  // The arguments take six cache lines: one wait for all of them, not one for each where its first word is needed
  asm volatile("" ::"s"(p.vp), "s"(p.lens), "s"(p.om.sn), "s"(p.causal), "s"(p.by_group.m), "s"(p.by_n.m));

  // ---- which rows and keys
  unsigned id = blockIdx.x, hkv, b = 0, rt, s;
  const bool prefix = !ONE && (int)id < p.n_prefix;
  if (prefix) {
    // The row tiles of a chunk read the same keys: they are 8 apart, since workgroups go to the 8 XCDs in turn and each has a cache
    // of its own.  (The last chunks, fewer than 8, have a chunk's side by side.)
    if ((int)id < p.full) {
      const unsigned group = split_by(id, p.by_group);
      s = group * 8 + id % 8;
      rt = id / 8;
    } else {
      rt = id - (unsigned)p.full;
      const unsigned before = div_by((unsigned)p.full, p.by_rtp);
      s = before + split_by(rt, p.by_rtp);
    }
    hkv = s;
    s = split_by(hkv, p.by_hkv);
  } else {
    rt = id - (unsigned)p.n_prefix;
    hkv = split_by(rt, p.by_rto);
    b = split_by(hkv, p.by_hkv);
    s = split_by(b, p.by_b);
  }
  const int GN = p.G * p.N, rows = prefix ? p.B * GN : GN, r0 = (int)rt * ROWS;
  const int nr = min(ROWS, rows - r0);            // rows of this workgroup
  const int nk = prefix ? p.P : own_len(p, (int)b);
  const int tp = ONE ? (p.P + SH_KEYS - 1) / SH_KEYS : 0, tiles = tp + (nk + SH_KEYS - 1) / SH_KEYS;     // tiles of the prefix come first
  int j0 = 0, j1 = tiles;
  if constexpr (!ONE) {
    const int per = prefix ? (int)div_by((unsigned)(tiles + p.Sp - 1), p.by_sp) : (int)div_by((unsigned)(tiles + p.So - 1), p.by_so);
    j0 = min((int)s * per, tiles);
    j1 = min(j0 + per, tiles);
  }
  const int sp = (int)s + (prefix ? 0 : p.Sp);
  const int i0 = prefix ? r0 : (int)b * GN + r0;  // first row in the numbering of part_row

  // Wavefronts: 32 rows each; where half of them do for the rows, two share rows and take every other 32 keys.  In the end they share
  // the channels too: each gives its upper CT / 2 channel tiles to the other, so the second has its tiles in the other order
  // (tile c in place c ^ CT / 2).
  const int WK = nr <= ROWS / 2 ? 2 : 1;
  const int kg = WK == 2 ? wave & 1 : 0, rg = WK == 2 ? wave >> 1 : wave;
  const bool active = rg * 32 < nr;

  if (!ONE && j0 >= j1) {                         // no keys: a partial result that the merge skips
    for (int i = t; i < nr; i += 64 * W) {
      float* ml = p.part_ml + part_row(p, sp, (int)hkv, i0 + i) * 2;
      ml[0] = -INFINITY;
      ml[1] = 0.0f;
    }
    return;
  }

  // ---- my row's query as the B operand, and how many keys it sees
  const int row = min(rg * 32 + col, nr - 1);
  const int i = i0 + row;
  unsigned rn = (unsigned)i;
  const unsigned rb = split_by(rn, p.by_gn), rh = split_by(rn, p.by_n);
  const size_t qrow = row_offset(p.qm, head_offset_of(p.qm, (int)rb, (int)(hkv * p.G + rh)), (int)rn);
  v4i q[KS];
#pragma unroll
  for (int st = 0; st < KS; ++st) q[st] = *reinterpret_cast<const v4i*>(p.q + qrow + 16 * st + 8 * half);
  const int coff = max(nk - p.N, 0);
  const int vis = prefix || !p.causal ? nk : min(coff + (int)rn + 1, nk);
  const int vis_all = prefix || !p.causal ? nk : min(coff + 1, nk);       // keys that every query sees
  const bool part_seen = vis_all < nk;            // ... and others that some do

  // ---- copies of a tile: rows behind the last key repeat it
  const TensorMap& m = prefix ? p.pm : p.om;      // (a step from token to token is the same in both)
  const size_t head = head_offset_of(m, (int)b, (int)hkv);
  const char* gk = uniform_ptr(reinterpret_cast<const char*>((prefix ? p.kp : p.ko) + head));
  const char* gv = uniform_ptr(reinterpret_cast<const char*>((prefix ? p.vp : p.vo) + head));
  const size_t first = ONE ? head_offset_of(p.pm, 0, (int)hkv) : 0;
  const char* gkp = uniform_ptr(reinterpret_cast<const char*>(p.kp + first));       // (ONE: the prefix's)
  const char* gvp = uniform_ptr(reinterpret_cast<const char*>(p.vp + first));
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)&s_kv[0][0];
  const unsigned step = (unsigned)m.sn * 2;       // bytes from token to token
  constexpr int COPIES = TILE / (64 * W);         // of a tile of K (or V), by a wavefront
  unsigned offs[COPIES];
#pragma unroll
  for (int x = 0; x < COPIES; ++x) {
    const int pc = (x * W + wave) * 64 + lane, r = pc / NP;
    offs[x] = (unsigned)r * step + (unsigned)((pc % NP) ^ swizzle<D>(r)) * 16;
  }
  // What one workgroup alone reads passes the caches by.  The prefix only where it has few rows: with more, its workgroups leave partial
  // results of as many bytes, and reads from memory itself make them later (us, kept in the caches / past them: 16 sequences of up to
  // 3000 own keys over 20000, 128 channels 56.5 / 52.9; 4 over 100000 84.5 / 75.3; 6 of 5 tokens of 256 channels over 5003, 120
  // rows: 30.4 / 34.2).  In one launch every sequence reads the prefix: with more than one to an XCD it is kept (sequences of 380 + 60 keys of
  // 128 channels, kept / past the caches: 512 106.4 / 108.4, 128 29.4 / 30.3, 32 13.4 / 13.6; 4 of 300 + 50 of 64 the kernel 9.6 / 9.4).
  const bool once = prefix ? rows <= 64 : p.rto == 1 && (!ONE || p.B <= 8);
  auto copy = [&](int j, int stage) __attribute__((always_inline)) {
    const bool before = ONE && j < tp;
    if (!before) j -= tp;
    const size_t at = (size_t)j * SH_KEYS * m.sn * 2;
    const char *fk = before ? gkp : gk, *fv = before ? gvp : gv;
    const unsigned to = lds0 + (unsigned)(stage * 2 * TILE + wave * 64) * 16;
    const int last = (before ? p.P : nk) - 1 - j * SH_KEYS;
    if (last >= SH_KEYS - 1) {
      if (once) {
#pragma unroll
        for (int x = 0; x < COPIES; ++x) {
          dma_b128_once(fk + at, offs[x], to + x * (W * 1024));
          dma_b128_once(fv + at, offs[x], to + TILE * 16 + x * (W * 1024));
        }
      } else {
#pragma unroll
        for (int x = 0; x < COPIES; ++x) {
          dma_b128(fk + at, offs[x], to + x * (W * 1024));
          dma_b128(fv + at, offs[x], to + TILE * 16 + x * (W * 1024));
        }
      }
    } else {
#pragma unroll 1
      for (int x = 0; x < COPIES; ++x) {
        const int pc = (x * W + wave) * 64 + lane, r = pc / NP, c = (pc % NP) ^ swizzle<D>(r);
        const unsigned off = (unsigned)min(r, last) * step + (unsigned)c * 16;
        dma_b128(fk + at, off, to + x * (W * 1024));
        dma_b128(fv + at, off, to + TILE * 16 + x * (W * 1024));
      }
    }
  };
  // The first tile is on its way while the queries come; the wait for them is one for it too, since loads are counted in order.  From
  // there on two tiles are in flight.
  if (!ONE || j0 < j1) copy(j0, 0);
#pragma unroll
  for (int st = 0; st < KS; ++st)
#pragma unroll
    for (int x = 0; x < 4; ++x) use_now(q[st][x]);
  if (j0 + 1 < j1) copy(j0 + 1, 1);

  v16f o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[c][v] = 0.0f;
  // A value that is not finite, of a key that some queries of a tile see and others do not: 0 times it would reach those that do not.  Such
  // tiles - the last ones of a causal chunk of queries, looked at only there - have these values taken out before the
  // products; in the end they are added to the outputs of the queries that see them.
  bool taken_out = false;
  auto take_out = [&](int stage) {
    v4i* tv = &s_kv[stage][TILE];
    int odd = 0;
#pragma unroll 1
    for (int x = t; x < TILE; x += 64 * W) {
      const v4i u = tv[x];
#pragma unroll
      for (int y = 0; y < 4; ++y) odd |= not_finite<BF16>((unsigned)u[y] & 0xffff) || not_finite<BF16>((unsigned)u[y] >> 16);
    }
    if (__syncthreads_or(odd) == 0) return;
    taken_out = true;
#pragma unroll 1
    for (int x = t; x < TILE; x += 64 * W) {
      v4i u = tv[x];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if (not_finite<BF16>((unsigned)u[y] & 0xffff)) u[y] &= (int)0xffff0000;
        if (not_finite<BF16>((unsigned)u[y] >> 16)) u[y] &= 0xffff;
      }
      tv[x] = u;
    }
    __syncthreads();
  };
  // Values behind the last key (copies of the last, which need not be finite): zeros
  auto clear = [&](int stage, int from) {
#pragma unroll 1
    for (int x = from * NP + t; x < TILE; x += 64 * W) {
      int zero = 0;
      asm volatile("" : "+v"(zero));              // (or four registers of zeros would be kept over the loop)
      s_kv[stage][TILE + x] = v4i{zero, zero, zero, zero};
    }
    __syncthreads();
  };
  float mx = -INFINITY, l = 0.0f;                 // running maximum (of both halves; fp16: less 14) and this half's sum

  // Where my operands start in a tile.  A row's first byte has its low bits zero and the swizzle of a row repeats every 16 rows, so a
  // step to another piece of a row is one exclusive or and a step of 16 or 32 rows an offset: no address is kept over the loop.
  // K: row of key 16 (g / 2) + 8h + 4 (g % 2) + r for operand row 8g + 4h + r, piece 2 st + half.  V: row 8 half + (l % 16) / 4 - the
  // transposed read gives lane l channel l % 16 of the four keys whose rows its group of 16 lanes point at - and, for
  // the upper four keys, four rows on, where the swizzle differs in its lowest bit.
  constexpr unsigned ROW = D * 2;
  typedef __attribute__((address_space(3))) const v4i* lds_v4i;
  typedef short v4s __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4s* lds_v4s;
  const int kr = 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3), vr = 8 * half + ((lane & 15) >> 2);
  const int vc = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);                  // first channel that my lane points at
  const unsigned k_at = (unsigned)row_piece<D>(kr, half) * 16, v_at = ((unsigned)row_piece<D>(vr, vc >> 3) * 16 + (vc & 4) * 2) ^ (kg * (CT / 2) * 64);

  // NS times 32 keys of a tile, from the sub0-th on: scores, weights and their product with V
  auto tile_keys = [&](auto ns, unsigned stage0, int tile0, int sub0, int vis, int vis_all) __attribute__((always_inline)) {
    constexpr int NS = decltype(ns)::value;
    const int key0 = tile0 + 32 * sub0;
    // S^T = K Q^T: with the rows as above, half h of the lanes has keys 8h + 0..7 and 16 + 8h + 0..7 of its query, in the order in
    // which the second product wants them
    const unsigned ka = stage0 + 32 * sub0 * ROW + k_at, va = stage0 + TILE * 16 + 32 * sub0 * ROW + v_at;
    v16f sc[NS];
#pragma unroll
    for (int y = 0; y < NS; ++y)
#pragma unroll
      for (int v = 0; v < 16; ++v) sc[y][v] = 0.0f;
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int y = 0; y < NS; ++y) sc[y] = mfma16<BF16>(*(lds_v4i)(uintptr_t)((ka ^ (32 * st)) + 32 * y * ROW), q[st], sc[y]);
    if (key0 + 32 * NS > vis_all) {
#pragma unroll
      for (int y = 0; y < NS; ++y)
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[y][v] = key0 + 32 * y + 16 * (v >> 3) + 8 * half + (v & 7) < vis ? sc[y][v] : -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v)
#pragma unroll
      for (int y = 0; y < NS; ++y) top = fmaxf(top, sc[y][v]);
    top = half_max(top) * p.kappa;
    // (m is a whole step or less off for scores below 2^24, so weights stay below 2^15; beyond, where a step of 14 may be lost, none is taken)
    if (!BF16) top = fabsf(top) < 16777216.0f ? top - 14.0f : top;
    const float m_new = fmaxf(mx, top);
    const float base = m_new == -INFINITY ? 0.0f : m_new;       // (no key seen yet: every weight 2^-inf)
    if (__ballot(m_new > mx) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(mx - base);
      l *= alpha;
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[c][v] *= alpha;
      mx = m_new;
    }
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    v4i pb[NS][2];
#pragma unroll
    for (int y = 0; y < NS; ++y)
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        const float e0 = __builtin_amdgcn_exp2f(__fmaf_rn(sc[y][v], p.kappa, -base));
        const float e1 = __builtin_amdgcn_exp2f(__fmaf_rn(sc[y][v + 1], p.kappa, -base));
        sum[v & 2] += e0;
        sum[(v & 2) + 1] += e1;
        pb[y][v >> 3][(v & 7) >> 1] = (int)pack16x2<BF16>(e0, e1);
      }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    // O^T += V^T P^T
#pragma unroll
    for (int y = 0; y < NS; ++y)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          const unsigned rows = (32 * y + 16 * ks) * ROW;
          const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)((va ^ (64 * c)) + rows));
          const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)((va ^ (64 * c + 16)) + rows + 4 * ROW));
          const v8s a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          o[c] = mfma16<BF16>(__builtin_bit_cast(v4i, a), pb[y][ks], o[c]);
        }
      }
  };

  constexpr int PER_TILE = 2 * COPIES;            // copies of a tile that a wavefront starts
  for (int j = j0; j < j1; ++j) {
    const int stage = (j - j0) & 1;
    if (j + 1 < j1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PER_TILE) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();                 // tile j is there
    asm volatile("" ::: "memory");
    const unsigned at = lds0 + (unsigned)stage * (2 * TILE * 16);
    const bool before = ONE && j < tp;
    const int tile0 = (before ? j : j - tp) * SH_KEYS, end = before ? p.P : nk;
    const int seen = before ? p.P : vis, seen_all = before ? p.P : vis_all;
    if (tile0 + SH_KEYS > end) clear(stage, end - tile0);
    if (!before && part_seen && tile0 + SH_KEYS > vis_all) take_out(stage);
    if (active) {
      if (D < 256 && WK == 1 && tile0 + 32 < end) tile_keys(std::integral_constant<int, 2>{}, at, tile0, 0, seen, seen_all);
      else for (int sub = kg; sub < 2 && tile0 + 32 * sub < end; sub += WK) tile_keys(std::integral_constant<int, 1>{}, at, tile0, sub, seen, seen_all);
    }
    if (j + 2 < j1) {                             // the next tile but one takes this one's place when all have read it
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      copy(j + 2, stage);
    }
  }
  l = half_sum(l);

  // ---- the two key groups of the same rows into one
  if (WK == 2) {
    v4f* x = reinterpret_cast<v4f*>(&s_kv[0][0]);
    __syncthreads();
    if (active) {
#pragma unroll
      for (int c = 0; c < CT / 2; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          x[((wave * (CT / 2) + c) * 4 + g) * 64 + lane] = v4f{o[CT / 2 + c][4 * g], o[CT / 2 + c][4 * g + 1], o[CT / 2 + c][4 * g + 2], o[CT / 2 + c][4 * g + 3]};
      if (half == 0) {
        s_ml[wave][2 * col] = mx;
        s_ml[wave][2 * col + 1] = l;
      }
    }
    __syncthreads();
    if (active) {
      const int other = wave ^ 1;
      const float m1 = s_ml[other][2 * col], l1 = s_ml[other][2 * col + 1];
      const float m_new = fmaxf(mx, m1), base = m_new == -INFINITY ? 0.0f : m_new;
      const float a0 = __builtin_amdgcn_exp2f(mx - base), a1 = __builtin_amdgcn_exp2f(m1 - base);
      l = l * a0 + l1 * a1;
      mx = m_new;
#pragma unroll
      for (int c = 0; c < CT / 2; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const v4f y = x[((other * (CT / 2) + c) * 4 + g) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[c][4 * g + e] = o[c][4 * g + e] * a0 + y[e] * a1;
        }
    }
  }
  if (!active || rg * 32 + col >= nr) return;
  const int mine = kg * (CT / 2);                 // channel tile of o[c]: c ^ mine; mine to write are CT / 2 of them, or all
  if (taken_out) {
    const int to = min(vis, (j1 - tp) * SH_KEYS);
#pragma unroll 1
    for (int k = max(vis_all, (j0 - tp) * SH_KEYS) / SH_KEYS * SH_KEYS; k < to; ++k) {      // (whole tiles were looked at)
      const char* v = gv + (size_t)k * step + 8 * half;
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const uint2 u = *reinterpret_cast<const uint2*>(v + 64 * (c ^ mine) + 16 * g);
          const unsigned y[4] = {u.x & 0xffff, u.x >> 16, u.y & 0xffff, u.y >> 16};
#pragma unroll
          for (int e = 0; e < 4; ++e) o[c][4 * g + e] += not_finite<BF16>(y[e]) ? load16<BF16>((unsigned short)y[e]) : 0.0f;
        }
    }
  }
  if constexpr (ONE) {
    const bool none = mx == -INFINITY && l == 0.0f;      // no key at all: zeros
    const float inv = none ? 0.0f : __fdiv_rn(1.0f, l);
    if (p.lse && half == 0 && kg == 0)
      p.lse[((size_t)rb * p.H + hkv * p.G + rh) * p.N + rn] = none ? -INFINITY : LN2 * (mx + __builtin_amdgcn_logf(l));
    unsigned short* y = p.out + qrow + 4 * half;
#pragma unroll
    for (int c = 0; c < CT; ++c)
      if (c < CT / 2 || WK == 1) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<uint2*>(y + 32 * (c ^ mine) + 8 * g) = make_uint2(pack16x2<BF16>(o[c][4 * g] * inv, o[c][4 * g + 1] * inv),
                                                                             pack16x2<BF16>(o[c][4 * g + 2] * inv, o[c][4 * g + 3] * inv));
      }
    return;
  }
  const size_t pr = part_row(p, sp, (int)hkv, i);
  if (half == 0 && kg == 0) {
    p.part_ml[pr * 2] = mx;
    p.part_ml[pr * 2 + 1] = l;
  }
  float* po = p.part_o + pr * D + 4 * half;
#pragma unroll
  for (int c = 0; c < CT; ++c)
    if (c < CT / 2 || WK == 1) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const v4f y = {o[c][4 * g], o[c][4 * g + 1], o[c][4 * g + 2], o[c][4 * g + 3]};
        *reinterpret_cast<v4f*>(po + 32 * (c ^ mine) + 8 * g) = y;
      }
    }
}

// The partial results of a row into its output, a wavefront per row, or per 64 channels of 256 (7.2 us, so 6.0, for 480 rows of 34 partial
// results; of 128 channels halves cost 1 to 4 us on large batches): lane s looks at partial results s, s + 64, .. for the
// maximum and the weights; then a lane takes four channels of every GRP-th partial result, MERGE_LOADS of them in flight.  Bound by
// the two trips to memory, not by bytes.  Scores that are NaN leave their mark in the sum, whatever the maximum.
template <int D> constexpr int merge_channels() { return D == 256 ? 64 : D; }
constexpr int MERGE_LOADS = 8, MERGE_PER_LANE = 4;
constexpr int MAX_PARTS = 64 * MERGE_PER_LANE;
template <int D, bool BF16>
__global__ void __launch_bounds__(256) k_shared_merge(const SharedParams p) {
  constexpr int MC = merge_channels<D>(), LPR = MC / 4, GRP = 64 / LPR, SLICES = D / MC;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned row = (blockIdx.y * gridDim.x + blockIdx.x) * (4 / SLICES) + (unsigned)wave / SLICES;
  if (row >= (unsigned)(p.B * p.G * p.N * p.Hkv)) return;
  const int hkv = (int)split_by(row, p.by_rows);
  const long long i = row;
  unsigned n = row;
  const int b = (int)split_by(n, p.by_gn), g = (int)split_by(n, p.by_n);
  const int S = p.Sp + p.So, c = MC * (wave % SLICES) + 4 * (lane % LPR), grp = lane / LPR;
  float ms[MERGE_PER_LANE], w[MERGE_PER_LANE], m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int x = 0; x < MERGE_PER_LANE; ++x) {
    ms[x] = -INFINITY; w[x] = 0.0f;
    if (64 * x + lane < S) {
      const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + part_row(p, 64 * x + lane, hkv, i) * 2);
      ms[x] = ml.x; w[x] = ml.y;
    }
    m = fmaxf(m, ms[x]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
#pragma unroll
  for (int x = 0; x < MERGE_PER_LANE; ++x) {
    const float ls = w[x];
    w[x] = ms[x] == -INFINITY && ls == 0.0f ? -1.0f : __builtin_amdgcn_exp2f(ms[x] - m);    // (-1: no key is seen: O may not even be there)
    if (w[x] != -1.0f) l = __fmaf_rn(w[x], ls, l);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o);
  v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int x = 0; x < MERGE_PER_LANE; ++x) {
    const int end = min(S - 64 * x, 64);
    for (int s0 = 0; s0 < end; s0 += GRP * MERGE_LOADS) {
      v4f o4[MERGE_LOADS];
      float ws[MERGE_LOADS];
#pragma unroll
      for (int k = 0; k < MERGE_LOADS; ++k) {
        const int s = s0 + k * GRP + grp;
        ws[k] = __shfl(w[x], s & 63);
        ws[k] = s < end ? ws[k] : -1.0f;
        o4[k] = *reinterpret_cast<const v4f*>(p.part_o + part_row(p, 64 * x + min(s, end - 1), hkv, i) * D + c);
      }
#pragma unroll
      for (int k = 0; k < MERGE_LOADS; ++k)
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[y] = ws[k] == -1.0f ? acc[y] : __fmaf_rn(ws[k], o4[k][y], acc[y]);
    }
  }
#pragma unroll
  for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
    for (int y = 0; y < 4; ++y) acc[y] += __shfl_xor(acc[y], o);
  if (grp != 0) return;
  const int h = hkv * p.G + g;
  const bool none = m == -INFINITY && l == 0.0f;  // no key at all: zeros
  const float inv = none ? 0.0f : __fdiv_rn(1.0f, l);
  if (p.lse && c == 0) p.lse[((size_t)b * p.H + h) * p.N + n] = none ? -INFINITY : LN2 * (m + __builtin_amdgcn_logf(l));
  unsigned short* y = p.out + row_offset(p.qm, head_offset_of(p.qm, b, h), (int)n) + c;
  *reinterpret_cast<uint2*>(y) = make_uint2(pack16x2<BF16>(acc[0] * inv, acc[1] * inv), pack16x2<BF16>(acc[2] * inv, acc[3] * inv));
}

// Tiles of a key chunk.  The chip has room for 256, 512 or 768 workgroups (of 256, 128, 64 channels), and each has its start to pay
// for, so 512 / d tiles at least.  A workgroup of the prefix takes an even share of all tiles - it has up to 128 rows of partial
// results to leave - and where it has few rows and is bound by reading, so many that there is one to a CU.  The own keys of a
// sequence have few rows, and lengths that the host does not know: they are cut finer, 12 tiles at most, so that the chip fills up to
// the end.  Us, an even share for both / this, caches read from memory: 64 sequences of up to 4096 tokens over 32768, 128 channels 173 /
// 158; 1 of 300 over 32768 32.4 / 32.1; 4 of 2000 over 100000 84 / 76; 32 of 3000 over 200 55.9 / 54.3.
void choose_chunks(SharedParams* p, int d, long long rows) {
  const long long tp = (p->P + SH_KEYS - 1) / SH_KEYS, to = (p->Nk + SH_KEYS - 1) / SH_KEYS;
  // So few tiles that a workgroup is over them before a second kernel could start: one launch, in which each sequence reads the prefix for
  // itself.  (Us, chunks / this: 4 heads of 300 + 50 keys of 64 channels 17.7 / 15.1, 128 of 380 + 128 of 128 16.6 / 15.2, of 500 + 250 16.7 /
  // 19.6; of 256 channels 128 of 180 + 60 18.2 / 14.9, of 300 + 50 18.2 / 18.5; 512 of 60 + 60 29.6 / 19.5.)
  p->one = tp + to <= 2 + 640 / d;
  if (p->one) {
    p->Sp = p->So = 0;
    return;
  }
  const long long prefix = (long long)p->Hkv * p->rtp * tp, own = (long long)p->B * p->Hkv * p->rto * to;
  const long long places = 256LL * (d == 64 ? 3 : d == 128 ? 2 : 1), least = 512 / d;
  long long share = (prefix + own + places - 1) / places;
  if (rows <= 64) share = std::max(share, (prefix + 255) / 256);
  const long long pp = std::max(least, share), po = std::max(least, std::min(12LL, (own + places - 1) / places));
  // The merge takes MAX_PARTS in all: half for each part, and what the other leaves where half would leave places of the chip empty, with one KV head
  // or two.  (Us, half / this: 1 sequence of 1000000 own keys, one KV head of 128 channels 160 / 97; 1 of 512 over 131072 35.8 / 33.5; 4
  // over 200000 of 256 channels 73 / 50; 8 of 200000 own keys, where half does, 143, with all 153.)
  const long long wp = (tp + pp - 1) / pp, wo = (to + po - 1) / po, half = MAX_PARTS / 2;
  const long long fp = places / ((long long)p->Hkv * p->rtp), fo = places / ((long long)p->B * p->Hkv * p->rto);
  p->Sp = (int)std::min(wp, std::max(half, std::min(MAX_PARTS - wo, fp)));
  p->So = (int)std::min(wo, std::max(half, std::min(MAX_PARTS - wp, fo)));
}

int shared_params(const sage_attn_shared_prefix_args* a, SharedParams* p, bool need_io) {
  if (!a || a->B <= 0 || a->H <= 0 || a->H_kv <= 0 || a->N <= 0 || a->N_prefix < 0 || a->N_kv < 0) return SAGE_ERR_INVALID_ARG;
  if (a->H % a->H_kv != 0) return SAGE_ERR_INVALID_ARG;
  if (a->d != 64 && a->d != 128 && a->d != 256) return SAGE_ERR_UNSUPPORTED;
  if (a->dtype != SAGE_DT_FP16 && a->dtype != SAGE_DT_BF16) return SAGE_ERR_UNSUPPORTED;
  if (a->layout != SAGE_LAYOUT_HND && a->layout != SAGE_LAYOUT_NHD) return SAGE_ERR_UNSUPPORTED;
  if (a->N > MAX_TOKENS || a->N_prefix > MAX_TOKENS || a->N_kv > MAX_TOKENS || (long long)a->B * a->H > 65535) return SAGE_ERR_UNSUPPORTED;
  if (need_io) {
    if (!a->q || !a->out || (a->N_prefix > 0 && (!a->k_prefix || !a->v_prefix)) || (a->N_kv > 0 && (!a->k || !a->v))) return SAGE_ERR_INVALID_ARG;
    if ((((uintptr_t)a->q | (uintptr_t)a->out | (uintptr_t)a->k_prefix | (uintptr_t)a->v_prefix | (uintptr_t)a->k | (uintptr_t)a->v) & 15u) != 0)
      return SAGE_ERR_INVALID_ARG;
    if ((((uintptr_t)a->lse | (uintptr_t)a->kv_lens) & 3u) != 0) return SAGE_ERR_INVALID_ARG;
  }
  p->q = (const unsigned short*)a->q; p->kp = (const unsigned short*)a->k_prefix; p->vp = (const unsigned short*)a->v_prefix;
  p->ko = (const unsigned short*)a->k; p->vo = (const unsigned short*)a->v; p->out = (unsigned short*)a->out;
  p->lse = a->lse; p->lens = a->kv_lens;
  p->B = a->B; p->H = a->H; p->Hkv = a->H_kv; p->G = a->H / a->H_kv; p->N = a->N; p->P = a->N_prefix; p->Nk = a->N_kv;
  p->causal = a->causal != 0;
  p->kappa = (a->sm_scale > 0.0f ? a->sm_scale : (float)(1.0 / std::sqrt((double)a->d))) * LOG2E;
  const int nhd = a->layout == SAGE_LAYOUT_NHD;
  p->qm = make_tensor_map(nhd, a->H, a->N, a->d);
  p->pm = make_tensor_map(nhd, a->H_kv, a->N_prefix, a->d);
  p->om = make_tensor_map(nhd, a->H_kv, a->N_kv, a->d);
  const long long gn = (long long)p->G * p->N, rows = gn * p->B;
  if (rows * p->Hkv > (1LL << 24)) return SAGE_ERR_UNSUPPORTED;
  const int per = shared_rows(a->d);
  p->rtp = (int)((rows + per - 1) / per);
  p->rto = (int)((gn + per - 1) / per);
  choose_chunks(p, a->d, rows);
  const long long np = (long long)p->Sp * p->Hkv * p->rtp, no = (long long)p->So * p->B * p->Hkv * p->rto;
  if ((np + no) * (a->d == 256 ? 64 * shared_waves<256>() : 64 * shared_waves<128>()) > MAX_THREADS) return SAGE_ERR_UNSUPPORTED;
  p->n_prefix = (int)np;
  p->full = p->Sp * a->H_kv / 8 * 8 * p->rtp;
  p->by_group = fast_div(8u * p->rtp); p->by_rtp = fast_div(p->rtp); p->by_hkv = fast_div(a->H_kv); p->by_rto = fast_div(p->rto);
  p->by_b = fast_div(a->B); p->by_gn = fast_div((unsigned)gn); p->by_n = fast_div(a->N); p->by_rows = fast_div((unsigned)rows);
  p->by_sp = fast_div(std::max(p->Sp, 1)); p->by_so = fast_div(std::max(p->So, 1));
  return SAGE_OK;
}

size_t part_rows(const SharedParams& p) { return (size_t)(p.Sp + p.So) * p.Hkv * p.B * p.G * p.N; }
size_t shared_bytes(const SharedParams& p, int d) {
  return align256(part_rows(p) * 2 * sizeof(float)) + align256(part_rows(p) * d * sizeof(float));
}

template <int D, bool BF16> hipError_t launch_shared(const SharedParams& p, hipStream_t s) {
  if (p.one) {
    k_shared<D, BF16, true><<<(unsigned)(p.B * p.Hkv * p.rto), 64 * shared_waves<D>(), 0, s>>>(p);
    return hipGetLastError();
  }
  const long long own = (long long)p.So * p.B * p.Hkv * p.rto, blocks = p.n_prefix + own;
  if (blocks > 0) {
    k_shared<D, BF16, false><<<(unsigned)blocks, 64 * shared_waves<D>(), 0, s>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // (2^24 rows of 256 channels are 2^32 threads: more than a million workgroups are in the second dimension too)
  const long long merges = ((long long)p.B * p.G * p.N * p.Hkv * (D / merge_channels<D>()) + 3) / 4, wide = std::min(merges, 1LL << 20);
  k_shared_merge<D, BF16><<<dim3((unsigned)wide, (unsigned)((merges + wide - 1) / wide)), 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace
}  // namespace sage

using namespace sage;

extern "C" size_t sage_attn_shared_prefix_workspace_bytes(const sage_attn_shared_prefix_args* a) {
  SharedParams p;
  if (shared_params(a, &p, false) != SAGE_OK) return 0;
  return shared_bytes(p, a->d);
}

extern "C" int sage_attn_shared_prefix(const sage_attn_shared_prefix_args* a) {
  SharedParams p;
  int st = shared_params(a, &p, true);
  if (st != SAGE_OK) return st;
  const size_t need = shared_bytes(p, a->d);
  if (need > 0 && (!a->workspace || a->workspace_bytes < need || ((uintptr_t)a->workspace & 255u) != 0)) return SAGE_ERR_WORKSPACE;
  // (a row's query is read before its output is written, by the same workgroup or a kernel before: out may be q)
  const size_t rows = (size_t)a->B * a->H * a->N, bytes = (size_t)a->d * 2, prefix = (size_t)a->H_kv * a->N_prefix, own = (size_t)a->B * a->H_kv * a->N_kv;
  const Span in[6] = {{a->out == a->q ? nullptr : a->q, rows * bytes}, {prefix > 0 ? a->k_prefix : nullptr, prefix * bytes}, {prefix > 0 ? a->v_prefix : nullptr, prefix * bytes},
                      {own > 0 ? a->k : nullptr, own * bytes}, {own > 0 ? a->v : nullptr, own * bytes}, {a->kv_lens, (size_t)a->B * 4}};
  const Span out[3] = {{a->out, rows * bytes}, {a->lse, rows * 4}, {need > 0 ? a->workspace : nullptr, need}};
  for (int i = 0; i < 3; ++i) {
    for (const Span& x : in) if (overlap(out[i], x)) return SAGE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j) if (overlap(out[i], out[j])) return SAGE_ERR_INVALID_ARG;
  }
  p.part_ml = (float*)a->workspace;
  p.part_o = (float*)((char*)a->workspace + align256(part_rows(p) * 2 * sizeof(float)));
  const hipStream_t s = (hipStream_t)a->stream;
  const bool bf16 = a->dtype == SAGE_DT_BF16;
  hipError_t e;
  if (a->d == 64) e = bf16 ? launch_shared<64, true>(p, s) : launch_shared<64, false>(p, s);
  else if (a->d == 128) e = bf16 ? launch_shared<128, true>(p, s) : launch_shared<128, false>(p, s);
  else e = bf16 ? launch_shared<256, true>(p, s) : launch_shared<256, false>(p, s);
  return op_status(e);
}
