// Attention over a cache of 8 bits and pages (sage_attn_paged).
//
// O = softmax(kappa Q K^T) V with K = codes 2^ek, V = codes 2^ev, one exponent for each block of 32 tokens.  E4M3 codes are exact in both 16-bit types, so
// Q stays as it is and the products are 16-bit ones with FP32 sums.  A block is one 32 x 32 tile of scores: 2^ek is a scalar beside kappa, 2^ev goes into the instruction
// that converts the codes of V.  Softmax in one pass with the running maximum m and sum l (Sec. 2.1, Eq. 1); chunks of the keys are independent workgroups that leave
// (m, l, O), and a second kernel merges them: O = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i.
// P is rounded to the 16-bit type for its product with V (half a step, which averages out over the keys).  fp16 has no numbers for weights below 2^-25 of the largest, which
// are in the sum all the same: there m is kept 14 below the maximum, so that weights are up to 2^14 and vanish from 2^-39 of the largest on.
//
// With few queries it reads the cache and nothing else should bound it.  A block's K (or V) is 32 d contiguous bytes whatever the size of a page; each wavefront copies its own blocks
// into LDS, two tiles ahead.  Where all queries of a KV head are 32 rows at most (256 channels: 16), it also attends to just those blocks, with no barrier; more rows are divided over the wavefronts.
// 32 heads of 128 over 8: 16 sequences of up to 32768 tokens 115 to 124 us by card (5.7 to 6.0 TB/s), 32 in a window of 4096 47.6 us (5.7 TB/s).  Chunks of 512 queries over 2 x 16384 tokens 263 to 288 us
// (0.76 to 0.83 PFLOP/s), bound by vector issue: of some 170 instructions of a block 64 widen its codes.  A lone workgroup takes 5 us to its first tile and from its last, and 0.65 us a tile.
#include "sage_paged.h"

#include <algorithm>
#include <type_traits>

namespace sage {
namespace {

constexpr int PT_BLOCKS = 4;         // blocks of a tile: one for each wavefront to copy

struct PagedParams {
  PagedCache c;
  const unsigned short* q;
  unsigned short* out;
  float* lse;
  const int *lens, *qlens;
  float *part_o, *part_ml;           // [chunk][B H_kv][G N][d], [chunk][B H_kv][G N][2]
  TensorMap qm;
  int B, H, N, G, cap;               // cap: max_pages * page
  int causal, window, sink, clear;
  float kappa;                       // sm_scale log2(e)
  int S, rt, units;                  // key chunks, row tiles, workgroups of one row tile: B H_kv S
  FastDiv by_rt8, by_s, by_hkv, by_g, by_gn;      // 8 rt, S, H_kv, G, G N
};

__device__ __forceinline__ int len_of(const PagedParams& p, int b) { return p.lens ? min(max(p.lens[b], 0), p.cap) : p.cap; }
__device__ __forceinline__ int count_of(const PagedParams& p, int b) { return p.qlens ? min(max(p.qlens[b], 0), p.N) : p.N; }

// The tokens that the query at `pos` sees: t < to, and t >= from or t < sink.
struct Seen { int sink, from, to; };
__device__ __forceinline__ Seen seen_from(const PagedParams& p, int len, int pos) {
  Seen s;
  s.to = p.causal ? min(len, pos + 1) : len;
  s.from = p.window > 0 ? max(pos + 1 - p.window, 0) : 0;
  s.sink = p.window > 0 ? min(p.sink, s.to) : 0;
  return s;
}
__device__ __forceinline__ bool sees(const Seen& s, int t) { return t < s.to && (t >= s.from || t < s.sink); }

// A block in LDS: 32 rows of D bytes, D / 16 pieces of 16; piece c of row r stands at piece c ^ turn(r), so that the pieces which a matrix operand takes together -
// the same one of rows 0..3 and 8..11, or of rows 0..7 - fall on different banks.
template <int D> __device__ __forceinline__ int turn(int r) {
  const int x = ((r >> 2) ^ (r >> 3)) & 1;
  if constexpr (D == 64) return ((r >> 1) & 1) | x << 1;
  return (r & 3) | x << 2;
}

// Eight codes (two dwords) as 16-bit numbers times a power of two: exact but below fp16's normal numbers.
template <bool BF16> __device__ __forceinline__ v4i widen(int u, int w, float scale) {
  v4i a;
  if constexpr (BF16) {
    a[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)u, scale, false));
    a[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)u, scale, true));
    a[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w, scale, false));
    a[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w, scale, true));
  } else {
    a[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)u, scale, false));
    a[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)u, scale, true));
    a[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)w, scale, false));
    a[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)w, scale, true));
  }
  return a;
}

// A byte of each active lane's own address into LDS, a dword a lane.
__device__ __forceinline__ void dma_u8(const void* from, unsigned lds_byte) {
  unsigned m0_after;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ubyte %2, off" : "={m0}"(m0_after) : "s"(lds_byte), "v"(from) : "memory");
}

// Sum / maximum of a value over the four lanes 16 apart, in all of them.
__device__ __forceinline__ float quarter_sum(float x) {
  const unsigned u = __float_as_uint(half_sum(x));
  const auto sw = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}
__device__ __forceinline__ float quarter_max(float x) {
  const unsigned u = __float_as_uint(half_max(x));
  const auto sw = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

// Wavefronts that share their rows' channels: of 256, whose outputs and queries would take all registers of a SIMD with 32 rows, two form the same scores and have half of the
// outputs each.  (One on a SIMD with 512 registers: 6 caches of 5120, 5 queries of 4 heads, window 3001: 30 us, so 20.)
template <int D, int COLS> constexpr int channel_groups() { return D == 256 && COLS == 32 ? 2 : 1; }
template <int D, int COLS> constexpr int paged_threads() { return 256 * channel_groups<D, COLS>(); }
template <int D, int COLS> constexpr int paged_occupancy() { return D == 64 ? (COLS == 16 ? 4 : 3) : 2; }   // wavefronts per SIMD

// COLS: rows of a wavefront, the columns of its score tiles: 32 (32 x 32 products, two parts of the lanes with eight tokens a step) or, with few, 16 (16 x 16, four parts), which halves the
// products, the exponentials and the chain of products that a block's scores are.
// RG: groups of them in a workgroup.  Its wavefronts are RG row groups times KG = 4 / RG key groups (which take the blocks kg, kg + KG, .. of a tile) times CG channel groups.
// ONE: a workgroup takes all keys and leaves the output itself.
// Two tiles are in LDS, the one that is attended to and the next.  (Four, where no other workgroup needs the room: 8 x 8 tiles of 128 channels 12.0 us, with two 11.6; it is a
// wavefront's chain of instructions, 0.75 us a block, that a tile takes where few are busy.)  They are dynamic LDS: were their size known, the compiler would see one wavefront on a SIMD with 256
// channels, hence 512 registers, and move outputs to and from the upper ones (4 x 8192 of 16 heads 16.0 us, so 14.6).
template <int D> constexpr unsigned lds_bytes() { return 2 * PT_BLOCKS * 2 * BLOCK * D; }
template <int D, bool BF16, int COLS, int RG, bool ONE>
__global__ void __launch_bounds__((paged_threads<D, COLS>()), (paged_occupancy<D, COLS>())) k_paged(const PagedParams p) {
  constexpr int CG = channel_groups<D, COLS>(), THREADS = paged_threads<D, COLS>();
  constexpr bool WIDE = COLS == 32;
  constexpr int KS = D / (WIDE ? 16 : 32), KST = WIDE ? 2 : 1;      // contraction steps of the two products
  constexpr int ST = WIDE ? 1 : 2, NSC = WIDE ? 16 : 8;            // score tiles of a block; scores of a lane
  constexpr int CT = D / COLS / CG, AV = WIDE ? 16 : 4;            // channel tiles of a wavefront, values of one in a lane
  constexpr int KG = 4 / RG, ROWS = COLS * RG;
  typedef typename std::conditional<WIDE, v16f, v4f>::type acc_t;
  constexpr bool SHARED = RG > 1 || CG > 1;       // wavefronts read blocks that others copied
  constexpr unsigned BYTES = BLOCK * D;           // of a block of K or V
  constexpr int COPIES = D / 32;                  // copies of 64 pieces of a block of K (or V)
  extern __shared__ __align__(1024) v4i s_kv[];   // [stage][block][K, V]
  __shared__ float s_ml[4 * CG][64];
  __shared__ unsigned s_scale[4 * CG][2][64];     // of the blocks in at_lo, at_hi: K's, V's
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int col = lane & (COLS - 1), part = lane / COLS, cg = wave % CG, own = wave / CG, kg = own % KG, rg = own / KG;      // own: the block of a tile that this one copies

  // The arguments take five cache lines: one wait for all of them, not one for each where its first word is needed
  asm volatile("" ::"s"(p.c.table), "s"(p.c.by_bpp.m), "s"(p.lens), "s"(p.qm.sn), "s"(p.kappa), "s"(p.by_s.m), "s"(p.by_gn.m));

  // ---- which rows and keys.  The row tiles of the same keys are 8 apart: workgroups go to the 8 XCDs in turn and each has a cache of its own.
  unsigned rt = blockIdx.x;
  unsigned unit = split_by(rt, p.by_rt8) * 8 + rt % 8;
  rt /= 8;
  if ((int)unit >= p.units) return;
  unsigned s = unit;
  const unsigned bh = split_by(s, p.by_s);
  unsigned hkv = bh;
  const unsigned b = split_by(hkv, p.by_hkv);
  const int len = len_of(p, (int)b), count = count_of(p, (int)b);
  const int rows = count * p.G, r0 = (int)rt * ROWS, nr = min(ROWS, rows - r0);      // rows: (query, head of the group)
  if (p.clear != 0 && s == 0) {                   // rows behind the last query
    for (int i = max(r0, rows) + t / (D / 8); i < min(r0 + ROWS, p.N * p.G); i += THREADS / (D / 8)) {
      unsigned g = (unsigned)i;
      const unsigned n = split_by(g, p.by_g), h = hkv * p.G + g;
      if (p.clear & SAGE_CLEAR_OUT) *reinterpret_cast<uint4*>(p.out + row_offset(p.qm, head_offset_of(p.qm, (int)b, (int)h), (int)n) + 8 * (t % (D / 8))) = make_uint4(0, 0, 0, 0);
      if ((p.clear & SAGE_CLEAR_LSE) && p.lse && t % (D / 8) == 0) p.lse[((size_t)b * p.H + h) * p.N + n] = 0.0f;
    }
  }
  if (nr <= 0) return;
  const int coff = max(len - count, 0);
  const Seen first = seen_from(p, len, coff + (int)div_by((unsigned)r0, p.by_g)), last = seen_from(p, len, coff + (int)div_by((unsigned)(r0 + nr - 1), p.by_g));
  // Blocks that some row sees: those of the sinks, then from the first row's window to the last row's end
  const int ns = (last.sink + BLOCK - 1) / BLOCK, w0 = max(ns, first.from / BLOCK), nb = ns + max((last.to + BLOCK - 1) / BLOCK - w0, 0);
  const int tiles = (nb + PT_BLOCKS - 1) / PT_BLOCKS;
  int j0 = 0, j1 = tiles;
  if constexpr (!ONE) {
    const int per = (int)div_by((unsigned)(tiles + p.S - 1), p.by_s);
    j0 = min((int)s * per, tiles);
    j1 = min(j0 + per, tiles);
  }
  const bool active = rg * COLS < nr;
  const size_t part0 = ((size_t)s * (p.B * p.c.Hkv) + bh) * ((size_t)p.G * p.N) + r0;      // of the partial results' rows
  if (!ONE && j0 >= j1) {                         // no keys: a partial result that the merge skips
    for (int i = t; i < nr; i += THREADS) {
      p.part_ml[(part0 + i) * 2] = -INFINITY;
      p.part_ml[(part0 + i) * 2 + 1] = 0.0f;
    }
    return;
  }

  // ---- my row's query as the B operand: 16 channels of each part are two steps
  const int i0 = r0 + min(rg * COLS + col, nr - 1);
  unsigned rh = (unsigned)i0;
  const unsigned rn = split_by(rh, p.by_g);
  const size_t qrow = row_offset(p.qm, head_offset_of(p.qm, (int)b, (int)(hkv * p.G + rh)), (int)rn);
  v4i q[KS];
#pragma unroll
  for (int st = 0; st < KS; ++st) q[st] = *reinterpret_cast<const v4i*>(p.q + qrow + 16 * ((64 / COLS) * (st >> 1) + part) + 8 * (st & 1));
  const Seen mine = seen_from(p, len, coff + (int)rn);
  // ---- where the next 16 tiles' blocks are in the pool, one block a lane, and their scales, which go to LDS like the blocks do, so that no wait for them is one for what
  // is copied after them.  Half of the lanes are refilled every 8 tiles.
  int at_lo = -1, at_hi = -1, token0 = 0;        // (no page, or past the last block: -1); the block's first token
  unsigned about = 0;                             // its scales, K's and V's, and from bit 16 on whether there is one, whether all rows see all of it and
  constexpr unsigned OUTER = 1u << 18;            // whether its scores may be FAR from zero, or kappa times K's scale is beyond FP32
  float factor = 0.0f;                            // kappa times K's
  auto fetch = [&](int j, int from, int to) __attribute__((always_inline)) {      // lanes from .. to - 1, the first of them tile j's first block
    const int i = 4 * j + lane - from;
    if (lane < from || lane >= to) return;
    long long at = -1;
    const int block = i < ns ? i : i - ns + w0;
    if (i < nb) at = pool_block(p.c, (int)b, (int)hkv, block);
    token0 = BLOCK * block;
    at_lo = (int)at; at_hi = (int)(at >> 32);
    if (at < 0) return;
    const unsigned dst = (unsigned)(size_t)(__attribute__((address_space(3))) char*)&s_scale[wave][0][0];
    dma_u8(p.c.ks + at, dst);
    dma_u8(p.c.vs + at, dst + 256);
  };
  fetch(j0, 0, 64);
#pragma unroll
  for (int st = 0; st < KS; ++st)                 // (the queries are there with the page numbers: no wait for them is one for a copy)
#pragma unroll
    for (int x = 0; x < 4; ++x) use_now(q[st][x]);
  // What a score (to the base 2) of these rows may reach, for a K scale of 1: the largest magnitude of a query times 448, d of them.  Infinities and NaN make their own scores whatever they make.
  // (32 caches in a window of 4096 take 0.3 us more for it.  Looked for block by block instead, far scores cost chunks of 512 queries 2 %.  Where all blocks are such, these take 675 us for 285, a step over
  // 32768 tokens 147 for 126.)
  unsigned most = 0;
#pragma unroll
  for (int st = 0; st < KS; ++st)
#pragma unroll
    for (int x = 0; x < 4; ++x) most = larger_pair(most, (unsigned)q[st][x] & 0x7fff7fff);
  most = largest_of_all(most);
  if (most >= (BF16 ? 0x7f80u : 0x7c00u)) {
    most = 0;
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int x = 0; x < 4; ++x) most = larger_pair(most, finite_pair<BF16>((unsigned)q[st][x]));
    most = largest_of_all(most);
  }
  const float reach = load16<BF16>((unsigned short)most) * (448.0f * D) * p.kappa;

  // ---- copies
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)&s_kv[0];
  unsigned offs[COPIES];
#pragma unroll
  for (int x = 0; x < COPIES; ++x) {
    const int pc = x * 64 + lane, r = pc / (D / 16);
    offs[x] = (unsigned)(r * D + ((pc % (D / 16)) ^ turn<D>(r)) * 16);
  }
  const bool once = p.rt == 1;                    // what one workgroup alone reads passes the caches by (16 x 32768: 123 us, through them 135)
  auto copy = [&](int j, int stage) __attribute__((always_inline)) -> bool {      // my block of tile j; whether there is one
    const int at_lane = ((j - j0) & 15) * 4 + own;
    const int hi = __builtin_amdgcn_readlane(at_hi, at_lane);
    if (hi < 0) return false;
    const size_t at = (size_t)((unsigned long long)(unsigned)hi << 32 | (unsigned)__builtin_amdgcn_readlane(at_lo, at_lane)) * BYTES;
    const unsigned to = lds0 + (unsigned)(stage * PT_BLOCKS + own) * (2 * BYTES);
    if constexpr (CG == 1) {
      const unsigned char *gk = p.c.k + at, *gv = p.c.v + at;
      if (once) {
#pragma unroll
        for (int x = 0; x < COPIES; ++x) {
          dma_b128_once(gk, offs[x], to + x * 1024);
          dma_b128_once(gv, offs[x], to + BYTES + x * 1024);
        }
      } else {
#pragma unroll
        for (int x = 0; x < COPIES; ++x) {
          dma_b128(gk, offs[x], to + x * 1024);
          dma_b128(gv, offs[x], to + BYTES + x * 1024);
        }
      }
    } else {                                      // (one the keys, the other the values)
      const unsigned char* g = (cg ? p.c.v : p.c.k) + at;
      if (once) {
#pragma unroll
        for (int x = 0; x < COPIES; ++x) dma_b128_once(g, offs[x], to + cg * BYTES + x * 1024);
      } else {
#pragma unroll
        for (int x = 0; x < COPIES; ++x) dma_b128(g, offs[x], to + cg * BYTES + x * 1024);
      }
    }
    return true;
  };
  copy(j0, 0);
  bool next = j0 + 1 < j1 && copy(j0 + 1, 1);     // whether tile j + 1 is on its way
  acc_t o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int v = 0; v < AV; ++v) o[c][v] = 0.0f;
  float mx = -INFINITY, l = 0.0f;                 // running maximum (of all parts; fp16: less 14) and this part's sum
  unsigned long long saw = 0;                     // lanes that have seen a token, whatever its score

  // Where my operands start in a block; steps to other pieces are exclusive ors.  K: rows in an order that gives each part of the lanes the scores of the tokens whose weights the
  // second product wants of it: tokens 8 part + 0..7 (32 columns: and 16 on), score i of a lane being token_of(i).  V: the transposed read gives lane l channel l % 16 of the
  // eight tokens whose rows its group of 16 lanes point at, two lanes a row.
  typedef __attribute__((address_space(3))) const v4i* lds_v4i;
  typedef __attribute__((address_space(3))) v2i* lds_v2i;
  unsigned k_at[ST];
#pragma unroll
  for (int y = 0; y < ST; ++y) {
    const int kr = WIDE ? 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3) : 8 * (col >> 2) + 4 * y + (col & 3);
    k_at[y] = (unsigned)(kr * D + (part ^ turn<D>(kr)) * 16);
  }
  const int vr = 8 * part + ((lane & 15) >> 1);
  const unsigned v_at = BYTES + ((unsigned)(vr * D + ((WIDE ? (lane >> 4) & 1 : 0) ^ turn<D>(vr)) * 16 + 8 * (lane & 1)) ^ (unsigned)(COLS * CT * cg));
  auto token_of = [&](int i) __attribute__((always_inline)) { return WIDE ? 16 * (i >> 3) + 8 * part + (i & 7) : 8 * part + i; };
  auto mfma = [](v4i x, v4i y, acc_t c) __attribute__((always_inline)) {
    if constexpr (WIDE) return mfma16<BF16>(x, y, c);
    else return mfma16_small<BF16>(x, y, c);
  };

  // One block: scores, weights and their product with V.  w: its `about`.  PART: some row does not see some token of it, its values may not fit the 16-bit type or it is OUTER; kk: kappa times
  // K's scale, or where that is beyond FP32 kappa alone, and the products are multiplied by the scale first.
  constexpr unsigned FITS = BF16 ? 246 : 134;      // 448 2^119 and 448 2^7 are numbers of the type
  constexpr float FAR = 16777216.0f;              // 2^24
  auto attend = [&](auto partly, unsigned base, int t0, float kk, unsigned w) __attribute__((always_inline)) {
    constexpr bool PART = decltype(partly)::value;
    const int ev = (int)(w >> 8 & 255);
    const float vs = scale_of(PART ? min((unsigned)ev, FITS) : (unsigned)ev);
    const unsigned va = base + v_at;              // (a block's first byte has its low bits zero: steps to other pieces need no address kept over the loop)
    acc_t tile[ST];
#pragma unroll
    for (int y = 0; y < ST; ++y)
#pragma unroll
      for (int v = 0; v < AV; ++v) tile[y][v] = 0.0f;
    constexpr int AHEAD = PART ? 1 : KS / 2 < 4 / ST ? KS / 2 : 4 / ST;      // reads of K in flight
#pragma unroll
    for (int u0 = 0; u0 < KS / 2; u0 += AHEAD) {
      v4i x[AHEAD][ST];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int y = 0; y < ST; ++y) x[u][y] = *(lds_v4i)(uintptr_t)((base + k_at[y]) ^ (16 * (64 / COLS) * (u0 + u)));
      if constexpr (!PART) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
#pragma unroll
        for (int y = 0; y < ST; ++y) tile[y] = mfma(widen<BF16>(x[u][y][0], x[u][y][1], 1.0f), q[2 * (u0 + u)], tile[y]);
#pragma unroll
        for (int y = 0; y < ST; ++y) tile[y] = mfma(widen<BF16>(x[u][y][2], x[u][y][3], 1.0f), q[2 * (u0 + u) + 1], tile[y]);
      }
    }
    // The values are read while the weights are worked out
    v2i xv[PART ? 1 : KST][CT];
    if constexpr (!PART) {
#pragma unroll
      for (int ks = 0; ks < KST; ++ks)
#pragma unroll
        for (int c = 0; c < CT; ++c) xv[ks][c] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i)(uintptr_t)((va ^ (COLS * c)) + ks * 16 * D));
      __builtin_amdgcn_sched_barrier(0);
    }
    float sc[NSC];
#pragma unroll
    for (int i = 0; i < NSC; ++i) sc[i] = tile[i / AV][i % AV];
    unsigned seen = 0xffff;                       // bit i: my row sees score i's token
    if constexpr (PART) {
      if (w & OUTER) {
        const float first_by = p.kappa * scale_of(w & 255) == INFINITY ? scale_of(w & 255) : 1.0f;
#pragma unroll
        for (int i = 0; i < NSC; ++i) sc[i] *= first_by;
      }
      seen = 0;
#pragma unroll
      for (int i = 0; i < NSC; ++i) {
        const bool see = sees(mine, t0 + token_of(i));
        seen |= (unsigned)see << i;
        sc[i] = see ? sc[i] : -INFINITY;
      }
      saw |= __ballot(seen != 0);
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NSC; ++i) top = fmaxf(top, sc[i]);
    top = (WIDE ? half_max(top) : quarter_max(top)) * kk;
    // (Up to a score of 2^24 m is a whole step or less off, so weights stay below 2^15; beyond, where a step of 14 may be lost, none is taken)
    if (!BF16) top = PART && fabsf(top) >= FAR ? top : top - 14.0f;
    const float m_new = fmaxf(mx, top);
    const float m = m_new == -INFINITY ? 0.0f : m_new;          // (no token seen yet: every weight 2^-inf)
    if (__ballot(m_new > mx) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(mx - m);
      l *= alpha;
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int v = 0; v < AV; ++v) o[c][v] *= alpha;
      mx = m_new;
    }
    // m is a rounded product and a weight's exponent is formed from the exact one, so the largest weight is 2^(that rounding): as good as 1, but from 2^24 on a whole step and soon anything.
    // There the products are rounded like m, and the largest weight is 1.  (Under such an m of another block all weights of this one are zero.)
    float by = kk;
    if constexpr (PART) {
      if (w & OUTER) {
        const bool is_far = fabsf(m) >= FAR;
#pragma unroll
        for (int i = 0; i < NSC; ++i) sc[i] = is_far ? sc[i] * kk : sc[i];
        by = is_far ? 1.0f : kk;
      }
    }
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    v4i pb[KST];
#pragma unroll
    for (int v = 0; v < NSC; v += 2) {
      float e0 = __builtin_amdgcn_exp2f(__fmaf_rn(sc[v], by, -m)), e1 = __builtin_amdgcn_exp2f(__fmaf_rn(sc[v + 1], by, -m));
      if constexpr (PART) {                       // (where kk is NaN, or m infinite, a hidden token's weight would not be zero)
        e0 = seen >> v & 1 ? e0 : 0.0f;
        e1 = seen >> (v + 1) & 1 ? e1 : 0.0f;
      }
      sum[v & 2] += e0;
      sum[(v & 2) + 1] += e1;
      pb[v >> 3][(v & 7) >> 1] = (int)pack16x2<BF16>(e0, e1);
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    if constexpr (!PART) {
#pragma unroll
      for (int ks = 0; ks < KST; ++ks)
#pragma unroll
        for (int c = 0; c < CT; ++c) o[c] = mfma(widen<BF16>(xv[ks][c][0], xv[ks][c][1], vs), pb[ks], o[c]);
    } else {
      // A NaN among V times a weight of zero would reach rows that do not see it: NaN is taken out before the product.  How many of a channel's a row sees is a product
      // too, of ones; where that is not zero, the output is NaN.  What no row sees counts as zeros.
      constexpr unsigned UNIT = BF16 ? 0x3f80 : 0x3c00;
      const float more = (unsigned)ev <= FITS ? 1.0f : scale_of(127 + (unsigned)ev - FITS);      // what vs leaves out
      v4i sb[KST];
      unsigned keep[KST][2];                      // bytes of tokens that some row sees
#pragma unroll
      for (int ks = 0; ks < KST; ++ks)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          keep[ks][y] = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = t0 + token_of(8 * ks + 4 * y + e);
            keep[ks][y] |= tok < last.to && (tok >= first.from || tok < last.sink) ? 0xffu << (8 * e) : 0u;
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const unsigned two = seen >> (8 * ks + 4 * y + 2 * e);
            sb[ks][2 * y + e] = (int)((two & 1 ? UNIT : 0u) | (two & 2 ? UNIT << 16 : 0u));
          }
        }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        unsigned nan[KST][2], any = 0;
        acc_t sum_of;
#pragma unroll
        for (int v = 0; v < AV; ++v) sum_of[v] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KST; ++ks) {
          v2i x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i)(uintptr_t)((va ^ (COLS * c)) + ks * 16 * D));
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const unsigned u = (unsigned)x[y] & keep[ks][y];
            nan[ks][y] = ((u & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u;      // 0x7f and 0xff
            any |= nan[ks][y];
            x[y] = (int)(u & ~(nan[ks][y] * 0xffu));
          }
          sum_of = mfma(widen<BF16>(x[0], x[1], vs), pb[ks], sum_of);
        }
#pragma unroll
        for (int v = 0; v < AV; ++v) o[c][v] = __fmaf_rn(sum_of[v], more, o[c][v]);
        if (__ballot(any != 0) != 0) {
          acc_t hits;
#pragma unroll
          for (int v = 0; v < AV; ++v) hits[v] = 0.0f;
#pragma unroll
          for (int ks = 0; ks < KST; ++ks) {
            v4i a;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const unsigned n = nan[ks][y];
              a[2 * y] = (int)((n & 1 ? UNIT : 0u) | (n >> 8 & 1 ? UNIT << 16 : 0u));
              a[2 * y + 1] = (int)((n >> 16 & 1 ? UNIT : 0u) | (n >> 24 & 1 ? UNIT << 16 : 0u));
            }
            hits = mfma(a, sb[ks], hits);
          }
#pragma unroll
          for (int v = 0; v < AV; ++v) o[c][v] = hits[v] > 0.0f ? NAN : o[c][v];
        }
        __builtin_amdgcn_sched_barrier(0);        // (channel tiles one after the other: side by side they take more registers than there are)
      }
    }
  };

  constexpr int PER_TILE = 2 * COPIES / CG;       // copies that a wavefront starts for a tile
  for (int j = j0; j < j1; ++j) {
    const int stage = (j - j0) & 1;
    if (next) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PER_TILE) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    if constexpr (SHARED) __builtin_amdgcn_s_barrier();      // tile j is there
    asm volatile("" ::: "memory");
    if (((j - j0) & 7) == 0) {
      // Values that may not fit the 16-bit type, scores that may be far from zero and factors beyond FP32 go the way of partly seen blocks.
      const unsigned ek = s_scale[wave][0][lane] & 255, ev = s_scale[wave][1][lane] & 255;
      const float by_scale = p.kappa * scale_of(ek);
      const bool outer = reach * scale_of(ek) >= 0.5f * FAR || by_scale == INFINITY;
      const bool all = (ev <= FITS || ev == 255) && !outer && token0 + BLOCK <= first.to && (token0 >= last.from || token0 + BLOCK <= first.sink);
      about = at_hi < 0 ? 0 : ek | (ev == 255 ? 127 : ev) << 8 | 1u << 16 | (unsigned)all << 17 | (outer ? OUTER : 0);
      factor = ev == 255 ? NAN : by_scale == INFINITY ? p.kappa : by_scale;      // a NaN among the scales makes the rows NaN that see the block, through kk
    }
    if (active) {
      // Blocks that all rows see whole first, then the others.  (In one loop, or with a way round the products, the outputs are copied from register to register for each block.)
      unsigned whole = 0, others = 0;
#pragma unroll
      for (int x = kg; x < PT_BLOCKS; x += KG) {
        const unsigned w = (unsigned)__builtin_amdgcn_readlane((int)about, ((j - j0) & 15) * 4 + x) >> 16;
        whole |= (w >> 1 & 1) << x;
        others |= (w & ~(w >> 1) & 1) << x;
      }
      auto block = [&](auto partly, int x) __attribute__((always_inline)) {
        const int at_lane = ((j - j0) & 15) * 4 + x;
        const unsigned w = (unsigned)__builtin_amdgcn_readlane((int)about, at_lane);
        const float kk = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(factor), at_lane));
        attend(partly, lds0 + (unsigned)(stage * PT_BLOCKS + x) * (2 * BYTES), __builtin_amdgcn_readlane(token0, at_lane), kk, w);
      };
      if (whole != 0) saw = ~0ull;
#pragma unroll 1
      for (; whole != 0; whole &= whole - 1) block(std::false_type{}, __builtin_ctz(whole));
#pragma unroll 1
      for (; others != 0; others &= others - 1) block(std::true_type{}, __builtin_ctz(others));
    }
    next = false;
    if (j + 2 < j1) {                             // the next tile but one takes this one's place when all have read it
      if (j + 2 - j0 >= 16 && ((j + 2 - j0) & 7) == 0) fetch(j + 2, 4 * ((j + 2 - j0) & 8), 4 * ((j + 2 - j0) & 8) + 32);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if constexpr (SHARED) __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      next = copy(j + 2, stage);
    } else {
      next = false;
    }
  }
  l = WIDE ? half_sum(l) : quarter_sum(l);
  // Scores of minus infinity alone: the sum of 1 tells them from no token at all, and goes with a weight of zero beside a finite maximum
  saw |= saw >> 32 | saw << 32;
  if constexpr (!WIDE) saw |= saw >> 16 | saw << 48;
  if (mx == -INFINITY && l == 0.0f && (saw >> lane & 1)) l = 1.0f;

  // ---- the key groups of the same rows into one, each wavefront's share of the channels: units of four of them a lane, unit u being channels (256 / COLS) u + 4 part + 0..3
  constexpr int ALL = CT * AV / 4, UN = ALL / KG;
  const int unit0 = ALL * cg + kg * UN;           // the first that I write
  auto mine_of = [&](int u) __attribute__((always_inline)) { return v4f{o[4 * u / AV][4 * u % AV], o[4 * u / AV][4 * u % AV + 1], o[4 * u / AV][4 * u % AV + 2], o[4 * u / AV][4 * u % AV + 3]}; };
  v4f res[UN];
  if constexpr (KG == 1) {
#pragma unroll
    for (int u = 0; u < UN; ++u) res[u] = mine_of(u);
  } else {
    v4f* x = reinterpret_cast<v4f*>(&s_kv[0]);
    __syncthreads();
    if (active) {
#pragma unroll
      for (int u = 0; u < ALL; ++u) x[(wave * ALL + u) * 64 + lane] = mine_of(u);
      if (part == 0) {
        s_ml[wave][2 * col] = mx;
        s_ml[wave][2 * col + 1] = l;
      }
    }
    __syncthreads();
    if (active) {
      float a[KG], m = -INFINITY;
#pragma unroll
      for (int k = 0; k < KG; ++k) m = fmaxf(m, s_ml[(rg * KG + k) * CG + cg][2 * col]);
      l = 0.0f;
#pragma unroll
      for (int k = 0; k < KG; ++k) {
        a[k] = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(s_ml[(rg * KG + k) * CG + cg][2 * col] - m);
        l = __fmaf_rn(a[k], s_ml[(rg * KG + k) * CG + cg][2 * col + 1], l);
      }
      mx = m;
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        res[u] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < KG; ++k) {
          const v4f y = x[(((rg * KG + k) * CG + cg) * ALL + kg * UN + u) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) res[u][e] = __fmaf_rn(a[k], y[e], res[u][e]);
        }
      }
    }
  }
  if (!active || rg * COLS + col >= nr) return;
  if constexpr (ONE) {
    const bool none = mx == -INFINITY && l == 0.0f;      // no token at all: zeros
    const float inv = none ? 0.0f : mx == -INFINITY ? NAN : __fdiv_rn(1.0f, l);
    if (p.lse && part == 0 && kg == 0 && cg == 0) p.lse[((size_t)b * p.H + hkv * p.G + rh) * p.N + rn] = none ? -INFINITY : LN2 * (mx + __builtin_amdgcn_logf(l));
    unsigned short* y = p.out + qrow + 4 * part;
#pragma unroll
    for (int u = 0; u < UN; ++u)
      *reinterpret_cast<uint2*>(y + (256 / COLS) * (unit0 + u)) = make_uint2(pack16x2<BF16>(res[u][0] * inv, res[u][1] * inv), pack16x2<BF16>(res[u][2] * inv, res[u][3] * inv));
  } else {
    const size_t pr = part0 + rg * COLS + col;
    if (part == 0 && kg == 0 && cg == 0) {
      p.part_ml[pr * 2] = mx;
      p.part_ml[pr * 2 + 1] = l;
    }
    float* po = p.part_o + pr * D + 4 * part;
#pragma unroll
    for (int u = 0; u < UN; ++u) *reinterpret_cast<v4f*>(po + (256 / COLS) * (unit0 + u)) = res[u];
  }
}

// The partial results of a row into its output, a wavefront per row, or per 64 channels of 256: lane s looks at partial results s, s + 64, .. for the maximum and the weights;
// then a lane takes four channels of every GRP-th partial result, MERGE_LOADS of them in flight.  Bound by the two trips to memory, not by bytes.
template <int D> constexpr int merge_channels() { return D == 256 ? 64 : D; }
constexpr int MERGE_LOADS = 8, MERGE_PER_LANE = 2, MAX_PARTS = 64 * MERGE_PER_LANE;
template <int D, bool BF16>
__global__ void __launch_bounds__(256) k_paged_merge(const PagedParams p) {
  constexpr int MC = merge_channels<D>(), LPR = MC / 4, GRP = 64 / LPR, SLICES = D / MC;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned rows = (unsigned)p.B * p.H * p.N;
  const unsigned row = blockIdx.x * (4 / SLICES) + (unsigned)wave / SLICES;
  if (row >= rows) return;
  unsigned g = row;                               // row: (batch and KV head, query, head of the group)
  unsigned hkv = split_by(g, p.by_gn);
  const unsigned b = split_by(hkv, p.by_hkv), n = split_by(g, p.by_g);
  if ((int)n >= count_of(p, (int)b)) return;
  const int S = p.S, c = MC * (wave % SLICES) + 4 * (lane % LPR), grp = lane / LPR;
  float ms[MERGE_PER_LANE], w[MERGE_PER_LANE], m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int x = 0; x < MERGE_PER_LANE; ++x) {
    ms[x] = -INFINITY; w[x] = 0.0f;
    if (64 * x + lane < S) {
      const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + ((size_t)(64 * x + lane) * rows + row) * 2);
      ms[x] = ml.x; w[x] = ml.y;
    }
    m = fmaxf(m, ms[x]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
#pragma unroll
  for (int x = 0; x < MERGE_PER_LANE; ++x) {
    const float ls = w[x];
    w[x] = ms[x] == -INFINITY && ls == 0.0f ? -1.0f : m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ms[x] - m);    // (-1: no token is seen: O may not even be there)
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
        o4[k] = *reinterpret_cast<const v4f*>(p.part_o + ((size_t)(64 * x + min(s, end - 1)) * rows + row) * D + c);
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
  const unsigned h = hkv * p.G + g;
  const bool none = m == -INFINITY && l == 0.0f;  // no token at all: zeros
  const float inv = none ? 0.0f : m == -INFINITY ? NAN : __fdiv_rn(1.0f, l);
  if (p.lse && c == 0) p.lse[((size_t)b * p.H + h) * p.N + n] = none ? -INFINITY : LN2 * (m + __builtin_amdgcn_logf(l));
  unsigned short* y = p.out + row_offset(p.qm, head_offset_of(p.qm, (int)b, (int)h), (int)n) + c;
  *reinterpret_cast<uint2*>(y) = make_uint2(pack16x2<BF16>(acc[0] * inv, acc[1] * inv), pack16x2<BF16>(acc[2] * inv, acc[3] * inv));
}

// The same of up to FEW partial results: a thread has four channels of a row and all of their loads in flight (32768 rows of two: 8.3 us, a wavefront per row 18).
constexpr int FEW = 8;
template <int D, bool BF16>
__global__ void __launch_bounds__(256) k_paged_merge_few(const PagedParams p) {
  const unsigned rows = (unsigned)p.B * p.H * p.N, row = blockIdx.x * (1024 / D) + threadIdx.x / (D / 4);
  if (row >= rows) return;
  const int c = 4 * (int)(threadIdx.x % (D / 4));
  float2 ml[FEW];
  v4f o4[FEW];
#pragma unroll
  for (int s = 0; s < FEW; ++s) {
    ml[s] = make_float2(-INFINITY, 0.0f);
    if (s < p.S) {
      ml[s] = *reinterpret_cast<const float2*>(p.part_ml + ((size_t)s * rows + row) * 2);
      o4[s] = *reinterpret_cast<const v4f*>(p.part_o + ((size_t)s * rows + row) * D + c);
    }
  }
  unsigned g = row;                               // row: (batch and KV head, query, head of the group)
  unsigned hkv = split_by(g, p.by_gn);
  const unsigned b = split_by(hkv, p.by_hkv), n = split_by(g, p.by_g);
  if ((int)n >= count_of(p, (int)b)) return;
  float m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int s = 0; s < FEW; ++s) m = fmaxf(m, ml[s].x);
  v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int s = 0; s < FEW; ++s) {
    if (ml[s].x == -INFINITY && ml[s].y == 0.0f) continue;      // (no token is seen: O may not even be there)
    const float w = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml[s].x - m);
    l = __fmaf_rn(w, ml[s].y, l);
#pragma unroll
    for (int y = 0; y < 4; ++y) acc[y] = __fmaf_rn(w, o4[s][y], acc[y]);
  }
  const unsigned h = hkv * p.G + g;
  const bool none = m == -INFINITY && l == 0.0f;  // no token at all: zeros
  const float inv = none ? 0.0f : m == -INFINITY ? NAN : __fdiv_rn(1.0f, l);
  if (p.lse && c == 0) p.lse[((size_t)b * p.H + h) * p.N + n] = none ? -INFINITY : LN2 * (m + __builtin_amdgcn_logf(l));
  unsigned short* y = p.out + row_offset(p.qm, head_offset_of(p.qm, (int)b, (int)h), (int)n) + c;
  *reinterpret_cast<uint2*>(y) = make_uint2(pack16x2<BF16>(acc[0] * inv, acc[1] * inv), pack16x2<BF16>(acc[2] * inv, acc[3] * inv));
}

// Rows of a workgroup.
int rows_of(const PagedParams& p) { return p.G * p.N <= 16 ? 16 : p.G * p.N <= 32 ? 32 : p.G * p.N <= 64 ? 64 : 128; }

// Key chunks of a row tile, S.  Workgroups beyond one on each CU (two of 64 channels, and where rows are many and products count, but of 256 channels, which fill the LDS) share
// what the chip reads, so what counts is rounds of them times the tiles of each, a tile's or two's worth of a start, and, with a merge, some 9 us of a second launch.  (A tile takes a
// wavefront of many rows as long as four of few.)  Us, sequences x tokens of 8 KV heads of 128 channels, 32 heads, chunks in parentheses: 32 in a window of 4096 48 (1) 49 (2) 52 (4);
// 1 x 32768 20 (32) 21 (64) 23 (16); 8 x 4096, 40 queries 51 (4) 56 (3) 54 (6); 1 x 4096, 600 queries 68 (3) 78 (4) 87 (2); 16 heads of 256 over 4 in 4 x 8192 18 (16) 21 (8) 23 (24); 8 heads
// over 2 in 4 x 1024 13 (1) 18 (8).
// Lengths that the host does not know are cut finer, 8 tiles or 2048 workgroups, so that the chip stays full up to the end: 8 x 8192 23 (8) 24 (4); 16 x 32768 125 (16) 127 (8) 132 (32).
void choose_chunks(PagedParams* p, int d) {
  const int rows = rows_of(*p);
  const long long gn = (long long)p->G * p->N;
  p->rt = (int)((gn + rows - 1) / rows);
  long long keys = p->cap, seen = keys;
  if (p->window > 0) seen = (long long)p->sink + p->window + std::min((long long)p->N, (long long)(rows + p->G - 1) / p->G + 1) + 2 * BLOCK;
  const bool even = p->B == 1 || 3 * seen < 2 * keys;      // all sequences about as long, as far as is known here
  const long long tiles = (std::min(keys, seen) + BLOCK * PT_BLOCKS - 1) / (BLOCK * PT_BLOCKS);
  const long long heads = (long long)p->B * p->c.Hkv * p->rt, start = rows > 64 ? 1 : 2, merge = (d == 64 ? 15 : d == 128 ? 8 : 4) * 32 / std::max(rows, 32);
  const int places = d == 64 || (rows > 32 && d == 128) ? 9 : 8;      // log2 of them
  auto rounds = [&](unsigned chunks) { return (heads * chunks + (1 << places) - 1) >> places; };
  long long best = rounds(1) * (tiles + start), chosen = 1;
  if (best > merge + start + 1)
    for (unsigned S : {2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 96, 128}) {
      if (S > tiles) break;
      const unsigned per = ((unsigned)tiles + S - 1) / S;
      const long long cost = rounds(((unsigned)tiles + per - 1) / per) * (per + start) + merge;
      if (cost < best) { best = cost; chosen = S; }
    }
  if (chosen > 1 && rows <= 32 && !even) chosen = std::max(chosen, tiles / std::max(8LL, heads * tiles / 2048));
  chosen = std::min(chosen, (long long)MAX_PARTS);
  const long long per = (tiles + chosen - 1) / chosen;
  p->S = (int)((tiles + per - 1) / per);
  p->units = p->B * p->c.Hkv * p->S;
}

int paged_params(const sage_attn_paged_args* a, PagedParams* p, bool need_io) {
  if (!a || a->H <= 0 || a->N <= 0) return SAGE_ERR_INVALID_ARG;
  const int st = cache_shape(&p->c, a->B, a->H_kv, a->d, a->n_pages, a->page, a->max_pages);
  if (st != SAGE_OK) return st;
  if (a->H % a->H_kv != 0 || a->window < 0 || a->sink < 0 || (a->causal & ~1) != 0 || (a->clear & ~3) != 0 || (a->window > 0 && !a->causal) || !std::isfinite(a->sm_scale))
    return SAGE_ERR_INVALID_ARG;
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
  p->clear = a->q_lens ? a->clear : 0;
  p->causal = a->causal; p->window = std::min(a->window, MAX_TOKENS * 2); p->sink = std::min(a->sink, MAX_TOKENS);
  p->kappa = (a->sm_scale > 0.0f ? a->sm_scale : (float)(1.0 / std::sqrt((double)a->d))) * LOG2E;
  if (!std::isfinite(p->kappa)) return SAGE_ERR_INVALID_ARG;
  choose_chunks(p, a->d);
  if (((long long)p->units + 7) / 8 * 8 * p->rt * 512 > MAX_THREADS) return SAGE_ERR_UNSUPPORTED;
  p->by_rt8 = fast_div(8u * p->rt); p->by_s = fast_div(p->S); p->by_hkv = fast_div(a->H_kv); p->by_g = fast_div(p->G);
  p->by_gn = fast_div((unsigned)p->G * a->N);
  return SAGE_OK;
}

size_t part_rows(const PagedParams& p) { return p.S > 1 ? (size_t)p.S * p.B * p.H * p.N : 0; }
size_t paged_bytes(const PagedParams& p, int d) { return align256(part_rows(p) * 2 * sizeof(float)) + align256(part_rows(p) * d * sizeof(float)); }

template <int D, bool BF16, bool ONE> void launch_rows(const PagedParams& p, hipStream_t s) {
  const unsigned grid = (unsigned)((p.units + 7) / 8 * 8) * p.rt;
  const int rows = rows_of(p);
  if (rows == 16) k_paged<D, BF16, 16, 1, ONE><<<grid, paged_threads<D, 16>(), lds_bytes<D>(), s>>>(p);
  else if (rows == 32) k_paged<D, BF16, 32, 1, ONE><<<grid, paged_threads<D, 32>(), lds_bytes<D>(), s>>>(p);
  else if (rows == 64) k_paged<D, BF16, 32, 2, ONE><<<grid, paged_threads<D, 32>(), lds_bytes<D>(), s>>>(p);
  else k_paged<D, BF16, 32, 4, ONE><<<grid, paged_threads<D, 32>(), lds_bytes<D>(), s>>>(p);
}
template <int D, bool BF16> hipError_t launch(const PagedParams& p, hipStream_t s) {
  if (p.S == 1) {
    launch_rows<D, BF16, true>(p, s);
    return hipGetLastError();
  }
  launch_rows<D, BF16, false>(p, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.S <= FEW) {
    k_paged_merge_few<D, BF16><<<((unsigned)(p.B * p.H) * p.N + 1024 / D - 1) / (1024 / D), 256, 0, s>>>(p);
    return hipGetLastError();
  }
  const unsigned per = 4 * merge_channels<D>() / D;
  k_paged_merge<D, BF16><<<((unsigned)(p.B * p.H) * p.N + per - 1) / per, 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace
}  // namespace sage

using namespace sage;

extern "C" size_t sage_attn_paged_workspace_bytes(const sage_attn_paged_args* a) {
  PagedParams p;
  if (paged_params(a, &p, false) != SAGE_OK) return 0;
  return paged_bytes(p, a->d);
}

extern "C" int sage_attn_paged(const sage_attn_paged_args* a) {
  PagedParams p;
  const int st = paged_params(a, &p, true);
  if (st != SAGE_OK) return st;
  const size_t rows = (size_t)a->B * a->H * a->N, blocks = cache_blocks(p.c), bytes = blocks * BLOCK * a->d, need = paged_bytes(p, a->d);
  if (need > 0 && (!a->workspace || a->workspace_bytes < need || ((uintptr_t)a->workspace & 255u) != 0)) return SAGE_ERR_WORKSPACE;
  // (a row's query is read before its output is written, by the same workgroup or a kernel before: out may be q)
  const Span in[8] = {{a->out == a->q ? nullptr : a->q, rows * a->d * 2}, {a->k_cache, bytes}, {a->v_cache, bytes}, {a->k_scale, blocks}, {a->v_scale, blocks},
                      {a->page_table, (size_t)a->B * a->max_pages * 4}, {a->kv_lens, (size_t)a->B * 4}, {a->q_lens, (size_t)a->B * 4}};
  const Span out[3] = {{a->out, rows * a->d * 2}, {a->lse, rows * 4}, {need > 0 ? a->workspace : nullptr, need}};
  for (int i = 0; i < 3; ++i) {
    for (const Span& x : in) if (overlap(out[i], x)) return SAGE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j) if (overlap(out[i], out[j])) return SAGE_ERR_INVALID_ARG;
  }
  p.part_ml = (float*)a->workspace;
  p.part_o = (float*)((char*)a->workspace + align256(part_rows(p) * 2 * sizeof(float)));
  const hipStream_t s = (hipStream_t)a->stream;
  const bool bf16 = a->dtype == SAGE_DT_BF16;
  hipError_t e;
  if (a->d == 64) e = bf16 ? launch<64, true>(p, s) : launch<64, false>(p, s);
  else if (a->d == 128) e = bf16 ? launch<128, true>(p, s) : launch<128, false>(p, s);
  else e = bf16 ? launch<256, true>(p, s) : launch<256, false>(p, s);
  return op_status(e);
}
