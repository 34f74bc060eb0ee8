// Shared by the operators around attention (sage_rope.hip, sage_attn_shared.hip, sage_key_weights.hip, sage_cache.hip).
#pragma once
#include "sage_attn_core.h"

namespace sage {

// The status of a launch: argument errors are found before it, so what is left is HIP's.  The error is cleared.
inline int op_status(hipError_t e) {
  if (e == hipSuccess) return 0;
  (void)hipGetLastError();
  return -4;      // SAGE_ERR_HIP
}

// A contiguous tensor, and whether two share a byte (none does with what is not there).
struct Span { const void* at; size_t bytes; };
inline bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = (uintptr_t)a.at, y = (uintptr_t)b.at;
  return a.at && b.at && x < y + b.bytes && y < x + a.bytes;
}

// Most threads of a grid in one of its dimensions: the launch packet counts them in 32 bits.
constexpr long long MAX_THREADS = 0xffffffffLL;

// Element offset of head h of batch b.
__device__ __forceinline__ size_t head_offset_of(const TensorMap& m, int b, int h) { return (size_t)b * m.sb + (size_t)h * m.sh; }

// 16-bit products on the matrix unit, 32 x 32 x 16: lane l supplies row (A) or column (B) l % 32 and contraction slots
// 8 (l / 32) + 0..7; accumulator v of lane l is row 8 (v / 4) + 4 (l / 32) + v % 4, column l % 32.
typedef short v8s __attribute__((ext_vector_type(8)));
template <bool BF16> __device__ __forceinline__ v16f mfma16(v4i a, v4i b, v16f c) {
  if constexpr (BF16) {
    typedef __bf16 v8b __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  } else {
    typedef _Float16 v8h __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
}

// The same, 16 x 16 x 32: row or column l % 16, contraction slots 8 (l / 16) + 0..7; accumulator v is row 4 (l / 16) + v, column l % 16.
template <bool BF16> __device__ __forceinline__ v4f mfma16_small(v4i a, v4i b, v4f c) {
  if constexpr (BF16) {
    typedef __bf16 v8b __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  } else {
    typedef _Float16 v8h __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
}

// Division by a number that the host knows (numerators and divisors below 2^31): a product's high half and two shifts, where the
// instruction sequence for an unknown divisor has some thirty.  With l = ceil(log2 d) and m = floor(2^32 (2^l - d) / d) + 1,
// floor(n / d) = (t + (n - t >> s1)) >> s2 for t = the high half of m n, s1 = min(l, 1), s2 = max(l - 1, 0).
struct FastDiv {
  unsigned d, m, s1, s2;
};
inline FastDiv fast_div(unsigned d) {
  unsigned l = 0;
  while (l < 32 && (1ull << l) < d) ++l;
  FastDiv f;
  f.d = d;
  f.m = (unsigned)(((1ull << 32) * ((1ull << l) - d)) / d + 1);
  f.s1 = l < 1 ? l : 1;
  f.s2 = l > 1 ? l - 1 : 0;
  return f;
}
__device__ __forceinline__ unsigned div_by(unsigned n, const FastDiv& f) {
  const unsigned t = (unsigned)(((unsigned long long)f.m * n) >> 32);
  return (t + ((n - t) >> f.s1)) >> f.s2;
}
// Quotient; n becomes the remainder.
__device__ __forceinline__ unsigned split_by(unsigned& n, const FastDiv& f) {
  const unsigned q = div_by(n, f);
  n -= q * f.d;
  return q;
}

// Sum / maximum of a value over the two halves of the wavefront, in both.
__device__ __forceinline__ float half_sum(float x) {
  const unsigned u = __float_as_uint(x);
  const auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}
__device__ __forceinline__ float half_max(float x) {
  const unsigned u = __float_as_uint(x);
  const auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

// Rows of D 16-bit values in LDS, D / 8 pieces of 16 bytes each, as an LDS-DMA lays them down: piece c of row r stands at
// piece c ^ swizzle(r) of the row.  Without it, the same piece of the rows that a matrix operand takes together would fall on the
// same banks (a row is a multiple of 128 bytes).  The low two row bits go to piece bits 2 and 3 because a transposed read takes four
// consecutive pieces of each of rows 4i .. 4i + 3 together.
template <int D> __device__ __forceinline__ int swizzle(int r) {
  if constexpr (D == 64) return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
  return (r & 3) << 2 | ((r >> 2) & 3);
}
template <int D> __device__ __forceinline__ int row_piece(int r, int c) { return r * (D / 8) + (c ^ swizzle<D>(r)); }

// dma_b128 of what is read once: it does not stay in the caches.
__device__ __forceinline__ void dma_b128_once(const void* gbase, unsigned voff, unsigned lds_byte) {
  unsigned m0_after;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3 nt"
               : "={m0}"(m0_after) : "s"(lds_byte), "v"(voff), "s"(gbase) : "memory");
}

}  // namespace sage
