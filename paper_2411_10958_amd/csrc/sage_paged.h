// A cache of keys and values in 8 bits and pages, as sage_cache_append writes it and sage_attn_paged reads it.
#pragma once
#include "sage_attn.h"
#include "sage_ops.h"
#include "sage_quant.h"

#include <cmath>

namespace sage {

constexpr int BLOCK = 32;            // tokens that share a scale: one tile of scores, so that the scale is one number of it

struct PagedCache {
  unsigned char *k, *v, *ks, *vs;    // codes [n_pages, H_kv, page, d], scales [n_pages, H_kv, bpp]
  const int* table;                  // [B, max_pages]
  int n_pages, bpp, max_pages, Hkv, d;      // bpp: blocks of a page
  FastDiv by_bpp;
};

// Block i of a sequence: which block of the pool's head hkv it is - codes at that times 32 d, scale at it - or -1: no page.
__device__ __forceinline__ long long pool_block(const PagedCache& c, int b, int hkv, int i) {
  unsigned j = (unsigned)i;
  const unsigned at = split_by(j, c.by_bpp);
  const int page = c.table[(size_t)b * c.max_pages + at];
  return (unsigned)page < (unsigned)c.n_pages ? ((long long)page * c.Hkv + hkv) * c.bpp + j : -1;
}
// A scale byte as the FP32 number 2^(byte - 127); 255 is NaN.
__device__ __forceinline__ float scale_of(unsigned byte) { return byte == 0 ? 0x1p-127f : byte == 255 ? NAN : __uint_as_float(byte << 23); }

// Magnitudes of 16-bit values are numbers of the same order.  The larger of two pairs; a pair without what is not finite; the largest of all lanes' pairs.
__device__ __forceinline__ unsigned larger_pair(unsigned a, unsigned b) {
  typedef unsigned short v2u __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(v2u, a), __builtin_bit_cast(v2u, b)));
}
template <bool BF16> __device__ __forceinline__ unsigned finite_pair(unsigned two) {
  constexpr unsigned EXP = BF16 ? 0x7f80 : 0x7c00;
  const unsigned lo = two & 0x7fff, hi = two >> 16 & 0x7fff;
  return (lo < EXP ? lo : 0) | (hi < EXP ? hi : 0) << 16;
}
__device__ __forceinline__ unsigned largest_of_all(unsigned two) { return (unsigned)(int)wave_max((float)max(two & 0xffff, two >> 16)); }

// The shape of a cache, checked; every offset into it stays within 48 bits.
inline int cache_shape(PagedCache* c, int B, int Hkv, int d, int n_pages, int page, int max_pages) {
  if (B <= 0 || Hkv <= 0 || n_pages <= 0 || page <= 0 || max_pages <= 0) return SAGE_ERR_INVALID_ARG;
  if (d != 64 && d != 128 && d != 256) return SAGE_ERR_UNSUPPORTED;
  if (page % BLOCK != 0 || (long long)max_pages * page > MAX_TOKENS || (long long)B * Hkv > 65535) return SAGE_ERR_UNSUPPORTED;
  if ((double)n_pages * Hkv * page * d > (double)(1LL << 47)) return SAGE_ERR_UNSUPPORTED;
  c->n_pages = n_pages; c->bpp = page / BLOCK; c->max_pages = max_pages; c->Hkv = Hkv; c->d = d;
  c->by_bpp = fast_div((unsigned)c->bpp);
  return SAGE_OK;
}
// Its pointers.
inline int cache_arrays(PagedCache* c, const void* k, const void* v, const void* ks, const void* vs, const int* table) {
  if (!k || !v || !ks || !vs || !table) return SAGE_ERR_INVALID_ARG;
  if ((((uintptr_t)k | (uintptr_t)v) & 15u) != 0 || ((uintptr_t)table & 3u) != 0) return SAGE_ERR_INVALID_ARG;
  c->k = (unsigned char*)const_cast<void*>(k); c->v = (unsigned char*)const_cast<void*>(v);
  c->ks = (unsigned char*)const_cast<void*>(ks); c->vs = (unsigned char*)const_cast<void*>(vs);
  c->table = table;
  return SAGE_OK;
}
inline size_t cache_blocks(const PagedCache& c) { return (size_t)c.n_pages * c.Hkv * c.bpp; }

}  // namespace sage
