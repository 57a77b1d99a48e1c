// The cache of keys and values in 4 bits (gfx950): layout, and codes -> bf16 in registers.
//
// Values are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times one power of two for every
// 32 values of a row, held as a byte (2^(byte - 127); 255: the block held a value that is not
// finite, and reads as NaN).  Every product of the two is a bf16 value exactly.
//
// A page holds P tokens (a multiple of 16) of one key head, P (d + d / 16) bytes:
//   K codes   [P][d / 2]              a token's row, two values to a byte, the lower 4 bits first
//   K scales  [d / 32][P]
//   V codes   [P / 4][16][4][d / 32]  quads of tokens: chunk c (values c d / 16 ..) of each in turn
//   V scales  [d / 32][P]
// The MFMA operands follow from it with no exchange between lanes: K rows are read 16 (8) bytes to
// a lane along d, V 16 (8) bytes to a lane along the tokens, the scales of 4 or 16 tokens at once.
#pragma once

#include "la_internal.h"

namespace la {

struct CacheGeom {
  const uint8_t* pages;    // [n_pages][Hkv][page bytes]
  const int32_t* table;    // [S][max_pages]
  int n_pages, max_pages;
  int log_p;               // log2 of the tokens of a page
  int Hkv;
};

namespace {

template <int D>
struct Kv4 {
  static constexpr int ROW = D / 2;                 // bytes of a token's codes
  static constexpr int NB = D / 32;                 // scale blocks of a row
  static constexpr int WB = D / 32;                 // bytes of a V chunk of one token
  __device__ __host__ static constexpr int page_bytes(int P) { return P * (D + D / 16); }
  __device__ static __forceinline__ int k_scale(int P) { return P * ROW; }
  __device__ static __forceinline__ int v_code(int P) { return P * (ROW + NB); }
  __device__ static __forceinline__ int v_scale(int P) { return P * (2 * ROW + NB); }
};

// Bytes of page `id` of key head h; a page number out of range gives page 0 and ok = false.
template <int D>
__device__ __forceinline__ const uint8_t* page_of(const CacheGeom& cg, int id, int h, bool* ok) {
  *ok = (uint32_t)id < (uint32_t)cg.n_pages;
  return cg.pages + ((uint64_t)(*ok ? id : 0) * (uint32_t)cg.Hkv + (uint32_t)h) *
                        (uint64_t)Kv4<D>::page_bytes(1 << cg.log_p);
}

// Two e2m1 codes (byte `sel` of w) times the scale -> two bf16.
template <int sel>
__device__ __forceinline__ uint32_t fp4x2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, sel));
}
// Byte i of a word of scale bytes as the power of two that it stands for.
__device__ __forceinline__ float scale_of(uint32_t bytes, int i) {
  return __uint_as_float(((bytes >> (8 * i)) & 0xffu) << 23);
}
// Eight codes of one block -> eight bf16.
__device__ __forceinline__ u32x4 fp4x8(uint32_t w, float scale) {
  return u32x4{fp4x2<0>(w, scale), fp4x2<1>(w, scale), fp4x2<2>(w, scale), fp4x2<3>(w, scale)};
}

}  // namespace
}  // namespace la
