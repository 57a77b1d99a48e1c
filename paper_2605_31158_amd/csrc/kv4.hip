// Entering keys and values into the 4-bit cache, and reading back the values they stand for
// (layout: kv4.h).
//
// Per 32 values of a row, x -> code(x / 2^e) with the smallest power of two under which the largest
// value is rounded by less than half a step: amax < 7 2^e, since 6 is the largest code and 7 lies half a
// step above it.  In bf16 bits that is one addition: with 32 added to the magnitude's bits a
// mantissa of 1.75 or more carries into the exponent.  e is held to [-125, 125], so that every value
// read back is a normal, finite bf16.  A block with a value that is not finite gets the scale byte
// 255 and reads as NaN.  Rounding is to nearest, ties to the even code, by the conversion
// instruction, after an exact multiplication by 2^-e.
//
// Both are streaming passes bound by HBM: 2 bytes per value on one side, 17/32 on the other.  A group
// of d / 8 lanes has a token's row of one head, 16 bytes a lane; four lanes share a block's maximum.  6240
// tokens of 16 heads, d 128 (65 MB either way): 11.0 us entered, 10.7 read, 5.9 TB/s, since part of it is
// found in the last-level cache; 64 tokens of 8 heads 3.7 us each, which is the launch and a chain of
// loads (starts, length, page number, row).
#include "kv4.h"

namespace la {
namespace {

constexpr int kKvThreads = 256;
constexpr int kCuLds = 1024;             // starts that a workgroup holds in LDS for its search

struct KvRows {
  const int32_t *cu, *lens;              // [S + 1], [S]
  int S, T, Hkv;
  int64_t k_tok, k_head, v_tok, v_head;
};

// Where the tokens of a workgroup lie: slot[i] = page << 16 | place for token t0 + i, or -1 where the
// token belongs to no sequence, -2 where its place does not exist (a position below zero or past the
// table, a page number out of range).  The search for a token's sequence goes through at most kCuLds
// of the starts in LDS and then through those between two of them.  (S may come near 2^31: no sum of two
// places among the starts is formed.)
template <int TOKENS>
__device__ void find_slots(const KvRows& r, const CacheGeom& cg, int t0, int64_t* slot, int32_t* cu) {
  const int step = (r.S + 1 + kCuLds - 1) / kCuLds, n = r.S / step + 1;     // starts 0, step, 2 step, ..
  for (int i = threadIdx.x; i < n; i += kKvThreads) cu[i] = r.cu[i * step];
  __syncthreads();
  if (threadIdx.x < TOKENS) {
    const int t = t0 + threadIdx.x;
    // the last start that is not behind t
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cu[mid] <= t) lo = mid;
      else hi = mid;
    }
    int s = lo * step, left = min(r.S + 1 - s, step);      // it is among starts s, .., s + left - 1
    while (left > 1) {
      const int half = left >> 1;
      if (r.cu[s + half] <= t) {
        s += half;
        left -= half;
      } else {
        left = half;
      }
    }
    int64_t x = -1;
    if (t < r.T && s < r.S && r.cu[s] <= t && t < r.cu[s + 1]) {
      const int n_new = r.cu[s + 1] - r.cu[s];
      const int64_t pos = (int64_t)r.lens[s] - n_new + (t - r.cu[s]);
      x = -2;
      if (pos >= 0 && (pos >> cg.log_p) < cg.max_pages) {
        const int id = cg.table[(int64_t)s * cg.max_pages + (pos >> cg.log_p)];
        if ((uint32_t)id < (uint32_t)cg.n_pages) x = (int64_t)id << 16 | (pos & ((1 << cg.log_p) - 1));
      }
    }
    slot[threadIdx.x] = x;
  }
  __syncthreads();
}

// Eight values -> their codes (value i in bits 4 i) and the scale byte of their block of 32, which this
// lane and the three beside it hold.
__device__ __forceinline__ uint32_t quantise8(u32x4 x, uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) top = max(top, max(x[e] & 0x7fffu, (x[e] >> 16) & 0x7fffu));
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xf, 0xf, true));   // quad_perm 1,0,3,2
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xf, 0xf, true));   // quad_perm 2,3,0,1
  const uint32_t b = (uint32_t)min(max((int)((top + 0x20u) >> 7) - 2, 2), 252);
  const bool bad = top >= 0x7f80u;
  *byte = bad ? 255u : b;
  const float f = __uint_as_float((254u - b) << 23);
  uint32_t w = 0;
#define LA_PAIR(e) \
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[e] << 16) * f, __uint_as_float(x[e] & 0xffff0000u) * f, 1.0f, e)
  LA_PAIR(0);
  LA_PAIR(1);
  LA_PAIR(2);
  LA_PAIR(3);
#undef LA_PAIR
  return bad ? 0u : w;
}

template <int D>
__global__ __launch_bounds__(kKvThreads) void kv4_append_kernel(const uint16_t* __restrict__ k,
                                                                const uint16_t* __restrict__ v, KvRows r, CacheGeom cg,
                                                                uint8_t* __restrict__ pages) {
  using F = Kv4<D>;
  constexpr int L = D / 8, TOKENS = kKvThreads / L;
  __shared__ int64_t slot[TOKENS];
  __shared__ int32_t cu[kCuLds];
  const int t0 = blockIdx.x * TOKENS, h = blockIdx.y;
  const int i = threadIdx.x / L, j = threadIdx.x % L;
  const int t = min(t0 + i, r.T - 1);
  const u32x4 xk = *(const u32x4*)(k + (int64_t)t * r.k_tok + (int64_t)h * r.k_head + 8 * j);
  const u32x4 xv = *(const u32x4*)(v + (int64_t)t * r.v_tok + (int64_t)h * r.v_head + 8 * j);
  find_slots<TOKENS>(r, cg, t0, slot, cu);
  uint32_t bk, bv;
  const uint32_t wk = quantise8(xk, &bk), wv = quantise8(xv, &bv);
  const int64_t at = slot[i];
  if (at < 0) return;
  const int P = 1 << cg.log_p, in = (int)(at & 0xffff);
  uint8_t* pg = pages + ((uint64_t)(at >> 16) * (uint32_t)cg.Hkv + (uint32_t)h) * (uint64_t)F::page_bytes(P);
  *(uint32_t*)(pg + in * F::ROW + 4 * j) = wk;
  if constexpr (D == 128) {
    *(uint32_t*)(pg + F::v_code(P) + ((in >> 2) * 16 + j) * 16 + (in & 3) * 4) = wv;
  } else {
    uint8_t* p = pg + F::v_code(P) + ((in >> 2) * 16 + 2 * j) * 8 + (in & 3) * 2;
    *(uint16_t*)p = (uint16_t)wv;
    *(uint16_t*)(p + 8) = (uint16_t)(wv >> 16);
  }
  if ((j & 3) == 0) {
    pg[F::k_scale(P) + (j >> 2) * P + in] = (uint8_t)bk;
    pg[F::v_scale(P) + (j >> 2) * P + in] = (uint8_t)bv;
  }
}

template <int D>
__global__ __launch_bounds__(kKvThreads) void kv4_read_kernel(KvRows r, CacheGeom cg, uint16_t* __restrict__ k,
                                                              uint16_t* __restrict__ v) {
  using F = Kv4<D>;
  constexpr int L = D / 8, TOKENS = kKvThreads / L;
  __shared__ int64_t slot[TOKENS];
  __shared__ int32_t cu[kCuLds];
  const int t0 = blockIdx.x * TOKENS, h = blockIdx.y;
  const int i = threadIdx.x / L, j = threadIdx.x % L;
  find_slots<TOKENS>(r, cg, t0, slot, cu);
  const int64_t at = slot[i];
  if (at == -1) return;
  u32x4 xk = u32x4{0u, 0u, 0u, 0u}, xv = xk;
  if (at >= 0) {
    const int P = 1 << cg.log_p, in = (int)(at & 0xffff);
    const uint8_t* pg = cg.pages + ((uint64_t)(at >> 16) * (uint32_t)cg.Hkv + (uint32_t)h) * (uint64_t)F::page_bytes(P);
    const uint32_t wk = *(const uint32_t*)(pg + in * F::ROW + 4 * j);
    uint32_t wv;
    if constexpr (D == 128) {
      wv = *(const uint32_t*)(pg + F::v_code(P) + ((in >> 2) * 16 + j) * 16 + (in & 3) * 4);
    } else {
      const uint8_t* p = pg + F::v_code(P) + ((in >> 2) * 16 + 2 * j) * 8 + (in & 3) * 2;
      wv = *(const uint16_t*)p | (uint32_t) * (const uint16_t*)(p + 8) << 16;
    }
    xk = fp4x8(wk, scale_of(pg[F::k_scale(P) + (j >> 2) * P + in], 0));
    xv = fp4x8(wv, scale_of(pg[F::v_scale(P) + (j >> 2) * P + in], 0));
  }
  const int64_t t = t0 + i;
  *(u32x4*)(k + t * r.k_tok + (int64_t)h * r.k_head + 8 * j) = xk;
  *(u32x4*)(v + t * r.v_tok + (int64_t)h * r.v_head + 8 * j) = xv;
}

KvRows kv_rows(const la_seqs& s, const int32_t* cu, const int32_t* lens) {
  return KvRows{cu, lens, s.S, s.Tk, s.Hkv, s.k_token, s.k_head, s.v_token, s.v_head};
}

dim3 kv_grid(const la_seqs& s) {
  const int tokens = kKvThreads / (s.d / 8);
  return dim3((s.Tk + tokens - 1) / tokens, s.Hkv);
}

}  // namespace

hipError_t launch_kv4_append(const la_seqs& s, const CacheGeom& cg, const void* k, const void* v, const int32_t* cu,
                             const int32_t* lens, void* pages, hipStream_t st) {
  const KvRows r = kv_rows(s, cu, lens);
  if (s.d == 128)
    hipLaunchKernelGGL(kv4_append_kernel<128>, kv_grid(s), dim3(kKvThreads), 0, st, (const uint16_t*)k,
                       (const uint16_t*)v, r, cg, (uint8_t*)pages);
  else
    hipLaunchKernelGGL(kv4_append_kernel<64>, kv_grid(s), dim3(kKvThreads), 0, st, (const uint16_t*)k,
                       (const uint16_t*)v, r, cg, (uint8_t*)pages);
  return hipGetLastError();
}

hipError_t launch_kv4_read(const la_seqs& s, const CacheGeom& cg, const int32_t* cu, const int32_t* lens, void* k,
                           void* v, hipStream_t st) {
  const KvRows r = kv_rows(s, cu, lens);
  if (s.d == 128)
    hipLaunchKernelGGL(kv4_read_kernel<128>, kv_grid(s), dim3(kKvThreads), 0, st, r, cg, (uint16_t*)k, (uint16_t*)v);
  else
    hipLaunchKernelGGL(kv4_read_kernel<64>, kv_grid(s), dim3(kKvThreads), 0, st, r, cg, (uint16_t*)k, (uint16_t*)v);
  return hipGetLastError();
}

}  // namespace la
