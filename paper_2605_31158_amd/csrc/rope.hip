// Rotary positions on gfx950: pair j of a head's first `rot` values is turned by the angle
// p f_j of its token's position p (of the axis that the pair belongs to),
//   (a, b) -> (a cos - b sin, b cos + a sin),
// with pairs (j, j + rot / 2) or (2 j, 2 j + 1); the values behind `rot` pass through.
//
// Bound by HBM: every value is read once and written once.  A workgroup has 4 tokens and all their
// heads, queries and keys in one launch, so an angle is computed once for all heads: one of the
// 4 x 64 at most per thread, in 64 bits as turns (p f / 2 pi less its whole turns: three roundings, 2^-24
// of a turn at positions of 10^9) and then sin and cos in fp32.  A lane moves 16 values of a row, the two
// halves of 8 pairs or 8 neighbouring ones, and holds their 8 cosines and sines in registers over the
// heads; four rows are in flight per lane.  6240 tokens of 16 + 16 bf16 heads of 128 (102 MB) take 23.0 us,
// 4.4 TB/s, 8191 tokens of 16 + 8 fp32 heads (201 MB) 47.3 us, 4.3 TB/s; a large copy reaches 5.1.  8 tokens
// take 3.1 us.
#include <math.h>

#include "la_internal.h"

namespace la {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;

struct RopeArgs {
  const void *q, *k;
  void *qo, *ko;
  const int32_t* pos;      // [axes][L]
  const double* freqs;     // [rot / 2], radians
  int L, Hq, Hk, rot;
  int axes, s0, s1;        // pairs below s0 turn by axis 0, below s1 by axis 1, the others by axis 2
  float amplitude;
  int64_t q_b, q_t, q_h, qo_b, qo_t, qo_h, k_b, k_t, k_h, ko_b, ko_t, ko_h;
};

// Eight values at p, as fp32.
template <bool BF16>
struct Chunk {
  u32x4 w[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const char* p) {
    const u32x4* s = (const u32x4*)p;
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) w[i] = __builtin_nontemporal_load(s + i);
  }
  __device__ __forceinline__ void store(char* p) const {
    u32x4* d = (u32x4*)p;
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) d[i] = w[i];
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (BF16) x[e] = __uint_as_float((e & 1) ? w[0][e >> 1] & 0xffff0000u : w[0][e >> 1] << 16);
      else x[e] = __uint_as_float(w[BF16 ? 0 : e >> 2][e & 3]);
    }
  }
  __device__ __forceinline__ void set(const float* x) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (BF16) {
        if ((e & 1) == 0) {
          const f2 f = {x[e], x[e + 1]};
          w[0][e >> 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, b2));
        }
      } else {
        w[BF16 ? 0 : e >> 2][e & 3] = __float_as_uint(x[e]);
      }
    }
  }
};

template <int D, bool BF16, bool NEIGHBOURS>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  constexpr int LANES = D / 16;                              // of a row
  constexpr int HEADS = kRopeThreads / (LANES * kRopeTokens);  // rows of a token at a time
  constexpr int UNROLL = 4, SIZE = BF16 ? 2 : 4;
  __shared__ float cs[kRopeTokens][D / 2], sn[kRopeTokens][D / 2];
  const int pairs = a.rot / 2, t0 = blockIdx.x * kRopeTokens, b = blockIdx.y, H = a.Hq + a.Hk;
  const int lane = threadIdx.x % LANES, hl = threadIdx.x / LANES % HEADS, tt = threadIdx.x / (LANES * HEADS);
  const int t = t0 + tt;
  // this lane's two chunks of 8 values, and whether they turn
  const bool turn = NEIGHBOURS ? 16 * lane < a.rot : lane < a.rot / 16;
  const int o1 = NEIGHBOURS ? 16 * lane : (turn ? 8 * lane : 16 * lane);
  const int o2 = !NEIGHBOURS && turn ? pairs + 8 * lane : o1 + 8;
  const char* const qs = (const char*)a.q + (b * a.q_b + t * a.q_t) * SIZE;
  const char* const ks = (const char*)a.k + (b * a.k_b + t * a.k_t) * SIZE;
  char* const qd = (char*)a.qo + (b * a.qo_b + t * a.qo_t) * SIZE;
  char* const kd = (char*)a.ko + (b * a.ko_b + t * a.ko_t) * SIZE;
  Chunk<BF16> x[UNROLL], y[UNROLL];
  // rows h0, h0 + HEADS, ..: the queries' heads, then the keys'
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int h = h0 + u * HEADS;
      if (h < H && t < a.L) {
        const char* p = h < a.Hq ? qs + h * a.q_h * SIZE : ks + (h - a.Hq) * a.k_h * SIZE;
        x[u].load(p + o1 * SIZE);
        y[u].load(p + o2 * SIZE);
      }
    }
  };
  load(hl);
  for (int i = threadIdx.x; i < kRopeTokens * pairs; i += kRopeThreads) {
    const int j = i % pairs, ti = i / pairs;
    const int axis = j < a.s0 ? 0 : (j < a.s1 ? 1 : 2);
    const int p = a.pos[(int64_t)axis * a.L + min(t0 + ti, a.L - 1)];
    const double turns = (double)p * a.freqs[j] * 0.15915494309189533577;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    cs[ti][j] = c * a.amplitude;
    sn[ti][j] = s * a.amplitude;
  }
  __syncthreads();
  if (t >= a.L) return;
  float c[8], s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    c[e] = turn ? cs[tt][8 * lane + e] : 1.f;
    s[e] = turn ? sn[tt][8 * lane + e] : 0.f;
  }
  for (int h0 = hl; h0 < H; h0 += UNROLL * HEADS) {
    if (h0 != hl) load(h0);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int h = h0 + u * HEADS;
      if (h >= H) break;
      if (turn) {
        float p[8], r[8], pn[8], rn[8];
        x[u].get(p);
        y[u].get(r);
        if (NEIGHBOURS) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            pn[2 * e] = p[2 * e] * c[e] - p[2 * e + 1] * s[e];
            pn[2 * e + 1] = p[2 * e + 1] * c[e] + p[2 * e] * s[e];
            rn[2 * e] = r[2 * e] * c[4 + e] - r[2 * e + 1] * s[4 + e];
            rn[2 * e + 1] = r[2 * e + 1] * c[4 + e] + r[2 * e] * s[4 + e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            pn[e] = p[e] * c[e] - r[e] * s[e];
            rn[e] = r[e] * c[e] + p[e] * s[e];
          }
        }
        x[u].set(pn);
        y[u].set(rn);
      }
      char* d = h < a.Hq ? qd + h * a.qo_h * SIZE : kd + (h - a.Hq) * a.ko_h * SIZE;
      x[u].store(d + o1 * SIZE);
      y[u].store(d + o2 * SIZE);
    }
  }
}

template <int D, bool BF16>
void launch(const RopeArgs& a, bool neighbours, int B, hipStream_t st) {
  const dim3 grid((a.L + kRopeTokens - 1) / kRopeTokens, B);
  if (neighbours) hipLaunchKernelGGL((rope_kernel<D, BF16, true>), grid, dim3(kRopeThreads), 0, st, a);
  else hipLaunchKernelGGL((rope_kernel<D, BF16, false>), grid, dim3(kRopeThreads), 0, st, a);
}

// Rows that are written lie apart: no stride of 0 (of the batch, where there is one).
bool bad_rows(int64_t batch, int64_t token, int64_t head, int B, bool written) {
  return batch < (written && B > 1 ? 1 : 0) || token < (written ? 1 : 0) || head < (written ? 1 : 0) ||
         ((batch | token | head) & 7);
}

}  // namespace
}  // namespace la

using namespace la;

extern "C" la_status la_rope(const la_rope_shape* s, const void* q, void* q_out, const void* k, void* k_out,
                             const int32_t* positions, const double* freqs, float amplitude, void* stream) {
  if (!s) return LA_ERR_ARG;
  if (s->B < 0 || s->L < 0 || s->Hq < 0 || s->Hk < 0 || s->B > 65535 || (s->d != 64 && s->d != 128)) return LA_ERR_SHAPE;
  if (s->L > (1 << 26) - 4) return LA_ERR_SHAPE;    // 64 threads a token, below 2^32 in all
  if (s->rot < 16 || s->rot > s->d || s->rot % 16) return LA_ERR_SHAPE;
  if (s->interleaved != 0 && s->interleaved != 1) return LA_ERR_SHAPE;
  if (s->axes < 1 || s->axes > 3) return LA_ERR_SHAPE;
  int pairs = 0;
  for (int i = 0; i < s->axes; ++i) {
    if (s->section[i] < 0 || s->section[i] > s->rot) return LA_ERR_SHAPE;
    pairs += s->section[i];
  }
  if (pairs != s->rot / 2) return LA_ERR_SHAPE;
  if (s->dtype != LA_DTYPE_F32 && s->dtype != LA_DTYPE_BF16) return LA_ERR_ARG;
  if (isnan(amplitude) || isinf(amplitude)) return LA_ERR_ARG;
  if (s->B == 0 || s->L == 0 || (s->Hq == 0 && s->Hk == 0)) return LA_OK;
  if (s->Hq > 0) {
    if (bad_rows(s->q_batch, s->q_token, s->q_head, s->B, false) ||
        bad_rows(s->qo_batch, s->qo_token, s->qo_head, s->B, true))
      return LA_ERR_SHAPE;
    if (!q || !q_out || ((uintptr_t)q & 15u) || ((uintptr_t)q_out & 15u)) return LA_ERR_ARG;
  }
  if (s->Hk > 0) {
    if (bad_rows(s->k_batch, s->k_token, s->k_head, s->B, false) ||
        bad_rows(s->ko_batch, s->ko_token, s->ko_head, s->B, true))
      return LA_ERR_SHAPE;
    if (!k || !k_out || ((uintptr_t)k & 15u) || ((uintptr_t)k_out & 15u)) return LA_ERR_ARG;
  }
  if (!positions || !freqs || ((uintptr_t)positions & 3u) || ((uintptr_t)freqs & 7u)) return LA_ERR_ARG;
  RopeArgs a{q, k, q_out, k_out, positions, freqs, s->L, s->Hq, s->Hk, s->rot, s->axes,
             s->axes > 1 ? s->section[0] : s->rot, s->axes > 2 ? s->section[0] + s->section[1] : s->rot, amplitude,
             s->q_batch, s->q_token, s->q_head, s->qo_batch, s->qo_token, s->qo_head,
             s->k_batch, s->k_token, s->k_head, s->ko_batch, s->ko_token, s->ko_head};
  const bool nb = s->interleaved, bf = s->dtype == LA_DTYPE_BF16;
  if (s->d == 128) bf ? launch<128, true>(a, nb, s->B, (hipStream_t)stream) : launch<128, false>(a, nb, s->B, (hipStream_t)stream);
  else bf ? launch<64, true>(a, nb, s->B, (hipStream_t)stream) : launch<64, false>(a, nb, s->B, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? LA_OK : LA_ERR_HIP;
}
