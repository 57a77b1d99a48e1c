// Attention of few query rows per sequence over a 4-bit cache on gfx950: the next token of every
// sequence, or a handful of proposed ones (many rows: seq_attn.hip).
//
// Bound by reading the cache once: (d + d / 16) bytes per token and key head.  The codes go from HBM to
// registers and to the MFMAs with no LDS between: K is the A operand of S^T = K Q^T, and its rows are
// 16 bytes a lane along d (which value of d stands where in the contraction is free, as long as Q
// follows); V is the A operand of O^T = V^T P^T, 16 bytes a lane along 4 tokens, and the P that its
// lanes need are the S that they hold: with keys 4 c + kt in row c of the kt-th S tile, lane (c, g)
// holds the keys 16 g .. 16 g + 15 of query row c, which are the keys of its V words.  Conversions cost
// one instruction per two values, and V's pairs lie along d where the operand wants them along the
// tokens: one more byte permutation per two values.
//
// A workgroup's four waves take the tiles (64 keys) of a piece in turn, each with its own (m, l, O);
// they are joined in LDS at the end of the piece.  Pieces are shares of one line of work (seq_walk.h),
// cut units are joined by seq_merge (seq_attn.hip).  Each wave issues the next tile's codes, and the page
// numbers of the one behind, before it works on one.  (The compiler joins the paths with and without a
// next tile and waits for the loads of the shorter one, so a wave may wait for most of what it issued;
// loads without the branch, with waits for exactly the present tile, took the same time, 40.4 against
// 41.0 us on 32 sequences: eight waves to a CU cover one another.)
//
// 32 sequences of 1000 to 16000 tokens (32 query heads over 8, d 128: 190 MB) take 49 us, 4 of them
// before the first codes arrive and 4.5 for the join: 4.7 TB/s while it streams, a large copy's rate being
// 5.1; with most of it in the last-level cache 41 us, 5.8 TB/s.  One sequence of 1000 tokens takes 11 us.
// 8 sequences of 5 queries (32 query heads over 4: 40 packed rows, two units of up to 32) over 700 to 9000 tokens
// take 24 us at d 128.  The 32-row instance has all 256 vector registers there and spills two, written before its
// tile loop and read behind it.
//
// The weights 2^(s - m) are rounded to bf16 for the product with V, as in seq_attn.hip; m, l (of the weights
// before they are rounded) and O are fp32.
#include <math.h>

#include <type_traits>

#include "kv4.h"
#include "la_internal.h"
#include "seq_walk.h"

namespace la {
namespace {

constexpr int kTokenWaves = 4;
constexpr int kTokenThreads = 64 * kTokenWaves;

template <int D>
struct TokenTile {                       // a lane's codes of one tile
  uint32_t k[4][D / 32];                 // K of key 4 c + kt: its g-th quarter
  uint32_t v[4][D / 32];                 // V of keys 16 g + 4 q ..: chunk c of each
  uint32_t ks, vs[4];                    // their scales
  bool kok, vok;                         // their pages exist
};

template <int D>
__device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p) {
  if constexpr (D == 128) {
    const u32x4 x = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
  } else {
    const u32x2 x = *(const u32x2*)p;
    w[0] = x[0];
    w[1] = x[1];
  }
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  const f2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, b2));
}

// max over the four lanes c, c + 16, c + 32, c + 48
__device__ __forceinline__ float group_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float((uint32_t)a[0]), __uint_as_float((uint32_t)a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float((uint32_t)b[0]), __uint_as_float((uint32_t)b[1]));
}

template <int D, int QT>
__global__ __launch_bounds__(kTokenThreads, 2) void token_attn_kernel(SeqGeom g, SeqIo io, CacheGeom cg) {
  using F = Kv4<D>;
  constexpr int R = 16 * QT, KS = D / 32, DT = D / 16;
  constexpr int OS = D + 4;                           // row stride of the joint O, in floats
  __shared__ float sm_o[kTokenWaves][R][OS];
  __shared__ float sm_m[kTokenWaves][R], sm_l[kTokenWaves][R];

  const int P = gridDim.x;
  const int lambda = (blockIdx.x & 7) * (P >> 3) + (blockIdx.x >> 3);
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (g.cuts && tid == 0) io.cut[2 * lambda] = io.cut[2 * lambda + 1] = int4{0, 0, 0, 0};
  Walk wk = start_walk<true>(g, lambda, P);
  const int page = 1 << cg.log_p;

  while (wk.more()) {
    uint64_t unit_end;
    const Piece pc = walk_piece(g, wk, &unit_end);
    if (pc.tb > pc.ta) {
      const int kvh = wk.kvh, lk = wk.q.lk;
      const int32_t* row_pages = cg.table + (int64_t)wk.s * cg.max_pages;
      // Q: lane (c, g) has values (d / 4) g + 8 ks .. of row c, as its K words have
      bf16x8 qreg[KS][QT];
      int limit[QT];
      f32x4 oacc[DT][QT];
      float m_run[QT], l_run[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const Row row = unit_row(g, wk, 16 * qt + c);
        const uint16_t* src = io.q + (int64_t)(wk.q.q0 + row.token) * io.q_tok + (int64_t)row.head * io.q_head + (D / 4) * lg;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          u32x4 x = u32x4{0u, 0u, 0u, 0u};
          if (row.ok) x = *(const u32x4*)(src + 8 * ks);
          qreg[ks][qt] = __builtin_bit_cast(bf16x8, x);
        }
        limit[qt] = row.ok ? token_keys(g, wk.q, row.token) : 0x7fffffff;
        m_run[qt] = -INFINITY;
        l_run[qt] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) oacc[t][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      // first tile that some row does not see whole
      const int open = g.causal ? min(lk, max(0, lk - wk.q.lq + wk.b * g.TB + 1)) : lk;

      auto load_ids = [&](int t, int* kid, int* vid) {
        const int last = cg.max_pages - 1;
        *kid = row_pages[min((64 * t + 4 * c) >> cg.log_p, last)];
        *vid = row_pages[min((64 * t + 16 * lg) >> cg.log_p, last)];
      };
      auto load_tile = [&](int t, int kid, int vid, TokenTile<D>& x) {
        const int kin = (64 * t + 4 * c) & (page - 1), vin = (64 * t + 16 * lg) & (page - 1);
        const uint8_t* kp = page_of<D>(cg, kid, kvh, &x.kok);
        const uint8_t* vp = page_of<D>(cg, vid, kvh, &x.vok);
        const uint8_t* kc = kp + kin * F::ROW + lg * (F::ROW / 4);
        const uint8_t* vc = vp + F::v_code(page) + ((vin >> 2) * 16 + c) * (4 * F::WB);
#pragma unroll
        for (int i = 0; i < 4; ++i) load_words<D>(x.k[i], kc + i * F::ROW);
#pragma unroll
        for (int i = 0; i < 4; ++i) load_words<D>(x.v[i], vc + i * (64 * F::WB));
        x.ks = *(const uint32_t*)(kp + F::k_scale(page) + (lg * D / 128) * page + kin);
        const u32x4 vs = *(const u32x4*)(vp + F::v_scale(page) + (c * D / 512) * page + vin);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.vs[i] = vs[i];
      };
      auto work = [&](int t, TokenTile<D>& x) {
        const int key0 = 64 * t;
        // pages that do not exist read as zeros; V behind the last key must be finite to meet its weight 0
        if (__any(!x.kok || !x.vok)) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
              x.k[i][j] = x.kok ? x.k[i][j] : 0u;
              x.v[i][j] = x.vok ? x.v[i][j] : 0u;
            }
          x.ks = x.kok ? x.ks : 0x7f7f7f7fu;
#pragma unroll
          for (int i = 0; i < 4; ++i) x.vs[i] = x.vok ? x.vs[i] : 0x7f7f7f7fu;
        }
        if (key0 + 64 > lk) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int n = lk - (key0 + 16 * lg + 4 * i);       // of these 4 tokens, those that exist
            const uint32_t behind = n >= 4 ? 0u : (n <= 0 ? ~0u : ~0u << (8 * n));
            x.vs[i] = (x.vs[i] & ~behind) | (0x7f7f7f7fu & behind);
          }
        }
        // S^T: tile kt, row 4 lg + i of it is key 16 lg + 4 i + kt
        f32x4 s[4][QT];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
          const float sc = scale_of(x.ks, kt);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) s[kt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const bf16x8 a = __builtin_bit_cast(bf16x8, fp4x8(x.k[kt][ks], sc));
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
              s[kt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qreg[ks][qt], s[kt][qt], 0, 0, 0);
          }
        }
        if (key0 + 64 > open) {
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) {
            const int lim = limit[qt] - key0 - 16 * lg;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (4 * i + kt >= lim) s[kt][qt][i] = -INFINITY;
          }
        }
        bf16x8 pb[2][QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          float mx = -INFINITY;
#pragma unroll
          for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[kt][qt][i]);
          mx *= io.scale_log2;
          // the maximum is raised where a weight would pass 2^8, so that most tiles need no rescale
          if (__any(!(mx <= m_run[qt] + 8.0f))) {
            const float mt = group_max(mx);
            if (mt > m_run[qt]) {
              const float a = __builtin_amdgcn_exp2f(m_run[qt] - mt);
              m_run[qt] = mt;
              l_run[qt] *= a;
#pragma unroll
              for (int t2 = 0; t2 < DT; ++t2) oacc[t2][qt] *= a;
            }
          }
          const float m_use = m_run[qt] == -INFINITY ? 0.f : m_run[qt];
          float p[4][4];
          float sum = 0.f;
#pragma unroll
          for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              p[kt][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][qt][i], io.scale_log2, -m_use));
              sum += p[kt][i];
            }
          l_run[qt] += sum;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            pb[h][qt] = __builtin_bit_cast(
                bf16x8, u32x4{pack2(p[0][2 * h], p[1][2 * h]), pack2(p[2][2 * h], p[3][2 * h]),
                              pack2(p[0][2 * h + 1], p[1][2 * h + 1]), pack2(p[2][2 * h + 1], p[3][2 * h + 1])});
        }
        // O^T: slot e of step h is key 16 lg + 8 h + e; row c of tile t is value c DT + t
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float sc[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) sc[e] = scale_of(x.vs[2 * h + (e >> 2)], e & 3);
          auto pairs = [&](auto B) {
            constexpr int b = decltype(B)::value;
            uint32_t y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t* w = x.v[2 * h + (e >> 2)];
              if constexpr (D == 128) y[e] = fp4x2<b>(w[e & 3], sc[e]);
              else y[e] = (e & 1) ? fp4x2<2 + b>(w[(e & 3) >> 1], sc[e]) : fp4x2<b>(w[(e & 3) >> 1], sc[e]);
            }
            u32x4 lo, hi;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              lo[e] = __builtin_amdgcn_perm(y[2 * e + 1], y[2 * e], 0x05040100u);
              hi[e] = __builtin_amdgcn_perm(y[2 * e + 1], y[2 * e], 0x07060302u);
            }
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
              oacc[2 * b][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), pb[h][qt],
                                                                       oacc[2 * b][qt], 0, 0, 0);
              oacc[2 * b + 1][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), pb[h][qt],
                                                                           oacc[2 * b + 1][qt], 0, 0, 0);
            }
          };
          pairs(std::integral_constant<int, 0>{});
          pairs(std::integral_constant<int, 1>{});
          if constexpr (D == 128) {
            pairs(std::integral_constant<int, 2>{});
            pairs(std::integral_constant<int, 3>{});
          }
        }
      };

      // this wave's tiles: ta + wave, + 4, ..; the next one's codes in flight, and the page numbers behind it
      int t = pc.ta + wave;
      if (t < pc.tb) {
        TokenTile<D> x0, x1;
        int kid, vid;
        load_ids(t, &kid, &vid);
        load_tile(t, kid, vid, x0);
        load_ids(t + kTokenWaves, &kid, &vid);
        for (;;) {
          if (t + kTokenWaves < pc.tb) {
            load_tile(t + kTokenWaves, kid, vid, x1);
            load_ids(t + 2 * kTokenWaves, &kid, &vid);
          }
          work(t, x0);
          t += kTokenWaves;
          if (t >= pc.tb) break;
          if (t + kTokenWaves < pc.tb) {
            load_tile(t + kTokenWaves, kid, vid, x0);
            load_ids(t + 2 * kTokenWaves, &kid, &vid);
          }
          work(t, x1);
          t += kTokenWaves;
          if (t >= pc.tb) break;
        }
      }

      // join the waves; lane (c, g) holds values 4 g DT .. of row c: O^T[(4 g + i) DT + t]
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        float l = l_run[qt];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const int r = 16 * qt + c;
        if (lg == 0) {
          sm_m[wave][r] = m_run[qt];
          sm_l[wave][r] = l;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int t2 = 0; t2 < DT; t2 += 4)
            *(f32x4*)&sm_o[wave][r][(4 * lg + i) * DT + t2] =
                f32x4{oacc[t2][qt][i], oacc[t2 + 1][qt][i], oacc[t2 + 2][qt][i], oacc[t2 + 3][qt][i]};
      }
      __syncthreads();
      constexpr int TPR = kTokenThreads / R, W = D / TPR;      // threads of a row, values of a thread
      const int r = tid / TPR, part = tid % TPR;
      const Row row = unit_row(g, wk, r);
      float mx = -INFINITY;
#pragma unroll
      for (int w = 0; w < kTokenWaves; ++w) mx = fmaxf(mx, sm_m[w][r]);
      const float base = mx == -INFINITY ? 0.f : mx;
      float l = 0.f, acc[W];
#pragma unroll
      for (int e = 0; e < W; ++e) acc[e] = 0.f;
#pragma unroll
      for (int w = 0; w < kTokenWaves; ++w) {
        const float a = __builtin_amdgcn_exp2f(sm_m[w][r] - base);
        l += a * sm_l[w][r];
#pragma unroll
        for (int e = 0; e < W; e += 4) {
          const f32x4 x = *(const f32x4*)&sm_o[w][r][part * W + e];
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[e + u] += a * x[u];
        }
      }
      const bool whole = pc.ta == 0 && pc.tb == pc.n;
      const int slot = 2 * lambda + (pc.ta == 0 ? 1 : 0);
      if (!whole && tid == 0) io.cut[slot] = unit_record(g, wk);
      if (!row.ok) {
      } else if (whole) {
        const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);   // a NaN stays one
        uint16_t* dst = io.o + (int64_t)(wk.q.q0 + row.token) * io.o_tok + (int64_t)row.head * io.o_head + part * W;
#pragma unroll
        for (int e = 0; e < W; e += 4)
          *(u32x2*)(dst + e) = u32x2{pack2(acc[e] * inv, acc[e + 1] * inv), pack2(acc[e + 2] * inv, acc[e + 3] * inv)};
        if (io.lse && part == 0)
          io.lse[(int64_t)(wk.q.q0 + row.token) * g.Hq + row.head] =
              l == 0.f ? -INFINITY : (mx + log2f(l)) * 0.69314718055994531f;
      } else {
        const size_t prow = (size_t)slot * R + r;
#pragma unroll
        for (int e = 0; e < W; e += 4)
          *(f32x4*)(io.part_o + prow * D + part * W + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
        if (part == 0) {
          io.part_m[prow] = mx;
          io.part_l[prow] = l;
        }
      }
      __syncthreads();
    }
    walk_on<true>(g, wk, unit_end);
  }
}

template <int D, int QT>
hipError_t launch_qt(const SeqGeom& g, const SeqIo& io, const CacheGeom& cg, int P, hipStream_t st) {
  hipLaunchKernelGGL((token_attn_kernel<D, QT>), dim3(P), dim3(kTokenThreads), 0, st, g, io, cg);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_tokens(const SeqGeom& g, const SeqIo& io, const CacheGeom& cg, int d, int rows, int P,
                               hipStream_t st) {
  hipError_t e;
  if (rows == 16) e = d == 128 ? launch_qt<128, 1>(g, io, cg, P, st) : launch_qt<64, 1>(g, io, cg, P, st);
  else e = d == 128 ? launch_qt<128, 2>(g, io, cg, P, st) : launch_qt<64, 2>(g, io, cg, P, st);
  return e == hipSuccess && g.cuts ? launch_cache_merge(g, io, d, rows, P, st) : e;
}

}  // namespace la
