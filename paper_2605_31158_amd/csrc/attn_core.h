// The tile core of the attention kernels on gfx950 (attn.hip, seq_attn.hip): tiles of 64 keys in
// LDS, S^T = K Q^T and O^T += V^T P^T on MFMA for 32 query rows per wave, and the online softmax
// between them.  What bounds it and why it is cut like this is said where the loops are, in attn.hip.
#pragma once

#include <math.h>

#include <type_traits>

#include "la_internal.h"

namespace la {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int KT = 64;          // keys per tile
constexpr int QW = 32;          // query rows per wave
constexpr int QR = 256;         // query rows per unit (workgroup)
constexpr int kMaxPersist = 256;        // persistent workgroups: one per CU, at most 256

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef short v8i16 __attribute__((ext_vector_type(8)));
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

// Shape of the MFMAs for head dimension D (MR x MR x KC) and what follows from it: lane l is row or
// column l % MR of group l / MR; it holds AR accumulator values, of rows acc_row(i) + 4 (l / MR).
template <int D>
struct Mma {
  static constexpr int MR = D == 128 ? 16 : 32;
  static constexpr int NG = 64 / MR;         // lane groups
  static constexpr int KC = 8 * NG;          // contraction depth: 8 values per lane
  static constexpr int QT = 32 / MR;         // MFMA columns of a wave's 32 query rows
  static constexpr int AR = MR * MR / 64;
  typedef typename std::conditional<MR == 16, f32x4, f32x16>::type Acc;
  __device__ static constexpr int acc_row(int i) { return 8 * (i >> 2) + (i & 3); }
  __device__ static __forceinline__ Acc mma(bf16x8 a, bf16x8 b, Acc c) {
    if constexpr (MR == 16)
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
typedef float f32x2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
#define LDS_AS __attribute__((address_space(3)))

// Two floats -> two bf16 (round to nearest even) in one v_cvt_pk_bf16_f32.
__device__ inline uint32_t pack_bf16x2(float lo, float hi) {
  const f32x2v f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2v));
}

// Workgroup barrier for waves with asynchronous tile loads in flight that they do not wait for
// here (an LDS release fence would wait for them: they write LDS).  The empty asm statements keep
// the compiler from moving memory accesses across the barrier; every LDS read of the wave has been
// consumed by then.  The barrier waits for nothing else: a wave whose tile other waves read behind it
// has waited for that tile itself, by vmcnt where it came by asynchronous loads and by lgkmcnt(0) where
// it was stored (the tiles of a 4-bit cache).
__device__ __forceinline__ void phase_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Waits until at most n of this wave's vector memory operations are outstanding (n < 16).
template <int n>
__device__ __forceinline__ void wait_vmem() {
  __builtin_amdgcn_s_waitcnt(0x0F70 | n);   // vmcnt(n), expcnt and lgkmcnt left at their maximum
}

// LDS layout: K and V tiles of 64 key rows of D bf16, row-major and not padded, so that a tile is
// an even share of four loads for each of four waves.  In a K row the 16-byte slots are permuted
// (slot c of row r is stored at slot c ^ kswz(r)): an MFMA operand read touches 16 rows per LDS
// cycle at one c.  In a V row the chunks of 2 MR bytes are (chunk c at chunk c ^ vswz(r)): a
// transpose read touches, per half-wave, 8 consecutive rows x 32 bytes (MR = 16) or 4 x 64 (32).
// Both spread over all 64 banks.  Every K operand read is one of D/KC lane bases (base ^ 16 NG ks)
// plus a compile-time offset, every V read one of D/MR (base ^ 2 MR dt).
template <int D>
struct Tile {
  static constexpr int STRIDE = D * 2;                 // bytes per row
  static constexpr int SLOTS = STRIDE / 16;            // 16-byte slots per row
  static constexpr int BYTES = KT * STRIDE;
  static constexpr int PER = BYTES / 4096;             // 1 KiB loads per loading wave (four load a tile)
  // slot permutation of K row r: the 16 rows one LDS cycle of an operand read touches lie in
  // distinct 16-byte bank groups (D = 64: two rows share the 256 bytes of all banks)
  __device__ static constexpr int kswz(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
  // chunk permutation of V row r: eight 32-byte chunks (D = 128), or two of 64 bytes, with two rows
  // sharing the 256 bytes of all banks (D = 64)
  __device__ static constexpr int vswz(int r) { return D == 128 ? (r & 7) : ((r >> 1) & 1); }
};

// Global byte offset that lane `lane` of the i-th load of loading wave lw fetches, less the 1024 i
// of the instruction's immediate (rows `stride` bytes apart, at least T::STRIDE): LDS slot 64 i + lane of the wave's quarter of the tile holds
// slot s ^ kswz(row) of its row (K) or part w of chunk pc ^ vswz(row) (V).
template <int D, bool V>
__device__ inline uint32_t slot_offset(int lw, int i, int lane, uint32_t stride = Tile<D>::STRIDE) {
  using T = Tile<D>;
  const int slot = 64 * i + lane;
  const int row = slot / T::SLOTS, sp = slot % T::SLOTS;
  constexpr int CS = Mma<D>::MR / 8;           // slots of a V chunk
  const int src = V ? ((sp / CS) ^ T::vswz(row)) * CS + sp % CS : (sp ^ T::kswz(row));
  return (uint32_t)(lw * (KT / 4) + row) * stride + (uint32_t)(src * 16 - 1024 * i);
}

// This wave's quarter of one tile of K or V (base: the tensor): a buffer descriptor that starts at
// the tile and ends at its head's Lk (rows past Lk read as zero; nrec 0 reads nothing).  The
// immediate offset of a load counts for both its addresses, so one LDS base (M0) serves all of
// them.  Written as one asm statement (the loads return nothing to registers): for the builtin the
// compiler waits for every load in flight before LDS reads whose stage it cannot tell apart.  M0 is
// an operand, so that the compiler writes it and knows what it holds.  The s_nop covers M0 and a
// descriptor word written just before by a VALU instruction (v_readlane).
template <int D>
__device__ __forceinline__ void issue_tile(unsigned char* dst, const uint16_t* base, uint64_t off, uint32_t nrec,
                                           const uint32_t* lane_off) {
  const uint64_t b = (uint64_t)(uintptr_t)base + off;
  const u32x4 rsrc = u32x4{(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, nrec, 0x00020000u};
  const uint32_t m0 = (uint32_t)(uintptr_t)(LDS_AS unsigned char*)dst;
  if constexpr (Tile<D>::PER == 4)
    asm volatile("s_nop 4\n\t"
                 "buffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %2, %5, 0 offen offset:1024 lds\n\t"
                 "buffer_load_dwordx4 %3, %5, 0 offen offset:2048 lds\n\t"
                 "buffer_load_dwordx4 %4, %5, 0 offen offset:3072 lds"
                 ::"{m0}"(m0), "v"(lane_off[0]), "v"(lane_off[1]), "v"(lane_off[2]), "v"(lane_off[3]), "s"(rsrc)
                 : "memory");
  else
    asm volatile("s_nop 4\n\t"
                 "buffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %2, %3, 0 offen offset:1024 lds"
                 ::"{m0}"(m0), "v"(lane_off[0]), "v"(lane_off[1]), "s"(rsrc)
                 : "memory");
}

// Per-wave constants of the tile loop (klimit changes with the unit).
struct WaveCtx {
  int klimit[2];             // keys >= klimit[qt] are invisible to this lane's query row of column qt
  int kbase, vbase;          // LDS read bases of this lane inside a K / V tile
  int g4;                    // 4 (lane / MR)
  float scale_log2;
};

// Scheduling-group masks of __builtin_amdgcn_sched_group_barrier.
constexpr int kSgMfma = 0x008;
constexpr int kSgDsRead = 0x100;

// S^T = K Q^T for one 64-key tile: accumulators [MR keys][MR queries].  The K operand reads run
// AHEAD operands ahead of their use, so LDS latency overlaps the matrix pipeline.
template <int D>
__device__ __forceinline__ void qk_tile(const unsigned char* __restrict__ kb,
                                        const bf16x8 (*qreg)[Mma<D>::QT],
                                        typename Mma<D>::Acc (*sacc)[Mma<D>::QT], int kbase) {
  using X = Mma<D>;
  constexpr int NT = KT / X::MR;                   // key groups
  constexpr int NO = NT * (D / X::KC);             // K operands per tile
  constexpr int AHEAD = X::MR == 16 ? 6 : 4;
  bf16x8 ka[NO];
#pragma unroll
  for (int i = 0; i < NO; ++i)
    ka[i] = *(const bf16x8*)(kb + (kbase ^ (16 * X::NG * (i / NT))) + (i % NT) * X::MR * Tile<D>::STRIDE);
#pragma unroll
  for (int kt = 0; kt < NT; ++kt)
#pragma unroll
    for (int qt = 0; qt < X::QT; ++qt)
#pragma unroll
      for (int i = 0; i < X::AR; ++i) sacc[kt][qt][i] = 0.f;
#pragma unroll
  for (int i = 0; i < NO; ++i)
#pragma unroll
    for (int qt = 0; qt < X::QT; ++qt) sacc[i % NT][qt] = X::mma(ka[i], qreg[i / NT][qt], sacc[i % NT][qt]);
  __builtin_amdgcn_sched_group_barrier(kSgDsRead, AHEAD, 0);
#pragma unroll
  for (int i = 0; i < NO - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(kSgMfma, X::QT, 0);
    __builtin_amdgcn_sched_group_barrier(kSgDsRead, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kSgMfma, X::QT * AHEAD, 0);
}

// O^T += V^T P^T for one 64-key tile (P: B operands [step of KC keys][MR queries]).  Slot e of lane
// group g of a step's contraction index is key 4 g + e (e < 4) or KC/2 + 4 g + e - 4 of the step,
// which is how the S accumulators lie; the two transpose reads of a V^T operand follow it.  They
// run AHEAD operands ahead of their use.
template <int D>
__device__ __forceinline__ void pv_tile(const unsigned char* __restrict__ vb, const bf16x8 (*pb)[Mma<D>::QT],
                                        typename Mma<D>::Acc (*oacc)[Mma<D>::QT], int vbase) {
  using X = Mma<D>;
  constexpr int DT = D / X::MR;
  constexpr int NO = (KT / X::KC) * DT;            // V^T operands per tile
  constexpr int AHEAD = X::MR == 16 ? 3 : 2;
  bf16x8 va[NO];
#pragma unroll
  for (int i = 0; i < NO; ++i) {
    const unsigned char* vp = vb + (vbase ^ (2 * X::MR * (i % DT))) + (X::KC * (i / DT)) * Tile<D>::STRIDE;
    const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS v4i16*)(vp));
    const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS v4i16*)(vp + X::KC / 2 * Tile<D>::STRIDE));
    const v8i16 a8 = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    va[i] = __builtin_bit_cast(bf16x8, a8);
  }
#pragma unroll
  for (int i = 0; i < NO; ++i)
#pragma unroll
    for (int qt = 0; qt < X::QT; ++qt) oacc[i % DT][qt] = X::mma(va[i], pb[i / DT][qt], oacc[i % DT][qt]);
  __builtin_amdgcn_sched_group_barrier(kSgDsRead, 2 * AHEAD, 0);
#pragma unroll
  for (int i = 0; i < NO - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(kSgMfma, X::QT, 0);
    __builtin_amdgcn_sched_group_barrier(kSgDsRead, 2, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kSgMfma, X::QT * AHEAD, 0);
}

// Masks of one tile (ragged tail, frame-causal pairs, padding at the end of the tile): invisible
// keys get -inf.  Lane holds keys key0 + MR kt + acc_row(i) + 4 (l / MR) of its query rows
// MR qt + l % MR; the NG lanes of one l % MR together hold a row's 64 keys.  The record's flag says
// that some row of the unit needs a mask; in a unit of several frames most waves do not (without
// the test the 78-of-1560 case of plan_union_kernel takes 564 instead of 515 us).
template <int D>
__device__ __forceinline__ void mask_tile(typename Mma<D>::Acc (*sacc)[Mma<D>::QT], int key0, int pad,
                                          const WaveCtx& w) {
  using X = Mma<D>;
  int vis[X::QT];                    // visible keys at the front of the tile
  bool need = false;
#pragma unroll
  for (int qt = 0; qt < X::QT; ++qt) {
    vis[qt] = min(w.klimit[qt] - key0, KT - pad);
    need = need || vis[qt] < KT;
  }
  if (!__any(need)) return;
#pragma unroll
  for (int qt = 0; qt < X::QT; ++qt) {
    const int lim = vis[qt] - w.g4;
#pragma unroll
    for (int kt = 0; kt < KT / X::MR; ++kt)
#pragma unroll
      for (int i = 0; i < X::AR; ++i)
        if (X::MR * kt + X::acc_row(i) >= lim) sacc[kt][qt][i] = -INFINITY;
  }
}

// P = 2^(S*scale - m) of the query column qt rounded to bf16 into the B operands of the P.V
// product; returns the sum of the lane's values (fp32, before rounding).
template <int D>
__device__ __forceinline__ float softmax_exp(const typename Mma<D>::Acc (*sacc)[Mma<D>::QT],
                                             bf16x8 (*pb)[Mma<D>::QT], int qt, float m_use, float scale_log2) {
  using X = Mma<D>;
  float rs0 = 0.f, rs1 = 0.f;
#pragma unroll
  for (int s = 0; s < KT / X::KC; ++s) {
    u32x4 pw;
#pragma unroll
    for (int j2 = 0; j2 < 4; ++j2) {
      const int e = 8 * s + 2 * j2;
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[e / X::AR][qt][e % X::AR], scale_log2, -m_use));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[e / X::AR][qt][e % X::AR + 1], scale_log2, -m_use));
      pw[j2] = pack_bf16x2(p0, p1);
      rs0 += p0;
      rs1 += p1;
    }
    pb[s][qt] = __builtin_bit_cast(bf16x8, pw);
  }
  return rs0 + rs1;
}

// Max over the NG lanes that hold a query row's keys.
template <int D>
__device__ __forceinline__ float row_max(float x) {
  if constexpr (Mma<D>::NG == 4) {
    const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x),
                                                    false, false);
    x = fmaxf(__builtin_bit_cast(float, (uint32_t)s[0]), __builtin_bit_cast(float, (uint32_t)s[1]));
  }
  const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x),
                                                  false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)s[0]), __builtin_bit_cast(float, (uint32_t)s[1]));
}

// Softmax of one tile with a lazily raised running max (base 2).  P is first formed against the
// current max m_run, which is left alone while every sum of a row's values over half of the tile's
// keys stays within 2^8 (so no value exceeds 2^8 and the O accumulators keep their range); otherwise
// the row max of the tile is taken, m_run raised to it, O and l rescaled, and P formed again.  Most
// tiles thus skip both the row max and the rescale.  On the first tile of a piece m_run is -inf: the
// first pass then gives inf or NaN sums, which fail the test too.
// A raised max makes the largest P exactly 1, with no rounding to bf16, so the limit matters to the
// precision: with 2^8 over a lane's 16 values alone (d = 128) the error against 64 bits was up to
// 0.15 % larger, 0.0023393 instead of 0.0023358 at 720P.  A lane tests its own values first, at half
// the limit where it holds a quarter of the keys; the sums of the halves are taken where that fails
// (in every tile they cost 2 % of the call).
template <int D>
__device__ __forceinline__ void softmax_tile(typename Mma<D>::Acc (*sacc)[Mma<D>::QT], bf16x8 (*pb)[Mma<D>::QT],
                                             typename Mma<D>::Acc (*oacc)[Mma<D>::QT], float* m_run, float* l_run,
                                             float scale_log2) {
  using X = Mma<D>;
  float rs[X::QT];
  bool over = false;
#pragma unroll
  for (int qt = 0; qt < X::QT; ++qt) {
    rs[qt] = softmax_exp<D>(sacc, pb, qt, m_run[qt], scale_log2);
    over = over || !(rs[qt] <= (X::NG == 4 ? 128.f : 256.f));
  }
  if (__builtin_expect(__any(over), 0)) {
    if constexpr (X::NG == 4) {
      over = false;
#pragma unroll
      for (int qt = 0; qt < X::QT; ++qt) {
        const uint32_t r = __builtin_bit_cast(uint32_t, rs[qt]);
        const auto h = __builtin_amdgcn_permlane32_swap(r, r, false, false);      // lanes l and l ^ 32
        over = over || !(__builtin_bit_cast(float, (uint32_t)h[0]) + __builtin_bit_cast(float, (uint32_t)h[1]) <= 256.f);
      }
    }
    if (X::NG == 2 || __any(over)) {
#pragma unroll
      for (int qt = 0; qt < X::QT; ++qt) {
        float mx = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < KT / X::MR; ++kt)
#pragma unroll
          for (int i = 0; i < X::AR; ++i) mx = fmaxf(mx, sacc[kt][qt][i]);
        const float mt = row_max<D>(mx) * scale_log2;
        if (mt > m_run[qt]) {
          const float alpha = __builtin_amdgcn_exp2f(m_run[qt] - mt);   // 0 while m_run is -inf
          m_run[qt] = mt;
          l_run[qt] *= alpha;
#pragma unroll
          for (int dt = 0; dt < D / X::MR; ++dt) oacc[dt][qt] *= alpha;
        }
        rs[qt] = softmax_exp<D>(sacc, pb, qt, m_run[qt] == -INFINITY ? 0.f : m_run[qt], scale_log2);
      }
    }
  }
#pragma unroll
  for (int qt = 0; qt < X::QT; ++qt) l_run[qt] += rs[qt];
}

}  // namespace
}  // namespace la
