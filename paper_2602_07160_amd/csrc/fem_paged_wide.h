// The FEM read of many query rows over a paged cache: a chunk of a prompt.
//
// The mathematics, the phases of an iteration and their schedule are those of
// the dense read (fem_softmax_kernel.h): S^T = K Q^T, the online softmax, the
// tilt shared by the workgroup's eight waves, O^T += E^T P^T, one barrier per
// 64-key tile.  What differs:
//
//   * Rows.  A block's 256 rows are (token, query head of the group) pairs of one
//     sequence and cached head, so a group's heads share the tile's loads and its
//     tilt.  A block with at most 128 rows runs the form with two key groups.
//   * Tiles come from pages.  Waves 2 i and 2 i + 1 fill the tile's rows 16 i ..
//     16 i + 15, which lie in one page whatever its size, so a wave's loads have
//     one base in scalar registers and the lane offsets of every tile alike.
//   * A quantised cache's codes are loaded as they are into an LDS area of the
//     wave's own; at the end of the iteration before the tile's, the wave turns
//     them into the tile's bf16 rows (exact).  The phases cannot tell the types
//     apart.
//   * Few row blocks are split over the keys; the splits' sums leave as
//     logarithms and are merged by paged_merge_kernel.
//   * Range.  P is lost below 2^-126 and E is at most 2^80, so a term that
//     underflows is at most 2^-46 of the frame; a sum below 2^-20 is formed again,
//     exactly.
//
// MFMA-bound, like the dense read: 4096 tokens behind 12288, 16 heads of 128 in bf16,
// 665 to 696 us by card, 690 to 724 TFLOP/s.
#pragma once

#include "fem_paged_rows.h"
#include "fem_softmax_kernel.h"

namespace fem {
namespace {

constexpr int kWideRows = 256;
constexpr int kWideTile = 64;
constexpr float kWideLow = 0x1p-20f;
constexpr float kNoMax = -3e38f;  // row maximum before the first visible key

template <class C, int KV>
struct WideLds {
  static constexpr bool MX = KV != FEM_KV_BF16;
  static constexpr int RAWK = 1024, RAWV = 1024;  // of a wave
  static constexpr size_t OFF_RAW = (C::LDS + 15) / 16 * 16;
  static constexpr size_t OFF_BAD = OFF_RAW + (MX ? C::NW * (RAWK + RAWV) : 0);
  static constexpr size_t BYTES = OFF_BAD + 16;
  static_assert(BYTES + kItemInts * 4 <= 160 * 1024, "LDS budget");
};

// Lane offset, inside the 16 rows that a pair of waves fills, of the 16-byte slot
// that this lane loads with its wave's u-th instruction, and whether there is one.
template <int W>
struct PairSlots {
  static constexpr int SPR = (W + 8) / 8;       // slots of a padded row
  static constexpr int N = 16 * SPR;            // of the 16 rows
  static constexpr int LOADS = (N + 127) / 128;  // instructions of a wave
  __device__ static __forceinline__ int slot(int u, int half, int lane) {
    return (half + 2 * u) * 64 + lane;
  }
  __device__ static __forceinline__ unsigned offset(int s) {
    const int row = s / SPR, chunk = s % SPR;
    return (unsigned)(row * W + (chunk < W / 8 ? chunk * 8 : 0)) * 2u;
  }
};

// The softmax of a paged read keeps its maximum m in the scores' own scale.  One fma a
// score, s scale2 - m scale2, is off by half the last place of m scale2: 2^-15 at 2^10,
// more than a 2^x can hold from 2^30 on.  A tile with such a row has m subtracted first.
// (It costs 1 %: 4096 rows over 16384 keys took 702 us for 695.  Subtracted always, two
// operations a score, it was 2.8 %.)
template <int NKB>
struct WideSoftmax : Softmax<NKB> {
  float mm;  // what the fma subtracts
  __device__ __forceinline__ void update(float& m, float& apend, float scale2) {
    const float x = fmaxf(this->mx, other_half(this->mx));
    const float mnew = (x - m) * scale2 > kRowLag ? x : m;
    apend = mnew == m ? 1.f : exp2_hw((m - mnew) * scale2);
    m = mnew;
  }
  __device__ __forceinline__ void shift(f32x16 (&sc)[NKB], float m, float scale2) {
    const float ms = fmaxf(m, -3e38f);  // (no key yet: every score is -inf)
    mm = ms * scale2;
    if (__any(fabsf(mm) > 0x1p10f)) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kb][i] -= ms;
      mm = 0.f;
    }
  }
  __device__ __forceinline__ void prob_arg(const f32x16 (&sc)[NKB], f32x2& x, int q, float,
                                           float scale2) const {
    const int ks = q >> 2, u = 2 * (q & 3), kb = ks >> 1, s0 = (ks & 1) * 8;
    x[0] = fmaf(sc[kb][s0 + u], scale2, -mm);
    x[1] = fmaf(sc[kb][s0 + u + 1], scale2, -mm);
  }
};

template <class C, int KV, int NLO>
__device__ __forceinline__ void wide_body(const PagedArgs& a, const ReadArgs& r, const RowItem& it,
                                          int g, int slot_id, unsigned char* smem, int nneed) {
  constexpr bool SPLIT = NLO > 0 && NLO < C::NCB;  // columns hold reordered channels
  constexpr bool MX = KV != FEM_KV_BF16;
  using L = WideLds<C, KV>;
  using PK = PairSlots<C::DK>;
  using PV = PairSlots<C::DV>;
  const Smem<C> sm{smem};
  int* const badflag = reinterpret_cast<int*>(smem + L::OFF_BAD);

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wave_s = __builtin_amdgcn_readfirstlane(wave);
  const int n = lane & 31, hl = lane >> 5;
  const Seq& sq = it.seq;
  const bool causal = r.causal != 0;
  const int r0 = it.rb * kWideRows;
  const int nr = (int)min((long long)sq.n * r.G - r0, (long long)kWideRows);
  const int n_eff = row_limit(sq, r0 + nr - 1, r.G, causal);  // keys of the block's last row
  const int all = (n_eff + kWideTile - 1) / kWideTile;
  const int tb = (int)((long long)it.s * all / it.ns);
  const int te = (int)((long long)(it.s + 1) * all / it.ns);
  const int ntiles = te - tb;
  if (ntiles <= 0) {  // an early block of a sequence has fewer tiles than splits
    float* p = r.wide_part + (size_t)slot_id * r.wide_rps * part_row(C::DV);
    for (int e = tid; e < nr * part_row(C::DV); e += C::NT) p[e] = -INFINITY;
    return;
  }

  if (!SPLIT) {
    for (int j = tid; j < C::DV; j += C::NT) {
      const float bl = r.beta[g * C::DV + j] * kLog2e;
      sm.bl()[j] = bl;
      sm.inv()[j] = 1.f / bl;
    }
  } else if (wave == 0) {
    // the channels that need the lo product first, each group in input order
    int below_lo = 0, below_hi = 0;
#pragma unroll
    for (int c0 = 0; c0 < C::DV; c0 += 64) {
      const int j = c0 + lane;
      const bool valid = j < C::DV;
      const float b = valid ? r.beta[g * C::DV + j] : 1.f;
      const bool need = valid && !(b >= kLoBeta);
      const uint64_t mlo = __ballot(need), mhi = __ballot(valid && !need);
      const int col = need ? below_lo + bits_below(mlo) : nneed + below_hi + bits_below(mhi);
      if (valid) {
        sm.chan()[col] = j;
        sm.bl()[col] = b * kLog2e;
        sm.inv()[col] = 1.f / (b * kLog2e);
      }
      below_lo += __popcll(mlo);
      below_hi += __popcll(mhi);
    }
  }
  if (tid == 0) *badflag = 0;

  const int rw = C::KG == 1 ? wave : wave % C::RW;  // row block of this wave
  const int kg = C::KG == 1 ? 0 : wave / C::RW;     // its half of every tile's keys
  const int wr0 = rw * 32;                          // first row of this wave in the block
  const bool wave_live = wr0 < nr;
  const int row = r0 + min(wr0 + n, nr - 1);        // rows past the last repeat it
  const int tm = row_limit(sq, row, r.G, causal) - 1;  // last key of this lane's row
  // first tile (of the split) that holds a key the wave's first row does not see
  const int wlast =
      row_limit(sq, r0 + min(wr0, nr - 1), r.G, causal) / kWideTile - tb;

  // ---- tile loads: this wave's 16 rows of a tile
  const int pair = wave_s >> 1, half = wave_s & 1;
  const unsigned lds0 = lds_addr(smem);
  unsigned koff[PK::LOADS], voff[PV::LOADS];
  if constexpr (!MX) {
#pragma unroll
    for (int u = 0; u < PK::LOADS; ++u) koff[u] = PK::offset(PK::slot(u, half, lane));
#pragma unroll
    for (int u = 0; u < PV::LOADS; ++u)
      voff[u] = C::SAME ? koff[u] : PV::offset(PV::slot(u, half, lane));
  }
  const int* const table = a.table + (size_t)it.b * a.table_len;
  const int last_group = (n_eff - 1) & ~15;
  // page of this wave's rows of tile k (rows past the last key read the last group)
  auto group_of = [&](int k) { return min((tb + k) * kWideTile + pair * 16, last_group); };
  auto page_of = [&](int k) {
    return __builtin_amdgcn_readfirstlane(table[group_of(k) >> a.page_log2]);
  };
  // first pool row of that group; a page outside the pool reads page 0 and is noted
  auto row_of = [&](int k, int p) {
    if ((unsigned)p >= (unsigned)a.pages) {
      if (lane == 0) *badflag = 1;
      p = 0;
    }
    return (((size_t)p * a.heads + g) << a.page_log2) + (group_of(k) & (a.page - 1));
  };
  auto kload = [&](int u, const rsrc_t& rs, int buf) {
    if (PK::slot(u, half, lane) < PK::N)
      dma16b(rs, koff[u],
             lds0 + C::OFF_K + buf * C::KB + pair * 16 * C::KROW * 2 + (half + 2 * u) * 1024);
  };
  auto vload = [&](int u, const rsrc_t& rs, int buf) {
    if (PV::slot(u, half, lane) < PV::N)
      dma16b(rs, voff[u],
             lds0 + C::OFF_V + buf * C::VB + pair * 16 * C::VROW * 2 + (half + 2 * u) * 1024);
  };
  auto krsrc = [&](size_t at) { return buffer_rsrc(a.k + at * (C::DK * 2), 16 * C::DK * 2); };
  auto vrsrc = [&](size_t at) { return buffer_rsrc(a.v + at * (C::DV * 2), 16 * C::DV * 2); };
  // quantised: the wave's half of the group's codes (8 rows), 16 a lane
  constexpr int KL = C::DK / 2, VL = C::DV / 2;  // lanes with a piece
  const unsigned raw = L::OFF_RAW + (unsigned)wave_s * (L::RAWK + L::RAWV);
  unsigned kscale = 0, vscale = 0;
  auto load_raw = [&](size_t at) {
    const size_t h8 = at + half * 8;
    if (lane < KL) {
      dma16b(buffer_rsrc(a.k + h8 * C::DK, 8 * C::DK), lane * 16, lds0 + raw);
      kscale = a.ks[h8 * (C::DK / kScaleBlock) + (lane >> 1)];
    }
    if (lane < VL) {
      dma16b(buffer_rsrc(a.v + h8 * C::DV, 8 * C::DV), lane * 16, lds0 + raw + L::RAWK);
      vscale = a.vs[h8 * (C::DV / kScaleBlock) + (lane >> 1)];
    }
  };
  auto convert_one = [&](int lanes, unsigned from, unsigned to, int w, int rowbytes, unsigned sc) {
    if (lane < lanes) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(smem + from + lane * 16);
      const int per = w / 16;  // pieces of a row
      const float s = scale_of(sc);
      u32x4* d = reinterpret_cast<u32x4*>(
          smem + to + (pair * 16 + half * 8 + lane / per) * rowbytes + (lane % per) * 32);
      d[0] = dequant8<KV>(x[0], x[1], s);
      d[1] = dequant8<KV>(x[2], x[3], s);
    }
  };
  auto convert = [&](int buf) {
    if constexpr (MX) {
      convert_one(KL, raw, C::OFF_K + buf * C::KB, C::DK, C::KROW * 2, kscale);
      convert_one(VL, raw + L::RAWK, C::OFF_V + buf * C::VB, C::DV, C::VROW * 2, vscale);
    }
  };

  int pnext;  // page of the next tile to load
  {
    const size_t at = row_of(0, page_of(0));
    if constexpr (MX) {
      load_raw(at);
    } else {
      const rsrc_t rk = krsrc(at), rv = vrsrc(at);
#pragma unroll
      for (int u = 0; u < PK::LOADS; ++u) kload(u, rk, 0);
#pragma unroll
      for (int u = 0; u < PV::LOADS; ++u) vload(u, rv, 0);
    }
    pnext = page_of(1);
  }
  bf16x8 qf[C::NKS];
  {
    const bf16* qp = r.q + (size_t)(sq.q0 + row / r.G) * (size_t)r.qld +
                     (size_t)(g * r.G + row % r.G) * C::DK + hl * 8;
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
  }
  wait_vmem();
  if constexpr (MX) {
    convert(0);
    if (ntiles > 1) load_raw(row_of(1, pnext));
    pnext = page_of(2);
  }
  __syncthreads();
  const int vcol = SPLIT ? sm.chan()[wave * C::CPW + lane % C::CPW] : wave * C::CPW + lane % C::CPW;

  f32x16 acc[C::NCB];
#pragma unroll
  for (int cb = 0; cb < C::NCB; ++cb) acc[cb] = f32x16{};
  f32x16 sacc[C::NKB] = {};
  bf16x8 pbuf[2][C::KS] = {};
  float m = kNoMax;   // finite: a row of a split may see none of its first keys
  float apend = 1.f;
  f32x4 lacc = {};
  bf16x8 lsel;
  {
    const int rr = lane & 15, b = lane >> 4;
    const __bf16 one = ((rr & 3) == 0 && ((rr >> 2) & 1) == (b & 1)) ? (__bf16)1.f : (__bf16)0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) lsel[e] = one;
  }
  const float scale2 = kLog2e / sqrtf((float)C::DK);
  const int kofs = (kg * 32 + n) * C::KROW * 2 + hl * 16;
  const int eofs = n * C::EROW * 2 + kg * 64 + hl * 16;

  // bf16: the next tile's loads, one per slot of phase 1
  constexpr int LD0 = 2;
  auto loads_in_slots = [&](int k) {
    const bool more = !MX && k + 1 < ntiles;
    const size_t at = more ? row_of(k + 1, pnext) : 0;
    const rsrc_t rk = krsrc(at), rv = vrsrc(at);
    if (!MX) pnext = page_of(k + 2);
    return [=](int st) __attribute__((always_inline)) {
      if (!more) return;
      const int u = st - LD0, w = u - PK::LOADS;
      if (u >= 0 && u < PK::LOADS) kload(u, rk, (k + 1) & 1);
      if (w >= 0 && w < PV::LOADS) vload(w, rv, (k + 1) & 1);
    };
  };
  // The end of iteration k: tile k + 1 is in LDS.  8-bit: its codes, loaded an
  // iteration ago, become its rows here, where no operand is live (between the
  // phases: 482 to 498 us for a batch of chunks and tokens), and tile k + 2's are
  // sent for.
  auto arrived = [&](int k) {
    wait_vmem();
    if (MX && k + 1 < ntiles) {
      convert((k + 1) & 1);
      if (k + 2 < ntiles) load_raw(row_of(k + 2, pnext));
      pnext = page_of(k + 3);
    }
    __syncthreads();
  };
  auto rescale = [&](int j, const i32x4& any4) {
    const bool col = (any4[0] | any4[1] | any4[2] | any4[3]) != 0;
    if (col || __any(apend != 1.f)) {
      const float* gcol = sm.g(j & 1);
#pragma unroll
      for (int cb = 0; cb < C::NCB; ++cb) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4 gg = {apend, apend, apend, apend};
          if (col) gg *= *reinterpret_cast<const f32x4*>(gcol + cb * 32 + q * 8 + hl * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[cb][q * 4 + e] *= gg[e];
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      lacc[0] *= apend;
    }
  };
  auto flags_of = [&](int j) {
    const i32x4* uf = reinterpret_cast<const i32x4*>(sm.upd(j & 1));
    i32x4 any4 = uf[0];
#pragma unroll
    for (int w = 1; w < C::NW / 4; ++w) any4 |= uf[w];
    return any4;
  };
#define FEM_WIDE1(PVA, QKT, PPREV, SIDE)                                                       \
  phase1<C, NLO, PVA, QKT>(sm, tl, k, n_eff - (tb + k) * kWideTile, wave, lane, kofs, eofs, vcol, qf, \
                           sacc, acc, lacc, PPREV, lsel, SIDE)
#define FEM_WIDE2(PVB, SM, MK, PPREV, PNEXT)                                                  \
  phase2<C, NLO, PVB, SM, MK, WideSoftmax<C::NKB>>(sm, acc, PPREV, PNEXT, sacc, m, apend, k - 1, eofs,             \
                              (tb + k) * kWideTile + kg * 32, tm, hl, scale2)
  const auto none = [](auto...) __attribute__((always_inline)) {};
  {
    const int k = 0;
    const auto loads = loads_in_slots(0);
    Tilt<C> tl;
    FEM_WIDE1(false, true, pbuf[1], loads);
    if (wlast <= 0) FEM_WIDE2(false, true, true, pbuf[1], pbuf[0]);
    else FEM_WIDE2(false, true, false, pbuf[1], pbuf[0]);
    arrived(0);
  }
  auto body = [&](const int k, auto par) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par)::value;
    if (k > 1) rescale(k - 1, flags_of(k - 1));
    Tilt<C> tl;
    __builtin_amdgcn_s_setprio(1);
    FEM_WIDE1(true, true, pbuf[PAR ^ 1], loads_in_slots(k));
    __builtin_amdgcn_s_setprio(0);
    if (k >= wlast) FEM_WIDE2(true, true, true, pbuf[PAR ^ 1], pbuf[PAR]);
    else FEM_WIDE2(true, true, false, pbuf[PAR ^ 1], pbuf[PAR]);
    arrived(k);
  };
  int kk = 1;
  for (; kk + 1 < ntiles; kk += 2) {
    body(kk, std::integral_constant<int, 1>());
    body(kk + 1, std::integral_constant<int, 0>());
  }
  if (kk < ntiles) body(kk, std::integral_constant<int, 1>());
  auto tail = [&](auto par) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par)::value;
    const int k = ntiles;
    if (k > 1) rescale(k - 1, flags_of(k - 1));
    Tilt<C> tl;
    FEM_WIDE1(true, false, pbuf[PAR], none);
    FEM_WIDE2(true, false, false, pbuf[PAR], pbuf[PAR]);
  };
  if ((ntiles - 1) & 1) tail(std::integral_constant<int, 1>());
  else tail(std::integral_constant<int, 0>());
#undef FEM_WIDE1
#undef FEM_WIDE2

  // ---- epilogue: rows staged in LDS (the tile buffers are free) in channel order
  constexpr int SROW = C::DV + 4;
  static_assert(C::RW * 32 * SROW * 4 <= C::OFF_F, "staging must not reach the tables");
  __syncthreads();
  float* stage = reinterpret_cast<float*>(smem) + rw * 32 * SROW;
  if constexpr (C::KG == 2) {
    // the second key group's sums meet the first's: same column frame, own row maxima
    constexpr int NX = C::NCB * 16;
    static_assert(64 * (NX + 2) <= 32 * SROW, "a row block's area holds the group's state");
    if (kg == 1) {
#pragma unroll
      for (int cb = 0; cb < C::NCB; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) stage[(cb * 16 + i) * 64 + lane] = acc[cb][i];
      stage[NX * 64 + lane] = m;
      stage[(NX + 1) * 64 + lane] = lacc[0];
    }
    __syncthreads();
    if (kg == 1) return;
    const float m1 = stage[NX * 64 + lane], l1 = stage[(NX + 1) * 64 + lane];
    const float mm = fmaxf(m, m1);
    const float f0 = exp2_hw((m - mm) * scale2), f1 = exp2_hw((m1 - mm) * scale2);
#pragma unroll
    for (int cb = 0; cb < C::NCB; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        acc[cb][i] = fmaf(acc[cb][i], f0, stage[(cb * 16 + i) * 64 + lane] * f1);
    lacc[0] = fmaf(lacc[0], f0, l1 * f1);
    m = mm;
  }
  if (!wave_live) return;
  const bool bad = *badflag != 0;
  const int kbeg = tb * kWideTile, kend = min(te * kWideTile, n_eff);
  const int seen = min(kend, tm + 1);  // end of this row's keys in the range
  const bool empty = seen <= kbeg, single = it.ns == 1;
  const float lt = lacc[0], rl = 0x1p-64f / lt;
  const float lp = empty ? -INFINITY : log2_hw(lt);  // (less m, as the channels' sums)
  const float* cw = sm.c((ntiles - 1) & 1);
  const float* inv = sm.inv();
  const auto low = [&](float x) { return !(x >= kWideLow && x * rl >= 0x1p-120f); };
  const bool mine = wr0 + n < nr;
  uint64_t flags = 0;
  {
    float amin = INFINITY;
#pragma unroll
    for (int cb = 0; cb < C::NCB; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i) amin = fminf(amin, acc[cb][i]);
    if (__ballot(low(amin) && mine && !empty && !bad) != 0) {
#pragma unroll
      for (int cb = 0; cb < C::NCB; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (low(acc[cb][i]) && mine && !empty && !bad) flags |= 1ull << (cb * 16 + i);
    }
  }
  // one split: F; else log2 of the joint sum less m, log2 acc - bias + c
#pragma unroll
  for (int cb = 0; cb < C::NCB; ++cb) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int ch0 = cb * 32 + q * 8 + hl * 4;
      const i32x4 oc = SPLIT ? *reinterpret_cast<const i32x4*>(sm.chan() + ch0)
                             : i32x4{ch0, ch0 + 1, ch0 + 2, ch0 + 3};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = acc[cb][q * 4 + e];
        float o = single ? (log2_hw(x * rl) + cw[ch0 + e]) * inv[ch0 + e]
                         : log2_hw(x * rl) + log2_hw(lt) + cw[ch0 + e];
        if (empty) o = -INFINITY;  // (never with one split)
        stage[n * SROW + oc[e]] = bad ? __builtin_nanf("") : o;
      }
    }
  }
  // flagged outputs: exact, over the range's keys
  uint64_t who = __ballot(flags != 0);
  while (who != 0) {
    const int src = __builtin_ctzll(who);
    who &= who - 1;
    const uint64_t fw =
        (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(flags >> 32), src) << 32 |
        (unsigned)__builtin_amdgcn_readlane((int)(unsigned)flags, src);
    const int rr = __builtin_amdgcn_readlane(row, src), ee = __builtin_amdgcn_readlane(seen, src);
    auto lane_of = [src](float x) {
      return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(x), src));
    };
    const float dl = lane_of(lp), ref = lane_of(m);
    const bf16* qp = r.q + (size_t)(sq.q0 + rr / r.G) * (size_t)r.qld +
                     (size_t)(g * r.G + rr % r.G) * C::DK;
    for (uint64_t f = fw; f != 0; f &= f - 1) {
      const int e = __builtin_ctzll(f), cb = e >> 4, i = e & 15;
      const int col = cb * 32 + (i >> 2) * 8 + (src >> 5) * 4 + (i & 3);
      const int j = SPLIT ? sm.chan()[col] : col;
      const float bl = sm.bl()[col];
      const float y = exact_joint<C::DK, C::DV, KV>(a, qp, it.b, g, j, bl, kbeg, ee, scale2, ref);
      if (lane == 0) stage[(src & 31) * SROW + j] = single ? (y - dl) / bl : y;
    }
  }
  // whole rows: lane l stores channels 4 (l % LPR) .. +3 of row l / LPR of each group
  constexpr int LPR = C::DV / 4, RPI = 64 / LPR;
  const int c4 = (lane % LPR) * 4;
  if (!single) {
    constexpr int PR = part_row(C::DV);
    float* p = r.wide_part + ((size_t)slot_id * r.wide_rps + wr0) * PR;
    if (hl == 0 && mine) {
      p[n * PR + C::DV] = bad ? __builtin_nanf("") : lp;
      p[n * PR + C::DV + 1] = empty ? -INFINITY : m;
    }
#pragma unroll 4
    for (int q = 0; q < 32; q += RPI) {
      const int rr = q + lane / LPR;
      const f32x4 o = *reinterpret_cast<const f32x4*>(stage + rr * SROW + c4);
      if (wr0 + rr < nr) *reinterpret_cast<f32x4*>(p + rr * PR + c4) = o;
    }
    return;
  }
#pragma unroll 4
  for (int q = 0; q < 32; q += RPI) {
    const int rr = q + lane / LPR, x = r0 + wr0 + rr;
    const f32x4 o = *reinterpret_cast<const f32x4*>(stage + rr * SROW + c4);
    if (wr0 + rr >= nr) continue;
    put4(r, ((size_t)(sq.q0 + x / r.G) * r.H + g * r.G + x % r.G) * C::DV + c4, o);
  }
}

// Dispatch on the column blocks that take the lo product.
template <class C, int KV, int N>
__device__ __forceinline__ void wide_nlo(int nlo, const PagedArgs& a, const ReadArgs& r,
                                         const RowItem& it, int g, int slot, unsigned char* smem,
                                         int nneed) {
  if constexpr (N == C::NCB) {
    wide_body<C, KV, N>(a, r, it, g, slot, smem, nneed);
  } else {
    if (nlo == N) wide_body<C, KV, N>(a, r, it, g, slot, smem, nneed);
    else wide_nlo<C, KV, N + 1>(nlo, a, r, it, g, slot, smem, nneed);
  }
}

__host__ __device__ __forceinline__ Work wide_work(const PagedArgs& a, const ReadArgs& r) {
  return Work{r.G, kWideRows, kWideTile, r.wide_least, 1ll << 60, a.max_q, r.causal != 0, true};
}

constexpr int kWideUnits = 256;  // compute units, which hold one workgroup each
constexpr int kMostSplitBlocks = kWideUnits / 2;
constexpr int kSplitCost = 8;    // a split's store and its part of the merge, in tiles
constexpr int kLeastTiles = 4;   // of a split

// Tiles of a split of the wide kernel.  Where the row blocks leave at least half of
// the compute units idle, the smallest with which all splits still have a unit each,
// if that saves more tiles than the splits cost.
__device__ __forceinline__ int wide_tiles(const Planner& plan, const ReadArgs& r) {
  if (!r.split_wide) return kWhole;
  const auto count = [&](int tps) {
    return plan.total(
        [=](const RowCounts& c) { return (long long)c.nrb * ((c.nt + (long long)tps - 1) / tps); });
  };
  const long long items = count(kWhole);
  if (items == 0 || items > kMostSplitBlocks) return kWhole;
  const int longest = plan.longest();
  int lo = kLeastTiles, hi = longest;  // the smallest that fits is in lo .. hi
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (count(mid) <= kWideUnits) hi = mid;
    else lo = mid + 1;
  }
  return lo + kSplitCost < longest ? lo : kWhole;
}

// Workgroup x * heads + g: item x of cached head g, the longest sequences' first.  A
// block's last rows, if at most 128, take the form with two key groups.  In a call
// that may have sequences of few rows too (r.rows_too), their splits follow, read as
// paged_rows_kernel reads them but by eight waves: they fill the units that the last
// wide items leave idle (twelve sequences of 1 to 700 tokens, of which two with one:
// 496 us with a launch of their own, 471 so, then).
template <int DK, int DV, int KV>
__global__ __launch_bounds__(512) void paged_wide_kernel(PagedArgs a, ReadArgs r) {
  using C1 = Cfg<DK, DV, 8, kFem, true, false, 1>;
  using C2 = Cfg<DK, DV, 8, kFem, true, false, 2>;
  static_assert(WideLds<C1, KV>::BYTES == WideLds<C2, KV>::BYTES, "one LDS layout");
  static_assert(row_lds<DK, DV>(8) <= WideLds<C1, KV>::BYTES, "few rows fit");
  __shared__ __align__(16) unsigned char smem[WideLds<C1, KV>::BYTES];
  __shared__ int item[kItemInts];
  const int g = blockIdx.x % a.heads, x = blockIdx.x / a.heads;
  const RowItem it = shared_item(item, [&] {
    const Work w = wide_work(a, r);
    const Planner plan(a, w);
    const int tps = wide_tiles(plan, r);
    const bool first = blockIdx.x == 0;
    if (r.split_wide && first && threadIdx.x == 0) r.tps[1] = tps;
    RowItem i = plan.template find<true>(tps, x);
    i.wide = 1;
    if (r.rows_too && (first || !i.found)) {
      const Work wr = rows_work(a, r);
      const Planner rows(a, wr);
      const int t = rows.tiles_per_split(r.target, kRowLeast);
      if (r.target != 0 && first && threadIdx.x == 0) r.tps[0] = t;
      if (!i.found) {
        i = rows.template find<true>(t, x - i.slot);
        i.wide = 0;
      }
    }
    return i;
  });
  if (!it.found) return;
  if (!it.seq.ok || it.seq.len == 0) {
    all_nan<DV>(r, it, g, it.wide ? kWideRows : kRowsMax, 512);
    return;
  }
  const int br = it.wide ? kWideRows : kRowsMax;
  const long long nr = (long long)it.seq.n * r.G - (long long)it.rb * br;
  const int slot = it.slot * a.heads + g;
  if (!it.wide) {
    if (nr <= 16) rows_body<DK, DV, KV, 1, 8>(a, r, it, g, slot, smem);
    else rows_body<DK, DV, KV, 2, 8>(a, r, it, g, slot, smem);
    return;
  }
  const int nneed = lo_channels<C1>(r.beta + g * DV, threadIdx.x & 63);
  if (nr > kWideRows / 2) wide_nlo<C1, KV, 0>((nneed + 31) >> 5, a, r, it, g, slot, smem, nneed);
  else wide_nlo<C2, KV, 0>((nneed + 31) >> 5, a, r, it, g, slot, smem, nneed);
}

}  // namespace
}  // namespace fem
