// The FEM read of few query rows over a paged cache: one decoding token, a
// group of query heads, a handful of drafted tokens.
//
//   out_j = (1/beta_j) [ log sum_i exp(s_i + beta_j v_ij) - log sum_i exp(s_i) ]
//
// The rows that share a cached head (tokens of a sequence times query heads of
// the group) are read together, up to 32 at a time, so that the cache is read
// once for all of them.
//
// Work.  The keys of a row block are split over workgroups (below) and, inside
// one, dealt to its four waves in tiles of 32 keys.  A wave works alone, with
// no barrier until its last tile: its scores, running row maxima, tilted
// values and running column shifts are its own.
//
//   * S^T = K Q^T on v_mfma_f32_16x16x32_bf16, K's fragments loaded straight
//     from the cache (a lane holds 8 dimensions of one key);
//   * P = 2^(s - m + 40), m a row maximum raised only past a lag of 8;
//   * V goes through the wave's own LDS area and comes back transposed
//     (ds_read_tr16_b64), so that a lane holds eight keys of one channel:
//     E = 2^(beta log2e v - c + 40), c a channel's shift raised likewise,
//     formed once for all rows; bf16, hi + lo where beta < 0.5;
//   * O += P E with P's registers as the scores left them (the contraction's
//     key order is permuted the same way on both sides).
//   * The next tile's K and V are loaded into the registers that this tile's
//     products and LDS writes have just freed, so a whole tilt hides them.
//
// What bounds it: HBM where there are enough keys.  8 x 16 heads of up to 4096 keys
// of d = 128 in bf16: 41.5 us, 4.65 TB/s of the 4.94 that a copy reaches; 16 x 8 heads
// of up to 32768 keys in e4m3, four query heads each: 160 us, 4.5 TB/s (672 vector
// instructions a tile, the vector units busy for 106 us of it).  Short splits are
// bound by a workgroup's start and end, int8 by its conversion too (13 sequences of
// 16 rows, d = 64: 30 us for 13 of bytes).
//
// Range.  P and E carry a bias of 40 and a lag of 8 each: their product is at
// most 2^96, and a term that underflows in either factor is at most 2^-70 of
// the frame (m, c), so a sum of at least 2^-40 has lost nothing that fp32 would
// keep.  A smaller sum (every visible key with a large score has a small value
// and the other way round, by 120 octaves together) is formed again, exactly,
// from the keys of the workgroup's range.
#pragma once

#include "fem_internal.h"
#include "fem_paged.h"

namespace fem {

// Workgroups of a compute unit (of kRowWaves waves, one a SIMD).  A third one helps
// nothing: 16 sequences of up to 8192 keys, one token, 8 heads, d = 64, 38.2 us with
// two and 38.8 with three; e4m3 34.5 and 35.2; d = 128 e4m3, whose registers then
// spill, 166 and 196 us at 16 x 32768 keys.
constexpr int kRowGroups = 2;

constexpr int kRowsMax = 32;       // query rows of a block
constexpr int kRowLeast = 8;       // tiles of a split at least, two a wave
constexpr int kRowTile = 32;       // keys of a wave's tile
constexpr int kRowWaves = 4;       // of a workgroup; calls with short contexts take twice as
                                   // many and do not split (kShortKeys)
constexpr float kRowBias = 40.f;   // of P and of E
constexpr float kLag = 8.f;        // of m and of c
constexpr float kNone = -3e38f;    // m and c before the first key: finite, so that a hidden
                                   // key's exponent is -inf and not NaN
constexpr float kLoBelow = 0.5f;   // channels with beta below this take E as hi + lo

// ---- who does what ------------------------------------------------------------

// The part of a call that one kernel takes: the sequences with lo < rows <= hi
// (rows: new tokens times query heads of a group), in row blocks of `br` rows and
// key tiles of `tk` keys.
struct Work {
  int G, br, tk;
  long long lo, hi;
  int max_q;
  bool causal;
  bool longest_first;  // items in the order of falling lengths (up to 64 sequences)
};

// A workgroup's piece of the work.
struct RowItem {
  int b, rb, s, ns;  // sequence, row block, split and the number of splits
  int slot;          // number of split s among those of one head (not found: of all splits)
  int wide;          // of the wide kernel's own items
  Seq seq;
  bool found;
};

struct RowCounts {
  int nrb, nt;  // row blocks, and key tiles of one
};

constexpr int kWhole = 1 << 30;  // tiles of a split where nothing is split

// The split of the work, formed from the lengths by one wave of every workgroup: a
// lane has a sequence (the first 64 in registers).
struct Planner {
  const PagedArgs& a;
  const Work& w;
  int lane;
  RowCounts first;

  __device__ __forceinline__ Planner(const PagedArgs& a_, const Work& w_)
      : a(a_), w(w_), lane(threadIdx.x & 63) {
    first = fetch(0);
  }
  __device__ __forceinline__ RowCounts fetch(int b0) const {
    RowCounts c = {0, 0};
    if (b0 + lane >= a.nseq) return c;
    const Seq q = seq_of(a, b0 + lane, w.causal);
    // a sequence that cannot be read is one item, whatever its rows (see all_nan)
    const bool ok = q.ok && q.n <= w.max_q;
    const long long rows = ok ? (long long)q.n * w.G : q.n > 0 ? 1 : 0;
    if (rows > w.lo && rows <= w.hi) {
      c.nrb = (int)((rows + w.br - 1) / w.br);
      c.nt = ok ? max((q.len + w.tk - 1) / w.tk, 1) : 1;
    }
    return c;
  }
  __device__ __forceinline__ RowCounts counts(int b0) const { return b0 == 0 ? first : fetch(b0); }
  __device__ __forceinline__ int lanes(int b0) const { return min(64, a.nseq - b0); }

  // Sum of f(counts) over the sequences and heads, the same in every lane.
  template <class F>
  __device__ __forceinline__ long long total(F&& f) const {
    long long t = 0;
    for (int b0 = 0; b0 < a.nseq; b0 += 64) t += f(counts(b0));
    const int m = lanes(0);
    for (int o = 1; o < m; o <<= 1) t += __shfl_xor(t, o);
    return ((long long)(unsigned)__builtin_amdgcn_readfirstlane((int)t) |
            (long long)__builtin_amdgcn_readfirstlane((int)(t >> 32)) << 32) * a.heads;
  }
  __device__ __forceinline__ int longest() const {
    int t = 0;
    for (int b0 = 0; b0 < a.nseq; b0 += 64) t = max(t, counts(b0).nt);
    const int m = lanes(0);
    for (int o = 1; o < m; o <<= 1) t = max(t, __shfl_xor(t, o));
    return __builtin_amdgcn_readfirstlane(t);
  }

  // Tiles of a split such that all splits of all heads number at most `target`: the
  // smallest of 64 candidates (a lane each) between a target-th of the tiles and
  // three times that; kWhole where none will do or nothing is to be split.
  __device__ __forceinline__ int tiles_per_split(int target, int least_tiles) const {
    if (target == 0) return kWhole;
    const long long t = total([](const RowCounts& c) { return (long long)c.nrb * c.nt; });
    const long long least = max((t + target - 1) / target, (long long)least_tiles);
    const int cand = (int)min(least + (least * lane + 31) / 32, (long long)kWhole);
    const float inv = 1.f / (float)cand;
    float n = 0.f;  // splits of a head with this lane's candidate (exact up to 2^24)
    for (int b0 = 0; b0 < a.nseq; b0 += 64) {
      const RowCounts c = counts(b0);
      const float nrb = (float)c.nrb, nt = (float)c.nt;
      const int m = lanes(b0);
      for (int i = 0; i < m; ++i) {
        // ceil(nt / cand), or one more where the product rounds up to a whole number
        n = fmaf(lane_of(nrb, i), floorf(lane_of(nt, i) * inv) + 1.f, n);
      }
    }
    const uint64_t fits = __ballot(n * (float)a.heads <= (float)target);
    return fits == 0 ? kWhole : __builtin_amdgcn_readlane(cand, __builtin_ctzll(fits));
  }
  __device__ __forceinline__ static float lane_of(float x, int i) {
    return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(x), i));
  }

  // Item x of all heads' alike: a split of a row block (SPLITS), or a whole row
  // block.  Items are numbered by sequence, row block and split; longest_first takes
  // the sequences by length and a sequence's last row block first.
  template <bool SPLITS>
  __device__ __forceinline__ RowItem find(int tps, int x) const {
    RowItem it;
    it.found = false;
    it.wide = 0;
    int base = 0, slot = 0;
    for (int b0 = 0; b0 < a.nseq; b0 += 64) {
      RowCounts c = counts(b0);
      const int m64 = lanes(b0);
      int who = b0 + lane;  // this lane's sequence
      if (w.longest_first && a.nseq <= 64) {
        int rank = lane;
        if (lane < m64) {
          rank = 0;
          for (int i = 0; i < m64; ++i) {
            const int t = __builtin_amdgcn_readlane(c.nt, i);
            rank += t > c.nt || (t == c.nt && i < lane);
          }
        }
        who = __builtin_amdgcn_ds_permute(rank * 4, who);
        c.nt = __builtin_amdgcn_ds_permute(rank * 4, c.nt);
        c.nrb = __builtin_amdgcn_ds_permute(rank * 4, c.nrb);
      }
      const int nrb = c.nrb, ns = tps >= c.nt ? 1 : (c.nt + tps - 1) / tps;
      const int mine = SPLITS ? nrb * ns : nrb, slots = nrb * ns;
      int end = mine, send = slots;
      for (int o = 1; o < m64; o <<= 1) {
        const int u = __shfl_up(end, o), v = SPLITS ? u : __shfl_up(send, o);
        if (lane >= o) {
          end += u;
          send += v;
        }
      }
      const uint64_t m = __ballot(lane < m64 && base + end > x);
      if (m != 0) {
        const int l = __builtin_ctzll(m);
        it.found = true;
        it.b = __builtin_amdgcn_readlane(who, l);
        const int at = x - base - __builtin_amdgcn_readlane(end - mine, l);
        it.ns = __builtin_amdgcn_readlane(ns, l);
        const int block = SPLITS ? at / it.ns : at;
        it.s = SPLITS ? at % it.ns : 0;
        it.slot = slot + __builtin_amdgcn_readlane(send - slots, l) + block * it.ns + it.s;
        it.rb = w.longest_first ? __builtin_amdgcn_readlane(nrb, l) - 1 - block : block;
        break;
      }
      base += __builtin_amdgcn_readlane(end, m64 - 1);
      slot += __builtin_amdgcn_readlane(send, m64 - 1);
    }
    if (it.found) {
      it.seq = seq_of(a, it.b, w.causal);
      it.seq.ok = it.seq.ok && it.seq.n <= w.max_q;
    } else {
      it.slot = slot;
    }
    return it;
  }
};

// An item that wave 0 has found, for the whole workgroup (barriers on both sides).
constexpr int kItemInts = 12;
template <class F>
__device__ __forceinline__ RowItem shared_item(int* lds, F&& find) {
  __syncthreads();  // the last item's LDS is free
  if (threadIdx.x < 64) {
    const RowItem it = find();
    if (threadIdx.x == 0) {
      lds[0] = it.found;
      if (it.found) {
        lds[1] = it.b;
        lds[2] = it.rb;
        lds[3] = it.s;
        lds[4] = it.ns;
        lds[5] = it.slot;
        lds[6] = it.seq.q0;
        lds[7] = it.seq.n;
        lds[8] = it.seq.len;
        lds[9] = it.seq.ok;
        lds[10] = it.wide;
      }
    }
  }
  __syncthreads();
  auto get = [lds](int i) { return __builtin_amdgcn_readfirstlane(lds[i]); };
  RowItem it;
  it.found = get(0) != 0;
  it.b = get(1);
  it.rb = get(2);
  it.s = get(3);
  it.ns = get(4);
  it.slot = get(5);
  it.seq.q0 = get(6);
  it.seq.n = get(7);
  it.seq.len = get(8);
  it.seq.ok = get(9) != 0;
  it.wide = get(10);
  return it;
}

// Keys that row r of a sequence's group sees.
__device__ __forceinline__ int row_limit(const Seq& s, int r, int G, bool causal) {
  return causal ? s.len - s.n + r / G + 1 : s.len;
}

// ---- exact form ---------------------------------------------------------------

// log2 sum over keys [k0, k1) of 2^((s_i - ref) scale2 + bl v_ij), formed by a whole
// wave in fp32; returns -inf for no keys.
template <int DK, int DV, int KV>
__device__ float exact_joint(const PagedArgs& a, const bf16* qrow, int b, int g, int j, float bl,
                             int k0, int k1, float scale2, float ref) {
  Lse2 t;
  for (int i = k0 + (threadIdx.x & 63); i < k1; i += 64) {
    bool bad = false;
    const size_t row = paged_row(a, b, g, i, bad);
    float dot = 0.f;
#pragma unroll 1  // registers: this is rare
    for (int c = 0; c < DK / 8; ++c) {
      const bf16x8 x = reinterpret_cast<const bf16x8*>(qrow)[c];
      float f[8];
      row8<KV, DK>(a.k, a.ks, row, c, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot = fmaf((float)x[e], f[e], dot);
    }
    float f[8], v = 0.f;
    row8<KV, DV>(a.v, a.vs, row, j >> 3, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) v = (j & 7) == e ? f[e] : v;
    t.add(fmaf(v, bl, (dot - ref) * scale2));
  }
  return t.wave_total();
}

__device__ __forceinline__ float max8(const float (&x)[8]) {  // three v_max3 and one v_max
  return fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), fmaxf(fmaxf(x[3], x[4]), x[5])), x[6]),
               x[7]);
}

// max(x over the lanes with the same l16), by lane swaps.
__device__ __forceinline__ float max_groups(float x) {
  unsigned u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  u = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// ---- the read -------------------------------------------------------------------

template <int DK, int DV>
struct RowCfg {
  static constexpr int NKS = DK / 32;          // k-steps of K Q^T
  static constexpr int NCB = DV / 16;          // 16-channel blocks
  static constexpr int VROW = DV * 2 + 32;     // LDS row of a V tile (bytes): conflict-free
  static constexpr int VT = kRowTile * VROW;   // a wave's V area
  static constexpr int OROW = DV + 4;          // LDS row of a merge area (floats)
  static constexpr int MT = 16 * OROW * 4;     // a wave's merge area
  static constexpr int AREA = VT > MT ? VT : MT;
};

// One wave's part of a read; NW waves share the keys.
template <int DK, int DV, int KV, int RB, int NW>
struct RowRead {
  using C = RowCfg<DK, DV>;
  static constexpr bool MX = KV != FEM_KV_BF16;
  static constexpr int KN = C::NKS;                       // K pieces of a block
  static constexpr int VN = MX ? (DV + 63) / 64 : DV / 32;  // V pieces of a block

  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

  const PagedArgs& a;
  int b, g, n_eff;  // sequence, cached head, keys the block may see at all
  int lane, l16, grp;
  unsigned char* vt;  // this wave's LDS area
  bool bad = false;

  bf16x8 qf[RB][C::NKS];
  f32x4 acc[RB][C::NCB];
  float m[RB];     // of the scores before scale2
  f32x4 lsum[RB];  // sums of rows 4 grp + i, the same in every lane of the group
  float bl[C::NCB], c[C::NCB];
  unsigned lo_blocks;  // bit cb: a channel of the block takes hi + lo

  u32x4 kw[2][KN];        // bf16: 8 values; 8-bit: words 0, 1 hold 8 codes
  unsigned ksc[2];        // scale bytes of the lane's key
  u32x4 vw[2][VN];
  unsigned vsc[2][VN];

  __device__ __forceinline__ RowRead(const PagedArgs& a_) : a(a_) {}

  // Pages of this wave's next 32 tiles (lane 2 n + kb: 16-key block kb of its n-th
  // tile from tile t on), so that the loop waits for no page number.  Blocks past the
  // last visible key stand for the last one.
  int pages;
  __device__ __forceinline__ int block_key(int t, int kb) const {
    return min(t * kRowTile + kb * 16, (n_eff - 1) & ~15);
  }
  __device__ __forceinline__ void load_pages(int t) {
    const int k = block_key(min(t + (lane >> 1) * NW, 1 << 25), lane & 1);
    pages = a.table[(size_t)b * a.table_len + (k >> a.page_log2)];
  }
  // First row of block kb of tile t, the n-th of those.
  __device__ __forceinline__ size_t block_row(int t, int kb, int n) {
    int p = __builtin_amdgcn_readlane(pages, 2 * n + kb);
    if ((unsigned)p >= (unsigned)a.pages) {
      bad = true;
      p = 0;
    }
    return (((size_t)p * a.heads + g) << a.page_log2) + (block_key(t, kb) & (a.page - 1));
  }
  __device__ __forceinline__ void load(int t, int n) {
    const size_t row[2] = {block_row(t, 0, n), block_row(t, 1, n)};
    load_k(row);
    load_v(row);
  }

  // Lane offsets in a block: the loads take them with a scalar base each.
  unsigned koff, ksoff, voff, vsoff;
  __device__ __forceinline__ void lane_offsets() {
    koff = MX ? l16 * DK + grp * 8 : l16 * (DK * 2) + grp * 16;
    ksoff = l16 * KN;
    const unsigned piece = MX && DV == 32 ? lane & 31 : lane;  // 16 bytes of V's rows in order
    voff = piece * 16;
    vsoff = piece >> 1;
  }
  __device__ __forceinline__ void load_k(const size_t (&row)[2]) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const uint8_t* p = a.k + row[kb] * (MX ? DK : DK * 2);
#pragma unroll
      for (int ks = 0; ks < KN; ++ks) {
        if constexpr (!MX) {
          kw[kb][ks] = *reinterpret_cast<const u32x4*>(p + koff + ks * 64);
        } else {
          const u32x2v w = *reinterpret_cast<const u32x2v*>(p + koff + ks * 32);
          kw[kb][ks][0] = w[0];
          kw[kb][ks][1] = w[1];
        }
      }
      if constexpr (MX) {
        const uint8_t* sp = a.ks + row[kb] * KN + ksoff;
        if constexpr (KN == 4) ksc[kb] = *reinterpret_cast<const unsigned*>(sp);
        else if constexpr (KN == 2) ksc[kb] = *reinterpret_cast<const unsigned short*>(sp);
        else ksc[kb] = *sp;
      }
    }
  }
  __device__ __forceinline__ void load_v(const size_t (&row)[2]) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const uint8_t* p = a.v + row[kb] * (MX ? DV : DV * 2);
#pragma unroll
      for (int i = 0; i < VN; ++i) {
        vw[kb][i] = *reinterpret_cast<const u32x4*>(p + voff + i * 1024);
        if constexpr (MX) vsc[kb][i] = a.vs[row[kb] * (DV / kScaleBlock) + i * 32 + vsoff];
      }
    }
  }
  __device__ __forceinline__ bf16x8 k_frag(int kb, int ks) const {
    if constexpr (!MX) return __builtin_bit_cast(bf16x8, kw[kb][ks]);
    return __builtin_bit_cast(bf16x8, dequant8<KV>(kw[kb][ks][0], kw[kb][ks][1],
                                                   scale_of(ksc[kb] >> (8 * ks) & 0xffu)));
  }
  // The tile's V into LDS as [32][DV] bf16; rows at or past `live` become -inf
  // (E = 0 there, and the column maximum does not see them).
  __device__ __forceinline__ void store_v(int live) {
    constexpr unsigned kNegInf2 = 0xff80ff80u;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int i = 0; i < VN; ++i) {
        if constexpr (!MX) {
          constexpr int PPR = DV / 8;  // pieces of a row
          const int piece = i * 64 + lane, row = kb * 16 + piece / PPR, col = piece % PPR;
          u32x4 w = vw[kb][i];
          if (live < kRowTile && row >= live) w = u32x4{kNegInf2, kNegInf2, kNegInf2, kNegInf2};
          *reinterpret_cast<u32x4*>(vt + row * C::VROW + col * 16) = w;
        } else {
          constexpr int PPR = DV / 16;
          const int piece = DV == 32 ? lane & 31 : i * 64 + lane;  // as loaded
          const int row = kb * 16 + piece / PPR, col = piece % PPR;
          const float s = scale_of(vsc[kb][i]);
          u32x4 w0 = dequant8<KV>(vw[kb][i][0], vw[kb][i][1], s);
          u32x4 w1 = dequant8<KV>(vw[kb][i][2], vw[kb][i][3], s);
          if (live < kRowTile && row >= live) {
            w0 = u32x4{kNegInf2, kNegInf2, kNegInf2, kNegInf2};
            w1 = w0;
          }
          u32x4* d = reinterpret_cast<u32x4*>(vt + row * C::VROW + col * 32);
          d[0] = w0;
          d[1] = w1;
        }
      }
    }
  }

  // One tile of keys k0 .. k0+31.  `masked`: some row does not see all of it;
  // lim[rb]: keys that the lane's row sees.  The next tile's rows are loaded
  // where `more` is set.
  __device__ __forceinline__ void tile(int k0, bool masked, const int (&lim)[RB], bool more,
                                       int tnext, int nnext, float scale2) {
    // ---- S^T = K Q^T
    f32x4 s[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb][0] = s[rb][1] = f32x4{};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int ks = 0; ks < KN; ++ks) {
        const bf16x8 kf = k_frag(kb, ks);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          s[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rb][ks], s[rb][kb], 0, 0, 0);
      }
    }
    store_v(n_eff - k0);
    if (more) load(tnext, nnext);

    // ---- P, in the A operand's layout: row l16, keys 4 grp + i, 16 + 4 grp + i
    bf16x8 p[RB], ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float x[8];
      // m is subtracted from the scores as they are: a product rounded otherwise than
      // m's own would leave the largest score off by half its last place
      auto exponents = [&] {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(s[rb][e >> 2][e & 3] - m[rb], scale2, kRowBias);
        return max8(x);
      };
      if (masked) {
        const int left = lim[rb] - k0 - 4 * grp;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if ((e & 3) + 16 * (e >> 2) >= left) s[rb][e >> 2][e & 3] = -INFINITY;
      }
      if (__any(exponents() > kRowBias + kLag)) {
        float mx = fmaxf(fmaxf(fmaxf(s[rb][0][0], s[rb][0][1]), fmaxf(s[rb][0][2], s[rb][0][3])),
                         fmaxf(fmaxf(s[rb][1][0], s[rb][1][1]), fmaxf(s[rb][1][2], s[rb][1][3])));
        mx = max_groups(mx);
        const float mn = (mx - m[rb]) * scale2 > kLag ? mx : m[rb];
        const float f = mn == m[rb] ? 1.f : exp2_hw((m[rb] - mn) * scale2);
        m[rb] = mn;
        f32x4 fr;
#pragma unroll
        for (int i = 0; i < 4; ++i) fr[i] = __shfl(f, 4 * grp + i);
        lsum[rb] *= fr;
#pragma unroll
        for (int cb = 0; cb < C::NCB; ++cb) acc[rb][cb] *= fr;
        exponents();
      }
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        // rounded to bf16 (at most 2^-8 relative); lsum adds the same rounded
        // values, so the rounding cancels from the mean over the keys
        const bf16x2 p2 = to_bf16x2(exp2_hw(x[e]), exp2_hw(x[e + 1]));
        p[rb][e] = p2[0];
        p[rb][e + 1] = p2[1];
      }
      lsum[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[rb], ones, lsum[rb], 0, 0, 0);
    }

    // ---- E and O += P E, 16 channels at a time
    const int tr = (4 * grp + (l16 >> 2)) * C::VROW + (l16 & 3) * 8;
    auto read_v = [&](int cb, int kb) {
      return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4*)(vt + tr + kb * 16 * C::VROW + cb * 32));
    };
    s16x4 n0 = read_v(0, 0), n1 = read_v(0, 1);  // one block ahead
#pragma unroll
    for (int cb = 0; cb < C::NCB; ++cb) {
      const s16x4 v0 = n0, v1 = n1;
      if (cb + 1 < C::NCB) {
        n0 = read_v(cb + 1, 0);
        n1 = read_v(cb + 1, 1);
      }
      float v[8], x[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = __uint_as_float((unsigned)(unsigned short)v0[e] << 16);
        v[4 + e] = __uint_as_float((unsigned)(unsigned short)v1[e] << 16);
      }
      auto exponents = [&] {
        const float sh = kRowBias - c[cb];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(v[e], bl[cb], sh);
        return max8(x);
      };
      if (__any(exponents() > kRowBias + kLag)) {
        const float mx = max_groups(max8(v)) * bl[cb];
        const float cn = mx > c[cb] + kLag ? mx : c[cb];
        const float f = cn == c[cb] ? 1.f : exp2_hw(c[cb] - cn);
        c[cb] = cn;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) acc[rb][cb] *= f;
        exponents();
      }
      float e8[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) e8[e] = exp2_hw(x[e]);
      if ((lo_blocks >> cb) & 1) {
        // beta < 0.5 turns a rounding of E to bf16 into more than 2^-8 of the
        // read: E = hi (truncated) + lo (the rest, rounded), 2^-16 relative
        bf16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const unsigned u0 = __float_as_uint(e8[e]), u1 = __float_as_uint(e8[e + 1]);
          const bf16x2 h = __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(u1, u0, 0x07060302u));
          const bf16x2 l = to_bf16x2(e8[e] - __uint_as_float(u0 & 0xffff0000u),
                                     e8[e + 1] - __uint_as_float(u1 & 0xffff0000u));
          hi[e] = h[0];
          hi[e + 1] = h[1];
          lo[e] = l[0];
          lo[e + 1] = l[1];
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          acc[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[rb], hi, acc[rb][cb], 0, 0, 0);
          acc[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[rb], lo, acc[rb][cb], 0, 0, 0);
        }
      } else {
        bf16x8 hi;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const bf16x2 h = to_bf16x2(e8[e], e8[e + 1]);
          hi[e] = h[0];
          hi[e + 1] = h[1];
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          acc[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[rb], hi, acc[rb][cb], 0, 0, 0);
      }
    }
  }
};

// Arguments of a read besides the cache and the sequences.
struct ReadArgs {
  const bf16* q;       // token t, head h at t * qld + h * DK
  long long qld;
  const float* beta;   // [heads][DV]
  void* out;           // [ntok][H][DV] float32 or bf16
  int* tps;            // [2] tiles of a split, as the two kernels have chosen them
  float* part;         // [slot][rps][part_row]
  float* wide_part;    // of the wide kernel
  int H, G;            // query heads, of a cached head
  int rps, wide_rps;   // rows of a slot
  int target;          // see tiles_per_split
  int split_wide;      // whether the wide kernel may split
  int rows_too;        // whether it takes the sequences of few rows too
  long long most_rows, wide_least;  // the kernels' sequences: rows <= most, rows > least
  int causal, obf16;
};

__host__ __device__ __forceinline__ Work rows_work(const PagedArgs& a, const ReadArgs& r) {
  return Work{r.G, kRowsMax, kRowTile, 0, r.most_rows, a.max_q, r.causal != 0, false};
}

// A row of partial results: log2 of its channels' joint sums and of its own sum, both
// less the row's maximum in the range (which may be far larger than what they differ
// by), that maximum in the scores' own scale, and room to keep the next row aligned for
// loads of four.
__host__ __device__ constexpr int part_row(int dv) { return dv + 4; }

__device__ __forceinline__ void put4(const ReadArgs& r, size_t at, f32x4 x) {
  if (r.obf16) {
    const bf16x2 a = to_bf16x2(x[0], x[1]), b = to_bf16x2(x[2], x[3]);
    *reinterpret_cast<u32x2v*>(static_cast<bf16*>(r.out) + at) =
        u32x2v{__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b)};
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(r.out) + at) = x;
  }
}

__device__ __forceinline__ void put(const ReadArgs& r, size_t at, float x) {
  if (r.obf16) static_cast<bf16*>(r.out)[at] = (bf16)x;
  else static_cast<float*>(r.out)[at] = x;
}

// LDS of a workgroup of nw waves: their areas, and the tables in which they meet.
template <int DK, int DV>
constexpr int row_lds(int nw) {
  return nw * (RowCfg<DK, DV>::AREA + (2 * kRowsMax + DV) * 4 + 4) + (2 * kRowsMax + DV) * 4;
}

// The read of one split of one row block (at most 16 RB rows) of cached head g.
template <int DK, int DV, int KV, int RB, int NW>
__device__ __forceinline__ void rows_body(const PagedArgs& a, const ReadArgs& r, const RowItem& it,
                                          int g, int slot, unsigned char* smem) {
  using C = RowCfg<DK, DV>;
  RowRead<DK, DV, KV, RB, NW> w(a);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  w.lane = tid & 63;
  w.l16 = tid & 15;
  w.grp = (tid & 63) >> 4;
  w.vt = smem + wave * C::AREA;
  w.lane_offsets();
  w.b = it.b;
  w.g = g;
  const Seq& sq = it.seq;
  const bool causal = r.causal != 0;
  const int r0 = it.rb * kRowsMax, nr = min((int)min((long long)sq.n * r.G - r0, 32ll), 16 * RB);
  w.n_eff = row_limit(sq, r0 + nr - 1, r.G, causal);
  const int tiles = (w.n_eff + kRowTile - 1) / kRowTile;
  const int tb = (int)((long long)it.s * tiles / it.ns);
  const int te = (int)((long long)(it.s + 1) * tiles / it.ns);
  const float scale2 = kLog2e / sqrtf((float)DK);

  int t = tb + wave;
  if (t < te) w.load_pages(t);
  int lim[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = r0 + min(rb * 16 + w.l16, nr - 1);  // rows past the last repeat it
    const int tok = row / r.G, h = g * r.G + row % r.G;
    const bf16* qp = r.q + (size_t)(sq.q0 + tok) * (size_t)r.qld + (size_t)h * DK + w.grp * 8;
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks) w.qf[rb][ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 32);
    lim[rb] = row_limit(sq, row, r.G, causal);
    w.m[rb] = kNone;
    w.lsum[rb] = f32x4{};
#pragma unroll
    for (int cb = 0; cb < C::NCB; ++cb) w.acc[rb][cb] = f32x4{};
  }
  const int least = row_limit(sq, r0, r.G, causal);  // keys that every row sees
  w.lo_blocks = 0;
#pragma unroll
  for (int cb = 0; cb < C::NCB; ++cb) {
    const float b = r.beta[g * DV + cb * 16 + w.l16];
    w.bl[cb] = b * kLog2e;
    w.c[cb] = kNone;
    if (__any(!(b >= kLoBelow))) w.lo_blocks |= 1u << cb;
  }
  if (t < te) w.load(t, 0);
  for (int n = 1; t < te; t += NW, n = (n + 1) & 31) {
    const int k0 = t * kRowTile, next = t + NW;
    if (n == 0 && next < te) w.load_pages(next);
    w.tile(k0, k0 + kRowTile > least, lim, next < te, next, n, scale2);
  }

  // ---- the waves meet: common frames M (row) and Cc (channel)
  float* const fm = reinterpret_cast<float*>(smem + NW * C::AREA);  // [NW][32] row maxima
  float* const fl = fm + NW * kRowsMax;                            // [NW][32] row sums
  float* const fc = fl + NW * kRowsMax;                            // [NW][DV] shifts
  float* const rm = fc + NW * DV;                                  // [32] a row's M
  float* const rl = rm + kRowsMax;                                 // [32] and its sum there
  float* const ct = rl + kRowsMax;                                 // [DV] a channel's Cc
  int* const fbad = reinterpret_cast<int*>(ct + DV);               // [NW]
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (w.grp == 0) fm[wave * kRowsMax + rb * 16 + w.l16] = w.m[rb];
    if (w.l16 == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) fl[wave * kRowsMax + rb * 16 + 4 * w.grp + i] = w.lsum[rb][i];
    }
  }
  if (w.grp == 0) {
#pragma unroll
    for (int cb = 0; cb < C::NCB; ++cb) fc[wave * DV + cb * 16 + w.l16] = w.c[cb];
  }
  if (w.lane == 0) fbad[wave] = w.bad;
  __syncthreads();
  int any_bad = 0;
#pragma unroll
  for (int x = 0; x < NW; ++x) any_bad |= fbad[x];
  const bool bad = any_bad != 0;
  auto top_of = [](const float* p, int stride) {  // over the waves
    float t = p[0];
#pragma unroll
    for (int x = 1; x < NW; ++x) t = fmaxf(t, p[x * stride]);
    return t;
  };
  // (for all to read after the next barrier)
  if (tid < 16 * RB) {
    const float M = top_of(fm + tid, kRowsMax);
    float l = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) l += fl[x * kRowsMax + tid] * exp2_hw((fm[x * kRowsMax + tid] - M) * scale2);
    rm[tid] = M;
    rl[tid] = l;
  }
  if (tid >= 64 * NW - DV) ct[tid - (64 * NW - DV)] = top_of(fc + tid - (64 * NW - DV), DV);
  float cf[C::NCB];
#pragma unroll
  for (int cb = 0; cb < C::NCB; ++cb) {
    const float top = top_of(fc + cb * 16 + w.l16, DV);
    cf[cb] = exp2_hw(w.c[cb] - top);
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (rb > 0) __syncthreads();
    f32x4 rf;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = rb * 16 + 4 * w.grp + i;
      rf[i] = exp2_hw((fm[wave * kRowsMax + q] - top_of(fm + q, kRowsMax)) * scale2);
    }
    float* area = reinterpret_cast<float*>(smem + wave * C::AREA);
#pragma unroll
    for (int cb = 0; cb < C::NCB; ++cb) {
      const f32x4 x = w.acc[rb][cb] * rf * cf[cb];
#pragma unroll
      for (int i = 0; i < 4; ++i) area[(4 * w.grp + i) * C::OROW + cb * 16 + w.l16] = x[i];
    }
    __syncthreads();
    const int kbeg = tb * kRowTile, kend = min(te * kRowTile, w.n_eff);
    for (int e = tid; e < 16 * DV; e += 64 * NW) {
      const int q = e / DV, j = e % DV, row = r0 + rb * 16 + q;
      if (rb * 16 + (e & ~63) / DV >= nr) break;  // the wave's rows are past the last
      const bool live = rb * 16 + q < nr;
      const float M = rm[rb * 16 + q], l = rl[rb * 16 + q], top = ct[j];
      float sum = 0.f;
#pragma unroll
      for (int x = 0; x < NW; ++x)
        sum += reinterpret_cast<const float*>(smem + x * C::AREA)[q * C::OROW + j];
      const float blj = r.beta[g * DV + j] * kLog2e;
      const int seen = min(kend, row_limit(sq, row, r.G, causal));  // of this range, up to here
      const bool none = !live || seen <= kbeg;
      // logarithms of the joint sum and of the row's sum, both less M
      float y = none ? -INFINITY : log2_hw(sum) + (top - 2.f * kRowBias);
      const float lp = none ? -INFINITY : log2_hw(l) - kRowBias;
      bool redo = !none && !bad && !(sum >= 0x1p-40f);
      uint64_t who = __ballot(redo);
      while (who != 0) {
        const int src = __builtin_ctzll(who);
        who &= who - 1;
        const int rr = __builtin_amdgcn_readlane(row, src), jj = __builtin_amdgcn_readlane(j, src);
        const int ee = __builtin_amdgcn_readlane(seen, src);
        const bf16* qp = r.q + (size_t)(sq.q0 + rr / r.G) * (size_t)r.qld +
                         (size_t)(g * r.G + rr % r.G) * DK;
        const float ref = __uint_as_float(
            (unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(M), src));
        const float x = exact_joint<DK, DV, KV>(a, qp, it.b, g, jj, r.beta[g * DV + jj] * kLog2e,
                                                kbeg, ee, scale2, ref);
        if (w.lane == src) y = x;
      }
      if (!live) continue;
      if (it.ns == 1) {
        // one logarithm of a ratio near 1 where the sums allow it
        const float x = sum / l * 0x1p-40f;
        float o = !redo && x >= 0x1p-120f ? (log2_hw(x) + top) / blj : (y - lp) / blj;
        if (bad) o = NAN;
        put(r, ((size_t)(sq.q0 + row / r.G) * r.H + g * r.G + row % r.G) * DV + j, o);
      } else {
        float* p = r.part + ((size_t)slot * r.rps + rb * 16 + q) * part_row(DV);
        p[j] = bad ? NAN : y;
        if (j == 0) {
          p[DV] = bad ? NAN : lp;
          p[DV + 1] = none ? -INFINITY : M;
        }
      }
    }
  }
}

// The rows of an item that has nothing to read: all of its sequence's where the
// sequence contradicts itself, the block's where it has no keys.
template <int DV>
__device__ __forceinline__ void all_nan(const ReadArgs& r, const RowItem& it, int g, int br,
                                        int threads) {
  const long long rows = (long long)it.seq.n * r.G;
  const long long r0 = it.seq.ok ? (long long)it.rb * br : 0;
  const long long r1 = it.seq.ok ? min(rows, r0 + br) : rows;
  for (long long e = r0 * DV + threadIdx.x; e < r1 * DV; e += threads) {
    const int row = (int)(e / DV);
    put(r, ((size_t)(it.seq.q0 + row / r.G) * r.H + g * r.G + row % r.G) * DV + e % DV, NAN);
  }
}

// Workgroup i takes the pieces i, i + gridDim, ...: piece x * heads + g is item x
// of cached head g.  RB = 1: no sequence has more than 16 rows.
template <int DK, int DV, int KV, int RB, int NW>
__global__ __launch_bounds__(64 * NW, 2)
void paged_rows_kernel(PagedArgs a, ReadArgs r) {
  __shared__ __align__(16) unsigned char smem[row_lds<DK, DV>(NW)];
  __shared__ int item[kItemInts];
  const Work wk = rows_work(a, r);
  int tps = 0;  // (wave 0's)
  for (int piece = blockIdx.x;; piece += gridDim.x) {
    const int g = piece % a.heads;
    const RowItem it = shared_item(item, [&] {
      const Planner plan(a, wk);
      if (tps == 0) {
        tps = plan.tiles_per_split(r.target, kRowLeast);
        if (r.target != 0 && blockIdx.x == 0 && threadIdx.x == 0) r.tps[0] = tps;
      }
      return plan.template find<true>(tps, piece / a.heads);
    });
    if (!it.found) return;
    if (!it.seq.ok || it.seq.len == 0) {
      all_nan<DV>(r, it, g, kRowsMax, 64 * NW);
      continue;
    }
    const long long left = (long long)it.seq.n * r.G - (long long)it.rb * kRowsMax;
    if (RB == 1 || left <= 16) rows_body<DK, DV, KV, 1, NW>(a, r, it, g, piece, smem);
    else rows_body<DK, DV, KV, 2, NW>(a, r, it, g, piece, smem);
  }
}

// ---- merge of the splits -------------------------------------------------------

// (max, sum) of 2^x over a set, joined with another; a NaN, which the maxima pass
// over, stays in the sum.
__device__ __forceinline__ void lse_join(float& m, float& s, float m2, float s2) {
  const float mn = fmaxf(m, m2);
  if (mn == -INFINITY) {  // nothing on either side, or NaN
    s += s2;
    return;
  }
  s = s * exp2_hw(m - mn) + s2 * exp2_hw(m2 - mn);
  m = mn;
}

// One of the two kernels' partial results, in chunks of `rows` rows of a row block.
struct MergePart {
  Work w;
  const int* tps;
  const float* part;
  int rps, rows, groups;  // rows of a slot, of a chunk; workgroups
  float scale2;           // of the scores
};

constexpr int kMergeThreads = 256;
constexpr int kMergeBatch = 8;

// Bound by latency: about 5.5 us for 13 x 8 heads of 16 rows in five splits.
// Workgroup (chunk of a row block, cached head); the first p.groups of them for p,
// the others for o.  A thread has four channels of a row; a row's splits are shared
// by so many threads (a power of two) that each takes one batch of them, if there
// are enough, and these meet in LDS.
template <int DV>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedArgs a, ReadArgs r,
                                                                    MergePart p, MergePart o) {
  constexpr int TPR = DV / 4, NG = kMergeThreads / TPR;  // threads of a row, groups of them
  __shared__ f32x4 meet_m[NG][TPR], meet_s[NG][TPR];
  __shared__ float meet_d[NG][3];
  __shared__ int item[kItemInts];
  const bool second = (int)blockIdx.x >= p.groups;
  const MergePart& x = second ? o : p;
  const int tps = *x.tps;
  if (tps >= kWhole) return;
  const int id = second ? blockIdx.x - p.groups : blockIdx.x;
  const int chunks = (min(x.w.br, x.rps) + x.rows - 1) / x.rows;  // of a row block
  const int g = id % a.heads, xc = id / a.heads;
  const RowItem it = shared_item(item, [&] {
    return Planner(a, x.w).template find<false>(tps, xc / chunks);
  });
  if (!it.found || it.ns == 1) return;
  const int c0 = xc % chunks * x.rows;  // first row of the block that is merged here
  const int r0 = it.rb * x.w.br + c0;
  const int nr = (int)min((long long)it.seq.n * r.G - r0, (long long)x.rows);
  if (nr <= 0) return;
  int per = 1;  // groups of a row
  while (per < NG && per * kMergeBatch < it.ns) per <<= 1;
  const int rows = NG / per, grp = threadIdx.x / TPR, c = threadIdx.x % TPR, sub = grp % per;
  f32x4 bl;
#pragma unroll
  for (int e = 0; e < 4; ++e) bl[e] = r.beta[g * DV + c * 4 + e] * kLog2e;
  constexpr int PR = part_row(DV);
  const size_t step = (size_t)a.heads * x.rps * PR;  // from split to split
  const float* base = x.part + ((size_t)((size_t)it.slot * a.heads + g) * x.rps + c0) * PR;
  const f32x4 kNone4 = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  for (int q0 = 0; q0 < nr; q0 += rows) {
    const int q = q0 + grp / per;
    // sums as (max, sum) of 2^x, x less the largest row maximum so far, ref
    f32x4 M = kNone4, S = {0.f, 0.f, 0.f, 0.f};
    float md = -INFINITY, sd = 0.f, ref = kNone;
    if (q < nr) {
      const float* pq = base + (size_t)q * PR;
      for (int s0 = sub; s0 < it.ns; s0 += kMergeBatch * per) {
        f32x4 y[kMergeBatch];
        float d[kMergeBatch], m[kMergeBatch];
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) {
          const int s = s0 + u * per;
          const float* ps = pq + step * min(s, it.ns - 1);
          y[u] = *reinterpret_cast<const f32x4*>(ps + c * 4);
          d[u] = ps[DV];
          m[u] = ps[DV + 1];
          if (s >= it.ns) {
            y[u] = kNone4;
            d[u] = -INFINITY;
            m[u] = -INFINITY;
          }
        }
        float now = ref;
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) now = fmaxf(now, m[u]);
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) m[u] = (m[u] - now) * x.scale2;
        const float old = (ref - now) * x.scale2;
        ref = now;
        // the batch's maximum first: its exponentials then wait for nothing else
        auto fold = [&](float& mm, float& z, auto&& at) {
          float top = at(0), sum = 0.f;
#pragma unroll
          for (int u = 1; u < kMergeBatch; ++u) top = fmaxf(top, at(u));
          const float zero = fmaxf(top, -3e38f);  // none of the batch: zeros, or NaN
#pragma unroll
          for (int u = 0; u < kMergeBatch; ++u) sum += exp2_hw(at(u) - zero);
          mm += old;
          lse_join(mm, z, top, sum);
        };
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float mm = M[e], z = S[e];
          fold(mm, z, [&](int u) { return y[u][e] + m[u]; });
          M[e] = mm;
          S[e] = z;
        }
        fold(md, sd, [&](int u) { return d[u] + m[u]; });
      }
    }
    const int row = r0 + q;
    const size_t at = ((size_t)(it.seq.q0 + row / r.G) * r.H + g * r.G + row % r.G) * DV + c * 4;
    if (per == 1) {  // the same for the whole workgroup
      f32x4 f;
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = ((M[e] - md) + (log2_hw(S[e]) - log2_hw(sd))) / bl[e];
      if (q < nr) put4(r, at, f);
      continue;
    }
    if (q0 > 0) __syncthreads();
    meet_m[grp][c] = M;
    meet_s[grp][c] = S;
    if (c == 0) {
      meet_d[grp][0] = md;
      meet_d[grp][1] = sd;
      meet_d[grp][2] = ref;
    }
    __syncthreads();
    if (q >= nr) continue;
    // the row's groups share its channels
    const int g0 = grp - sub;
    float top = meet_d[g0][2];
    for (int u = 1; u < per; ++u) top = fmaxf(top, meet_d[g0 + u][2]);
    auto join = [&](auto&& max_of, auto&& sum_of, float& m, float& z) {
      auto at_top = [&](int u) { return max_of(u) + (meet_d[g0 + u][2] - top) * x.scale2; };
      m = at_top(0);
      for (int u = 1; u < per; ++u) m = fmaxf(m, at_top(u));
      const float zero = fmaxf(m, -3e38f);
      z = 0.f;
      for (int u = 0; u < per; ++u) z += sum_of(u) * exp2_hw(at_top(u) - zero);
    };
    join([&](int u) { return meet_d[g0 + u][0]; }, [&](int u) { return meet_d[g0 + u][1]; }, md, sd);
    for (int e = sub; e < 4; e += per) {
      float m, z;
      join([&](int u) { return reinterpret_cast<const float*>(&meet_m[g0 + u][c])[e]; },
           [&](int u) { return reinterpret_cast<const float*>(&meet_s[g0 + u][c])[e]; }, m, z);
      put(r, at + e, ((m - md) + (log2_hw(z) - log2_hw(sd))) / (r.beta[g * DV + c * 4 + e] * kLog2e));
    }
  }
}

}  // namespace fem
