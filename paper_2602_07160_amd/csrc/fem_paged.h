// The paged key/value cache as the kernels see it: addresses, stored values,
// and the sequences of a call.
#pragma once

#include "fem.h"
#include "fem_device.h"

namespace fem {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2v;

constexpr int kScaleBlock = 32;   // channels that share a scale
constexpr int kLeastExp = -100;   // smallest scale exponent: every stored value is a normal bf16

// One call's cache and sequences (the public structs with derived sizes).
struct PagedArgs {
  const uint8_t* k;        // [pages][heads][page][dk] codes or bf16
  const uint8_t* v;        // [pages][heads][page][dv]
  const uint8_t* ks;       // [pages][heads][page][dk / 32] scale bytes
  const uint8_t* vs;
  const int* q_start;      // [nseq + 1]
  const int* lens;         // [nseq]
  const int* table;        // [nseq][table_len]
  int pages, page, page_log2, heads;
  int nseq, table_len, ntok, max_q;
};

// Scale 2^(byte - 127).  255 gives +inf, which makes the zeros of such a block NaN.
__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte << 23); }

// Two words (8 codes) as 8 bf16 values: exact, since a code has at most eight
// significant bits.
template <int KV>
__device__ __forceinline__ u32x4 dequant8(unsigned w0, unsigned w1, float s) {
  if constexpr (KV == FEM_KV_E4M3) {
    // two codes to bf16, scaled, in one instruction (checked for every code and
    // scale byte from 27 on against the conversion to float and a product)
    auto pair = [s](unsigned w, bool hi) {
      return __builtin_bit_cast(unsigned, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)
                                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
    };
    return u32x4{pair(w0, false), pair(w0, true), pair(w1, false), pair(w1, true)};
  } else {
    // code + 128 as an unsigned byte, so that one conversion and one
    // multiply-add (a single rounding of an exact result) give the value, whose
    // high half is the bf16
    const float o = -128.f * s;
    auto pair = [s, o](unsigned u, int e) {
      const float x = fmaf((float)((u >> (8 * e)) & 0xffu), s, o);
      const float y = fmaf((float)((u >> (8 * e + 8)) & 0xffu), s, o);
      return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
    };
    w0 ^= 0x80808080u;
    w1 ^= 0x80808080u;
    return u32x4{pair(w0, 0), pair(w0, 2), pair(w1, 0), pair(w1, 2)};
  }
}

// Eight consecutive values (chunk c) of a stored row as floats.
template <int KV, int W>
__device__ __forceinline__ void row8(const uint8_t* pool, const uint8_t* scales, size_t row, int c,
                                     float (&f)[8]) {
  u32x4 w;
  if constexpr (KV == FEM_KV_BF16) {
    w = *reinterpret_cast<const u32x4*>(pool + (row * W + c * 8) * 2);
  } else {
    const u32x2v r = *reinterpret_cast<const u32x2v*>(pool + row * W + c * 8);
    w = dequant8<KV>(r[0], r[1], scale_of(scales[row * (W / kScaleBlock) + c / 4]));
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __uint_as_float(w[e] << 16);
    f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}

// A sequence of the call.  Its token range is always inside [0, ntok]; `ok` is
// false where the lengths contradict each other or the table: such a
// sequence's tokens read NaN and its new rows are not stored.
struct Seq {
  int q0, n, len;
  bool ok;
};

__device__ __forceinline__ Seq seq_of(const PagedArgs& a, int b, bool causal) {
  Seq s;
  const int q0 = a.q_start[b], q1 = a.q_start[b + 1];
  s.len = a.lens[b];
  s.q0 = min(max(q0, 0), a.ntok);
  s.n = max(min(q1, a.ntok) - s.q0, 0);
  s.ok = q0 >= 0 && q1 >= q0 && q1 <= a.ntok && s.len >= (causal ? s.n : 0) &&
         (unsigned long long)s.len <= (unsigned long long)a.table_len << a.page_log2;
  return s;
}

// Row index (of [pages * heads * page] rows) of key i of sequence b, head g; a
// page id outside the pool makes `bad` true and reads page 0.
__device__ __forceinline__ size_t paged_row(const PagedArgs& a, int b, int g, int i, bool& bad) {
  int p = a.table[(size_t)b * a.table_len + (i >> a.page_log2)];
  if ((unsigned)p >= (unsigned)a.pages) {
    bad = true;
    p = 0;
  }
  return (((size_t)p * a.heads + g) << a.page_log2) + (i & (a.page - 1));
}

}  // namespace fem
