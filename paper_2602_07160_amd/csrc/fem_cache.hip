// Writing the paged key/value cache and reading it back.
//
// A stored row (token, head) is bf16, or 8-bit codes with one power-of-two
// scale 2^e for every 32 channels:
//
//   e = the smallest integer >= -100 with max |x| <= M 2^e,
//       M = 448 (e4m3) or 127 (int8);
//   code = x 2^-e rounded to nearest even;  value = code 2^e.
//
// No code saturates, and every value is a bf16 number (a code has at most
// eight significant bits), so a read over a quantised cache is the bf16 read
// over its values.  A power-of-two scale costs an e4m3 code nothing (the
// format is floating itself) and an int8 code at most one bit.
//
// Both kernels are copies with a conversion, bound by HBM bandwidth; for a few
// tokens by the launch's latency.

#include "fem_internal.h"
#include "fem_paged.h"

namespace fem {
namespace {

constexpr int kThreads = 256;

// ---- append -----------------------------------------------------------------

// The smallest exponent e >= kLeastExp with top <= M 2^e, M = m 2^p with
// m in [1, 2): the exponent of top less p, one more where top's significand
// exceeds m.
template <int KV>
__device__ __forceinline__ int scale_exp(float top) {
  constexpr int p = KV == FEM_KV_E4M3 ? 8 : 6;
  constexpr unsigned frac = KV == FEM_KV_E4M3 ? 0x600000u : 0x7e0000u;  // 1.75, 127 / 64
  const unsigned u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 127 - p + ((u & 0x7fffffu) > frac ? 1 : 0);
  return max(e, kLeastExp);
}

// Eight bf16 of one row's chunk into the pool; four neighbouring lanes hold a
// scale's 32 channels.
template <int KV>
__device__ __forceinline__ void store8(u32x4 x, uint8_t* pool, uint8_t* scales, size_t row, int w,
                                       int c) {
  if constexpr (KV == FEM_KV_BF16) {
    *reinterpret_cast<u32x4*>(pool + (row * w + c * 8) * 2) = x;
    return;
  }
  // the largest |x| as its bits: ordered like the values, inf and NaN on top
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  u16x2 t2 = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    t2 = __builtin_elementwise_max(t2, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
  unsigned top = max(t2[0], t2[1]);
  top = max(top, (unsigned)__shfl_xor((int)top, 1));
  top = max(top, (unsigned)__shfl_xor((int)top, 2));
  const bool fine = top < 0x7f80u;
  const int e = fine ? scale_exp<KV>(__uint_as_float(top << 16)) : 0;
  const float inv = __uint_as_float((unsigned)(127 - e) << 23);
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(x[i] << 16);
    f[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
  }
  unsigned w0 = 0, w1 = 0;
  if (fine) {
    if constexpr (KV == FEM_KV_E4M3) {
      w0 = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[0] * inv, f[1] * inv, (int)w0, false);
      w0 = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[2] * inv, f[3] * inv, (int)w0, true);
      w1 = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[4] * inv, f[5] * inv, (int)w1, false);
      w1 = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[6] * inv, f[7] * inv, (int)w1, true);
    } else {
      // added to 1.5 * 2^23, the (exact) product is rounded to a whole number, ties
      // to even, that stands in the low byte
      auto four = [&](int i) {
        unsigned u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = __float_as_uint(fmaf(f[i + j], inv, 12582912.f));
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u),
                                     __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), 0x05040100u);
      };
      w0 = four(0);
      w1 = four(4);
    }
  }
  *reinterpret_cast<u32x2v*>(pool + row * w + c * 8) = u32x2v{w0, w1};
  if ((c & 3) == 0) scales[row * (w / kScaleBlock) + c / 4] = (uint8_t)(fine ? e + 127 : 255);
}

// The sequence of token t: the last b with q_start[b] <= t (sequences without
// new tokens share their start with the next one).
__device__ __forceinline__ int sequence_of(const int* q_start, int nseq, int t) {
  int lo = 0, hi = nseq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (q_start[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

constexpr int kAppendTokens = 32;  // of a workgroup
constexpr int kAppendBatch = 2;    // loads in flight of a thread

// Workgroup (32 tokens, head): the tokens' slots are found once (a thread each), then
// every thread takes 16-byte chunks of their K rows and of their V rows.  Consecutive
// tokens of one head are neighbours in the pool: their rows and, above all, their few
// scale bytes leave as whole cache lines.  (With the workgroups on tokens instead, all
// heads of a few, 10713 tokens of 16 heads of 128 took 38.5 us in int8, 34.8
// so, 3.8 TB/s.)
template <int KV>
__global__ __launch_bounds__(kThreads) void append_kernel(PagedArgs a, uint8_t* kp, uint8_t* vp,
                                                          uint8_t* ksp, uint8_t* vsp,
                                                          const bf16* __restrict__ k, long long kld,
                                                          const bf16* __restrict__ v, long long vld,
                                                          int dk, int dv) {
  __shared__ long long slot[kAppendTokens];  // the token's row, or -1
  const int g = blockIdx.x % a.heads, t0 = blockIdx.x / a.heads * kAppendTokens, tid = threadIdx.x;
  if (tid < kAppendTokens) {
    const int t = t0 + tid;
    long long s = -1;
    if (t < a.ntok) {
      const int b = sequence_of(a.q_start, a.nseq, t);
      const Seq q = seq_of(a, b, true);
      const int i = t - q.q0;
      if (q.ok && i >= 0 && i < q.n) {
        bool bad = false;
        const size_t r = paged_row(a, b, g, q.len - q.n + i, bad);
        if (!bad) s = (long long)r;
      }
    }
    slot[tid] = s;
  }
  __syncthreads();
  auto rows = [&](const bf16* x, long long ld, int w, uint8_t* pool, uint8_t* scales) {
    const int sh = 28 - __builtin_clz(w);  // log2 of the row's chunks
    const int all = min(kAppendTokens, a.ntok - t0) << sh;
    for (int x0 = tid; x0 < all; x0 += kThreads * kAppendBatch) {
      u32x4 c[kAppendBatch];
#pragma unroll
      for (int u = 0; u < kAppendBatch; ++u) {
        const int i = x0 + u * kThreads;
        if (i < all)
          c[u] = *reinterpret_cast<const u32x4*>(x + (size_t)(t0 + (i >> sh)) * (size_t)ld + g * w +
                                                 (i & ((1 << sh) - 1)) * 8);
      }
#pragma unroll
      for (int u = 0; u < kAppendBatch; ++u) {
        const int i = x0 + u * kThreads;
        if (i >= all) continue;
        const long long s = slot[i >> sh];  // (the same for the four lanes of a scale)
        if (s >= 0) store8<KV>(c[u], pool, scales, (size_t)s, w, i & ((1 << sh) - 1));
      }
    }
  };
  rows(k, kld, dk, kp, ksp);
  rows(v, vld, dv, vp, vsp);
}

// ---- gather -----------------------------------------------------------------

constexpr int kGatherRows = 64;

// Workgroup (b, g, block of 64 rows): K's rows, then V's, 8 values a thread.  At the
// rate of a copy: 95 k tokens of 8 heads of 128 in e4m3, 587 MB, 116 us, 5.05 TB/s.
template <int KV>
__device__ __forceinline__ void gather_rows(const PagedArgs& a, const uint8_t* pool,
                                            const uint8_t* scales, bf16* out, int w, int n,
                                            const long long* rows) {
  const int cw = w / 8;  // a power of two
  const int sh = 31 - __builtin_clz(cw);
  for (int x = threadIdx.x; x < n * cw; x += kThreads) {
    const int r = x >> sh, c = x & (cw - 1);
    const long long row = rows[r];
    u32x4 o = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    if (row >= 0) {
      if constexpr (KV == FEM_KV_BF16) {
        o = *reinterpret_cast<const u32x4*>(pool + ((size_t)row * w + c * 8) * 2);
      } else {
        const u32x2v q = *reinterpret_cast<const u32x2v*>(pool + (size_t)row * w + c * 8);
        o = dequant8<KV>(q[0], q[1], scale_of(scales[(size_t)row * (w / kScaleBlock) + c / 4]));
      }
    }
    *reinterpret_cast<u32x4*>(out + (size_t)r * w + c * 8) = o;
  }
}

template <int KV>
__global__ __launch_bounds__(kThreads) void gather_kernel(PagedArgs a, bf16* __restrict__ ko,
                                                          bf16* __restrict__ vo, int L, int dk,
                                                          int dv, int nblk) {
  __shared__ long long rows[kGatherRows];
  const int blk = blockIdx.x % nblk, bg = blockIdx.x / nblk;
  const int b = bg / a.heads, g = bg % a.heads;
  const int len = a.lens[b], i0 = blk * kGatherRows;
  if ((unsigned long long)(unsigned)max(len, 0) > (unsigned long long)a.table_len << a.page_log2)
    return;
  const int n = min(min(len, L) - i0, kGatherRows);
  if (n <= 0) return;
  if ((int)threadIdx.x < n) {
    bool bad = false;
    const size_t r = paged_row(a, b, g, i0 + threadIdx.x, bad);
    rows[threadIdx.x] = bad ? -1 : (long long)r;
  }
  __syncthreads();
  const size_t at = (size_t)bg * L + i0;
  if (ko) gather_rows<KV>(a, a.k, a.ks, ko + at * dk, dk, n, rows);
  if (vo) gather_rows<KV>(a, a.v, a.vs, vo + at * dv, dv, n, rows);
}

}  // namespace

hipError_t launch_cache_append(const PagedArgs& a, int kv, int dk, int dv, void* kp, void* vp,
                               void* ksp, void* vsp, const void* k, long long kld, const void* v,
                               long long vld, hipStream_t stream) {
  const int groups = (a.ntok + kAppendTokens - 1) / kAppendTokens;
  const dim3 grid((unsigned)groups * (unsigned)a.heads), block(kThreads);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, static_cast<uint8_t*>(kp),
                       static_cast<uint8_t*>(vp), static_cast<uint8_t*>(ksp),
                       static_cast<uint8_t*>(vsp), static_cast<const bf16*>(k), kld,
                       static_cast<const bf16*>(v), vld, dk, dv);
  };
  if (kv == FEM_KV_BF16) go(append_kernel<FEM_KV_BF16>);
  else if (kv == FEM_KV_E4M3) go(append_kernel<FEM_KV_E4M3>);
  else go(append_kernel<FEM_KV_INT8>);
  return hipGetLastError();
}

hipError_t launch_cache_gather(const PagedArgs& a, int kv, int dk, int dv, void* ko, void* vo, int L,
                               hipStream_t stream) {
  const int nblk = (L + kGatherRows - 1) / kGatherRows;
  const dim3 grid((unsigned)((size_t)nblk * a.nseq * a.heads)), block(kThreads);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, static_cast<bf16*>(ko),
                       static_cast<bf16*>(vo), L, dk, dv, nblk);
  };
  if (kv == FEM_KV_BF16) go(gather_kernel<FEM_KV_BF16>);
  else if (kv == FEM_KV_E4M3) go(gather_kernel<FEM_KV_E4M3>);
  else go(gather_kernel<FEM_KV_INT8>);
  return hipGetLastError();
}

}  // namespace fem
