// The paged FEM read: how a call's work is split, and its launches.

#include "fem_internal.h"
#include "fem_paged_rows.h"

#include <algorithm>

namespace fem {

namespace {
constexpr int kTarget = 1024;   // splits aimed at
constexpr int kShortKeys = 128; // contexts that one workgroup reads in one round
}  // namespace

PagedPlan paged_plan(const PagedArgs& a, int H, int dv) {
  PagedPlan p;
  const long long G = H / a.heads, rows = (long long)a.ntok * G, most = a.max_q * G;
  const long long blocks = std::min(rows / kRowsMax + a.nseq,
                                    (most + kRowsMax - 1) / kRowsMax * (long long)a.nseq);
  p.row_blocks = (int)std::min(blocks, 1ll << 30);
  p.target = ((long long)a.table_len << a.page_log2) <= kShortKeys ? 0 : kTarget;
  p.rps = (int)std::min<long long>(kRowsMax, most);
  p.slots = (size_t)p.target + (size_t)p.row_blocks * a.heads;
  p.ws_bytes = p.target ? p.slots * p.rps * (dv + 1) * sizeof(float) : 0;
  return p;
}

hipError_t launch_paged_read(const PagedArgs& a, const PagedPlan& plan, int kv, int dk, int dv,
                             const void* q, long long qld, const float* beta, void* out, int H,
                             bool causal, bool obf16, void* ws, hipStream_t stream) {
  ReadArgs r;
  r.q = static_cast<const bf16*>(q);
  r.qld = qld;
  r.beta = beta;
  r.out = out;
  r.part = static_cast<float*>(ws);
  r.H = H;
  r.G = H / a.heads;
  r.rps = plan.rps;
  r.target = plan.target;
  r.causal = causal;
  r.obf16 = obf16;
  if (dk == 32 && dv == 32) return paged_rows<32, 32>(a, r, plan, kv, stream);
  if (dk == 64 && dv == 64) return paged_rows<64, 64>(a, r, plan, kv, stream);
  if (dk == 64 && dv == 32) return paged_rows<64, 32>(a, r, plan, kv, stream);
  if (dk == 128 && dv == 128) return paged_rows<128, 128>(a, r, plan, kv, stream);
  if (dk == 128 && dv == 64) return paged_rows<128, 64>(a, r, plan, kv, stream);
  return hipErrorInvalidValue;
}

}  // namespace fem
