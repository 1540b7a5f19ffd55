// The paged FEM read: which kernels a call takes, and their scratch.

#include "fem_internal.h"
#include "fem_paged_wide.h"

#include <algorithm>

namespace fem {

namespace {
constexpr int kUnits = 256;      // compute units
// Contexts that are not split: eight waves have four tiles each at most, which
// takes about as long as the merge of splits would (one token, 8 heads,
// 701 keys, d = 64: 12.5 us, and 14.4 with four waves, splits and a merge).
constexpr int kShortKeys = 1024;
constexpr int kMergeRows = 8;    // of a merge's workgroup, few rows a block

// Rows of a merge's workgroup, many rows a block: as many as leave about four
// workgroups a compute unit, whose cost is mostly finding their rows (one block of
// 256 rows and eight heads in 32 splits: 48 us with 4 rows, 51 with 8, 59 with 16;
// ten blocks and twelve heads in two: 64 with 8 and 58 with 16).
int wide_merge_rows(size_t rows) {
  int n = 4;
  while (n < 16 && rows / (2 * n) >= 4 * kUnits) n *= 2;
  return n;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }
}  // namespace

// Up to 32 rows a sequence the kernel for few rows; more, the one for many; both
// where max_q allows either.
PagedPlan paged_plan(const PagedArgs& a, int H, int dv) {
  PagedPlan p = {};
  const long long G = H / a.heads, rows = (long long)a.ntok * G, most = a.max_q * G;
  const long long keys = (long long)a.table_len << a.page_log2;
  auto blocks = [&](long long most_, int br) {
    return (int)std::min(rows / br + a.nseq, (most_ + br - 1) / br * (long long)a.nseq);
  };
  p.wide = most > kRowsMax;
  p.rows = !p.wide || a.nseq > 1;
  p.most_rows = kRowsMax;
  p.wide_least = p.rows ? kRowsMax : 0;
  size_t at = 256;  // the two kernels' split sizes
  p.part_at = at;
  if (p.rows) {  // in a launch of their own, or in the other kernel's
    const long long m = std::min<long long>(most, kRowsMax);
    p.row_blocks = blocks(m, kRowsMax);
    p.rps = (int)m;
    const bool brief = keys <= kShortKeys;
    p.waves = brief ? 2 * kRowWaves : kRowWaves;
    const int room = kUnits * (brief || p.wide ? 1 : kRowGroups);
    p.target = brief ? 0 : room;
    p.groups = p.target ? room : std::min<size_t>((size_t)p.row_blocks * a.heads, room);
    if (p.target) at += up256((size_t)p.target * p.rps * part_row(dv) * sizeof(float));
  }
  p.wide_at = at;
  if (p.wide) {
    p.wide_blocks = blocks(most, kWideRows);
    p.split_wide = keys > kLeastTiles * kWideTile;
    p.wide_rps = (int)std::min<long long>(most, kWideRows);
    p.wide_groups = (size_t)p.wide_blocks * a.heads;
    if (p.split_wide) {
      p.wide_groups = std::max<size_t>(p.wide_groups, kWideUnits);
      at += up256((size_t)kWideUnits * p.wide_rps * part_row(dv) * sizeof(float));
    }
  }
  if (p.wide && p.rows)
    p.wide_groups += std::max<size_t>((size_t)p.row_blocks * a.heads, p.target);
  p.ws_bytes = p.target || p.split_wide ? at : 0;
  return p;
}

hipError_t launch_paged_read(const PagedArgs& a, const PagedPlan& plan, int kv, int dk, int dv,
                             const void* q, long long qld, const float* beta, void* out, int H,
                             bool causal, bool obf16, void* ws, hipStream_t stream) {
  ReadArgs r = {};
  r.q = static_cast<const bf16*>(q);
  r.qld = qld;
  r.beta = beta;
  r.out = out;
  r.tps = static_cast<int*>(ws);
  r.part = reinterpret_cast<float*>(static_cast<char*>(ws) + plan.part_at);
  r.wide_part = reinterpret_cast<float*>(static_cast<char*>(ws) + plan.wide_at);
  r.H = H;
  r.G = H / a.heads;
  r.rps = plan.rps;
  r.wide_rps = plan.wide_rps;
  r.target = plan.target;
  r.split_wide = plan.split_wide;
  r.rows_too = plan.wide && plan.rows;
  r.most_rows = plan.most_rows;
  r.wide_least = plan.wide_least;
  r.causal = causal;
  r.obf16 = obf16;
  // The merge's workgroups: calls of more blocks than splits are aimed at are not split.
  MergePart few = {}, many = {};
  auto part = [&](MergePart& m, const Work& w, const int* tps, const float* at, int rps,
                  size_t blocks, int rows) {
    m = MergePart{w, tps, at, rps, rows, 0, kLog2e / sqrtf((float)dk)};
    m.groups = (int)(blocks * ((rps + m.rows - 1) / m.rows));
  };
  if (plan.rows && plan.target)
    part(few, rows_work(a, r), r.tps, r.part, plan.rps,
         std::min<size_t>((size_t)plan.row_blocks * a.heads, plan.target), kMergeRows);
  if (plan.wide && plan.split_wide) {
    const size_t blocks = std::min<size_t>((size_t)plan.wide_blocks * a.heads, kMostSplitBlocks);
    part(many, wide_work(a, r), r.tps + 1, r.wide_part, plan.wide_rps, blocks,
         wide_merge_rows(blocks * plan.wide_rps));
  }
  auto go = [&](auto rows, auto wide, auto merge) {
    hipError_t e = hipSuccess;
    e = plan.wide ? wide(a, r, plan, kv, stream) : rows(a, r, plan, kv, stream);
    if (e == hipSuccess && few.groups + many.groups > 0) {
      hipLaunchKernelGGL(merge, dim3((unsigned)(few.groups + many.groups)), dim3(kMergeThreads), 0,
                         stream, a, r, few, many);
      e = hipGetLastError();
    }
    return e;
  };
  if (dk == 32 && dv == 32) return go(paged_rows<32, 32>, paged_wide<32, 32>, paged_merge_kernel<32>);
  if (dk == 64 && dv == 64) return go(paged_rows<64, 64>, paged_wide<64, 64>, paged_merge_kernel<64>);
  if (dk == 64 && dv == 32) return go(paged_rows<64, 32>, paged_wide<64, 32>, paged_merge_kernel<32>);
  if (dk == 128 && dv == 128)
    return go(paged_rows<128, 128>, paged_wide<128, 128>, paged_merge_kernel<128>);
  if (dk == 128 && dv == 64)
    return go(paged_rows<128, 64>, paged_wide<128, 64>, paged_merge_kernel<64>);
  return hipErrorInvalidValue;
}

}  // namespace fem
