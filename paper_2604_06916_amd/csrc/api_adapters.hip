// C-ABI entry points of the low-rank adapters (declared and documented in
// solfp4.h).  Every argument check happens on the host before the first HIP
// call.
#include "solfp4.h"
#include "kernels.h"
#include "operand_checks.h"

namespace {

using namespace solfp4::checks;

int adapter_dims(int64_t tokens, int64_t adapters) {
  if (tokens < 0 || adapters < 1) return SOLFP4_EINVAL;
  return tokens >= solfp4::kAdapterMaxTokens || adapters > solfp4::kAdapterMaxAdapters ? SOLFP4_ESHAPE : SOLFP4_OK;
}

// Sizes, the adapters' weights and the plan, which both passes read.
struct Weights {
  const uint16_t *a, *b;
  const float* scales;
  const void* plan;
  int64_t adapters, tokens, N, K, rank;

  int check() const {
    const int rc = adapter_dims(tokens, adapters);
    if (rc) return rc;
    if (N < 0 || K < 0 || rank < 1) return SOLFP4_EINVAL;
    if (N >= solfp4::kAdapterMaxFeatures || K >= solfp4::kAdapterMaxFeatures || rank > solfp4::kAdapterMaxRank)
      return SOLFP4_ESHAPE;
    if (!plan && adapters != 1) return SOLFP4_EINVAL;
    if ((K > 0 && !a) || (N > 0 && !b)) return SOLFP4_EINVAL;
    return (uintptr_t)a & 1u || (uintptr_t)b & 1u || (uintptr_t)scales & 3u || !aligned16(plan) ? SOLFP4_EALIGN
                                                                                               : SOLFP4_OK;
  }
  // Whether what is written shares no byte with any of them.
  bool apart_from(const Region& o) const {
    return apart(o, block_of(a, a ? adapters * rank * K * 2 : 0)) && apart(o, block_of(b, b ? adapters * N * rank * 2 : 0)) &&
           apart(o, block_of(scales, scales ? adapters * 4 : 0)) &&
           apart(o, block_of(plan, plan ? (int64_t)solfp4::adapter_plan_bytes(tokens, adapters) : 0));
  }
};

// Sizes of a call, and its tokens.  Without a plan tiles start at every 32nd
// token, with one every adapter starts a tile.
bool sized(int64_t tokens, int64_t adapters, int planned, int64_t N, int64_t K, int64_t rank, solfp4::AdapterTokens* t) {
  if (adapter_dims(tokens, adapters) || rank < 1 || rank > solfp4::kAdapterMaxRank) return false;
  if (N < 0 || K < 0 || N >= solfp4::kAdapterMaxFeatures || K >= solfp4::kAdapterMaxFeatures) return false;
  *t = solfp4::adapter_tokens(planned ? t : nullptr, tokens, adapters);
  return true;
}

}  // namespace

extern "C" {

size_t solfp4_adapter_plan_bytes(int64_t tokens, int64_t adapters) {
  return adapter_dims(tokens, adapters) ? 0 : solfp4::adapter_plan_bytes(tokens, adapters);
}

int solfp4_adapter_plan(const void* index, int index_bytes, int64_t tokens, int64_t adapters, void* plan,
                        size_t plan_bytes, void* stream) {
  const int rc = adapter_dims(tokens, adapters);
  if (rc) return rc;
  if (index_bytes != 4 && index_bytes != 8) return SOLFP4_EINVAL;
  if (!plan || (tokens > 0 && !index)) return SOLFP4_EINVAL;
  if (!aligned16(plan) || ((uintptr_t)index & (uintptr_t)(index_bytes - 1))) return SOLFP4_EALIGN;
  const size_t need = solfp4::adapter_plan_bytes(tokens, adapters);
  if (plan_bytes < need) return SOLFP4_EWORKSPACE;
  if (!apart(block_of(plan, (int64_t)need), block_of(index, tokens * index_bytes))) return SOLFP4_EINVAL;
  const hipError_t e = solfp4::launch_adapter_plan(index, index_bytes, tokens, adapters, plan,
                                                   static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

size_t solfp4_add_adapters_workspace_bytes(int64_t tokens, int64_t adapters, int planned, int64_t N, int64_t K,
                                           int64_t rank) {
  solfp4::AdapterTokens t;
  return sized(tokens, adapters, planned, N, K, rank, &t) ? solfp4::add_adapters_bytes(t, K, rank) : 0;
}

int solfp4_add_adapters(const uint16_t* y, int64_t y_stride, const uint16_t* x, int64_t x_stride, const uint16_t* a,
                        const uint16_t* b, const float* scales, int64_t adapters, const void* plan, uint16_t* out,
                        int64_t out_stride, float* hidden, void* workspace, size_t workspace_bytes, int64_t tokens,
                        int64_t N, int64_t K, int64_t rank, void* stream) {
  const Weights w = {a, b, scales, plan, adapters, tokens, N, K, rank};
  int rc = w.check();
  if (rc) return rc;
  if (tokens == 0) return SOLFP4_OK;
  if (N > 0) {
    if ((rc = check_rows(SOLFP4_BF16, y, y_stride, tokens, N, false))) return rc;
    if ((rc = check_rows(SOLFP4_BF16, out, out_stride, tokens, N, true))) return rc;
  }
  if (K > 0 && (rc = check_rows(SOLFP4_BF16, x, x_stride, tokens, K, false))) return rc;
  if ((uintptr_t)hidden & 3u) return SOLFP4_EALIGN;
  const Region ry = rows_region(SOLFP4_BF16, N > 0 ? y : nullptr, y_stride, tokens, N);
  const Region rx = rows_region(SOLFP4_BF16, K > 0 ? x : nullptr, x_stride, tokens, K);
  const Region o = rows_region(SOLFP4_BF16, N > 0 ? out : nullptr, out_stride, tokens, N);
  const Region h = block_of(hidden, hidden ? tokens * rank * 4 : 0);
  if (!same_or_apart(ry, o) || !apart(rx, o) || !w.apart_from(o)) return SOLFP4_EINVAL;
  if (!apart(ry, h) || !apart(rx, h) || !apart(o, h) || !w.apart_from(h)) return SOLFP4_EINVAL;
  const solfp4::AdapterTokens t = solfp4::adapter_tokens(plan, tokens, adapters);
  const size_t need = solfp4::add_adapters_bytes(t, K, rank);
  if (need && !workspace) return SOLFP4_EWORKSPACE;
  if (!aligned16(workspace)) return SOLFP4_EALIGN;
  if (workspace_bytes < need) return SOLFP4_EWORKSPACE;
  const Region s = block_of(workspace, (int64_t)need);
  if (!apart(ry, s) || !apart(rx, s) || !apart(o, s) || !apart(h, s) || !w.apart_from(s)) return SOLFP4_EINVAL;
  solfp4::AdapterArgs args = {};
  args.t = t, args.y = y, args.y_stride = y_stride, args.x = x, args.x_stride = x_stride;
  args.a = a, args.b = b, args.scales = scales, args.out = out, args.out_stride = out_stride, args.hidden = hidden;
  args.N = (int)N, args.K = (int)K, args.rank = (int)rank;
  const hipError_t e = solfp4::launch_add_adapters(args, workspace, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

size_t solfp4_adapters_backward_workspace_bytes(int64_t tokens, int64_t adapters, int planned, int64_t N, int64_t K,
                                                int64_t rank) {
  solfp4::AdapterTokens t;
  return sized(tokens, adapters, planned, N, K, rank, &t) ? solfp4::adapters_backward_bytes(t, N, K, rank) : 0;
}

int solfp4_adapters_backward(const uint16_t* dy, int64_t dy_stride, const uint16_t* x, int64_t x_stride,
                             const float* hidden, const uint16_t* a, const uint16_t* b, const float* scales,
                             int64_t adapters, const void* plan, const uint16_t* past, int64_t past_stride,
                             uint16_t* dx, int64_t dx_stride, float* da, float* db, void* workspace,
                             size_t workspace_bytes, int64_t tokens, int64_t N, int64_t K, int64_t rank, void* stream) {
  const Weights w = {a, b, scales, plan, adapters, tokens, N, K, rank};
  int rc = w.check();
  if (rc) return rc;
  if ((K > 0 && !da) || (N > 0 && !db) || (tokens > 0 && !hidden)) return SOLFP4_EINVAL;
  if (((uintptr_t)da & 3u) || ((uintptr_t)db & 3u) || ((uintptr_t)hidden & 3u)) return SOLFP4_EALIGN;
  if (tokens > 0) {
    if (N > 0 && (rc = check_rows(SOLFP4_BF16, dy, dy_stride, tokens, N, false))) return rc;
    if (K > 0) {
      if ((rc = check_rows(SOLFP4_BF16, x, x_stride, tokens, K, false))) return rc;
      if (past && (rc = check_rows(SOLFP4_BF16, past, past_stride, tokens, K, false))) return rc;
      if ((rc = check_rows(SOLFP4_BF16, dx, dx_stride, tokens, K, true))) return rc;
    }
  }
  const solfp4::AdapterTokens t = solfp4::adapter_tokens(plan, tokens, adapters);
  const size_t need = solfp4::adapters_backward_bytes(t, N, K, rank);
  if (need && !workspace) return SOLFP4_EWORKSPACE;
  if (!aligned16(workspace)) return SOLFP4_EALIGN;
  if (workspace_bytes < need) return SOLFP4_EWORKSPACE;
  const bool n = tokens > 0 && N > 0, k = tokens > 0 && K > 0;
  const Region in[4] = {rows_region(SOLFP4_BF16, n ? dy : nullptr, dy_stride, tokens, N),
                        rows_region(SOLFP4_BF16, k ? x : nullptr, x_stride, tokens, K),
                        block_of(hidden, tokens > 0 ? tokens * rank * 4 : 0),
                        rows_region(SOLFP4_BF16, k ? past : nullptr, past_stride, tokens, K)};
  const Region out[4] = {rows_region(SOLFP4_BF16, k ? dx : nullptr, dx_stride, tokens, K),
                         block_of(da, K > 0 ? adapters * rank * K * 4 : 0),
                         block_of(db, N > 0 ? adapters * N * rank * 4 : 0), block_of(workspace, (int64_t)need)};
  for (int o = 0; o < 4; ++o) {
    for (int i = 0; i < 4; ++i)   // dx in the place of past alone
      if (!(o == 0 && i == 3 ? same_or_apart(in[i], out[o]) : apart(in[i], out[o]))) return SOLFP4_EINVAL;
    for (int i = 0; i < o; ++i)
      if (!apart(out[i], out[o])) return SOLFP4_EINVAL;
    if (!w.apart_from(out[o])) return SOLFP4_EINVAL;
  }
  const solfp4::AdapterBackArgs args = {t, dy, dy_stride, x, x_stride, hidden, a, b, scales, past, past_stride, dx,
                                        dx_stride, da, db, (int)N, (int)K, (int)rank};
  const hipError_t e = solfp4::launch_adapters_backward(args, workspace, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

}  // extern "C"
