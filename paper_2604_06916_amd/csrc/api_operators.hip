// C-ABI entry points of the operators around the linears (declared and
// documented in solfp4.h).  Every argument check happens on the host before
// the first HIP call.
#include <math.h>

#include "solfp4.h"
#include "kernels.h"
#include "operand_checks.h"

namespace {

constexpr int64_t kMaxK = (int64_t)1 << 24, kMaxN = (int64_t)1 << 22;

using namespace solfp4::checks;

int norm_checks(int type, const solfp4::NormArgs& a, const void* shift_rows, int64_t shift_stride, int64_t groups, int out) {
  if (!type_ok(type)) return SOLFP4_EINVAL;
  int rc = check_dims(a.rows, a.width);
  if (rc) return rc;
  if (groups < 1 || !(a.eps >= 0.0f)) return SOLFP4_EINVAL;
  if (a.width > solfp4::kNormMaxWidth || a.rows % groups || (out != solfp4::kNormSame && a.width % 32))
    return SOLFP4_ESHAPE;
  if (a.rows == 0 || a.width == 0) return SOLFP4_OK;
  if ((rc = check_rows(type, a.x, a.x_stride, a.rows, a.width, false))) return rc;
  if (a.residual) {
    if ((rc = check_rows(type, a.residual, a.residual_stride, a.rows, a.width, false))) return rc;
    if ((rc = check_rows(type, a.sum, a.sum_stride, a.rows, a.width, true))) return rc;
  }
  if (a.gain && (rc = check_rows(type, a.gain, a.gain_stride, groups, a.width, false))) return rc;
  if (shift_rows && (rc = check_rows(type, shift_rows, shift_stride, groups, a.width, false))) return rc;
  // what is written over nothing else, except in place
  const Region x = rows_region(type, a.x, a.x_stride, a.rows, a.width);
  const Region residual = rows_region(type, a.residual, a.residual_stride, a.rows, a.width);
  const Region gain = rows_region(type, a.gain, a.gain_stride, groups, a.width);
  const Region shift = rows_region(type, shift_rows, shift_stride, groups, a.width);
  const Region sum = rows_region(type, a.residual ? a.sum : nullptr, a.sum_stride, a.rows, a.width);
  if (!same_or_apart(x, sum) || !same_or_apart(residual, sum) || !apart(gain, sum) || !apart(shift, sum))
    return SOLFP4_EINVAL;
  if (out == solfp4::kNormSame) {
    if ((rc = check_rows(type, a.out, a.out_stride, a.rows, a.width, true))) return rc;
    const Region o = rows_region(type, a.out, a.out_stride, a.rows, a.width);
    return same_or_apart(x, o) && apart(residual, o) && apart(gain, o) && apart(shift, o) && apart(sum, o)
               ? SOLFP4_OK : SOLFP4_EINVAL;
  }
  if (!a.codes || !a.scales) return SOLFP4_EINVAL;
  if (!aligned16(a.codes) || !aligned16(a.scales)) return SOLFP4_EALIGN;
  const Region codes = block_of(a.codes, a.rows * (out == solfp4::kNormMxfp8 ? a.width : a.width / 2));
  const Region scales = block_of(a.scales, a.rows * (a.width / 32));
  for (const Region& o : {codes, scales})
    if (!apart(x, o) || !apart(residual, o) || !apart(gain, o) || !apart(shift, o) || !apart(sum, o))
      return SOLFP4_EINVAL;
  return apart(codes, scales) ? SOLFP4_OK : SOLFP4_EINVAL;
}

int add_rmsnorm(int type, int kind, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                const void* gain, int64_t gain_stride, int64_t groups, float eps, void* sum, int64_t sum_stride,
                void* out, int64_t out_stride, uint8_t* codes, uint8_t* scales, int64_t rows, int64_t width,
                void* stream) {
  const solfp4::NormArgs a = {x, x_stride, residual, residual_stride, gain, gain_stride,
                              groups > 0 && rows > 0 ? rows / groups : 1, eps, sum, sum_stride, out, out_stride,
                              codes, scales, rows, width, 0};
  const int rc = norm_checks(type, a, nullptr, 0, groups, kind);
  if (rc) return rc;
  const hipError_t e = solfp4::launch_add_rmsnorm(type, kind, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

int add_layernorm(int type, int kind, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                  const void* gain, int64_t gain_stride, const void* shift, int64_t shift_stride, int64_t groups,
                  float eps, void* sum, int64_t sum_stride, void* out, int64_t out_stride, uint8_t* codes,
                  uint8_t* scales, int64_t rows, int64_t width, void* stream) {
  const solfp4::LayerNormArgs a = {{x, x_stride, residual, residual_stride, gain, gain_stride,
                                    groups > 0 && rows > 0 ? rows / groups : 1, eps, sum, sum_stride, out, out_stride,
                                    codes, scales, rows, width, 0}, shift, shift_stride};
  const int rc = norm_checks(type, a.n, shift, shift_stride, groups, kind);
  if (rc) return rc;
  const hipError_t e = solfp4::launch_add_layernorm(type, kind, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

size_t back_workspace(int64_t rows, int64_t width, int64_t groups) {
  const int64_t parts = solfp4::rmsnorm_backward_parts(rows, width, groups);
  if (parts == 0) return 0;
  // one part needs none, but a caller need not tell its sizes apart
  const size_t bytes = parts == 1 ? 1 : (size_t)(parts * groups) * (size_t)width * sizeof(float);
  return (bytes + 255) / 256 * 256;
}

int back_dims(int64_t rows, int64_t width, int64_t groups) {
  const int rc = check_dims(rows, width);
  if (rc) return rc;
  if (groups < 1) return SOLFP4_EINVAL;
  return width > solfp4::kNormMaxWidth || groups > 65535 || rows % groups ? SOLFP4_ESHAPE : SOLFP4_OK;
}

int linear_checks(const void* x, const void* x_scales, bool scaled_x, const void* wc, const void* ws, const float* wg,
                  bool has_global, const uint16_t* bias, const uint16_t* out, int64_t M, int64_t N, int64_t K,
                  int64_t block) {
  int rc = check_dims(M, N);
  if (rc) return rc;
  rc = check_dims(K, 0);
  if (rc) return rc;
  if (K % block || K >= kMaxK || N >= kMaxN) return SOLFP4_ESHAPE;
  if (M == 0 || N == 0) return SOLFP4_OK;
  if (!out || (has_global && !wg)) return SOLFP4_EINVAL;
  if (K > 0 && (!x || !wc || !ws || (scaled_x && !x_scales))) return SOLFP4_EINVAL;
  if (!aligned16(out) || (bias && !aligned16(bias)) || (has_global && !aligned16(wg))) return SOLFP4_EALIGN;
  if (K > 0 && (!aligned16(x) || !aligned16(wc) || !aligned16(ws) || (scaled_x && !aligned16(x_scales))))
    return SOLFP4_EALIGN;
  const Region o = block_of(out, M * N * 2);
  const Region in[6] = {block_of(x, M * K * (scaled_x ? 1 : 2)), block_of(x_scales, scaled_x ? M * (K / 32) : 0),
                        block_of(wc, N * (K / 2)), block_of(ws, N * (K / block)),
                        block_of(wg, has_global ? 4 : 0), block_of(bias, bias ? N * 2 : 0)};
  for (const Region& i : in)
    if (!apart(i, o)) return SOLFP4_EINVAL;
  return SOLFP4_OK;
}

int run_linear(int format, bool x8, const solfp4::WeightLinearArgs& a, void* stream) {
  const hipError_t e = solfp4::launch_weight_linear(format, x8, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

int rotary_operand(int type, solfp4::RotaryOperand* o, const void* in, int64_t it, int64_t ih, void* out, int64_t ot,
                   int64_t oh, int64_t heads, int64_t tokens, int64_t dim) {
  if (heads < 0) return SOLFP4_EINVAL;
  if (heads >= 1 << 20) return SOLFP4_ESHAPE;
  *o = {in, it, ih, out, ot, oh, (int)heads};
  if (heads == 0 || tokens == 0 || dim == 0) return SOLFP4_OK;
  if (!in || !out || it < 0 || ih < 0 || ot < 0 || oh < 0) return SOLFP4_EINVAL;
  if (!span_ok(it, tokens) || !span_ok(ih, heads) || !span_ok(ot, tokens) || !span_ok(oh, heads)) return SOLFP4_ESHAPE;
  if (!element_aligned(type, in) || !element_aligned(type, out)) return SOLFP4_EALIGN;
  // heads of the output must not overlap: either order of tokens and heads
  const bool by_token = (heads == 1 || oh >= dim) && (tokens == 1 || ot >= (heads - 1) * oh + dim);
  const bool by_head = (tokens == 1 || ot >= dim) && (heads == 1 || oh >= (tokens - 1) * ot + dim);
  return by_token || by_head ? SOLFP4_OK : SOLFP4_EINVAL;
}

Region heads_region(int type, const void* p, int64_t token, int64_t head, int64_t heads, int64_t tokens, int64_t dim) {
  const int64_t bytes = type == SOLFP4_F32 ? 4 : 2;
  return {(uintptr_t)p, tokens, tokens > 1 ? token * bytes : 0, heads, heads > 1 ? head * bytes : 0, dim * bytes};
}

bool rotary_in_place(const solfp4::RotaryOperand& o, int64_t tokens) {
  return o.in == o.out && (o.in_token == o.out_token || tokens == 1) && (o.in_head == o.out_head || o.heads == 1);
}

}  // namespace

extern "C" {

int solfp4_add_rmsnorm(int type, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                       const void* gain, int64_t gain_stride, int64_t groups, float eps, void* sum,
                       int64_t sum_stride, void* out, int64_t out_stride, int64_t rows, int64_t width, void* stream) {
  return add_rmsnorm(type, solfp4::kNormSame, x, x_stride, residual, residual_stride, gain, gain_stride, groups, eps,
                     sum, sum_stride, out, out_stride, nullptr, nullptr, rows, width, stream);
}

int mxfp8_add_rmsnorm(int type, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                      const void* gain, int64_t gain_stride, int64_t groups, float eps, void* sum, int64_t sum_stride,
                      uint8_t* codes, uint8_t* scales, int64_t rows, int64_t width, void* stream) {
  return add_rmsnorm(type, solfp4::kNormMxfp8, x, x_stride, residual, residual_stride, gain, gain_stride, groups, eps,
                     sum, sum_stride, nullptr, 0, codes, scales, rows, width, stream);
}

int mxfp4_add_rmsnorm(int type, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                      const void* gain, int64_t gain_stride, int64_t groups, float eps, void* sum, int64_t sum_stride,
                      uint8_t* codes, uint8_t* scales, int64_t rows, int64_t width, void* stream) {
  return add_rmsnorm(type, solfp4::kNormMxfp4, x, x_stride, residual, residual_stride, gain, gain_stride, groups, eps,
                     sum, sum_stride, nullptr, 0, codes, scales, rows, width, stream);
}

size_t solfp4_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t width, int64_t groups) {
  return back_dims(rows, width, groups) ? 0 : back_workspace(rows, width, groups);
}

int solfp4_rmsnorm_backward(int type, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride,
                            const void* gain, int64_t gain_stride, int64_t groups, const void* dsum,
                            int64_t dsum_stride, float eps, void* dx, int64_t dx_stride, float* dgain,
                            void* workspace, size_t workspace_bytes, int64_t rows, int64_t width, void* stream) {
  if (!type_ok(type)) return SOLFP4_EINVAL;
  int rc = back_dims(rows, width, groups);
  if (rc) return rc;
  if (!(eps >= 0.0f)) return SOLFP4_EINVAL;
  if (width == 0) return SOLFP4_OK;
  if (rows > 0) {
    if ((rc = check_rows(type, dy, dy_stride, rows, width, false))) return rc;
    if ((rc = check_rows(type, x, x_stride, rows, width, false))) return rc;
    if (gain && (rc = check_rows(type, gain, gain_stride, groups, width, false))) return rc;
    if (dsum && (rc = check_rows(type, dsum, dsum_stride, rows, width, false))) return rc;
    if ((rc = check_rows(type, dx, dx_stride, rows, width, true))) return rc;
  }
  const size_t need = dgain ? back_workspace(rows, width, groups) : 0;
  if (dgain) {
    if ((uintptr_t)dgain & 3u) return SOLFP4_EALIGN;
    if (need && !workspace) return SOLFP4_EWORKSPACE;
    if (!aligned16(workspace)) return SOLFP4_EALIGN;
    if (workspace_bytes < need) return SOLFP4_EWORKSPACE;
  }
  if (rows > 0) {
    const Region in[4] = {rows_region(type, dy, dy_stride, rows, width), rows_region(type, x, x_stride, rows, width),
                          rows_region(type, dsum, dsum_stride, rows, width),
                          rows_region(type, gain, gain_stride, groups, width)};
    const Region out = rows_region(type, dx, dx_stride, rows, width);
    const Region sums = block_of(dgain, dgain ? groups * width * 4 : 0), scratch = block_of(workspace, (int64_t)need);
    for (int i = 0; i < 4; ++i)
      if (!(i < 3 ? same_or_apart(in[i], out) : apart(in[i], out)) || !apart(in[i], sums) || !apart(in[i], scratch))
        return SOLFP4_EINVAL;
    if (!apart(out, sums) || !apart(out, scratch) || !apart(sums, scratch)) return SOLFP4_EINVAL;
  }
  solfp4::NormBackArgs a = {};
  a.dy = dy, a.dy_stride = dy_stride, a.x = x, a.x_stride = x_stride;
  a.gain = gain, a.gain_stride = gain_stride, a.groups = groups;
  a.dsum = dsum, a.dsum_stride = dsum_stride, a.eps = eps;
  a.dx = dx, a.dx_stride = dx_stride;
  a.partial = dgain ? static_cast<float*>(workspace) : nullptr;
  a.rows = rows, a.width = width;
  const hipError_t e = solfp4::launch_rmsnorm_backward(type, a, dgain, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

int solfp4_add_layernorm(int type, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                         const void* gain, int64_t gain_stride, const void* shift, int64_t shift_stride,
                         int64_t groups, float eps, void* sum, int64_t sum_stride, void* out, int64_t out_stride,
                         int64_t rows, int64_t width, void* stream) {
  return add_layernorm(type, solfp4::kNormSame, x, x_stride, residual, residual_stride, gain, gain_stride, shift,
                       shift_stride, groups, eps, sum, sum_stride, out, out_stride, nullptr, nullptr, rows, width, stream);
}

int mxfp8_add_layernorm(int type, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                        const void* gain, int64_t gain_stride, const void* shift, int64_t shift_stride, int64_t groups,
                        float eps, void* sum, int64_t sum_stride, uint8_t* codes, uint8_t* scales, int64_t rows,
                        int64_t width, void* stream) {
  return add_layernorm(type, solfp4::kNormMxfp8, x, x_stride, residual, residual_stride, gain, gain_stride, shift,
                       shift_stride, groups, eps, sum, sum_stride, nullptr, 0, codes, scales, rows, width, stream);
}

int mxfp4_add_layernorm(int type, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                        const void* gain, int64_t gain_stride, const void* shift, int64_t shift_stride, int64_t groups,
                        float eps, void* sum, int64_t sum_stride, uint8_t* codes, uint8_t* scales, int64_t rows,
                        int64_t width, void* stream) {
  return add_layernorm(type, solfp4::kNormMxfp4, x, x_stride, residual, residual_stride, gain, gain_stride, shift,
                       shift_stride, groups, eps, sum, sum_stride, nullptr, 0, codes, scales, rows, width, stream);
}

size_t solfp4_layernorm_backward_workspace_bytes(int64_t rows, int64_t width, int64_t groups) {
  return back_dims(rows, width, groups) ? 0 : 2 * back_workspace(rows, width, groups);
}

int solfp4_layernorm_backward(int type, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride,
                              const void* gain, int64_t gain_stride, int64_t groups, const void* dsum,
                              int64_t dsum_stride, float eps, void* dx, int64_t dx_stride, float* dgain, float* dshift,
                              void* workspace, size_t workspace_bytes, int64_t rows, int64_t width, void* stream) {
  if (!type_ok(type)) return SOLFP4_EINVAL;
  int rc = back_dims(rows, width, groups);
  if (rc) return rc;
  if (!(eps >= 0.0f)) return SOLFP4_EINVAL;
  if (width == 0) return SOLFP4_OK;
  if (rows > 0) {
    if ((rc = check_rows(type, dy, dy_stride, rows, width, false))) return rc;
    if ((rc = check_rows(type, x, x_stride, rows, width, false))) return rc;
    if (gain && (rc = check_rows(type, gain, gain_stride, groups, width, false))) return rc;
    if (dsum && (rc = check_rows(type, dsum, dsum_stride, rows, width, false))) return rc;
    if ((rc = check_rows(type, dx, dx_stride, rows, width, true))) return rc;
  }
  // the gain's shares first, then the shift's
  const size_t half = back_workspace(rows, width, groups), gain_bytes = dgain ? half : 0;
  const size_t need = gain_bytes + (dshift ? half : 0);
  if (dgain || dshift) {
    if (((uintptr_t)dgain & 3u) || ((uintptr_t)dshift & 3u)) return SOLFP4_EALIGN;
    if (need && !workspace) return SOLFP4_EWORKSPACE;
    if (!aligned16(workspace)) return SOLFP4_EALIGN;
    if (workspace_bytes < need) return SOLFP4_EWORKSPACE;
  }
  const Region sums[2] = {block_of(dgain, dgain ? groups * width * 4 : 0), block_of(dshift, dshift ? groups * width * 4 : 0)};
  if (!apart(sums[0], sums[1])) return SOLFP4_EINVAL;
  if (rows > 0) {
    const Region in[4] = {rows_region(type, dy, dy_stride, rows, width), rows_region(type, x, x_stride, rows, width),
                          rows_region(type, dsum, dsum_stride, rows, width),
                          rows_region(type, gain, gain_stride, groups, width)};
    const Region out = rows_region(type, dx, dx_stride, rows, width), scratch = block_of(workspace, (int64_t)need);
    for (int i = 0; i < 4; ++i)
      if (!(i < 3 ? same_or_apart(in[i], out) : apart(in[i], out)) || !apart(in[i], sums[0]) ||
          !apart(in[i], sums[1]) || !apart(in[i], scratch))
        return SOLFP4_EINVAL;
    if (!apart(out, sums[0]) || !apart(out, sums[1]) || !apart(out, scratch) || !apart(sums[0], scratch) ||
        !apart(sums[1], scratch))
      return SOLFP4_EINVAL;
  }
  solfp4::LayerNormBackArgs a = {};
  a.n.dy = dy, a.n.dy_stride = dy_stride, a.n.x = x, a.n.x_stride = x_stride;
  a.n.gain = gain, a.n.gain_stride = gain_stride, a.n.groups = groups;
  a.n.dsum = dsum, a.n.dsum_stride = dsum_stride, a.n.eps = eps;
  a.n.dx = dx, a.n.dx_stride = dx_stride;
  a.n.partial = dgain ? static_cast<float*>(workspace) : nullptr;
  a.shift_partial = dshift ? reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + gain_bytes) : nullptr;
  a.n.rows = rows, a.n.width = width;
  const hipError_t e = solfp4::launch_layernorm_backward(type, a, dgain, dshift, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

int solfp4_rotary_table(const int64_t* positions, int64_t rows, const double* frequencies, int64_t pairs,
                        const int64_t* axis_pairs, int axes, double magnitude, float* table, void* stream) {
  int rc = check_dims(rows, pairs);
  if (rc) return rc;
  if (axes < 1 || (axes > 1 && (!axis_pairs || !positions))) return SOLFP4_EINVAL;
  if (axes > solfp4::kRotaryMaxAxes || pairs >= 1 << 20) return SOLFP4_ESHAPE;
  solfp4::RotaryTableArgs a = {positions, frequencies, rows, (int)pairs, axes, {}, magnitude, table, 0};
  int64_t end = axis_pairs ? 0 : pairs;
  for (int i = 0; i < axes; ++i) {
    if (axis_pairs) {
      if (axis_pairs[i] < 0) return SOLFP4_EINVAL;
      if (axis_pairs[i] > pairs - end) return SOLFP4_ESHAPE;
      end += axis_pairs[i];
    }
    a.axis_end[i] = (int)end;
  }
  if (end != pairs) return SOLFP4_ESHAPE;
  if (rows == 0 || pairs == 0) return SOLFP4_OK;
  if (!frequencies || !table) return SOLFP4_EINVAL;
  if (((uintptr_t)positions & 7u) || ((uintptr_t)frequencies & 7u) || ((uintptr_t)table & 3u)) return SOLFP4_EALIGN;
  const Region out = block_of(table, rows * pairs * 8);
  if (!apart(out, block_of(frequencies, pairs * 8)) ||
      !apart(out, block_of(positions, positions ? rows * axes * 8 : 0)))
    return SOLFP4_EINVAL;
  const hipError_t e = solfp4::launch_rotary_table(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

int solfp4_rotary(int type, int layout, int inverse, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                  void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, int64_t q_heads, const void* k,
                  int64_t k_token_stride, int64_t k_head_stride, void* k_out, int64_t k_out_token_stride,
                  int64_t k_out_head_stride, int64_t k_heads, const float* table, int64_t table_rows,
                  const void* positions, int position_bytes, int64_t tokens, int64_t dim, int64_t rotated,
                  void* stream) {
  if (!type_ok(type) || (layout != SOLFP4_ROTARY_HALF && layout != SOLFP4_ROTARY_INTERLEAVED)) return SOLFP4_EINVAL;
  int rc = check_dims(tokens, dim);
  if (rc) return rc;
  if (rotated < 0 || table_rows < 0) return SOLFP4_EINVAL;
  if (rotated % 2 || rotated > dim || dim >= 1 << 20) return SOLFP4_ESHAPE;
  if (position_bytes != 0 && position_bytes != 4 && position_bytes != 8) return SOLFP4_EINVAL;
  solfp4::RotaryArgs a = {};
  if ((rc = rotary_operand(type, &a.q, q, q_token_stride, q_head_stride, q_out, q_out_token_stride, q_out_head_stride,
                           q_heads, tokens, dim)))
    return rc;
  if ((rc = rotary_operand(type, &a.k, k, k_token_stride, k_head_stride, k_out, k_out_token_stride, k_out_head_stride,
                           k_heads, tokens, dim)))
    return rc;
  if ((q_heads + k_heads) * dim >= kMaxDim) return SOLFP4_ESHAPE;
  if (tokens == 0 || dim == 0 || q_heads + k_heads == 0) return SOLFP4_OK;
  if ((position_bytes != 0) != (positions != nullptr)) return SOLFP4_EINVAL;
  if (rotated > 0 && (!table || table_rows == 0)) return SOLFP4_EINVAL;
  if (rotated > 0 && table_rows > kMaxSpan / rotated) return SOLFP4_ESHAPE;
  if ((uintptr_t)table & 3u) return SOLFP4_EALIGN;
  if (position_bytes && ((uintptr_t)positions & (uintptr_t)(position_bytes - 1))) return SOLFP4_EALIGN;
  // neither output over what the call reads, except in place, nor over the other
  const solfp4::RotaryOperand* const both[2] = {&a.q, &a.k};
  for (int i = 0; i < 2; ++i) {
    const solfp4::RotaryOperand &o = *both[i], &other = *both[1 - i];
    if (!o.heads) continue;
    const Region out = heads_region(type, o.out, o.out_token, o.out_head, o.heads, tokens, dim);
    if (!rotary_in_place(o, tokens) && !apart(out, heads_region(type, o.in, o.in_token, o.in_head, o.heads, tokens, dim)))
      return SOLFP4_EINVAL;
    if (other.heads &&
        (!apart(out, heads_region(type, other.in, other.in_token, other.in_head, other.heads, tokens, dim)) ||
         !apart(out, heads_region(type, other.out, other.out_token, other.out_head, other.heads, tokens, dim))))
      return SOLFP4_EINVAL;
    if ((rotated && !apart(out, block_of(table, table_rows * rotated * 4))) ||
        (positions && !apart(out, block_of(positions, tokens * position_bytes))))
      return SOLFP4_EINVAL;
  }
  a.table = table, a.table_rows = table_rows > 0 ? table_rows : 1;
  a.positions = positions, a.tokens = tokens, a.dim = (int)dim, a.rotated = (int)rotated;
  const hipError_t e = solfp4::launch_rotary(type, layout == SOLFP4_ROTARY_INTERLEAVED, inverse != 0, position_bytes,
                                             a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SOLFP4_OK : SOLFP4_EHIP;
}

int nvfp4_weight_linear(const uint16_t* x, const uint8_t* w_codes, const uint8_t* w_scales,
                        const float* w_global_scale, const uint16_t* bias, uint16_t* out, int64_t M, int64_t N,
                        int64_t K, void* stream) {
  const int rc = linear_checks(x, nullptr, false, w_codes, w_scales, w_global_scale, true, bias, out, M, N, K, 16);
  if (rc) return rc;
  return run_linear(SOLFP4_FORMAT_NVFP4, false, {x, nullptr, w_codes, w_scales, w_global_scale, bias, out, M, N, K},
                    stream);
}

int mxfp4_weight_linear(const uint16_t* x, const uint8_t* w_codes, const uint8_t* w_scales, const uint16_t* bias,
                        uint16_t* out, int64_t M, int64_t N, int64_t K, void* stream) {
  const int rc = linear_checks(x, nullptr, false, w_codes, w_scales, nullptr, false, bias, out, M, N, K, 32);
  if (rc) return rc;
  return run_linear(SOLFP4_FORMAT_MXFP4, false, {x, nullptr, w_codes, w_scales, nullptr, bias, out, M, N, K}, stream);
}

int mxfp8_linear(const uint8_t* x_codes, const uint8_t* x_scales, const uint8_t* w_codes, const uint8_t* w_scales,
                 const uint16_t* bias, uint16_t* out, int64_t M, int64_t N, int64_t K, void* stream) {
  const int rc = linear_checks(x_codes, x_scales, true, w_codes, w_scales, nullptr, false, bias, out, M, N, K, 32);
  if (rc) return rc;
  return run_linear(SOLFP4_FORMAT_MXFP4, true, {x_codes, x_scales, w_codes, w_scales, nullptr, bias, out, M, N, K},
                    stream);
}

}  // extern "C"
