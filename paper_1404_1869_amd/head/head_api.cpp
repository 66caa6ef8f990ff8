// C ABI entry points of the head's operators: argument validation, size queries and dispatch.  Every check happens on the
// host before any device work is enqueued.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "head.h"

namespace dn {
namespace head {
namespace {

// One traced launch: the launcher's HIP status mapped to a dn_status naming the step.
template <typename F>
int run_step(const char* name, void* stream, F&& launch) {
  TraceScope trace(name, stream);
  const int err = launch();
  if (err == 0) return DN_OK;
  return fail(DN_E_HIP, std::string(name) + ": " + hipGetErrorString((hipError_t)err));
}

bool valid_dtype(dn_dtype dt) { return dt == DN_F32 || dt == DN_F16 || dt == DN_BF16; }

// Rows of C elements: a pointer (where there are rows) aligned to its elements, and a stride that keeps rows apart.
int check_rows(const char* what, const void* p, int64_t stride, int64_t n, int32_t C, size_t elem) {
  if (n > 0 && !p) return fail(DN_E_INVALID_ARG, std::string(what) + ": null pointer");
  if ((uintptr_t)p % elem) return fail(DN_E_INVALID_ARG, std::string(what) + ": not aligned to its elements");
  if (n > 1 && stride < C) return fail(DN_E_INVALID_ARG, std::string(what) + ": rows overlap (stride < C)");
  if (stride > (1LL << 40)) return fail(DN_E_TOO_LARGE, std::string(what) + ": stride");
  return DN_OK;
}
size_t elem_size(dn_dtype dt) { return dt == DN_F8 ? 1 : dtype_size(dt); }

int check_work(const void* work, size_t bytes, size_t need, size_t* needed) {
  if (needed) *needed = need;
  if (!work) return DN_OK;
  if (bytes < need) return fail(DN_E_BUFFER_TOO_SMALL, "workspace too small");
  if ((uintptr_t)work % 256) return fail(DN_E_INVALID_ARG, "workspace must be aligned to 256 bytes");
  return DN_OK;
}

constexpr int64_t MAX_ROWS = (1LL << 31) - 256;
constexpr int64_t MAX_BACK_ROWS = (1LL << 30) - 256;  // twice their number is a product's k in fp32
constexpr int64_t MAX_TILES = MAX_LAUNCH_THREADS / 256;
// What a call of the 8-bit head's asks for: never 0, so that a caller's workspace is never the null pointer of a size query, and
// DN_NO_WORKSPACE exactly where nothing is written there.
size_t at_least(size_t bytes) { return bytes ? bytes + DN_NO_WORKSPACE : DN_NO_WORKSPACE; }

int check_loss(const LossArgs& a, dn_dtype dtype, bool backward) {
  if (!valid_dtype(dtype)) return fail(DN_E_UNSUPPORTED, "unknown dtype");
  if (a.n < 0 || a.C <= 0 || a.V <= 0) return fail(DN_E_INVALID_ARG, "n must be >= 0, C and V positive");
  if (a.n > MAX_ROWS || a.V > MAX_ROWS || a.C > (1 << 20)) return fail(DN_E_TOO_LARGE, "n, V or C");
  const int64_t tn = (a.n + 127) / 128, tv = (a.V + 127) / 128, tc = (a.C + 127) / 128;
  if (tn * tv > 0x7fffffffLL || tn * tc > 0x7fffffffLL || tv * tc > 0x7fffffffLL)
    return fail(DN_E_TOO_LARGE, "n times V, n times C or V times C");
  // (the forward pass goes over n in pieces, the gradient over V)
  if (backward && (a.n > MAX_BACK_ROWS || tn * tc > MAX_TILES || tv * tc > MAX_TILES))
    return fail(DN_E_TOO_LARGE, "n, n times C or V times C");
  const size_t e = dtype_size(dtype);
  int st;
  if ((st = check_rows("h", a.h, a.h_stride, a.n, a.C, e))) return st;
  if ((st = check_rows("w", a.w, a.w_stride, a.V, a.C, e))) return st;
  if (a.n > 0 && !a.label) return fail(DN_E_INVALID_ARG, "null label pointer");
  return DN_OK;
}

int64_t blocks_of(int64_t x) { return (x + DN_SCALE_BLOCK - 1) / DN_SCALE_BLOCK; }

int check_scores(const void* logits, int64_t stride, const int64_t* token, int64_t n, int32_t V, dn_dtype dtype, float scale, int32_t top) {
  if (!valid_dtype(dtype)) return fail(DN_E_UNSUPPORTED, "unknown dtype");
  if (n < 0 || V <= 0) return fail(DN_E_INVALID_ARG, "n must be >= 0 and V positive");
  if (n > MAX_ROWS || V >= MAX_ROWS) return fail(DN_E_TOO_LARGE, "n or V");
  // (times log2 e, which the exponentials take, it has to be finite too)
  if (!(scale > 0) || scale > 0x1p127f) return fail(DN_E_INVALID_ARG, "scale must be positive and at most 2^127");
  if (top < 0 || top > DN_MAX_TOP) return fail(DN_E_UNSUPPORTED, "top must be 0 .. DN_MAX_TOP");
  if ((uintptr_t)token % 8) return fail(DN_E_INVALID_ARG, "tokens: not aligned");
  return check_rows("logits", logits, stride, n, V, dtype_size(dtype));
}

}  // namespace
}  // namespace head
}  // namespace dn

using namespace dn;
using namespace dn::head;

extern "C" {

int densenet_rms_norm(const void* d_x, int64_t x_stride, const void* d_res, int64_t res_stride, const float* d_gamma, int64_t n,
                      int32_t C, dn_dtype dtype, float eps, void* d_sum, int64_t sum_stride, void* d_y, int64_t y_stride,
                      dn_dtype y_dtype, int32_t block, float* d_scale, void* stream) {
  try {
    if (!valid_dtype(dtype) || !(valid_dtype(y_dtype) || y_dtype == DN_F8)) return fail(DN_E_UNSUPPORTED, "unknown dtype");
    if (n < 0 || C <= 0) return fail(DN_E_INVALID_ARG, "n must be >= 0 and C positive");
    if (C > DN_MAX_NORM_C) return fail(DN_E_TOO_LARGE, "rows are limited to DN_MAX_NORM_C values");
    if (n > MAX_ROWS) return fail(DN_E_TOO_LARGE, "too many rows");
    if (!(eps >= 0) || std::isinf(eps)) return fail(DN_E_INVALID_ARG, "eps must be finite and >= 0");
    if (y_dtype == DN_F8) {
      if (block != 0 && block != 32 && block != 64 && block != 128)
        return fail(DN_E_UNSUPPORTED, "block must be 0, 32, 64 or 128");
      if (n > 0 && !d_scale) return fail(DN_E_INVALID_ARG, "an 8-bit output needs d_scale");
    } else if (block != 0 || d_scale) {
      return fail(DN_E_INVALID_ARG, "block and d_scale belong to an 8-bit output");
    }
    int st;
    const size_t e = dtype_size(dtype);
    if ((st = check_rows("x", d_x, x_stride, n, C, e))) return st;
    if (d_res && (st = check_rows("residual", d_res, res_stride, n, C, e))) return st;
    if (d_sum && (st = check_rows("sum", d_sum, sum_stride, n, C, e))) return st;
    if ((st = check_rows("y", d_y, y_stride, n, C, elem_size(y_dtype)))) return st;
    if ((uintptr_t)d_gamma % 4 || (uintptr_t)d_scale % 4) return fail(DN_E_INVALID_ARG, "gamma or scale: not aligned");
    if (n == 0) return DN_OK;
    NormArgs a{d_x, d_res, d_gamma, d_sum, d_y, d_scale, x_stride, res_stride, sum_stride, y_stride, n, C, block, eps};
    return run_step("rms_norm", stream, [&] { return launch_rms_norm(a, dtype, y_dtype, stream); });
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

int densenet_rms_norm_backward(const void* d_dy, int64_t dy_stride, dn_dtype dy_dtype, const void* d_sum, int64_t sum_stride,
                               const void* d_dsum, int64_t dsum_stride, const float* d_gamma, int64_t n, int32_t C,
                               dn_dtype dtype, float eps, void* d_dx, int64_t dx_stride, float* d_dgamma, void* d_workspace,
                               size_t workspace_bytes, size_t* bytes_needed, void* stream) {
  try {
    if (!valid_dtype(dtype) || !valid_dtype(dy_dtype)) return fail(DN_E_UNSUPPORTED, "unknown dtype");
    if (n < 0 || C <= 0) return fail(DN_E_INVALID_ARG, "n must be >= 0 and C positive");
    if (C > DN_MAX_NORM_C) return fail(DN_E_TOO_LARGE, "rows are limited to DN_MAX_NORM_C values");
    if (n > MAX_ROWS) return fail(DN_E_TOO_LARGE, "too many rows");
    if (!(eps >= 0) || std::isinf(eps)) return fail(DN_E_INVALID_ARG, "eps must be finite and >= 0");
    const int32_t groups = norm_back_groups(n, C);
    // (never 0, so that a caller's workspace is never the null pointer of a size query: without rows, dgamma is still to be written)
    const size_t need = 4 * (size_t)std::max(groups, 1) * C;
    int st;
    if ((st = check_work(d_workspace, workspace_bytes, need, bytes_needed)) || !d_workspace) return st;
    const size_t e = dtype_size(dtype);
    if ((st = check_rows("dy", d_dy, dy_stride, n, C, dtype_size(dy_dtype)))) return st;
    if ((st = check_rows("sum", d_sum, sum_stride, n, C, e))) return st;
    if (d_dsum && (st = check_rows("dsum", d_dsum, dsum_stride, n, C, e))) return st;
    if ((st = check_rows("dx", d_dx, dx_stride, n, C, e))) return st;
    if ((uintptr_t)d_gamma % 4 || (uintptr_t)d_dgamma % 4) return fail(DN_E_INVALID_ARG, "gamma: not aligned");
    if (n == 0 && !d_dgamma) return DN_OK;
    NormBackArgs a{d_dy,      d_sum,      d_dsum,      d_gamma,   d_dx, d_dgamma, (float*)d_workspace,
                   dy_stride, sum_stride, dsum_stride, dx_stride, n,    C,        groups,
                   eps};
    return run_step("rms_norm_backward", stream, [&] { return launch_rms_norm_backward(a, dtype, dy_dtype, stream); });
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

int densenet_softmax_loss(const void* d_h, int64_t h_stride, const void* d_w, int64_t w_stride, const int64_t* d_label, int64_t n,
                          int32_t C, int32_t V, dn_dtype dtype, float* d_loss, float* d_lse, void* d_workspace,
                          size_t workspace_bytes, size_t* bytes_needed, void* stream) {
  try {
    LossArgs a{};
    a.h = d_h, a.w = d_w, a.label = d_label, a.h_stride = h_stride, a.w_stride = w_stride;
    a.n = n, a.C = C, a.V = V, a.loss = d_loss, a.lse = d_lse;
    int st;
    if ((st = check_loss(a, dtype, false))) return st;
    const size_t need = n ? softmax_loss_bytes(a, dtype) : 0;
    if ((st = check_work(d_workspace, workspace_bytes, need, bytes_needed)) || !d_workspace) return st;
    if (n == 0) return DN_OK;
    if (!d_loss || !d_lse) return fail(DN_E_INVALID_ARG, "null output pointer");
    return run_step("softmax_loss", stream, [&] { return launch_softmax_loss(a, dtype, d_workspace, stream); });
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

int densenet_softmax_loss_backward(const void* d_h, int64_t h_stride, const void* d_w, int64_t w_stride, const int64_t* d_label,
                                   const float* d_lse, const float* d_dloss, float scale, int64_t n, int32_t C, int32_t V,
                                   dn_dtype dtype, void* d_dh, int64_t dh_stride, void* d_dw, int64_t dw_stride,
                                   void* d_workspace, size_t workspace_bytes, size_t* bytes_needed, void* stream) {
  try {
    LossArgs a{};
    a.h = d_h, a.w = d_w, a.label = d_label, a.h_stride = h_stride, a.w_stride = w_stride;
    a.n = n, a.C = C, a.V = V, a.lse_in = d_lse, a.dloss = d_dloss, a.scale = scale;
    a.dh = d_dh, a.dw = d_dw, a.dh_stride = dh_stride, a.dw_stride = dw_stride;
    int st;
    if ((st = check_loss(a, dtype, true))) return st;
    const size_t need = softmax_loss_backward_bytes(a, dtype);
    if ((st = check_work(d_workspace, workspace_bytes, need, bytes_needed)) || !d_workspace) return st;
    const size_t e = dtype_size(dtype);
    if ((st = check_rows("dh", d_dh, dh_stride, n, C, e))) return st;
    if ((st = check_rows("dw", d_dw, dw_stride, V, C, e))) return st;
    if (n > 0 && !d_lse) return fail(DN_E_INVALID_ARG, "null lse pointer");
    return run_step("softmax_loss_backward", stream,
                    [&] { return launch_softmax_loss_backward(a, dtype, d_workspace, stream); });
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

int densenet_adamw(const dn_adamw_tensor* tensors, int32_t count, dn_dtype p_dtype, dn_dtype g_dtype, dn_dtype copy_dtype,
                   const dn_adamw_params* params, void* d_m, void* d_v, float* d_m_scale, float* d_v_scale, int64_t n_blocks,
                   void* stream) {
  try {
    if (!params || count < 0 || (count > 0 && !tensors)) return fail(DN_E_INVALID_ARG, "null table or parameters");
    const dn_adamw_params& k = *params;
    if (!valid_dtype(p_dtype) || !valid_dtype(g_dtype)) return fail(DN_E_UNSUPPORTED, "unknown dtype");
    if (copy_dtype != DN_F16 && copy_dtype != DN_BF16) return fail(DN_E_UNSUPPORTED, "copies are DN_F16 or DN_BF16");
    if (k.state_bits != 8 && k.state_bits != 32) return fail(DN_E_UNSUPPORTED, "state_bits must be 8 or 32");
    if (!(k.beta1 >= 0 && k.beta1 < 1 && k.beta2 >= 0 && k.beta2 < 1)) return fail(DN_E_INVALID_ARG, "betas must be in [0, 1)");
    if (!(k.eps > 0) || k.step < 1) return fail(DN_E_INVALID_ARG, "eps must be positive, step at least 1");
    if (!std::isfinite(k.lr) || !std::isfinite(k.weight_decay) || !std::isfinite(k.grad_scale) || !std::isfinite(k.eps))
      return fail(DN_E_INVALID_ARG, "parameters must be finite");
    if (n_blocks < 0 || n_blocks > (1LL << 40)) return fail(DN_E_INVALID_ARG, "bad n_blocks");
    if (n_blocks > 0 && (!d_m || !d_v)) return fail(DN_E_INVALID_ARG, "null state pointer");
    if ((uintptr_t)d_m % 16 || (uintptr_t)d_v % 16) return fail(DN_E_INVALID_ARG, "states must be aligned to 16 bytes");
    if (k.state_bits == 8 && n_blocks > 0 && (!d_m_scale || !d_v_scale))
      return fail(DN_E_INVALID_ARG, "8-bit states need their scales");
    for (int32_t i = 0; i < count; ++i) {
      const dn_adamw_tensor& t = tensors[i];
      if (t.n < 0) return fail(DN_E_INVALID_ARG, "a tensor's n must be >= 0");
      if (t.n == 0) continue;
      if (!t.p || !t.g) return fail(DN_E_INVALID_ARG, "null tensor pointer");
      if ((uintptr_t)t.p % dtype_size(p_dtype) || (uintptr_t)t.g % dtype_size(g_dtype) || (uintptr_t)t.copy % 2)
        return fail(DN_E_INVALID_ARG, "a tensor is not aligned to its elements");
      if (t.block < 0 || t.n > n_blocks * ADAMW_BLOCK || t.block > n_blocks - (t.n + ADAMW_BLOCK - 1) / ADAMW_BLOCK)
        return fail(DN_E_INVALID_ARG, "a tensor's states lie outside the blocks");
    }
    AdamWArgs a{};
    a.seed = k.seed, a.m = d_m, a.v = d_v, a.m_scale = d_m_scale, a.v_scale = d_v_scale;
    a.beta1 = (float)k.beta1, a.beta2 = (float)k.beta2;
    a.one_beta1 = (float)(1 - k.beta1), a.one_beta2 = (float)(1 - k.beta2);
    a.rate = (float)(k.lr / (1 - std::pow(k.beta1, (double)k.step)));
    a.root = (float)(1 / std::sqrt(1 - std::pow(k.beta2, (double)k.step)));
    a.eps = (float)k.eps, a.decay = (float)(1 - k.lr * k.weight_decay), a.grad_scale = (float)k.grad_scale;
    if (!(a.eps > 0)) return fail(DN_E_INVALID_ARG, "eps is below fp32's range");
    int64_t groups = 0;
    const auto flush = [&]() -> int {
      if (!a.count) return DN_OK;
      const int st = run_step("adamw", stream,
                              [&] { return launch_adamw(a, groups, p_dtype, g_dtype, copy_dtype, k.state_bits, stream); });
      a.count = 0, groups = 0;
      return st;
    };
    for (int32_t i = 0; i < count; ++i) {
      const dn_adamw_tensor& t = tensors[i];
      // a tensor of more workgroups than a launch can have goes in several parts, at whole tiles
      constexpr int64_t most = MAX_LAUNCH_THREADS / 256;
      for (int64_t at = 0; at < t.n;) {
        const int64_t n = std::min<int64_t>(t.n - at, most * ADAMW_TILE), own = (n + ADAMW_TILE - 1) / ADAMW_TILE;
        if (a.count == ADAMW_TENSORS || groups + own > most) {
          const int st = flush();
          if (st) return st;
        }
        a.t[a.count++] = AdamWTensor{(char*)t.p + at * (int64_t)dtype_size(p_dtype), (const char*)t.g + at * (int64_t)dtype_size(g_dtype),
                                     t.copy ? (char*)t.copy + at * 2 : nullptr, n, t.block * ADAMW_BLOCK + at, groups};
        groups += own;
        at += n;
      }
    }
    return flush();
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

int densenet_quantize_blocks(const void* d_x, int64_t x_stride, int64_t n, int32_t C, dn_dtype dtype, int32_t rows, void* d_codes,
                             int64_t codes_stride, float* d_scale, void* d_turned, int64_t turned_stride, float* d_turned_scale,
                             void* stream) {
  try {
    if (!valid_dtype(dtype)) return fail(DN_E_UNSUPPORTED, "unknown dtype");
    if (rows != 1 && rows != DN_SCALE_BLOCK) return fail(DN_E_UNSUPPORTED, "rows must be 1 or DN_SCALE_BLOCK");
    if (n < 0 || C <= 0) return fail(DN_E_INVALID_ARG, "n must be >= 0 and C positive");
    if (n > MAX_ROWS) return fail(DN_E_TOO_LARGE, "too many rows");
    const int64_t tiles = blocks_of(n) * blocks_of(C);
    if (tiles > MAX_TILES) return fail(DN_E_TOO_LARGE, "n times C");
    if (!d_codes && !d_turned) return n ? fail(DN_E_INVALID_ARG, "no output asked for") : DN_OK;
    if (!d_codes != !d_scale || !d_turned != !d_turned_scale) return fail(DN_E_INVALID_ARG, "codes and their scales belong together");
    int st;
    if ((st = check_rows("x", d_x, x_stride, n, C, dtype_size(dtype)))) return st;
    if (d_codes && (st = check_rows("codes", d_codes, codes_stride, n, C, 1))) return st;
    // (turned rows are n long, which is within 31 bits)
    if (d_turned && (st = check_rows("turned", d_turned, turned_stride, C, (int32_t)n, 1))) return st;
    if ((uintptr_t)d_scale % 4 || (uintptr_t)d_turned_scale % 4) return fail(DN_E_INVALID_ARG, "scale: not aligned");
    if (n == 0) return DN_OK;
    QuantArgs a{d_x,      x_stride, n, C, rows, (uint8_t*)d_codes, (uint8_t*)d_turned, codes_stride, turned_stride, d_scale,
                d_turned_scale};
    return run_step("quantize_blocks", stream, [&] { return launch_quantize_blocks(a, dtype, stream); });
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

int densenet_block_product(const void* d_a, int64_t a_stride, const float* d_a_scale, const void* d_w, int64_t w_stride,
                           const float* d_w_scale, int64_t n, int32_t C, int32_t V, void* d_y, int64_t y_stride, dn_dtype y_dtype,
                           void* d_workspace, size_t workspace_bytes, size_t* bytes_needed, void* stream) {
  try {
    if (!valid_dtype(y_dtype)) return fail(DN_E_UNSUPPORTED, "unknown dtype");
    if (n < 0 || C <= 0 || V <= 0) return fail(DN_E_INVALID_ARG, "n must be >= 0, C and V positive");
    if (n > MAX_ROWS || V > MAX_ROWS || C > (1 << 20)) return fail(DN_E_TOO_LARGE, "n, V or C");
    if (blocks_of(n) * blocks_of(V) > MAX_TILES) return fail(DN_E_TOO_LARGE, "n times V");
    ProductArgs a{(const uint8_t*)d_a, (const uint8_t*)d_w, d_a_scale, d_w_scale, a_stride, w_stride, n, C, V, d_y, y_stride};
    int st;
    if ((st = check_rows("a", d_a, a_stride, n, C, 1))) return st;
    if ((st = check_rows("w", d_w, w_stride, V, C, 1))) return st;
    const size_t need = at_least(n ? block_product_bytes(a, y_dtype) : 0);
    if ((st = check_work(d_workspace, workspace_bytes, need, bytes_needed)) || !d_workspace) return st;
    if (n == 0) return DN_OK;
    if (!d_a_scale || !d_w_scale) return fail(DN_E_INVALID_ARG, "null scale pointer");
    if ((uintptr_t)d_a_scale % 4 || (uintptr_t)d_w_scale % 4) return fail(DN_E_INVALID_ARG, "scale: not aligned");
    if ((st = check_rows("y", d_y, y_stride, n, V, dtype_size(y_dtype)))) return st;
    return run_step("block_product", stream, [&] { return launch_block_product(a, y_dtype, d_workspace, stream); });
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

int densenet_token_scores(const void* d_logits, int64_t stride, const int64_t* d_token, int64_t n, int32_t V, dn_dtype dtype,
                          float scale, int32_t top, float* d_logp, float* d_entropy, float* d_lse, int64_t* d_top_id,
                          float* d_top_logp, void* d_workspace, size_t workspace_bytes, size_t* bytes_needed, void* stream) {
  try {
    int st;
    if ((st = check_scores(d_logits, stride, d_token, n, V, dtype, scale, top))) return st;
    const size_t need = at_least(scores_bytes(n, V, top));
    if ((st = check_work(d_workspace, workspace_bytes, need, bytes_needed)) || !d_workspace) return st;
    if (n == 0) return DN_OK;
    if (!d_lse) return fail(DN_E_INVALID_ARG, "null lse pointer");
    if (top > 0 && (!d_top_id || !d_top_logp)) return fail(DN_E_INVALID_ARG, "alternatives need d_top_id and d_top_logp");
    if ((uintptr_t)d_logp % 4 || (uintptr_t)d_entropy % 4 || (uintptr_t)d_lse % 4 || (uintptr_t)d_top_logp % 4 ||
        (uintptr_t)d_top_id % 8)
      return fail(DN_E_INVALID_ARG, "an output is not aligned to its elements");
    ScoresArgs a{d_logits, d_token, stride,    n,     V,        top,        scores_parts(n, V, top), scale,
                 d_logp,   d_entropy, d_lse, d_top_id, d_top_logp, d_workspace};
    return run_step("token_scores", stream, [&] { return launch_token_scores(a, dtype, stream); });
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

int densenet_token_scores_backward(const void* d_logits, int64_t stride, const int64_t* d_token, const float* d_lse,
                                   const float* d_entropy, const float* d_dlogp, const float* d_dentropy, const float* d_dlse,
                                   const int64_t* d_top_id, const float* d_dtop, int64_t n, int32_t V, dn_dtype dtype, float scale,
                                   int32_t top, void* d_dlogits, int64_t dlogits_stride, void* stream) {
  try {
    int st;
    if ((st = check_scores(d_logits, stride, d_token, n, V, dtype, scale, top))) return st;
    if ((st = check_rows("dlogits", d_dlogits, dlogits_stride, n, V, dtype_size(dtype)))) return st;
    if (d_dlogits == d_logits && n > 1 && dlogits_stride != stride)
      return fail(DN_E_INVALID_ARG, "dlogits in the logits' own memory: with their stride");
    if (n == 0) return DN_OK;
    if (!d_lse) return fail(DN_E_INVALID_ARG, "null lse pointer");
    if (d_dentropy && !d_entropy) return fail(DN_E_INVALID_ARG, "dentropy needs the entropy");
    if (d_dlogp && !d_token) return fail(DN_E_INVALID_ARG, "dlogp needs the tokens");
    if (top > 0 && d_dtop && !d_top_id) return fail(DN_E_INVALID_ARG, "dtop needs the ids");
    for (const void* p : {(const void*)d_lse, (const void*)d_entropy, (const void*)d_dlogp, (const void*)d_dentropy,
                          (const void*)d_dlse, (const void*)d_dtop})
      if ((uintptr_t)p % 4) return fail(DN_E_INVALID_ARG, "a vector is not aligned to its elements");
    if ((uintptr_t)d_top_id % 8) return fail(DN_E_INVALID_ARG, "ids: not aligned");
    ScoresBackArgs a{d_logits, d_token,   d_top_id, d_lse, d_entropy, d_dlogp, d_dentropy, d_dlse, top > 0 ? d_dtop : nullptr,
                     d_dlogits, stride, dlogits_stride, n, V, top, 1, scale};
    return run_step("token_scores_backward", stream, [&] { return launch_token_scores_backward(a, dtype, stream); });
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

int densenet_muon(const dn_muon_tensor* tensors, int32_t count, dn_dtype p_dtype, dn_dtype g_dtype, dn_dtype copy_dtype,
                  const dn_muon_params* params, void* d_workspace, size_t workspace_bytes, size_t* bytes_needed, void* stream) {
  try {
    if (!params || count < 0 || (count > 0 && !tensors)) return fail(DN_E_INVALID_ARG, "null table or parameters");
    const dn_muon_params& k = *params;
    if (!valid_dtype(p_dtype) || !valid_dtype(g_dtype)) return fail(DN_E_UNSUPPORTED, "unknown dtype");
    if (copy_dtype != DN_F16 && copy_dtype != DN_BF16) return fail(DN_E_UNSUPPORTED, "copies are DN_F16 or DN_BF16");
    if (k.steps < 1 || k.steps > DN_MAX_NS_STEPS) return fail(DN_E_UNSUPPORTED, "steps must be 1 .. DN_MAX_NS_STEPS");
    if (k.parts < 0 || k.parts > 2) return fail(DN_E_UNSUPPORTED, "parts must be 0, 1 or 2");
    if (!(k.momentum >= 0 && k.momentum < 1)) return fail(DN_E_INVALID_ARG, "momentum must be in [0, 1)");
    // (2^13 / eps, which an update of zeros is multiplied by, has to be finite)
    if (!(k.eps >= 1e-30) || !std::isfinite((float)k.eps)) return fail(DN_E_INVALID_ARG, "eps must be 1e-30 or more, and finite in fp32");
    // (in fp32, which the step is computed in)
    const auto finite = [](double v) { return std::isfinite((float)v); };
    if (!finite(k.lr) || !finite(k.weight_decay) || !finite(k.grad_scale) || !finite(1 - k.lr * k.weight_decay))
      return fail(DN_E_INVALID_ARG, "parameters must be finite in fp32");
    for (int32_t s = 0; s < k.steps; ++s) {
      const double* c = k.coefficients[s];
      if (!(std::fabs(c[0]) <= 64) || !(std::fabs(c[1]) <= 64) || !(std::fabs(c[2]) <= 64))
        return fail(DN_E_INVALID_ARG, "coefficients must be in [-64, 64]");
    }
    int64_t tiles = 0;
    for (int32_t i = 0; i < count; ++i) {
      const dn_muon_tensor& t = tensors[i];
      if (t.rows <= 0 || t.cols <= 0) return fail(DN_E_INVALID_ARG, "a matrix's rows and cols must be positive");
      // (256 rows of the larger side in fp16 are within the 31 bits of a buffer's offsets)
      if (t.rows > (1 << 21) || t.cols > (1 << 21) || std::min(t.rows, t.cols) > (1 << 15))
        return fail(DN_E_TOO_LARGE, "a matrix's rows or cols");
      if (!finite(t.rate) || !finite(k.lr * t.rate)) return fail(DN_E_INVALID_ARG, "a matrix's rate, and lr times it, must be finite in fp32");
      // (more workgroups than any launch has for it: pieces of 2048 values, and twice the tiles of 64 x 64 of its smaller side)
      tiles += (t.rows * t.cols + 2047) / 2048 + ((std::min(t.rows, t.cols) + 63) / 64) * ((std::min(t.rows, t.cols) + 127) / 64) + 16384;
    }
    if (tiles > MAX_TILES) return fail(DN_E_TOO_LARGE, "the matrices of a call");
    int st;
    const size_t need = muon_bytes(tensors, count, p_dtype, k);
    if ((st = check_work(d_workspace, workspace_bytes, need, bytes_needed)) || !d_workspace) return st;
    for (int32_t i = 0; i < count; ++i) {
      const dn_muon_tensor& t = tensors[i];
      if (!t.p || !t.g) return fail(DN_E_INVALID_ARG, "null tensor pointer");
      if (!t.m && k.momentum != 0) return fail(DN_E_INVALID_ARG, "momentum needs its state");
      if ((uintptr_t)t.p % dtype_size(p_dtype) || (uintptr_t)t.g % dtype_size(g_dtype) || (uintptr_t)t.copy % 2 || (uintptr_t)t.m % 4)
        return fail(DN_E_INVALID_ARG, "a tensor is not aligned to its elements");
    }
    if (count == 0) return DN_OK;
    return run_step("muon", stream, [&] { return launch_muon(tensors, count, p_dtype, g_dtype, copy_dtype, k, d_workspace, stream); });
  } catch (...) {
    return fail(DN_E_INTERNAL, "unexpected exception");
  }
}

}  // extern "C"
