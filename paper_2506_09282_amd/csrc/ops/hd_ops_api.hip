// C ABI of the operators behind answers and learning: argument checks on the host,
// then the launch on the caller's stream.
#include <math.h>

#include "../../../include/hd.h"
#include "hd_ops.hpp"

namespace {

constexpr int64_t kMaxDim = int64_t(1) << 30;

bool float_dt(int dt) { return dt == HD_F32 || dt == HD_BF16; }
bool known_dt(int dt) { return float_dt(dt) || dt == HD_I8; }
size_t esize(int dt) { return dt == HD_F32 ? 4 : 2; }
bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
hd_status from_hip(hipError_t e) { return e == hipSuccess ? HD_OK : HD_ERR_HIP; }

constexpr int64_t kMaxRows = 4096;  // of X in one 4-bit product

// The sizes of a 4-bit matrix: HD_OK, or what is wrong with them.
hd_status nibble_sizes(int64_t outer, int64_t inner, int64_t group) {
  if (outer < 1 || inner < 1 || (group != 32 && group != 64 && group != 128)) return HD_ERR_ARG;
  if (outer > kMaxDim || inner > kMaxDim) return HD_ERR_UNSUPPORTED;
  const hd::ops::NibbleLayout L = hd::ops::nibble_layout(outer, inner, (int)group);
  return L.otiles * L.itiles <= (int64_t(1) << 24) ? HD_OK : HD_ERR_UNSUPPORTED;
}

hd_status logprobs_args(const void* scores, int64_t ld, const uint8_t* mask, int64_t ldm,
                        const int32_t* y, float scale, int64_t N, int64_t K, int dt) {
  if (N < 0 || K < 1 || !known_dt(dt) || !(scale > 0.0f) || !isfinite(scale)) return HD_ERR_ARG;
  if (ld < K || (mask && ldm != 0 && ldm < K)) return HD_ERR_ARG;
  if (N > kMaxDim || K > kMaxDim || ld > (int64_t(1) << 40) || !float_dt(dt))
    return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if (!scores || !aligned(scores, esize(dt)) || !aligned(y, 4)) return HD_ERR_ARG;
  return HD_OK;
}

constexpr int64_t kMaxCkptRows = int64_t(65535) * hd::ops::kCkptRows;

hd_status ckpt_sizes(int64_t N, int64_t D) {
  if (N < 0 || D < 1) return HD_ERR_ARG;
  return N <= kMaxCkptRows && D <= kMaxDim ? HD_OK : HD_ERR_UNSUPPORTED;
}
hd_status ckpt_grad_sizes(int64_t N, int64_t D, int64_t K, int dt) {
  if (K < 1 || !known_dt(dt)) return HD_ERR_ARG;
  const hd_status st = ckpt_sizes(N, D);
  if (st != HD_OK) return st;
  if (K > (int64_t(1) << 20) || !float_dt(dt) ||
      hd::cdiv(N, hd::ops::kCkptRows) * hd::cdiv(K, 32) >= (int64_t(1) << 23))
    return HD_ERR_UNSUPPORTED;
  return HD_OK;
}

// Strides that the tiles of a product take (tile::kMaxStride).
constexpr int64_t kMaxStride = int64_t(1) << 22;
constexpr int64_t kMaxValues = int64_t(1) << 38;  // of a matrix that tiles cover

hd_status byte_sizes(int64_t outer, int64_t inner) {
  if (outer < 1 || inner < 1) return HD_ERR_ARG;
  if (inner > 131071 || outer > (int64_t(1) << 23) ||
      hd::cdiv(outer, 32) * hd::cdiv(inner, 128) > (int64_t(1) << 23))
    return HD_ERR_UNSUPPORTED;
  return HD_OK;
}
hd_status byte_product_sizes(int64_t N, int64_t outer, int64_t inner, int x_dt) {
  if (N < 0 || !known_dt(x_dt)) return HD_ERR_ARG;
  const hd_status st = byte_sizes(outer, inner);
  if (st != HD_OK) return st;
  return N <= (int64_t(1) << 23) && N * outer <= kMaxValues ? HD_OK : HD_ERR_UNSUPPORTED;
}

hd_status class_sizes(int64_t N, int64_t D, int64_t K, int dt) {
  if (N < 0 || D < 1 || K < 1 || !known_dt(dt)) return HD_ERR_ARG;
  constexpr int64_t kMost = int64_t(1) << 24;
  if (N > kMost || K > kMost || D > (int64_t(1) << 20) || !float_dt(dt) || N * K > kMaxValues ||
      N * D > kMaxValues || K * D > kMaxValues)
    return HD_ERR_UNSUPPORTED;
  return HD_OK;
}
hd_status class_args(const void* H, int64_t ldh, const void* C, int64_t ldc, const int32_t* y,
                     float scale, const float* stats, int64_t N, int64_t D, int64_t K, int dt) {
  const hd_status st = class_sizes(N, D, K, dt);
  // (the kernels take scale log2(e), under 2 scale)
  if (st == HD_ERR_ARG || !(scale > 0.0f) || !isfinite(2.0f * scale) || ldh < D || ldc < D)
    return HD_ERR_ARG;
  if (st != HD_OK || ldh > kMaxStride || ldc > kMaxStride) return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if (!H || !C || !y || !stats || !aligned(H, esize(dt)) || !aligned(C, esize(dt)) ||
      !aligned(y, 4) || !aligned(stats, 4))
    return HD_ERR_ARG;
  return HD_OK;
}

}  // namespace

extern "C" {

size_t hd_nibble_bytes(int64_t outer, int64_t inner, int64_t group) {
  if (nibble_sizes(outer, inner, group) != HD_OK) return 0;
  return hd::ops::nibble_layout(outer, inner, (int)group).total;
}

hd_status hd_nibble_pack(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros,
                         int64_t outer, int64_t inner, int64_t group, void* image,
                         size_t image_bytes, hipStream_t stream) {
  const hd_status st = nibble_sizes(outer, inner, group);
  if (st != HD_OK) return st;
  if (!codes || !scales || !image || !aligned(scales, 2) || !aligned(image, 256))
    return HD_ERR_ARG;
  if (image_bytes < hd_nibble_bytes(outer, inner, group)) return HD_ERR_WORKSPACE;
  return from_hip(hd::ops::launch_nibble_pack(codes, scales, zeros, outer, inner, (int)group,
                                              image, stream));
}

hd_status hd_nibble_quantize(const void* W, int64_t ldw, int inner_rows, int zeros, int64_t outer,
                             int64_t inner, int64_t group, hd_dtype dt, void* image,
                             size_t image_bytes, hipStream_t stream) {
  const hd_status st = nibble_sizes(outer, inner, group);
  if (!known_dt(dt)) return HD_ERR_ARG;
  if (st != HD_OK) return st;
  if (!float_dt(dt)) return HD_ERR_UNSUPPORTED;
  if (ldw < (inner_rows ? outer : inner) || !W || !image || !aligned(W, esize(dt)) ||
      !aligned(image, 256))
    return HD_ERR_ARG;
  if (image_bytes < hd_nibble_bytes(outer, inner, group)) return HD_ERR_WORKSPACE;
  return from_hip(hd::ops::launch_nibble_quantize(W, ldw, inner_rows != 0, outer, inner,
                                                  (int)group, zeros != 0, dt, image, stream));
}

hd_status hd_nibble_unpack(const void* image, int zeros, float* W, int64_t outer, int64_t inner,
                           int64_t group, hipStream_t stream) {
  const hd_status st = nibble_sizes(outer, inner, group);
  if (st != HD_OK) return st;
  if (!image || !W || !aligned(image, 256) || !aligned(W, 4)) return HD_ERR_ARG;
  return from_hip(
      hd::ops::launch_nibble_unpack(image, W, outer, inner, (int)group, zeros != 0, stream));
}

size_t hd_nibble_workspace_bytes(int64_t N, int64_t inner, hd_dtype x_dt) {
  if (N < 1 || N > kMaxRows || inner < 1 || inner > kMaxDim || !float_dt(x_dt)) return 0;
  return hd::ops::nibble_ws_bytes(N, inner, x_dt);
}

hd_status hd_nibble_product(const void* X, int64_t ldx, const void* image, int zeros, void* Y,
                            int64_t ldy, int64_t N, int64_t outer, int64_t inner, int64_t group,
                            hd_dtype x_dt, hd_dtype y_dt, hd_act act, void* workspace,
                            size_t workspace_bytes, hipStream_t stream) {
  const hd_status st = nibble_sizes(outer, inner, group);
  if (N < 0 || !known_dt(x_dt) || !known_dt(y_dt) ||
      (act != HD_ACT_HARDSIGN && act != HD_ACT_IDENTITY))
    return HD_ERR_ARG;
  if (st != HD_OK) return st;
  if (N > kMaxRows || !float_dt(x_dt) || !float_dt(y_dt)) return HD_ERR_UNSUPPORTED;
  if (ldx < inner || ldy < outer) return HD_ERR_ARG;
  if (N == 0) return HD_OK;
  if (!X || !image || !Y || !aligned(X, esize(x_dt)) || !aligned(Y, esize(y_dt)) ||
      !aligned(image, 256) || !aligned(workspace, 256))
    return HD_ERR_ARG;
  const size_t need = hd::ops::nibble_ws_bytes(N, inner, x_dt);
  if (need > 0 && !workspace) return HD_ERR_ARG;
  if (workspace_bytes < need) return HD_ERR_WORKSPACE;
  return from_hip(hd::ops::launch_nibble_product(X, ldx, image, Y, ldy, N, outer, inner,
                                                 (int)group, zeros != 0, x_dt, y_dt, act,
                                                 workspace, stream));
}

size_t hd_logprobs_workspace_bytes(int64_t N, int64_t K, hd_dtype dt) {
  if (N < 1 || K < 1 || N > kMaxDim || K > kMaxDim || !float_dt(dt)) return 0;
  return hd::ops::logprobs_ws_bytes(N, K, dt);
}

hd_status hd_logprobs(const void* scores, int64_t ld, const uint8_t* mask, int64_t ldm,
                      const int32_t* y, float scale, float* logp, float* entropy, float* stats,
                      int32_t* ids, float* top_logp, int64_t N, int64_t K, int64_t top,
                      hd_dtype dt, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const hd_status st = logprobs_args(scores, ld, mask, ldm, y, scale, N, K, dt);
  if (st != HD_OK) return st;
  if (top < 0) return HD_ERR_ARG;
  if (top > hd::ops::kMaxTop) return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if ((y && !logp) || !entropy || !stats || (top > 0 && (!ids || !top_logp))) return HD_ERR_ARG;
  if (!aligned(logp, 4) || !aligned(entropy, 4) || !aligned(stats, 4) || !aligned(ids, 4) ||
      !aligned(top_logp, 4) || !aligned(workspace, 256))
    return HD_ERR_ARG;
  const size_t need = hd::ops::logprobs_ws_bytes(N, K, dt);
  if (need > 0 && !workspace) return HD_ERR_ARG;
  if (workspace_bytes < need) return HD_ERR_WORKSPACE;
  const hd::ops::LogprobsArgs a{scores, ld, mask, ldm, y, scale, N, K, dt};
  return from_hip(hd::ops::launch_logprobs(a, logp, entropy, stats, ids, top_logp, (int)top,
                                           workspace, stream));
}

hd_status hd_logprobs_grad(const void* scores, int64_t ld, const uint8_t* mask, int64_t ldm,
                           const int32_t* y, float scale, const float* stats,
                           const float* entropy, const float* g_logp, const float* g_entropy,
                           void* dscores, int64_t ldd, int64_t N, int64_t K, hd_dtype dt,
                           hipStream_t stream) {
  const hd_status st = logprobs_args(scores, ld, mask, ldm, y, scale, N, K, dt);
  if (st != HD_OK) return st;
  if (ldd < K) return HD_ERR_ARG;
  if (ldd > (int64_t(1) << 40)) return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if (!stats || !entropy || !dscores || !aligned(stats, 4) || !aligned(entropy, 4) ||
      !aligned(g_logp, 4) || !aligned(g_entropy, 4) || !aligned(dscores, esize(dt)))
    return HD_ERR_ARG;
  if (dscores == scores && ldd != ld) return HD_ERR_ARG;
  const hd::ops::LogprobsArgs a{scores, ld, mask, ldm, y, scale, N, K, dt};
  return from_hip(hd::ops::launch_logprobs_grad(a, stats, entropy, g_logp, g_entropy, dscores,
                                                ldd, stream));
}

size_t hd_ckpt_bytes(int64_t N, int64_t D) {
  if (N < 1 || ckpt_sizes(N, D) != HD_OK) return 0;
  return hd::ops::ckpt_image_bytes(N, D);
}

hd_status hd_ckpt_store(const void* H, int64_t ldh, int64_t N, int64_t D, hd_dtype dt, void* image,
                        size_t image_bytes, hipStream_t stream) {
  const hd_status st = ckpt_sizes(N, D);
  if (!known_dt(dt)) return HD_ERR_ARG;
  if (st != HD_OK) return st;
  if (!float_dt(dt)) return HD_ERR_UNSUPPORTED;
  if (ldh < D) return HD_ERR_ARG;
  if (N == 0) return HD_OK;
  if (!H || !image || !aligned(H, esize(dt)) || !aligned(image, 256)) return HD_ERR_ARG;
  if (image_bytes < hd::ops::ckpt_image_bytes(N, D)) return HD_ERR_WORKSPACE;
  return from_hip(hd::ops::launch_ckpt_store(H, ldh, N, D, dt, image, stream));
}

hd_status hd_ckpt_load(const void* image, void* H, int64_t ldh, int64_t N, int64_t D, hd_dtype dt,
                       hipStream_t stream) {
  const hd_status st = ckpt_sizes(N, D);
  if (!known_dt(dt)) return HD_ERR_ARG;
  if (st != HD_OK) return st;
  if (!float_dt(dt)) return HD_ERR_UNSUPPORTED;
  if (ldh < D) return HD_ERR_ARG;
  if (N == 0) return HD_OK;
  if (!H || !image || !aligned(H, esize(dt)) || !aligned(image, 256)) return HD_ERR_ARG;
  return from_hip(hd::ops::launch_ckpt_load(image, H, ldh, N, D, dt, stream));
}

size_t hd_ckpt_class_grad_workspace_bytes(int64_t N, int64_t D, int64_t K, hd_dtype dt) {
  if (N < 1 || ckpt_grad_sizes(N, D, K, dt) != HD_OK) return 0;
  return hd::ops::ckpt_grad_ws_bytes(N, D, K, dt);
}

hd_status hd_ckpt_class_grad(const void* dS, int64_t lds, const void* image, float* dC, int64_t N,
                             int64_t D, int64_t K, hd_dtype dt, int accumulate, void* workspace,
                             size_t workspace_bytes, hipStream_t stream) {
  const hd_status st = ckpt_grad_sizes(N, D, K, dt);
  if (st != HD_OK) return st;
  if (lds < K) return HD_ERR_ARG;
  if (N == 0 && accumulate) return HD_OK;
  if (!dC || !aligned(dC, 4)) return HD_ERR_ARG;
  if (N == 0)  // an empty sum
    return from_hip(hd::launch_zero(dC, (size_t)(K * D) * 4, stream));
  if (!dS || !image || !aligned(dS, esize(dt)) || !aligned(image, 256) ||
      !aligned(workspace, 256))
    return HD_ERR_ARG;
  const size_t need = hd::ops::ckpt_grad_ws_bytes(N, D, K, dt);
  if (need > 0 && !workspace) return HD_ERR_ARG;
  if (workspace_bytes < need) return HD_ERR_WORKSPACE;
  return from_hip(hd::ops::launch_ckpt_class_grad(dS, lds, image, dC, N, D, K, dt,
                                                  accumulate != 0, workspace, stream));
}

size_t hd_byte_bytes(int64_t outer, int64_t inner) {
  return byte_sizes(outer, inner) == HD_OK ? hd::ops::byte_image_bytes(outer, inner) : 0;
}

hd_status hd_byte_pack(const int8_t* codes, const float* scales, int64_t outer, int64_t inner,
                       void* image, size_t image_bytes, hipStream_t stream) {
  const hd_status st = byte_sizes(outer, inner);
  if (st != HD_OK) return st;
  if (!codes || !scales || !image || !aligned(scales, 4) || !aligned(image, 256))
    return HD_ERR_ARG;
  if (image_bytes < hd::ops::byte_image_bytes(outer, inner)) return HD_ERR_WORKSPACE;
  return from_hip(hd::ops::launch_byte_pack(codes, scales, outer, inner, image, stream));
}

hd_status hd_byte_quantize(const void* W, int64_t ldw, int inner_rows, int64_t outer,
                           int64_t inner, hd_dtype dt, void* image, size_t image_bytes,
                           hipStream_t stream) {
  const hd_status st = byte_sizes(outer, inner);
  if (!known_dt(dt)) return HD_ERR_ARG;
  if (st != HD_OK) return st;
  if (!float_dt(dt) || ldw > (int64_t(1) << 40)) return HD_ERR_UNSUPPORTED;
  if (ldw < (inner_rows ? outer : inner) || !W || !image || !aligned(W, esize(dt)) ||
      !aligned(image, 256))
    return HD_ERR_ARG;
  if (image_bytes < hd::ops::byte_image_bytes(outer, inner)) return HD_ERR_WORKSPACE;
  return from_hip(
      hd::ops::launch_byte_quantize(W, ldw, inner_rows != 0, outer, inner, dt, image, stream));
}

hd_status hd_byte_unpack(const void* image, float* W, int64_t outer, int64_t inner,
                         hipStream_t stream) {
  const hd_status st = byte_sizes(outer, inner);
  if (st != HD_OK) return st;
  if (!image || !W || !aligned(image, 256) || !aligned(W, 4)) return HD_ERR_ARG;
  return from_hip(hd::ops::launch_byte_unpack(image, W, outer, inner, stream));
}

hd_status hd_byte_rows(const void* X, int64_t ldx, int64_t N, int64_t inner, hd_dtype dt,
                       int8_t* codes, float* scales, hipStream_t stream) {
  const hd_status st = byte_product_sizes(N, 1, inner, dt);
  if (st == HD_ERR_ARG || ldx < inner) return HD_ERR_ARG;
  if (st != HD_OK || !float_dt(dt) || ldx > (int64_t(1) << 40)) return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if (!X || !codes || !scales || !aligned(X, esize(dt)) || !aligned(scales, 4)) return HD_ERR_ARG;
  return from_hip(hd::ops::launch_byte_rows(X, ldx, N, inner, dt, codes, scales, stream));
}

size_t hd_byte_workspace_bytes(int64_t N, int64_t outer, int64_t inner, hd_dtype x_dt) {
  if (N < 1 || byte_product_sizes(N, outer, inner, x_dt) != HD_OK) return 0;
  return hd::ops::byte_ws_bytes(N, outer, inner, x_dt);
}

hd_status hd_byte_product(const void* X, int64_t ldx, const float* row_scales, const void* image,
                          void* Y, int64_t ldy, int64_t N, int64_t outer, int64_t inner,
                          hd_dtype x_dt, hd_dtype y_dt, hd_act act, void* workspace,
                          size_t workspace_bytes, hipStream_t stream) {
  const hd_status st = byte_product_sizes(N, outer, inner, x_dt);
  if (st == HD_ERR_ARG || !known_dt(y_dt) || (act != HD_ACT_HARDSIGN && act != HD_ACT_IDENTITY) ||
      ldx < inner || ldy < outer || (row_scales && x_dt != HD_I8))
    return HD_ERR_ARG;
  if (st != HD_OK || !float_dt(y_dt) || ldx > kMaxStride || ldy > (int64_t(1) << 40))
    return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if (!X || !image || !Y || (x_dt != HD_I8 && !aligned(X, esize(x_dt))) ||
      !aligned(Y, esize(y_dt)) || !aligned(row_scales, 4) || !aligned(image, 256) ||
      !aligned(workspace, 256))
    return HD_ERR_ARG;
  const size_t need = hd::ops::byte_ws_bytes(N, outer, inner, x_dt);
  if (need > 0 && !workspace) return HD_ERR_ARG;
  if (workspace_bytes < need) return HD_ERR_WORKSPACE;
  return from_hip(hd::ops::launch_byte_product(X, ldx, row_scales, image, Y, ldy, N, outer, inner,
                                               x_dt, y_dt, act, workspace, stream));
}

size_t hd_class_loss_workspace_bytes(int64_t N, int64_t D, int64_t K, hd_dtype dt) {
  if (N < 1 || class_sizes(N, D, K, dt) != HD_OK) return 0;
  return hd::ops::class_loss_ws_bytes(N, D, K);
}

hd_status hd_class_loss(const void* H, int64_t ldh, const void* C, int64_t ldc,
                        const uint8_t* mask, const int32_t* y, float scale, float* loss,
                        float* stats, int64_t N, int64_t D, int64_t K, hd_dtype dt,
                        void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const hd_status st = class_args(H, ldh, C, ldc, y, scale, stats, N, D, K, dt);
  if (st != HD_OK || N == 0) return st;
  if (!loss || !aligned(loss, 4) || !workspace || !aligned(workspace, 256)) return HD_ERR_ARG;
  if (workspace_bytes < hd::ops::class_loss_ws_bytes(N, D, K)) return HD_ERR_WORKSPACE;
  const hd::ops::ClassArgs a{H, ldh, C, ldc, mask, y, scale, N, D, K, dt};
  return from_hip(hd::ops::launch_class_loss(a, loss, stats, workspace, stream));
}

size_t hd_class_loss_grad_workspace_bytes(int64_t N, int64_t D, int64_t K, hd_dtype dt) {
  return hd_class_loss_grad_workspace_bytes_of(N, D, K, dt, 1, 1);
}
size_t hd_class_loss_grad_workspace_bytes_of(int64_t N, int64_t D, int64_t K, hd_dtype dt,
                                             int with_dH, int with_dC) {
  if (N < 1 || class_sizes(N, D, K, dt) != HD_OK || (!with_dH && !with_dC)) return 0;
  return hd::ops::class_grad_ws_bytes(N, D, K, dt, with_dH != 0, with_dC != 0);
}

hd_status hd_class_loss_grad(const void* H, int64_t ldh, const void* C, int64_t ldc,
                             const uint8_t* mask, const int32_t* y, float scale,
                             const float* stats, const float* g_loss, void* dH, void* dC,
                             int64_t N, int64_t D, int64_t K, hd_dtype dt, void* workspace,
                             size_t workspace_bytes, hipStream_t stream) {
  const hd_status st = class_args(H, ldh, C, ldc, y, scale, stats, N, D, K, dt);
  if (st != HD_OK) return st;
  if (N > 0 ? !dH && !dC : false) return HD_ERR_ARG;
  if (!aligned(dH, esize(dt)) || !aligned(dC, esize(dt))) return HD_ERR_ARG;
  if (N == 0)  // an empty sum
    return dC ? from_hip(hd::launch_zero(dC, (size_t)(K * D) * esize(dt), stream)) : HD_OK;
  if (!g_loss || !aligned(g_loss, 4) || !workspace || !aligned(workspace, 256)) return HD_ERR_ARG;
  if (workspace_bytes < hd::ops::class_grad_ws_bytes(N, D, K, dt, dH != nullptr, dC != nullptr))
    return HD_ERR_WORKSPACE;
  const hd::ops::ClassArgs a{H, ldh, C, ldc, mask, y, scale, N, D, K, dt};
  return from_hip(
      hd::ops::launch_class_loss_grad(a, stats, g_loss, dH, dC, workspace, stream));
}

hd_status hd_dropout(const void* X, int64_t ldx, void* Y, int64_t ldy, int64_t N, int64_t D,
                     double p, uint64_t seed, uint64_t step, const uint64_t* step_at, hd_dtype dt,
                     hipStream_t stream) {
  if (N < 0 || D < 1 || !known_dt(dt) || !(p >= 0.0 && p <= 1.0) || ldx < D || ldy < D)
    return HD_ERR_ARG;
  if (N > kMaxDim || D > kMaxDim || !float_dt(dt) || ldx > (int64_t(1) << 40) ||
      ldy > (int64_t(1) << 40))
    return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if (!X || !Y || !aligned(X, esize(dt)) || !aligned(Y, esize(dt)) || !aligned(step_at, 8) ||
      (X == Y && ldx != ldy))
    return HD_ERR_ARG;
  const double scale = p < 1.0 ? 1.0 / (1.0 - p) : 0.0;
  return from_hip(hd::ops::launch_dropout(X, ldx, Y, ldy, N, D, (uint64_t)llrint(p * 4294967296.0),
                                          (float)scale, seed, step, step_at, dt, stream));
}

}  // extern "C"
