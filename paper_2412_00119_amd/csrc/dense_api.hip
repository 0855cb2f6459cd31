// C entries of the dense operators: argument checks, then one launcher each.
#include <math.h>

#include "dense.h"

using namespace bmlp;

namespace {

bool type_ok(int32_t t) { return t == BMLP_TYPE_F32 || t == BMLP_TYPE_BF16 || t == BMLP_TYPE_F16; }
int type_size(int32_t t) { return t == BMLP_TYPE_F32 ? 4 : 2; }

// a matrix of n rows: its base aligned to an element, its rows apart
bool rows_ok(const void *p, int64_t ld, int32_t n, int32_t cols, int size) {
  return p != nullptr && reinterpret_cast<uintptr_t>(p) % size == 0 && (n <= 1 || ld >= cols);
}
bool rows_ok_or_null(const void *p, int64_t ld, int32_t n, int32_t cols, int size) {
  return p == nullptr || rows_ok(p, ld, n, cols, size);
}
bool f32_ok(const void *p) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % 4 == 0; }
bool f32_ok_or_null(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }
hipStream_t stream_of(void *s) { return static_cast<hipStream_t>(s); }

}  // namespace

extern "C" {

int bmlp_norm_quant(int32_t type, int32_t n, int32_t K, const void *d_x, int64_t ldx, const void *d_res,
                    int64_t ldr, const void *d_weight, int32_t weight_type, float eps, int8_t *d_q, int64_t ldq,
                    float *d_scale, float *d_rstd, void *d_h, int64_t ldh, void *d_y, int64_t ldy, void *stream) {
  if (!type_ok(type) || !(eps >= 0.f) || !isfinite(eps)) return BMLP_EINVAL;
  if (d_weight != nullptr && weight_type != type && weight_type != BMLP_TYPE_F32) return BMLP_EINVAL;
  if (n < 0 || K < 1 || K > BMLP_MAX_NORM_WIDTH) return BMLP_ESHAPE;
  if (n == 0) return BMLP_OK;
  const int sz = type_size(type);
  if (!rows_ok(d_x, ldx, n, K, sz) || !rows_ok_or_null(d_res, ldr, n, K, sz) || !rows_ok(d_q, ldq, n, K, 1) ||
      !rows_ok_or_null(d_h, ldh, n, K, sz) || !rows_ok_or_null(d_y, ldy, n, K, sz) || !f32_ok(d_scale) ||
      !f32_ok_or_null(d_rstd) || reinterpret_cast<uintptr_t>(d_weight) % type_size(weight_type) != 0)
    return BMLP_EINVAL;
  NormArgs a{};
  a.x = d_x; a.res = d_res; a.w = d_weight;
  a.ldx = ldx; a.ldr = ldr; a.ldq = ldq; a.ldh = ldh; a.ldy = ldy;
  a.q = d_q; a.scale = d_scale; a.rstd = d_rstd; a.h = d_h; a.y = d_y;
  a.n = n; a.K = K; a.eps = eps; a.norm = true; a.w_f32 = weight_type == BMLP_TYPE_F32;
  BMLP_LAUNCH(launch_norm_quant(type, a, stream_of(stream)));
  return BMLP_OK;
}

int bmlp_quantize_rows(int32_t type, int32_t n, int32_t K, const void *d_x, int64_t ldx, int8_t *d_q, int64_t ldq,
                       float *d_scale, void *stream) {
  if (!type_ok(type)) return BMLP_EINVAL;
  if (n < 0 || K < 1 || K > BMLP_MAX_NORM_WIDTH) return BMLP_ESHAPE;
  if (n == 0) return BMLP_OK;
  if (!rows_ok(d_x, ldx, n, K, type_size(type)) || !rows_ok(d_q, ldq, n, K, 1) || !f32_ok(d_scale))
    return BMLP_EINVAL;
  NormArgs a{};
  a.x = d_x; a.ldx = ldx; a.q = d_q; a.ldq = ldq; a.scale = d_scale; a.n = n; a.K = K;
  BMLP_LAUNCH(launch_norm_quant(type, a, stream_of(stream)));
  return BMLP_OK;
}

size_t bmlp_norm_quant_backward_workspace_bytes(int32_t n, int32_t K) {
  return n < 1 || K < 1 || K > BMLP_MAX_NORM_WIDTH ? 0 : norm_back_ws_bytes(n, K);
}

int bmlp_norm_quant_backward(int32_t type, int32_t n, int32_t K, const void *d_dy, int64_t lddy, const void *d_h,
                             int64_t ldh, const float *d_rstd, const void *d_weight, int32_t weight_type,
                             const void *d_dh, int64_t lddh, void *d_dx, int64_t lddx, float *d_dweight, void *d_ws,
                             size_t ws_bytes, void *stream) {
  if (!type_ok(type)) return BMLP_EINVAL;
  if (d_weight != nullptr && weight_type != type && weight_type != BMLP_TYPE_F32) return BMLP_EINVAL;
  if (n < 0 || K < 1 || K > BMLP_MAX_NORM_WIDTH) return BMLP_ESHAPE;
  if (!f32_ok_or_null(d_dweight)) return BMLP_EINVAL;
  if (n == 0) {
    if (d_dweight != nullptr)
      BMLP_LAUNCH(launch_fill_i32(reinterpret_cast<int32_t *>(d_dweight), K, 0, stream_of(stream)));
    return BMLP_OK;
  }
  const int sz = type_size(type);
  if (!rows_ok(d_dy, lddy, n, K, sz) || !rows_ok(d_h, ldh, n, K, sz) || !rows_ok_or_null(d_dh, lddh, n, K, sz) ||
      !rows_ok(d_dx, lddx, n, K, sz) || !f32_ok(d_rstd) ||
      reinterpret_cast<uintptr_t>(d_weight) % type_size(weight_type) != 0)
    return BMLP_EINVAL;
  if (d_dweight != nullptr &&
      (d_ws == nullptr || ws_bytes < norm_back_ws_bytes(n, K) || (reinterpret_cast<uintptr_t>(d_ws) & 15)))
    return BMLP_EINVAL;
  NormBackArgs a{};
  a.dy = d_dy; a.h = d_h; a.w = d_weight; a.dh = d_dh;
  a.lddy = lddy; a.ldh = ldh; a.lddh = lddh; a.lddx = lddx;
  a.rstd = d_rstd; a.dx = d_dx; a.dw = d_dweight; a.part = static_cast<float *>(d_ws);
  a.n = n; a.K = K; a.w_f32 = weight_type == BMLP_TYPE_F32;
  BMLP_LAUNCH(launch_norm_quant_backward(type, a, stream_of(stream)));
  return BMLP_OK;
}

size_t bmlp_qlinear_packed_bytes(int32_t N, int32_t K) {
  if (N < 1 || K < 1 || K > BMLP_MAX_LINEAR_INPUTS || (int64_t)N * K > ((int64_t)1 << 40)) return 0;
  return (size_t)((N - 1) / kPackRows + 1) * (size_t)((K - 1) / kPackK + 1) * kPackBytes;
}

int bmlp_qlinear_pack(const int8_t *d_w, int64_t ldw, int32_t N, int32_t K, void *d_packed, void *stream) {
  if (bmlp_qlinear_packed_bytes(N, K) == 0) return BMLP_ESHAPE;
  if (!rows_ok(d_w, ldw, N, K, 1) || d_packed == nullptr || (reinterpret_cast<uintptr_t>(d_packed) & 15))
    return BMLP_EINVAL;
  BMLP_LAUNCH(launch_qlinear_pack(d_w, ldw, N, K, static_cast<uint8_t *>(d_packed), stream_of(stream)));
  return BMLP_OK;
}

int bmlp_qlinear(int32_t type, int32_t n, int32_t N, int32_t K, const int8_t *d_q, int64_t ldq, const float *d_scale,
                 const void *d_packed, const float *d_wscale, const float *d_bias, void *d_out, int64_t ldo,
                 void *stream) {
  if (!type_ok(type)) return BMLP_EINVAL;
  if (n < 0 || bmlp_qlinear_packed_bytes(N, K) == 0) return BMLP_ESHAPE;
  if (n == 0) return BMLP_OK;
  if (!rows_ok(d_q, ldq, n, K, 1) || !f32_ok_or_null(d_scale) || d_packed == nullptr ||
      (reinterpret_cast<uintptr_t>(d_packed) & 15) || !f32_ok(d_wscale) || !f32_ok_or_null(d_bias) ||
      !rows_ok(d_out, ldo, n, N, type_size(type)))
    return BMLP_EINVAL;
  QLinearArgs a{};
  a.q = d_q; a.ldq = ldq; a.ldo = ldo; a.scale = d_scale; a.wscale = d_wscale; a.bias = d_bias;
  a.w = static_cast<const uint8_t *>(d_packed); a.out = d_out; a.n = n; a.N = N; a.K = K;
  BMLP_LAUNCH(launch_qlinear(type, a, stream_of(stream)));
  return BMLP_OK;
}

int bmlp_distill(int32_t type, int32_t n, int32_t c, const void *d_z, int64_t ldz, int32_t k, const int32_t *d_idx,
                 const void *d_t, int32_t t_type, const float *d_lse, const float *d_weight, float tau, float *d_loss,
                 void *d_dz, int64_t lddz, void *stream) {
  // the kernel multiplies by log2(e) / tau
  if (!type_ok(type) || !type_ok(t_type) || !(tau > 0.f) || !isfinite(tau) || !isfinite(1.44269504f / tau)) return BMLP_EINVAL;
  if (n < 0 || c < 2 || c > BMLP_MAX_DISTILL_CLASSES || k < 1 || k > BMLP_MAX_DISTILL_LISTED) return BMLP_ESHAPE;
  if (n == 0) return BMLP_OK;
  if (!rows_ok(d_z, ldz, n, c, type_size(type)) || !f32_ok(d_idx) || !rows_ok(d_t, k, n, k, type_size(t_type)) ||
      !f32_ok_or_null(d_lse) || !f32_ok_or_null(d_weight) || !f32_ok(d_loss) ||
      !rows_ok_or_null(d_dz, lddz, n, c, type_size(type)))
    return BMLP_EINVAL;
  DistillArgs a{};
  a.z = d_z; a.t = d_t; a.ldz = ldz; a.lddz = lddz; a.idx = d_idx; a.lse = d_lse; a.weight = d_weight;
  a.loss = d_loss; a.dz = d_dz; a.n = n; a.c = c; a.k = k; a.tau = tau;
  BMLP_LAUNCH(launch_distill(type, t_type, a, stream_of(stream)));
  return BMLP_OK;
}

}  // extern "C"
