// Declarations and device helpers of the dense operators (norm with int8 rows,
// 8-bit product, distillation loss).
#pragma once

#include "bmlp_internal.h"

namespace bmlp {

struct NormArgs {
  const void *x, *res, *w;
  int64_t ldx, ldr, ldq, ldh, ldy;
  int8_t *q;
  float *scale, *rstd;
  void *h, *y;
  int n, K;
  float eps, down;         // down: set by the launcher
  bool norm, w_f32;        // norm off: scale = max|x| / 127; weights are 32-bit whatever x's type
};
hipError_t launch_norm_quant(int type, const NormArgs &all, hipStream_t s);

struct NormBackArgs {
  const void *dy, *h, *w, *dh;
  int64_t lddy, ldh, lddh, lddx;
  const float *rstd;
  void *dx;
  float *dw, *part;        // part: [rows of partial sums][K]
  int n, K, parts;         // parts: set by the launcher
  bool w_f32;
};
hipError_t launch_norm_quant_backward(int type, NormBackArgs &a, hipStream_t s);
size_t norm_back_ws_bytes(int n, int K);

// 8-bit weights in the order of the matrix cores: blocks of 32 weight rows and
// 64 inputs (2048 bytes), block (j / 32) * ceil(K / 64) + k / 64, and within
// it chunk c = (k % 64) / 16 of row r = j % 32 at byte 512 c + 16 r.  A
// 32x32x32 MFMA's operand is 1 KB in running order, lane by lane; zeros stand
// past N and K.
constexpr int kPackRows = 32, kPackK = 64, kPackBytes = kPackRows * kPackK;
struct QLinearArgs {
  const int8_t *q;
  int64_t ldq, ldo;
  const float *scale, *wscale, *bias;
  const uint8_t *w;        // packed
  void *out;
  int n, N, K;
};
hipError_t launch_qlinear_pack(const int8_t *w, int64_t ldw, int N, int K, uint8_t *packed, hipStream_t s);
hipError_t launch_qlinear(int type, const QLinearArgs &all, hipStream_t s);

struct DistillArgs {
  const void *z, *t;
  int64_t ldz, lddz;
  const int32_t *idx;
  const float *lse, *weight;
  float *loss;
  void *dz;
  int n, c, k;
  float tau;
};
hipError_t launch_distill(int type, int t_type, const DistillArgs &all, hipStream_t s);

// A launch holds fewer than 2^32 threads: more rows than this take several.
constexpr int kRowsPerLaunch = 1 << 20;

// ---------------------------------------------------------------------------
// Device helpers
// ---------------------------------------------------------------------------

template <typename T, int N>
using vec_t = T __attribute__((ext_vector_type(N)));

// N values to p, which is aligned to a value only
template <typename T, int N>
__device__ __forceinline__ void store_as(T *p, const vec_t<float, N> &f) {
  const vec_t<T, N> v = __builtin_convertvector(f, vec_t<T, N>);
  __builtin_memcpy(p, &v, sizeof(v));
}

// what one wave wrote to LDS, before its other lanes read it
__device__ __forceinline__ void wave_sync_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Joins a value over the wave, the same in every lane, without LDS: pairs at
// distances 1, 2, 4 and 8 by DPP (quad permutations, half-row and row mirror: the
// lanes of a pair's halves are equal by then), 16 and 32 by lane swaps.  `op` is
// commutative.  (Shuffles through LDS take several times as long, and a row's
// work is a chain of such joins.)
template <int CTRL, typename T>
__device__ __forceinline__ T dpp(T v) {
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  u = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, CTRL, 0xF, 0xF, false);
  __builtin_memcpy(&v, &u, 4);
  return v;
}
template <int D, typename T>
__device__ __forceinline__ void swap_halves(T v, T &a, T &b) {   // D = 16 or 32
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  uint32_t x, y;
  if constexpr (D == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = r[0], y = r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    x = r[0], y = r[1];
  }
  __builtin_memcpy(&a, &x, 4);
  __builtin_memcpy(&b, &y, 4);
}
template <typename T, typename F>
__device__ __forceinline__ T wave_all(T v, F op) {
  v = op(v, dpp<0xB1>(v));
  v = op(v, dpp<0x4E>(v));
  v = op(v, dpp<0x141>(v));
  v = op(v, dpp<0x140>(v));
  T a, b;
  swap_halves<16>(v, a, b);
  v = op(a, b);
  swap_halves<32>(v, a, b);
  return op(a, b);
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_all(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_all(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  return wave_all(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}

}  // namespace bmlp
