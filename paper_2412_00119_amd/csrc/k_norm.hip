// Root-mean-square norm with the residual's addition and int8 rows with a
// scale each, its gradient, and the plain row quantisation.
//
// Forward.  With h = x + r and t = h w, the int8 row is round(t 127 / max|t|):
// the norm's factor 1 / rms multiplies every t alike and cancels, and only
// enters the scale.  So one pass over a row yields both statistics, the sum of
// h^2 and the largest |t|, a single exchange between its waves joins them, and
// what follows needs t alone, which stays in registers: every input is read
// once and every output written once.  |t| is compared as its bits, an order in
// which NaN and infinity come last and so are not lost.  8192 x 4096 bf16 with
// residual and values (302 MB): 55 us a pass among others, 5.5 TB/s, where a large
// copy reaches 4.9.  Rows above 32768 spill: 2048 x 32768 bf16 123 us, but 1024 x
// 40000 1046 and 1024 x 65536 1076 (f16 867, f32 273).
//
// Backward.  dx needs one sum per row, of g h with g = dy w; dweight needs one
// sum per column over all rows.  A work-group keeps its columns' sums in
// registers over the rows it walks and writes them once; a second launch adds
// the work-groups' sums in a fixed order.  4096 x 8192 bf16 (268 MB): 52.5 us a pass
// among others, 5.1 TB/s (43 and 4 of it the kernels, alone).
//
// Rounding: h, dx and y are rounded to their type once, from 32 bits; q to whole
// numbers, half to even; the scale is what it is in 32 bits.
#include <type_traits>

#include "dense.h"

namespace bmlp {
namespace {

// A row's vector from element e0 on: all of it before K, or none, or (one lane
// of the row) K % VEC elements, the same number for every row.  That part is
// loaded as the row's last 16 bytes, without a branch, shifted down where it is
// used (settle), and stored in pieces of 4, 2 and 1 elements: element by element,
// the lane's 48 loads and stores took as long as the rest of the row, and a
// shift right after the load would wait for it (8192 x 1025 bf16 backward 58 us).
// Elements past K are 0.
template <typename T, int VEC>
__device__ __forceinline__ vec_t<T, VEC> load_raw(const T *row, int e0, int K) {
  vec_t<T, VEC> x = (vec_t<T, VEC>)((T)0.f);
  if (K >= VEC) {
    if (e0 < K) __builtin_memcpy(&x, row + min(e0, K - VEC), sizeof(x));
  } else {   // a row shorter than a vector
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (e0 + i < K) x[i] = row[e0 + i];
  }
  return x;
}
template <typename T, int VEC>
__device__ __forceinline__ void settle(vec_t<T, VEC> &x, int e0, int K) {
  if (K % VEC == 0 || K < VEC) return;   // the same for all lanes
  if (e0 >= K || e0 + VEC <= K) return;
  constexpr int kDwords = sizeof(x) / 4;   // 4, or 8 for 32-bit weights beside 16-bit rows
  uint32_t d[kDwords];
  __builtin_memcpy(d, &x, sizeof(x));
  const int drop = (VEC - K % VEC) * (int)sizeof(T);   // bytes
#pragma unroll
  for (int step = kDwords / 2; step > 0; step >>= 1)
    if (drop & 4 * step) {
#pragma unroll
      for (int i = 0; i < kDwords; ++i) d[i] = i + step < kDwords ? d[i + step] : 0u;
    }
  if (drop & 2) {
#pragma unroll
    for (int i = 0; i < kDwords; ++i)
      d[i] = __builtin_amdgcn_alignbyte(i + 1 < kDwords ? d[i + 1 < kDwords ? i + 1 : 0] : 0u, d[i], 2);
  }
  __builtin_memcpy(&x, d, sizeof(x));
}
template <typename T, int VEC>
__device__ __forceinline__ vec_t<float, VEC> load_part(const T *row, int e0, int K) {
  vec_t<T, VEC> x = load_raw<T, VEC>(row, e0, K);
  settle<T, VEC>(x, e0, K);
  return __builtin_convertvector(x, vec_t<float, VEC>);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_raw(T *row, int e0, int K, const vec_t<T, VEC> &x) {
  if (e0 + VEC <= K) {
    __builtin_memcpy(row + e0, &x, sizeof(x));
  } else if (e0 < K) {
    T v[VEC];
    __builtin_memcpy(v, &x, sizeof(x));
    const int m = K % VEC;
    T *o = row + e0;
    if constexpr (VEC > 4) {
      if (m & 4) {
        __builtin_memcpy(o, v, 4 * sizeof(T));
        o += 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = v[i + 4];
      }
    }
    if (m & 2) {
      __builtin_memcpy(o, v, 2 * sizeof(T));
      o += 2;
      v[0] = v[2];
    }
    if (m & 1) *o = v[0];
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_part(T *row, int e0, int K, const vec_t<float, VEC> &f) {
  store_raw<T, VEC>(row, e0, K, __builtin_convertvector(f, vec_t<T, VEC>));
}
template <typename T, int VEC>
__device__ __forceinline__ vec_t<float, VEC> load_weight(const void *w, bool f32, int e0, int K) {
  if (w == nullptr) return (vec_t<float, VEC>)(1.f);
  if (f32) return load_part<float, VEC>(static_cast<const float *>(w), e0, K);
  return load_part<T, VEC>(static_cast<const T *>(w), e0, K);
}

constexpr float kTiny = 0x1p-118f;   // 127 / kTiny is still finite

// Squares are summed times p.down, about 1 / K, so that the sum stays in range
// wherever the mean does.  What a square loses to the range's low end (2^-150 at
// most) is below 2^-33 of a mean of kSmallMean or more.  Where the mean with eps is
// smaller, which takes an eps that is (SMALL), a second sum of (h kUp)^2 is used:
// it has every digit down to h = 2^-149 and stays in range up to means far above.
// A template parameter, since the second sum spills in the widest shape (1024 x 65536
// f32 277 us without, 289 with).
constexpr float kSmallMean = 0x1p-100f, kUp = 0x1p90f;
template <bool SMALL>
__device__ __forceinline__ float norm_rstd(float ss, float ss_up, const NormArgs &p) {
  if (!p.norm) return 1.f;
  const float mean = ss / ((float)p.K * p.down) + p.eps;
  if (!SMALL || !(mean < kSmallMean)) return 1.f / sqrtf(mean);   // (NaN too)
  const float up = ss_up / (float)p.K + p.eps * kUp * kUp;
  return up > kTiny * kUp * (kTiny * kUp) ? kUp / sqrtf(up) : 0.f;
}

// NT threads and R vectors of 16 bytes of x per thread to a row; a wave per
// row (four in a work-group) or a work-group per row.
template <typename T, int NT, int R, bool SMALL>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_quant_kernel(NormArgs p) {
  constexpr int VEC = 16 / sizeof(T), G = NT < 256 ? 256 / NT : 1, W = NT / 64;
  static_assert(NT == 64 || NT >= 256, "a wave or a whole work-group per row");
  typedef vec_t<float, VEC> fv;
  __shared__ float s_ss[W], s_up[SMALL ? W : 1];
  __shared__ uint32_t s_top[W];
  const int g = G > 1 ? (int)threadIdx.x / NT : 0, t = G > 1 ? (int)threadIdx.x % NT : (int)threadIdx.x;
  const int64_t row = (int64_t)blockIdx.x * G + g;
  if (G > 1 && row >= p.n) return;   // a whole wave, and no barrier follows
  const int K = p.K;
  const T *x = static_cast<const T *>(p.x) + row * p.ldx;
  const T *r = p.res != nullptr ? static_cast<const T *>(p.res) + row * p.ldr : nullptr;
  T *ho = p.h != nullptr ? static_cast<T *>(p.h) + row * p.ldh : nullptr;
  fv tv[R];
  float ss = 0.f, ss_up = 0.f;
  uint32_t top = 0u;
  vec_t<T, VEC> xv[R], rv[R];
#pragma unroll
  for (int v = 0; v < R; ++v) xv[v] = load_raw<T, VEC>(x, (v * NT + t) * VEC, K);
  if (r != nullptr) {
#pragma unroll
    for (int v = 0; v < R; ++v) rv[v] = load_raw<T, VEC>(r, (v * NT + t) * VEC, K);
  }
#pragma unroll
  for (int v = 0; v < R; ++v) {
    settle<T, VEC>(xv[v], (v * NT + t) * VEC, K);
    tv[v] = __builtin_convertvector(xv[v], fv);
    if (r != nullptr) {
      settle<T, VEC>(rv[v], (v * NT + t) * VEC, K);
      tv[v] += __builtin_convertvector(rv[v], fv);
    }
  }
#pragma unroll
  for (int v = 0; v < R; ++v) {
    const int e0 = (v * NT + t) * VEC;
    const fv w = load_weight<T, VEC>(p.w, p.w_f32, e0, K);
    if (ho != nullptr) store_part<T, VEC>(ho, e0, K, tv[v]);
    if constexpr (SMALL) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) ss_up += (tv[v][i] * kUp) * (tv[v][i] * kUp);
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      ss += tv[v][i] * (tv[v][i] * p.down);
      tv[v][i] *= w[i];
      // a place that does not exist: h is 0, and the weight 0 or 1
      top = max(top, __float_as_uint(tv[v][i]) & 0x7FFFFFFFu);
    }
  }
  ss = wave_sum(ss);
  top = wave_max_u32(top);
  if constexpr (SMALL) ss_up = wave_sum(ss_up);
  if constexpr (W > 1) {
    if ((t & 63) == 0) {
      s_ss[t >> 6] = ss;
      s_top[t >> 6] = top;
      if constexpr (SMALL) s_up[t >> 6] = ss_up;
    }
    __syncthreads();
    ss = 0.f;
    top = 0u;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      ss += s_ss[w];
      top = max(top, s_top[w]);
    }
    if constexpr (SMALL) {
      ss_up = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) ss_up += s_up[w];
    }
  }
  const float rstd = norm_rstd<SMALL>(ss, ss_up, p);
  const bool bad = top >= 0x7F800000u;
  const float amax = __uint_as_float(top);
  const float inv = !bad && amax > kTiny ? 1.f / amax * 127.f : 0.f;
  const float scale = bad ? __uint_as_float(0x7FC00000u) : inv > 0.f ? amax * rstd / 127.f : 0.f;
  if (t == 0) {
    p.scale[row] = scale;
    if (p.rstd != nullptr) p.rstd[row] = rstd;
  }
  int8_t *q = p.q + row * p.ldq;
  T *y = p.y != nullptr ? static_cast<T *>(p.y) + row * p.ldy : nullptr;
#pragma unroll
  for (int v = 0; v < R; ++v) {
    const int e0 = (v * NT + t) * VEC;
    fv qf;
    vec_t<int8_t, VEC> b;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      qf[i] = bad ? 0.f : rintf(tv[v][i] * inv);   // |t| 127 / max|t| rounds to 127 at most
      b[i] = (int8_t)(int)qf[i];
    }
    store_raw<int8_t, VEC>(q, e0, K, b);
    if (y != nullptr) store_part<T, VEC>(y, e0, K, qf * scale);
  }
}

// NT threads and R vectors per thread to a row, G rows at a time in a
// work-group.  Two rows of each are in registers, in the type they have in
// memory: one that is worked on and the next one's loads.
template <typename T, typename TW, int NT, int R, int G>
__global__ __launch_bounds__(NT *G) void norm_back_kernel(NormBackArgs p) {
  constexpr int VEC = 16 / sizeof(T), W = NT / 64, kCols = NT * R * VEC;
  typedef vec_t<float, VEC> fv;
  typedef vec_t<T, VEC> raw;
  __shared__ float s_sum[2][G][W];
  __shared__ float s_dw[G > 1 ? G * kCols : 1];
  const int g = threadIdx.x / NT, t = threadIdx.x % NT;
  const int K = p.K;
  vec_t<TW, VEC> w[R];
  fv dw[R];
#pragma unroll
  for (int v = 0; v < R; ++v) {
    w[v] = (vec_t<TW, VEC>)((TW)1.f);
    if (p.w != nullptr) {
      w[v] = load_raw<TW, VEC>(static_cast<const TW *>(p.w), (v * NT + t) * VEC, K);
      settle<TW, VEC>(w[v], (v * NT + t) * VEC, K);
    }
    dw[v] = (fv)(0.f);
  }
  raw dy[R], h[R];   // (zeros, for a row that is not there)
#pragma unroll
  for (int v = 0; v < R; ++v) dy[v] = h[v] = (raw)((T)0.f);
  float rstd = 0.f;
  auto load = [&](int64_t row, raw (&y)[R], raw (&x)[R], float &rs) {
    const T *yp = static_cast<const T *>(p.dy) + row * p.lddy, *xp = static_cast<const T *>(p.h) + row * p.ldh;
#pragma unroll
    for (int v = 0; v < R; ++v) {
      y[v] = load_raw<T, VEC>(yp, (v * NT + t) * VEC, K);
      x[v] = load_raw<T, VEC>(xp, (v * NT + t) * VEC, K);
    }
    rs = p.rstd[row];
  };
  const int64_t step = (int64_t)p.parts * G;
  int64_t row = (int64_t)blockIdx.x * G + g;
  if (row < p.n) load(row, dy, h, rstd);
  int turn = 0;
  // as many turns for every row of the work-group, for the barrier's sake
  for (int64_t first = (int64_t)blockIdx.x * G; first < p.n; first += step, row += step) {
    raw dh[R], dy2[R], h2[R];
    float rstd2 = 0.f;
#pragma unroll
    for (int v = 0; v < R; ++v) dy2[v] = h2[v] = (raw)((T)0.f);
    if (p.dh != nullptr && row < p.n) {
      const T *dp = static_cast<const T *>(p.dh) + row * p.lddh;
#pragma unroll
      for (int v = 0; v < R; ++v) dh[v] = load_raw<T, VEC>(dp, (v * NT + t) * VEC, K);
    }
    if (row + step < p.n) load(row + step, dy2, h2, rstd2);
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < R; ++v) {
      settle<T, VEC>(dy[v], (v * NT + t) * VEC, K);
      settle<T, VEC>(h[v], (v * NT + t) * VEC, K);
      const fv a = __builtin_convertvector(dy[v], fv), n = __builtin_convertvector(h[v], fv) * rstd;
      const fv an = a * n, wn = __builtin_convertvector(w[v], fv);
      dw[v] += an;
#pragma unroll
      for (int i = 0; i < VEC; ++i) sum += an[i] * wn[i];
    }
    sum = wave_sum(sum);
    if constexpr (W > 1) {   // two sets of slots in turn: one barrier a row
      if ((t & 63) == 0) s_sum[turn][g][t >> 6] = sum;
      __syncthreads();
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) sum += s_sum[turn][g][i];
      turn ^= 1;
    }
    const float c = sum / (float)K * rstd;   // rstd^2 mean(g h) = rstd mean(g h rstd)
    if (row < p.n) {
      T *dx = static_cast<T *>(p.dx) + row * p.lddx;
#pragma unroll
      for (int v = 0; v < R; ++v) {
        const int e0 = (v * NT + t) * VEC;
        fv d = rstd * (__builtin_convertvector(dy[v], fv) * __builtin_convertvector(w[v], fv) - __builtin_convertvector(h[v], fv) * c);
        if (p.dh != nullptr) {
          settle<T, VEC>(dh[v], e0, K);
          d += __builtin_convertvector(dh[v], fv);
        }
        store_part<T, VEC>(dx, e0, K, d);
      }
    }
#pragma unroll
    for (int v = 0; v < R; ++v) {
      dy[v] = dy2[v];
      h[v] = h2[v];
    }
    rstd = rstd2;
  }
  if (p.dw == nullptr) return;
  float *part = p.part + (size_t)blockIdx.x * K;
  if constexpr (G == 1) {
#pragma unroll
    for (int v = 0; v < R; ++v) store_part<float, VEC>(part, (v * NT + t) * VEC, K, dw[v]);
  } else {   // the work-group's rows together
#pragma unroll
    for (int v = 0; v < R; ++v) __builtin_memcpy(&s_dw[g * kCols + (v * NT + t) * VEC], &dw[v], sizeof(fv));
    __syncthreads();
    for (int col = threadIdx.x; col < kCols && col < K; col += NT * G) {
      float sum = s_dw[col];
#pragma unroll
      for (int i = 1; i < G; ++i) sum += s_dw[i * kCols + col];
      part[col] = sum;
    }
  }
}

// The widest rows: only the columns' sums stay in registers, a row is read again
// for dx.  Its registers spill all the same (16-bit rows 26-34 up to 32768 wide,
// 172-269 above; 32-bit rows 80 up to 32768 wide, 314 above), much less than with
// rows and weights held (1024 x 32768 bf16 741 us).  us a call with dh and dweight:
// bf16 2048 x 20000 125, 1024 x 32768 103, 1024 x 65536 450; f32 4096 x 16384 241,
// 1024 x 32768 204, 1024 x 65536 664: 1.2 to 4.5 TB/s.
template <typename T, typename TW, int R>
__global__ __launch_bounds__(1024) void norm_back_wide_kernel(NormBackArgs p) {
  constexpr int VEC = 16 / sizeof(T), NT = 1024;
  typedef vec_t<float, VEC> fv;
  __shared__ float s_sum[2][NT / 64];
  const int t = threadIdx.x, K = p.K;
  fv dw[R];
#pragma unroll
  for (int v = 0; v < R; ++v) dw[v] = (fv)(0.f);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.n; row += p.parts) {
    const T *dy = static_cast<const T *>(p.dy) + row * p.lddy, *h = static_cast<const T *>(p.h) + row * p.ldh;
    const float rstd = p.rstd[row];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < R; ++v) {
      const int e0 = (v * NT + t) * VEC;
      const fv an = load_part<T, VEC>(dy, e0, K) * (load_part<T, VEC>(h, e0, K) * rstd);
      const fv wn = load_weight<T, VEC>(p.w, std::is_same<TW, float>::value, e0, K);
      dw[v] += an;
#pragma unroll
      for (int i = 0; i < VEC; ++i) sum += an[i] * wn[i];
    }
    sum = wave_sum(sum);
    if ((t & 63) == 0) s_sum[turn][t >> 6] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) sum += s_sum[turn][i];
    turn ^= 1;
    const float c = sum / (float)K * rstd;
    T *dx = static_cast<T *>(p.dx) + row * p.lddx;
    for (int e0 = t * VEC; e0 < K; e0 += NT * VEC) {
      fv d = rstd * (load_part<T, VEC>(dy, e0, K) * load_weight<T, VEC>(p.w, std::is_same<TW, float>::value, e0, K) -
                     load_part<T, VEC>(h, e0, K) * c);
      if (p.dh != nullptr) d += load_part<T, VEC>(static_cast<const T *>(p.dh) + row * p.lddh, e0, K);
      store_part<T, VEC>(dx, e0, K, d);
    }
  }
  if (p.dw == nullptr) return;
#pragma unroll
  for (int v = 0; v < R; ++v) store_part<float, VEC>(p.part + (size_t)blockIdx.x * K, (v * NT + t) * VEC, K, dw[v]);
}

// dweight: a wave adds 64 columns over every 16th row of partial sums
__global__ __launch_bounds__(1024) void norm_back_join_kernel(const float *part, int parts, int K, float *dw) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = (int)blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (col < K) {
    const float *c = part + col;
    int i = wave;
    for (; i + 7 * 16 < parts; i += 8 * 16) {
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = c[(size_t)(i + 16 * q) * K];
#pragma unroll
      for (int q = 0; q < 8; ++q) sum += v[q];
    }
    for (; i < parts; i += 16) sum += c[(size_t)i * K];
  }
  s[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && col < K) {
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += s[i][lane];
    dw[col] = sum;
  }
}

// Work-groups of the backward launch, a partial sum of every column each: one
// to a compute unit, which the prefetched row keeps busy (us for 256 / 512 /
// 1024: 4096 x 8192 bf16 49.3, 52.8, 60.8; 8192 x 1024 18.4, 21.0, 21.0; 777 x 2025
// f16 14.2, 12.8, 16.4).
int back_groups(int n) { return min(n, 256); }

// Shape by the vectors of a row, measured with residual, h and y, us, bf16 / f32 rows
// of that many, the one taken first:
//   16384 rows of 60   64 x 1 14.1 / 12.5, 256 x 1 29.9 / 21.8
//   16384 rows of 128  64 x 2 24.2 / 22.6, 256 x 1 29.9 / 25.3
//   8192 rows of 129   256 x 1 17.4 / 15.6, 64 x 3 14.3 / 13.4
//   8192 rows of 256   256 x 1 24.5 / 23.1, 64 x 4 24.8 / 22.5
//   8192 rows of 300   256 x 2 29.1 / 27.9, 64 x 8 35.8 / 29.3, 512 x 1 29.6 / 27.3
//   8192 rows of 512   256 x 2 49.2 / 53.3, 64 x 8 58.7 / 48.3, 512 x 1 48.8 / 51.2
//   8192 rows of 1024  256 x 4 111 / 109, 512 x 2 109 / 104, 1024 x 1 107 / 106
//   4096 rows of 1500  512 x 4 85.5 / 84.7, 256 x 8 91.1 / 92.0, 1024 x 2 85.1 / 80.7
//   4096 rows of 2048  512 x 4 114 / 110, 256 x 8 118 / 112, 1024 x 2 115 / 106
//   2048 rows of 4096  1024 x 4 122 / 113, 512 x 8 130 / 119
//   300 rows of 512    256 x 2 4.9 / 4.2, 64 x 8 8.8 / 8.1, 512 x 1 4.7 / 4.2
// What is wider has no other shape that fits a work-group.
template <typename T, bool SMALL>
hipError_t norm_quant_of(const NormArgs &a, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  const int vecs = (a.K - 1) / VEC + 1;   // 16-byte vectors of a row
#define BMLP_NORM(NT_, R_)                                                                        \
  if (vecs <= NT_ * (R_)) {                                                                       \
    const int rows = NT_ < 256 ? 256 / NT_ : 1;                                                   \
    hipLaunchKernelGGL((norm_quant_kernel<T, NT_, R_, SMALL>), dim3((a.n - 1) / rows + 1), dim3(NT_ < 256 ? 256 : NT_), 0, s, a); \
    return hipGetLastError();                                                                     \
  }
  BMLP_NORM(64, 1)
  BMLP_NORM(64, 2)
  BMLP_NORM(256, 1)
  BMLP_NORM(256, 2)
  BMLP_NORM(256, 4)
  BMLP_NORM(512, 4)
  BMLP_NORM(1024, 4)
  BMLP_NORM(1024, 8)
  if constexpr (sizeof(T) == 4) BMLP_NORM(1024, 16)
#undef BMLP_NORM
  return hipErrorInvalidValue;
}
template <typename T>
hipError_t norm_quant_of(const NormArgs &a, hipStream_t s) {
  return a.norm && a.eps < kSmallMean ? norm_quant_of<T, true>(a, s) : norm_quant_of<T, false>(a, s);
}

template <typename T, typename TW>
hipError_t norm_back_of(NormBackArgs &a, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  const int vecs = (a.K - 1) / VEC + 1;
#define BMLP_NORM(NT_, R_, G_)                                                                    \
  if (vecs <= NT_ * (R_)) {                                                                       \
    a.parts = min((a.n - 1) / G_ + 1, back_groups(a.n));                                          \
    hipLaunchKernelGGL((norm_back_kernel<T, TW, NT_, R_, G_>), dim3(a.parts), dim3(NT_ * G_), 0, s, a); \
    return hipGetLastError();                                                                     \
  }
  // one vector a thread where that is enough (4096 x 8192 bf16, 1024 x 1 / 512 x 2 /
  // 256 x 4: 49.3, 50.1, 55.2 us)
  BMLP_NORM(64, 1, 16)
  BMLP_NORM(128, 1, 8)
  BMLP_NORM(256, 1, 4)
  BMLP_NORM(512, 1, 2)
  BMLP_NORM(1024, 1, 1)
  // 4096 x 16384 bf16: 512 x 4, which spills 30-42 registers, 112 us; 1024 x 2 520; rows
  // read twice 124.  4096 x 12288: 85, 495, 102
  if constexpr (sizeof(T) == 4) {
    BMLP_NORM(1024, 2, 1)
  } else {
    BMLP_NORM(512, 4, 1)
  }
#undef BMLP_NORM
#define BMLP_NORM(R_)                                                                             \
  if (vecs <= 1024 * R_) {                                                                        \
    a.parts = back_groups(a.n);                                                                   \
    hipLaunchKernelGGL((norm_back_wide_kernel<T, TW, R_>), dim3(a.parts), dim3(1024), 0, s, a);   \
    return hipGetLastError();                                                                     \
  }
  BMLP_NORM(4)
  BMLP_NORM(8)
  if constexpr (sizeof(T) == 4) BMLP_NORM(16)
#undef BMLP_NORM
  return hipErrorInvalidValue;
}
template <typename T>
hipError_t norm_back_of(NormBackArgs &a, hipStream_t s) {
  return a.w_f32 ? norm_back_of<T, float>(a, s) : norm_back_of<T, T>(a, s);
}

}  // namespace

hipError_t launch_norm_quant(int type, const NormArgs &all, hipStream_t s) {
  NormArgs a = all;
  a.down = 1.f;   // the largest power of two up to 1 / K
  while (a.down * (float)a.K > 1.f) a.down *= 0.5f;
  const int64_t size = type == BMLP_TYPE_F32 ? 4 : 2;
  auto rows_on = [](auto *p, int64_t bytes) {
    return p == nullptr ? p : reinterpret_cast<decltype(p)>(reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes);
  };
  for (int64_t i = 0; i < all.n; i += kRowsPerLaunch) {
    a.n = (int)min((int64_t)kRowsPerLaunch, all.n - i);
    a.x = rows_on(all.x, i * all.ldx * size);
    a.res = rows_on(all.res, i * all.ldr * size);
    a.h = rows_on(all.h, i * all.ldh * size);
    a.y = rows_on(all.y, i * all.ldy * size);
    a.q = all.q + i * all.ldq;
    a.scale = all.scale + i;
    a.rstd = rows_on(all.rstd, i * 4);
    const hipError_t e = type == BMLP_TYPE_F32    ? norm_quant_of<float>(a, s)
                         : type == BMLP_TYPE_BF16 ? norm_quant_of<__bf16>(a, s)
                                                  : norm_quant_of<_Float16>(a, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t norm_back_ws_bytes(int n, int K) { return (size_t)back_groups(n) * (size_t)K * sizeof(float); }

hipError_t launch_norm_quant_backward(int type, NormBackArgs &a, hipStream_t s) {
  hipError_t e;
  if (type == BMLP_TYPE_F32)
    e = norm_back_of<float>(a, s);
  else if (type == BMLP_TYPE_BF16)
    e = norm_back_of<__bf16>(a, s);
  else
    e = norm_back_of<_Float16>(a, s);
  if (e != hipSuccess || a.dw == nullptr) return e;
  hipLaunchKernelGGL(norm_back_join_kernel, dim3((a.K - 1) / 64 + 1), dim3(1024), 0, s, a.part, a.parts, a.K, a.dw);
  return hipGetLastError();
}

}  // namespace bmlp
