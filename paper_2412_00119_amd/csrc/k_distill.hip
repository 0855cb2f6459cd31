// Distillation from a teacher's top logits: loss and gradient in one launch.
//
// With m the largest logit of the classes that the teacher did not list and
// S = sum over them of exp((z - m) / tau), the student's log-sum-exp is
//   L = log(exp(m / tau + log S) + sum over listed classes of exp(z / tau)),
// the unlisted classes' probability is exp(m / tau + log S - L), and the
// gradient of an unlisted class is e_v (exp(m / tau - L) - p_r / S) with
// e_v = exp((z_v - m) / tau).  So the listed classes never enter S, and S is
// never the small difference of two large sums.
//
// A work-group takes a row and holds it in registers between the sum and the
// gradient, so that the row is read once; what does not fit is read again (from
// the caches, mostly).  Vectors of 16 bytes are cut at 16-byte boundaries of
// memory, whatever the row's start: position = class + shift.  Which classes
// are listed is a bit per position in LDS; a vector's listed places become -inf,
// so that they drop out of maximum, sum and gradient alike, and their gradients
// are written at the end.  The first wave works on the list (teacher's softmax,
// the listed part of L, the loss) while the others sum; where a row has one wave
// only, before it sums.
//
// What bounds it: 4 bytes of traffic a class in 16 bits, and two exponentials
// a class at a quarter of the vector rate.  2048 x 131072 bf16 (1.07 GB): 254 us, 4.2
// TB/s; 8192 x 8192: 61 us, 4.4 TB/s.  Few or short rows: a chain of dependent loads
// and joins of about 5 us (1 x 1000 f32), to which 4096 rows of 1000 add 6.
#include "dense.h"

namespace bmlp {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float finite_or_0(float m) { return m == kNegInf ? 0.f : m; }

// Maximum and sum of exponentials relative to it (in steps of s2 = log2(e) / tau).
struct MaxSum {
  float m, S;
};
__device__ __forceinline__ MaxSum join(const MaxSum &a, const MaxSum &b, float s2) {
  const float m = fmaxf(a.m, b.m), m0 = finite_or_0(m);
  return {m, a.S * exp2_of((a.m - m0) * s2) + b.S * exp2_of((b.m - m0) * s2)};
}
// over the wave: its maximum first, then the sums, which add
__device__ __forceinline__ MaxSum wave_join(const MaxSum &v, float s2) {
  const float m = wave_max(v.m);
  return {m, wave_sum(v.S * exp2_of((v.m - finite_or_0(m)) * s2))};
}

// A row's entries in LDS: k of each.
struct List {
  int *idx;      // the class, or -1: no entry, or a class's later entry
  float *z, *p;  // its logit; t / tau, then p (a class listed twice: the sum, at its first entry)
};
// What the list's wave leaves for the others.
struct ListSums {
  float tmax, psum;   // largest t / tau; sum of p (before it is divided by itself where there is no lse)
  MaxSum z;           // of the listed classes
};

// The list's part, by one wave.  On entry idx holds classes or -1.
template <typename T, typename TT>
__device__ ListSums work_on_list(const List &l, int k, const T *z, const TT *t, float inv_tau, float s2, bool has_lse,
                                 float lse, bool twice) {
  const int lane = threadIdx.x & 63;
  ListSums r{kNegInf, 0.f, {kNegInf, 0.f}};
  for (int j = lane; j < k; j += 64) {
    const int v = l.idx[j];
    const float x = v >= 0 ? (float)t[j] * inv_tau : kNegInf;
    l.p[j] = x;
    l.z[j] = v >= 0 ? (float)z[v] : 0.f;
    r.tmax = fmaxf(r.tmax, x != x ? 0.f : x);   // NaN: the row counts, and becomes NaN
  }
  r.tmax = wave_max(r.tmax);
  const float ref = has_lse ? lse : finite_or_0(r.tmax);
  for (int j = lane; j < k; j += 64) {
    const float e = l.idx[j] >= 0 ? exp2_of((l.p[j] - ref) * kLog2e) : 0.f;
    l.p[j] = e;
    r.psum += e;
  }
  r.psum = wave_sum(r.psum);
  if (twice) {   // the sums in the list's order; all are read before any is written
    constexpr int kPer = BMLP_MAX_DISTILL_LISTED / 64;
    float sum[kPer];
    uint32_t later = 0u;
    wave_sync_lds();
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int j = lane + 64 * q;
      sum[q] = 0.f;
      if (j < k && l.idx[j] >= 0)
        for (int i = 0; i < k; ++i)
          if (l.idx[i] == l.idx[j]) {
            sum[q] += l.p[i];
            if (i < j) later |= 1u << q;
          }
    }
    wave_sync_lds();
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int j = lane + 64 * q;
      if (j < k) {
        l.p[j] = sum[q];
        if (later >> q & 1u) l.idx[j] = -1;
      }
    }
  }
  for (int j = lane; j < k; j += 64)
    if (l.idx[j] >= 0) r.z.m = fmaxf(r.z.m, l.z[j]);
  const float m0 = finite_or_0(wave_max(r.z.m));
  for (int j = lane; j < k; j += 64)
    if (l.idx[j] >= 0) r.z.S += exp2_of((l.z[j] - m0) * s2);
  r.z.m = m0;
  r.z.S = wave_sum(r.z.S);
  return r;
}

// The row's constants, from the unlisted classes' maximum and sum and the
// list's; `some_rest`: there is a class that is not listed.
struct RowSums {
  float z0, log_sum;      // L = z0 / tau + log_sum
  float m0, f;            // gradient of an unlisted class: f exp((z - m0) / tau)
  float g, pscale;        // of a listed one: g (exp((z - z0) / tau - log_sum) - p pscale)
  float p_rest, log_rest; // the rest's p and log q
};
__device__ __forceinline__ RowSums row_sums(const MaxSum &u, const ListSums &l, float inv_tau, float s2, float g, bool has_lse,
                                            bool some_rest) {
  RowSums r;
  r.m0 = finite_or_0(u.m);
  r.z0 = u.S == 0.f ? l.z.m : l.z.S == 0.f ? r.m0 : fmaxf(r.m0, l.z.m);
  // unlisted classes relative to z0 (S = 0: none, or all of them -inf)
  const float out = u.S == 0.f ? 0.f : u.S * exp2_of((r.m0 - r.z0) * s2);
  const float in = l.z.S == 0.f ? 0.f : l.z.S * exp2_of((l.z.m - r.z0) * s2);
  r.log_sum = logf(in + out);
  r.pscale = has_lse ? 1.f : 1.f / l.psum;
  r.p_rest = has_lse && some_rest ? fmaxf(1.f - l.psum, 0.f) : 0.f;
  r.log_rest = logf(u.S) + (r.m0 - r.z0) * inv_tau - r.log_sum;
  r.g = l.psum != l.psum ? l.psum : g;   // a NaN of the teacher's: the whole row
  const float q_m = exp2_of(((r.m0 - r.z0) * inv_tau - r.log_sum) * kLog2e);   // q of an unlisted class with logit m0
  r.f = u.S == 0.f ? 0.f * r.g : r.g * (q_m - r.p_rest / u.S);
  return r;
}
// The loss, by the list's wave.
__device__ __forceinline__ float row_loss(const List &l, int k, const RowSums &r, float inv_tau) {
  float loss = 0.f;
  for (int j = threadIdx.x & 63; j < k; j += 64)
    if (l.idx[j] >= 0) {
      const float p = l.p[j] * r.pscale;
      if (p != 0.f) loss += p * (logf(p) - ((l.z[j] - r.z0) * inv_tau - r.log_sum));
    }
  loss = wave_sum(loss);
  if (r.p_rest > 0.f) loss += r.p_rest * (logf(r.p_rest) - r.log_rest);
  return loss;
}

// 16-byte vectors of a row, cut at 16-byte boundaries; positions [lo, hi) exist
template <typename T>
struct Vectors {
  static constexpr int N = 16 / sizeof(T);
  typedef vec_t<T, N> raw;
  typedef vec_t<float, N> val;
  int lo, hi;

  __device__ bool whole(int v) const { return v * N >= lo && v * N + N <= hi; }
  __device__ raw load(const T *base, int v) const {   // base: position 0, 16-byte aligned
    raw x;
    if (whole(v)) {
      x = *reinterpret_cast<const raw *>(base + v * N);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = v * N + i;
        x[i] = e >= lo && e < hi ? base[e] : (T)kNegInf;
      }
    }
    return x;
  }
  // base: the output's position 0, aligned to an element
  __device__ void store(T *base, int v, const val &f) const {
    if (whole(v)) {
      store_as<T, N>(base + v * N, f);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = v * N + i;
        if (e >= lo && e < hi) base[e] = (T)f[i];
      }
    }
  }
  // listed places become -inf
  static __device__ void drop(raw &x, const uint32_t *bits, int v) {
    const uint32_t b = (bits[v * N >> 5] >> (v * N & 31)) & ((1u << N) - 1u);
    if (b) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (b >> i & 1u) x[i] = (T)kNegInf;
    }
  }
  static __device__ float largest(const raw &x, float m) {
    const val f = __builtin_convertvector(x, val);
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, f[i]);
    return m;
  }
  static __device__ float sum(const raw &x, float m0, float s2) {
    const val f = __builtin_convertvector(x, val);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s += exp2_of((f[i] - m0) * s2);
    return s;
  }
  static __device__ val gradient(const raw &x, float m0, float s2, float g) {
    val f = __builtin_convertvector(x, val);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = g * exp2_of((f[i] - m0) * s2);
    return f;
  }
};

// NT threads to a row, R vectors of it in each thread's registers.
template <typename T, typename TT, int NT, int R, int OCC>
__global__ __launch_bounds__(NT, OCC) void distill_kernel(DistillArgs p) {
  typedef Vectors<T> V;
  constexpr int NW = NT / 64, kHeld = NT * R;
  extern __shared__ uint32_t s_bits[];
  __shared__ MaxSum s_part[NW];
  __shared__ ListSums s_list;
  __shared__ int s_twice, s_listed;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), c = p.c, k = p.k;
  const int64_t row = blockIdx.x;
  const T *z = static_cast<const T *>(p.z) + row * p.ldz;
  T *dz = p.dz != nullptr ? static_cast<T *>(p.dz) + row * p.lddz : nullptr;
  const int32_t *idx = p.idx + row * k;
  const float weight = p.weight != nullptr ? p.weight[row] : 1.f, lse = p.lse != nullptr ? p.lse[row] : 0.f, inv_tau = 1.f / p.tau, s2 = inv_tau * kLog2e;
  const int shift = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const T *zb = z - shift;
  const V vec{shift, c + shift};
  const int vecs = (c + shift + V::N - 1) / V::N, words = (c + shift + 31) / 32;
  List l;
  l.idx = reinterpret_cast<int *>(s_bits + words);
  l.z = reinterpret_cast<float *>(l.idx + k);
  l.p = l.z + k;

  typename V::raw x[R];
#pragma unroll
  for (int v = 0; v < R; ++v)
    if (v * NT + t < vecs) x[v] = vec.load(zb, v * NT + t);
  for (int i = t; i < words; i += NT) s_bits[i] = 0u;
  if (t == 0) s_twice = s_listed = 0;
  __syncthreads();
  for (int j = t; j < k; j += NT) {
    int v = idx[j];
    if (v >= 0 && v < c) {
      const uint32_t bit = 1u << ((v + shift) & 31);
      if (atomicOr(&s_bits[(v + shift) >> 5], bit) & bit)
        s_twice = 1;
      else
        atomicAdd(&s_listed, 1);
    } else {
      v = -1;
    }
    l.idx[j] = v;
  }
  __syncthreads();
  const int listed = s_listed;
  bool counts = listed > 0 && weight != 0.f;

  MaxSum u{kNegInf, 0.f};
  if (counts) {
    if (wave == 0) {
      const ListSums r = work_on_list<T, TT>(l, k, z, static_cast<const TT *>(p.t) + row * k, inv_tau, s2,
                                             p.lse != nullptr, lse, s_twice != 0);
      if (t == 0) s_list = r;
    }
#pragma unroll
    for (int v = 0; v < R; ++v)
      if (v * NT + t < vecs) {
        V::drop(x[v], s_bits, v * NT + t);
        u.m = V::largest(x[v], u.m);
      }
    const float m0 = finite_or_0(u.m);
#pragma unroll
    for (int v = 0; v < R; ++v)
      if (v * NT + t < vecs) u.S += V::sum(x[v], m0, s2);
    for (int v = kHeld + t; v < vecs; v += NT) {
      typename V::raw y = vec.load(zb, v);
      V::drop(y, s_bits, v);
      MaxSum w{V::largest(y, u.m), 0.f};
      const float w0 = finite_or_0(w.m);
      w.S = u.S * exp2_of((u.m - w0) * s2) + V::sum(y, w0, s2);
      u = w;
    }
    u = wave_join(u, s2);
    if ((t & 63) == 0) s_part[wave] = u;
    __syncthreads();
    u = s_part[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) u = join(u, s_part[w], s2);
    counts = s_list.tmax != kNegInf;
  }
  if (!counts) {   // nothing to learn from
    if (t == 0) p.loss[row] = 0.f;
    if (dz != nullptr)
      for (int v = t; v < vecs; v += NT) vec.store(dz - shift, v, (typename V::val)(0.f));
    return;
  }
  const RowSums r = row_sums(u, s_list, inv_tau, s2, weight * p.tau, p.lse != nullptr, listed < c);
  if (wave == 0) {
    const float loss = row_loss(l, k, r, inv_tau);
    if (t == 0) p.loss[row] = (s_list.psum != s_list.psum ? s_list.psum : loss) * p.tau * p.tau * weight;
  }
  if (dz == nullptr) return;
#pragma unroll
  for (int v = 0; v < R; ++v)
    if (v * NT + t < vecs) vec.store(dz - shift, v * NT + t, V::gradient(x[v], r.m0, s2, r.f));
  for (int v = kHeld + t; v < vecs; v += NT) {
    typename V::raw y = vec.load(zb, v);
    V::drop(y, s_bits, v);
    vec.store(dz - shift, v, V::gradient(y, r.m0, s2, r.f));
  }
  __syncthreads();
  for (int j = t; j < k; j += NT)
    if (l.idx[j] >= 0)
      dz[l.idx[j]] = (T)(r.g * (exp2_of(((l.z[j] - r.z0) * inv_tau - r.log_sum) * kLog2e) - l.p[j] * r.pscale));
}

// Threads to a row and vectors held by each: enough of both that a row, or
// nearly all of it, stays in registers, and few enough threads that several
// rows share a compute unit and one loads or stores while another computes.
// Measured, us: 8192 x 4096 bf16 (512 vectors a row) 64 threads x 8 38, 128 x 4 39,
// 256 x 4 45; 8192 x 8192 bf16 (1024) 256 x 4 61, 128 x 8 61, 64 x 8 79, 512 x 8 89;
// 8192 x 5000 f32 (1250) 256 x 8 71, 256 x 4 79, 512 x 8 104; 4096 x 32000 bf16 (4000)
// 512 x 8 119, 512 x 16 122, 256 x 8 146, 1024 x 8 195; 2048 x 65536 bf16 (8192)
// 512 x 16 128, 1024 x 4 132, 1024 x 8 162; 2048 x 131072 bf16 (16384) 1024 x 6, the most
// that two rows a compute unit have registers for and most of the row read twice, 254, 1024 x 5
// 258, 1024 x 4 263, 512 x 16 274, 1024 x 16 275, 512 x 8 298.
template <typename T, typename TT>
hipError_t distill_of(const DistillArgs &a, hipStream_t s) {
  constexpr int N = 16 / sizeof(T);
  const int vecs = (a.c + 2 * (N - 1)) / N;   // at most, for any shift
  const size_t lds = (size_t)((a.c + N - 1 + 31) / 32) * 4 + (size_t)a.k * 12;
#define BMLP_DISTILL(NT_, R_, OCC_) \
  hipLaunchKernelGGL((distill_kernel<T, TT, NT_, R_, OCC_>), dim3(a.n), dim3(NT_), lds, s, a)
  if (vecs <= 256)
    BMLP_DISTILL(64, 4, 8);
  else if (vecs <= 512)
    BMLP_DISTILL(64, 8, 4);
  else if (vecs <= 1024)
    BMLP_DISTILL(256, 4, 8);
  else if (vecs <= 2048)
    BMLP_DISTILL(256, 8, 4);
  else if (vecs <= 4096)
    BMLP_DISTILL(512, 8, 4);
  else if (vecs <= 8192)
    BMLP_DISTILL(512, 16, 4);
  else
    BMLP_DISTILL(1024, 6, 8);
#undef BMLP_DISTILL
  return hipGetLastError();
}

template <typename T>
hipError_t distill_of(int t_type, const DistillArgs &a, hipStream_t s) {
  if (t_type == BMLP_TYPE_F32) return distill_of<T, float>(a, s);
  if (t_type == BMLP_TYPE_BF16) return distill_of<T, __bf16>(a, s);
  return distill_of<T, _Float16>(a, s);
}

}  // namespace

hipError_t launch_distill(int type, int t_type, const DistillArgs &all, hipStream_t s) {
  DistillArgs a = all;
  const int64_t size = type == BMLP_TYPE_F32 ? 4 : 2, t_size = t_type == BMLP_TYPE_F32 ? 4 : 2;
  for (int64_t i = 0; i < all.n; i += kRowsPerLaunch) {
    a.n = (int)min((int64_t)kRowsPerLaunch, all.n - i);
    a.z = static_cast<const char *>(all.z) + i * all.ldz * size;
    a.t = static_cast<const char *>(all.t) + i * all.k * t_size;
    a.idx = all.idx + i * all.k;
    a.lse = all.lse != nullptr ? all.lse + i : nullptr;
    a.weight = all.weight != nullptr ? all.weight + i : nullptr;
    a.loss = all.loss + i;
    a.dz = all.dz != nullptr ? static_cast<char *>(all.dz) + i * all.lddz * size : nullptr;
    const hipError_t e = type == BMLP_TYPE_F32    ? distill_of<float>(t_type, a, s)
                         : type == BMLP_TYPE_BF16 ? distill_of<__bf16>(t_type, a, s)
                                                  : distill_of<_Float16>(t_type, a, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace bmlp
