// Product of int8 rows with packed int8 weights on the matrix cores, exact in
// int32 (128 * 128 * K < 2^31), with the scales and the bias applied in 32 bits
// as the tile is written, and one rounding to the output's type.
//
// The weights lie in the order of the matrix cores' operands (dense.h), so that
// they need no swizzle in LDS and a wave's load of them is 1 KB in running order;
// the zeros past K in them make whatever is read past the end of a row of q
// harmless.
#include "dense.h"
#include "qlinear_plan.h"

#include <algorithm>

namespace bmlp {
namespace {

// a launch holds fewer than 2^32 threads
constexpr int64_t kMaxThreads = UINT32_MAX;

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

// One thread per 16-byte chunk of the packed buffer.
__global__ __launch_bounds__(256) void qlinear_pack_kernel(const int8_t *w, int64_t ldw, int N, int K, int kblocks,
                                                           int64_t chunks, uint8_t *packed) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= chunks) return;
  const int64_t block = i >> 7;
  const int c = (int)(i >> 5) & 3, r = (int)i & 31;
  const int64_t j = block / kblocks * kPackRows + r;
  const int k = (int)(block % kblocks) * kPackK + 16 * c;
  uint8_t b[16] = {};
  if (j < N) {
    const int8_t *src = w + j * ldw + k;
    if (k + 16 <= K) {
      __builtin_memcpy(b, src, 16);
    } else {
#pragma unroll
      for (int q = 0; q < 16; ++q)
        if (k + q < K) b[q] = (uint8_t)src[q];
    }
  }
  __builtin_memcpy(__builtin_assume_aligned(packed + 16 * i, 16), b, 16);
}

bool ragged(const QLinearArgs &a) { return qlinear_ragged(reinterpret_cast<uintptr_t>(a.q), a.n, a.ldq, a.K); }

// 16 bytes of row i at byte k: past K they are not used (the packed weights
// are zero there), so reading on into the next row is fine, past the last
// row's end is not.
__device__ __forceinline__ v4i load_row16(const QLinearArgs &p, int64_t i, int k) {
  const int64_t off = i * p.ldq + k, end = (int64_t)(p.n - 1) * p.ldq + p.K;
  v4i v = (v4i)(0);
  if (off + 16 <= end) {
    __builtin_memcpy(&v, p.q + off, 16);
  } else {
    uint8_t b[16] = {};
#pragma unroll
    for (int q = 0; q < 16; ++q)
      if (off + q < end) b[q] = (uint8_t)p.q[off + q];
    __builtin_memcpy(&v, b, 16);
  }
  return v;
}

// 16 bytes from any address, as 4-byte aligned words: those that hold the first
// and the last of them and all between.  (A 16-byte load that starts inside a
// word takes several times as long: 16 rows of 8191 inputs against 8192 weight
// rows 23.1 us with such loads.)
struct Words {
  v4i a;
  int b;
};
__device__ __forceinline__ Words load_words(const int8_t *p) {
  const int m = (int)(reinterpret_cast<uintptr_t>(p) & 3);
  Words w;
  __builtin_memcpy(&w.a, __builtin_assume_aligned(p - m, 4), 16);
  w.b = *reinterpret_cast<const int *>(p - m + (m ? 16 : 12));
  return w;
}
__device__ __forceinline__ v4i bytes_of(const Words &w, const int8_t *p) {
  const uint32_t m = (uint32_t)reinterpret_cast<uintptr_t>(p) & 3u;
  const uint32_t d[5] = {(uint32_t)w.a.x, (uint32_t)w.a.y, (uint32_t)w.a.z, (uint32_t)w.a.w, (uint32_t)w.b};
  v4i v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (int)__builtin_amdgcn_alignbyte(d[i + 1], d[i], m);   // (m = 0: d[i])
  return v;
}

// ---------------------------------------------------------------------------
// Few rows: a work-group computes a tile of S rows and S columns, its waves
// taking the 64-input blocks in turn (wave w blocks w, w + NW, ...), U of them
// in flight at a time, operands straight from memory; the waves' sums are
// joined in LDS.  S is the MFMA's size, 16 (one MFMA a block) or 32 (two).  The
// weights' bytes bound it, each read once: 16 rows of 8192 inputs against 8192
// weight rows (67 MB) in 12.5 us, 5.4 TB/s, where the weights are still in the
// last-level cache from the call before, and 16.1 us, 4.2 TB/s, over twelve layers in
// turn (805 MB), which that cache does not hold.
// ---------------------------------------------------------------------------
template <typename T, int S, int NW, int U, bool RAGGED>
__global__ __launch_bounds__(64 * NW) void qlinear_direct_kernel(QLinearArgs p, int kblocks, int row_tiles) {
  constexpr int H = S == 32 ? 2 : 1, A = S * S / 64;   // MFMAs of a block; accumulators of an MFMA
  typedef int vacc __attribute__((ext_vector_type(A)));
  __shared__ __align__(16) int s_part[NW][S * S];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane % S, lc = lane / S;     // the lane's row of an operand, and its 16-byte chunk
  const int jt = (int)(blockIdx.x / row_tiles);
  const int64_t i0 = (int64_t)(blockIdx.x % row_tiles) * S;
  const int n_blocks = (p.N - 1) / kPackRows + 1;
  const int64_t row = min(i0 + lr, (int64_t)p.n - 1);   // past the last row: that row again
  const int8_t *q = p.q + row * p.ldq + 16 * lc;
  const int64_t c = (int64_t)S * jt + lr;
  const int64_t block = min(c / kPackRows, (int64_t)n_blocks - 1);   // past the last block: that block again
  const uint8_t *w = p.w + (size_t)block * kblocks * kPackBytes + 512 * lc + 16 * (int)(c % kPackRows);
  vacc acc = (vacc)(0);
  auto multiply = [&](const v4i &a, const v4i &b) {
    if constexpr (S == 32)
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc, 0, 0, 0);
    else
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, acc, 0, 0, 0);
  };
  auto load_w = [&](int kb, int h) { return *reinterpret_cast<const v4i *>(w + (size_t)kb * kPackBytes + 1024 * h); };
  // every block but the last lies inside its rows
  int kb = wave;
  for (; kb + (U - 1) * NW < kblocks - 1; kb += U * NW) {
    v4i a[U][H], b[U][H];
    Words r[RAGGED ? U : 1][H];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < H; ++h) {
        b[u][h] = load_w(kb + u * NW, h);
        const int8_t *src = q + (kb + u * NW) * kPackK + 32 * h;
        if constexpr (RAGGED)
          r[u][h] = load_words(src);
        else
          a[u][h] = *reinterpret_cast<const v4i *>(src);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < H; ++h) {
        if constexpr (RAGGED) a[u][h] = bytes_of(r[u][h], q);   // (steps of 32 bytes: the same place in a word)
        multiply(a[u][h], b[u][h]);
      }
  }
  for (; kb < kblocks; kb += NW) {
    v4i a[H], b[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      b[h] = load_w(kb, h);
      a[h] = load_row16(p, row, kb * kPackK + 32 * h + 16 * lc);
    }
#pragma unroll
    for (int h = 0; h < H; ++h) multiply(a[h], b[h]);
  }
#pragma unroll
  for (int e = 0; e < A; ++e)   // result element e: row 8 (e / 4) + 4 lc + e % 4, column lr
    s_part[wave][(8 * (e >> 2) + 4 * lc + (e & 3)) * S + lr] = acc[e];
  __syncthreads();
  // four columns of a row per thread
  if (tid >= S * S / 4) return;
  const int64_t i = i0 + 4 * tid / S, j = (int64_t)jt * S + 4 * tid % S;
  if (i >= p.n || j >= p.N) return;
  v4i sum = *reinterpret_cast<const v4i *>(&s_part[0][4 * tid]);
#pragma unroll
  for (int v = 1; v < NW; ++v) sum += *reinterpret_cast<const v4i *>(&s_part[v][4 * tid]);
  const float sc = p.scale != nullptr ? p.scale[i] : 1.f;
  vec_t<float, 4> f;
  const int left = (int)min((int64_t)4, p.N - j);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) {
      f[e] = (float)sum[e] * sc * p.wscale[j + e];
      if (p.bias != nullptr) f[e] += p.bias[j + e];
    }
  T *o = static_cast<T *>(p.out) + i * p.ldo + j;
  if (left == 4) {
    store_as<T, 4>(o, f);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < left) o[e] = (T)f[e];
  }
}

template <typename T, int S, int NW, int U>
hipError_t qlinear_direct(const QLinearArgs &a, hipStream_t s) {
  static_assert(S * S / 4 <= 64 * NW, "a thread for four columns");
  const int kblocks = (a.K - 1) / kPackK + 1;
  const int64_t row_tiles = ((int64_t)a.n - 1) / S + 1;
  // columns of as many launches as their number of threads takes, in whole blocks of weights
  const int64_t cols = std::max((int64_t)1, kMaxThreads / (64 * NW) / row_tiles * S / kPackRows) * kPackRows;
  for (int64_t j = 0; j < a.N; j += cols) {
    QLinearArgs p = a;
    p.N = (int)std::min(cols, a.N - j);
    p.w += (size_t)(j / kPackRows) * kblocks * kPackBytes;
    p.wscale += j;
    if (p.bias != nullptr) p.bias += j;
    p.out = static_cast<T *>(a.out) + j;
    const dim3 grid((unsigned)(row_tiles * (((int64_t)p.N - 1) / S + 1)));
    if (ragged(a))
      hipLaunchKernelGGL((qlinear_direct_kernel<T, S, NW, U, true>), grid, dim3(64 * NW), 0, s, p, kblocks, (int)row_tiles);
    else
      hipLaunchKernelGGL((qlinear_direct_kernel<T, S, NW, U, false>), grid, dim3(64 * NW), 0, s, p, kblocks, (int)row_tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------------------
// Tiles through LDS.  A work-group of WM x WN waves computes a tile of
// 32 FM WM rows and 32 FN WN columns; K is walked in steps of 64 through a
// ring of SLOTS LDS slots.  Both operands come by direct-to-LDS loads of 16
// bytes a lane, SLOTS - 2 steps ahead of the barrier that admits them; a row of q
// lies in its slot with its 16-byte units XOR-ed so that an operand read
// touches every bank once (conflicts: 1% of the LDS cycles), and the packed weights lie in
// the order of the reads already.  A wave's operands for one half of a step (32
// inputs) are read while the MFMAs of the half before run, and the loads are
// issued between MFMAs too.  Where rows of q do not start at 16-byte boundaries
// (RAGGED) they go through registers instead.
//
// What bounds it.  Large products: the card's power.  8192^3 in 468 us, 2350 TOP/s:
// the matrix cores are busy for 76% of the cycles, at 1.5 GHz instead of 2.4; a
// loop of the same MFMAs on random operands that stay in registers reaches 3300
// to 3450 (at full issue and 1.6 GHz), the library's product 2070.  Few tiles:
// a compute unit takes in about 55 GB/s whatever the tile, the ring's depth or a
// step's width (of the tried ones 64 x 64 to 256 x 256, 24 to 120 KB in flight,
// 64 and 128 bytes), so eight slots instead of four help small tiles (256 x 4096
// x 4096 15.6 -> 9.8 us) and no more than that.
// ---------------------------------------------------------------------------
typedef __attribute__((address_space(3))) void lds_void;
constexpr int kStepBytes = 64;

__device__ __forceinline__ void bdma16(__amdgpu_buffer_rsrc_t rs, uint32_t voff, void *dst_wave_base) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)dst_wave_base, 16, voff, 0, 0, 0);
}
// waits until at most N vector-memory operations of this wave are outstanding
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt field");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0xF70);
}
__device__ __forceinline__ int swz(int r) { return (r >> 2) & 3; }

template <typename T, int FM, int FN, int WM, int WN, int SLOTS, bool RAGGED>
__global__ __launch_bounds__(64 * WM *WN) void qlinear_tile_kernel(QLinearArgs p, int kblocks, int row_tiles, int col_tiles,
                                                                 int per_xcd) {
  constexpr int NW = WM * WN, TM = 32 * FM * WM, TN = 32 * FN * WN;
  constexpr int kSlot = (TM + TN) * kStepBytes;
  static_assert(SLOTS == 4 || SLOTS == 8, "named arrays below");
  constexpr int kSlotHi = SLOTS == 8 ? kSlot : 16;
  constexpr int kDmaA = TM / 16 / NW, kDmaB = TN / 16 / NW;   // KB-sized loads per wave and step
  constexpr int kDma = (RAGGED ? 0 : kDmaA) + kDmaB;          // direct to LDS
  constexpr int kIssue = kDmaA + kDmaB;                       // all
  // one array a slot, which the compiler can tell apart: an operand read then
  // waits for no load into another slot
  __shared__ __align__(16) uint8_t s0[kSlot], s1[kSlot], s2[kSlot], s3[kSlot];
  __shared__ __align__(16) uint8_t s4[kSlotHi], s5[kSlotHi], s6[kSlotHi], s7[kSlotHi];
  uint8_t *const slot[8] = {s0, s1, s2, s3, s4, s5, s6, s7};
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int wm = wave / WN, wn = wave % WN, lr = lane & 31, lh = lane >> 5;

  // XCD x (work-group id mod 8) takes the x-th eighth of the tiles in an order
  // that runs down eight row tiles, then to the next column tile: what the
  // 32 compute units of an XCD work on at a time shares rows and columns in
  // its L2.
  const int t = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);   // below 2^31 (the grid)
  if (t >= row_tiles * col_tiles) return;
  const int band = t / (8 * col_tiles), r0_ = t - band * 8 * col_tiles, band_rows = min(8, row_tiles - 8 * band);
  // wave-uniform, which the buffer descriptors built from them have to be
  const int nt = __builtin_amdgcn_readfirstlane(r0_ / band_rows);
  const int mt = __builtin_amdgcn_readfirstlane(8 * band + r0_ % band_rows);
  const int64_t m0 = (int64_t)mt * TM;
  const int n_blocks = (p.N - 1) / kPackRows + 1, nb0 = nt * (TN / 32);
  const int rows_left = (int)min((int64_t)TM, p.n - m0), blocks_left = min(TN / 32, n_blocks - nb0);

  // sources: rows and blocks past the end repeat the last one
  const int64_t tile_bytes = (int64_t)(rows_left - 1) * p.ldq + p.K;
  const __amdgpu_buffer_rsrc_t rsA =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p.q + m0 * p.ldq), 0, (int)tile_bytes, kRawRsrcWord3);
  const __amdgpu_buffer_rsrc_t rsB = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t *>(p.w + (size_t)nb0 * kblocks * kPackBytes), 0, blocks_left * kblocks * kPackBytes, kRawRsrcWord3);
  uint32_t voffA[kDmaA], voffB[kDmaB];
#pragma unroll
  for (int h = 0; h < kDmaA; ++h) {   // 16 rows a load, four lanes a row
    const int r = 16 * (kDmaA * wave + h) + lane / 4, u = (lane & 3) ^ swz(r);
    voffA[h] = (uint32_t)min(r, rows_left - 1) * (uint32_t)p.ldq + 16 * u;
  }
#pragma unroll
  for (int h = 0; h < kDmaB; ++h) {   // half a block a load
    const int b = kDmaB * wave + h;
    voffB[h] = (uint32_t)min(b >> 1, blocks_left - 1) * (uint32_t)(kblocks * kPackBytes) + 1024 * (b & 1) + 16 * lane;
  }
  constexpr int kAhead = SLOTS == 8 ? 4 : 1;   // RAGGED: steps of rows in registers
  v4i regA[kAhead][kDmaA];
  auto issue_one = [&](int ks, uint8_t *d, int h) {
    if (h < kDmaB)
      bdma16(rsB, voffB[h < kDmaB ? h : 0] + (uint32_t)(ks * kPackBytes), d + TM * kStepBytes + (kDmaB * wave + h) * 1024);
    else
      bdma16(rsA, voffA[h - kDmaB < kDmaA ? h - kDmaB : 0] + (uint32_t)(ks * kStepBytes),
             d + (kDmaA * wave + h - kDmaB) * 1024);
  };
  auto issue = [&](int ks, uint8_t *d) {
#pragma unroll
    for (int h = 0; h < kDma; ++h) issue_one(ks, d, h);
  };
  const int last = kblocks - 1;
  // RAGGED: rows into registers, by aligned words, and steps later on into their
  // slot.  A unit's 16 bytes lie in five words: its lane loads the last four,
  // the first one is the last of the unit before, which the lane beside it
  // loaded, or for a step's first unit the last unit's lane a step ago.  (Loads
  // that start inside a word take several times as long: 8192 x 8191 x 8192 613 us.)
  // The last step reaches past the end of its rows: on into the next row, whose
  // bytes meet weights that are zero, or past the last row's last word, where the
  // descriptor makes it zeros, word by word.
  const int first = (int)(reinterpret_cast<uintptr_t>(p.q) & 3);
  const int64_t base = (first + m0 * p.ldq) & ~(int64_t)3;   // from the first row's first word
  const __amdgpu_buffer_rsrc_t rsW = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t *>(p.q - first + base), 0, (int)((first + m0 * p.ldq - base + tile_bytes + 3) & ~(int64_t)3), kRawRsrcWord3);
  uint32_t voffW[kDmaA], mW[kDmaA], carry[kDmaA];
  int putW[kDmaA];
  bool lastW[kDmaA];
  if constexpr (RAGGED) {
#pragma unroll
    for (int h = 0; h < kDmaA; ++h) {
      const int r = 16 * (kDmaA * wave + h) + lane / 4, u = lane & 3;
      const int64_t row = first + (m0 + min(r, rows_left - 1)) * p.ldq;
      voffW[h] = (uint32_t)((row & ~(int64_t)3) - base) + 16 * u + 4;   // the unit's second word
      mW[h] = (uint32_t)row & 3u;
      lastW[h] = u == 3;
      putW[h] = r * kStepBytes + 16 * (u ^ swz(r));
      carry[h] = __builtin_amdgcn_raw_buffer_load_b32(rsW, voffW[h] - 16 * u - 4, 0, 0);   // a row's first word
    }
  }
  auto fetch = [&](int ks, v4i (&r)[kDmaA]) {
#pragma unroll
    for (int h = 0; h < kDmaA; ++h) r[h] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(rsW, voffW[h] + (uint32_t)(ks * kStepBytes), 0, 0);
  };
  auto put = [&](uint8_t *d, const v4i (&r)[kDmaA]) {
#pragma unroll
    for (int h = 0; h < kDmaA; ++h) {
      const uint32_t w[4] = {(uint32_t)r[h].x, (uint32_t)r[h].y, (uint32_t)r[h].z, (uint32_t)r[h].w};
      // quad_perm [3,0,1,2]: from the lane before
      const uint32_t w0 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(lastW[h] ? carry[h] : w[3]), 0x93, 0xF, 0xF, false);
      carry[h] = w[3];
      v4i v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (int)__builtin_amdgcn_alignbyte(w[i], i ? w[i ? i - 1 : 0] : w0, mW[h]);
      *reinterpret_cast<v4i *>(d + putW[h]) = v;
    }
  };

  v16i acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = (v16i)(0);
  struct Ops {
    v4i a[FM], b[FN];
  };
  // operand x of a half step: first those of the weights, then those of q
  auto read_one = [&](Ops &o, const uint8_t *t, int h, int x) {
    if (x < FN) {
      o.b[x < FN ? x : 0] = *reinterpret_cast<const v4i *>(t + TM * kStepBytes + (wn * FN + x) * kPackBytes + 1024 * h + 16 * lane);
    } else {
      const int r = (wm * FM + x - FN) * 32 + lr;
      o.a[x - FN < FM ? x - FN : 0] = *reinterpret_cast<const v4i *>(t + r * kStepBytes + (((2 * h + lh) ^ swz(r)) * 16));
    }
  };
  auto read = [&](Ops &o, const uint8_t *t, int h) {
#pragma unroll
    for (int x = 0; x < FM + FN; ++x) read_one(o, t, h, x);
  };
  // The MFMAs of a half step, each followed by its share of `count` other
  // operations: nothing stands between two MFMAs for longer than one of them
  // runs.
  auto multiply = [&](const Ops &o, int count, auto other) {
    int done = 0;
#pragma unroll
    for (int x = 0; x < FM * FN; ++x) {
      const int i = x / FN, j = i & 1 ? FN - 1 - x % FN : x % FN;   // one operand stays from MFMA to MFMA
      acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(o.a[i], o.b[j], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < count; ++q)
        if (q >= done && q < (count * (x + 1) + FM * FN - 1) / (FM * FN)) other(q);
      done = (count * (x + 1) + FM * FN - 1) / (FM * FN);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  Ops r0, r1;
  if constexpr (RAGGED) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      fetch(min(x, last), regA[0]);
      put(slot[x], regA[0]);
    }
#pragma unroll
    for (int x = 0; x < kAhead; ++x) fetch(min(2 + x, last), regA[x]);
  }
#pragma unroll
  for (int x = 0; x < SLOTS - 1; ++x) issue(min(x, last), slot[x]);
  __builtin_amdgcn_sched_barrier(0);
  wait_vm<RAGGED ? 0 : (SLOTS - 2) * kDma>();   // (RAGGED: every step's, so that the count below holds from the start)
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): the rows put into LDS
  __builtin_amdgcn_s_barrier();
  read(r0, slot[0], 0);
  // Step ks, in slot x = ks % SLOTS: its second half's operands are read under
  // the first half's MFMAs, and the next step's first ones under the second's.
  // The slot of step ks - 1 is free once every wave has passed this step's
  // barrier, and takes step ks + SLOTS - 1 (RAGGED: and the rows fetched for
  // step ks + 2 go into their slot).  Past the last step the loads repeat it
  // into slots nobody reads, so that the count in flight stays the same.  The
  // wait leaves in flight what was issued after step ks + 1's loads: SLOTS - 3
  // steps of loads to LDS (RAGGED: issued in the steps up to this one, each
  // after its fetch).
  auto step = [&](int ks, int x) {
    multiply(r0, FM + FN, [&](int q) { read_one(r1, slot[x], 1, q); });
    wait_vm<(SLOTS - 3) * kIssue>();
    if constexpr (RAGGED) __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (RAGGED) {
      put(slot[(x + 2) % SLOTS], regA[x % kAhead]);
      fetch(min(ks + 2 + kAhead, last), regA[x % kAhead]);
      __builtin_amdgcn_sched_barrier(0);
    }
    const int kn = min(ks + SLOTS - 1, last);
    multiply(r1, kDma + FM + FN, [&](int q) {
      if (q < kDma)
        issue_one(kn, slot[(x + SLOTS - 1) % SLOTS], q);
      else
        read_one(r0, slot[(x + 1) % SLOTS], 0, q - kDma);
    });
  };
  int ks = 0;
  for (; ks + SLOTS <= kblocks; ks += SLOTS)
#pragma unroll
    for (int x = 0; x < SLOTS; ++x) step(ks + x, x);
#pragma unroll
  for (int x = 0; x < SLOTS - 1; ++x)
    if (ks + x < kblocks) step(ks + x, x);

  // ---- the tile's values, 32 rows of a wave at a time through LDS, so that
  // a lane stores 16 bytes of a row
  wait_vm<0>();
  __syncthreads();
  constexpr int kCols = 32 * FN, VEC = 16 / (int)sizeof(T), kLd = kCols + VEC;
  static_assert(NW % 4 == 0 && NW / 4 * 32 * kLd * sizeof(T) <= kSlot, "a quarter of the waves stages in each slot");
  const int sl = wave / (NW / 4);
  T *stage = reinterpret_cast<T *>(sl == 0 ? s0 : sl == 1 ? s1 : sl == 2 ? s2 : s3) + (wave % (NW / 4)) * 32 * kLd;
  const int64_t col0 = (int64_t)nt * TN + wn * kCols;
  float ws[FN], bias[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int64_t c = min(col0 + 32 * j + lr, (int64_t)p.N - 1);
    ws[j] = p.wscale[c];
    bias[j] = p.bias != nullptr ? p.bias[c] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int64_t row0 = m0 + (wm * FM + i) * 32;
    float sc[16];
#pragma unroll
    for (int e = 0; e < 16; ++e)
      sc[e] = p.scale != nullptr ? p.scale[min(row0 + 8 * (e >> 2) + 4 * lh + (e & 3), (int64_t)p.n - 1)] : 1.f;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float f = (float)acc[i][j][e] * sc[e] * ws[j];
        if (p.bias != nullptr) f += bias[j];
        stage[(8 * (e >> 2) + 4 * lh + (e & 3)) * kLd + 32 * j + lr] = (T)f;
      }
    wave_sync_lds();
    constexpr int kLanes = kCols / VEC;   // lanes to a row
#pragma unroll
    for (int r = 0; r < 32; r += 64 / kLanes) {
      const int rr = r + lane / kLanes, cc = lane % kLanes * VEC;
      const int64_t row = row0 + rr, col = col0 + cc;
      if (row < p.n && col < p.N) {
        T *o = static_cast<T *>(p.out) + row * p.ldo + col;
        const T *v = stage + rr * kLd + cc;
        if (col + VEC <= p.N) {
          __builtin_memcpy(o, __builtin_assume_aligned(v, 16), 16);
        } else {
          for (int q = 0; q < VEC && col + q < p.N; ++q) o[q] = v[q];
        }
      }
    }
    wave_sync_lds();
  }
}

template <typename T, int FM, int FN, int WM, int WN, int SLOTS>
hipError_t qlinear_tiles(const QLinearArgs &a, hipStream_t s) {
  constexpr int TM = 32 * FM * WM, TN = 32 * FN * WN;
  const int kblocks = (a.K - 1) / kPackK + 1, row_tiles = (a.n - 1) / TM + 1, col_tiles = (a.N - 1) / TN + 1;
  const int64_t tiles = (int64_t)row_tiles * col_tiles, per_xcd = (tiles + 7) / 8;
  if (8 * per_xcd > kMaxThreads / (64 * WM * WN) || col_tiles > INT32_MAX / 8) return hipErrorInvalidValue;
  // buffer descriptors and their offsets are 32 bits: a tile of q and of w
  if (a.ldq > INT32_MAX / (2 * TM)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(8 * per_xcd)), block(64 * WM * WN);
  if (ragged(a))
    hipLaunchKernelGGL((qlinear_tile_kernel<T, FM, FN, WM, WN, SLOTS, true>), grid, block, 0, s, a, kblocks, row_tiles, col_tiles,
                       (int)per_xcd);
  else
    hipLaunchKernelGGL((qlinear_tile_kernel<T, FM, FN, WM, WN, SLOTS, false>), grid, block, 0, s, a, kblocks, row_tiles, col_tiles,
                       (int)per_xcd);
  return hipGetLastError();
}

template <typename T>
hipError_t qlinear_of(const QLinearArgs &a, hipStream_t s) {
  switch (qlinear_kernel(a.n, a.N, a.ldq)) {
    case kDirect16: return qlinear_direct<T, 16, 8, 4>(a, s);
    case kDirect32: return qlinear_direct<T, 32, 16, 2>(a, s);
    case kTile256x256: return qlinear_tiles<T, 4, 2, 2, 4, 4>(a, s);
    case kTile128x256: return qlinear_tiles<T, 2, 2, 2, 4, 4>(a, s);
    case kTile128x128: return qlinear_tiles<T, 2, 2, 2, 2, 8>(a, s);
    case kTile64x128: return qlinear_tiles<T, 1, 2, 2, 2, 8>(a, s);
    default: return qlinear_tiles<T, 1, 1, 2, 2, 8>(a, s);
  }
}

}  // namespace

hipError_t launch_qlinear_pack(const int8_t *w, int64_t ldw, int N, int K, uint8_t *packed, hipStream_t s) {
  const int kblocks = (K - 1) / kPackK + 1;
  const int64_t block_chunks = (int64_t)kblocks * (kPackBytes / 16);          // of 32 weight rows
  const int64_t rows = kMaxThreads / 256 * 256 / block_chunks * kPackRows;   // that a launch takes
  for (int64_t j = 0; j < N; j += rows) {
    const int n = (int)std::min(rows, N - j);
    const int64_t chunks = ((int64_t)(n - 1) / kPackRows + 1) * block_chunks;
    hipLaunchKernelGGL(qlinear_pack_kernel, dim3((unsigned)((chunks - 1) / 256 + 1)), dim3(256), 0, s, w + j * ldw, ldw, n, K,
                       kblocks, chunks, packed + (size_t)(j / kPackRows) * kblocks * kPackBytes);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_qlinear(int type, const QLinearArgs &all, hipStream_t s) {
  QLinearArgs a = all;
  const int64_t size = type == BMLP_TYPE_F32 ? 4 : 2;
  for (int64_t i = 0; i < all.n; i += kRowsPerLaunch) {
    a.n = (int)std::min((int64_t)kRowsPerLaunch, all.n - i);
    a.q = all.q + i * all.ldq;
    a.scale = all.scale != nullptr ? all.scale + i : nullptr;
    a.out = static_cast<char *>(all.out) + i * all.ldo * size;
    const hipError_t e = type == BMLP_TYPE_F32    ? qlinear_of<float>(a, s)
                         : type == BMLP_TYPE_BF16 ? qlinear_of<__bf16>(a, s)
                                                  : qlinear_of<_Float16>(a, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace bmlp
