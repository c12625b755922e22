// vocab.hip -- the vocabulary loss in bf16 (gfx950), what both types share, and the C entry points.
//
// Per piece of the vocabulary: vocab_logits computes the logits of 256 x 256 tiles and, while they are in
// registers, turns them into exponentials relative to the row's reference (P, with the target's term left
// out), with their sums; vocab_fold adds the tiles' sums of a row and, where the reference moved, brings
// the piece's terms to it; vocab_grad adds P W to the row's running sum.  vocab_finish forms the loss and
//     dx = weight (sum_{v != t} e_v W_v - others W_t) / (others + e_t).
// So the logits are computed once: 4 T K V operations where recomputing them would take 6.  A piece is as wide as P's
// room (kPieceBytes) allows, so that what one kernel writes of it the next one finds in the last-level cache.
// 256 rows against 128256 of 4096, with the head transposed at hand: 0.57 ms, 0.42 at the rate of a large product on
// this card (1290 TFLOP/s); 4096 rows against 128256 of 8192: 13.1 ms (1320 TFLOP/s).  The exponentials are rounded to
// bf16 for the second product; dX is off from 64 bits by 0.17% in the root mean square either way: its own rounding.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "device_common.h"
#include "dsv.h"
#include "gemm_tile.h"
#include "vocab.h"

namespace dsv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// ---- logits -------------------------------------------------------------------------------------------
// GRAD: P is written.  Tiles of 32 FM rows and 32 FN columns; NB: buffers (2: tile_nt, else tile_ring).  Up to 128 rows
// the stream of a large head is what bounds it: one row against 128256 of 4096 takes 185 us with the fold, 5.7 TB/s, 128 rows 206.
// Else the matrix core: 4096 rows, 32256 x 8192 a piece, 1.61 ms (1340 TFLOP/s).
template <bool GRAD, int FM, int FN, int NB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, NB == 2 ? 1 : 2))) void vocab_logits_kernel(VocabArgs a) {
  constexpr int WM = 16 * FM, TM = 2 * WM, WN = 16 * FN, TN = 2 * WN;
  constexpr int kStage = NB == 2 ? kTileStage : kRingStage<FM, FN>;
  __shared__ __attribute__((aligned(1024))) char smem0[kStage];
  __shared__ __attribute__((aligned(1024))) char smem1[kStage];
  __shared__ float red[3][2][TM];  // [maximum, sum, reference][column half][row]
  const int n_m = (a.T + TM - 1) / TM;
  int mt, nt;
  tile_at(tile_of(blockIdx.x, gridDim.x), n_m, a.n_ct, mt, nt);
  const int m0 = mt * TM, n0 = nt * TN, cols = min(TN, a.vn - n0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, l15 = lane & 15, g4 = lane >> 4;
  f32x4 acc[FM][FN];
  // with one row tile the head's rows come from memory once, and neighbouring tiles begin a step apart (one row
  // against 128256 of 4096: 215 us in step, 185 so; with more row tiles it changes nothing)
  const int turn = n_m == 1 ? nt : 0;
  const uint16_t* const X = static_cast<const uint16_t*>(a.X) + (int64_t)m0 * a.ldx;
  const uint16_t* const W = static_cast<const uint16_t*>(a.W) + (int64_t)(a.v0 + n0) * a.ldw;
  char* idle = smem0;
  if constexpr (NB == 2) {
    idle = tile_nt<FM>(X, a.ldx, a.T - m0, W, a.ldw, cols, a.K, turn, smem0, smem1, acc);
  } else {
    __shared__ __attribute__((aligned(1024))) char smem2[kStage];
    if constexpr (NB == 3) {
      char* const ring[3] = {smem0, smem1, smem2};
      tile_ring<uint16_t, FM, FN, 3>(X, a.ldx, a.T - m0, W, a.ldw, cols, a.K, turn, ring, acc);
    } else if constexpr (NB == 4) {
      __shared__ __attribute__((aligned(1024))) char smem3[kStage];
      char* const ring[4] = {smem0, smem1, smem2, smem3};
      tile_ring<uint16_t, FM, FN, 4>(X, a.ldx, a.T - m0, W, a.ldw, cols, a.K, turn, ring, acc);
    } else {
      static_assert(NB == 6, "buffers");
      __shared__ __attribute__((aligned(1024))) char smem3[kStage];
      __shared__ __attribute__((aligned(1024))) char smem4[kStage];
      __shared__ __attribute__((aligned(1024))) char smem5[kStage];
      char* const ring[6] = {smem0, smem1, smem2, smem3, smem4, smem5};
      tile_ring<uint16_t, FM, FN, 6>(X, a.ldx, a.T - m0, W, a.ldw, cols, a.K, turn, ring, acc);
    }
  }
  const int c0 = wn * WN + 4 * g4;  // column of acc[.][j][v]: c0 + 16 j + v
  // The sums are read twice and never written: in registers of the matrix core from the first to the last.
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    float m = -INFINITY;
    if (cols == TN) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, acc[i][j][v]);
    } else {
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, c0 + 16 * j + v < cols ? acc[i][j][v] : -INFINITY);
    }
    m = quad_max(m);
    if (lane < 16) red[0][wn][wm * WM + 16 * i + l15] = m;
  }
  __syncthreads();
  // Terms: 32 rows of 16 FN columns per wave at a time, whose P goes through the idle buffer for 16-byte stores.
  constexpr int SRS = WN * 2 + 16, RPS = 64 / (2 * FN);  // rows a store instruction covers
  static_assert(4 * 32 * SRS <= kStage, "slices");
  char* const slice = idle + wave * 32 * SRS;
  uint16_t* const P = static_cast<uint16_t*>(a.P) + (int64_t)(m0 + wm * WM) * a.ldp + n0 + wn * WN;
#pragma unroll
  for (int t = 0; t < FM / 2; ++t) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = 2 * t + h, r = wm * WM + 16 * i + l15, row = m0 + r;
      const bool in = row < a.T;
      const float m = fmaxf(red[0][0][r], red[0][1][r]) * kLog2e;
      const float have = !a.first && in ? a.ref[row] : 0.f;
      const float ref = tile_reference(m, have, a.first), base = ref == -INFINITY ? 0.f : ref;
      const int tc = in ? a.target[row] - a.v0 - n0 - c0 : -1;  // the target's column, from the lane's first
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        f32x4 e;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float z = acc[i][j][v];
          e[v] = __builtin_amdgcn_exp2f(z * kLog2e - base);
          if (tc == 16 * j + v) e[v] = 0.f;
          if (cols < TN && c0 + 16 * j + v >= cols) e[v] = 0.f;
          sum += e[v];
        }
        if constexpr (GRAD)
          *reinterpret_cast<uint2*>(slice + (16 * h + l15) * SRS + 2 * (16 * j + 4 * g4)) =
              make_uint2(f2bf2(e[0], e[1]), f2bf2(e[2], e[3]));
      }
      sum = quad_sum(sum);
      if (lane < 16) {
        red[1][wn][r] = sum;
        if (wn == 0) red[2][0][r] = ref;
      }
    }
    if constexpr (GRAD) {
      asm volatile("" ::: "memory");  // a wave's LDS accesses run in order
#pragma unroll
      for (int q = 0; q < FN; ++q) {
        const int r = RPS * q + lane / (2 * FN), c = lane % (2 * FN);
        const u32x4 v = *reinterpret_cast<const u32x4*>(slice + r * SRS + 16 * c);
        if (m0 + wm * WM + 32 * t + r < a.T) *reinterpret_cast<u32x4*>(P + (int64_t)(32 * t + r) * a.ldp + 8 * c) = v;
      }
      asm volatile("" ::: "memory");
    }
  }
  __syncthreads();
  for (int r = threadIdx.x; r < TM; r += 256)
    if (m0 + r < a.T) a.stats[(int64_t)(m0 + r) * a.ld_stats + nt] = make_float2(red[2][0][r], red[1][0][r] + red[1][1][r]);
}

// ---- second product -------------------------------------------------------------------------------------
// Range `part` of the piece's contraction: O[part] = alpha O[part] + P W (O[part] = P W for the first piece).  Matrix
// core: 4096 rows, 32256 x 8192 a piece, 1.59 ms (1360 TFLOP/s).  With few tiles the contraction is cut into
// ranges with sums of their own, which vocab_finish adds (256 rows of 4096, 128256 columns: 16 tiles in 16 ranges,
// 0.28 ms).
template <bool NN, int FM>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void vocab_grad_kernel(VocabArgs a) {
  constexpr int WM = 16 * FM, TM = 2 * WM;
  __shared__ __attribute__((aligned(1024))) char smem0[NN ? kTileStageNN : kTileStage];
  __shared__ __attribute__((aligned(1024))) char smem1[NN ? kTileStageNN : kTileStage];
  const int n_m = (a.T + TM - 1) / TM, n_n = (a.K + 255) / 256, tiles = n_m * n_n;
  // ranges one after the other: those that run together read the same columns of P and W
  const int lin = tile_of(blockIdx.x, gridDim.x), part = lin / tiles;
  int mt, nt;
  tile_at(lin - part * tiles, n_m, n_n, mt, nt);
  const int m0 = mt * TM, n0 = nt * 256;
  const int c0 = part * a.split_len, C = min(a.vn - c0, a.split_len);
  const uint16_t* W = static_cast<const uint16_t*>(NN ? a.W : a.Wt);
  W += NN ? (int64_t)(a.v0 + c0) * a.ldw + n0 : (int64_t)n0 * a.ldwt + a.v0 + c0;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  auto put = [&](auto value) {
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int row = m0 + wm * WM + 16 * i + (lane & 15);
      if (row >= a.T) continue;
      const float f = a.first ? 0.f : a.alpha[row];
      float* o = a.O + ((int64_t)part * a.T + row) * a.K;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int col = n0 + wn * 128 + 16 * j + 4 * (lane >> 4);
        if (col >= a.K) continue;
        f32x4 x = value(i, j);
        if (!a.first) x += *reinterpret_cast<const f32x4*>(o + col) * f;
        *reinterpret_cast<f32x4*>(o + col) = x;
      }
    }
  };
  if (C <= 0) {  // a short last piece ends before this range
    put([](int, int) { return f32x4{0.f, 0.f, 0.f, 0.f}; });
    return;
  }
  f32x4 acc[FM][8];
  const uint16_t* const P = static_cast<const uint16_t*>(a.P) + (int64_t)m0 * a.ldp + c0;
  if constexpr (NN) {
    __shared__ __attribute__((aligned(1024))) char smem2[kTileStageNN];
    __shared__ __attribute__((aligned(1024))) char smem3[kTileStageNN];
    tile_nn<FM>(P, a.ldp, a.T - m0, W, a.ldw, a.K - n0, C, smem0, smem1, smem2, smem3, acc);
  } else {
    tile_nt<FM>(P, a.ldp, a.T - m0, W, a.ldwt, a.K - n0, C, 0, smem0, smem1, acc);
  }
  put([&](int i, int j) { return acc[i][j]; });
}

// ---- rows -------------------------------------------------------------------------------------------------
template <int N>
__device__ __forceinline__ float block_max(float x, float* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int w = 1; w < N; ++w) x = fmaxf(x, red[w]);
  __syncthreads();
  return x;
}
template <int N>
__device__ __forceinline__ float block_sum(float x, float* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int w = 1; w < N; ++w) x += red[w];
  __syncthreads();
  return x;
}

template <int N>
__device__ __forceinline__ double block_sum(double x, double* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int w = 1; w < N; ++w) x += red[w];
  return x;
}

// Eight values from p on.
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(v[i] << 16), x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i + e] = v[e];
  }
}

// One row: the piece's sums into the row's, at the larger of the references; the terms of tiles at another
// reference are brought to the row's.  After the last piece the target's logit, its term and the loss, in 64 bits: the
// logarithm and the logit nearly cancel for a sure row, and there is one of each per row (one row against 128256 of
// 4096: the loss is off by 8e-7 in the root mean square with the logit from the products, whose sums are fp32).
template <typename T>
__global__ __launch_bounds__(256) void vocab_fold_kernel(VocabArgs a) {
  __shared__ float red[4];
  __shared__ double red64[4];
  const int row = blockIdx.x;
  const int target = a.last ? a.target[row] : -1;
  const bool has = target >= 0 && target < a.V;
  double zt = 0.;
  if (has) {
    const T* x = static_cast<const T*>(a.X) + row * a.ldx;
    const T* w = static_cast<const T*>(a.W) + target * a.ldw;
    for (int c = 8 * threadIdx.x; c < a.K; c += 8 * 256) {
      float xs[8], ws[8];
      load8(x + c, xs);
      load8(w + c, ws);
#pragma unroll
      for (int e = 0; e < 8; ++e) zt += (double)xs[e] * ws[e];
    }
    zt = block_sum<4>(zt, red64);
  }
  const float2* st = a.stats + (int64_t)row * a.ld_stats;
  const float have = a.first ? -INFINITY : a.ref[row];
  float m = have;
  for (int t = threadIdx.x; t < a.n_ct; t += 256) m = fmaxf(m, st[t].x);
  const float ref = block_max<4>(m, red);
  float sum = 0.f;
  bool moved = false;
  for (int t = threadIdx.x; t < a.n_ct; t += 256) {
    const float2 x = st[t];
    sum += x.x == -INFINITY ? x.y : x.y * exp2f(x.x - ref);
    moved |= x.x != ref;
  }
  sum = block_sum<4>(sum, red);
  if (threadIdx.x == 0) {
    const float f = have == -INFINITY ? 0.f : exp2f(have - ref);
    const float others = (a.first ? 0.f : a.others[row] * f) + sum;
    a.others[row] = others;
    a.ref[row] = ref;
    a.alpha[row] = f;
    if (a.last) {
      const double et = has ? exp2(zt * 1.4426950408889634 - ref) : 1.;
      a.term[row] = (float)et;
      // near 0 the loss keeps its relative accuracy
      if (a.loss)
        a.loss[row] = !has           ? 0.f
                      : et >= others ? (float)log1p(others / et)
                                     : (float)(log(others + et) + ref * 0.69314718055994531 - zt);
    }
  }
  if (!a.grad || !__syncthreads_or(moved)) return;
  T* P = static_cast<T*>(a.P) + (int64_t)row * a.ldp;
  constexpr int E = 16 / sizeof(T);
  for (int64_t c = threadIdx.x * E; c < (int64_t)a.n_ct * a.tw; c += 256 * E) {
    const float r = st[c / a.tw].x;
    if (r == ref || r == -INFINITY) continue;
    const float f = ldexpf(1.f, (int)fmaxf(r - ref, -1000.f));  // both are whole numbers, ref the larger one
    u32x4 v = *reinterpret_cast<const u32x4*>(P + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (E == 8)
        v[i] = f2bf2(__uint_as_float(v[i] << 16) * f, __uint_as_float(v[i] & 0xffff0000u) * f);
      else
        v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
    }
    *reinterpret_cast<u32x4*>(P + c) = v;
  }
}

__device__ __forceinline__ f32x4 load4(const uint16_t* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
               __uint_as_float(v.y & 0xffff0000u)};
}
__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ void store4(uint16_t* p, f32x4 x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]));
}
__device__ __forceinline__ void store4(float* p, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }

template <typename T>
__global__ __launch_bounds__(256) void vocab_finish_kernel(VocabArgs a) {
  const int row = blockIdx.x, t = a.target[row];
  T* dx = static_cast<T*>(a.dX) + (int64_t)row * a.lddx;
  const bool has = t >= 0 && t < a.V;
  const T* w = static_cast<const T*>(a.W) + (int64_t)(has ? t : 0) * a.ldw;
  const float others = a.others[row], f = (a.weight ? a.weight[row] : 1.f) / (others + a.term[row]);
  // 1024 columns a workgroup
  const int c = 1024 * blockIdx.y + 4 * threadIdx.x;
  if (c < a.K) {
    f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
    if (has) {
#pragma unroll 4
      for (int s = 0; s < a.split; ++s) x += *reinterpret_cast<const f32x4*>(a.O + ((int64_t)s * a.T + row) * a.K + c);
      x = (x - load4(w + c) * others) * f;
    }
    store4(dx + c, x);
  }
}

// ---- host -------------------------------------------------------------------------------------------------
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

int device_cus() {
  static int cached[64] = {};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 256;
  if (dev < 64 && cached[dev] > 0) return cached[dev];
  int n = 0;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
  if (dev < 64) cached[dev] = n;
  return n;
}

// Pieces of the vocabulary and ranges of the second product's contraction.
struct Pieces {
  int32_t tw, width, n;         // column tile, piece width (a multiple of it), pieces
  int32_t split, split_len;     // ranges per piece and their length
  size_t p, stats, rows, o, total;
};

// Column tile of the logits: whole tiles (256, of 256 or 128 rows) where they fill the CUs, else 128 x 128 or 64 x 64 ones,
// whichever takes the least time in rounds of one tile a CU.  Microseconds a round and 64 contraction values: 1.5 for
// 256 x 256, 1.05 for 128 x 256, 0.62 and 0.28 for the small ones, each measured at 5000, 20000 and 50000 columns.
// Losses of rows of 4096, in microseconds, whole / 128 / 64: 64 rows against 5000 75 / 45 / 26, against 20000 78 / 49 /
// 51, against 50000 88 / 94 / 97; 500 rows against 5000 101 / 49 / 65, against 20000 108 / 130 / 186.
int logits_tile(int32_t T, int64_t width, int cus) {
  auto rounds = [&](int tm, int tn) {
    const int64_t n = ((T + tm - 1) / tm) * ((width + tn - 1) / tn);
    return (double)((n + cus - 1) / cus);
  };
  const double whole = T <= 128 ? 1.05 * rounds(128, 256) : 1.5 * rounds(256, 256);
  const double t128 = 0.62 * rounds(128, 128), t64 = 0.28 * rounds(64, 64);
  return whole <= std::min(t128, t64) ? 256 : t128 <= t64 ? 128 : 64;
}

constexpr int64_t kPieceBytes = 256 << 20;  // of P: the size of the last-level cache

Pieces pieces(dsv_dtype dt, int32_t T, int32_t K, int32_t V, int64_t ldw, bool grad, int cus) {
  Pieces r{};
  const bool bf = dt == DSV_BF16;
  const int64_t size = bf ? 2 : 4;
  r.tw = bf ? 256 : 128;
  int64_t width = (V + r.tw - 1) / r.tw * r.tw;
  r.split = 1;
  if (grad) {
    // P within its room; 32-bit offsets of the second product's reads of W and of a tile's (up to 256) rows of P
    const int64_t most = std::min({kPieceBytes / (size * std::max(T, 1)), ((int64_t)1 << 30) / (size * ldw),
                                   (((int64_t)1 << 31) - 1) / (size * 256)}) / r.tw * r.tw;
    const int64_t n = (V + std::max<int64_t>(most, r.tw) - 1) / std::max<int64_t>(most, r.tw);
    width = ((V + n - 1) / n + r.tw - 1) / r.tw * r.tw;
  }
  r.width = (int32_t)width;
  r.n = (int32_t)((V + width - 1) / width);
  r.split_len = r.width;
  if (bf) r.tw = logits_tile(T, r.width, cus);
  if (grad && T > 0) {
    // Ranges: whole rounds of tiles against the traffic of the ranges' own sums, in microseconds.
    const int tm = bf ? (T <= 128 ? 128 : 256) : vocab_f32_rows(T), tn = bf ? 256 : 128;
    const int64_t tiles = (int64_t)((T + tm - 1) / tm) * ((K + tn - 1) / tn);
    const double step = bf ? (tm == 128 ? 0.8 : 1.45) : (tm == 32 ? 1.0 : 1.9);  // of 64 contraction values
    double best = 1e30;
    for (int s = 1; s <= 32; ++s) {
      const int64_t len = (width / 64 + s - 1) / s * 64;
      if (s > 1 && len < 512) break;
      const double t = (double)((tiles * s + cus - 1) / cus) * (len / 64) * step + s * (double)T * K * 8 / 4.5e6;
      if (t < best) best = t, r.split = s, r.split_len = (int32_t)len;
    }
    r.split = (int32_t)((width + r.split_len - 1) / r.split_len);
  }
  size_t at = 0;
  auto room = [&](size_t bytes) {
    const size_t o = at;
    at += align256(bytes);
    return o;
  };
  r.p = room(grad ? (size_t)T * r.width * size : 0);
  r.stats = room((size_t)T * (r.width / r.tw) * sizeof(float2));
  r.rows = room((size_t)T * 4 * sizeof(float));
  r.o = room(grad ? (size_t)r.split * T * K * sizeof(float) : 0);
  r.total = std::max<size_t>(at, 256);
  return r;
}

int stride(int32_t given, int32_t len, int64_t* out) {
  if (given == 0) {
    *out = len;
    return DSV_OK;
  }
  if (given < len || (given & 7) || given > (1 << 20)) return DSV_ERR_SIZE;
  *out = given;
  return DSV_OK;
}

bool aligned(const void* p, size_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check_shape(dsv_dtype dt, int32_t T, int32_t K, int32_t V, int32_t ldw, int64_t* w) {
  if (T < 0) return DSV_ERR_ARG;
  if (dt != DSV_BF16 && dt != DSV_F32) return DSV_ERR_RANGE;
  if (K <= 0 || (K & 7) || K > (1 << 20) || V < 1 || V > (1 << 24)) return DSV_ERR_SIZE;
  return stride(ldw, K, w);
}

// Tiles of 64 rows have six buffers where each has a CU to itself, else four, which leave room for two on a CU (one row of
// 4096 against 5000: 22 us with six, 25 with four; 45 rows of 816 against 113000: 65 and 57).
template <bool GRAD>
hipError_t launch_logits(const VocabArgs& a, int cus, hipStream_t s) {
  const int tm = a.tw < 256 ? a.tw : a.T <= 128 ? 128 : 256;
  const dim3 grid((unsigned)(a.n_ct * (int64_t)((a.T + tm - 1) / tm)));
  if (a.tw == 64 && grid.x <= (unsigned)cus)
    hipLaunchKernelGGL((vocab_logits_kernel<GRAD, 2, 2, 6>), grid, dim3(256), 0, s, a);
  else if (a.tw == 64) hipLaunchKernelGGL((vocab_logits_kernel<GRAD, 2, 2, 4>), grid, dim3(256), 0, s, a);
  else if (a.tw == 128) hipLaunchKernelGGL((vocab_logits_kernel<GRAD, 4, 4, 3>), grid, dim3(256), 0, s, a);
  else if (tm == 128) hipLaunchKernelGGL((vocab_logits_kernel<GRAD, 4, 8, 2>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((vocab_logits_kernel<GRAD, 8, 8, 2>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_grad(const VocabArgs& a, hipStream_t s) {
  const int64_t tm = a.T <= 128 ? 128 : 256;
  const dim3 grid((unsigned)(((a.T + tm - 1) / tm) * ((a.K + 255) / 256) * a.split));
  if (a.Wt) {
    if (tm == 128) hipLaunchKernelGGL((vocab_grad_kernel<false, 4>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((vocab_grad_kernel<false, 8>), grid, dim3(256), 0, s, a);
  } else {
    if (tm == 128) hipLaunchKernelGGL((vocab_grad_kernel<true, 4>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((vocab_grad_kernel<true, 8>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

int run(VocabArgs a, dsv_dtype dt, void* ws, size_t ws_bytes, hipStream_t s) {
  const bool bf = dt == DSV_BF16;
  const int cus = device_cus();
  const Pieces pc = pieces(dt, a.T, a.K, a.V, a.ldw, a.grad != 0, cus);
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return DSV_ERR_ARG;
  if (ws_bytes < pc.total) return DSV_ERR_SIZE;
  if (a.T == 0) return DSV_OK;
  char* b = static_cast<char*>(ws);
  a.P = a.grad ? b + pc.p : nullptr;
  a.ldp = pc.width;
  a.stats = reinterpret_cast<float2*>(b + pc.stats);
  a.ld_stats = pc.width / pc.tw;
  a.ref = reinterpret_cast<float*>(b + pc.rows);
  a.others = a.ref + a.T;
  a.term = a.others + a.T;
  a.alpha = a.term + a.T;
  a.O = reinterpret_cast<float*>(b + pc.o);
  a.tw = pc.tw;
  a.split_len = pc.split_len;
  for (int i = 0; i < pc.n; ++i) {
    a.v0 = i * pc.width;
    a.vn = std::min(pc.width, a.V - a.v0);
    a.n_ct = (a.vn + pc.tw - 1) / pc.tw;
    a.first = i == 0;
    a.last = i + 1 == pc.n;
    a.split = pc.split;
    hipError_t e = !bf ? launch_vocab_f32_logits(a, cus, s) : a.grad ? launch_logits<true>(a, cus, s) : launch_logits<false>(a, cus, s);
    if (e != hipSuccess) return DSV_ERR_DEVICE;
    if (bf) hipLaunchKernelGGL(vocab_fold_kernel<uint16_t>, dim3((unsigned)a.T), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(vocab_fold_kernel<float>, dim3((unsigned)a.T), dim3(256), 0, s, a);
    if (hipGetLastError() != hipSuccess) return DSV_ERR_DEVICE;
    if (!a.grad) continue;
    e = bf ? launch_grad(a, s) : launch_vocab_f32_grad(a, s);
    if (e != hipSuccess) return DSV_ERR_DEVICE;
  }
  if (!a.grad) return DSV_OK;
  if (bf) hipLaunchKernelGGL(vocab_finish_kernel<uint16_t>, dim3((unsigned)a.T, (a.K + 1023) / 1024), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(vocab_finish_kernel<float>, dim3((unsigned)a.T, (a.K + 1023) / 1024), dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? DSV_OK : DSV_ERR_DEVICE;
}

}  // namespace
}  // namespace dsv

using namespace dsv;

extern "C" int dsv_vocab_workspace(dsv_dtype dt, int32_t T, int32_t K, int32_t V, int32_t ldw, int32_t grad,
                                   size_t* bytes) {
  if (!bytes) return DSV_ERR_ARG;
  int64_t w = 0;
  const int rc = check_shape(dt, T, K, V, ldw, &w);
  if (rc != DSV_OK) return rc;
  *bytes = pieces(dt, T, K, V, w, grad != 0, device_cus()).total;
  return DSV_OK;
}

extern "C" int dsv_vocab_loss(dsv_dtype dt, int32_t T, int32_t K, int32_t V, const void* X, int32_t ldx, const void* W,
                              int32_t ldw, const int32_t* target, float* loss, void* ws, size_t ws_bytes,
                              void* hip_stream) {
  VocabArgs a{};
  int rc = check_shape(dt, T, K, V, ldw, &a.ldw);
  if (rc == DSV_OK) rc = stride(ldx, K, &a.ldx);
  if (rc != DSV_OK) return rc;
  if (!aligned(W, 16) || (T > 0 && (!aligned(X, 16) || !aligned(target, 4) || !aligned(loss, 4)))) return DSV_ERR_ARG;
  a.T = T, a.K = K, a.V = V;
  a.X = X, a.W = W, a.target = target, a.loss = loss;
  return run(a, dt, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
}

extern "C" int dsv_vocab_loss_grad(dsv_dtype dt, int32_t T, int32_t K, int32_t V, const void* X, int32_t ldx,
                                   const void* W, int32_t ldw, const void* Wt, int32_t ldwt, const int32_t* target,
                                   const float* weight, float* loss, void* dX, int32_t lddx, void* ws, size_t ws_bytes,
                                   void* hip_stream) {
  VocabArgs a{};
  int rc = check_shape(dt, T, K, V, ldw, &a.ldw);
  if (rc == DSV_OK) rc = stride(ldx, K, &a.ldx);
  if (rc == DSV_OK) rc = stride(lddx, K, &a.lddx);
  bool use_t = Wt && dt == DSV_BF16 && (V & 7) == 0;
  if (rc == DSV_OK && use_t) rc = stride(ldwt, V, &a.ldwt);
  use_t = use_t && 256 * 2 * a.ldwt < (int64_t)1 << 31;  // tile_nt's offsets over a tile's 256 rows
  if (rc != DSV_OK) return rc;
  if (!aligned(W, 16) || (use_t && !aligned(Wt, 16)) || (reinterpret_cast<uintptr_t>(weight) & 3) ||
      (reinterpret_cast<uintptr_t>(loss) & 3))
    return DSV_ERR_ARG;
  if (T > 0 && (!aligned(X, 16) || !aligned(target, 4) || !aligned(dX, 16))) return DSV_ERR_ARG;
  a.T = T, a.K = K, a.V = V;
  a.X = X, a.W = W, a.Wt = use_t ? Wt : nullptr;
  a.target = target, a.weight = weight, a.loss = loss, a.dX = dX;
  a.grad = 1;
  return run(a, dt, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
}
