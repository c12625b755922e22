// vocab_f32.hip -- the vocabulary loss's two products in fp32, on the fp32 matrix instructions.
//
// 64 x 64 tiles, 4 waves of 32 x 32 (2 x 2 blocks of v_mfma_f32_16x16x4_f32), steps of 32 contraction values
// staged through registers into LDS.  A lane's values of a row are eight neighbours of the step (the
// order of a step's contraction values is free), so fragments are 16-byte reads.  333 rows against 5003 of 512: 27 us
// and 29 us for the products (62 TFLOP/s; a large fp32 product reaches 132), 64 us in all.  What bounds it is each
// step's loads: two workgroups a CU cannot cover them (two LDS buffers and one barrier a step: 28 and 30 us).
#include <hip/hip_runtime.h>

#include "device_common.h"
#include "vocab.h"

namespace dsv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kLd = 36;  // LDS row of a step, padded

// Sums of a 64 x 64 tile: acc[i][j][v] is row 32 wm + 16 i + l % 16, column 32 wn + 16 j + 4 (l / 16) + v.
// NT: Q [n][C]; NN: Q [C][n].  Rows, columns and contraction values that do not exist count as zeros.
template <bool NN>
__device__ __forceinline__ void tile64(const float* P, int64_t ldp, int p_rows, const float* Q, int64_t ldq, int q_cols,
                                       int C, float* sa, float* sb, f32x4 (&acc)[2][2]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  const int l15 = lane & 15, g4 = lane >> 4;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  f32x4 ra[2], rb[2];
  // C is a multiple of 4 in the rows of P and Q that are read four at a time
  auto fetch = [&](int k0) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = (tid >> 3) + 32 * e, c = k0 + 4 * (tid & 7);
      ra[e] = r < p_rows && c < C ? *reinterpret_cast<const f32x4*>(P + r * ldp + c) : f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (!NN) {
        rb[e] = r < q_cols && c < C ? *reinterpret_cast<const f32x4*>(Q + r * ldq + c) : f32x4{0.f, 0.f, 0.f, 0.f};
      } else {
        const int k = (tid >> 4) + 16 * e, n = 4 * (tid & 15);
        rb[e] = k0 + k < C && n < q_cols ? *reinterpret_cast<const f32x4*>(Q + (k0 + k) * ldq + n) : f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
  };
  fetch(0);
  for (int k0 = 0; k0 < C; k0 += 32) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = (tid >> 3) + 32 * e;
      *reinterpret_cast<f32x4*>(sa + r * kLd + 4 * (tid & 7)) = ra[e];
      if constexpr (!NN) {
        *reinterpret_cast<f32x4*>(sb + r * kLd + 4 * (tid & 7)) = rb[e];
      } else {
        const int k = (tid >> 4) + 16 * e, n = 4 * (tid & 15);
#pragma unroll
        for (int v = 0; v < 4; ++v) sb[(n + v) * kLd + k] = rb[e][v];
      }
    }
    __syncthreads();
    if (k0 + 32 < C) fetch(k0 + 32);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f32x4 fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = *reinterpret_cast<const f32x4*>(sa + (32 * wm + 16 * i + l15) * kLd + 8 * g4 + 4 * s);
        fb[i] = *reinterpret_cast<const f32x4*>(sb + (32 * wn + 16 * i + l15) * kLd + 8 * g4 + 4 * s);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[j][e], fa[i][e], acc[i][j], 0, 0, 0);
    }
  }
}

__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

__global__ __launch_bounds__(256) void vocab_f32_logits_kernel(VocabArgs a) {
  __shared__ __attribute__((aligned(16))) float sa[64 * kLd], sb[64 * kLd];
  __shared__ float red[2][2][64];
  const int n_m = (a.T + 63) / 64;
  const int mt = blockIdx.x % n_m, nt = blockIdx.x / n_m;
  const int m0 = 64 * mt, n0 = 64 * nt, cols = min(64, a.vn - n0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, l15 = lane & 15;
  f32x4 acc[2][2];
  tile64<false>(static_cast<const float*>(a.X) + (int64_t)m0 * a.ldx, a.ldx, a.T - m0,
                static_cast<const float*>(a.W) + (int64_t)(a.v0 + n0) * a.ldw, a.ldw, cols, a.K, sa, sb, acc);
  const int c0 = 32 * wn + 4 * (lane >> 4);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        if (c0 + 16 * j + v >= cols) acc[i][j][v] = -INFINITY;
        m = fmaxf(m, acc[i][j][v]);
      }
    m = quad_max(m);
    if (lane < 16) red[0][wn][32 * wm + 16 * i + l15] = m;
  }
  __syncthreads();
  float ref[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 32 * wm + 16 * i + l15, row = m0 + r;
    const bool in = row < a.T;
    const float m = fmaxf(red[0][0][r], red[0][1][r]) * kLog2e;
    const float have = !a.first && in ? a.ref[row] : 0.f;
    ref[i] = own_reference(m, have, a.first) ? m : have;
    const float base = ref[i] == -INFINITY ? 0.f : ref[i];
    const int t = in ? a.target[row] - a.v0 - n0 - c0 : -1;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float z = acc[i][j][v];
        float e = exp2f(z * kLog2e - base);
        if (t == 16 * j + v) e = 0.f;
        sum += e;
        acc[i][j][v] = e;
      }
      if (a.grad && in)
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.P) + (int64_t)row * a.ldp + n0 + c0 + 16 * j) = acc[i][j];
    }
    sum = quad_sum(sum);
    if (lane < 16) red[1][wn][r] = sum;
  }
  __syncthreads();
  if (wn == 0 && lane < 16) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 32 * wm + 16 * i + l15;
      if (m0 + r < a.T) a.stats[(int64_t)(m0 + r) * a.ld_stats + nt] = make_float2(ref[i], red[1][0][r] + red[1][1][r]);
    }
  }
}

__global__ __launch_bounds__(256) void vocab_f32_grad_kernel(VocabArgs a) {
  __shared__ __attribute__((aligned(16))) float sa[64 * kLd], sb[64 * kLd];
  const int n_m = (a.T + 63) / 64, n_n = (a.K + 63) / 64;
  const int part = blockIdx.x / (n_m * n_n), tile = blockIdx.x % (n_m * n_n);
  const int m0 = 64 * (tile % n_m), n0 = 64 * (tile / n_m);
  const int c0 = part * a.split_len;
  // the piece's columns up to a whole step hold zeros in P, so its rows may be read four at a time; W
  // is read row by row, and rows past the piece are left out
  const int C = min(a.vn - c0, a.split_len);
  f32x4 acc[2][2];
  tile64<true>(static_cast<const float*>(a.P) + (int64_t)m0 * a.ldp + c0, a.ldp, a.T - m0,
               static_cast<const float*>(a.W) + (int64_t)(a.v0 + c0) * a.ldw + n0, a.ldw, a.K - n0, C, sa, sb, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = m0 + 32 * wm + 16 * i + (lane & 15);
    if (row >= a.T) continue;
    const float f = a.first ? 0.f : a.alpha[row];
    float* o = a.O + ((int64_t)part * a.T + row) * a.K;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int col = n0 + 32 * wn + 16 * j + 4 * (lane >> 4);
      if (col >= a.K) continue;
      f32x4 x = acc[i][j];
      if (!a.first) x += *reinterpret_cast<const f32x4*>(o + col) * f;
      *reinterpret_cast<f32x4*>(o + col) = x;
    }
  }
}

}  // namespace

hipError_t launch_vocab_f32_logits(const VocabArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(vocab_f32_logits_kernel, dim3((unsigned)(a.n_ct * (int64_t)((a.T + 63) / 64))), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_vocab_f32_grad(const VocabArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(vocab_f32_grad_kernel, dim3((unsigned)((int64_t)((a.T + 63) / 64) * ((a.K + 63) / 64) * a.split)),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace dsv
