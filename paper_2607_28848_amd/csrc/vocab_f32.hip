// vocab_f32.hip -- the vocabulary loss's two products in fp32, on the fp32 matrix instructions.
//
// Tiles of 32 FM rows and 128 columns, 4 waves in a 2 x 2 grid, each FM x 4 blocks of v_mfma_f32_16x16x4_f32, steps of 32
// contraction values through three LDS buffers that global memory is loaded straight into.  A step's order of
// contraction values is free: slot l / 16 of instruction e stands for value 16 s + 4 (l / 16) + e, so a lane's
// values of a row of P (and of Q, NT) are a 16-byte chunk.  The loads of a step have two steps' time to arrive, and one
// barrier a step: 600 rows against 20000 of 1024, losses 250 us, with the gradient 478 (103 TFLOP/s; a large fp32 product
// reaches 132; 64 x 64 tiles staged through registers, two barriers a step: 290 and 571).  333 rows against 5003 of 512:
// 25 us and 23 for the products, 52 a pass: two waves a SIMD for 16 steps, and the tiles' start and end.
#include <hip/hip_runtime.h>

#include "device_common.h"
#include "gemm_tile.h"
#include "vocab.h"

namespace dsv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kStage = kRingStage<2, 4>;

// out[m][n] = sum_c P[m][c] Q[c][n] of a tile of 32 FM rows and 128 columns: tile_ring's loop with three buffers, and with
// Q's rows as they lie.  P's rows hold zeros from C to a multiple of 4; rows, columns and contraction values that do not
// exist count as zeros.
template <int FM>
__device__ __forceinline__ void tile_nn_f32(const float* P, int64_t ldp, int p_rows, const float* Q, int64_t ldq_, int q_cols,
                                         int C, char* b0, char* b1, char* b2, f32x4 (&acc)[FM][4]) {
  constexpr int A_BYTES = 32 * FM * 128, N = FM + 4, TK = 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, l15 = lane & 15, g4 = lane >> 4, lr = lane >> 3;
  const int ld = (int)ldp, ldq = (int)ldq_, nk = (C + TK - 1) / TK;
  const i32x4 ra = tile_rsrc(P, ((int64_t)(min(32 * FM, p_rows) - 1) * ld + ((C + 3) & ~3)) * 4);
  const i32x4 rb = tile_rsrc(Q, ((int64_t)(C - 1) * ldq + q_cols) * 4);
  // P: chunk c of row r in slot c ^ r % 8 ^ r / 8 % 8.  Q, rows of 512 bytes: the 64-byte block b of row c in block
  // b ^ c / 4 % 4 (a read's four rows in different banks).
  constexpr int kNone = 0x7FFFFFF0;  // past every descriptor
  int chunk_a[FM], chunk_b[4];
#pragma unroll
  for (int i = 0; i < FM; ++i) chunk_a[i] = (lane & 7) ^ lr ^ ((FM * wave + i) & 7);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    chunk_b[i] = (lane & 31) ^ 4 * ((2 * wave + (i >> 1)) & 3);
  // Load e of step kt (P's first).  Past the last step the last is loaded again, for a buffer that is not read: so each
  // step's loads are followed by the same number of others.
  auto load = [&](int kt, char* st, int e) {
    const int k0 = min(kt, nk - 1) * TK;
    if (e < FM) {
      const int q = wave * FM + e;
      llvm_amdgcn_raw_buffer_load_lds_t(ra, (lds_u32*)(st + q * 1024), 16,
                                        k0 + 4 * chunk_a[e] < C ? 16 * chunk_a[e] + lr * ld * 4 : kNone,
                                        __builtin_amdgcn_readfirstlane((q * 8 * ld + k0) * 4), 0, 0);
    } else {
      const int q = wave * 4 + e - FM;
      llvm_amdgcn_raw_buffer_load_lds_t(rb, (lds_u32*)(st + A_BYTES + q * 1024), 16,
                                        16 * chunk_b[e - FM] + (lane >> 5) * ldq * 4,
                                        __builtin_amdgcn_readfirstlane((k0 + 2 * q) * ldq * 4), 0, 0);
    }
  };
#pragma unroll
  for (int e = 0; e < N; ++e) load(0, b0, e);
#pragma unroll
  for (int e = 0; e < N; ++e) load(1, b1, e);
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // Fragment addresses: a lane part picked by the half step and block (the chunk swizzle), plus an immediate.
  const int part = g4 ^ (l15 & 7) ^ (l15 >> 3);
  int off_a[4], off_b[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    off_a[x] = (16 * FM * wm + l15) * 128 + 16 * (part ^ (2 * FM * wm) ^ (2 * x));
    off_b[x] = A_BYTES + 4 * g4 * 512 + 256 * wn + 64 * (x ^ g4) + 4 * l15;
  }
  // Step kt in `st`, with the loads of step kt + 2 into `nxt`, which the step before this one has read; behind the
  // step's own loads are those of AFTER more.
  auto step = [&](auto with, auto after, int kt, const char* st, char* nxt) {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(decltype(after)::value * N));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();  // not __syncthreads(), which would wait for every load
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    f32x4 fa[2][FM], fb[2][4];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[s][i] = *reinterpret_cast<const f32x4*>(st + off_a[(2 * s) ^ i] + 2048 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) fb[s][j][e] = *reinterpret_cast<const float*>(st + off_b[j] + 8192 * s + 512 * e);
      }
    }
    if constexpr (decltype(with)::value) {
#pragma unroll
      for (int e = 0; e < N; ++e) load(kt + 2, nxt, e);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < FM; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[s][j][e], fa[s][i][e], acc[i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  int kt = 0;
  for (; kt + 3 <= nk; kt += 3) {
    step(flag_c<true>{}, num_c<1>{}, kt, b0, b2);
    step(flag_c<true>{}, num_c<1>{}, kt + 1, b1, b0);
    step(flag_c<true>{}, num_c<1>{}, kt + 2, b2, b1);
  }
  if (kt < nk) step(flag_c<false>{}, num_c<1>{}, kt, b0, nullptr);
  if (kt + 1 < nk) step(flag_c<false>{}, num_c<0>{}, kt, b1, nullptr);
  vmem_wait_all();  // nothing lands in the buffers any more
  __syncthreads();
}

__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

template <int FM>
__global__ __launch_bounds__(256) void vocab_f32_logits_kernel(VocabArgs a) {
  constexpr int WM = 16 * FM, TM = 2 * WM;
  __shared__ __attribute__((aligned(1024))) char b0[kStage];
  __shared__ __attribute__((aligned(1024))) char b1[kStage];
  __shared__ __attribute__((aligned(1024))) char b2[kStage];
  __shared__ float red[2][2][TM];
  // the row tiles of a column tile one after the other: they share the head's rows in L2
  const int n_m = (a.T + TM - 1) / TM, lin = tile_of(blockIdx.x, gridDim.x);
  const int mt = lin % n_m, nt = lin / n_m;
  const int m0 = TM * mt, n0 = 128 * nt, cols = min(128, a.vn - n0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, l15 = lane & 15;
  f32x4 acc[FM][4];
  char* const ring[3] = {b0, b1, b2};
  tile_ring<float, FM, 4, 3>(static_cast<const float*>(a.X) + (int64_t)m0 * a.ldx, a.ldx, a.T - m0,
                             static_cast<const float*>(a.W) + (int64_t)(a.v0 + n0) * a.ldw, a.ldw, cols, a.K, 0, ring, acc);
  const int c0 = 64 * wn + 4 * (lane >> 4);
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        if (c0 + 16 * j + v >= cols) acc[i][j][v] = -INFINITY;
        m = fmaxf(m, acc[i][j][v]);
      }
    m = quad_max(m);
    if (lane < 16) red[0][wn][WM * wm + 16 * i + l15] = m;
  }
  __syncthreads();
  float ref[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int r = WM * wm + 16 * i + l15, row = m0 + r;
    const bool in = row < a.T;
    const float m = fmaxf(red[0][0][r], red[0][1][r]) * kLog2e;
    const float have = !a.first && in ? a.ref[row] : 0.f;
    ref[i] = tile_reference(m, have, a.first);
    const float base = ref[i] == -INFINITY ? 0.f : ref[i];
    const int t = in ? a.target[row] - a.v0 - n0 - c0 : -1;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float e = exp2f(acc[i][j][v] * kLog2e - base);
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
    for (int i = 0; i < FM; ++i) {
      const int r = WM * wm + 16 * i + l15;
      if (m0 + r < a.T) a.stats[(int64_t)(m0 + r) * a.ld_stats + nt] = make_float2(ref[i], red[1][0][r] + red[1][1][r]);
    }
  }
}

// Range `part` of the piece's contraction, as in bf16.
template <int FM>
__global__ __launch_bounds__(256) void vocab_f32_grad_kernel(VocabArgs a) {
  constexpr int WM = 16 * FM, TM = 2 * WM;
  __shared__ __attribute__((aligned(1024))) char b0[kStage];
  __shared__ __attribute__((aligned(1024))) char b1[kStage];
  __shared__ __attribute__((aligned(1024))) char b2[kStage];
  const int n_m = (a.T + TM - 1) / TM, n_n = (a.K + 127) / 128, lin = tile_of(blockIdx.x, gridDim.x);
  const int part = lin / (n_m * n_n), tile = lin % (n_m * n_n);
  const int m0 = TM * (tile % n_m), n0 = 128 * (tile / n_m);
  const int c0 = part * a.split_len;
  // the piece's columns up to a whole tile hold zeros in P; W's rows past the piece are left out
  const int C = min(a.vn - c0, a.split_len);
  f32x4 acc[FM][4];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (C > 0)  // a short last piece ends before some ranges
    tile_nn_f32<FM>(static_cast<const float*>(a.P) + (int64_t)m0 * a.ldp + c0, a.ldp, a.T - m0,
                    static_cast<const float*>(a.W) + (int64_t)(a.v0 + c0) * a.ldw + n0, a.ldw, a.K - n0, C, b0, b1, b2, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int row = m0 + WM * wm + 16 * i + (lane & 15);
    if (row >= a.T) continue;
    const float f = a.first ? 0.f : a.alpha[row];
    float* o = a.O + ((int64_t)part * a.T + row) * a.K;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = n0 + 64 * wn + 16 * j + 4 * (lane >> 4);
      if (col >= a.K) continue;
      f32x4 x = acc[i][j];
      if (!a.first) x += *reinterpret_cast<const f32x4*>(o + col) * f;
      *reinterpret_cast<f32x4*>(o + col) = x;
    }
  }
}

}  // namespace

// Tiles of 64 rows fewer than the CUs are taken as tiles of 32 (64 rows against 5003 of 512: 19 us, 27 else).
hipError_t launch_vocab_f32_logits(const VocabArgs& a, int cus, hipStream_t s) {
  const int tm = (int64_t)a.n_ct * ((a.T + 63) / 64) <= cus ? 32 : vocab_f32_rows(a.T);
  const dim3 grid((unsigned)(a.n_ct * (int64_t)((a.T + tm - 1) / tm)));
  if (tm == 32) hipLaunchKernelGGL(vocab_f32_logits_kernel<1>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(vocab_f32_logits_kernel<2>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_vocab_f32_grad(const VocabArgs& a, hipStream_t s) {
  const int tm = vocab_f32_rows(a.T);
  const dim3 grid((unsigned)((int64_t)((a.T + tm - 1) / tm) * ((a.K + 127) / 128) * a.split));
  if (tm == 32) hipLaunchKernelGGL(vocab_f32_grad_kernel<1>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(vocab_f32_grad_kernel<2>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace dsv
