// attn_f32.hip -- fp32 attention (forward, dQ, dK and dV) on the fp32 matrix instructions.
//
// Every product is a 16 x 16 tile of v_mfma_f32_16x16x4_f32 (lane l holds A[l % 16][l / 16],
// B[l / 16][l % 16] and C[4 (l / 16) + v][l % 16]).  Which four contraction values a step takes is
// free as long as both operands agree, so a lane's values of a row of Q or K are D / 4 neighbours,
// and the scores of a tile, as the matrix core leaves them (four keys of one query per lane, or four
// queries of one key), are the second product's operand where they are.
//
// Bounds: the matrix core (two products of D = 64 at 16 x 16 tiles need one LDS read per step) and,
// for the small batches that this mode serves, the latency of one tile after the other.
#include <hip/hip_runtime.h>

#include "attn.h"
#include "attn_plan.h"
#include "device_common.h"

namespace dsv {
namespace {

constexpr int kTK = 32;  // rows of the staged tiles (keys in forward and dQ, queries in dK and dV)

__device__ __forceinline__ float quad_max(float x) {  // over the four lanes l, l ^ 16, l ^ 32, l ^ 48
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

struct Seq {
  int q0, ql, k0, kl, cq, ck;
  __device__ __forceinline__ Seq(const AttnArgs& a, int i) {
    const int32_t* w = a.seqs + (int64_t)i * kAttnSeqWords;
    q0 = w[0], ql = w[1], k0 = w[2], kl = w[3], cq = w[4], ck = w[5];
  }
};

// A lane's D / 4 values of a row (zeros where the row does not exist).
template <int D>
__device__ __forceinline__ void load_quarter(const AttnView& t, int64_t row, int h, bool in, float (&x)[D / 4]) {
  const float* p = static_cast<const float*>(t.ptr) + row * t.row + h * t.head + (threadIdx.x >> 4 & 3) * (D / 4);
#pragma unroll
  for (int c = 0; c < D / 4; c += 4) {
    const f32x4 v = in ? *reinterpret_cast<const f32x4*>(p + c) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) x[c + e] = v[e];
  }
}

// Rows [r0, r0 + kTK) of a head into LDS, rows from r_end on as zeros.
template <int D>
__device__ __forceinline__ void stage(const AttnView& t, int64_t base, int r0, int r_end, int h, float* lds) {
  constexpr int LD = D + 4;
  const float* p = static_cast<const float*>(t.ptr) + h * t.head;
  for (int i = threadIdx.x; i < kTK * D / 4; i += 256) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    const bool in = r0 + r < r_end;
    const f32x4 v = in ? *reinterpret_cast<const f32x4*>(p + (base + r0 + r) * t.row + c) : f32x4{0.f, 0.f, 0.f, 0.f};
    *reinterpret_cast<f32x4*>(lds + r * LD + c) = v;
  }
}

// C[row][col] = sum over D of the staged rows 16 sub .. and the lane's own row x.
template <int D>
__device__ __forceinline__ f32x4 dot_tile(const float* lds, int sub, const float (&x)[D / 4]) {
  const int lane = threadIdx.x & 63;
  const float* p = lds + (16 * sub + (lane & 15)) * (D + 4) + (lane >> 4) * (D / 4);
  f32x4 c = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < D / 4; s += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + s);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], x[s + e], c, 0, 0, 0);
  }
  return c;
}

// acc[d][lane's column] += sum over the staged rows 16 sub + 4 (l / 16) + v of row[d] w[v].
template <int D>
__device__ __forceinline__ void add_rows(const float* lds, int sub, f32x4 w, f32x4 (&acc)[D / 16]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float* p = lds + (16 * sub + 4 * (lane >> 4) + v) * (D + 4) + (lane & 15);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[16 * t], w[v], acc[t], 0, 0, 0);
  }
}

template <int D>
__device__ __forceinline__ void store_row(const AttnView& t, int64_t row, int h, const f32x4 (&acc)[D / 16], float f) {
  float* p = static_cast<float*>(t.ptr) + row * t.row + h * t.head + 4 * (threadIdx.x >> 4 & 3);
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
    *reinterpret_cast<f32x4*>(p + 16 * i) = f32x4{acc[i][0] * f, acc[i][1] * f, acc[i][2] * f, acc[i][3] * f};
}

// 64 queries of one head, 16 a wave, over the keys that the last of them sees.
template <int D>
__global__ __launch_bounds__(256) void attn_f32_fwd_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) float ks[kTK * (D + 4)], vs[kTK * (D + 4)];
  const int item = blockIdx.x / a.hq, h = blockIdx.x % a.hq;
  const Seq s(a, a.items[2 * item]);
  const int qt = a.items[2 * item + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15;
  const int q = qt + 16 * wave + l15;  // the lane's query
  const int off = s.kl - s.ql;
  float qv[D / 4];
  load_quarter<D>(a.Q, (int64_t)s.q0 + q, h, q < s.ql, qv);
  f32x4 acc[D / 16];
#pragma unroll
  for (int t = 0; t < D / 16; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  const int k_end = min(s.kl, min(qt + kAttnF32Rows, s.ql) + off);
  for (int kt = 0; kt < k_end; kt += kTK) {
    __syncthreads();
    stage<D>(a.K, s.k0, kt, s.kl, h / a.group, ks);
    stage<D>(a.V, s.k0, kt, s.kl, h / a.group, vs);
    __syncthreads();
    f32x4 x[kTK / 16];
    float mx = m;
#pragma unroll
    for (int u = 0; u < kTK / 16; ++u) {
      x[u] = dot_tile<D>(ks, u, qv);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        x[u][v] = kt + 16 * u + 4 * (lane >> 4) + v <= q + off ? x[u][v] * a.scale : -INFINITY;
        mx = fmaxf(mx, x[u][v]);
      }
    }
    mx = quad_max(mx);
    const float ref = mx == -INFINITY ? 0.f : mx;  // nothing seen yet: every term below is exp(-inf) = 0
    const float f = expf(m - ref);
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < kTK / 16; ++u)
#pragma unroll
      for (int v = 0; v < 4; ++v) sum += x[u][v] = expf(x[u][v] - ref);
    l = l * f + quad_sum(sum);
    m = mx;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) acc[t] *= f;
#pragma unroll
    for (int u = 0; u < kTK / 16; ++u) add_rows<D>(vs, u, x[u], acc);
  }
  if (q >= s.ql) return;
  store_row<D>(a.O, (int64_t)s.q0 + q, h, acc, l > 0.f ? 1.f / l : l);  // l is 0 where no key is seen, NaN stays NaN
  if (a.lse && lane < 16) a.lse[(int64_t)h * a.n_q + s.q0 + q] = l > 0.f ? m + logf(l) : l == 0.f ? -INFINITY : l;
}

// dQ of 64 queries of one head, and delta = do . o for the launch of dK and dV.
template <int D>
__global__ __launch_bounds__(256) void attn_f32_dq_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) float ks[kTK * (D + 4)], vs[kTK * (D + 4)];
  const int item = blockIdx.x / a.hq, h = blockIdx.x % a.hq;
  const Seq s(a, a.items[2 * item]);
  const int qt = a.items[2 * item + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15;
  const int q = qt + 16 * wave + l15;
  const int off = s.kl - s.ql;
  const bool in = q < s.ql;
  float qv[D / 4], dv[D / 4], ov[D / 4];
  load_quarter<D>(a.Q, (int64_t)s.q0 + q, h, in, qv);
  load_quarter<D>(a.dO, (int64_t)s.cq + q, h, in, dv);
  load_quarter<D>(a.O, (int64_t)s.q0 + q, h, in, ov);
  float dot = 0.f;
#pragma unroll
  for (int c = 0; c < D / 4; ++c) dot += dv[c] * ov[c];
  const float delta = quad_sum(dot);
  if (in && lane < 16) a.delta[h * a.train_q + s.cq + q] = delta;
  const float lse = in ? a.lse[(int64_t)h * a.n_q + s.q0 + q] : 0.f;
  f32x4 acc[D / 16];
#pragma unroll
  for (int t = 0; t < D / 16; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int k_end = min(s.kl, min(qt + kAttnF32Rows, s.ql) + off);
  for (int kt = 0; kt < k_end; kt += kTK) {
    __syncthreads();
    stage<D>(a.K, s.k0, kt, s.kl, h / a.group, ks);
    stage<D>(a.V, s.k0, kt, s.kl, h / a.group, vs);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kTK / 16; ++u) {
      const f32x4 x = dot_tile<D>(ks, u, qv), dp = dot_tile<D>(vs, u, dv);
      f32x4 ds;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const bool seen = kt + 16 * u + 4 * (lane >> 4) + v <= q + off;
        ds[v] = seen ? expf(x[v] * a.scale - lse) * (dp[v] - delta) * a.scale : 0.f;
      }
      add_rows<D>(ks, u, ds, acc);
    }
  }
  if (in) store_row<D>(a.dQ, (int64_t)s.cq + q, h, acc, 1.f);
}

// dK and dV of 64 keys of one key head, 16 a wave, over the queries that see the first of them, the
// key head's query heads one after the other (so the sums over them need no atomics).
template <int D>
__global__ __launch_bounds__(256) void attn_f32_dk_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) float qs[kTK * (D + 4)], os[kTK * (D + 4)];
  __shared__ float st[2][kTK];  // lse and delta of the staged queries
  const int item = blockIdx.x / a.hkv, g = blockIdx.x % a.hkv;
  const Seq s(a, a.items[2 * item]);
  const int k0 = a.items[2 * item + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15;
  const int k = k0 + 16 * wave + l15;  // the lane's key
  const int off = s.kl - s.ql;
  const bool in = k < s.kl;
  float kv[D / 4], vv[D / 4];
  load_quarter<D>(a.K, (int64_t)s.k0 + k, g, in, kv);
  load_quarter<D>(a.V, (int64_t)s.k0 + k, g, in, vv);
  f32x4 dk[D / 16], dv[D / 16];
#pragma unroll
  for (int t = 0; t < D / 16; ++t) dk[t] = dv[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int q_first = max(0, k0 - off);
  for (int h = g * a.group; h < (g + 1) * a.group; ++h) {
    for (int qt = q_first; qt < s.ql; qt += kTK) {
      __syncthreads();
      stage<D>(a.Q, s.q0, qt, s.ql, h, qs);
      stage<D>(a.dO, s.cq, qt, s.ql, h, os);
      if (threadIdx.x < kTK) {
        const int q = min(qt + (int)threadIdx.x, s.ql - 1);
        st[0][threadIdx.x] = a.lse[(int64_t)h * a.n_q + s.q0 + q];
        st[1][threadIdx.x] = a.delta[h * a.train_q + s.cq + q];
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kTK / 16; ++u) {
        const f32x4 x = dot_tile<D>(qs, u, kv), dp = dot_tile<D>(os, u, vv);
        f32x4 p, ds;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int r = 16 * u + 4 * (lane >> 4) + v, q = qt + r;
          p[v] = q < s.ql && k <= q + off ? expf(x[v] * a.scale - st[0][r]) : 0.f;
          ds[v] = q < s.ql && k <= q + off ? p[v] * (dp[v] - st[1][r]) * a.scale : 0.f;
        }
        add_rows<D>(os, u, p, dv);
        add_rows<D>(qs, u, ds, dk);
      }
    }
  }
  if (!in) return;
  store_row<D>(a.dK, (int64_t)s.ck + k, g, dk, 1.f);
  store_row<D>(a.dV, (int64_t)s.ck + k, g, dv, 1.f);
}

}  // namespace

hipError_t launch_attn_f32_fwd(const AttnArgs& a, hipStream_t s) {
  if (a.n_items <= 0) return hipSuccess;
  const dim3 grid((unsigned)(a.n_items * (int64_t)a.hq));
  if (a.d == 64) hipLaunchKernelGGL(attn_f32_fwd_kernel<64>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(attn_f32_fwd_kernel<128>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_attn_f32_dq(const AttnArgs& a, hipStream_t s) {
  if (a.n_items <= 0) return hipSuccess;
  const dim3 grid((unsigned)(a.n_items * (int64_t)a.hq));
  if (a.d == 64) hipLaunchKernelGGL(attn_f32_dq_kernel<64>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(attn_f32_dq_kernel<128>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_attn_f32_dk(const AttnArgs& a, hipStream_t s) {
  if (a.n_items <= 0) return hipSuccess;
  const dim3 grid((unsigned)(a.n_items * (int64_t)a.hkv));
  if (a.d == 64) hipLaunchKernelGGL(attn_f32_dk_kernel<64>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(attn_f32_dk_kernel<128>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace dsv
