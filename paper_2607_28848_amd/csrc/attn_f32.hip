// attn_f32.hip -- fp32 attention (forward, dQ, dK and dV) on the fp32 matrix instructions.
//
// Every product is a 16 x 16 tile of v_mfma_f32_16x16x4_f32 (lane l holds A[l % 16][l / 16],
// B[l / 16][l % 16] and C[4 (l / 16) + v][l % 16]).  Which four contraction values a step takes is
// free as long as both operands agree, so a lane's values of a row of Q or K are D / 4 neighbours,
// and the scores of a tile, as the matrix core leaves them (four keys of one query per lane, or four
// queries of one key), are the second product's operand where they are.
//
// A workgroup has 16 queries (or keys) of one head, and its waves take 16 keys (queries) each by turns, straight
// from global memory (the rows that several workgroups read come from L2), and add their sums at the end: the
// batches of this mode are small, and what bounds them is the number of tiles that one wave walks one after the other,
// each with its loads' time in front.  Rows are read through descriptors, whose lanes need no pointers and no
// predicates of their own (with pointers the dK kernel of heads of 128 kept 215 registers in memory: 157 us against 58).
// Two samples of 96 and three of 157 rows, 8 heads on 2 of 64: forward 7.7 us, dQ 9.7, dK and dV 10.3, their join 4.0
// (four waves on 64 rows with staged tiles: 135 in all).  Two of 200 and three of 300, 16 on 2 of 128: 39, 46, 57, 5.
#include <hip/hip_runtime.h>

#include "attn.h"
#include "attn_plan.h"
#include "device_common.h"

namespace dsv {
namespace {

static_assert(kAttnF32Rows == 16, "rows of a tile");

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

// Descriptor over `n` rows (none if n <= 0) of head h from `row` on: what lies past them reads zeros.
template <int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const AttnView& t, int64_t row, int h, int n) {
  const uint64_t p = reinterpret_cast<uint64_t>(static_cast<const float*>(t.ptr) + row * t.row + h * t.head);
  const int64_t bytes = n > 0 ? ((int64_t)(min(n, 16) - 1) * t.row + D) * 4 : 0;
  const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p),
                 hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(lo | hi << 32), 0,
                                           __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}

// A lane's D / 4 values of row l % 16.
template <int D>
__device__ __forceinline__ void load_quarter(__amdgpu_buffer_rsrc_t t, int64_t stride, float (&x)[D / 4]) {
  const int at = (int)(threadIdx.x & 15) * (int)stride * 4 + (threadIdx.x >> 4 & 3) * D;
#pragma unroll
  for (int c = 0; c < D / 4; c += 4) {
    const f32x4 v = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(t, at + 4 * c, 0, 0));
#pragma unroll
    for (int e = 0; e < 4; ++e) x[c + e] = v[e];
  }
}

// C[row][col] = the dot product of the lanes' rows a (as rows of C) and b (as columns).
template <int D>
__device__ __forceinline__ f32x4 dot_tile(const float (&a)[D / 4], const float (&b)[D / 4]) {
  f32x4 c = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < D / 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s], b[s], c, 0, 0, 0);
  return c;
}

// Values [16 i + l % 16] of rows 4 (l / 16) + v.
template <int D>
__device__ __forceinline__ void load_columns(__amdgpu_buffer_rsrc_t t, int64_t stride, float (&x)[4][D / 16]) {
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int at = (int)(4 * (threadIdx.x >> 4 & 3) + v) * (int)stride * 4 + (threadIdx.x & 15) * 4;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
      x[v][i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(t, at + 64 * i, 0, 0));
  }
}

// acc[d][lane's column] += sum over the loaded rows of row[d] w[v].
template <int D>
__device__ __forceinline__ void add_rows(const float (&x)[4][D / 16], f32x4 w, f32x4 (&acc)[D / 16]) {
#pragma unroll
  for (int v = 0; v < 4; ++v)
#pragma unroll
    for (int t = 0; t < D / 16; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[v][t], w[v], acc[t], 0, 0, 0);
}

template <int D>
__device__ __forceinline__ void clear(f32x4 (&acc)[D / 16]) {
#pragma unroll
  for (int t = 0; t < D / 16; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// The waves' sums times f, through LDS: afterwards red[wave][row][d].
template <int D>
__device__ __forceinline__ void spread(const f32x4 (&acc)[D / 16], float f, float* red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* p = red + (wave * 16 + (lane & 15)) * (D + 4) + 4 * (lane >> 4);
#pragma unroll
  for (int t = 0; t < D / 16; ++t)
    *reinterpret_cast<f32x4*>(p + 16 * t) = f32x4{acc[t][0] * f, acc[t][1] * f, acc[t][2] * f, acc[t][3] * f};
}
// Elements c .. c + 3 of row r, the waves' parts added in order.
template <int D, int NW>
__device__ __forceinline__ f32x4 gather(const float* red, int r, int c) {
  f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < NW; ++w) x += *reinterpret_cast<const f32x4*>(red + (w * 16 + r) * (D + 4) + c);
  return x;
}

// The blocks of 16 keys that a tile of 16 queries walks, as the plan lays them down for the bf16 tiles.
template <bool WIN>
__device__ __forceinline__ AttnKeys<WIN> keys_of(const AttnArgs& a, const Seq& s, int qt, int& end) {
  const int off = s.kl - s.ql;
  end = min(s.kl, min(qt + 16, s.ql) + off);
  if (!WIN || end <= 0 || qt + off < a.window || qt + off - a.window + 1 <= a.sinks) return AttnKeys<WIN>(0, 0);
  const int sink = (a.sinks + 15) & ~15, shift = qt + off - a.window + 1 - sink;
  end -= shift;
  return AttnKeys<WIN>(sink, shift);
}

// 16 queries of one head over the keys that the last of them sees.
template <int D, bool WIN>
__global__ __launch_bounds__(256) void attn_f32_fwd_kernel(AttnArgs a) {
  constexpr int NW = 4;
  __shared__ __attribute__((aligned(16))) float red[NW * 16 * (D + 4)];
  __shared__ float ml[2][NW][16];
  const int item = blockIdx.x / a.hq, h = blockIdx.x % a.hq;
  const Seq s(a, a.items[2 * item]);
  const int qt = a.items[2 * item + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15;
  const int hk = h / a.group, q = qt + l15, off = s.kl - s.ql;  // the lane's query
  float qv[D / 4];
  load_quarter<D>(rows_of<D>(a.Q, (int64_t)s.q0 + qt, h, s.ql - qt), a.Q.row, qv);
  f32x4 acc[D / 16];
  clear<D>(acc);
  float m = -INFINITY, l = 0.f;
  int k_end;
  const AttnKeys<WIN> keys = keys_of<WIN>(a, s, qt, k_end);
  for (int b = 16 * wave; b < k_end; b += 16 * NW) {
    const int kt = keys.at(b), n = keys.end(a, b, s.kl) - kt;
    const uint32_t back = keys.back(a, b);
    float kv[D / 4], vv[4][D / 16];
    load_quarter<D>(rows_of<D>(a.K, (int64_t)s.k0 + kt, hk, n), a.K.row, kv);
    load_columns<D>(rows_of<D>(a.V, (int64_t)s.k0 + kt, hk, n), a.V.row, vv);
    f32x4 x = dot_tile<D>(kv, qv);
    float mx = m;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      x[v] = AttnKeys<WIN>::sees(a, back, WIN ? max(q + off, -1) : q + off, kt + 4 * (lane >> 4) + v) ? x[v] * a.scale : -INFINITY;
      mx = fmaxf(mx, x[v]);
    }
    mx = quad_max(mx);
    const float ref = mx == -INFINITY ? 0.f : mx;  // nothing seen yet: every term below is exp(-inf) = 0
    const float f = expf(m - ref);
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) sum += x[v] = expf(x[v] - ref);
    l = l * f + quad_sum(sum);
    m = mx;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) acc[t] *= f;
    add_rows<D>(vv, x, acc);
  }
  if (lane < 16) {
    ml[0][wave][l15] = m;
    ml[1][wave][l15] = l;
  }
  __syncthreads();
  // the waves' sums at one reference
  float ref = -INFINITY, total = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) ref = fmaxf(ref, ml[0][w][l15]);
#pragma unroll
  for (int w = 0; w < NW; ++w)
    total += ml[0][w][l15] == -INFINITY ? ml[1][w][l15] : ml[1][w][l15] * expf(ml[0][w][l15] - ref);
  spread<D>(acc, (m == -INFINITY ? 1.f : expf(m - ref)) * (total == 0.f ? 0.f : 1.f / total), red);
  if (a.lse && wave == 0 && lane < 16 && q < s.ql)
    a.lse[(int64_t)h * a.n_q + s.q0 + q] = total == 0.f ? -INFINITY : ref + logf(total);
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * D / 4; i += 64 * NW) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    if (qt + r < s.ql)
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.O.ptr) + ((int64_t)s.q0 + qt + r) * a.O.row + h * a.O.head + c) =
          gather<D, NW>(red, r, c);
  }
}

// dQ of 16 queries of one head, and delta = do . o for the launch of dK and dV (none where a.delta is null).
template <int D, bool WIN, int NW>
__device__ __forceinline__ void dq_tile(const AttnArgs& a, const int32_t* items, int block, float* red) {
  const int item = block / a.hq, h = block % a.hq;
  const Seq s(a, items[2 * item]);
  const int qt = items[2 * item + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15;
  const int hk = h / a.group, q = qt + l15, off = s.kl - s.ql;
  const bool in = q < s.ql;
  float qv[D / 4], dv[D / 4], dot = 0.f;
  load_quarter<D>(rows_of<D>(a.Q, (int64_t)s.q0 + qt, h, s.ql - qt), a.Q.row, qv);
  load_quarter<D>(rows_of<D>(a.dO, (int64_t)s.cq + qt, h, s.ql - qt), a.dO.row, dv);
  {
    float ov[D / 4];
    load_quarter<D>(rows_of<D>(a.O, (int64_t)s.q0 + qt, h, s.ql - qt), a.O.row, ov);
#pragma unroll
    for (int c = 0; c < D / 4; ++c) dot += dv[c] * ov[c];
  }
  const float delta = quad_sum(dot);
  if (in && wave == 0 && lane < 16 && a.delta) a.delta[h * a.train_q + s.cq + q] = delta;
  const float lse = in ? exp_from(a.lse[(int64_t)h * a.n_q + s.q0 + q]) : 0.f;
  f32x4 acc[D / 16];
  clear<D>(acc);
  int k_end;
  const AttnKeys<WIN> keys = keys_of<WIN>(a, s, qt, k_end);
  for (int b = 16 * wave; b < k_end; b += 16 * NW) {
    const int kt = keys.at(b), n = keys.end(a, b, s.kl) - kt;
    const uint32_t back = keys.back(a, b);
    float kv[D / 4], vv[D / 4], kc[4][D / 16];
    const auto kr = rows_of<D>(a.K, (int64_t)s.k0 + kt, hk, n);
    const auto vr = rows_of<D>(a.V, (int64_t)s.k0 + kt, hk, n);
    load_quarter<D>(kr, a.K.row, kv);
    load_quarter<D>(vr, a.V.row, vv);
    load_columns<D>(kr, a.K.row, kc);
    const f32x4 x = dot_tile<D>(kv, qv), dp = dot_tile<D>(vv, dv);
    f32x4 ds;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const bool seen = AttnKeys<WIN>::sees(a, back, WIN ? max(q + off, -1) : q + off, kt + 4 * (lane >> 4) + v);
      ds[v] = seen ? expf(x[v] * a.scale - lse) * (dp[v] - delta) * a.scale : 0.f;
    }
    add_rows<D>(kc, ds, acc);
  }
  if (lse == INFINITY) clear<D>(acc);  // 0 times an infinite key
  spread<D>(acc, 1.f, red);
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * D / 4; i += 64 * NW) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    if (qt + r < s.ql)
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.dQ.ptr) + ((int64_t)s.cq + qt + r) * a.dQ.row + h * a.dQ.head + c) =
          gather<D, NW>(red, r, c);
  }
}

template <int D>
__global__ __launch_bounds__(256) void attn_f32_dq_kernel(AttnArgs a) {
  constexpr int NW = 4;
  __shared__ __attribute__((aligned(16))) float red[NW * 16 * (D + 4)];
  dq_tile<D, false, NW>(a, a.items, blockIdx.x, red);
}

// dK and dV of 16 keys of one key head over the queries that see the first of them, of all the key head's query
// heads (so the sums over them need no atomics), or of one of a.parts ranges of them, whose sums go to the workspace
// (32 us whole, 10.3 and 4.0 for the join in four parts: the first batch above).
// WIN: in one launch with dq_tile, so delta is formed here as it is there; the parts are ranges of all the tile's steps, and
// the tiles behind the first a.cut are whole.
template <int D, bool WIN, int NW>
__device__ __forceinline__ void dk_tile(const AttnArgs& a, int block, float* red) {
  const int whole = WIN ? block - a.cut * a.hkv * a.parts : -1, parts = whole < 0 ? a.parts : 1;
  const int part = whole < 0 ? block % parts : 0, tile = whole < 0 ? block / parts : a.cut * a.hkv + whole;
  const int item = tile / a.hkv, g = tile % a.hkv;
  const Seq s(a, a.items[2 * item]);
  const int k0 = a.items[2 * item + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15;
  const int k = k0 + l15, off = s.kl - s.ql;  // the lane's key
  float kv[D / 4], vv[D / 4];
  load_quarter<D>(rows_of<D>(a.K, (int64_t)s.k0 + k0, g, s.kl - k0), a.K.row, kv);
  load_quarter<D>(rows_of<D>(a.V, (int64_t)s.k0 + k0, g, s.kl - k0), a.V.row, vv);
  f32x4 dk[D / 16], dv[D / 16];
  clear<D>(dk);
  clear<D>(dv);
  const int q_first = max(0, k0 - off);
  // the keys' last query: with a window that of the last key, but the sinks are seen to the end
  const int q_end = WIN && k0 >= a.sinks ? (int)min((int64_t)s.ql, (int64_t)min(k0 + 16, s.kl) - 1 - off + a.window) : s.ql;
  const int per_head = q_first < q_end ? (q_end - q_first + 15) / 16 : 0;
  const int64_t all = WIN ? (int64_t)per_head * a.group : a.group;
  const int step = WIN ? 1 : per_head, n0 = (int)(part * all / parts) * step, n1 = (int)((part + 1) * all / parts) * step;
  for (int n = n0 + wave; n < n1; n += NW) {
    const int h = g * a.group + n / per_head, qt = q_first + n % per_head * 16;
    float qv[D / 4], ov[D / 4], qc[4][D / 16], oc[4][D / 16], lse[4], delta[4];
    const auto qr = rows_of<D>(a.Q, (int64_t)s.q0 + qt, h, s.ql - qt);
    const auto dr = rows_of<D>(a.dO, (int64_t)s.cq + qt, h, s.ql - qt);
    load_quarter<D>(qr, a.Q.row, qv);
    load_quarter<D>(dr, a.dO.row, ov);
    float mine = 0.f;  // do . o of row l % 16
    if constexpr (WIN) {
      float rows[D / 4];
      load_quarter<D>(rows_of<D>(a.O, (int64_t)s.q0 + qt, h, s.ql - qt), a.O.row, rows);
#pragma unroll
      for (int c = 0; c < D / 4; ++c) mine += ov[c] * rows[c];
      mine = quad_sum(mine);
    }
    load_columns<D>(dr, a.dO.row, oc);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int q = min(qt + 4 * (lane >> 4) + v, s.ql - 1);
      lse[v] = a.lse[(int64_t)h * a.n_q + s.q0 + q];
      delta[v] = WIN ? __shfl(mine, 4 * (lane >> 4) + v) : a.delta[h * a.train_q + s.cq + q];
    }
    const f32x4 x = dot_tile<D>(qv, kv);
    // Q's columns take the registers of its rows (with heads of 128 both do not fit)
    if constexpr (!WIN || D == 128) __builtin_amdgcn_sched_barrier(0);
    load_columns<D>(qr, a.Q.row, qc);
    const f32x4 dp = dot_tile<D>(ov, vv);
    f32x4 p, ds;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int q = qt + 4 * (lane >> 4) + v;
      const bool seen = q < s.ql && AttnKeys<WIN>::sees(a, a.window, WIN ? max(q + off, -1) : q + off, k) && lse[v] != -INFINITY;  // as exp_from(), which spills here
      p[v] = seen ? expf(x[v] * a.scale - lse[v]) : 0.f;
      ds[v] = seen ? p[v] * (dp[v] - delta[v]) * a.scale : 0.f;
    }
    add_rows<D>(oc, p, dv);
    add_rows<D>(qc, ds, dk);
  }
  if (AttnKeys<WIN>::unseen(a, off, k)) {  // 0 times an infinite value
    clear<D>(dk);
    clear<D>(dv);
  }
  auto put = [&](const f32x4 (&acc)[D / 16], const AttnView& t, int half) {
    __syncthreads();
    spread<D>(acc, 1.f, red);
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * D / 4; i += 64 * NW) {
      const int r = i / (D / 4), c = 4 * (i % (D / 4));
      const f32x4 x = gather<D, NW>(red, r, c);
      if (parts > 1)
        *reinterpret_cast<f32x4*>(a.part_o + (((int64_t)block * 2 + half) * 16 + r) * D + c) = x;
      else if (k0 + r < s.kl)
        *reinterpret_cast<f32x4*>(static_cast<float*>(t.ptr) + ((int64_t)s.ck + k0 + r) * t.row + g * t.head + c) = x;
    }
  };
  put(dk, a.dK, 0);
  put(dv, a.dV, 1);
}

template <int D>
__global__ __launch_bounds__(512) void attn_f32_dk_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) float red[8 * 16 * (D + 4)];
  dk_tile<D, false, 8>(a, blockIdx.x, red);
}

// Both gradients of a plan with a window: a.first_groups workgroups for dK and dV, then those of dQ (a.first_join's items).
// The key tiles are short there but for the sinks', and two launches would leave most of the card to the other's latency:
// three samples of 357 rows, 8 heads on 2 of 64, window 101: 13.6 and 21 us one after the other.
template <int D>
__global__ __launch_bounds__(256) void attn_f32_grad_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) float red[4 * 16 * (D + 4)];
  if ((int)blockIdx.x < a.first_groups) dk_tile<D, true, 4>(a, blockIdx.x, red);
  else dq_tile<D, true, 4>(a, a.first_join, blockIdx.x - a.first_groups, red);
}

// dK and dV of 16 keys from the parts' sums, in order: one workgroup a tile and gradient.
template <int D>
__global__ __launch_bounds__(256) void attn_f32_dk_join_kernel(AttnArgs a) {
  const int half = blockIdx.x & 1, tile = blockIdx.x >> 1, item = tile / a.hkv, g = tile % a.hkv;
  const Seq s(a, a.items[2 * item]);
  const int k0 = a.items[2 * item + 1];
  const AttnView& t = half ? a.dV : a.dK;
  for (int i = threadIdx.x; i < 16 * D / 4; i += 256) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    if (k0 + r >= s.kl) break;
    const float* p = a.part_o + (((int64_t)tile * a.parts * 2 + half) * 16 + r) * D + c;
    f32x4 x = *reinterpret_cast<const f32x4*>(p);
    for (int n = 1; n < a.parts; ++n) x += *reinterpret_cast<const f32x4*>(p + (int64_t)n * 32 * D);
    *reinterpret_cast<f32x4*>(static_cast<float*>(t.ptr) + ((int64_t)s.ck + k0 + r) * t.row + g * t.head + c) = x;
  }
}

}  // namespace

hipError_t launch_attn_f32_fwd(const AttnArgs& a, bool windowed, hipStream_t s) {
  if (a.n_items <= 0) return hipSuccess;
  const dim3 grid((unsigned)(a.n_items * (int64_t)a.hq));
  if (windowed && a.d == 64) hipLaunchKernelGGL((attn_f32_fwd_kernel<64, true>), grid, dim3(256), 0, s, a);
  else if (windowed) hipLaunchKernelGGL((attn_f32_fwd_kernel<128, true>), grid, dim3(256), 0, s, a);
  else if (a.d == 64) hipLaunchKernelGGL((attn_f32_fwd_kernel<64, false>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attn_f32_fwd_kernel<128, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_attn_f32_dq(const AttnArgs& a, hipStream_t s) {
  if (a.n_items <= 0) return hipSuccess;
  const dim3 grid((unsigned)(a.n_items * (int64_t)a.hq));
  if (a.d == 64) hipLaunchKernelGGL(attn_f32_dq_kernel<64>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(attn_f32_dq_kernel<128>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

namespace {

// The join of dK's and dV's parts, where there are some.
hipError_t join_parts(const AttnArgs& a, int64_t tiles, hipStream_t s) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1 || tiles == 0) return e;
  if (a.d == 64) hipLaunchKernelGGL(attn_f32_dk_join_kernel<64>, dim3((unsigned)(2 * tiles)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(attn_f32_dk_join_kernel<128>, dim3((unsigned)(2 * tiles)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_f32_dk(const AttnArgs& a, hipStream_t s) {
  if (a.n_items <= 0) return hipSuccess;
  const int64_t tiles = a.n_items * (int64_t)a.hkv;
  const dim3 grid((unsigned)(tiles * a.parts));
  if (a.d == 64) hipLaunchKernelGGL(attn_f32_dk_kernel<64>, grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL(attn_f32_dk_kernel<128>, grid, dim3(512), 0, s, a);
  return join_parts(a, tiles, s);
}

hipError_t launch_attn_f32_grad(AttnArgs a, const int32_t* dq_items, int32_t n_dq, hipStream_t s) {
  const int64_t cut = a.cut * (int64_t)a.hkv;
  a.first_groups = (int32_t)(cut * a.parts + (a.n_items - a.cut) * (int64_t)a.hkv);
  a.first_join = dq_items;
  a.delta = nullptr;
  const dim3 grid((unsigned)(a.first_groups + (int64_t)n_dq * a.hq));
  if (grid.x == 0) return hipSuccess;
  if (a.d == 64) hipLaunchKernelGGL(attn_f32_grad_kernel<64>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(attn_f32_grad_kernel<128>, grid, dim3(256), 0, s, a);
  return join_parts(a, cut, s);
}

}  // namespace dsv
