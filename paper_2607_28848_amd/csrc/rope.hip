// rope.hip -- norms of queries and keys and the position rotation, forward and backward (gfx950), and the C entry points.
//
// A head's vector is held by D / 16 lanes, 16 elements each, as two chunks of 8 (16 or 32 bytes a load): lane l has
// chunks l and l + rotated / 16, or 2 l and 2 l + 1 where neighbours turn together, so both elements of a pair lie in
// one lane and in both orders the lane's pairs are i = 8 l .. 8 l + 7.  A wave takes 64 / (D / 16) heads of one row at a
// time.  The row's cosines and sines are formed once a wave, one angle a lane, and go to the lanes through LDS.
//
// Memory's rate bounds both directions: 16384 rows of 64 + 8 heads of 128 and the values, bf16, 127 us (5.3 TB/s); 6144 of 32 + 8
// 34 us (4.4 TB/s); 8192 rows of gradients of 32 + 8 63 us (4.0 TB/s).  A few rows cost a launch: 8 rows 3.3 us.  Loading the
// next heads before the present ones are turned was slower (44 us for the 6144 rows: more registers, fewer waves).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "device_common.h"
#include "view.h"

namespace dsv {
namespace {

// The backward of the queries or the keys.
struct RopeBack {
  int32_t heads, split, groups;  // waves a row, workgroups
  const float* weight;
  AttnView dy, x, dx;
  float* dw;  // nullptr: not wanted
};

struct RopeArgs {
  int32_t n;            // rows of the forward's tensors
  int32_t hq, hkv, hv;  // hv: heads of V that are copied (0: none)
  int32_t rot;
  int32_t split;        // waves a row
  float eps;
  const int32_t* pos;
  const double* freq;
  const float *qw, *kw;
  AttnView Q, K, V, Qo, Ko, Vo;
  const int32_t* slots;  // nullptr: row i to row i
  int32_t n_slots;
  // backward
  int32_t n_rows;
  const int32_t* rows;  // nullptr: row i
  RopeBack q, k;
  float* part;          // [groups of both][D] sums of the weights' gradients (nullptr: none)
};

template <typename T>
struct Chunk;  // eight elements as they lie in memory
template <>
struct Chunk<uint16_t> {
  u32x4 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<u32x4*>(p) = v; }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(v[i] << 16), x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
  __device__ __forceinline__ void set(const float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = f2bf2(x[2 * i], x[2 * i + 1]);
  }
};
template <>
struct Chunk<float> {
  f32x4 v[2];
  __device__ __forceinline__ void load(const float* p) {
    v[0] = *reinterpret_cast<const f32x4*>(p), v[1] = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ __forceinline__ void store(float* p) const {
    *reinterpret_cast<f32x4*>(p) = v[0], *reinterpret_cast<f32x4*>(p + 4) = v[1];
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i / 4][i % 4];
  }
  __device__ __forceinline__ void set(const float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i / 4][i % 4] = x[i];
  }
};

// Cosine and sine of pos * freq radians.  The frequency in quarter turns is held in two 64-bit parts, and the angle less its
// whole quarters, in [-1/2, 1/2], is one fma, so nothing is rounded before the reduction (an angle of 2^31 quarters in 64 bits
// is up to 2.4e-7 of one off); what is left, at most pi / 4, goes through the Taylor series of both (next terms below 3e-9 and
// 2e-10 of the value).
__device__ __forceinline__ float2 turn_of(int pos, double freq) {
  constexpr double kHigh = 0.6366197723675814, kLow = -3.935735335036497e-17;  // 2 / pi
  const double f = freq * kHigh, f_low = fma(freq, kHigh, -f) + freq * kLow;
  const double p = pos, whole = rint(p * f);
  const float x = (float)((fma(p, f, -whole) + p * f_low) * 1.57079632679489661923), x2 = x * x;
  const float s = x + x * x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880))));
  const float c = 1.f + x2 * (-0.5f + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 + x2 * (-1.f / 3628800)))));
  const int turn = (int)(whole - 4. * floor(whole * 0.25));  // 0 to 3
  const float a = turn & 1 ? s : c, b = turn & 1 ? c : s;    // cosine and sine but for their signs
  return make_float2(turn == 1 || turn == 2 ? -a : a, turn >= 2 ? -b : b);
}

// The sum over the LPH lanes of a head.
template <int LPH>
__device__ __forceinline__ float head_sum(float x) {
  auto add = [&](auto ctrl) {
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  add(std::integral_constant<int, 0xB1>{});   // quads: lanes 1 0 3 2
  add(std::integral_constant<int, 0x4E>{});   // lanes 2 3 0 1
  if constexpr (LPH == 8) add(std::integral_constant<int, 0x141>{});  // eights reversed: the other quad's sum
  return x;
}

// A lane's place in its wave's heads.
template <int D>
struct Lane {
  static constexpr int LPH = D / 16, HPW = 64 / LPH;
  int l, g, a, b;  // lane of the head, head, first elements of the two chunks
  bool turns;
  __device__ __forceinline__ Lane(int rot, bool next) {
    const int lane = threadIdx.x & 63, nr = rot / 16;
    l = lane % LPH, g = lane / LPH;
    turns = l < nr;
    const bool half = turns && !next;
    a = half ? 8 * l : 16 * l;
    b = half ? 8 * (l + nr) : 16 * l + 8;
  }
};

// cos and sin of the row's pairs, for the lane's own eight; cs: the wave's room.
template <int D>
__device__ __forceinline__ void row_turns(const RopeArgs& a, int pos, const Lane<D>& at, float (*cs)[64], float (&c)[8],
                                          float (&s)[8]) {
  const int lane = threadIdx.x & 63;
  asm volatile("" ::: "memory");  // the row before has read its own (a wave's LDS accesses run in order)
  if (lane < a.rot / 2) {
    const float2 t = turn_of(pos, a.freq[lane]);
    cs[0][lane] = t.x, cs[1][lane] = t.y;
  }
  asm volatile("" ::: "memory");
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(&cs[0][8 * at.l + i]), y = *reinterpret_cast<const f32x4*>(&cs[1][8 * at.l + i]);
#pragma unroll
    for (int e = 0; e < 4; ++e) c[i + e] = x[e], s[i + e] = y[e];
  }
}

// The lane's pairs turned (BACK: the other way): x[0 .. 8) and x[8 .. 16) are its chunks.
template <bool NEXT, bool BACK = false>
__device__ __forceinline__ void turn(float (&x)[16], const float (&c)[8], const float (&s)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int a = NEXT ? 2 * i : i, b = NEXT ? 2 * i + 1 : 8 + i;
    const float u = x[a], v = x[b];
    if constexpr (BACK) x[a] = u * c[i] + v * s[i], x[b] = v * c[i] - u * s[i];
    else x[a] = u * c[i] - v * s[i], x[b] = v * c[i] + u * s[i];
  }
}

template <int D>
__device__ __forceinline__ void weight_of(const float* w, const Lane<D>& at, float (&x)[16]) {
  Chunk<float> a, b;
  a.load(w + at.a), b.load(w + at.b);
  a.get(x), b.get(x + 8);
}

__device__ __forceinline__ float square_sum(const float (&x)[16]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += x[i] * x[i];
  return s;
}

// 1 / sqrt(x) to half a step and a little: the instruction's result, off by up to a whole one, and a Newton step whose
// residue 1 - x r^2 is formed without rounding x r.  The kernels wait for memory meanwhile.
__device__ __forceinline__ float inverse_root(float x) {
  const float r = __builtin_amdgcn_rsqf(x), t = x * r;
  const float rest = fmaf(-fmaf(x, r, -t), r, fmaf(-t, r, 1.f));
  return x < INFINITY ? fmaf(0.5f * rest, r, r) : r;
}

template <typename T>
__device__ __forceinline__ T* element(const AttnView& t, int64_t row, int h) {
  return static_cast<T*>(t.ptr) + row * t.row + h * t.head;
}

// Heads of a row: queries, keys, values, one list; wave `part` of `split` takes every split-th 64 / (D / 16) of them.
template <typename T, int D, bool NEXT>
__global__ __launch_bounds__(256) void rope_fwd_kernel(RopeArgs a) {
  __shared__ __attribute__((aligned(16))) float cs[4][2][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t w = (int64_t)blockIdx.x * 4 + wave;
  const int row = (int)(w / a.split), part = (int)(w % a.split);
  if (row >= a.n) return;
  const Lane<D> at(a.rot, NEXT);
  constexpr int HPW = Lane<D>::HPW;
  const int heads = a.hq + a.hkv + a.hv, slot = a.slots ? a.slots[row] : row;
  const bool kept = !a.slots || (uint32_t)slot < (uint32_t)a.n_slots;
  float c[8], s[8];
  row_turns<D>(a, a.rot ? a.pos[row] : 0, at, cs[wave], c, s);
  for (int h0 = part * HPW; h0 < heads; h0 += a.split * HPW) {
    const int h = h0 + at.g;
    if (h >= heads) continue;
    const bool is_q = h < a.hq, is_v = h >= a.hq + a.hkv;
    const int hh = is_q ? h : is_v ? h - a.hq - a.hkv : h - a.hq;
    const T* x = element<const T>(is_q ? a.Q : is_v ? a.V : a.K, row, hh);
    T* y = element<T>(is_q ? a.Qo : is_v ? a.Vo : a.Ko, is_q ? row : slot, hh);
    Chunk<T> p, q;
    p.load(x + at.a), q.load(x + at.b);
    if (!is_v) {
      float v[16];
      p.get(v), q.get(v + 8);
      const float* weight = is_q ? a.qw : a.kw;
      const float sum = head_sum<Lane<D>::LPH>(square_sum(v));
      if (weight) {
        float wt[16];
        weight_of<D>(weight, at, wt);
        const float r = inverse_root(sum * (1.f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = v[i] * r * wt[i];
      }
      if (at.turns) turn<NEXT>(v, c, s);
      p.set(v), q.set(v + 8);
    }
    if (is_q || kept) p.store(y + at.a), q.store(y + at.b);
  }
}

// Gradient rows of the queries (the first a.q.groups workgroups) or of the keys: a wave takes every
// (4 groups / split)-th row and, of its heads, every split-th wave's share; the weight's gradient stays in registers over
// its rows.  With queries and keys in one wave the two sums took 155 registers, three waves a SIMD: 2048 rows of 8 + 2
// heads of 64 11.8 us with the weights' launch, 8.2 so; 16000 of 24 + 4 45.7 and 39.8 (4.3 TB/s).
template <typename T, int D, bool NEXT>
__global__ __launch_bounds__(256, 4) void rope_bwd_kernel(RopeArgs a) {
  constexpr int LPH = Lane<D>::LPH, HPW = Lane<D>::HPW;
  __shared__ __attribute__((aligned(16))) float cs[4][2][64];
  __shared__ __attribute__((aligned(16))) float red[4 * HPW][D];
  const bool is_q = (int)blockIdx.x < a.q.groups;
  const RopeBack& k = is_q ? a.q : a.k;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t w = (int64_t)(blockIdx.x - (is_q ? 0 : a.q.groups)) * 4 + wave;
  const int part = (int)(w % k.split);
  const int64_t step = (int64_t)k.groups * 4 / k.split;  // groups * 4 is a multiple of split
  const Lane<D> at(a.rot, NEXT);
  float dw[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) dw[i] = 0.f;
  for (int64_t i = w / k.split; i < a.n_rows; i += step) {
    const int row = a.rows ? a.rows[i] : (int)i;
    const bool in = (uint32_t)row < (uint32_t)a.n;
    float c[8], s[8];
    row_turns<D>(a, a.rot && in ? a.pos[row] : 0, at, cs[wave], c, s);
    for (int h = part * HPW + at.g; h < k.heads; h += k.split * HPW) {
      float g[16], x[16];
      Chunk<T> p, q, px, qx;
      const T* from = element<const T>(k.dy, i, h);
      p.load(from + at.a), q.load(from + at.b);
      if (k.weight && in) {
        const T* seen = element<const T>(k.x, row, h);
        px.load(seen + at.a), qx.load(seen + at.b);
      }
      p.get(g), q.get(g + 8);
      if (at.turns) turn<NEXT, true>(g, c, s);
      if (k.weight && in) {
        px.get(x), qx.get(x + 8);
        float wt[16], dot = 0.f;
        weight_of<D>(k.weight, at, wt);
        const float r = inverse_root(head_sum<LPH>(square_sum(x)) * (1.f / D) + a.eps);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[e] *= r;
          dw[e] += g[e] * x[e];
          g[e] *= wt[e];
          dot += g[e] * x[e];
        }
        dot = head_sum<LPH>(dot) * (1.f / D);
#pragma unroll
        for (int e = 0; e < 16; ++e) g[e] = r * (g[e] - x[e] * dot);
      }
      if (!in)
#pragma unroll
        for (int e = 0; e < 16; ++e) g[e] = 0.f;
      T* to = element<T>(k.dx, i, h);
      p.set(g), q.set(g + 8);
      p.store(to + at.a), q.store(to + at.b);
    }
  }
  if (!a.part || !k.dw) return;
  Chunk<float> p, q;
  p.set(dw), q.set(dw + 8);
  p.store(&red[wave * HPW + at.g][at.a]), q.store(&red[wave * HPW + at.g][at.b]);
  __syncthreads();
  if (threadIdx.x < D) {
    float x = 0.f;
#pragma unroll
    for (int g = 0; g < 4 * HPW; ++g) x += red[g][threadIdx.x];
    a.part[(int64_t)blockIdx.x * D + threadIdx.x] = x;
  }
}

// The workgroups' sums of 16 columns of a weight's gradient (the queries' first) added in order, in 64 bits: 16 ranges of
// the workgroups, then the ranges.
template <int D>
__global__ __launch_bounds__(256) void rope_weight_kernel(RopeArgs a) {
  __shared__ double red[16][17];
  const bool is_q = blockIdx.x < D / 16;
  const RopeBack& k = is_q ? a.q : a.k;
  if (!k.dw) return;
  const int col = blockIdx.x % (D / 16) * 16 + (threadIdx.x & 15), range = threadIdx.x >> 4;
  const float* part = a.part + (int64_t)(is_q ? 0 : a.q.groups) * D + col;
  double x = 0.;
#pragma unroll 16
  for (int g = range; g < k.groups; g += 16) x += (double)part[(int64_t)g * D];
  red[range][threadIdx.x & 15] = x;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  x = 0.;
#pragma unroll
  for (int r = 0; r < 16; ++r) x += red[r][threadIdx.x];
  k.dw[col] = (float)x;
}

// ---- host -----------------------------------------------------------------------------------------------------------
// Of a row's blocks of heads a forward wave takes three in bf16 (6 KiB) and one in fp32 (4 KiB), or one where that makes
// fewer waves than this.  16384 rows of 64 + 8 heads of 128 and the values, bf16, one, two or three blocks, or all ten a wave:
// 136, 127, 127 and 143 us; fp32 239, 248, 254 and 268.  6144 rows of 32 + 8: 35.8, 34.3, 33.9 and 36.5; fp32 54, 57, 59, 60.
constexpr int kFwdWaves = 4096;
// Workgroups of a backward, four on a CU: with 2048, 2048 rows of 32 + 8 heads 21.9 us and 19.6 with 1024, 8192 62.1 and 62.8.
constexpr int kBwdGroups = 1024;

// Waves that share a gradient row: a power of two, so that four waves a group divide evenly.
int split_of(int64_t rows, int blocks, int64_t waves) {
  int s = 1;
  while (s < blocks && rows * s < waves && s < 64) s *= 2;
  return s;
}

int heads_a_wave(int d) { return 64 / (d / 16); }

// Workgroups of the backward of `heads` heads, at most `most`: a number of waves that the split divides.
int bwd_groups(int32_t heads, int d, int32_t n_rows, int most, int* split) {
  *split = 1;
  if (heads == 0) return 0;
  const int hpw = heads_a_wave(d);
  *split = split_of(n_rows, (heads + hpw - 1) / hpw, 4 * most);
  const int64_t waves = std::min<int64_t>((int64_t)n_rows * *split, 4 * most);
  const int64_t per = std::max(1, *split / 4);  // groups of four waves that one row takes
  return (int)std::max<int64_t>(per, (waves + 4 * per - 1) / (4 * per) * per);
}

// Of both kinds, with the workgroups divided as the heads are.
void bwd_launch(const dsv_rope& r, int32_t n_rows, RopeBack* q, RopeBack* k) {
  const int hpw = heads_a_wave(r.head_dim), qb = (r.heads_q + hpw - 1) / hpw, kb = (r.heads_kv + hpw - 1) / hpw;
  const int most_q = std::max(1, kBwdGroups * qb / (qb + kb)), most_k = std::max(1, kBwdGroups * kb / (qb + kb));
  q->groups = bwd_groups(r.heads_q, r.head_dim, n_rows, most_q, &q->split);
  k->groups = bwd_groups(r.heads_kv, r.head_dim, n_rows, most_k, &k->split);
}

int check(const dsv_rope* r) {
  if (!r || r->n < 0) return DSV_ERR_ARG;
  if (r->heads_q < 0 || r->heads_q > 1024 || r->heads_kv < 0 || r->heads_kv > 1024 || r->heads_q + r->heads_kv == 0)
    return DSV_ERR_RANGE;
  if (r->head_dim != 64 && r->head_dim != 128) return DSV_ERR_RANGE;
  if (r->rotated < 0 || r->rotated > r->head_dim || (r->rotated & 15) || (r->interleaved != 0 && r->interleaved != 1))
    return DSV_ERR_RANGE;
  if (r->q_weight || r->k_weight) {
    const float e = (float)r->eps;
    if (!(e >= FLT_MIN) || !std::isfinite(e)) return DSV_ERR_RANGE;
  }
  auto off = [](const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; };
  if (off(r->pos, 4) || off(r->freq, 8) || off(r->q_weight, 16) || off(r->k_weight, 16)) return DSV_ERR_ARG;
  if (r->rotated > 0 && (!r->freq || (r->n > 0 && !r->pos))) return DSV_ERR_ARG;
  return DSV_OK;
}

RopeArgs common(const dsv_rope& r) {
  RopeArgs a{};
  a.n = r.n;
  a.hq = r.heads_q, a.hkv = r.heads_kv;
  a.rot = r.rotated;
  a.eps = (float)r.eps;
  a.pos = r.pos, a.freq = r.freq;
  a.qw = r.q_weight, a.kw = r.k_weight;
  return a;
}

int status(hipError_t e) { return e == hipSuccess ? DSV_OK : DSV_ERR_DEVICE; }

template <typename T, bool NEXT>
hipError_t launch_fwd(const RopeArgs& a, int d, int64_t groups, hipStream_t s) {
  if (d == 64) hipLaunchKernelGGL((rope_fwd_kernel<T, 64, NEXT>), dim3((unsigned)groups), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((rope_fwd_kernel<T, 128, NEXT>), dim3((unsigned)groups), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool NEXT>
hipError_t launch_bwd(const RopeArgs& a, int d, hipStream_t s) {
  if (d == 64) hipLaunchKernelGGL((rope_bwd_kernel<T, 64, NEXT>), dim3((unsigned)(a.q.groups + a.k.groups)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((rope_bwd_kernel<T, 128, NEXT>), dim3((unsigned)(a.q.groups + a.k.groups)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace dsv

using namespace dsv;

extern "C" int dsv_rope_fwd(dsv_dtype dt, const dsv_rope* r, const dsv_attn_view* Q, const dsv_attn_view* K,
                            const dsv_attn_view* V, const int32_t* slots, int32_t n_slots, const dsv_attn_view* Q_out,
                            const dsv_attn_view* K_out, const dsv_attn_view* V_out, void* hip_stream) {
  int rc = check(r);
  if (rc != DSV_OK) return rc;
  if (dt != DSV_BF16 && dt != DSV_F32) return DSV_ERR_RANGE;
  if ((!V) != (!V_out) || (slots && n_slots < 0) || (reinterpret_cast<uintptr_t>(slots) & 3)) return DSV_ERR_ARG;
  RopeArgs a = common(*r);
  const int32_t d = r->head_dim, kept = slots ? n_slots : r->n;
  if (a.hq > 0) {
    if ((rc = view(Q, r->n, a.hq, d, false, &a.Q)) != DSV_OK) return rc;
    if ((rc = view(Q_out, r->n, a.hq, d, true, &a.Qo)) != DSV_OK) return rc;
  }
  if (a.hkv > 0) {
    if ((rc = view(K, r->n, a.hkv, d, false, &a.K)) != DSV_OK) return rc;
    if ((rc = view(K_out, kept, a.hkv, d, true, &a.Ko)) != DSV_OK) return rc;
    if (V) {
      if ((rc = view(V, r->n, a.hkv, d, false, &a.V)) != DSV_OK) return rc;
      if ((rc = view(V_out, kept, a.hkv, d, true, &a.Vo)) != DSV_OK) return rc;
      a.hv = a.hkv;
    }
  }
  if (r->n == 0) return DSV_OK;
  a.slots = slots, a.n_slots = n_slots;
  const int hpw = heads_a_wave(d);
  const int blocks = (a.hq + a.hkv + a.hv + hpw - 1) / hpw, shared = dt == DSV_BF16 ? (blocks + 2) / 3 : blocks;
  a.split = (int64_t)r->n * shared < kFwdWaves ? blocks : shared;
  const int64_t groups = ((int64_t)r->n * a.split + 3) / 4;
  if (groups > UINT32_MAX / 256) return DSV_ERR_SIZE;  // a grid's work items are counted in 32 bits
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (dt == DSV_BF16)
    return status(r->interleaved ? launch_fwd<uint16_t, true>(a, d, groups, s) : launch_fwd<uint16_t, false>(a, d, groups, s));
  return status(r->interleaved ? launch_fwd<float, true>(a, d, groups, s) : launch_fwd<float, false>(a, d, groups, s));
}

extern "C" int dsv_rope_workspace(const dsv_rope* r, int32_t n_rows, size_t* bytes) {
  if (!bytes || n_rows < 0) return DSV_ERR_ARG;
  const int rc = check(r);
  if (rc != DSV_OK) return rc;
  RopeBack q, k;
  bwd_launch(*r, n_rows, &q, &k);
  *bytes = std::max<size_t>(256, (size_t)(q.groups + k.groups) * r->head_dim * sizeof(float));
  return DSV_OK;
}

extern "C" int dsv_rope_bwd(dsv_dtype dt, const dsv_rope* r, int32_t n_rows, const int32_t* rows, const dsv_attn_view* dQ,
                            const dsv_attn_view* dK, const dsv_attn_view* Q, const dsv_attn_view* K,
                            const dsv_attn_view* dQ_out, const dsv_attn_view* dK_out, float* dq_weight, float* dk_weight,
                            void* ws, size_t ws_bytes, void* hip_stream) {
  int rc = check(r);
  if (rc != DSV_OK) return rc;
  if (dt != DSV_BF16 && dt != DSV_F32) return DSV_ERR_RANGE;
  if (n_rows < 0 || (!rows && n_rows > r->n) || (reinterpret_cast<uintptr_t>(rows) & 3)) return DSV_ERR_ARG;
  if ((dq_weight && (!r->q_weight || r->heads_q == 0)) || (dk_weight && (!r->k_weight || r->heads_kv == 0)))
    return DSV_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(dq_weight) | reinterpret_cast<uintptr_t>(dk_weight)) & 15) return DSV_ERR_ARG;
  RopeArgs a = common(*r);
  const int32_t d = r->head_dim;
  if (a.hq > 0) {
    if ((rc = view(dQ, n_rows, a.hq, d, false, &a.q.dy)) != DSV_OK) return rc;
    if ((rc = view(dQ_out, n_rows, a.hq, d, true, &a.q.dx)) != DSV_OK) return rc;
    if (a.qw && (rc = view(Q, r->n, a.hq, d, false, &a.q.x)) != DSV_OK) return rc;
  }
  if (a.hkv > 0) {
    if ((rc = view(dK, n_rows, a.hkv, d, false, &a.k.dy)) != DSV_OK) return rc;
    if ((rc = view(dK_out, n_rows, a.hkv, d, true, &a.k.dx)) != DSV_OK) return rc;
    if (a.kw && (rc = view(K, r->n, a.hkv, d, false, &a.k.x)) != DSV_OK) return rc;
  }
  bwd_launch(*r, n_rows, &a.q, &a.k);
  a.q.heads = a.hq, a.k.heads = a.hkv;
  a.q.weight = a.qw, a.k.weight = a.kw;
  a.q.dw = dq_weight, a.k.dw = dk_weight;
  const bool sums = dq_weight || dk_weight;
  if (sums) {
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return DSV_ERR_ARG;
    if (ws_bytes < (size_t)(a.q.groups + a.k.groups) * d * sizeof(float)) return DSV_ERR_SIZE;
    a.part = static_cast<float*>(ws);
  }
  if (n_rows == 0 && !sums) return DSV_OK;
  a.n_rows = n_rows, a.rows = rows;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e =
      dt == DSV_BF16 ? (r->interleaved ? launch_bwd<uint16_t, true>(a, d, s) : launch_bwd<uint16_t, false>(a, d, s))
                     : (r->interleaved ? launch_bwd<float, true>(a, d, s) : launch_bwd<float, false>(a, d, s));
  if (e != hipSuccess || !sums) return status(e);
  hipLaunchKernelGGL(d == 64 ? rope_weight_kernel<64> : rope_weight_kernel<128>, dim3((unsigned)(d / 8)), dim3(256), 0, s, a);
  return status(hipGetLastError());
}
