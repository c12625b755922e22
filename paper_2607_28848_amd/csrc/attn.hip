// attn.hip -- CDNA4 (gfx950) attention of a mixed batch in bf16, and the C entry points.
//
//   attn_fwd    128 queries of one head against the keys they see, one pass with the running maximum
//               and sum of the softmax.
//   attn_split  the (query, head) pairs of a key head of a sequence of few queries (decode) against
//               one piece of its keys; attn_join adds the pieces of both forms.
//   attn_dq     dQ of 128 queries (and do . o); attn_dk: dK and dV of 128 keys; attn_grad_join adds their pieces.
//
// Products are v_mfma_f32_32x32x16_bf16: lane l holds A[l % 32][8 (l / 32) + e], B[8 (l / 32) + e][l % 32]
// (e < 8) and C[8 (v / 4) + 4 (l / 32) + v % 4][l % 32] (v < 16).  The scores are computed with the
// index that the second product sums over as rows, so a lane holds 16 of them for its own column, and
// values 8 t .. 8 t + 7, rounded to bf16, are the second product's operand as they are: its contraction
// slot (l / 32, e) stands for row 16 t + 8 (e / 4) + 4 (l / 32) + e % 4, and the other operand is read in that
// order (two transposing LDS reads of four rows each).  No value crosses lanes but for a query's maximum and
// sum, which two lanes share.
//
// p and ds are rounded to bf16 for the second product because an fp32 one takes 16 times as long on the matrix core.
// Against 64 bits the outputs are then off by 0.21 to 0.27% in the root mean square, where fp32 products of the same
// operands, rounded once at the end, leave 0.16 to 0.20%.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "attn.h"
#include "attn_plan.h"
#include "device_common.h"

namespace dsv {
namespace {

extern "C" __device__ void llvm_amdgcn_raw_buffer_load_lds_a(i32x4 rsrc, lds_u32* lds, int size, int voffset,
                                                             int soffset, int offset,
                                                             int aux) __asm("llvm.amdgcn.raw.buffer.load.lds");

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Seq {
  int q0, ql, k0, kl, cq, ck;
  __device__ __forceinline__ Seq(const AttnArgs& a, int i) {
    const int32_t* w = a.seqs + (int64_t)i * kAttnSeqWords;
    q0 = w[0], ql = w[1], k0 = w[2], kl = w[3], cq = w[4], ck = w[5];
  }
};

// Workgroup -> (item, query head): a key head's query heads are hkv apart, so that they land on one XCD
// (ids go round the 8 XCDs) when the key heads are 8, and share K and V in its L2.
__device__ __forceinline__ int head_of(const AttnArgs& a, int x) { return (x % a.hkv) * a.group + x / a.hkv; }

// LDS image of staged rows (D bf16 each): 16-byte chunk c of row r sits in slot c ^ swz(r).  Of the 64 banks'
// 256 bytes, 16 consecutive rows put one chunk in 16 different 16-byte groups (fragment reads), and four
// consecutive rows put four neighbouring chunks in four different 64-byte groups (transposing reads).
template <int D>
__device__ __forceinline__ constexpr int swz(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3);
}

// Descriptor over rows [r0, r_end) of a head (reads past them return zeros); rows are at most 64 at a
// time and at most 2^23 elements apart, so offsets fit in 31 bits.
__device__ __forceinline__ i32x4 rows_rsrc(const AttnView& t, int64_t row, int h, int n, int d) {
  const uint64_t p = reinterpret_cast<uint64_t>(static_cast<const uint16_t*>(t.ptr) + row * t.row + h * t.head);
  const int64_t range = n > 0 ? ((int64_t)(n - 1) * t.row + d) * 2 : 0;
  i32x4 r;
  r.x = __builtin_amdgcn_readfirstlane((int)(uint32_t)p);
  r.y = __builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32));
  r.z = __builtin_amdgcn_readfirstlane((int)range);
  r.w = 0x00020000;
  return r;
}

__device__ __forceinline__ i32x4 flat_rsrc(const void* base, int bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  i32x4 r;
  r.x = __builtin_amdgcn_readfirstlane((int)(uint32_t)p);
  r.y = __builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32));
  r.z = __builtin_amdgcn_readfirstlane(bytes);
  r.w = 0x00020000;
  return r;
}

// Rows [0, ROWS) of the descriptor into LDS, the work shared by NW waves.  A load fills 1 KiB of the image: RPL
// rows; row blocks go in the scalar offset and change the lane's slot by a constant xor.
template <int D, int ROWS, int NW>
__device__ __forceinline__ void stage(const i32x4& rs, int row_bytes, char* lds, int wave, int lane = threadIdx.x & 63) {
  constexpr int RB = 2 * D, RPL = 1024 / RB, CH = RB / 16;  // row bytes, rows a load, chunks a row
  constexpr int N = ROWS / RPL / NW;
  static_assert(N > 0 && N * RPL * NW == ROWS, "rows");
  const int own = 16 * ((lane % CH) ^ swz<D>(lane / CH)), row = lane / CH * row_bytes;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int q = wave * N + i;
    llvm_amdgcn_raw_buffer_load_lds_a(rs, (lds_u32*)(lds + q * 1024), 16, (own ^ (16 * swz<D>(q * RPL % 16))) + row,
                                      __builtin_amdgcn_readfirstlane(q * RPL * row_bytes), 0, 0);
  }
}

// The lane's number, read afresh: what is derived from it cannot be kept in registers across uses.
__device__ __forceinline__ int fresh_lane() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

// Fragment of rows 32 u ..: lane's row 32 u + l % 32, its 8 values of step s.  Steps and blocks of columns
// change single bits of the lane's slot, so an address is the lane's own part xor a constant.
template <int D>
__device__ __forceinline__ bf16x8 frag(const char* lds, int u, int s, int lane = threadIdx.x & 63) {
  const int r = lane & 31, own = r * 2 * D + 16 * ((lane >> 5) ^ swz<D>(r));
  return as_bf(*reinterpret_cast<const u32x4*>(lds + (own ^ (32 * s)) + u * 64 * D));
}

// Transposed fragment: lane's column 32 t + l % 32 of rows 16 w + 4 (l / 32) + {0..3} and 8 further on.
template <int D>
__device__ __forceinline__ bf16x8 frag_t(const char* lds, int w, int t, int lane = threadIdx.x & 63) {
  const int lam = lane & 15, r = 4 * (lane >> 5) + (lam >> 2);
  const int own = r * 2 * D + 16 * ((2 * ((lane >> 4) & 1) + ((lam & 3) >> 1)) ^ swz<D>(r)) + 8 * (lam & 1);
  static_assert(swz<D>(8) == 2 && swz<D>(16) == 0, "row 8 on: slot bit 1");
  u32x4 v;
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    const char* p = lds + (own ^ (64 * t + 32 * hh)) + (16 * w + 8 * hh) * 2 * D;
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
    v[2 * hh] = (uint32_t)(uint16_t)x[0] | ((uint32_t)(uint16_t)x[1] << 16);
    v[2 * hh + 1] = (uint32_t)(uint16_t)x[2] | ((uint32_t)(uint16_t)x[3] << 16);
  }
  return as_bf(v);
}

// A lane's fragments of its own row (zeros where it does not exist).
template <int D>
__device__ __forceinline__ void row_frags(const AttnView& t, int64_t row, int h, bool in, bf16x8 (&f)[D / 16]) {
  const uint16_t* p = static_cast<const uint16_t*>(t.ptr) + row * t.row + h * t.head + 8 * ((threadIdx.x >> 5) & 1);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) f[s] = as_bf(in ? ld16(p + 16 * s) : zero4());
}

// Scheduling of a run of N matrix instructions that consume DS LDS reads each: the reads of the first `ahead`
// of them, then one instruction and the reads of a later one by turns, so that no instruction waits for
// the read before it.
template <int N, int DS, int AHEAD>
__device__ __forceinline__ void feed() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * DS, 0);
#pragma unroll
  for (int i = 0; i < N - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, DS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}

// The same with V vector instructions (of other values) after each matrix instruction.
template <int N, int DS, int AHEAD, int V>
__device__ __forceinline__ void feed_beside() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * DS, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (i < N - AHEAD) __builtin_amdgcn_sched_group_barrier(0x100, DS, 0);
    __builtin_amdgcn_sched_group_barrier(0x402, V, 0);
  }
}

// Two values of [0, 2) in 16 bits each, rounded to nearest: sign and the exponent's first bit are zero, so 7 bits of
// exponent and 9 of mantissa hold fp32's range below 2.  (A NaN is lost; its query's delta is NaN, and with it ds.)
__device__ __forceinline__ uint32_t pack_p(float a, float b) {
  return __builtin_amdgcn_perm((__float_as_uint(b) << 2) + 0x8000u, (__float_as_uint(a) << 2) + 0x8000u, 0x07060302u);
}

template <bool B>
struct bool_c {  // a compile-time flag passed as a value
  static constexpr bool value = B;
};

// The larger / the sum of the two lanes that share a column.
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ bf16x8 pack8(const f32x16& x, int t) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = f2bf2(x[8 * t + 2 * i], x[8 * t + 2 * i + 1]);
  return as_bf(v);
}

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] = 0.f;
  return z;
}

// Row of value v of a 32 x 32 tile.
__device__ __forceinline__ int tile_row(int v) { return 8 * (v >> 2) + 4 * ((threadIdx.x >> 5) & 1) + (v & 3); }

// The running softmax of a lane's query: the reference that exponents are taken from (base 2, times
// scale) and the lane's own part of the sum.
struct Running {
  float ref = -INFINITY, sum = 0.f;
};

// Moves the reference (and with it the sums and acc) where a score c x exceeds it by more than 2^8: terms are
// bounded by that, and all but the first blocks of a row leave the reference as it is.
template <int N, int NA>
__device__ __forceinline__ void softmax_ref(const f32x16 (&x)[N], float c, Running& r, f32x16 (&acc)[NA]) {
  float mx = x[0][0];
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, x[u][v]);
  const float top = pair_max(mx) * c;
  if (__builtin_amdgcn_ballot_w64(top > r.ref + 8.f) != 0) {
    const float ref = fmaxf(top, r.ref);
    const float f = ref == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(r.ref - ref);
    r.ref = ref;
    r.sum *= f;
#pragma unroll
    for (int t = 0; t < NA; ++t) acc[t] *= f;
  }
}

// Values 8 w .. of a block's scores to terms exp2(c x - ref), into the sum and, as bf16, the second product's
// operand.  base: the reference, 0 where no key was seen so far (every term is exp2(-inf) = 0 then).
__device__ __forceinline__ bf16x8 softmax_terms(const f32x16& x, int w, float c, float base, float& sum) {
  f32x16 e;
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    e[v] = __builtin_amdgcn_exp2f(x[8 * w + v] * c - base);
    sum += e[v];
  }
  return pack8(e, 0);
}

__device__ __forceinline__ float lse_of(float ref, float sum) {
  return sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int D>
__device__ __forceinline__ void store_cols(const AttnView& t, int64_t row, int h, const f32x16 (&acc)[D / 32], float f) {
  uint16_t* p = static_cast<uint16_t*>(t.ptr) + row * t.row + h * t.head + 4 * ((threadIdx.x >> 5) & 1);
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const uint32_t w0 = f2bf2(acc[i][4 * a] * f, acc[i][4 * a + 1] * f);
      const uint32_t w1 = f2bf2(acc[i][4 * a + 2] * f, acc[i][4 * a + 3] * f);
      *reinterpret_cast<uint2*>(p + 32 * i + 8 * a) = make_uint2(w0, w1);
    }
}

// The same as they are, in fp32, to the row at p.
template <int D>
__device__ __forceinline__ void store_sums(float* p, const f32x16 (&acc)[D / 32]) {
  p += 4 * ((threadIdx.x >> 5) & 1);
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(p + 32 * t + 8 * i) =
          f32x4{acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]};
}

// ---------------------------------------------------------------------------------------------------
// O and lse of 128 queries of one head (or the sums of a piece of their keys): 32 queries a wave, 64 keys a step.
//
// A wave's products read a fragment of K or V from LDS for each matrix instruction, 1 KiB in the 32 cycles that one
// takes: all of a CU's LDS bandwidth with four waves at it, so two workgroups share a CU and one's softmax runs beside
// the other's products.  With heads of 64 the exponentials (one for 256 operations, a quarter of the vector rate) take
// as long as the products.  16384 queries, 32 heads of 128 on 8: 1.90 ms (1155 TFLOP/s; a large bf16 product reaches
// 1290 on the same card).  Nine prompts of about 700, 24 heads of 64 on 4: 36 us (570 TFLOP/s).
template <int D>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(AttnArgs a) {
  constexpr int TK = 64, TILE = TK * 2 * D;
  __shared__ __attribute__((aligned(1024))) char b0[2 * TILE];
  __shared__ __attribute__((aligned(1024))) char b1[2 * TILE];
  const int item = blockIdx.x / a.hq, h = head_of(a, blockIdx.x % a.hq);
  const int32_t* it = a.items + (int64_t)item * kAttnTileWords;
  const Seq s(a, it[0]);
  const int qt = it[1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int off = s.kl - s.ql, hk = h / a.group;
  const int q = qt + 32 * wave + (lane & 31);
  // the tile's keys, or a piece of them
  const int k_first = TK * it[2], k_end = min(min(s.kl, min(qt + kAttnFwdRows, s.ql) + off), TK * it[3]);
  const int krow = (int)a.K.row * 2, vrow = (int)a.V.row * 2;
  auto load = [&](int kt, char* b) {
    stage<D, TK, 4>(rows_rsrc(a.K, (int64_t)s.k0 + kt, hk, min(TK, s.kl - kt), D), krow, b, wave);
    stage<D, TK, 4>(rows_rsrc(a.V, (int64_t)s.k0 + kt, hk, min(TK, s.kl - kt), D), vrow, b + TILE, wave);
  };
  if (k_first < k_end) load(k_first, b0);
  bf16x8 qf[D / 16];
  row_frags<D>(a.Q, (int64_t)s.q0 + q, h, q < s.ql, qf);
  f32x16 acc[D / 32];
#pragma unroll
  for (int t = 0; t < D / 32; ++t) acc[t] = zero16();
  Running run;
  const float c = a.scale * kLog2e;
  const int seen = q + off;                                        // the lane's last key
  const int wave_all = qt + 32 * wave + off;                       // keys up to here are seen by the whole wave
  const int wave_end = min(s.kl, wave_all + 32);                   // keys from here on by none of it
  auto step = [&](int kt, const char* cur, char* nxt) {
    vmem_wait_all();
    __syncthreads();
    if (kt + TK < k_end) load(kt + TK, nxt);
    if (kt >= wave_end) return;
    f32x16 x[2];
    x[0] = x[1] = zero16();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) x[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag<D>(cur, u, i), qf[i], x[u], 0, 0, 0);
    feed<D / 8, 1, 4>();
    __builtin_amdgcn_sched_barrier(0);
    if (kt + TK - 1 > wave_all) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int v = 0; v < 16; ++v) x[u][v] = kt + 32 * u + tile_row(v) <= seen ? x[u][v] : -INFINITY;
    }
    softmax_ref(x, c, run, acc);
    const float base = run.ref == -INFINITY ? 0.f : run.ref;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const bf16x8 p = softmax_terms(x[w >> 1], w & 1, c, base, run.sum);
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_t<D>(cur + TILE, w, t), p, acc[t], 0, 0, 0);
    }
    // the terms of 16 keys are formed between the products of the 16 before
    __builtin_amdgcn_sched_group_barrier(0x100, D / 16, 0);
    __builtin_amdgcn_sched_group_barrier(0x402, 28, 0);
#pragma unroll
    for (int i = 0; i < 3 * D / 32; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, 28 * 32 / D, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, D / 32, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  for (int kt = k_first; kt < k_end; kt += 2 * TK) {
    step(kt, b0, b1);
    if (kt + TK < k_end) step(kt + TK, b1, b0);
  }
  const float sum = pair_sum(run.sum);
  if (q >= s.ql) return;
  if (it[5] > 1) {
    const int64_t slot = (int64_t)it[4] * a.hq + h;
    const int row = 32 * wave + (lane & 31);
    store_sums<D>(a.part_o + (slot * kAttnFwdRows + row) * D, acc);
    if (lane < 32) {
      a.part_ml[slot * 2 * kAttnFwdRows + row] = run.ref;
      a.part_ml[(slot * 2 + 1) * kAttnFwdRows + row] = sum;
    }
    return;
  }
  store_cols<D>(a.O, (int64_t)s.q0 + q, h, acc, sum == 0.f ? 0.f : 1.f / sum);
  if (a.lse && lane < 32) a.lse[(int64_t)h * a.n_q + s.q0 + q] = lse_of(run.ref, sum);
}

// ---------------------------------------------------------------------------------------------------
// One piece of the keys of a sequence for 32 (query, head) pairs of a key head, row r being query
// r / group and head r % group.  Each wave takes every fourth block of 32 keys through buffers of its
// own (no barrier until the end), then the four waves' sums are added.  Every key is read once for all of
// its head's queries: the stream of K and V is what bounds it where there are many keys (64 sequences of about 2600,
// 8 heads of 128: 577 MB in 105 us, 5.5 TB/s), and the loads' latency one after the other where there are few (8 of
// about 400: 10 us for 12 MB).
template <int D>
__global__ __launch_bounds__(256) void attn_split_kernel(AttnArgs a) {
  constexpr int TK = 32, TILE = TK * 2 * D, LDO = D + 4;
  constexpr int kOut = 4 * 32 * LDO * 4, kBuf = 4 * 2 * TILE;
  __shared__ __attribute__((aligned(1024))) char b0[kOut > kBuf ? kOut : kBuf];
  __shared__ __attribute__((aligned(1024))) char b1[kBuf];
  __shared__ float ml[2][4][32];
  const int item = blockIdx.x / a.hkv, hk = blockIdx.x % a.hkv;
  const int32_t* it = a.items + kAttnSplitWords * (int64_t)item;
  const struct { int q0, ql, k0, kl; } s = {it[0], it[1], it[2], it[3]};
  const int r0 = it[4], n_pieces = it[5], k_first = it[7], k_last = it[8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int off = s.kl - s.ql, rows = s.ql * a.group;
  const int r = r0 + (lane & 31), q = min(r, rows - 1) / a.group, h = hk * a.group + min(r, rows - 1) % a.group;
  const int krow = (int)a.K.row * 2, vrow = (int)a.V.row * 2;
  char* const w0 = b0 + wave * 2 * TILE;
  char* const w1 = b1 + wave * 2 * TILE;
  auto load = [&](int kt, char* b) {
    stage<D, TK, 1>(rows_rsrc(a.K, (int64_t)s.k0 + kt, hk, min(TK, s.kl - kt), D), krow, b, 0);
    stage<D, TK, 1>(rows_rsrc(a.V, (int64_t)s.k0 + kt, hk, min(TK, s.kl - kt), D), vrow, b + TILE, 0);
  };
  constexpr int LOADS = 2 * TILE / 1024;
  const int kb = k_first + TK * wave;
  if (kb < k_last) load(kb, w0);
  bf16x8 qf[D / 16];
  row_frags<D>(a.Q, (int64_t)s.q0 + q, h, r < rows, qf);
  asm volatile("" ::: "memory");  // before the next block's loads: what step() waits for covers them
  f32x16 acc[D / 32];
#pragma unroll
  for (int t = 0; t < D / 32; ++t) acc[t] = zero16();
  Running run;
  const float c = a.scale * kLog2e;
  const int seen = q + off;
  const int all = min(r0, rows - 1) / a.group + off;  // keys up to here are seen by every row
  auto step = [&](int kt, const char* cur, char* nxt) {
    if (kt + 4 * TK < k_last) {
      load(kt + 4 * TK, nxt);
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(LOADS));
    } else {
      vmem_wait_all();
    }
    asm volatile("" ::: "memory");
    f32x16 x[1];
    x[0] = zero16();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) x[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag<D>(cur, 0, i), qf[i], x[0], 0, 0, 0);
    feed<D / 16, 1, D / 16>();
    __builtin_amdgcn_sched_barrier(0);
    if (kt + TK - 1 > all || kt + TK > k_last) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        x[0][v] = kt + tile_row(v) <= seen && kt + tile_row(v) < k_last ? x[0][v] : -INFINITY;
    }
    softmax_ref(x, c, run, acc);
    const float base = run.ref == -INFINITY ? 0.f : run.ref;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const bf16x8 p = softmax_terms(x[0], w, c, base, run.sum);
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_t<D>(cur + TILE, w, t), p, acc[t], 0, 0, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, D / 8, 0);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // `cur` is read before it is loaded again
  };
  for (int kt = kb; kt < k_last; kt += 8 * TK) {
    step(kt, w0, w1);
    if (kt + 4 * TK < k_last) step(kt + 4 * TK, w1, w0);
  }
  const float sum = pair_sum(run.sum);
  __syncthreads();  // every wave is done with its buffers
  float* const out = reinterpret_cast<float*>(b0) + (wave * 32 + (lane & 31)) * LDO + 4 * (lane >> 5);
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(out + 32 * t + 8 * i) =
          f32x4{acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]};
  if (lane < 32) {
    ml[0][wave][lane] = run.ref;
    ml[1][wave][lane] = sum;
  }
  __syncthreads();
  // row tid / 8, D / 8 columns each
  const int row = threadIdx.x >> 3, c0 = (threadIdx.x & 7) * (D / 8);
  if (r0 + row >= rows) return;
  float ref = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) ref = fmaxf(ref, ml[0][w][row]);
  float f[4], total = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = ml[0][w][row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0][w][row] - ref);
    total += f[w] * ml[1][w][row];
  }
  const bool whole = n_pieces == 1;
  const float g = !whole ? 1.f : total == 0.f ? 0.f : 1.f / total;
  const int qr = (r0 + row) / a.group, hr = hk * a.group + (r0 + row) % a.group;
  const int64_t slot = (int64_t)it[6] * a.hkv + hk;
#pragma unroll
  for (int i = 0; i < D / 8; i += 4) {
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w)
      o += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(b0) + (w * 32 + row) * LDO + c0 + i) * f[w];
    o *= g;
    if (whole) {
      uint16_t* p = static_cast<uint16_t*>(a.O.ptr) + ((int64_t)s.q0 + qr) * a.O.row + hr * a.O.head + c0 + i;
      *reinterpret_cast<uint2*>(p) = make_uint2(f2bf2(o[0], o[1]), f2bf2(o[2], o[3]));
    } else {
      *reinterpret_cast<f32x4*>(a.part_o + (slot * kAttnPackRows + row) * D + c0 + i) = o;
    }
  }
  if ((threadIdx.x & 7) == 0) {
    if (!whole) {
      a.part_ml[slot * 2 * kAttnPackRows + row] = ref;
      a.part_ml[(slot * 2 + 1) * kAttnPackRows + row] = total;
    } else if (a.lse) {
      a.lse[(int64_t)hr * a.n_q + s.q0 + qr] = lse_of(ref, total);
    }
  }
}

// Pieces of a row added in order: columns c0 .. c0 + D / 8 of row `row` of `rows`, slots first, first + step, ..
template <int D>
__device__ __forceinline__ void join_row(const AttnArgs& a, const float* part_o, const float* part_ml, int64_t first, int64_t step,
                                         int n, int rows, int row, int c0, int64_t out_row, int h) {
  float ref = -INFINITY, total = 0.f;
#pragma unroll 4
  for (int k = 0; k < n; ++k) ref = fmaxf(ref, part_ml[(first + k * step) * 2 * rows + row]);
  f32x4 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int k = 0; k < n; ++k) {
    const int64_t slot = first + k * step;
    const float m = part_ml[slot * 2 * rows + row];
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - ref);
    total += f * part_ml[(slot * 2 + 1) * rows + row];
    const float* p = part_o + (slot * rows + row) * D + c0;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] += *reinterpret_cast<const f32x4*>(p + 4 * i) * f;
  }
  const float g = total == 0.f ? 0.f : 1.f / total;
  uint16_t* p = static_cast<uint16_t*>(a.O.ptr) + out_row * a.O.row + h * a.O.head + c0;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
    *reinterpret_cast<uint2*>(p + 4 * i) = make_uint2(f2bf2(o[i][0] * g, o[i][1] * g), f2bf2(o[i][2] * g, o[i][3] * g));
  if (a.lse && c0 == 0) a.lse[(int64_t)h * a.n_q + out_row] = lse_of(ref, total);
}

// Both forms' pieces in one launch: 32 rows a workgroup, row tid / 8, D / 8 columns each; forward tiles first.
// The launch and two reads one after the other: 4.9 us for 512 tiles of the split form, 8.0 for 48 sequences' beside
// 96 forward tiles in five pieces (two launches: 12.2).
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  const int at = blockIdx.x, row = threadIdx.x >> 3, c0 = (threadIdx.x & 7) * (D / 8);
  if (at < a.first_groups) {
    constexpr int BL = kAttnFwdRows / 32;
    const int item = at / (BL * a.hq), h = at / BL % a.hq;
    const int32_t* it = a.first_join + 4 * (int64_t)item;
    const Seq s(a, it[0]);
    const int r = 32 * (at % BL) + row, q = it[1] + r;
    if (q >= s.ql) return;
    join_row<D>(a, a.first_o, a.first_ml, (int64_t)it[2] * a.hq + h, a.hq, it[3], kAttnFwdRows, r, c0, (int64_t)s.q0 + q, h);
    return;
  }
  const int item = (at - a.first_groups) / a.hkv, hk = (at - a.first_groups) % a.hkv;
  const int32_t* it = a.items + kAttnSplitWords * (int64_t)item;
  const int r = it[4] + row;
  if (it[5] == 1 || r >= it[1] * a.group) return;  // one piece: written by it
  join_row<D>(a, a.part_o, a.part_ml, (int64_t)it[6] * a.hkv + hk, a.hkv, it[5], kAttnPackRows, row, c0,
              (int64_t)it[0] + r / a.group, hk * a.group + r % a.group);
}

// ---------------------------------------------------------------------------------------------------
// dQ of 128 queries of one head over the keys they see, 32 queries a wave, 64 keys a step, in three products: the scores
// again (p = 2^(c s - lse) needs no maximum), dO V^T, and ds K.  It also leaves delta = do . o and the base-2 lse of its
// rows for attn_dk, which runs after it.  Bound as attn_fwd is (three fragments of LDS for three matrix instructions),
// matrix core 49% busy: four samples of 2048, 64 heads of 128 on 8, 0.45 ms (412 GFLOP, 920 TFLOP/s).
template <int D>
__global__ __launch_bounds__(256, 2) void attn_dq_kernel(AttnArgs a) {
  constexpr int TK = 64, TILE = TK * 2 * D;
  __shared__ __attribute__((aligned(1024))) char b0[2 * TILE];
  __shared__ __attribute__((aligned(1024))) char b1[2 * TILE];
  const int item = blockIdx.x / a.hq, h = head_of(a, blockIdx.x % a.hq);
  const int32_t* it = a.items + (int64_t)item * kAttnTileWords;
  const Seq s(a, it[0]);
  const int qt = it[1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int off = s.kl - s.ql, hk = h / a.group;
  const int q = qt + 32 * wave + (lane & 31);
  const bool in = q < s.ql;
  const int k_first = TK * it[2], k_end = min(min(s.kl, min(qt + kAttnBwdRows, s.ql) + off), TK * it[3]);
  const int krow = (int)a.K.row * 2, vrow = (int)a.V.row * 2;
  auto load = [&](int kt, char* b) {
    const int ln = fresh_lane();  // the loads' addresses kept in registers would spill others
    stage<D, TK, 4>(rows_rsrc(a.K, (int64_t)s.k0 + kt, hk, min(TK, s.kl - kt), D), krow, b, wave, ln);
    stage<D, TK, 4>(rows_rsrc(a.V, (int64_t)s.k0 + kt, hk, min(TK, s.kl - kt), D), vrow, b + TILE, wave, ln);
  };
  if (k_first < k_end) load(k_first, b0);
  bf16x8 qf[D / 16], df[D / 16];
  row_frags<D>(a.Q, (int64_t)s.q0 + q, h, in, qf);
  row_frags<D>(a.dO, (int64_t)s.cq + q, h, in, df);
  float dot = 0.f;
  {
    bf16x8 of[D / 16];
    row_frags<D>(a.O, (int64_t)s.q0 + q, h, in, of);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) dot += (float)df[i][e] * (float)of[i][e];
  }
  const float delta = pair_sum(dot);
  const float lse2 = in ? exp_from(a.lse[(int64_t)h * a.n_q + s.q0 + q]) * kLog2e : 0.f;
  if (in && lane < 32 && k_first == 0) {
    a.delta[h * a.train_q + s.cq + q] = delta;
    a.lse2[h * a.train_q + s.cq + q] = lse2;
  }
  f32x16 acc[D / 32];
#pragma unroll
  for (int t = 0; t < D / 32; ++t) acc[t] = zero16();
  const float c = a.scale * kLog2e;
  const int seen = q + off, wave_all = qt + 32 * wave + off, wave_end = min(s.kl, wave_all + 32);
  // 64 keys as two blocks: the terms of one are formed beside the products of the other.  CUT: some query of
  // the wave does not see all of them.
  auto block = [&](auto cut, int kt, const char* cur) {
    constexpr bool CUT = decltype(cut)::value;
    constexpr int V = (CUT ? 104 : 72) * 8 / D + 1;
    f32x16 x[2], dp[2];
    auto scores = [&](int u) {
      x[u] = dp[u] = zero16();
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        x[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag<D>(cur, u, i), qf[i], x[u], 0, 0, 0);
        dp[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag<D>(cur + TILE, u, i), df[i], dp[u], 0, 0, 0);
      }
    };
    bf16x8 ds[2][2];
    auto terms = [&](int u) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float t = __builtin_amdgcn_exp2f(x[u][v] * c - lse2) * (dp[u][v] - delta);
        x[u][v] = !CUT || kt + 32 * u + tile_row(v) <= seen ? t : 0.f;
      }
      ds[u][0] = pack8(x[u], 0), ds[u][1] = pack8(x[u], 1);
    };
    auto product = [&](int u) {
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
          acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_t<D>(cur, 2 * u + w, t), ds[u][w], acc[t], 0, 0, 0);
    };
    __builtin_amdgcn_sched_barrier(0);
    scores(0);
    feed<D / 8, 1, 4>();
    __builtin_amdgcn_sched_barrier(0);
    scores(1);
    terms(0);
    feed_beside<D / 8, 1, 4, V>();
    __builtin_amdgcn_sched_barrier(0);
    product(0);
    terms(1);
    feed_beside<D / 16, 2, 2, 2 * V>();
    __builtin_amdgcn_sched_barrier(0);
    product(1);
    feed<D / 16, 2, 2>();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](int kt, const char* cur, char* nxt) {
    vmem_wait_all();
    __syncthreads();
    if (kt + TK < k_end) load(kt + TK, nxt);
    if (kt >= wave_end) return;
    if (kt + TK - 1 > wave_all) block(bool_c<true>{}, kt, cur);
    else block(bool_c<false>{}, kt, cur);
  };
  for (int kt = k_first; kt < k_end; kt += 2 * TK) {
    step(kt, b0, b1);
    if (kt + TK < k_end) step(kt + TK, b1, b0);
  }
  if (!in) return;
  if (lse2 == INFINITY)  // 0 times an infinite key
#pragma unroll
    for (int t = 0; t < D / 32; ++t) acc[t] = zero16();
  if (it[5] > 1) store_sums<D>(a.part_o + (((int64_t)it[4] * a.hq + h) * kAttnBwdRows + 32 * wave + (lane & 31)) * D, acc);
  else store_cols<D>(a.dQ, (int64_t)s.cq + q, h, acc, a.scale);
}

// ---------------------------------------------------------------------------------------------------
// dK and dV of 128 keys of one key head over 64 queries at a time, the key head's query heads one after
// the other: the sums over them stay in registers.
//
// Two waves share 32 keys, each with the sums of one output (32 x D, as many registers as one wave can
// keep beside another one on its SIMD): wave w forms p and dV, wave w + 4 do . v and dK. p goes from one to
// the other through LDS, lane to lane, a step late: in step n the second wave multiplies dO(n) with V and
// closes ds(n - 1), for which Q is kept for one step more.  It travels in 16 bits with 9 of mantissa
// (pack_p): in bf16 the second rounding of ds would show, dK being off by 0.31% instead of 0.25%.
//
// Four products of 2 D operations a score (attn_dq: three), because dQ's sums run along the other axis and would need
// atomics here.  The matrix core is 45% busy: 64 queries against 128 keys read 272 KB of LDS, 2200 cycles beside 2048 of
// products, and two waves a SIMD overlap them in part.  Four samples of 2048, 64 heads of 128 on
// 8: 0.65 ms (550 GFLOP, 845 TFLOP/s); two of 1024, 32 heads on 8: 72 us and 8 for the join.
template <int D>
__global__ __launch_bounds__(512) void attn_dk_kernel(AttnArgs a) {
  constexpr int TQ = 64, TILE = TQ * 2 * D, PB = 4 * 64 * TQ, ST = 2 * TILE + PB;
  // Q, dO, p of 4 x 32 keys, lse (base 2) and delta
  __shared__ __attribute__((aligned(1024))) char b0[ST + 8 * TQ];
  __shared__ __attribute__((aligned(1024))) char b1[ST + 8 * TQ];
  __shared__ __attribute__((aligned(1024))) char b2[ST + 8 * TQ];
  const int item = blockIdx.x / a.hkv, hk = blockIdx.x % a.hkv;
  const int32_t* it = a.items + (int64_t)item * kAttnTileWords;
  const Seq s(a, it[0]);
  const int k0 = it[1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool second = wave >= 4;
  const int blk = wave & 3;
  const int off = s.kl - s.ql;
  const int k = k0 + 32 * blk + (lane & 31);
  const bool in = k < s.kl;
  const int qrow = (int)a.Q.row * 2, drow = (int)a.dO.row * 2;
  const int q_first = max(0, k0 - off);
  // the tile's steps, or a piece of them
  const int per_head = q_first < s.ql ? (s.ql - q_first + TQ - 1) / TQ : 0, n0 = it[2], steps = it[3] - n0;
  // The last queries first, one query head after the other: the workgroups of a sequence's key tiles run
  // through the same rows at the same time, whatever their first query, and share them in L2 (heads
  // outside and queries upwards missed 56% of its lines, this order 25%: four samples of 2048, 64 heads on 8, 1156 us
  // and 1006 in an earlier form).
  auto q_of = [&](int n) { return q_first + (per_head - 1 - (n0 + n) / a.group) * TQ; };
  auto load = [&](int n, char* b, int ln) {
    const int h = hk * a.group + (n0 + n) % a.group, qt = q_of(n);
    stage<D, TQ, 8>(rows_rsrc(a.Q, (int64_t)s.q0 + qt, h, min(TQ, s.ql - qt), D), qrow, b, wave, ln);
    stage<D, TQ, 8>(rows_rsrc(a.dO, (int64_t)s.cq + qt, h, min(TQ, s.ql - qt), D), drow, b + TILE, wave, ln);
    // one load each: a value a lane (zeros past the last query, whose dO is zeros)
    if (blk == 0) {
      const float* v = (second ? a.delta : a.lse2) + h * a.train_q + s.cq + qt;
      llvm_amdgcn_raw_buffer_load_lds_a(flat_rsrc(v, 4 * min(TQ, s.ql - qt)), (lds_u32*)(b + ST + (second ? 4 * TQ : 0)), 4,
                                        4 * ln, 0, 0, 0);
    }
  };
  if (steps > 0) load(0, b0, lane);
  bf16x8 kv[D / 16];  // the lane's key: K (first wave) or V
  row_frags<D>(second ? a.V : a.K, (int64_t)s.k0 + k, hk, in, kv);
  f32x16 acc[D / 32];  // dV or dK
#pragma unroll
  for (int t = 0; t < D / 32; ++t) acc[t] = zero16();
  const float c = a.scale * kLog2e;
  // First wave: p of 64 queries as two blocks, the terms of one beside the products of the other.  CUT: some
  // key lies behind a query's last one, or some query does not exist (its scores are 0 times the key: NaN where that is
  // infinite).
  auto form_p = [&](auto cut, char* cur, int qt, int ln) {
    constexpr bool CUT = decltype(cut)::value;
    constexpr int V = (CUT ? 112 : 64) * 16 / D + 1;
    const int first = k0 + 32 * blk + (ln & 31) - off;  // the first query that sees the lane's key
    const int ahead = qt + 4 * (ln >> 5) - first;
    const uint32_t seen_by = s.ql - first;
    f32x16 x[2];
    f32x4 l4[2][4];
    bf16x8 p[2][2];
    auto scores = [&](int u) {
      x[u] = zero16();
#pragma unroll
      for (int i = 0; i < 4; ++i) l4[u][i] = *reinterpret_cast<const f32x4*>(cur + ST + 4 * (32 * u + 8 * i + 4 * (ln >> 5)));
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
        x[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag<D>(cur, u, i, ln), kv[i], x[u], 0, 0, 0);
    };
    auto terms = [&](int u) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float e = __builtin_amdgcn_exp2f(x[u][v] * c - l4[u][v >> 2][v & 3]);
        x[u][v] = !CUT || (uint32_t)(ahead + 32 * u + 8 * (v >> 2) + (v & 3)) < seen_by ? e : 0.f;
      }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        p[u][w] = pack8(x[u], w);
        u32x4 h;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          h[e] = pack_p(x[u][8 * w + 2 * e], x[u][8 * w + 2 * e + 1]);
        *reinterpret_cast<u32x4*>(cur + 2 * TILE + ((blk * 4 + 2 * u + w) * 64 + ln) * 16) = h;
      }
    };
    auto product = [&](int u) {
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
          acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_t<D>(cur + TILE, 2 * u + w, t, ln), p[u][w], acc[t], 0, 0, 0);
    };
    __builtin_amdgcn_sched_barrier(0);
    scores(0);
    feed<D / 16, 1, 4>();
    __builtin_amdgcn_sched_barrier(0);
    scores(1);
    terms(0);
    feed_beside<D / 16, 1, 4, V>();
    __builtin_amdgcn_sched_barrier(0);
    product(0);
    terms(1);
    feed_beside<D / 16, 2, 2, V>();
    __builtin_amdgcn_sched_barrier(0);
    product(1);
    feed<D / 16, 2, 2>();
    __builtin_amdgcn_sched_barrier(0);
  };
  // Second wave: do . v of step n (NOW), and ds of the step before (PAST) with its product, a block of 32
  // queries after the other.
  auto form_ds = [&](auto now_c, auto past_c, f32x16 (&dp)[2], const char* cur, const char* old, int ln) {
    constexpr bool NOW = decltype(now_c)::value, PAST = decltype(past_c)::value;
    constexpr int V = 72 * 16 / D;
    bf16x8 ds[2];
    auto terms = [&](int u) {
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const u32x4 p = *reinterpret_cast<const u32x4*>(old + 2 * TILE + ((blk * 4 + 2 * u + w) * 64 + ln) * 16);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const f32x4 d4 = *reinterpret_cast<const f32x4*>(old + ST + 4 * (TQ + 32 * u + 16 * w + 8 * i + 4 * (ln >> 5)));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t pw = p[2 * i + e / 2];
            const float pf = __uint_as_float(e & 1 ? pw >> 2 & 0x3fffc000u : (pw & 0xffffu) << 14);
            dp[u][8 * w + 4 * i + e] = pf * (dp[u][8 * w + 4 * i + e] - d4[e]);
          }
        }
        ds[w] = pack8(dp[u], w);
      }
    };
    auto product = [&](int u, const bf16x8 (&d)[2]) {
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
          acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_t<D>(old, 2 * u + w, t, ln), d[w], acc[t], 0, 0, 0);
    };
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (PAST) {
      terms(0);
      const bf16x8 d0[2] = {ds[0], ds[1]};
      __builtin_amdgcn_sched_barrier(0);
      product(0, d0);
      terms(1);
      feed_beside<D / 16, 2, 2, V>();
      __builtin_amdgcn_sched_barrier(0);
      product(1, ds);
      feed<D / 16, 2, 2>();
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (NOW) {
      dp[0] = dp[1] = zero16();
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          dp[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag<D>(cur + TILE, u, i, ln), kv[i], dp[u], 0, 0, 0);
      feed<D / 8, 1, 4>();
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Step n, 0 to steps: its rows have landed, the next ones are under way.  (The three buffers lie further apart
  // than an LDS offset reaches: kept in registers, three sets of addresses spill.)
  auto begin = [&](int n, char* nxt) {
    vmem_wait_all();
    __syncthreads();
    const int ln = fresh_lane();
    if (n + 1 < steps) load(n + 1, nxt, ln);
    return ln;
  };
  if (!second) {
    auto step = [&](int n, char* cur, char* nxt) {
      const int ln = begin(n, nxt);
      if (n == steps) return;
      const int qt = q_of(n);
      if (k0 + 32 * blk + 31 > qt + off || qt + TQ > s.ql) form_p(bool_c<true>{}, cur, qt, ln);
      else form_p(bool_c<false>{}, cur, qt, ln);
    };
    for (int n = 0; n <= steps; n += 3) {
      step(n, b0, b1);
      if (n + 1 <= steps) step(n + 1, b1, b2);
      if (n + 2 <= steps) step(n + 2, b2, b0);
    }
  } else {
    f32x16 dp[2];  // do . v of the step before
    auto step = [&](int n, const char* cur, const char* old, char* nxt) {
      const int ln = begin(n, nxt);
      if (n > 0) form_ds(bool_c<false>{}, bool_c<true>{}, dp, cur, old, ln);
      if (n < steps) form_ds(bool_c<true>{}, bool_c<false>{}, dp, cur, old, ln);
    };
    for (int n = 0; n <= steps; n += 3) {
      step(n, b0, b2, b1);
      if (n + 1 <= steps) step(n + 1, b1, b0, b2);
      if (n + 2 <= steps) step(n + 2, b2, b1, b0);
    }
  }
  if (!in) return;
  if (it[5] > 1) {
    float* p = a.part_o + ((((int64_t)it[4] * a.hkv + hk) * 2 + (second ? 0 : 1)) * kAttnBwdRows + 32 * blk + (lane & 31)) * D +
               4 * (lane >> 5);
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(p + 32 * t + 8 * i) =
            f32x4{acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]};
    return;
  }
  if (second) store_cols<D>(a.dK, (int64_t)s.ck + k, hk, acc, a.scale);
  else store_cols<D>(a.dV, (int64_t)s.ck + k, hk, acc, 1.f);
}

// Pieces of gradients, n of them `step` rows of D apart from p on, added in order and stored times f: columns
// c0 .. c0 + D / 8 of a row of t.
template <int D>
__device__ __forceinline__ void join_grad(const float* p, int64_t step, int n, const AttnView& t, int64_t row, int h, int c0,
                                          float f) {
  f32x4 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int k = 0; k < n; ++k)
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] += *reinterpret_cast<const f32x4*>(p + k * step * D + c0 + 4 * i);
  uint16_t* out = static_cast<uint16_t*>(t.ptr) + row * t.row + h * t.head + c0;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
    *reinterpret_cast<uint2*>(out + 4 * i) = make_uint2(f2bf2(o[i][0] * f, o[i][1] * f), f2bf2(o[i][2] * f, o[i][3] * f));
}

// Gradients of tiles in pieces, dQ first, then dK (half 0) and dV: 32 rows a workgroup, row tid / 8, D / 8 columns each.
template <int D>
__global__ __launch_bounds__(256) void attn_grad_join_kernel(AttnArgs a) {
  constexpr int BL = kAttnBwdRows / 32;
  const int c0 = (threadIdx.x & 7) * (D / 8);
  int at = blockIdx.x;
  if (at < a.first_groups) {
    const int h = at / BL % a.hq, r = 32 * (at % BL) + (threadIdx.x >> 3);
    const int32_t* it = a.first_join + 4 * (int64_t)(at / (BL * a.hq));
    const Seq s(a, it[0]);
    if (it[1] + r >= s.ql) return;
    join_grad<D>(a.first_o + (((int64_t)it[2] * a.hq + h) * kAttnBwdRows + r) * D, (int64_t)a.hq * kAttnBwdRows, it[3], a.dQ,
                 (int64_t)s.cq + it[1] + r, h, c0, a.scale);
    return;
  }
  at -= a.first_groups;
  const int half = at & 1, hk = at / (2 * BL) % a.hkv, r = 32 * (at / 2 % BL) + (threadIdx.x >> 3);
  const int32_t* it = a.items + 4 * (int64_t)(at / (2 * BL * a.hkv));
  const Seq s(a, it[0]);
  if (it[1] + r >= s.kl) return;
  join_grad<D>(a.part_o + ((((int64_t)it[2] * a.hkv + hk) * 2 + half) * kAttnBwdRows + r) * D,
               (int64_t)a.hkv * 2 * kAttnBwdRows, it[3], half ? a.dV : a.dK, (int64_t)s.ck + it[1] + r, hk, c0,
               half ? 1.f : a.scale);
}

// ---- host -------------------------------------------------------------------------------------------
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

struct Workspace {
  size_t split_o, split_ml, fwd_o, fwd_ml;  // forward
  size_t delta, lse2, dq, dk;               // backward (the two do not overlap on a stream: one room)
  size_t total;
};

// fp32 key tiles of short batches are fewer than the CUs: the query heads of a key head are then divided among so many
// workgroups.
int f32_parts(const dsv_attn_plan& p) {
  const int64_t tiles = std::max<int64_t>(1, (int64_t)p.n_f32_dk * p.hkv);
  return (int)std::min<int64_t>(p.hq / p.hkv, (kAttnDkSlots + tiles - 1) / tiles);
}

Workspace carve(const dsv_attn_plan& p, dsv_dtype dt) {
  Workspace w{};
  size_t at = 0;
  auto room = [&](size_t floats) {
    const size_t o = at;
    at += align256(floats * sizeof(float));
    return o;
  };
  const bool bf = dt == DSV_BF16;
  const size_t split = bf && p.n_split > p.n_join ? (size_t)p.n_split * p.hkv : 0;  // some tile has several pieces
  const size_t tiles = bf ? (size_t)p.fwd_slots * p.hq : 0;
  w.split_o = room(split * kAttnPackRows * p.d);
  w.split_ml = room(split * 2 * kAttnPackRows);
  w.fwd_o = room(tiles * kAttnFwdRows * p.d);
  w.fwd_ml = room(tiles * 2 * kAttnFwdRows);
  const size_t fwd = at;
  at = 0;
  w.delta = room((size_t)p.train_q * p.hq);
  w.lse2 = room(bf ? (size_t)p.train_q * p.hq : 0);
  w.dq = room(bf ? (size_t)p.dq_slots * p.hq * kAttnBwdRows * p.d : 0);
  const int parts = f32_parts(p);
  w.dk = room(bf          ? (size_t)p.dk_slots * p.hkv * 2 * kAttnBwdRows * p.d
              : parts > 1 ? (size_t)p.n_f32_dk * p.hkv * parts * 2 * kAttnF32Rows * p.d
                          : 0);
  w.total = std::max<size_t>(256, std::max(at, fwd));
  return w;
}

template <typename T>
T* at(void* ws, size_t off) {
  return reinterpret_cast<T*>(static_cast<char*>(ws) + off);
}

constexpr int64_t kMaxRowStride = 1 << 23, kMaxHeadStride = (int64_t)1 << 40;

// The view with dense strides filled in; out: its vectors must be apart.
int view(const dsv_attn_view* v, int64_t rows, int32_t heads, int32_t d, bool out, AttnView* to) {
  if (!v) return DSV_ERR_ARG;
  to->ptr = v->ptr;
  to->row = v->row == 0 ? (int64_t)heads * d : v->row;
  to->head = v->head == 0 ? d : v->head;
  if (reinterpret_cast<uintptr_t>(v->ptr) & 15) return DSV_ERR_ARG;
  if (rows > 0 && !v->ptr) return DSV_ERR_ARG;
  if (to->row < d || to->head < d || (to->row & 7) || (to->head & 7) || to->row > kMaxRowStride ||
      to->head > kMaxHeadStride)
    return DSV_ERR_SIZE;
  if (out && rows > 0 && to->row < (heads - 1) * to->head + d && to->head < (rows - 1) * to->row + d) return DSV_ERR_SIZE;
  return DSV_OK;
}

int check(const dsv_attn_plan* p, dsv_dtype dt, double scale) {
  if (!p || !p->d_meta) return DSV_ERR_ARG;
  if (dt != DSV_BF16 && dt != DSV_F32) return DSV_ERR_RANGE;
  const float f = (float)scale;  // what the kernels multiply with, and in bf16 mode f log2 e
  if (!std::isfinite(scale) || !(f > 0) || !std::isfinite(f * kLog2e)) return DSV_ERR_RANGE;
  return DSV_OK;
}

AttnArgs common(const dsv_attn_plan& p, double scale) {
  AttnArgs a{};
  a.seqs = p.dptr(p.lay.seqs);
  a.hq = p.hq;
  a.hkv = p.hkv;
  a.group = p.hq / p.hkv;
  a.d = p.d;
  a.n_q = p.n_q;
  a.train_q = p.train_q;
  a.scale = (float)scale;
  return a;
}

int status(hipError_t e) { return e == hipSuccess ? DSV_OK : DSV_ERR_DEVICE; }

template <typename K>
hipError_t launch(K k64, K k128, const AttnArgs& a, int64_t groups, hipStream_t s, int threads = 256) {
  if (groups <= 0) return hipSuccess;
  hipLaunchKernelGGL(a.d == 64 ? k64 : k128, dim3((unsigned)groups), dim3((unsigned)threads), 0, s, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace dsv

using namespace dsv;

extern "C" int dsv_attn_workspace(const dsv_attn_plan* p, dsv_dtype dt, size_t* bytes) {
  if (!p || !bytes) return DSV_ERR_ARG;
  if (dt != DSV_BF16 && dt != DSV_F32) return DSV_ERR_RANGE;
  *bytes = carve(*p, dt).total;
  return DSV_OK;
}

extern "C" int dsv_attn_fwd(const dsv_attn_plan* p, dsv_dtype dt, double scale, const dsv_attn_view* Q,
                            const dsv_attn_view* K, const dsv_attn_view* V, const dsv_attn_view* O, float* lse,
                            void* ws, size_t ws_bytes, void* hip_stream) {
  int rc = check(p, dt, scale);
  if (rc != DSV_OK) return rc;
  AttnArgs a = common(*p, scale);
  if ((rc = view(Q, p->n_q, p->hq, p->d, false, &a.Q)) != DSV_OK) return rc;
  if ((rc = view(K, p->n_kv, p->hkv, p->d, false, &a.K)) != DSV_OK) return rc;
  if ((rc = view(V, p->n_kv, p->hkv, p->d, false, &a.V)) != DSV_OK) return rc;
  if ((rc = view(O, p->n_q, p->hq, p->d, true, &a.O)) != DSV_OK) return rc;
  if (reinterpret_cast<uintptr_t>(lse) & 3) return DSV_ERR_ARG;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return DSV_ERR_ARG;
  const Workspace w = carve(*p, dt);
  if (ws_bytes < w.total) return DSV_ERR_SIZE;
  a.lse = lse;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (dt == DSV_F32) {
    a.items = p->dptr(p->lay.f32_items);
    a.n_items = p->n_f32;
    return status(launch_attn_f32_fwd(a, s));
  }
  const int64_t hq = p->hq, hkv = p->hkv;
  a.items = p->dptr(p->lay.fwd_items);
  a.first_o = a.part_o = at<float>(ws, w.fwd_o);
  a.first_ml = a.part_ml = at<float>(ws, w.fwd_ml);
  hipError_t e = launch(attn_fwd_kernel<64>, attn_fwd_kernel<128>, a, p->n_fwd * hq, s);
  if (e != hipSuccess) return status(e);
  a.items = p->dptr(p->lay.split_items);
  a.part_o = at<float>(ws, w.split_o);
  a.part_ml = at<float>(ws, w.split_ml);
  e = launch(attn_split_kernel<64>, attn_split_kernel<128>, a, p->n_split * hkv, s);
  if (e != hipSuccess) return status(e);
  a.items = p->dptr(p->lay.join_items);
  a.first_join = p->dptr(p->lay.fwd_join);
  a.first_groups = (int32_t)(p->n_fwd_join * hq * (kAttnFwdRows / 32));
  const int64_t split = p->n_split == p->n_join ? 0 : p->n_join * hkv;  // one piece each: nothing to join
  return status(launch(attn_join_kernel<64>, attn_join_kernel<128>, a, a.first_groups + split, s));
}

extern "C" int dsv_attn_bwd(const dsv_attn_plan* p, dsv_dtype dt, double scale, const dsv_attn_view* Q,
                            const dsv_attn_view* K, const dsv_attn_view* V, const dsv_attn_view* O, const float* lse,
                            const dsv_attn_view* dO, const dsv_attn_view* dQ, const dsv_attn_view* dK,
                            const dsv_attn_view* dV, void* ws, size_t ws_bytes, void* hip_stream) {
  int rc = check(p, dt, scale);
  if (rc != DSV_OK) return rc;
  AttnArgs a = common(*p, scale);
  if ((rc = view(Q, p->n_q, p->hq, p->d, false, &a.Q)) != DSV_OK) return rc;
  if ((rc = view(K, p->n_kv, p->hkv, p->d, false, &a.K)) != DSV_OK) return rc;
  if ((rc = view(V, p->n_kv, p->hkv, p->d, false, &a.V)) != DSV_OK) return rc;
  if ((rc = view(O, p->n_q, p->hq, p->d, false, &a.O)) != DSV_OK) return rc;
  if ((rc = view(dO, p->train_q, p->hq, p->d, false, &a.dO)) != DSV_OK) return rc;
  if ((rc = view(dQ, p->train_q, p->hq, p->d, true, &a.dQ)) != DSV_OK) return rc;
  if ((rc = view(dK, p->train_k, p->hkv, p->d, true, &a.dK)) != DSV_OK) return rc;
  if ((rc = view(dV, p->train_k, p->hkv, p->d, true, &a.dV)) != DSV_OK) return rc;
  if ((p->train_q > 0 && !lse) || (reinterpret_cast<uintptr_t>(lse) & 3)) return DSV_ERR_ARG;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return DSV_ERR_ARG;
  const Workspace w = carve(*p, dt);
  if (ws_bytes < w.total) return DSV_ERR_SIZE;
  a.lse = const_cast<float*>(lse);
  a.delta = at<float>(ws, w.delta);
  a.lse2 = at<float>(ws, w.lse2);
  a.part_o = at<float>(ws, w.dk);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int64_t hq = p->hq, hkv = p->hkv;
  if (dt == DSV_F32) {
    a.items = p->dptr(p->lay.f32_dq_items);
    a.n_items = p->n_f32_dq;
    const hipError_t e = launch_attn_f32_dq(a, s);
    if (e != hipSuccess) return status(e);
    a.items = p->dptr(p->lay.f32_dk_items);
    a.n_items = p->n_f32_dk;
    a.parts = f32_parts(*p);
    return status(launch_attn_f32_dk(a, s));
  }
  a.items = p->dptr(p->lay.dq_items);
  a.first_o = a.part_o = at<float>(ws, w.dq);
  hipError_t e = launch(attn_dq_kernel<64>, attn_dq_kernel<128>, a, p->n_dq * hq, s);
  if (e != hipSuccess) return status(e);
  a.items = p->dptr(p->lay.dk_items);
  a.part_o = at<float>(ws, w.dk);
  e = launch(attn_dk_kernel<64>, attn_dk_kernel<128>, a, p->n_dk * hkv, s, 512);
  if (e != hipSuccess) return status(e);
  a.items = p->dptr(p->lay.dk_join);
  a.first_join = p->dptr(p->lay.dq_join);
  constexpr int blocks = kAttnBwdRows / 32;
  a.first_groups = (int32_t)(p->n_dq_join * hq * blocks);
  return status(launch(attn_grad_join_kernel<64>, attn_grad_join_kernel<128>, a,
                       a.first_groups + p->n_dk_join * hkv * 2 * blocks, s));
}
