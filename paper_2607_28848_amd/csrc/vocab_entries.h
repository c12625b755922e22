// vocab_entries.h -- the entries' logits of a distillation, beside the tiles of the logits' launch.
#pragma once

#include "device_common.h"
#include "vocab.h"

namespace dsv {
namespace {

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

// A sum over a workgroup of four waves.
__device__ __forceinline__ double sum_of_four(double x, double* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}

// The teacher's shares of a row's entries: its softmax over them, in 64 bits.
__device__ __forceinline__ void teacher_shares(const VocabArgs& a, int64_t row) {
  __shared__ double red[4];
  __shared__ int32_t ids[kMaxEntries];
  const double c = a.inv_tau * 1.4426950408889634;
  // an entry's logit, -infinity where it is none
  auto logit = [&](int j) { return (uint32_t)ids[j] < (uint32_t)a.V ? a.teacher[row * a.k + j] * c : -INFINITY; };
  double top = -INFINITY;
  for (int j = threadIdx.x; j < a.k; j += 256) {
    ids[j] = a.ids[row * a.k + j];
    top = fmax(top, logit(j));
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmax(top, __shfl_xor(top, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmax(fmax(red[0], red[1]), fmax(red[2], red[3]));
  auto term = [&](double t) { return t == -INFINITY ? 0. : exp2(t - top); };
  double mass = 0.;
  for (int j = threadIdx.x; j < a.k; j += 256) mass += term(logit(j));
  mass = sum_of_four(mass, red);
  const double log_mass = log2(mass);
  for (int j = threadIdx.x; j < a.k; j += 256) {
    const double t = logit(j), x = term(t), q = x == 0. ? 0. : x / mass;
    bool again = false;  // the token stands at an earlier entry too
    for (int i = 0; i < j; ++i) again |= ids[i] == ids[j];
    a.share[row * a.k + j] = (float)(again ? -q : q);
    a.log_share[row * a.k + j] = t == -INFINITY ? t : t - top - log_mass;
  }
  if (threadIdx.x == 0) a.term[row] = mass == 0. ? 0.f : 1.f;
}

// A bit for each element of a logits tile that is an entry's, [rows][columns / 32]: the products' terms there are left out of
// P and of the sums.  The tile's rows of ids are one run of memory, four a load whatever their alignment.  The first B loads a
// thread go out at the start, and a barrier stands between that and put(); mark is complete behind the barrier after it.  16 rows
// of 20 entries against 128256 of 4096: 197 us a call so, 193 with the entries' terms left in the sums; 1024 of 64 and 8192, with
// the gradient, 3.75 ms and 3.73.
template <int TM, int TN, int B>
struct EntryMarks {
  struct __attribute__((packed, aligned(4))) Four {
    int32_t id[4];
  };
  const int32_t* ids;
  int n;
  float rows_per;  // the row of number i, up to 2^18, from a quotient at least 1 / (2 k) from a whole number
  Four x[B];
  __device__ __forceinline__ EntryMarks(const VocabArgs& a, int m0, uint32_t (&mark)[TM][TN / 32]) {
    ids = a.ids + (int64_t)m0 * a.k;
    n = min(TM, a.T - m0) * a.k;
    rows_per = 1.f / a.k;
    if (n >= 4) load(0);
    for (int i = threadIdx.x; i < TM * TN / 32; i += 256) (&mark[0][0])[i] = 0;
  }
  __device__ __forceinline__ void load(int i0) {
#pragma unroll
    for (int b = 0; b < B; ++b) x[b] = *reinterpret_cast<const Four*>(ids + min(i0 + 1024 * b + 4 * (int)threadIdx.x, n - 4));
  }
  // first, cols: the tile's columns of the vocabulary
  __device__ __forceinline__ void put(uint32_t (&mark)[TM][TN / 32], uint32_t first, int cols) {
    auto one = [&](int i, int id) {
      const uint32_t c = (uint32_t)id - first;
      if (c < (uint32_t)cols) atomicOr(&mark[(int)((i + 0.5f) * rows_per)][c >> 5], 1u << (c & 31));
    };
    for (int i0 = 0; i0 < n - 3;) {
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const int i = i0 + 1024 * b + 4 * (int)threadIdx.x;
        if (i < n - 3)
#pragma unroll
          for (int e = 0; e < 4; ++e) one(i + e, x[b].id[e]);
      }
      i0 += 1024 * B;
      if (i0 < n - 3) load(i0);
    }
    if ((int)threadIdx.x < (n & 3)) one((n & ~3) + threadIdx.x, ids[(n & ~3) + threadIdx.x]);
  }
};

// The student's exponents at a teacher's tokens: products of a row with the head's rows in 64 bits from 8 products on,
// times c.  The student's terms of the entries are kept out of P and of the sums and formed from these, so that where
// student and teacher agree their difference, not bf16's rounding of both, is what reaches dX, and a loss near 0 keeps its
// accuracy.  A workgroup of four waves takes kEntryGroup entries of a row, a wave four of them side by side.  They go in
// the launch of the first piece's logits, ahead of its tiles, which they do not wait for (16 rows of 4096, 20 entries:
// 18 us in a launch of their own).  A row's first group forms the teacher's shares as well where they are few
// (a.shares_ahead).
template <typename T, bool SHARES = true>
__device__ __forceinline__ void entry_exponents(const VocabArgs& a, int block) {
  const int groups = entry_groups(a.k);
  const int64_t row = block / groups;
  const int lane = threadIdx.x & 63, j0 = kEntryGroup * (block % groups) + 4 * (int)(threadIdx.x >> 6);
  const T* x = static_cast<const T*>(a.X) + row * a.ldx;
  const T* w[4];
  bool is[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int id = j0 + e < a.k ? a.ids[row * a.k + j0 + e] : -1;
    is[e] = (uint32_t)id < (uint32_t)a.V;
    w[e] = static_cast<const T*>(a.W) + (is[e] ? id : 0) * a.ldw;
  }
  double z[4] = {0., 0., 0., 0.};
#pragma unroll 2
  for (int at = 8 * lane; at < a.K; at += 512) {
    float xs[8], ws[4][8];
    load8(x + at, xs);
#pragma unroll
    for (int e = 0; e < 4; ++e) load8(w[e] + at, ws[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float part = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) part += xs[i] * ws[e][i];
      z[e] += part;
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) z[e] += __shfl_xor(z[e], d);
    if (lane == e && j0 + e < a.k) a.exponent[row * a.k + j0 + e] = is[e] ? z[e] * (a.inv_tau * 1.4426950408889634) : -INFINITY;
  }
  if constexpr (SHARES) {
    if (a.shares_ahead && block % groups == 0) teacher_shares(a, row);
  }
}

}  // namespace
}  // namespace dsv
