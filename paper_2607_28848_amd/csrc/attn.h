// attn.h -- arguments and host launchers of the attention kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

namespace dsv {

// A tensor [rows][heads][D] with its strides in elements.
struct AttnView {
  void* ptr;
  int64_t row, head;
};

struct AttnArgs {
  const int32_t* seqs;   // sequence descriptors (attn_plan.h)
  const int32_t* items;  // the launch's work items
  int32_t n_items;       // fp32 launches
  int32_t parts;         // fp32 dK and dV: ranges of a key head's query heads
  int32_t hq, hkv, group, d;
  int32_t n_q;           // row length of lse ([hq][n_q])
  int64_t train_q;       // row length of delta ([hq][train_q])
  float scale;           // of the scores
  AttnView Q, K, V, O, dO, dQ, dK, dV;
  float* lse;            // nullptr: not written (forward)
  float* delta;          // do . o of the compact rows, [hq][train_q]
  float* lse2;           // bf16: lse of the compact rows, base 2
  // Sums of pieces, by slot.  Split form: [slot][hkv][kAttnPackRows][D] sums of 2^(s - m) v, and
  // [slot][hkv][2][kAttnPackRows] m and sum of 2^(s - m).  Forward tiles: the same with hq and kAttnFwdRows.
  // Query tiles: [slot][hq][kAttnBwdRows][D].  Key tiles: [slot][hkv][dK, dV][kAttnBwdRows][D].  fp32 key tiles: [item][hkv][part][dK, dV][kAttnF32Rows][D].
  float* part_o;
  float* part_ml;
  // A join's first part (forward tiles, dQ): its sums, items and workgroups; the rest is as above.
  const float* first_o;
  const float* first_ml;
  const int32_t* first_join;
  int32_t first_groups;
};

// What the backward subtracts from a row's scores: its lse, or infinity where that is -infinity (no key, or none of a
// score above -infinity), so that every p of the row is 0.
__device__ __forceinline__ float exp_from(float lse) { return lse == -INFINITY ? INFINITY : lse; }

// fp32 mode: tiles of kAttnF32Rows.
hipError_t launch_attn_f32_fwd(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_f32_dq(const AttnArgs& a, hipStream_t s);  // dQ, and delta for the next launch
hipError_t launch_attn_f32_dk(const AttnArgs& a, hipStream_t s);  // dK, dV

}  // namespace dsv
