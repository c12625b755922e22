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
  int32_t parts;         // fp32 dK and dV: ranges of a key head's query heads, or of the steps of
  int32_t cut;           // the first `cut` items, with a window (the others are whole)
  int32_t hq, hkv, group, d;
  int32_t n_q;           // row length of lse ([hq][n_q])
  int64_t train_q;       // row length of delta ([hq][train_q])
  float scale;           // of the scores
  int32_t window, sinks; // kernels of plans with a window
  AttnView Q, K, V, O, dO, dQ, dK, dV;
  float* lse;            // nullptr: not written (forward)
  float* delta;          // do . o of the compact rows, [hq][train_q]
  float* lse2;           // bf16: lse of the compact rows, base 2
  // Sums of pieces, by slot.  Split form: [slot][hkv][kAttnPackRows][D] sums of 2^(s - m) v, and
  // [slot][hkv][2][kAttnPackRows] m and sum of 2^(s - m).  Forward tiles: the same with hq and kAttnFwdRows.
  // Query tiles: [slot][hq][kAttnBwdRows][D].  Key tiles: [slot][hkv][dK, dV][kAttnBwdRows][D].
  // fp32 key tiles (cut ones): [item][hkv][part][dK, dV][kAttnF32Rows][D].
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

// The keys that a tile of queries walks in a plan with a window (WIN): blocks of the sinks alone, which `sink` counts, and
// behind them blocks from the first key of the first query's window on.  Key kv of the count is key at(kv) of the sequence.
template <bool WIN>
struct AttnKeys {
  int sink, shift;
  __device__ __forceinline__ AttnKeys(int s, int further) : sink(WIN ? s : 0), shift(WIN ? further : 0) {}
  __device__ __forceinline__ int at(int kv) const { return WIN && kv >= sink ? kv + shift : kv; }
  // One past the last key that the block may hold.
  __device__ __forceinline__ int end(const AttnArgs& a, int kv, int kl) const { return WIN && kv < sink ? a.sinks : kl; }
  // Keys a query looks back over in the block, sinks apart.
  __device__ __forceinline__ uint32_t back(const AttnArgs& a, int kv) const { return WIN && kv < sink ? 0u : (uint32_t)a.window; }
  // Whether queries whose last keys are `first` and more have the n keys from kt on behind their windows.
  __device__ __forceinline__ static bool passed(const AttnArgs& a, int kt, int n, int first) {
    return WIN && kt >= a.sinks && first - (kt + n - 1) >= a.window;
  }
  // Whether queries whose last keys are up to `last` have some of the n keys from kt on behind their windows.
  __device__ __forceinline__ static bool cut(const AttnArgs& a, uint32_t back, int kt, int n, int last) {
    return WIN && kt + n > a.sinks && last - kt >= (int)back;
  }
  // Whether a query whose last key is `seen` (-1 or more) sees `key`; seen - key of a later key is a large unsigned number.
  __device__ __forceinline__ static bool sees(const AttnArgs& a, uint32_t back, int seen, int key) {
    return WIN ? (uint32_t)(seen - key) < (key < a.sinks ? 0x80000000u : back) : key <= seen;
  }
  // Whether no query of a sequence whose first query's last key is `off` sees the key.
  __device__ __forceinline__ static bool unseen(const AttnArgs& a, int off, int key) {
    return WIN && key >= a.sinks && off - key >= a.window;
  }
};

// fp32 mode: tiles of kAttnF32Rows.  windowed: the plan has a window.
hipError_t launch_attn_f32_fwd(const AttnArgs& a, bool windowed, hipStream_t s);
hipError_t launch_attn_f32_dq(const AttnArgs& a, hipStream_t s);  // dQ, and delta for the next launch
hipError_t launch_attn_f32_dk(const AttnArgs& a, hipStream_t s);  // dK, dV
// Plans with a window: dQ, dK and dV; a's items are the key tiles'.
hipError_t launch_attn_f32_grad(AttnArgs a, const int32_t* dq_items, int32_t n_dq, hipStream_t s);

}  // namespace dsv
