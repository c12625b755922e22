// vocab.h -- arguments and host launchers of the vocabulary loss's kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace dsv {

// One piece of the vocabulary: columns [v0, v0 + vn) of the logits, in column tiles of `tw`.
struct VocabArgs {
  int32_t T, K, V;
  const void* X;
  const void* W;
  const void* Wt;         // nullptr: the second product reads W
  int64_t ldx, ldw, ldwt, lddx;
  const int32_t* target;
  const float* weight;    // nullptr: ones
  float* loss;            // nullptr: not written
  void* dX;
  int32_t v0, vn;
  int32_t tw, n_ct;       // width and number of the piece's column tiles
  int32_t first, last;    // the piece is the first / the last
  int32_t grad;
  // Exponents are base 2: a row's reference r stands for 2^r.
  void* P;                // [T][ldp] 2^(z log2 e - reference) of the piece, the target's left out (grad)
  int64_t ldp;
  float2* stats;          // [T][ld_stats] per column tile: reference, sum of its P
  int64_t ld_stats;
  float* ref;             // [T] the row's reference
  float* others;          // [T] sum of the terms that are not the target's, at the reference
  float* term;            // [T] the target's term at the reference (after the last piece)
  float* alpha;           // [T] what the sums so far are multiplied by (the reference moved)
  // second product: contraction in `split` ranges of split_len columns, each with its own sums
  float* O;               // [split][T][K]
  int32_t split, split_len;
};

// References.  A row starts at 0, and a tile of the first piece takes its own maximum (m, base 2) where it lies
// further than kVocabSlack from that on either side; in later pieces where it exceeds the row's reference by
// more.  So terms stay below 2^kVocabSlack and the row's largest far from underflow, and for all but unusual
// logits every tile of a row has one reference: its terms need no second look.  References are whole numbers, so that
// terms go from one to another by a power of two, which rounds nothing.
constexpr float kVocabSlack = 60.f;

__device__ __forceinline__ float tile_reference(float m, float have, bool first) {
  return m > have + kVocabSlack || (first && m < have - kVocabSlack) ? ceilf(m) : have;
}

// Rows of an fp32 tile (20 rows against 20000 of 1024, with the gradient: 56 us in tiles of 32, 94 in one of 64 rows).
inline int vocab_f32_rows(int32_t T) { return T <= 32 ? 32 : 64; }

hipError_t launch_vocab_f32_logits(const VocabArgs& a, int cus, hipStream_t s);
hipError_t launch_vocab_f32_grad(const VocabArgs& a, hipStream_t s);

}  // namespace dsv
