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
  float c;                // log2 e over the temperature: exponents are c z
  const int32_t* target;
  const float* weight;    // nullptr: ones
  float* loss;            // nullptr: not written
  void* dX;
  int32_t v0, vn;
  int32_t tw, n_ct;       // width and number of the piece's column tiles
  int32_t first, last;    // the piece is the first / the last
  int32_t grad;
  // Exponents are base 2: a row's reference r stands for 2^r.
  void* P;                // [T][ldp] 2^(c z - reference) of the piece, the target's or the entries' left out (grad)
  int64_t ldp;
  float2* stats;          // [T][ld_stats] per column tile: reference, sum of its P
  int64_t ld_stats;
  float* ref;             // [T] the row's reference
  float* others;          // [T] sum of the terms that are not the target's or the entries', at the reference; distillation:
                          // after the last piece the sum of all
  float* term;            // [T] the target's term at the reference (after the last piece); distillation: whether the row has
                          // an entry of share > 0 (0: no, 2: and one of them names an earlier one's token)
  float* alpha;           // [T] what the sums so far are multiplied by (the reference moved)
  // Distillation: k entries a row, [T][k] each, and what the rows' sums of them come to.
  const int32_t* ids;
  const float* teacher;
  int32_t k;
  int32_t n_entry;        // workgroups of entry_exponents ahead of the launch's tiles
  int32_t shares_ahead;   // they form the teacher's shares too; else the first fold does
  double inv_tau;
  double* exponent;       // c z of the entry, -infinity where it is none; after the first fold also where its token stands
                          // at an earlier one
  float* share;           // the teacher's probability of it; below 0 (or -0) until the first fold where its token stands earlier
  double* log_share;      // its logarithm, base 2
  double* base;           // [T] sum of the probabilities (in 64 bits) times log_share - c z
  // second product: contraction in `split` ranges of split_len columns, each with its own sums
  float* O;               // [split][T][K]
  int32_t split, split_len;
};

// Distillation: the most entries a row, and how many of them a workgroup takes.
constexpr int kMaxEntries = 1024, kEntryGroup = 16;
__host__ __device__ inline int entry_groups(int k) { return (k + kEntryGroup - 1) / kEntryGroup; }

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
