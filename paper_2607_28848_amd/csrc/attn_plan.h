// attn_plan.h -- host plan and packed device metadata of a mixed batch's attention.
#pragma once

#include <cstddef>
#include <cstdint>
#include <vector>

#include "dsv.h"

namespace dsv {

// sequence descriptor: {q_start, q_len, k_start, k_len, compact q row, compact k row, 0, 0}
// (compact rows: -1 unless the sequence is a fine-tuning sample)
constexpr int kAttnSeqWords = 8;
// Rows of a forward tile (bf16), of a gradient tile (bf16: queries, keys) and of the fp32 tiles.
constexpr int kAttnFwdRows = 128;
constexpr int kAttnBwdRows = 128;
constexpr int kAttnF32Rows = 16;
// A sequence of up to kAttnSplitQ queries takes the split form: the (query, head) pairs of a
// key head form rows, kAttnPackRows to a tile, and the keys are split into pieces.  Heads of 128, split form and tiles:
// 16 queries behind 5000 keys, 32 heads on 8, 14.1 us and 22.4; 20 14.3 and 23.0; 64 18.5 and 26.6.  16 sequences of
// 16 or 20 queries behind 600 keys, 11.6 and 21.1 or 18.9 and 21.0; of 40, 27.9 and 21.8.  16 prompts of 16 tokens, 6.5
// and 5.9; of 20, 9.5 and 6.6.  So one limit on the queries is ahead up to 16 but for short prompts, and one sequence
// behind a long prefix would gain from a higher one.
constexpr int kAttnSplitQ = 16;
constexpr int kAttnPackRows = 32;
// Pieces of the split form: multiples of kAttnPieceKeys keys (each of the workgroup's four waves takes blocks of
// 32 of them by turns), of a length that makes about as many as run at a time (one workgroup per CU with heads of
// 128, two with 64; 64 sequences of 2600 keys: 104 us in 536 pieces, 114 in 1144).  Where no sequence has more than
// kAttnWholeKeys keys each is one piece: the join's launch costs more than the shorter walk saves.
// In pieces of 256 and whole, 8 sequences on 8 key heads of 128: 300 keys, 9.6 us and 7.5; 600 keys, 9.9 and 9.6; 1000 keys,
// 10.6 and 12.9; 1500 keys, 15.8 and 17.7 (1 or 2 sequences: 10 us in pieces of any of these; whole 7.4, 9.5, 12.3, 16;
// 32 sequences: the same either way from 600 keys on).  So the two cross between 600 and 1000 keys, and the limit lies
// above that by up to 2.5 us.
constexpr int kAttnPieceKeys = 256;
constexpr int kAttnWholeKeys = 1024;
constexpr int kAttnSplitTarget = 256;

// A forward, query or key tile with far more work than its share of the device (few tiles over long rows: a
// chunk behind a long prefix, short batches' gradients) is cut along its sum into pieces, whose fp32 sums another
// kernel adds.  Slots: workgroups that run at a time (two of attn_fwd per CU, one of attn_dk).  A piece is not shorter
// than so many steps of 64 rows: below that its start and the join cost more than it saves.  One sample of 2048, 8
// heads of 128: dQ 56 us whole, 31 in pieces and 3 more for the join; two samples of 111, 8 key heads for 32: dK and dV
// 25 us whole, 17 and 4 in pieces of 4 steps.  Forward pieces of 4 steps: 30 us with the join where those of 8 take 25
// (a sample of 1096 and three prompts, 14 heads on 2).
constexpr int kAttnFwdSlots = 512;
constexpr int kAttnDkSlots = 256;
constexpr int kAttnFwdPieceSteps = 8;
constexpr int kAttnGradPieceSteps = 4;

// A plan with a window: a query tile (or a sequence of the split form) walks blocks of the sinks alone and, behind them,
// blocks from the first key of its first query's window on; keys are counted through both.

// tile descriptor: {sequence, first row, first step, last step + 1, slot of its sums, pieces, x, y}
// query tiles: x keys' worth of sinks' blocks, y to be added to the count of a key behind them; key tiles: x one past the
// last query
constexpr int kAttnTileWords = 8;

// split form descriptor: {q_start, q_len, k_start, k_len, first row, pieces, slot (join: the first one's), first key,
// last key + 1, the tiles' x and y, 0}.  The sequence's fields stand in the item: short calls wait for every load that
// another one's address depends on.
constexpr int kAttnSplitWords = 12;

// Word offsets inside the packed blob (int32 words).
struct AttnLayout {
  int64_t seqs;         // [n_seqs][kAttnSeqWords]
  int64_t fwd_items;    // [n_fwd][kAttnTileWords]: bf16 forward tiles or their pieces, steps of 64 keys
  int64_t fwd_join;     // [n_fwd_join][4] {sequence, first query, first slot, pieces}
  int64_t f32_items;    // [n_f32][2] {sequence, first query}: fp32 forward tiles of every sequence
  int64_t split_items;  // [n_split][kAttnSplitWords]: pieces of the split form, longest first
  int64_t join_items;   // [n_join][kAttnSplitWords]: its tiles
  int64_t dq_items;     // [n_dq][kAttnTileWords]: fine-tuning samples, steps of 64 keys
  int64_t dq_join;      // [n_dq_join][4]
  int64_t dk_items;     // [n_dk][kAttnTileWords]: fine-tuning samples, steps of 64 queries of one head
  int64_t dk_join;      // [n_dk_join][4]
  int64_t f32_dq_items; // the same in fp32 tiles
  int64_t f32_dk_items;
  int64_t total_words;
};

}  // namespace dsv

struct dsv_attn_plan {
  int32_t n_seqs = 0, n_q = 0, n_kv = 0, hq = 0, hkv = 0, d = 0;
  bool windowed = false;  // some key that causality leaves is hidden by the window
  int32_t window = 0, sinks = 0;
  int64_t train_q = 0, train_k = 0;
  int32_t n_fwd = 0, n_fwd_join = 0, fwd_slots = 0, n_dk_join = 0, dk_slots = 0;  // *_slots: pieces with sums of their own
  int32_t n_dq_join = 0, dq_slots = 0;
  int32_t n_f32 = 0, n_split = 0, n_join = 0, n_dq = 0, n_dk = 0, n_f32_dq = 0, n_f32_dk = 0;
  int32_t f32_dk_long = 0;    // of the fp32 key tiles the first ones, with more than twice the usual one's queries
  std::vector<int32_t> meta;  // packed blob, host image
  dsv::AttnLayout lay{};
  void* d_meta = nullptr;     // device copy (nullptr: host-only plan)
  void* copy_done = nullptr;  // hipEvent_t recorded after the upload
  const int32_t* dptr(int64_t off) const { return static_cast<const int32_t*>(d_meta) + off; }
};
