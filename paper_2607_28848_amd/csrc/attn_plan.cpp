// attn_plan.cpp -- validation and packing of a mixed batch's attention (host only, plus
// one asynchronous host-to-device copy of the packed blob).
//
// The sequences of a batch (Sec. 3.2: inference entries and fine-tuning samples) are the
// same for every layer, so the tiles, their order and the pieces of long caches are laid
// down here, once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <array>
#include <functional>
#include <map>
#include <new>
#include <numeric>

#include "attn_plan.h"

namespace {

using namespace dsv;

// Tiles of `rows` rows, as {sequence, first row}, those with the most work first (ties: table
// order), so that the last workgroups to start are short ones.
struct Tiles {
  std::vector<std::pair<int64_t, std::pair<int32_t, int32_t>>> t;
  void add(int64_t work, int32_t seq, int64_t first) { t.push_back({-work, {seq, (int32_t)first}}); }
  std::vector<int32_t> words() {
    std::stable_sort(t.begin(), t.end(), [](const auto& a, const auto& b) { return a.first < b.first; });
    std::vector<int32_t> w;
    w.reserve(2 * t.size());
    for (const auto& e : t) w.insert(w.end(), {e.second.first, e.second.second});
    return w;
  }
};

// Tiles in steps of equal cost, `copies` (heads) of each, on `slots` workgroups at a time: every tile whole, or cut
// into pieces of at most `piece` steps, no shorter than `least`, if there are fewer tiles than most_tiles.
struct Cut {
  std::vector<int32_t> items, join;
  int32_t n_items = 0, n_join = 0, n_slots = 0;
};

// The time, in steps, that the tiles take in pieces of at most `piece` steps, longest first, each on the slot
// that is free first.  join: steps that a piece's own sums cost.  Pieces of one length and slots that are free at one time
// are taken together: the tiles behind a window are nearly all alike, and up to 16 schedules are tried (eight samples of 16384,
// window 64, sinks: 5.9 ms a plan piece by piece, 0.94 so, 0.86 without a window).
template <typename F>
int64_t makespan(const std::vector<int64_t>& steps, int64_t copies, F pieces_of, int slots, int64_t join) {
  std::map<int64_t, int64_t, std::greater<int64_t>> pieces;  // length: number
  for (int64_t s : steps) {
    const int64_t n = pieces_of(s);
    pieces[(s + n - 1) / n + (n > 1 ? join : 0)] += n * copies;
  }
  std::map<int64_t, int64_t> free_at{{0, slots}};  // time: slots
  int64_t end = 0;
  for (const auto& [length, number] : pieces) {
    for (int64_t left = number; left > 0;) {
      const auto first = free_at.begin();
      const int64_t n = std::min(left, first->second), t = first->first + length;
      left -= n;
      free_at[t] += n;
      end = std::max(end, t);
      if ((first->second -= n) == 0) free_at.erase(first);
    }
  }
  return end;
}

struct Tile {
  int64_t steps;
  int32_t seq, first;
  int32_t x = 0, y = 0;  // the descriptor's last words
};

// windowed: the sinks' tiles, several times as long as the others, may have pieces of a length of their own (two samples of
// 8192 behind a window of 1024, 32 heads on 8, forward and backward: 1606 us, 1635 with one length for all tiles).
Cut cut(std::vector<Tile> t, int64_t copies, int slots, int64_t least, int64_t join, int64_t most_tiles, bool windowed = false) {
  std::stable_sort(t.begin(), t.end(), [](const Tile& a, const Tile& b) { return a.steps > b.steps; });
  std::vector<int64_t> steps;
  int64_t all = 0, most = 0;
  for (const Tile& e : t) {
    steps.push_back(e.steps);
    all += e.steps;
    most = std::max(most, e.steps);
  }
  int64_t piece = std::max<int64_t>(most, 1);
  const int64_t share = all * copies / slots;
  int64_t far = most, far_piece = 0;  // tiles of more than `far` steps are cut into pieces of far_piece
  auto by = [&](int64_t p) { return [p](int64_t s) { return std::max<int64_t>(1, (s + p - 1) / p); }; };
  auto pieces_of = [&](int64_t s) { return by(s > far ? far_piece : piece)(s); };
  // With several rounds of tiles the short ones fill what the long ones leave.
  if ((int64_t)t.size() * copies < most_tiles && most > share + share / 4 && most > least) {
    int64_t best = makespan(steps, copies, by(piece), slots, 0);
    for (int64_t d = 2; d <= 8; ++d) {  // shares of eighths
      const int64_t p = std::max<int64_t>(least, share * d / 4);
      const int64_t m = makespan(steps, copies, by(p), slots, join);
      if (m < best) best = m, piece = p;
    }
    const int64_t usual = steps.empty() ? 0 : steps[steps.size() / 2];
    if (windowed && most > 2 * usual) {
      for (int64_t d = 1; d <= 8; ++d) {  // eighths of a usual tile
        const int64_t p = std::max<int64_t>(least, usual * d / 8);
        const int64_t m = makespan(
            steps, copies, [&](int64_t s) { return s > 2 * usual ? by(p)(s) : (int64_t)1; }, slots, join);
        if (m < best) best = m, piece = most, far = 2 * usual, far_piece = p;
      }
    }
  }
  Cut c;
  struct Piece {
    int64_t steps;
    int32_t w[kAttnTileWords];
  };
  std::vector<Piece> all_pieces;
  for (const Tile& e : t) {
    const int64_t s = e.steps, n = pieces_of(s), len = (s + n - 1) / n;
    if (n > 1) {
      c.join.insert(c.join.end(), {e.seq, e.first, c.n_slots, (int32_t)n});
      ++c.n_join;
    }
    for (int64_t k = 0; k < n; ++k) {
      const int64_t b = std::min(k * len, s), l = std::min((k + 1) * len, s);
      all_pieces.push_back({l - b, {e.seq, e.first, (int32_t)b, (int32_t)l, n > 1 ? c.n_slots++ : 0, (int32_t)n, e.x, e.y}});
    }
  }
  std::stable_sort(all_pieces.begin(), all_pieces.end(), [](const Piece& a, const Piece& b) { return a.steps > b.steps; });
  for (const Piece& p : all_pieces) c.items.insert(c.items.end(), p.w, p.w + kAttnTileWords);
  c.n_items = (int32_t)all_pieces.size();
  return c;
}

// Keys that queries [.., last] of a sequence see.
int64_t keys_seen(const dsv_attn_seq& s, int64_t last) {
  return std::max<int64_t>(0, std::min<int64_t>(s.k_len, last + 1 + s.k_len - s.q_len));
}

// The keys that queries [q0, q1) of a sequence see, in steps of `step` keys.  Where the window leaves a gap behind the
// sinks: `sink` keys' worth of steps for the sinks alone, and behind them the keys from the window's first one on, which
// lie `shift` keys from where they would without the gap (`shift` may be negative: a step of sinks may be short).  So no
// key is read that none of the queries sees.  Else sink and shift are 0.
struct Span {
  int64_t steps, sink, shift;
};
Span span_of(const dsv_attn_plan& p, const dsv_attn_seq& s, int64_t q0, int64_t q1, int64_t step) {
  const int64_t end = keys_seen(s, q1 - 1), all = (end + step - 1) / step;
  const int64_t first = q0 + s.k_len - s.q_len + 1 - p.window;
  if (!p.windowed || end == 0 || first <= p.sinks) return {all, 0, 0};
  const int64_t sink = (p.sinks + step - 1) / step;
  return {sink + (end - first + step - 1) / step, sink * step, first - sink * step};
}

// One past the last query that sees one of the keys [k0, k1): the sinks are seen to the end.
int64_t queries_end(const dsv_attn_plan& p, const dsv_attn_seq& s, int64_t k0, int64_t k1) {
  if (!p.windowed || k0 < p.sinks) return s.q_len;
  return std::min<int64_t>(s.q_len, std::min<int64_t>(k1, s.k_len) - 1 - ((int64_t)s.k_len - s.q_len) + p.window);
}

int build(const dsv_attn_seq* seqs, int32_t n, int32_t n_q, int32_t n_kv, int32_t hq, int32_t hkv, int32_t d,
          int32_t window, int32_t sinks, dsv_attn_plan& p) {
  if (n < 0 || n_q < 0 || n_kv < 0 || (n > 0 && !seqs)) return DSV_ERR_ARG;
  if (hkv < 1 || hq < hkv || hq > 1024 || hq % hkv != 0 || (d != 64 && d != 128)) return DSV_ERR_RANGE;
  if (window < 1 || sinks < 0) return DSV_ERR_RANGE;
  std::vector<int32_t> order(n);
  std::iota(order.begin(), order.end(), 0);
  for (int32_t i = 0; i < n; ++i) {
    const dsv_attn_seq& s = seqs[i];
    if (s.is_train != 0 && s.is_train != 1) return DSV_ERR_RANGE;
    if (s.q_start < 0 || s.q_len < 0 || s.k_start < 0 || s.k_len < 0) return DSV_ERR_LAYOUT;
    if ((int64_t)s.q_start + s.q_len > n_q || (int64_t)s.k_start + s.k_len > n_kv) return DSV_ERR_LAYOUT;
  }
  std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return seqs[a].q_start < seqs[b].q_start; });
  int64_t end = 0;
  for (int32_t i : order) {
    if (seqs[i].q_len == 0) continue;
    if (seqs[i].q_start < end) return DSV_ERR_LAYOUT;  // overlapping query ranges
    end = (int64_t)seqs[i].q_start + seqs[i].q_len;
  }

  // workgroups of a launch, before the work lists are laid down
  int64_t tiles_q = 0, tiles_k = 0;
  for (int32_t i = 0; i < n; ++i) {
    tiles_q += ((int64_t)seqs[i].q_len + kAttnF32Rows - 1) / kAttnF32Rows;
    tiles_k += ((int64_t)seqs[i].k_len + kAttnF32Rows - 1) / kAttnF32Rows;
  }
  if (8 * tiles_q * hq > INT32_MAX || 8 * tiles_k * hkv > INT32_MAX) return DSV_ERR_SIZE;

  // A window that hides nothing is none.
  for (int32_t i = 0; i < n; ++i)
    if (seqs[i].q_len > 0 && seqs[i].k_len > window && sinks < seqs[i].k_len - window) p.windowed = true;
  // counts of keys through the sinks' blocks and the window's
  for (int32_t i = 0; p.windowed && i < n; ++i)
    if (seqs[i].k_len > INT32_MAX - 1024) return DSV_ERR_SIZE;
  p.window = window;
  p.sinks = sinks;
  p.n_seqs = n;
  p.n_q = n_q;
  p.n_kv = n_kv;
  p.hq = hq;
  p.hkv = hkv;
  p.d = d;
  const int32_t group = hq / hkv;
  std::vector<int32_t> desc((size_t)n * kAttnSeqWords, 0);
  for (int32_t i : order) {
    const dsv_attn_seq& s = seqs[i];
    int32_t* w = &desc[(size_t)i * kAttnSeqWords];
    w[0] = s.q_start;
    w[1] = s.q_len;
    w[2] = s.k_start;
    w[3] = s.k_len;
    w[4] = w[5] = -1;
    if (s.is_train) {
      if (p.train_q + s.q_len > INT32_MAX || p.train_k + s.k_len > INT32_MAX) return DSV_ERR_SIZE;
      w[4] = (int32_t)p.train_q;
      w[5] = (int32_t)p.train_k;
      p.train_q += s.q_len;
      p.train_k += s.k_len;
    }
  }

  Tiles f32, f32_dq, f32_dk;
  std::vector<Tile> fwd, dq, dk;
  // query tiles: the words that their kernels find the keys by
  auto query_tile = [&](std::vector<Tile>& to, int32_t i, int64_t q, int64_t rows) {
    const Span sp = span_of(p, seqs[i], q, std::min<int64_t>(q + rows, seqs[i].q_len), 64);
    to.push_back({sp.steps, i, (int32_t)q, (int32_t)sp.sink, (int32_t)sp.shift});
  };
  auto f32_tile = [&](Tiles& to, int32_t i, int64_t q) {
    const dsv_attn_seq& s = seqs[i];
    const int64_t q1 = std::min<int64_t>(q + kAttnF32Rows, s.q_len);
    to.add(p.windowed ? 16 * span_of(p, s, q, q1, 16).steps : keys_seen(s, q1 - 1), i, q);
  };
  // keys that a sequence of the split form walks: those of all its queries, the sinks' blocks whole
  auto split_shift = [&](const dsv_attn_seq& s) { return span_of(p, s, 0, s.q_len, 32).shift; };
  auto split_keys = [&](const dsv_attn_seq& s) { return s.k_len - split_shift(s); };
  int64_t split_keys_all = 0, split_most = 0;  // keys that the split form's tiles read; the longest sequence's
  std::vector<int32_t> split;
  for (int32_t i = 0; i < n; ++i) {
    const dsv_attn_seq& s = seqs[i];
    for (int64_t q = 0; q < s.q_len; q += kAttnF32Rows) f32_tile(f32, i, q);
    if (s.q_len <= kAttnSplitQ) {
      if (s.q_len == 0) continue;
      split.push_back(i);
      const int64_t tiles = ((int64_t)s.q_len * group + kAttnPackRows - 1) / kAttnPackRows;
      split_keys_all += tiles * split_keys(s);
      split_most = std::max<int64_t>(split_most, split_keys(s));
    } else {
      for (int64_t q = 0; q < s.q_len; q += kAttnFwdRows) query_tile(fwd, i, q, kAttnFwdRows);
    }
  }
  for (int32_t i = 0; i < n; ++i) {
    const dsv_attn_seq& s = seqs[i];
    if (!s.is_train) continue;
    for (int64_t q = 0; q < s.q_len; q += kAttnBwdRows) query_tile(dq, i, q, kAttnBwdRows);
    for (int64_t q = 0; q < s.q_len; q += kAttnF32Rows) f32_tile(f32_dq, i, q);
    // queries that see keys from k on: from max(0, k - (k_len - q_len)) on, up to `end`
    auto seen_by = [&](int64_t k, int64_t end) { return end - std::max<int64_t>(0, k - ((int64_t)s.k_len - s.q_len)); };
    for (int64_t k = 0; k < s.k_len; k += kAttnBwdRows) {
      const int64_t end = std::max<int64_t>(0, queries_end(p, s, k, k + kAttnBwdRows));
      dk.push_back({std::max<int64_t>(0, (seen_by(k, end) + 63) / 64) * group, i, (int32_t)k, (int32_t)end, 0});
    }
    for (int64_t k = 0; k < s.k_len; k += kAttnF32Rows) f32_dk.add(seen_by(k, queries_end(p, s, k, k + kAttnF32Rows)), i, k);
  }

  // Pieces: one length for the whole call
  const int64_t target = d == 128 ? kAttnSplitTarget : 2 * kAttnSplitTarget;
  int64_t piece = (split_keys_all * hkv + target - 1) / target;
  piece = std::max<int64_t>(kAttnPieceKeys, (piece + kAttnPieceKeys - 1) / kAttnPieceKeys * kAttnPieceKeys);
  if (split_most <= kAttnWholeKeys) piece = kAttnWholeKeys;
  std::vector<std::array<int32_t, kAttnSplitWords>> pieces;
  std::vector<int32_t> split_items, join_items;
  for (int32_t i : split) {
    const dsv_attn_seq& s = seqs[i];
    const int64_t rows = (int64_t)s.q_len * group;
    // pieces of equal length (to a multiple of 32 keys)
    const Span sp = span_of(p, s, 0, s.q_len, 32);
    const int32_t sink = (int32_t)sp.sink, shift = (int32_t)sp.shift;
    const int64_t keys = split_keys(s);
    const int64_t np = std::max<int64_t>(1, (keys + piece - 1) / piece);
    const int64_t len = std::max<int64_t>(32, ((keys + np - 1) / np + 31) / 32 * 32);
    for (int64_t r = 0; r < rows; r += kAttnPackRows) {
      const int64_t first = (int64_t)pieces.size();
      if (first + np > INT32_MAX / kAttnSplitWords) return DSV_ERR_SIZE;
      join_items.insert(join_items.end(), {s.q_start, s.q_len, s.k_start, s.k_len, (int32_t)r, (int32_t)np, (int32_t)first, 0,
                                           s.k_len, 0, 0, 0});
      for (int64_t k = 0; k < np; ++k)
        pieces.push_back({s.q_start, s.q_len, s.k_start, s.k_len, (int32_t)r, (int32_t)np, (int32_t)(first + k),
                          (int32_t)std::min<int64_t>(k * len, keys), (int32_t)std::min<int64_t>((k + 1) * len, keys), sink,
                          shift, 0});
    }
  }
  std::stable_sort(pieces.begin(), pieces.end(), [](const auto& a, const auto& b) { return a[8] - a[7] > b[8] - b[7]; });
  for (const auto& w : pieces) split_items.insert(split_items.end(), w.begin(), w.end());

  std::vector<int32_t>& m = p.meta;
  auto put = [&](const std::vector<int32_t>& w) {
    const int64_t off = (int64_t)m.size();
    m.insert(m.end(), w.begin(), w.end());
    m.resize((m.size() + 3) & ~size_t(3), 0);
    return off;
  };
  AttnLayout& L = p.lay;
  auto count = [](const std::vector<int32_t>& w, int words, int32_t* out) {
    const int64_t c = (int64_t)w.size() / words;
    *out = (int32_t)c;
    return c;
  };
  const Cut cf = cut(std::move(fwd), hq, kAttnFwdSlots, kAttnFwdPieceSteps, 2, 4 * kAttnFwdSlots);
  // The sinks' key tile has every query of its sequence, however many tiles of a window there are beside it.
  const Cut ck = cut(std::move(dk), hkv, kAttnDkSlots, kAttnGradPieceSteps, 3, p.windowed ? INT64_MAX : 4 * kAttnDkSlots,
                     p.windowed);
  // Query tiles that fill the CUs run two to a CU, and the long ones faster when the short ones end: only fewer are cut.
  const Cut cq = cut(std::move(dq), hq, kAttnDkSlots, kAttnGradPieceSteps, 3, kAttnDkSlots);
  p.n_fwd = cf.n_items, p.n_fwd_join = cf.n_join, p.fwd_slots = cf.n_slots;
  p.n_dq = cq.n_items, p.n_dq_join = cq.n_join, p.dq_slots = cq.n_slots;
  p.n_dk = ck.n_items, p.n_dk_join = ck.n_join, p.dk_slots = ck.n_slots;
  const std::vector<int32_t> w3 = f32.words(), w3q = f32_dq.words(),
                             w3k = f32_dk.words();
  const auto& kt = f32_dk.t;  // sorted by now, and work is -first
  const size_t some = std::partition_point(kt.begin(), kt.end(), [](const auto& e) { return e.first < 0; }) - kt.begin();
  for (size_t i = 0; i < some; ++i) p.f32_dk_long += kt[i].first < 2 * kt[some / 2].first;
  int64_t most = std::max({p.n_fwd, p.n_dk, p.n_dq});
  most = std::max(most, count(w3, 2, &p.n_f32));
  most = std::max(most, count(split_items, kAttnSplitWords, &p.n_split));
  most = std::max(most, count(join_items, kAttnSplitWords, &p.n_join));
  most = std::max(most, count(w3q, 2, &p.n_f32_dq));
  most = std::max(most, count(w3k, 2, &p.n_f32_dk));
  if (8 * most * hq > INT32_MAX) return DSV_ERR_SIZE;  // workgroups of a launch
  L.seqs = put(desc);
  L.fwd_items = put(cf.items);
  L.fwd_join = put(cf.join);
  L.f32_items = put(w3);
  L.split_items = put(split_items);
  L.join_items = put(join_items);
  L.dq_items = put(cq.items);
  L.dq_join = put(cq.join);
  L.dk_items = put(ck.items);
  L.dk_join = put(ck.join);
  L.f32_dq_items = put(w3q);
  L.f32_dk_items = put(w3k);
  m.resize(std::max<size_t>(64, (m.size() + 63) & ~size_t(63)), 0);
  L.total_words = (int64_t)m.size();
  return DSV_OK;
}

}  // namespace

extern "C" int dsv_attn_build(const dsv_attn_seq* seqs, int32_t n_seqs, int32_t n_q, int32_t n_kv, int32_t heads_q,
                              int32_t heads_kv, int32_t head_dim, size_t* meta_bytes, dsv_attn_plan** out_plan) {
  return dsv_attn_build_window(seqs, n_seqs, n_q, n_kv, heads_q, heads_kv, head_dim, INT32_MAX, 0, meta_bytes, out_plan);
}

extern "C" int dsv_attn_build_window(const dsv_attn_seq* seqs, int32_t n_seqs, int32_t n_q, int32_t n_kv, int32_t heads_q,
                                     int32_t heads_kv, int32_t head_dim, int32_t window, int32_t sinks,
                                     size_t* meta_bytes, dsv_attn_plan** out_plan) {
  if (out_plan) *out_plan = nullptr;
  if (!meta_bytes || !out_plan) return DSV_ERR_ARG;
  dsv_attn_plan* p = nullptr;
  int rc = DSV_OK;
  try {
    p = new dsv_attn_plan();
    rc = build(seqs, n_seqs, n_q, n_kv, heads_q, heads_kv, head_dim, window, sinks, *p);
  } catch (const std::bad_alloc&) {
    rc = DSV_ERR_SIZE;
  } catch (...) {
    rc = DSV_ERR_ARG;
  }
  if (rc != DSV_OK) {
    delete p;
    return rc;
  }
  *meta_bytes = (size_t)p->lay.total_words * sizeof(int32_t);
  *out_plan = p;
  return DSV_OK;
}

extern "C" int dsv_attn_upload(dsv_attn_plan* p, void* d_meta, size_t meta_bytes, void* hip_stream) {
  if (!p || !d_meta || p->d_meta || reinterpret_cast<uintptr_t>(d_meta) % 256 != 0) return DSV_ERR_ARG;
  const size_t need = (size_t)p->lay.total_words * sizeof(int32_t);
  if (meta_bytes < need) return DSV_ERR_SIZE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipEvent_t ev = nullptr;
  hipError_t e = hipEventCreateWithFlags(&ev, hipEventDisableTiming);
  if (e == hipSuccess) e = hipMemcpyAsync(d_meta, p->meta.data(), need, hipMemcpyHostToDevice, st);
  if (e == hipSuccess) e = hipEventRecord(ev, st);
  if (e != hipSuccess) {
    if (ev) (void)hipEventDestroy(ev);
    return DSV_ERR_DEVICE;
  }
  p->copy_done = ev;
  p->d_meta = d_meta;
  return DSV_OK;
}

extern "C" int dsv_attn_train_rows(const dsv_attn_plan* p, int64_t out[2]) {
  if (!p || !out) return DSV_ERR_ARG;
  out[0] = p->train_q;
  out[1] = p->train_k;
  return DSV_OK;
}

extern "C" void dsv_attn_free(dsv_attn_plan* p) {
  if (!p) return;
  if (p->copy_done) {
    // the host image is the source of the asynchronous upload: wait for it
    hipEvent_t ev = static_cast<hipEvent_t>(p->copy_done);
    (void)hipEventSynchronize(ev);
    (void)hipEventDestroy(ev);
  }
  delete p;
}
