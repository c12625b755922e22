// gemm_tile.h -- the contraction loops of a 256-column bf16 tile (v_mfma_f32_16x16x32_bf16) as functions
// that leave the fp32 sums in registers for the caller's epilogue.
//
//   tile_nt: out[m][n] = sum_c P[m][c] Q[n][c]      tile_nn: out[m][n] = sum_c P[m][c] Q[c][n]
// 4 waves in a 2 x 2 grid, each FM x 8 blocks of 16 x 16 (FM 8: 256 rows, FM 4: 128).  Operand tiles go
// from global memory straight into LDS.  Rows and columns past the operands, and contraction values past C,
// read zeros.
// tile_ring is tile_nt's form for products of few tiles, in both types.
// Sums: acc[i][j][v] is row wm * 16 FM + 16 i + l % 16, column wn * 128 + 16 j + 4 (l / 16) + v.
#pragma once

#include "device_common.h"

namespace dsv {
namespace {

extern "C" __device__ void llvm_amdgcn_raw_buffer_load_lds_t(i32x4 rsrc, lds_u32* lds, int size, int voffset,
                                                             int soffset, int offset,
                                                             int aux) __asm("llvm.amdgcn.raw.buffer.load.lds");

template <bool B>
struct flag_c {  // a compile-time flag passed as a value
  static constexpr bool value = B;
};

template <int V>
struct num_c {
  static constexpr int value = V;
};

// f(num_c<U>) for U of [U, END)
template <int U, int END, typename F>
__device__ __forceinline__ void ring_tail(F&& f) {
  if constexpr (U < END) {
    f(num_c<U>{});
    ring_tail<U + 1, END>(f);
  }
}

constexpr int kTileStage = 2 * 256 * 64 * 2;    // bytes of one of tile_nt's two buffers (FM 8)
constexpr int kTileStageNN = 2 * 256 * 32 * 2;  // bytes of one of tile_nn's four buffers (FM 8)

// Descriptor over `bytes` bytes (at most 2^31) from base.
__device__ __forceinline__ i32x4 tile_rsrc(const void* base, int64_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  i32x4 r;
  r.x = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
  r.y = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
  r.z = __builtin_amdgcn_readfirstlane((int)(bytes > 0 ? bytes : 0));
  r.w = 0x00020000;
  return r;
}

// Consecutive workgroup ids go round the 8 XCDs: each gets a contiguous range of tiles.
__device__ __forceinline__ int tile_of(int bid, int n) {
  const int per = n >> 3, rem = n & 7, xcd = bid & 7;
  return xcd * per + min(xcd, rem) + (bid >> 3);
}

// Tile -> (row tile, column tile): groups of 4 row tiles, column by column.
__device__ __forceinline__ void tile_at(int lin, int n_m, int n_n, int& mt, int& nt) {
  const int span = 4 * n_n, grp = lin / span, first = grp * 4, size = min(n_m - first, 4);
  mt = first + (lin % span) % size;
  nt = (lin % span) / size;
}

// P: the tile's first row; p_rows, q_cols: rows and columns that exist; C: contraction length.  Steps of 64 through two
// buffers, a barrier each.
// turn: the step of 64 to begin with.  Tiles that run together and whose rows lie a power of two apart read from the
// same memory channels when they walk the contraction in step.
// Returns the buffer that the last step did not use.
template <int FM>
__device__ __forceinline__ char* tile_nt(const uint16_t* P, int64_t ldp, int p_rows, const uint16_t* Q, int64_t ldq_,
                                              int q_cols, int C, int turn, char* smem0, char* smem1, f32x4 (&acc)[FM][8]) {
  constexpr int WM = 16 * FM, TM = 2 * WM, TN = 256, TK = 64, FN = 8, ROWB = TK * 2;
  constexpr int A_BYTES = TM * ROWB, LOADS = 8, LOADS_A = FM;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, l15 = lane & 15, lr = lane >> 3;
  const int ld = (int)ldp, ldq = (int)ldq_, nk = (C + TK - 1) / TK;
  auto buf = [&](int stage) { return stage ? smem1 : smem0; };
  auto rswz = [](int row) { return (row ^ (row >> 3)) & 7; };
  // from the tile's first value to its last row's last one (P: rows are read eight values at a time)
  const i32x4 ra = tile_rsrc(P, ((int64_t)(min(TM, p_rows) - 1) * ld + ((C + 7) & ~7)) * 2);
  const i32x4 rb = tile_rsrc(Q, ((int64_t)(min(TN, q_cols) - 1) * ldq + C) * 2);
  int voff_a[LOADS_A], voff_b[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS_A; ++i) voff_a[i] = ((((lane & 7) ^ lr ^ ((LOADS_A * wave + i) & 7)) << 4)) + lr * ld * 2;
#pragma unroll
  for (int i = 0; i < LOADS; ++i) voff_b[i] = (((lane & 7) ^ lr ^ i) << 4) + lr * ldq * 2;
  // Steps in the order turn, turn + 1, .., nk - 1, 0, .. (where all are whole).
  const int first = C % TK == 0 ? turn % nk : 0;
  auto at = [&](int kt) { return kt + first < nk ? kt + first : kt + first - nk; };
  auto load_a = [&](int kt, char* st, int i) {
    const int q = wave * LOADS_A + i;
    llvm_amdgcn_raw_buffer_load_lds_t(ra, (lds_u32*)(st + q * 1024), 16, voff_a[i],
                                      __builtin_amdgcn_readfirstlane(q * 16 * ld + at(kt) * TK * 2), 0, 0);
  };
  auto load_b = [&](int kt, char* st, int i) {
    const int q = wave * LOADS + i;
    llvm_amdgcn_raw_buffer_load_lds_t(rb, (lds_u32*)(st + A_BYTES + q * 1024), 16, voff_b[i],
                                      __builtin_amdgcn_readfirstlane(q * 16 * ldq + at(kt) * TK * 2), 0, 0);
  };
  // any step: chunks past the contraction read zeros (C is a multiple of 8, or the rows hold zeros from C on)
  auto issue = [&](int kt, int stage) {
    const int k0 = kt * TK;
    char* st = buf(stage);
    if (k0 + TK <= C) {
#pragma unroll
      for (int i = 0; i < LOADS_A; ++i) load_a(kt, st, i);
#pragma unroll
      for (int i = 0; i < LOADS; ++i) load_b(kt, st, i);
      return;
    }
#pragma unroll
    for (int i = 0; i < LOADS_A; ++i) {
      const int q = wave * LOADS_A + i, row = 8 * q + lr, c = (lane & 7) ^ rswz(row);
      const int vo = k0 + 8 * c < C ? (row * ld + k0 + 8 * c) * 2 : (int)0x7FFFFFF0;
      llvm_amdgcn_raw_buffer_load_lds_t(ra, (lds_u32*)(st + q * 1024), 16, vo, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int q = wave * LOADS + i, row = 8 * q + lr, c = (lane & 7) ^ rswz(row);
      const int vo = k0 + 8 * c < C ? (row * ldq + k0 + 8 * c) * 2 : (int)0x7FFFFFF0;
      llvm_amdgcn_raw_buffer_load_lds_t(rb, (lds_u32*)(st + A_BYTES + q * 1024), 16, vo, 0, 0, 0);
    }
  };
  issue(0, 0);
  if (nk > 1) issue(1, 1);
  // Zeros placed in the matrix core's registers: left to itself the compiler rotates the sums through others
  // (252 moves beside 128 matrix instructions; 4096 rows of 8192 against 32256: 1.94 ms, 1.60 so).
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      asm volatile("" : "+a"(acc[i][j]));
    }

  // Fragment addresses: a lane part picked by the step and block (the chunk swizzle), plus an immediate.
  const int lanepart = (lane >> 4) ^ (l15 & 7) ^ (l15 >> 3);
  int off_a[4], off_b[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    off_a[c] = (wm * WM + l15) * ROWB + 16 * (lanepart ^ (2 * c));
    off_b[c] = A_BYTES + (wn * 128 + l15) * ROWB + 16 * (lanepart ^ (2 * c));
  }
  auto rd_a = [&](const char* st, int s, int i) {
    return as_bf(*reinterpret_cast<const u32x4*>(st + off_a[((2 * s) ^ i) & 3] + 16 * i * ROWB));
  };
  auto rd_b = [&](const char* st, int s, int j) {
    return as_bf(*reinterpret_cast<const u32x4*>(st + off_b[((2 * s) ^ j) & 3] + 16 * j * ROWB));
  };
  bf16x8 fa0[FM], fa1[FM], fb[FN];
  if (nk >= 2) __builtin_amdgcn_s_waitcnt(vmcnt_imm(LOADS_A + LOADS));  // the first step has landed
  else vmem_wait_all();
  __syncthreads();
#pragma unroll
  for (int j = 0; j < FN; ++j) fb[j] = rd_b(smem0, 0, j);
#pragma unroll
  for (int i = 0; i < FM; ++i) fa0[i] = rd_a(smem0, 0, i);
  // 32 contraction values with fragments (cur, fb), a column block at a time; per block two of the loads of
  // step kl into buffer ls, and the reads that replace the fragments it is done with.
  auto half = [&](bf16x8 (&cur)[FM], bf16x8 (&nxt)[FM], const char* st_next, int s_next, bool load, int kl, int ls) {
#pragma unroll
    for (int j = 0; j < FN; ++j) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], cur[i], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int e = 2 * j; e < 2 * j + 2; ++e)
        if (load && e < LOADS_A + LOADS) {
          if (e < LOADS_A) load_a(kl, buf(ls), e < LOADS_A ? e : 0);
          else load_b(kl, buf(ls), e - LOADS_A);
        }
      if (j < FM / 2) {
        nxt[2 * j] = rd_a(st_next, s_next, 2 * j);
        nxt[2 * j + 1] = rd_a(st_next, s_next, 2 * j + 1);
      }
      fb[j] = rd_b(st_next, s_next, j);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Step kt in buffer `stage`, another one to follow: the barrier between its halves publishes kt + 1 and
  // frees the buffer, which kt + 2 is loaded into.
  auto kstep = [&](int kt, int stage, bool load) {
    half(fa0, fa1, buf(stage), 1, false, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    vmem_wait_all();
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
    if (!load && kt + 2 < nk) issue(kt + 2, stage);  // a partial last step
    half(fa1, fa0, buf(stage ^ 1), 0, load, kt + 2, stage);
  };
  int kt = 0, stage = 0;
  const int main_end = C / TK - 2;  // kt < main_end: step kt + 2 is whole
  for (; kt < main_end; ++kt, stage ^= 1) kstep(kt, stage, true);
  for (; kt + 1 < nk; ++kt, stage ^= 1) kstep(kt, stage, false);
  half(fa0, fa1, buf(stage), 1, false, 0, 0);
#pragma unroll
  for (int j = 0; j < FN; ++j)
#pragma unroll
    for (int i = 0; i < FM; ++i)
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa1[i], acc[i][j], 0, 0, 0);
  return buf(stage ^ 1);
}

// Steps of 32 through four buffers, so that a step's loads have three steps' time to arrive: Q's rows come through
// transposing reads, twice as many as tile_nt's, and two buffers with steps of 64 leave no room between them for the
// loads (4096 rows, 32256 x 8192: 1.75 ms so, 1.61 in four.  tile_nt gains nothing: 1.64 ms and 1.72).
// P's rows hold zeros from C to a multiple of 32.
template <int FM>
__device__ __forceinline__ void tile_nn(const uint16_t* P, int64_t ldp, int p_rows, const uint16_t* Q, int64_t ldq_,
                                        int q_cols, int C, char* b0, char* b1, char* b2, char* b3, f32x4 (&acc)[FM][8]) {
  constexpr int WM = 16 * FM, TM = 2 * WM, TN = 256, TK = 32, FN = 8, ROWB = 2 * TK;
  constexpr int A_BYTES = TM * ROWB, LOADS = 4, LOADS_A = FM / 2, N = LOADS + LOADS_A;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, l15 = lane & 15, g4 = lane >> 4;
  const int ld = (int)ldp, ldq = (int)ldq_, nk = (C + TK - 1) / TK;
  const i32x4 ra = tile_rsrc(P, ((int64_t)(min(TM, p_rows) - 1) * ld + nk * TK) * 2);
  const i32x4 rb = tile_rsrc(Q, ((int64_t)(C - 1) * ldq + q_cols) * 2);
  // P's rows of 64 bytes: chunk c of row r in slot c ^ r / 4 % 4 (16 consecutive rows put a chunk in
  // 16 different bank groups).  A load fills 16 rows.
  const int voff_a = (lane >> 2) * ld * 2 + 16 * ((lane & 3) ^ g4);
  int voff_b[2];
#pragma unroll
  for (int par = 0; par < 2; ++par)
    voff_b[par] = ((lane >> 5) * ldq + 8 * ((lane & 31) ^ 2 * ((2 * par + (lane >> 5)) & 3))) * 2;
  // Load e of step kt (P's first).  Past the last step the last is loaded again, for a buffer that is not read: so each
  // step's loads are followed by the same number of others.
  auto load = [&](int kt, char* st, int e) {
    const int k = min(kt, nk - 1) * TK;
    if (e < LOADS_A) {
      const int q = wave * LOADS_A + e;
      llvm_amdgcn_raw_buffer_load_lds_t(ra, (lds_u32*)(st + q * 1024), 16, voff_a,
                                        __builtin_amdgcn_readfirstlane((q * 16 * ld + k) * 2), 0, 0);
    } else {
      const int q = wave * LOADS + e - LOADS_A;
      llvm_amdgcn_raw_buffer_load_lds_t(rb, (lds_u32*)(st + A_BYTES + q * 1024), 16, voff_b[(e - LOADS_A) & 1],
                                        __builtin_amdgcn_readfirstlane((k + 2 * q) * ldq * 2), 0, 0);
    }
  };
#pragma unroll
  for (int e = 0; e < N; ++e) load(0, b0, e);
#pragma unroll
  for (int e = 0; e < N; ++e) load(1, b1, e);
#pragma unroll
  for (int e = 0; e < N; ++e) load(2, b2, e);
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      asm volatile("" : "+a"(acc[i][j]));
    }
  const int off_a = (wm * WM + l15) * ROWB + 16 * (g4 ^ (l15 >> 2));
  int off_b[4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
    off_b[c] = A_BYTES + (8 * g4 + (l15 >> 2)) * (TN * 2) + 256 * wn + 32 * (c ^ (l15 >> 2)) + 16 * ((l15 & 3) >> 1) +
               8 * (l15 & 1);
  // Step kt in `st`, with the loads of step kt + 3 into `nxt`, which the step before this one has read; behind the
  // step's own loads are those of AFTER more.
  auto step = [&](auto with, auto after, int kt, const char* st, char* nxt) {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(decltype(after)::value * N));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();  // not __syncthreads(), which would wait for every load
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    auto rd_b = [&](int j) {
      typedef uint32_t u32x2t __attribute__((ext_vector_type(2)));
      const char* p = st + off_b[j & 3] + 128 * (j >> 2);
      const u32x2t a0 = __builtin_bit_cast(u32x2t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
      const u32x2t a1 = __builtin_bit_cast(u32x2t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * (TN * 2))));
      return as_bf(u32x4{a0[0], a0[1], a1[0], a1[1]});
    };
    bf16x8 fa[FM], fb[FN];
    fb[0] = rd_b(0);
#pragma unroll
    for (int i = 0; i < FM; ++i) fa[i] = as_bf(*reinterpret_cast<const u32x4*>(st + off_a + 16 * i * ROWB));
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      if (j + 1 < FN) fb[j + 1] = rd_b(j + 1);
      if (decltype(with)::value && j < N) load(kt + 3, nxt, j);
#pragma unroll
      for (int i = 0; i < FM; ++i)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int kt = 0;
  for (; kt + 4 <= nk; kt += 4) {
    step(flag_c<true>{}, num_c<2>{}, kt, b0, b3);
    step(flag_c<true>{}, num_c<2>{}, kt + 1, b1, b0);
    step(flag_c<true>{}, num_c<2>{}, kt + 2, b2, b1);
    step(flag_c<true>{}, num_c<2>{}, kt + 3, b3, b2);
  }
  if (kt < nk) step(flag_c<false>{}, num_c<2>{}, kt, b0, nullptr);
  if (kt + 1 < nk) step(flag_c<false>{}, num_c<1>{}, kt, b1, nullptr);
  if (kt + 2 < nk) step(flag_c<false>{}, num_c<0>{}, kt, b2, nullptr);
  vmem_wait_all();  // nothing lands in the buffers any more
  __syncthreads();  // the buffers are free
}

// NT tiles of 32 FM rows and 32 FN columns in either type, for products of few tiles: a step of 128 bytes of every row
// through a ring of NB buffers, so that its loads have NB - 1 steps' time to arrive.  T: uint16_t (bf16,
// v_mfma_f32_16x16x32_bf16, C a multiple of 8) or float (v_mfma_f32_16x16x4_f32, C a multiple of 4; slot l / 16 of
// instruction e stands for value 16 s + 4 (l / 16) + e, so a lane's values of a row are a 16-byte chunk here too).
// ring: NB buffers of kRingStage bytes.  Sums: acc[i][j][v] is row 16 FM wm + 16 i + l % 16, column
// 16 FN wn + 16 j + 4 (l / 16) + v.
template <int FM, int FN>
constexpr int kRingStage = 32 * (FM + FN) * 128;

template <typename T, int FM, int FN, int NB>
__device__ __forceinline__ void tile_ring(const T* P, int64_t ldp, int p_rows, const T* Q, int64_t ldq_, int q_cols, int C,
                                          int turn, char* const (&ring)[NB], f32x4 (&acc)[FM][FN]) {
  constexpr int A_BYTES = 32 * FM * 128, N = FM + FN, E = 16 / sizeof(T), TK = 8 * E;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, l15 = lane & 15, g4 = lane >> 4, lr = lane >> 3;
  const int nk = (C + TK - 1) / TK, lda = (int)ldp * (int)sizeof(T), ldb = (int)ldq_ * (int)sizeof(T);  // bytes
  const i32x4 ra = tile_rsrc(P, (int64_t)(min(32 * FM, p_rows) - 1) * lda + ((C + E - 1) / E) * 16);
  const i32x4 rb = tile_rsrc(Q, (int64_t)(min(32 * FN, q_cols) - 1) * ldb + ((C + E - 1) / E) * 16);
  constexpr int kNone = 0x7FFFFFF0;  // past every descriptor
  // chunk c of row r in slot c ^ r % 8 ^ r / 8 % 8: 16 rows put a chunk in 16 bank groups
  int chunk_a[FM], chunk_b[FN];
#pragma unroll
  for (int i = 0; i < FM; ++i) chunk_a[i] = (lane & 7) ^ lr ^ ((FM * wave + i) & 7);
#pragma unroll
  for (int i = 0; i < FN; ++i) chunk_b[i] = (lane & 7) ^ lr ^ ((FN * wave + i) & 7);
  // Steps in the order turn, turn + 1, .., nk - 1, 0, ..  Past the last one it is loaded again, for a buffer that is not
  // read: so each step's loads are followed by the same number of others.
  const int first = turn % nk;
  auto load = [&](int kt, char* st, int e) {
    const int at = min(kt, nk - 1) + first, k = at < nk ? at : at - nk;
    if (e < FM) {
      const int q = wave * FM + e;
      llvm_amdgcn_raw_buffer_load_lds_t(ra, (lds_u32*)(st + q * 1024), 16,
                                        k * TK + E * chunk_a[e] < C ? 16 * chunk_a[e] + lr * lda : kNone,
                                        __builtin_amdgcn_readfirstlane(q * 8 * lda + k * 128), 0, 0);
    } else {
      const int q = wave * FN + e - FM;
      llvm_amdgcn_raw_buffer_load_lds_t(rb, (lds_u32*)(st + A_BYTES + q * 1024), 16,
                                        k * TK + E * chunk_b[e - FM] < C ? 16 * chunk_b[e - FM] + lr * ldb : kNone,
                                        __builtin_amdgcn_readfirstlane(q * 8 * ldb + k * 128), 0, 0);
    }
  };
#pragma unroll
  for (int u = 0; u < NB - 1; ++u)
#pragma unroll
    for (int e = 0; e < N; ++e) load(u, ring[u], e);
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      asm volatile("" : "+a"(acc[i][j]));  // as in tile_nt
    }
  // Fragment addresses: a lane part picked by the half step and block (the chunk swizzle), plus an immediate.
  const int part = g4 ^ (l15 & 7) ^ (l15 >> 3);
  int off_a[4], off_b[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    off_a[x] = (16 * FM * wm + l15) * 128 + 16 * (part ^ ((2 * FM * wm) & 7) ^ (2 * x));
    off_b[x] = A_BYTES + (16 * FN * wn + l15) * 128 + 16 * (part ^ ((2 * FN * wn) & 7) ^ (2 * x));
  }
  // Step kt in `st`, with the loads of step kt + NB - 1 into `nxt`, which the step before this one has read; behind the
  // step's own loads are those of AFTER more.
  auto step = [&](auto with, auto after, int kt, const char* st, char* nxt) {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(decltype(after)::value * N));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();  // not __syncthreads(), which would wait for every load
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    u32x4 fa[2][FM], fb[2][FN];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[s][i] = *reinterpret_cast<const u32x4*>(st + off_a[((2 * s) ^ i) & 3] + 2048 * i);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[s][j] = *reinterpret_cast<const u32x4*>(st + off_b[((2 * s) ^ j) & 3] + 2048 * j);
    }
    if constexpr (decltype(with)::value) {
#pragma unroll
      for (int e = 0; e < N; ++e) load(kt + NB - 1, nxt, e);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int i = 0; i < FM; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf(fb[s][j]), as_bf(fa[s][i]), acc[i][j], 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(fb[s][j][e]), __uint_as_float(fa[s][i][e]),
                                                               acc[i][j], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  int kt = 0;
  for (; kt + NB <= nk; kt += NB) {
#pragma unroll
    for (int u = 0; u < NB; ++u) step(flag_c<true>{}, num_c<NB - 2>{}, kt + u, ring[u], ring[(u + NB - 1) % NB]);
  }
  ring_tail<0, NB - 1>([&](auto u) {
    constexpr int U = decltype(u)::value;
    if (kt + U < nk) step(flag_c<false>{}, num_c<NB - 2 - U>{}, kt, ring[U], nullptr);
  });
  vmem_wait_all();  // nothing lands in the buffers any more
  __syncthreads();
}

}  // namespace
}  // namespace dsv
