// Chunk attention: arguments, work partition and workspace, shared by its
// kernels (chunk.cu).
#pragma once

#include "decode_common.cuh"
#include "optr_internal.cuh"
#include "tc05.cuh"

namespace optr {

struct ChunkArgs {
  int n_tok;
  const int32_t *cu, *pos0;
  int max_new;
  const int32_t* bt;
  int B, max_pages;
  const uint8_t* pool;
  int num_pages;
  WinArgs win;
  int sink, recent, h_kv, compact;
  const uint16_t *Rk_query, *Rv_back;
  const float* muR;
  __nv_bfloat16* out;
  unsigned* err;
  // workspace
  struct ChunkSeg* seg;  // [W] segments begun by a CTA and ended by another
  float* part;           // partial results
  int rows;              // rows of a partial
  int W;                 // CTAs
  bool out32;            // out is 32-byte aligned
  const int32_t* parent; // trees: the rows' parents
};

// A segment that CTA w begins and another one ends: its pieces are those of the
// CTAs from w on whose ranges begin before `end`.
struct ChunkSeg {
  long long F, end;
  int c0, n_new, h, qb;
  int W;              // ranges that the line is cut into
  int valid;
};

constexpr int kQTok = 64;     // tokens of a query block: two tiles of 32 x 4 heads
constexpr int kTile = 128;    // keys per tile
constexpr float kLogit = 1.44269504088896340736f * 0.08838834764831844055f;  // log2(e) / sqrt(128)

// What one sequence asks for.
struct SeqWork {
  int c0, n_new, n_past;
  int n_int, n_win;  // cached INT2 positions (from `sink` on) and window rows
  int slot;
  unsigned bad;      // why the sequence is left out (device error bits)
};

__device__ __forceinline__ SeqWork seq_work(const ChunkArgs& A, int b) {
  SeqWork s;
  s.c0 = __ldcg(A.cu + b);
  const int c1 = __ldcg(A.cu + b + 1);
  s.n_past = __ldcg(A.pos0 + b);
  s.slot = A.win.win ? __ldcg(A.win.slot + b) : 0;
  s.n_new = c1 - s.c0;
  s.n_int = s.n_win = 0;
  s.bad = 0;
  if (s.c0 < 0 || c1 < s.c0 || c1 > A.n_tok || s.n_new > A.max_new)
    s.bad = OPTR_DEVERR_CU_NEW;
  else if (s.n_past < 0 || s.n_past > A.max_pages * kPage)
    s.bad = OPTR_DEVERR_SEQ_LEN;
  if (s.bad) {
    s.n_new = 0;
    return s;
  }
  const int e = int2_end(s.n_past, A.sink, A.recent);
  s.n_int = max(0, min(e, s.n_past) - A.sink);
  if (A.win.win && s.slot >= 0 && s.slot < A.win.n_slots) s.n_win = min(s.n_past, A.sink + A.recent);
  return s;
}

__device__ __forceinline__ int tiles_of(int keys) { return (keys + kTile - 1) / kTile; }

// Cost of the first m query blocks of a sequence (one head), in tiles, `past`
// cached tiles each: block qb sees own tiles 0 .. qb / 2, and begin_cost tiles'
// time goes into its start and end, more where INT2 tiles have the queries rotated
// and the output rotated back.  Measured: a ragged batch of 64 sequences takes 139 us,
// 160 with 2 for all; an 8192-token prompt 406 us, 415 with 5 where nothing is cached.
constexpr int kBegin = 2, kBeginInt2 = 6;
__device__ __forceinline__ int begin_cost(int n_int) { return n_int > 0 ? kBeginInt2 : kBegin; }
__device__ __forceinline__ long long block_cost(long long m, int past, int begin) {
  return m * (past + begin) + (m + 1) * (m + 1) / 4;
}

// A run of tiles of one (sequence, KV head, query block): tiles t0 .. t1-1 of
// its `total`, INT2 tiles first, then the windows', then the chunk's own.
struct Piece {
  int b, h, qb;
  int c0, n_new, n_int, n_win, slot;
  int I, Wt;         // INT2 and window tiles of the segment
  int t0, t1, total;
  __device__ __forceinline__ int int_tiles() const { return max(0, min(t1, I) - t0); }
  // query tiles that have rows: 2, or 1 that both softmax groups work on
  __device__ __forceinline__ int q_tiles() const { return n_new - qb * kQTok > kQTok / 2 ? 2 : 1; }
};

__device__ __forceinline__ long long seq_cost(const SeqWork& s) {
  return s.n_new > 0 ? block_cost((s.n_new + kQTok - 1) / kQTok, tiles_of(s.n_int) + tiles_of(s.n_win),
                                  begin_cost(s.n_int))
                     : 0;
}

// The flat index space orders units of cost as (sequence, KV head, query block,
// unit); CTA w takes [w F / W, (w + 1) F / W).  Of a block's begin_cost + tiles
// units the first begin_cost stand for no tile.  One warp goes through a CTA's range: lane
// i holds sequence b0 + i.
struct PieceFinder {
  long long f, f1, F;    // the next unit, the range's end, all units
  int W;                 // ranges: A.W, or fewer so that each has a unit (one token over 1024:
                         // 14.7 us, 19.4 with four units at least)
  long long f_seg;       // first unit of the last piece's segment
  int b0;                // the 32 sequences held, and what comes before them
  long long base, incl;  // (cost of one head); incl: up to and with the lane's
  SeqWork s;

  __device__ __forceinline__ void hold(const ChunkArgs& A, int first) {
    const int lane = threadIdx.x & 31;
    b0 = first;
    s.n_new = 0;
    if (b0 + lane < A.B) s = seq_work(A, b0 + lane);
    incl = seq_cost(s);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
  }

  __device__ __forceinline__ void start(const ChunkArgs& A, int w) {
    const int lane = threadIdx.x & 31;
    long long sum = 0;
#pragma unroll 4
    for (int b = lane; b < A.B; b += 32) sum += seq_cost(seq_work(A, b));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    F = sum * A.h_kv;
    W = (int)min((long long)A.W, max(1ll, F));
    f = w < W ? F * w / W : F;
    f1 = w < W ? F * (w + 1) / W : F;
    base = 0;
    hold(A, 0);
  }

  // The piece at f (< f1), in all lanes; it has no tile (t1 = t0) where the
  // range ends within begin_cost.
  __device__ __forceinline__ void next(const ChunkArgs& A, Piece& p) {
    unsigned over;  // lanes whose sequence ends after f
    while (!(over = __ballot_sync(0xffffffffu, (base + incl) * A.h_kv > f))) {
      if (b0 >= A.B) {  // (only where the tables change under the call)
        f = f1;
        p.t0 = p.t1 = 0;
        return;
      }
      base += __shfl_sync(0xffffffffu, incl, 31);
      hold(A, b0 + 32);
    }
    const int l = __ffs(over) - 1;
    auto of = [&](int x) { return __shfl_sync(0xffffffffu, x, l); };
    const long long c = __shfl_sync(0xffffffffu, seq_cost(s), l);
    const long long before = base + __shfl_sync(0xffffffffu, incl, l) - c;
    p.b = b0 + l;
    p.c0 = of(s.c0), p.n_new = of(s.n_new), p.n_int = of(s.n_int), p.n_win = of(s.n_win);
    p.slot = of(s.slot);
    p.I = tiles_of(p.n_int);
    p.Wt = tiles_of(p.n_win);
    long long r = f - before * A.h_kv;
    p.h = (int)(r / c);
    r -= p.h * c;
    const int begin = begin_cost(p.n_int);
    int q0 = 0, q1 = (p.n_new + kQTok - 1) / kQTok;
    while (q1 - q0 > 1) {
      const int mid = (q0 + q1) >> 1;
      if (block_cost(mid, p.I + p.Wt, begin) <= r) q0 = mid; else q1 = mid;
    }
    p.qb = q0;
    p.total = p.I + p.Wt + q0 / 2 + 1;
    const long long u0 = r - block_cost(q0, p.I + p.Wt, begin);
    const long long u1 = min((long long)p.total + begin, u0 + (f1 - f));
    p.t0 = (int)max(0ll, u0 - begin);
    p.t1 = (int)max(0ll, u1 - begin);
    f_seg = f - u0;
    f += u1 - u0;
  }
};

// Flags what is wrong with the sequences; one warp of a call's.
__device__ __forceinline__ void report_sequences(const ChunkArgs& A) {
  const int lane = threadIdx.x & 31;
  if (lane == 0 && (__ldcg(A.cu) != 0 || __ldcg(A.cu + A.B) != A.n_tok))
    atomicOr(A.err, OPTR_DEVERR_CU_NEW);
  for (int b = lane; b < A.B; b += 32) {
    const SeqWork x = seq_work(A, b);
    unsigned bad = x.bad;
    if (!bad && A.win.win && (x.slot < 0 || x.slot >= A.win.n_slots)) bad = OPTR_DEVERR_WIN_SLOT;
    if (bad) atomicOr(A.err, bad);
  }
}

// A partial: O [32 channel groups][rows][4], then m [rows] and l [rows].
// CTA w has two: of a segment begun by an earlier CTA, and of one that a later
// CTA ends.
__host__ __device__ constexpr size_t part_floats(int rows) { return (size_t)rows * (kD + 2); }
__device__ __forceinline__ float* part_of(const ChunkArgs& A, int w, bool begun) {
  return A.part + (2 * (size_t)w + (begun ? 1 : 0)) * part_floats(A.rows);
}

// A CTA's warp that finds its pieces for the others, kAhead ahead: a piece
// without tiles ends them.  then(n, p) follows the n-th one, and says whether to go on.
template <int kAhead, typename Then>
__device__ __forceinline__ void find_pieces(const ChunkArgs& A, int w, Piece* piece, uint64_t* full,
                                            uint64_t* empty, volatile int* abort, Then then) {
  const int lane = threadIdx.x & 31;
  if (w == 0) report_sequences(A);
  PieceFinder next;
  next.start(A, w);
  ChunkSeg seg{};
  bool more = true;
  for (uint32_t n = 0; more; ++n) {
    const uint32_t i = n % kAhead;
    Piece p;
    p.t0 = p.t1 = 0;
    while (next.f < next.f1 && p.t1 == p.t0) next.next(A, p);
    more = p.t1 > p.t0;
    if (more && p.t0 == 0 && p.t1 < p.total)
      seg = ChunkSeg{next.F, next.f_seg + begin_cost(p.n_int) + p.total, p.c0, p.n_new, p.h, p.qb, next.W, 1};
    if (n >= kAhead &&
        !__all_sync(0xffffffffu, tc05::bar_wait_spin(&empty[i], (n / kAhead - 1) & 1, abort)))
      break;
    if (lane == 0) {
      piece[i] = p;
      tc05::bar_arrive(&full[i]);
    }
    __syncwarp();
    if (more && !then(n, p)) break;
  }
  if (lane == 0) A.seg[w] = seg;
}

}  // namespace optr
