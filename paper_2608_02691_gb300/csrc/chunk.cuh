// Chunk attention: arguments, work partition and workspace, shared by its
// kernels (chunk.cu).
#pragma once

#include "decode_common.cuh"
#include "optr_internal.cuh"

namespace optr {

struct ChunkArgs {
  const __nv_bfloat16* q;
  int n_tok;
  const int32_t *cu, *pos0;
  int max_new;
  const int32_t* bt;
  int B, max_pages;
  const uint8_t* pool;
  int num_pages;
  WinArgs win;
  int sink, recent, h_kv, compact;
  const uint4* Rk_frag;
  const uint16_t* Rv_back;
  const float* mu;
  __nv_bfloat16* out;
  unsigned* err;
  // workspace
  long long* pref;       // [B + 1] cost of the sequences before b, one head
  __half* qrot;          // [n_tok][h_q][128] rotated queries, scaled, order of dequant.cuh
  float2* qinfo;         // [n_tok][h_q] logit scale of a rotated query; <q, mu>
  float* part;           // partial results, ChunkPart
  int rows;              // rows of a partial
  int W;                 // CTAs of the attention kernel
  bool out32;            // out is 32-byte aligned
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
// cached tiles each: block qb sees own tiles 0 .. qb / 2, and kBegin tiles' time
// goes into its start and end.
constexpr int kBegin = 2;
__device__ __forceinline__ long long block_cost(long long m, int past) {
  return m * (past + kBegin) + (m + 1) * (m + 1) / 4;
}

// A run of tiles of one (sequence, KV head, query block): tiles t0 .. t1-1 of
// its `total`, INT2 tiles first, then the windows', then the chunk's own.
struct Piece {
  int b, h, qb;
  int c0, n_new, n_int, n_win, slot;
  int I, Wt;         // INT2 and window tiles of the segment
  int t0, t1, total;
  __device__ __forceinline__ int int_tiles() const { return max(0, min(t1, I) - t0); }
  // query tiles that have rows
  __device__ __forceinline__ int q_tiles() const { return n_new - qb * kQTok > kQTok / 2 ? 2 : 1; }
};

// The flat index space orders units of cost as (sequence, KV head, query block,
// unit); CTA w takes [w F / W, (w + 1) F / W).  Of a block's kBegin + tiles units
// the first kBegin stand for no tile.  Called by a whole warp: the piece that
// starts at f < F of a range that ends at f1, in all lanes; *f_seg receives the
// flat index of the segment's first unit, the return value is the next piece's
// start.  The piece has no tile (t1 = t0) where the range ends within kBegin.
__device__ __forceinline__ long long locate_piece(const ChunkArgs& A, long long f, long long f1,
                                                  Piece& p, long long* f_seg) {
  const int lane = threadIdx.x & 31;
  // the last sequence b with pref[b] h_kv <= f, 32 probes at a time
  int lo = 0, hi = A.B;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const bool le = at < hi && __ldcg(A.pref + at) * A.h_kv <= f;
    lo += (__popc(__ballot_sync(0xffffffffu, le)) - 1) * step;
    hi = min(hi, lo + step);
  }
  const long long base = __ldcg(A.pref + lo), cost = __ldcg(A.pref + lo + 1) - base;
  const SeqWork s = seq_work(A, lo);
  long long r = f - base * A.h_kv;
  p.b = lo;
  p.h = (int)(r / cost);
  r -= p.h * cost;
  p.c0 = s.c0, p.n_new = s.n_new, p.n_int = s.n_int, p.n_win = s.n_win, p.slot = s.slot;
  p.I = tiles_of(s.n_int);
  p.Wt = tiles_of(s.n_win);
  int q0 = 0, q1 = (s.n_new + kQTok - 1) / kQTok;
  while (q1 - q0 > 1) {
    const int mid = (q0 + q1) >> 1;
    if (block_cost(mid, p.I + p.Wt) <= r) q0 = mid; else q1 = mid;
  }
  p.qb = q0;
  p.total = p.I + p.Wt + q0 / 2 + 1;
  const long long u0 = r - block_cost(q0, p.I + p.Wt);
  const long long u1 = min((long long)p.total + kBegin, u0 + (f1 - f));
  p.t0 = (int)max(0ll, u0 - kBegin);
  p.t1 = (int)max(0ll, u1 - kBegin);
  *f_seg = f - u0;
  return f + (u1 - u0);
}

// A partial: O [32 channel groups][rows][4], then m [rows] and l [rows].
// CTA w has two: of a segment begun by an earlier CTA, and of one that a later
// CTA ends.
__host__ __device__ constexpr size_t part_floats(int rows) { return (size_t)rows * (kD + 2); }
__device__ __forceinline__ float* part_of(const ChunkArgs& A, int w, bool begun) {
  return A.part + (2 * (size_t)w + (begun ? 1 : 0)) * part_floats(A.rows);
}

}  // namespace optr
