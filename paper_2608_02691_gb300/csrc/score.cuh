// Attention weights of the new tokens, summed by position: arguments, work partition
// and workspace, shared by its kernels (score.cu).
#pragma once

#include "decode_common.cuh"
#include "optr_internal.cuh"

namespace optr {

constexpr int kTok = 64;       // tokens of a query block
constexpr int kKeys = 128;     // keys of a tile
constexpr int kBlockCols = 4 * kTok;  // logit columns: token i, head j at 4 i + j
constexpr float kLogit = 1.44269504088896340736f * 0.08838834764831844055f;  // log2(e) / sqrt(128)

struct ScoreArgs {
  const __nv_bfloat16* q;
  int n_tok;
  const int32_t *cu, *pos0;
  int max_new, t0;       // t0: the query block's first token in its sequence
  const int32_t* bt;
  int B, max_pages;
  const uint8_t* pool;
  int num_pages;
  WinArgs win;
  int sink, recent, h_kv, compact;
  const float *R_k, *mu;
  float* score;
  int n_score;
  unsigned* err;
  // workspace
  int cols;              // columns kept for a block
  uint8_t* qop;          // query operands, by (sequence, KV head)
  float2* part;          // [W + segments][2][kKeys] maxima and sums of a CTA
  int W;                 // CTAs
};

// A decode step's few tokens (score_few.cu): its part of the workspace, and the launches.
constexpr int kFewTok = 4;
struct FewLayout {
  size_t part, logits, total;
  int W;  // warps
};
FewLayout few_layout(const optr_params* p, int B, int max_new, int max_pages);
bool few_tokens(const optr_params* p, int B, int max_new, int max_pages);
cudaError_t launch_score_few(const optr_params* p, const ScoreArgs& A, uint8_t* ws, cudaStream_t s);

// What one sequence asks for of the query block.
struct ScoreSeq {
  int c0, pos0, n;       // row of its first token, cached tokens before, and with them
  int rows;              // tokens of the block
  int n_int, n_win, slot;
  unsigned bad;          // why it is left out (device error bits)
};

__device__ __forceinline__ ScoreSeq score_seq(const ScoreArgs& A, int b) {
  ScoreSeq s;
  s.c0 = __ldcg(A.cu + b);
  const int c1 = __ldcg(A.cu + b + 1);
  s.pos0 = __ldcg(A.pos0 + b);
  s.slot = A.win.win ? __ldcg(A.win.slot + b) : 0;
  const int n_new = c1 - s.c0;
  s.n = s.rows = s.n_int = s.n_win = 0;
  s.bad = 0;
  if (s.c0 < 0 || c1 < s.c0 || c1 > A.n_tok || n_new > A.max_new) {
    s.bad = OPTR_DEVERR_CU_NEW;
    return s;
  }
  const long long n = (long long)s.pos0 + n_new;
  if (s.pos0 < 0 || n > (long long)A.max_pages * kPage || n > A.n_score) {
    s.bad = OPTR_DEVERR_SEQ_LEN;
    return s;
  }
  if (n_new <= A.t0) return s;
  s.n = (int)n;
  s.rows = min(n_new - A.t0, kTok);
  s.n_int = max(0, min(int2_end(s.n, A.sink, A.recent), s.n) - A.sink);
  if (A.win.win) {
    if (s.slot < 0 || s.slot >= A.win.n_slots)
      s.bad = OPTR_DEVERR_WIN_SLOT;  // (its window keys are left out)
    else
      s.n_win = win_count(s.n, A.sink, A.recent);
  }
  return s;
}

__device__ __forceinline__ int key_tiles(int keys) { return (keys + kKeys - 1) / kKeys; }
__device__ __forceinline__ int seq_tiles(const ScoreSeq& s) { return key_tiles(s.n_int) + key_tiles(s.n_win); }

// Flags what is wrong with the sequences; one warp of a call's.
__device__ __forceinline__ void report_sequences(const ScoreArgs& A) {
  const int lane = threadIdx.x & 31;
  if (lane == 0 && (__ldcg(A.cu) != 0 || __ldcg(A.cu + A.B) != A.n_tok))
    atomicOr(A.err, OPTR_DEVERR_CU_NEW);
  for (int b = lane; b < A.B; b += 32) {
    const unsigned bad = score_seq(A, b).bad;
    if (bad) atomicOr(A.err, bad);
  }
}

// Units t0 .. t1-1 of a (sequence, KV head), INT2 ones first, then the windows'.
struct ScorePiece {
  int seg, b, h;
  int c0, pos0, n, rows, n_int, n_win, slot;
  int t0, t1;
  int w0, w1;  // the workers that have a part in the segment
  __device__ __forceinline__ int I() const { return key_tiles(n_int); }  // INT2 tiles
  __device__ __forceinline__ int cols() const { return 4 * rows; }
  // columns of the products, a multiple of 16
  __device__ __forceinline__ int N() const { return (4 * rows + 15) / 16 * 16; }
};

// Units of a (sequence, KV head): tiles of 128 keys.
struct Tiles {
  __device__ __forceinline__ static int of(const ScoreSeq& s) { return seq_tiles(s); }
};

// The flat index space orders units as (sequence, KV head, unit); worker w of W takes
// [w F / W, (w + 1) F / W).  One warp goes through a range: lane i holds sequence
// b0 + i.
template <typename Unit>
struct ScoreFinder {
  long long f, f1, F, W;
  int b0;
  long long base, incl;  // units of one head before the 32 held; up to and with the lane's
  ScoreSeq s;

  __device__ __forceinline__ void hold(const ScoreArgs& A, int first) {
    const int lane = threadIdx.x & 31;
    b0 = first;
    s.rows = s.n_int = s.n_win = 0;
    if (b0 + lane < A.B) s = score_seq(A, b0 + lane);
    incl = Unit::of(s);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
  }

  __device__ __forceinline__ void start(const ScoreArgs& A, int w, int workers) {
    const int lane = threadIdx.x & 31;
    long long sum = 0;
    for (int b = lane; b < A.B; b += 32) sum += Unit::of(score_seq(A, b));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    F = sum * A.h_kv;
    W = min((long long)workers, max(1ll, F));  // each has a unit
    f = w < W ? F * w / W : F;
    f1 = w < W ? F * (w + 1) / W : F;
    base = 0;
    hold(A, 0);
  }

  // The piece at f (< f1), in all lanes.
  __device__ __forceinline__ void next(const ScoreArgs& A, ScorePiece& p) {
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
    const int T = of(Unit::of(s));
    const long long before = base + __shfl_sync(0xffffffffu, incl, l) - T;
    p.b = b0 + l;
    p.c0 = of(s.c0), p.pos0 = of(s.pos0), p.n = of(s.n), p.rows = of(s.rows);
    p.n_int = of(s.n_int), p.n_win = of(s.n_win), p.slot = of(s.slot);
    const long long r = f - before * A.h_kv;
    p.h = (int)(r / T);
    p.seg = p.b * A.h_kv + p.h;
    p.t0 = (int)(r - (long long)p.h * T);
    p.t1 = (int)min((long long)T, p.t0 + (f1 - f));
    p.w0 = 0, p.w1 = T;
    f += p.t1 - p.t0;
  }

  // The workers of the piece's segment (after next()).
  __device__ __forceinline__ void workers(const ScoreArgs& A, ScorePiece& p) {
    if (p.t1 <= p.t0) return;
    const long long f0 = f - p.t1, T = p.w1;  // the segment's first unit, and its units
    // the worker of a unit f: the largest w with w F / W <= f
    p.w0 = (int)(((f0 + 1) * W - 1) / F);
    p.w1 = (int)(((f0 + T) * W - 1) / F);
  }
};

// What comes before a (sequence, KV head) in the flat order: the workers that have a part
// in it, w0 .. w1 (none: w1 < w0).  A whole CTA; `sum` has an element a warp.
template <typename Unit>
__device__ __forceinline__ void workers_of(const ScoreArgs& A, int b, int h, int workers, long long* sum,
                                           int& w0, int& w1) {
  const int threads = blockDim.x, tid = threadIdx.x;
  long long x[2] = {0, 0};  // units of one head: before b, in all
  for (int i = tid; i < A.B; i += threads) {
    const int t = Unit::of(score_seq(A, i));
    x[1] += t;
    if (i < b) x[0] += t;
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x[e] += __shfl_xor_sync(0xffffffffu, x[e], o);
    __syncthreads();
    if ((tid & 31) == 0) sum[tid >> 5] = x[e];
    __syncthreads();
    x[e] = 0;
    for (int i = 0; i < threads / 32; ++i) x[e] += sum[i];
  }
  const long long F = x[1] * A.h_kv, W = min((long long)workers, max(1ll, F));
  const int T = Unit::of(score_seq(A, b));
  w0 = 0, w1 = -1;
  if (T == 0) return;
  const long long f0 = x[0] * A.h_kv + (long long)h * T;
  // the worker of a unit f: the largest w with w F / W <= f
  w0 = (int)(((f0 + 1) * W - 1) / F);
  w1 = (int)(((f0 + T) * W - 1) / F);
}

// Operands of a (sequence, KV head)'s query block: hi and lo parts of the rotated
// queries, the queries as given (with windows), 256 B a column each, and of four pairs a
// slot the groups' sums of the rotated ones, 32 B a column; then by column <q, mu> and the
// rotated query's sum, and for the block the factor that brings a product with the rotated
// ones to log2 units, and the largest sums of a column's magnitudes, rotated and as given.
__host__ __device__ __forceinline__ size_t qop_lines(int cols, bool win, bool compact) {
  return (size_t)cols * (256 * (win ? 3 : 2) + (compact ? 0 : 32));
}
__host__ __device__ __forceinline__ size_t qop_bytes(int cols, bool win, bool compact) {
  return qop_lines(cols, win, compact) + (size_t)cols * 8 + 16;
}
__device__ __forceinline__ uint8_t* qop_of(const ScoreArgs& A, int seg) {
  return A.qop + (size_t)seg * qop_bytes(A.cols, A.win.win != nullptr, A.compact);
}
// a CTA's partial of a segment: (CTA, segment) pairs lie on a staircase, so their sum is
// a slot of its own
__device__ __forceinline__ float2* score_part(const ScoreArgs& A, int w, int seg) {
  return A.part + (size_t)(w + seg) * 2 * kKeys;
}

}  // namespace optr
