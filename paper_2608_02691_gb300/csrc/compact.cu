// Eviction, the move (include/optr.h, "optr_kv_compact"): the records of the positions
// that stay move together, in place, and the windows' ring turns with them.
//
// Records.  kept[i] >= i and the list rises, so a source lies behind the destinations
// of all moves before its own: moves may be made in chunks as long as everything that
// a chunk and those before it read is in registers before the chunk is written.  A
// cluster of CTAs takes a (sequence, KV head) and goes over its list in chunks of
// kRecords records a CTA; between a chunk's loads and its stores lies one cluster
// barrier, and the next chunk's loads are already under way then (they read behind the
// chunk's destinations).  Addresses come from the list and the table a chunk earlier
// still.  Bound by memory: a record is read and written in pieces of 16 bytes, two lanes
// to a slot's 32 code bytes.
// Where every second of 8192 records stays, all of the cache is read (memory gives 64
// bytes at a time, a piece is 32 or 16) and half written: 16 x 8192 to 4096 take 31.5 us,
// 4.9 TB/s of those bytes.  Records brought into L2 three chunks ahead took 38.5, clusters
// of 8 CTAs with one chunk each 36.9.
//
// Windows.  A ring of r rows turns by n - n' rows: CTAs of their own take the rows of a
// (sequence, KV head, kind), all bytes or a half or quarter of them, load 64 KB and
// store them.
#include "cluster.cuh"
#include "optr_internal.cuh"

#include <algorithm>

namespace optr {
namespace {

constexpr int kThreads = 512;
constexpr int kRecords = 512;  // of a chunk, by CTA

struct CompactArgs {
  const int32_t *kept, *n_kept, *lens, *bt;
  int n_most, max_pages, num_pages, h_kv, B;
  uint8_t* pool;
  float* score;
  int n_score;
  WinArgs win;
  int sink, recent;
  int cs, n_rec;  // CTAs of a (sequence, KV head); of them in all
  int slices;     // of a window row: 1, 2 or 4
  unsigned* err;
};

// What a (sequence, KV head) asks for; n == m: nothing.
struct Job {
  int n, m;      // tokens before and after
  unsigned bad;
};

__device__ __forceinline__ Job job_of(const CompactArgs& A, int b, int h) {
  Job j;
  j.n = __ldcg(A.lens + b);
  j.m = __ldcg(A.n_kept + b);
  j.bad = 0;
  if (j.n < 0 || j.n > A.max_pages * (long long)kPage || (A.score && j.n > A.n_score) || j.m < 0 ||
      j.m > j.n || j.m > A.n_most)
    j.bad = OPTR_DEVERR_SEQ_LEN;
  if (!j.bad && A.win.win) {
    const int slot = __ldcg(A.win.slot + b);
    if (slot < 0 || slot >= A.win.n_slots) {
      j.bad = OPTR_DEVERR_WIN_SLOT;
    } else if (j.m < j.n) {
      // the windows' positions have to be kept: the list rises, so one look at either
      const int32_t* kept = A.kept + ((size_t)b * A.h_kv + h) * A.n_most;
      if (j.m < A.sink + A.recent || (A.sink && __ldcg(kept + A.sink - 1) != A.sink - 1) ||
          (A.recent && __ldcg(kept + j.m - A.recent) != j.n - A.recent))
        j.bad = OPTR_DEVERR_KEPT;
    }
  }
  if (j.bad) j.n = j.m = 0;
  return j;
}

// A thread's pieces of a chunk: of the codes of two records, half a slot each, and of
// the pairs and the score of a third.
template <bool kCompact>
struct Pieces {
  using Meta = typename std::conditional<kCompact, uint32_t, uint4>::type;
  uint4 code[2][2];  // [record][kind]
  Meta meta[2];
  float score;
};

struct Smem {
  // by record of a chunk: byte offset of the page's record, its slot in the low four
  // bits (offsets are multiples of 128), or -1; sources three chunks deep, as they are
  // written while those of the two before are in use
  long long src[3][kRecords], dst[3][kRecords];
};

template <bool kCompact>
__device__ void move_records(const CompactArgs& A, Smem& S) {
  constexpr int kMeta = meta_stride(kCompact);
  using Meta = typename Pieces<kCompact>::Meta;
  const int seg = blockIdx.x / A.cs, rank = A.cs > 1 ? cluster_rank_of() : 0;
  const int b = seg / A.h_kv, h = seg % A.h_kv, tid = threadIdx.x;
  const Job job = job_of(A, b, h);
  if (job.bad && rank == 0 && tid == 0) atomicOr(A.err, job.bad);
  if (job.n == job.m) return;  // the same for the whole cluster
  const int32_t* kept = A.kept + (size_t)seg * A.n_most;
  const int32_t* table = A.bt + (size_t)b * A.max_pages;
  float* score = A.score ? A.score + (size_t)seg * A.n_score : nullptr;
  const int step = A.cs * kRecords, chunks = (job.m + step - 1) / step;
  const int first = rank * kRecords;  // of a chunk
  // Record tid's source position and entries of chunk c
  struct Request {
    int i, from, before;
  };
  auto request = [&](int c) {
    Request r{c * step + first + tid, -1, -1};
    if (c < chunks && r.i < job.m) {
      r.from = __ldcg(kept + r.i);
      if (r.i > 0) r.before = __ldcg(kept + r.i - 1);
    }
    return r;
  };
  auto address = [&](int c, const Request& r) {
    long long src = -1, dst = -1;
    if (c < chunks && r.i < job.m) {
      unsigned bad = 0;
      if (r.from <= r.before || r.from < r.i || r.from >= job.n) {
        bad = OPTR_DEVERR_KEPT;
      } else if (r.from != r.i) {
        const int ps = __ldcg(table + r.from / kPage), pd = __ldcg(table + r.i / kPage);
        if (ps < 0 || ps >= A.num_pages || pd < 0 || pd >= A.num_pages) {
          bad = OPTR_DEVERR_PAGE_ID;
        } else {
          src = (long long)(((size_t)ps * A.h_kv + h) * chunk_bytes(kCompact)) | (r.from % kPage);
          dst = (long long)(((size_t)pd * A.h_kv + h) * chunk_bytes(kCompact)) | (r.i % kPage);
        }
      }
      if (bad) atomicOr(A.err, bad);
    }
    S.src[c % 3][tid] = src;
    S.dst[c % 3][tid] = dst;
  };
  static_assert(kRecords == kThreads && chunk_bytes(kCompact) % 16 == 0, "one record a thread");
  const int half = 16 * (tid & 1);
  // from[] of the score's move of chunk c: the thread's own record
  auto load = [&](int c, Pieces<kCompact>& x, int from) {
    if (c >= chunks) return;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const long long s = S.src[c % 3][(kThreads / 2) * e + tid / 2];
      if (s >= 0) {
        const uint8_t* r = A.pool + (s & ~15ll) + 32 * (s & 15) + half;
        x.code[e][0] = __ldcg(reinterpret_cast<const uint4*>(r + OPTR_K_CODES_OFFSET));
        x.code[e][1] = __ldcg(reinterpret_cast<const uint4*>(r + OPTR_V_CODES_OFFSET));
      }
    }
    const long long s = S.src[c % 3][tid];
    if (s >= 0) {
      const uint8_t* r = A.pool + (s & ~15ll) + kMeta * (s & 15);
      x.meta[0] = __ldcg(reinterpret_cast<const Meta*>(r + OPTR_K_META_OFFSET));
      x.meta[1] = __ldcg(reinterpret_cast<const Meta*>(r + vmeta_offset(kCompact)));
      if (score) x.score = __ldcg(score + from);
    }
  };
  auto store = [&](int c, const Pieces<kCompact>& x) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const long long d = S.dst[c % 3][(kThreads / 2) * e + tid / 2];
      if (d >= 0) {
        uint8_t* r = A.pool + (d & ~15ll) + 32 * (d & 15) + half;
        *reinterpret_cast<uint4*>(r + OPTR_K_CODES_OFFSET) = x.code[e][0];
        *reinterpret_cast<uint4*>(r + OPTR_V_CODES_OFFSET) = x.code[e][1];
      }
    }
    const long long d = S.dst[c % 3][tid];
    if (d >= 0) {
      uint8_t* r = A.pool + (d & ~15ll) + kMeta * (d & 15);
      *reinterpret_cast<Meta*>(r + OPTR_K_META_OFFSET) = x.meta[0];
      *reinterpret_cast<Meta*>(r + vmeta_offset(kCompact)) = x.meta[1];
      if (score) score[c * step + first + tid] = x.score;
    }
  };
  // requests two chunks ahead of the stores, loads one
  Pieces<kCompact> x[2];
  Request r = request(0);
  address(0, r);
  int from = r.from;
  r = request(1);
  __syncthreads();
  load(0, x[0], from);
  for (int c0 = 0; c0 < chunks; c0 += 2) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int c = c0 + e;
      if (c >= chunks) break;
      address(c + 1, r);
      from = r.from;
      r = request(c + 2);
      __syncthreads();
      load(c + 1, x[e ^ 1], from);
      // every CTA has read the chunk's sources
      if (A.cs > 1) cluster_barrier(); else __syncthreads();
      store(c, x[e]);
    }
  }
  if (score)
    for (int i = job.m + rank * kThreads + tid; i < job.n; i += A.cs * kThreads) score[i] = 0.f;
}

__device__ void turn_ring(const CompactArgs& A, int unit) {
  const int slice = unit % A.slices, kind = unit / A.slices % 2, seg = unit / (2 * A.slices);
  const int pieces = 16 / A.slices;  // of 16 bytes, of a row
  const int b = seg / A.h_kv, h = seg % A.h_kv, tid = threadIdx.x;
  if (b >= A.B) return;
  const Job job = job_of(A, b, h);
  const int d = job.n - job.m, rows = A.sink + A.recent;
  if (d == 0 || d % A.recent == 0) return;
  uint8_t* base = reinterpret_cast<uint8_t*>(A.win.win) +
                  (((size_t)__ldcg(A.win.slot + b) * A.h_kv + h) * 2 + kind) * (size_t)rows * (2 * kD) +
                  16 * (pieces * slice + tid % pieces);
  // position n - recent + j, at row sink + (n - recent + j - sink) % recent
  const int old0 = (job.n - A.sink) % A.recent, new0 = (job.m - A.sink) % A.recent;
  constexpr int kMost = 8;  // pieces of a thread
  uint4 x[kMost];
#pragma unroll
  for (int e = 0; e < kMost; ++e) {
    const int j = (kThreads * e + tid) / pieces;
    if (j < A.recent)
      x[e] = __ldcg(reinterpret_cast<const uint4*>(base + (size_t)(A.sink + (old0 + j) % A.recent) * (2 * kD)));
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kMost; ++e) {
    const int j = (kThreads * e + tid) / pieces;
    if (j < A.recent)
      *reinterpret_cast<uint4*>(base + (size_t)(A.sink + (new0 + j) % A.recent) * (2 * kD)) = x[e];
  }
}

template <bool kCompact>
__global__ void __launch_bounds__(kThreads, 2) compact_kernel(const __grid_constant__ CompactArgs A) {
  __shared__ Smem S;
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x < A.n_rec)
    move_records<kCompact>(A, S);
  else
    turn_ring(A, (int)blockIdx.x - A.n_rec);
}

}  // namespace
}  // namespace optr

using namespace optr;

extern "C" optr_status optr_kv_compact_win(const optr_params* p, const int32_t* kept, int n_most,
                                           const int32_t* n_kept, const int32_t* lens,
                                           const int32_t* block_table, int B, int max_pages,
                                           uint8_t* pool, int num_pages, void* win,
                                           const int32_t* win_slot, int n_slots, float* score,
                                           int n_score, cudaStream_t stream) {
  if (!p || !kept || !n_kept || !lens || !block_table || !pool || n_most <= 0 || B <= 0 ||
      max_pages <= 0 || num_pages <= 0 || !aligned(pool, 16) || !aligned(score, 4) || (score && n_score <= 0))
    return OPTR_ERR_INVALID_ARG;
  WinArgs w{nullptr, nullptr, 0};
  if (p->cfg.sink + p->cfg.recent > 0) {
    if (!win || !win_slot || n_slots <= 0 || !aligned(win, 16)) return OPTR_ERR_INVALID_ARG;
    w = WinArgs{(__nv_bfloat16*)win, win_slot, n_slots};
  }
  const long long segs = (long long)B * p->cfg.h_kv;
  if (segs > (1 << 24) || max_pages > (1 << 26) || (long long)max_pages * kPage > 0x7fffffffll)
    return OPTR_ERR_OUT_OF_RANGE;
  // CTAs of a (sequence, KV head): two per SM in all, each a chunk at least
  int cs = 1;
  while (cs < 8 && segs * 2 * cs <= 2 * p->num_sms && n_most > cs * kRecords) cs *= 2;
  // few long lists: 16 (one of 131072 to 30000, 8 heads: 39.9 -> 29.6 us)
  if (cs == 8 && segs * 16 <= p->num_sms && n_most > 16 * kRecords) cs = 16;
  const bool turn = w.win && p->cfg.recent > 0;
  const int slices = p->cfg.recent <= 256 ? 1 : p->cfg.recent <= 512 ? 2 : 4;  // 8 pieces a thread
  const long long n_rec = segs * cs, units = turn ? (segs * 2 * slices + cs - 1) / cs * cs : 0;
  const CompactArgs A{kept, n_kept, lens, block_table, n_most, max_pages, num_pages, p->cfg.h_kv, B,
                      pool, score, n_score, w, p->cfg.sink, p->cfg.recent, cs, (int)n_rec, slices, p->err};
  auto fn = p->cfg.group == 4 * kG ? compact_kernel<true> : compact_kernel<false>;
  if (cs > 8 && ensure_wide_clusters(reinterpret_cast<const void*>(fn)) != cudaSuccess) return OPTR_ERR_CUDA;
  return cuda_status(launch_pdl_cluster(fn, dim3((unsigned)(n_rec + units)), dim3(kThreads), cs, 0, stream, A));
}

extern "C" optr_status optr_kv_compact(const optr_params* p, const int32_t* kept, int n_most,
                                       const int32_t* n_kept, const int32_t* lens,
                                       const int32_t* block_table, int B, int max_pages, uint8_t* pool,
                                       int num_pages, float* score, int n_score, cudaStream_t stream) {
  if (p && (p->cfg.sink > 0 || p->cfg.recent > 0)) return OPTR_ERR_INVALID_ARG;
  return optr_kv_compact_win(p, kept, n_most, n_kept, lens, block_table, B, max_pages, pool, num_pages,
                             nullptr, nullptr, 0, score, n_score, stream);
}
