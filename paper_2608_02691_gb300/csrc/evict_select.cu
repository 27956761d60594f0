// Eviction, the choice of the positions that stay (include/optr.h,
// "optr_evict_select"): of a row of n scores the k largest, as a rising list.
//
// A cluster of CTAs takes a (sequence, KV head), each CTA a contiguous slice of its
// positions.  The scores become 32-bit keys that order as they do, kept in shared
// memory as far as they fit (kSlice of a CTA).  Three counts of 11, 11 and 10 bits
// from the top find the k-th largest key T: each CTA counts its slice's digits, the
// cluster's counts are added through distributed shared memory, and every CTA takes
// the digit at which the sum from the top reaches k.  Then all keys above T stay, and
// of those equal to it the lowest positions, as many as are missing.  A warp owns a
// contiguous part of the slice, so the number of kept positions before it, counted once
// and summed over warps and CTAs, is all it needs to write its own in order.
#include "cluster.cuh"
#include "optr_internal.cuh"

#include <algorithm>

namespace optr {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kSlice = 16384;  // keys of a CTA in shared memory, 64 KB

struct Smem {
  uint32_t hist[2][kBins];
  int sum[kWarps];
  int above[kWarps], equal[kWarps];  // by warp, then what lies before it
  int digit, rest;
  int count[2];                      // this CTA's keys above T, and equal to it
};

// Unsigned order = the scores' (-0 as 0, NaN above all).
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(__fadd_rn(x, 0.f));
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kThreads)
select_kernel(const float* __restrict__ score, int n_score, const int32_t* __restrict__ lens,
              const int32_t* __restrict__ keep, int h_kv, int first, int last,
              int32_t* __restrict__ kept, int n_most, int32_t* __restrict__ n_kept, int cs,
              int n_keys, unsigned* err) {
  __shared__ Smem S;
  extern __shared__ uint32_t keys[];
  const int seg = blockIdx.x / cs, rank = cs > 1 ? cluster_rank_of() : 0, b = seg / h_kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  pdl_trigger();
  const int n = __ldcg(lens + b);
  const long long ends = (long long)first + last;
  const int m = (int)min((long long)n, max((long long)max(__ldcg(keep + b), 0), min((long long)n, ends)));
  const bool bad = n < 0 || n > n_score || m > n_most;
  if (tid == 0 && rank == 0 && seg % h_kv == 0) {
    n_kept[b] = bad ? -1 : m;
    if (bad) atomicOr(err, OPTR_DEVERR_SEQ_LEN);
  }
  if (bad) return;  // the same for the whole cluster
  // positions a0 .. a1-1 are chosen from, k of them stay
  const int a0 = min(first, n), a1 = max(a0, n - min(last, n));
  const int k = m - (n - (a1 - a0));
  const float* row = score + (size_t)seg * n_score;
  int32_t* out = kept + (size_t)seg * n_most;
  const int lo = (int)((long long)n * rank / cs), hi = (int)((long long)n * (rank + 1) / cs);
  // the CTA's keys that are chosen from, and the warp's part of its slice
  const int c0 = max(lo, a0), c1 = max(c0, min(hi, a1));
  auto key_at = [&](int i) { return i - lo < n_keys ? keys[i - lo] : key_of(__ldcg(row + i)); };
  uint32_t T = 0u;
  int ties = 0;      // of the keys equal to T
  const bool choose = k > 0 && k < a1 - a0;
  if (choose) {
#pragma unroll 4
    for (int i = c0 + tid; i < min(c1, lo + n_keys); i += kThreads) keys[i - lo] = key_of(__ldcg(row + i));
    int rest = k;
    uint32_t prefix = 0u;
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass < 2 ? 11 : 10;
      uint32_t* hist = S.hist[pass & 1];
      for (int i = tid; i < kBins; i += kThreads) hist[i] = 0u;
      __syncthreads();
      for (int i0 = c0; i0 < c1; i0 += kThreads) {
        const int i = i0 + tid;
        const uint32_t x = i < c1 ? key_at(i) : 0u;
        const bool in = i < c1 && (pass == 0 || x >> (shift + bits) == prefix);
        const uint32_t digit = x >> shift & ((1u << bits) - 1u);
        // equal scores are common (positions that were never attended to): those that
        // share the first such lane's digit are counted at once
        const unsigned act = __ballot_sync(0xffffffffu, in);
        if (act == 0u) continue;
        const int lead = __ffs(act) - 1;
        const uint32_t d0 = __shfl_sync(0xffffffffu, digit, lead);
        const unsigned same = __ballot_sync(0xffffffffu, in && digit == d0);
        if (lane == lead)
          atomicAdd(&hist[d0], (uint32_t)__popc(same));
        else if (in && digit != d0)
          atomicAdd(&hist[digit], 1u);
      }
      if (cs > 1) cluster_barrier(); else __syncthreads();
      // four bins a thread from the top one down, over the cluster
      const int n_bins = 1 << bits, mine = n_bins / kThreads;  // 4 or 2
      uint32_t c[4] = {0u, 0u, 0u, 0u};
      for (int r = 0; r < cs; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < mine) {
            const uint32_t* x = &hist[n_bins - 1 - (tid * mine + j)];
            c[j] += cs > 1 ? cluster_ld32(x, r) : *x;
          }
      int incl = (int)(c[0] + c[1] + c[2] + c[3]);
      const int own = incl;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      if (lane == 31) S.sum[warp] = incl;
      __syncthreads();
      int before = incl - own;
      for (int i = 0; i < warp; ++i) before += S.sum[i];
      if (before < rest && rest <= before + own) {  // one thread: the digit is among its
        int j = 0;
        while (before + (int)c[j] < rest) before += (int)c[j++];
        S.digit = n_bins - 1 - (tid * mine + j);
        S.rest = rest - before;
      }
      __syncthreads();
      prefix = prefix << bits | (uint32_t)S.digit;
      rest = S.rest;
    }
    T = prefix;
    ties = rest;
  }
  // What lies before each warp's part: kept positions that do not hang on ties, and ties.
  const int w0 = lo + (int)((long long)(hi - lo) * warp / kWarps),
            w1 = lo + (int)((long long)(hi - lo) * (warp + 1) / kWarps);
  auto classify = [&](int i, bool& yes, bool& tie) {
    const bool end = i < w1 && (i < a0 || i >= a1), in = i < w1 && !end;
    yes = end || (in && k > 0 && !choose);
    tie = false;
    if (in && choose) {
      const uint32_t x = key_at(i);
      yes = x > T;
      tie = x == T;
    }
  };
  int above = 0, equal = 0;
  for (int i0 = w0; i0 < w1; i0 += 32) {
    bool yes, tie;
    classify(i0 + lane, yes, tie);
    above += __popc(__ballot_sync(0xffffffffu, yes));
    equal += __popc(__ballot_sync(0xffffffffu, tie));
  }
  if (lane == 0) {
    S.above[warp] = above;
    S.equal[warp] = equal;
  }
  __syncthreads();
  if (tid == 0) {
    int x = 0, y = 0;
    for (int i = 0; i < kWarps; ++i) {
      const int u = S.above[i], v = S.equal[i];
      S.above[i] = x;
      S.equal[i] = y;
      x += u;
      y += v;
    }
    S.count[0] = x;
    S.count[1] = y;
  }
  if (cs > 1) cluster_barrier(); else __syncthreads();
  above = S.above[warp];
  equal = S.equal[warp];
  for (int r = 0; r < rank; ++r) {
    above += (int)cluster_ld32(&S.count[0], r);
    equal += (int)cluster_ld32(&S.count[1], r);
  }
  const unsigned below = (1u << lane) - 1u;
  for (int i0 = w0; i0 < w1; i0 += 32) {
    bool yes, tie;
    classify(i0 + lane, yes, tie);
    const unsigned t = __ballot_sync(0xffffffffu, tie);
    // ties before this one are kept as long as there are any to keep
    const int rank_of = equal + __popc(t & below);
    const bool stays = yes || (tie && rank_of < ties);
    const unsigned s = __ballot_sync(0xffffffffu, stays);
    if (stays) out[above + min(equal, ties) + __popc(s & below)] = i0 + lane;
    const int u = __popc(t);
    above += __popc(s) - (min(equal + u, ties) - min(equal, ties));
    equal += u;
  }
  if (cs > 1) cluster_barrier();  // no CTA leaves while its shared memory may be read
}

}  // namespace
}  // namespace optr

extern "C" optr_status optr_evict_select(const optr_params* p, const float* score, int n_score,
                                         const int32_t* lens, const int32_t* keep, int B, int first,
                                         int last, int32_t* kept, int n_most, int32_t* n_kept,
                                         cudaStream_t stream) {
  using namespace optr;
  if (!p || !score || !lens || !keep || !kept || !n_kept || n_score <= 0 || B <= 0 || n_most <= 0 ||
      first < 0 || last < 0 || !aligned(score, 4))
    return OPTR_ERR_INVALID_ARG;
  const long long rows = (long long)B * p->cfg.h_kv;
  if (rows > (1 << 27) || n_score > (1 << 30)) return OPTR_ERR_OUT_OF_RANGE;
  // CTAs of a row: as few as leave each 4096 scores or fewer, two per SM in all
  int cs = 1;
  while (cs < 8 && n_score > 4096 * cs && rows * 2 * cs <= 2 * p->num_sms) cs *= 2;
  const int n_keys = std::min(kSlice, n_score / cs + 1);
  const size_t smem = sizeof(uint32_t) * (size_t)n_keys;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(select_kernel), smem);
  if (e != cudaSuccess) return OPTR_ERR_CUDA;
  return cuda_status(launch_pdl_cluster(select_kernel, dim3((unsigned)(rows * cs)), dim3(kThreads), cs, smem,
                                        stream, score, n_score, lens, keep, p->cfg.h_kv, first, last, kept,
                                        n_most, n_kept, cs, n_keys, p->err));
}
