// Eviction, the choice of the positions that stay (include/optr.h,
// "optr_evict_select"): of a row of n scores the k largest, as a rising list.
//
// A cluster of CTAs takes a (sequence, KV head), each CTA a contiguous slice of its
// positions and each warp a contiguous part of that, in registers as 32-bit keys that
// order as the scores do.  Counts of 11, 11 and 10 bits from the top find the k-th
// largest key T: each CTA counts its slice's digits and sums the bins in 64s (32 in the
// last), and after a cluster barrier every warp by itself adds the CTAs' sums up from
// the top, through distributed shared memory, until they reach k, then the bins of
// the sum where they do.  Where a bin stays whole the lower bits need no count (two
// counts do with all but rare scores).  Then all keys above T stay, and of those equal
// to it the lowest positions, as many as are missing: the number of kept positions
// before a warp's part, counted once and summed over warps and CTAs, is all it needs to
// write its own in order.
//
// Bound by a chain: up to three counts by shared atomics, the sums of each behind a barrier of
// the cluster, one more before the list; some 60 instructions a key of 32 lanes over its
// counts and 600 a warp beside fill 39% of the issue slots, and 6.9 MB are read.  64 rows of 20011 ..
// 32768 take 16.4 us, 8 rows of 2049 4.6 us, less than the host needs to call it (7 us).
#include "cluster.cuh"
#include "optr_internal.cuh"

#include <algorithm>

namespace optr {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kSums = 32;  // sums of a CTA's bins

struct Smem {
  alignas(16) uint32_t bins[2048 + 2048 + 1024];  // of the three counts
  uint32_t sums[3][kSums];                        // of 64 (32) bins, by count
  int above[kWarps], equal[kWarps];
  int count[2];  // this CTA's keys above T, and equal to it
};

// Unsigned order = the scores' (-0 as 0, NaN above all), between the keys of no position
// and of one that stays whatever its score.
constexpr uint32_t kNone = 0u, kZero = 0x80000000u, kNan = 0xfffffffeu, kEnd = 0xffffffffu;
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(__fadd_rn(x, 0.f));
  if ((u & 0x7fffffffu) > 0x7f800000u) return kNan;
  return u ^ ((uint32_t)((int32_t)u >> 31) | kZero);
}

// A word of shared memory, over the cluster.
__device__ __forceinline__ uint32_t cluster_sum(const uint32_t* x, int cs) {
  if (cs == 1) return *x;
  uint32_t y[8], sum = 0u;
#pragma unroll
  for (int r = 0; r < 8; ++r) y[r] = r < cs ? cluster_ld32(x, r) : 0u;
#pragma unroll
  for (int r = 0; r < 8; ++r) sum += y[r];
  return sum;
}

// Of counts by lane, from lane 31 down: the lane at which their sum reaches `rest`, which
// loses what lies above it; `own` becomes that lane's count.
__device__ __forceinline__ int reach(uint32_t& own, int& rest) {
  const int lane = threadIdx.x & 31;
  int incl = (int)own;  // of this lane and those above
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_down_sync(0xffffffffu, incl, o);
    if (lane + o < 32) incl += y;
  }
  // (none: only where the scores change under the call)
  const int at = max(0, 31 - __clz((int)__ballot_sync(0xffffffffu, incl >= rest)));
  rest -= __shfl_sync(0xffffffffu, incl - (int)own, at);
  own = __shfl_sync(0xffffffffu, own, at);
  return at;
}

// kPer: keys of a thread, in registers; 0: as many as there are, read from memory each time.
template <int kPer>
__global__ void __launch_bounds__(kThreads, kPer <= 16 ? 2 : 1)
select_kernel(const float* __restrict__ score, int n_score, const int32_t* __restrict__ lens,
              const int32_t* __restrict__ keep, int h_kv, int first, int last,
              int32_t* __restrict__ kept, int n_most, int32_t* __restrict__ n_kept, int log_cs,
              unsigned* err) {
  __shared__ Smem S;
  const int cs = 1 << log_cs, seg = blockIdx.x >> log_cs, rank = cs > 1 ? cluster_rank_of() : 0, b = seg / h_kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  for (int i = tid; i < (int)(sizeof(S.bins) / 16); i += kThreads)
    reinterpret_cast<uint4*>(S.bins)[i] = make_uint4(0u, 0u, 0u, 0u);
  pdl_wait();
  pdl_trigger();
  const int n = __ldcg(lens + b), budget = __ldcg(keep + b);
  const long long ends = (long long)first + last;
  const int m = (int)min((long long)n, max((long long)max(budget, 0), min((long long)n, ends)));
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
  const bool choose = k > 0 && k < a1 - a0;
  // the warp's part w0 .. w1-1 of the CTA's slice
  const int lo = (int)((long long)n * rank >> log_cs), hi = (int)((long long)n * (rank + 1) >> log_cs);
  const int w0 = lo + (int)((long long)(hi - lo) * warp / kWarps),
            w1 = lo + (int)((long long)(hi - lo) * (warp + 1) / kWarps);
  auto key_at = [&](int i) {
    uint32_t x = kZero;
    if (choose && i < w1) x = key_of(__ldcg(row + i));
    return i >= w1 ? kNone : i < a0 || i >= a1 ? kEnd : x;
  };
  uint32_t keys[kPer ? kPer : 1];
#pragma unroll
  for (int j = 0; j < kPer; ++j) keys[j] = key_at(w0 + 32 * j + lane);
  // f(32 positions, the lane's key) for each of the lane's, in order
  auto each = [&](auto f) {
    if constexpr (kPer > 0) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) f(w0 + 32 * j, keys[j]);
    } else {
      for (int i0 = w0; i0 < w1; i0 += 32) f(i0, key_at(i0 + lane));
    }
  };
  uint32_t T = k > 0 ? kNone : kNan;
  int ties = 0;  // of the keys equal to T
  if (choose) {
    __syncthreads();
    int rest = k, zeros = 0;
    uint32_t prefix = 0u;
    for (int pass = 0;; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass < 2 ? 11 : 10;
      uint32_t* bins = S.bins + 2048 * pass;
      // positions that were never attended to are common: their zeros are added at once
      if (pass == 0) {
        each([&](int, uint32_t x) {
          if (x == kZero)
            ++zeros;
          else if (x - 1u < kNan)
            atomicAdd(&bins[x >> 21], 1u);
        });
        zeros = __reduce_add_sync(0xffffffffu, zeros);
      } else if (pass == 1) {
        each([&](int, uint32_t x) {
          if (x >> 21 == prefix && x != kZero && x != kEnd) atomicAdd(&bins[x >> 10 & 0x7ffu], 1u);
        });
      } else {
        each([&](int, uint32_t x) {
          if (x >> 10 == prefix && x != kZero && x != kEnd) atomicAdd(&bins[x & 0x3ffu], 1u);
        });
      }
      if (lane == 0 && zeros > 0 && (pass == 0 || kZero >> (shift + bits) == prefix))
        atomicAdd(&bins[kZero >> shift & ((1u << bits) - 1u)], (uint32_t)zeros);
      __syncthreads();
      const int size = (1 << bits) / kSums;  // bins of a sum: 64, or 32
      {  // sums 2 warp and 2 warp + 1
        const uint2 x = reinterpret_cast<const uint2*>(bins + size * (2 * warp + (lane >> 4)))[lane & 15];
        uint32_t sum = x.x + x.y;
        if (size == 64) {
          const uint2 y = reinterpret_cast<const uint2*>(bins + size * (2 * warp + (lane >> 4)) + 32)[lane & 15];
          sum += y.x + y.y;
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if ((lane & 15) == 0) S.sums[pass][2 * warp + (lane >> 4)] = sum;
      }
      if (cs > 1) cluster_barrier(); else __syncthreads();
      uint32_t own = cluster_sum(&S.sums[pass][lane], cs);
      int digit = size * reach(own, rest);
      if (size == 64) {
        uint32_t low = cluster_sum(&bins[digit + lane], cs), high = cluster_sum(&bins[digit + 32 + lane], cs);
        const int upper = (int)__reduce_add_sync(0xffffffffu, high);
        if (upper >= rest) {
          digit += 32;
          own = high;
        } else {
          rest -= upper;
          own = low;
        }
      } else {
        own = cluster_sum(&bins[digit + lane], cs);
      }
      digit += reach(own, rest);
      prefix = prefix << bits | (uint32_t)digit;
      const bool whole = (int)own == rest;
      if (pass == 2 || whole) {
        T = prefix << shift;
        ties = rest;
        if (whole && shift > 0) {  // all keys from T on stay (T > 0: a number's key is)
          T -= 1u;
          ties = 0;
        }
        break;
      }
    }
  }
  // What lies before each warp's part: kept positions that do not hang on ties, and ties.
  int above = 0, equal = 0;
  each([&](int, uint32_t x) {
    above += x > T;
    equal += x == T;
  });
  above = __reduce_add_sync(0xffffffffu, above);
  equal = ties > 0 ? __reduce_add_sync(0xffffffffu, equal) : 0;
  const int mine = equal;
  if (lane == 0) {
    S.above[warp] = above;
    S.equal[warp] = equal;
  }
  __syncthreads();
  // (each warp sums up by itself)
  int x = lane < kWarps ? S.above[lane] : 0, y = lane < kWarps ? S.equal[lane] : 0;
  if (cs > 1) {
    if (warp == 0) {
      const int u = __reduce_add_sync(0xffffffffu, x), v = __reduce_add_sync(0xffffffffu, y);
      if (lane == 0) S.count[0] = u, S.count[1] = v;
    }
    cluster_barrier();
  }
  if (lane >= warp) x = y = 0;
  above = __reduce_add_sync(0xffffffffu, x);
  equal = __reduce_add_sync(0xffffffffu, y);
  if (cs > 1) {
    int u = lane < rank ? (int)cluster_ld32(&S.count[0], lane) : 0;
    int v = lane < rank ? (int)cluster_ld32(&S.count[1], lane) : 0;
    above += __reduce_add_sync(0xffffffffu, u);
    equal += __reduce_add_sync(0xffffffffu, v);
    cluster_arrive();  // no CTA leaves while its shared memory may be read
  }
  const unsigned below = (1u << lane) - 1u;
  if (mine == 0) {
    above += min(equal, ties);
    each([&](int i, uint32_t x) {
      const unsigned s = __ballot_sync(0xffffffffu, x > T);
      if (x > T) out[above + __popc(s & below)] = i + lane;
      above += __popc(s);
    });
  } else {
    each([&](int i, uint32_t x) {
      const unsigned t = __ballot_sync(0xffffffffu, x == T);
      // ties before this one are kept as long as there are any to keep
      const bool stays = x > T || (x == T && equal + __popc(t & below) < ties);
      const unsigned s = __ballot_sync(0xffffffffu, stays);
      if (stays) out[above + min(equal, ties) + __popc(s & below)] = i + lane;
      const int u = __popc(t);
      above += __popc(s) - (min(equal + u, ties) - min(equal, ties));
      equal += u;
    });
  }
  if (cs > 1) cluster_wait();
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
  // CTAs of a row: as few as leave each 4096 scores or fewer, one per SM in all (16 x 8 rows of
  // 8192: one CTA each 8.6 us, two 12.4), and as many as are resident at once (64 rows of 32768
  // in clusters of 8: 35 us, of 2 16.4)
  int log_cs = 0;
  while (log_cs < 3 && n_score > 4096 << log_cs &&
         (rows << (log_cs + 1)) <= (log_cs < 2 ? p->num_sms : p->num_sms * 3 / 4))
    ++log_cs;
  const int cs = 1 << log_cs;
  const int per = (n_score - 1) / (cs * kThreads) + 1;
  auto fn = per <= 8    ? select_kernel<8>
            : per <= 16 ? select_kernel<16>
            : per <= 32 ? select_kernel<32>
            : per <= 64 ? select_kernel<64>
                        : select_kernel<0>;
  return cuda_status(launch_pdl_cluster(fn, dim3((unsigned)(rows * cs)), dim3(kThreads), cs, 0, stream, score,
                                        n_score, lens, keep, p->cfg.h_kv, first, last, kept, n_most, n_kept, log_cs,
                                        p->err));
}
