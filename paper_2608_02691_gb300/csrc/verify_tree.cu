// Verification of a tree of drafted tokens against the target's probabilities
// from given random numbers (include/optr.h, "optr_verify_tree").
//
// From the root on, at row r with the children c_1 < c_2 < .. whose tokens were
// drawn independently from q_r: with w = p_r and S = 1, child c of token x is
// accepted if u_c q_r(x) S < w(x), that is with probability min(1, (w(x) / S) / q_r(x));
// if it is rejected, w becomes max(w - S q_r, 0) and S its sum, so that w / S is the
// residual that the next child is measured against and, after the last one, the
// next token is drawn from (as argmax w / e, see verify.cu).  By induction over the
// children the token that is kept has the distribution p_r.  Without probabilities
// q_r is 1 at each child's token: its w becomes 0, S loses w(x).
//
// A cluster of CTAs takes a sequence.  Every row's p, q, u at its own token are
// loaded at once into shared memory; each CTA walks down the tree by itself (one
// warp, in shared memory) until a sum S or the final draw needs the vocabulary.  Of
// that each CTA has a slice; w is not stored but computed from p, q and the S so
// far, and the warps' sums meet in shared memory across the cluster, in a fixed order
// (equal calls give equal bits).
//
// Bound by latency: offsets, tree, probabilities of the drafts, then a round of loads for
// each sum and for the draw, one cluster barrier each.  16 x 24 rows of 131072 take 20 to
// 28 us with the tree (the deepest way and the sums on it decide; of 26 on one, cold: 9 until
// the first row, 3.5 a sum without its loads), 1 x 8 of 32000 7.6 us.
#include "cluster.cuh"
#include "optr_internal.cuh"

namespace optr {
namespace {

constexpr int kTreeThreads = 512, kWarps = kTreeThreads / 32;
constexpr int kRows = OPTR_TREE_MAX_ROWS;
constexpr int kTerms = 256;  // probabilities of a float32 sum: 2^-16 of it at the very worst

struct Node {
  int parent, token;  // parent -2: never reached
  float px, qx, u;    // of its token: target and draft probability at the parent's row
};

struct Walk {
  int row;    // the last accepted row
  int last;   // children up to this row were rejected
  int n_cut;  // rejected children of `row`: their S (probabilities) or tokens in `cut`
  int depth;  // accepted rows after the root
  bool draw;  // no child is left
};

struct Smem {
  Node node[kRows];
  uint32_t cut[kRows];
  int16_t path[kRows];
  Walk walk;
  double sum[2][kWarps];                 // the warps' sums, by pass,
  unsigned long long best[2][kWarps];    // and their largest ratios
  unsigned long long all;
};

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// N consecutive values, past the caches that a kernel before may have left stale.
template <int N>
__device__ __forceinline__ void fetch(const float* p, float (&x)[N]) {
  if constexpr (N == 4) {
    const float4 y = __ldcg(reinterpret_cast<const float4*>(p));
    x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
  } else {
    x[0] = __ldcg(p);
  }
}
template <int N>
__device__ __forceinline__ void fetch(const __nv_bfloat16* p, float (&x)[N]) {
  if constexpr (N == 4) {
    const uint2 y = __ldcg(reinterpret_cast<const uint2*>(p));
    x[0] = __uint_as_float(y.x << 16), x[1] = __uint_as_float(y.x & 0xffff0000u);
    x[2] = __uint_as_float(y.y << 16), x[3] = __uint_as_float(y.y & 0xffff0000u);
  } else {
    x[0] = as_float(__ldcg(p));
  }
}

// What a rejection by probabilities leaves.
__device__ __forceinline__ float left(float w, float S, float q) {
  return fmaxf(__fsub_rn(w, __fmul_rn(S, q)), 0.f);
}

// Larger value first, then the lower token (values are not negative, -0 is a zero).
__device__ __forceinline__ unsigned long long ranked(float value, int token) {
  return (unsigned long long)__float_as_uint(__fadd_rn(value, 0.f)) << 32 | (0xffffffffu - (unsigned)token);
}

// One warp: the 16 words of each CTA of the cluster (8 at most), four a lane; the lanes of
// CTAs that there are not get `none`.
__device__ __forceinline__ void cluster_words(const void* x, int cs, unsigned long long none,
                                              unsigned long long (&y)[4]) {
  static_assert(kWarps == 16, "four words a lane, four lanes a CTA");
  const int lane = threadIdx.x & 31, rank = lane >> 2;
  const unsigned long long* at = static_cast<const unsigned long long*>(x) + 4 * (lane & 3);
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = rank < cs ? (cs > 1 ? cluster_ld64(at + i, rank) : at[i]) : none;
}

// x / e where it may pass the largest ratio so far.  Most cannot: the reciprocal's estimate
// says so (to 2^-20; estimates near nothing and what is not a number say nothing).
struct Largest {
  float top = -1.f, limit = -1.f;
  int at = 0;
  __device__ __forceinline__ void take(float x, float e, int token) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e));
    const float guess = x * r;
    if (guess < limit && (guess > 1e-30f || x == 0.f)) return;
    const float exact = __fdiv_rn(x, e);
    if (exact > top) {
      top = exact;
      limit = exact * 0.999999f;
      at = token;
    }
  }
};

// One warp: down from S.walk until a sum or the draw is needed.
__device__ __forceinline__ void descend(Smem& S, int n, bool probs) {
  const int lane = threadIdx.x & 31;
  Walk w = S.walk;
  float mass = 1.f;
  if (w.n_cut > 0 && probs) mass = __uint_as_float(S.cut[w.n_cut]);
  // w(x) of a child, from the masses of the rejected ones before it
  for (;;) {
    int child = n;
    for (int i0 = (w.last + 1) & ~31; i0 < n && child == n; i0 += 32) {
      const int i = i0 + lane;
      const unsigned m = __ballot_sync(0xffffffffu, i > w.last && i < n && S.node[i].parent == w.row);
      if (m) child = i0 + __ffs(m) - 1;
    }
    if (child == n) {
      w.draw = true;
      break;
    }
    const Node c = S.node[child];
    float x = c.px;
    bool known = true;  // whether S is
    if (probs) {
      for (int j = 0; j < w.n_cut; ++j) x = left(x, __uint_as_float(S.cut[j]), c.qx);
      known = !(mass < 0.f);
    } else {
      for (int j = 0; j < w.n_cut; ++j)
        if ((int)S.cut[j] == c.token) x = 0.f;
    }
    if (!known) break;  // (the mass of what is left comes first)
    if (__fmul_rn(__fmul_rn(c.u, c.qx), mass) < x) {
      w.row = w.last = child;
      w.n_cut = 0;
      mass = 1.f;
      ++w.depth;
      if (lane == 0) S.path[w.depth] = (int16_t)child;
      continue;
    }
    w.last = child;
    if (c.token < 0) continue;  // a draft out of range takes nothing from the target
    if (lane == 0) S.cut[w.n_cut] = probs ? __float_as_uint(mass) : (uint32_t)c.token;
    ++w.n_cut;
    mass = probs ? -1.f : __fsub_rn(mass, x);
    __syncwarp();
  }
  if (lane == 0) S.walk = w;
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kTreeThreads)
verify_tree_kernel(const T* __restrict__ tp, const T* __restrict__ dp,
                   const int32_t* __restrict__ tokens, const int32_t* __restrict__ parent,
                   const float* __restrict__ uniform, const float* __restrict__ noise,
                   const int32_t* __restrict__ cu, int n_tok, int V, int cs,
                   int32_t* __restrict__ accepted, int32_t* __restrict__ path,
                   int32_t* __restrict__ next, unsigned* err) {
  __shared__ Smem S;
  const int b = blockIdx.x / cs, rank = cluster_rank_of();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && tid == 64 && (__ldcg(cu) != 0 || __ldcg(cu + gridDim.x / cs) != n_tok))
    atomicOr(err, OPTR_DEVERR_CU_NEW);
  const int c0 = __ldcg(cu + b), c1 = __ldcg(cu + b + 1), n = c1 - c0;
  const bool bad = c0 < 0 || c1 < c0 || c1 > n_tok || n > kRows;
  if (bad || n == 0) {  // the same for the whole cluster
    if (rank == 0 && tid == 0) {
      accepted[b] = -1;
      if (bad) atomicOr(err, OPTR_DEVERR_CU_NEW);
    }
    return;
  }
  for (int i = tid; i < n; i += kTreeThreads) {
    Node x;
    x.parent = __ldcg(parent + c0 + i);
    x.token = __ldcg(tokens + c0 + i);
    x.u = __ldcg(uniform + c0 + i);
    x.px = x.qx = 0.f;
    unsigned flag = 0;
    if (i == 0 ? x.parent != -1 : x.parent < 0 || x.parent >= i) {
      flag |= OPTR_DEVERR_TREE;
      x.parent = -2;
    }
    if (i > 0) {
      if (x.token < 0 || x.token >= V) {
        flag |= OPTR_DEVERR_TOKEN;
        x.token = -1;
      } else if (x.parent >= 0) {
        const size_t at = ((size_t)c0 + x.parent) * V + x.token;
        x.px = as_float(__ldcg(tp + at));
        x.qx = dp ? as_float(__ldcg(dp + at)) : 1.f;
      }
    }
    S.node[i] = x;
    if (flag && rank == 0) atomicOr(err, flag);
  }
  if (tid == 0) {
    S.walk = Walk{0, 0, 0, 0, false};
    S.path[0] = 0;
  }
  const int n_vec = V / kVec;
  const int lo = (int)((long long)n_vec * rank / cs), hi = (int)((long long)n_vec * (rank + 1) / cs);
  const float* e = noise + (size_t)b * V;
  // the noise is wanted in any case: it comes into L2 while the walk goes on
  for (int v = lo + (128 / (4 * kVec)) * tid; v < hi; v += (128 / (4 * kVec)) * kTreeThreads)
    asm volatile("prefetch.global.L2 [%0];" ::"l"(e + (size_t)v * kVec));
  __syncthreads();
  if (warp == 0) descend(S, n, dp != nullptr);
  __syncthreads();
  // Sums until the walk ends
  Walk w;
  for (int pass = 0;; ++pass) {
    w = S.walk;
    if (w.draw) break;
    const T* p = tp + ((size_t)c0 + w.row) * V;
    const T* q = dp + ((size_t)c0 + w.row) * V;
    double total = 0.0;
    for (int v = lo + tid; v < hi;) {
      float sum = 0.f;
      const int end = min(hi, v + kTerms / kVec * kTreeThreads);
#pragma unroll 4
      for (; v < end; v += kTreeThreads) {
        float x[kVec], y[kVec];
        fetch(p + (size_t)v * kVec, x);
        fetch(q + (size_t)v * kVec, y);
        for (int j = 0; j < w.n_cut; ++j) {
          const float m = __uint_as_float(S.cut[j]);
#pragma unroll
          for (int i = 0; i < kVec; ++i) x[i] = left(x[i], m, y[i]);
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum += x[i];
      }
      total += sum;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    if (lane == 0) S.sum[pass & 1][warp] = total;
    if (cs > 1) cluster_barrier(); else __syncthreads();
    if (warp == 0) {
      unsigned long long y[4];
      cluster_words(S.sum[pass & 1], cs, 0ull, y);
      total = (__longlong_as_double((long long)y[0]) + __longlong_as_double((long long)y[1])) +
              (__longlong_as_double((long long)y[2]) + __longlong_as_double((long long)y[3]));
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
      // (the mass that the next child is measured against, where descend() looks for it)
      if (lane == 0) S.cut[w.n_cut] = __float_as_uint((float)total);
      __syncwarp();
      descend(S, n, true);
    }
    __syncthreads();
  }
  // The next token: first maximum of w / e; of p / e where w is zero everywhere
  const T* p = tp + ((size_t)c0 + w.row) * V;
  const T* q = dp ? dp + ((size_t)c0 + w.row) * V : nullptr;
  unsigned long long all = 0;
  for (int pass = 0; pass < 2; ++pass) {
    const int n_cut = pass == 0 ? w.n_cut : 0;
    Largest best;
#pragma unroll 4
    for (int v = lo + tid; v < hi; v += kTreeThreads) {
      float x[kVec], z[kVec], y[kVec];
      fetch(p + (size_t)v * kVec, x);
      fetch(e + (size_t)v * kVec, z);
      if (q && n_cut > 0) fetch(q + (size_t)v * kVec, y);
      for (int j = 0; j < n_cut; ++j) {
        const uint32_t cut = S.cut[j];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          if (q)
            x[i] = left(x[i], __uint_as_float(cut), y[i]);
          else if ((int)cut == v * kVec + i)
            x[i] = 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) best.take(x[i], z[i], v * kVec + i);
    }
    unsigned long long c = best.top >= 0.f ? ranked(best.top, best.at) : 0ull;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long y = __shfl_xor_sync(0xffffffffu, c, o);
      c = y > c ? y : c;
    }
    if (lane == 0) S.best[pass][warp] = c;
    if (cs > 1) cluster_barrier(); else __syncthreads();
    if (warp == 0) {
      unsigned long long y[4];
      cluster_words(S.best[pass], cs, 0ull, y);
#pragma unroll
      for (int i = 1; i < 4; ++i) y[0] = y[i] > y[0] ? y[i] : y[0];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long z = __shfl_xor_sync(0xffffffffu, y[0], o);
        y[0] = z > y[0] ? z : y[0];
      }
      if (lane == 0) S.all = y[0];
    }
    __syncthreads();
    all = S.all;
    if ((uint32_t)(all >> 32) != 0u) break;  // the same in the whole cluster
  }
  if (cs > 1) cluster_arrive();  // no CTA leaves while its shared memory may be read
  if (rank == 0) {
    const int token = (int)(0xffffffffu - (unsigned)all);
    if (tid == 0) accepted[b] = w.depth;
    for (int i = tid; i < n; i += kTreeThreads) {
      path[c0 + i] = i <= w.depth ? c0 + S.path[i] : -1;
      next[c0 + i] = i < w.depth ? S.node[S.path[i + 1]].token : i == w.depth ? token : -1;
    }
  }
  if (cs > 1) cluster_wait();
}

template <typename T>
cudaError_t launch_verify_tree(const optr_params* p, const void* tp, const void* dp,
                               const int32_t* tokens, const int32_t* parent, const float* u,
                               const float* noise, const int32_t* cu, int n_tok, int B, int V,
                               int32_t* accepted, int32_t* path, int32_t* next, cudaStream_t s) {
  // four values an access where the vocabulary and the rows' alignment admit it
  const bool wide = V % 4 == 0 && aligned(tp, 4 * sizeof(T)) && aligned(dp, 4 * sizeof(T)) &&
                    aligned(noise, 16);
  // CTAs per sequence: about two per SM in all, a round of loads each at least
  int cs = 8;
  while (cs > 1 && ((long long)B * cs > 2LL * p->num_sms || (long long)cs * kTreeThreads * 8 > 2LL * V))
    cs >>= 1;
  auto fn = wide ? verify_tree_kernel<T, 4> : verify_tree_kernel<T, 1>;
  return launch_pdl_cluster(fn, dim3((unsigned)B * cs), dim3(kTreeThreads), cs, 0, s, (const T*)tp,
                            (const T*)dp, tokens, parent, u, noise, cu, n_tok, V, cs, accepted, path,
                            next, p->err);
}

}  // namespace
}  // namespace optr

extern "C" optr_status optr_verify_tree(const optr_params* p, const void* target_probs,
                                        const void* draft_probs, int probs_dtype,
                                        const int32_t* tokens, const int32_t* parent,
                                        const float* uniform, const float* noise,
                                        const int32_t* cu_tree, int n_tok, int B, int vocab,
                                        int32_t* accepted, int32_t* path, int32_t* next,
                                        cudaStream_t stream) {
  using namespace optr;
  if (!p || n_tok < 0 || B <= 0 || vocab <= 0) return OPTR_ERR_INVALID_ARG;
  if (!cu_tree || !accepted || !noise ||
      (n_tok > 0 && (!target_probs || !tokens || !parent || !uniform || !path || !next)))
    return OPTR_ERR_INVALID_ARG;
  if (probs_dtype != OPTR_PROBS_F32 && probs_dtype != OPTR_PROBS_BF16) return OPTR_ERR_UNSUPPORTED;
  const size_t size = probs_dtype == OPTR_PROBS_F32 ? 4 : 2;
  if (!aligned(target_probs, size) || !aligned(draft_probs, size) || !aligned(noise, 4))
    return OPTR_ERR_INVALID_ARG;
  if (B > (1 << 24) || vocab > (1 << 30)) return OPTR_ERR_OUT_OF_RANGE;
  auto fn = probs_dtype == OPTR_PROBS_F32 ? launch_verify_tree<float> : launch_verify_tree<__nv_bfloat16>;
  return cuda_status(fn(p, target_probs, draft_probs, tokens, parent, uniform, noise, cu_tree, n_tok, B,
                        vocab, accepted, path, next, stream));
}
