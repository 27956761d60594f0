// Verification of drafted tokens against the target's probabilities from
// given random numbers (include/optr.h, "optr_verify_drafts").
//
// Sequence b has n drafts x_0 .. x_{n-1}, a target row p_i after each prefix
// and a draft row q_i for each draft.  Draft i is accepted while
// u_i q_i(x_i) < p_i(x_i); with a drafts accepted the next token is drawn from
//   r = max(p_a - q_a, 0)   (a < n: the first rejected draft's residual)
//   r = p_n                 (a = n: all accepted)
// as argmax_v r(v) / e(v), where e holds independent exponential numbers: the
// smallest of exponential clocks of rates r(v) rings first with probability
// r(v) / sum r, so neither r's sum nor a prefix sum is needed, the rows are
// read once and no rounding of a sum can move the choice.
//
// A cluster of CTAs takes a sequence: each CTA finds a on its own (a few
// dependent loads), then the first maximum of r / e over its slice of the
// vocabulary, and the CTAs' maxima meet in shared memory across the cluster.
// The maximum does not depend on the order in which slices meet, and the
// lowest token wins a tie.  A thread divides only where an approximate quotient
// comes near its warp's largest: dividing everywhere takes 16.9 us where this
// takes 10.0 (16 sequences of 4 drafts, 131072 tokens, float32), and batches
// loaded while others are looked at took it from 32.5 us to 29.2 (128 ragged
// sequences, 100003 tokens; its bytes take 19 at the copy rate).  Bound by
// memory for a serving batch, by the chain of loads (offsets, draft, its
// probabilities, rows: 7 us in all) for one sequence.
#include "optr_internal.cuh"

namespace optr {
namespace {

constexpr int kVerifyThreads = 512;

__device__ __forceinline__ float prob(float x) { return x; }
__device__ __forceinline__ float prob(__nv_bfloat16 x) { return __bfloat162float(x); }

// A candidate as one number: the larger value first, then the lower token
// (values are not negative, so their bits order as they do; the sum makes -0 a
// zero like any other).
__device__ __forceinline__ unsigned long long candidate(float value, int token) {
  return ((unsigned long long)__float_as_uint(__fadd_rn(value, 0.f)) << 32) | (0xFFFFFFFFu - (unsigned)token);
}

__device__ __forceinline__ unsigned long long warp_max(unsigned long long x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned long long y = __shfl_xor_sync(0xffffffffu, x, o);
    if (y > x) x = y;
  }
  return x;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;"
               ::: "memory");
}

__device__ __forceinline__ unsigned long long cluster_load(const unsigned long long* x, int rank) {
  unsigned long long v;
  asm volatile("{\n .reg .u32 r;\n mapa.shared::cluster.u32 r, %1, %2;\n"
               " ld.shared::cluster.u64 %0, [r];\n}\n"
               : "=l"(v)
               : "r"((uint32_t)__cvta_generic_to_shared(x)), "r"(rank)
               : "memory");
  return v;
}

// kVec consecutive probabilities or noise values, as float (the kernel may have
// started while their producer ran: not through the non-coherent path).
template <int kVec>
__device__ __forceinline__ void load_vec(const float* p, float (&x)[kVec]) {
  if constexpr (kVec == 1) {
    x[0] = __ldcg(p);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; i += 4) {
      const float4 y = __ldcg(reinterpret_cast<const float4*>(p + i));
      x[i] = y.x, x[i + 1] = y.y, x[i + 2] = y.z, x[i + 3] = y.w;
    }
  }
}
template <int kVec>
__device__ __forceinline__ void load_vec(const __nv_bfloat16* p, float (&x)[kVec]) {
  if constexpr (kVec == 1) {
    x[0] = __bfloat162float(__ldcg(p));
  } else {
    const uint2 y = __ldcg(reinterpret_cast<const uint2*>(p));
    x[0] = __uint_as_float(y.x << 16), x[1] = __uint_as_float(y.x & 0xffff0000u);
    x[2] = __uint_as_float(y.y << 16), x[3] = __uint_as_float(y.y & 0xffff0000u);
  }
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kVerifyThreads)
verify_kernel(const T* __restrict__ tp, const T* __restrict__ dp,
              const int32_t* __restrict__ drafts, const float* __restrict__ u,
              const float* __restrict__ noise, const int32_t* __restrict__ cu, int n_draft,
              int V, int cs, int32_t* __restrict__ accepted, int32_t* __restrict__ tokens,
              unsigned* err) {
  constexpr int kUnroll = kVec == 1 ? 4 : 1;  // accesses of a batch (wide, 2: 13.6 us for 10.0)
  __shared__ int head[2];
  __shared__ unsigned long long wbest[kVerifyThreads / 32];
  __shared__ unsigned long long best[2];  // this CTA's, by pass
  const int b = blockIdx.x / cs, rank = (int)cluster_rank();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  pdl_trigger();
  // drafts before the first sequence's or after the last one's
  if (blockIdx.x == 0 && tid == 64 && (__ldcg(cu) != 0 || __ldcg(cu + gridDim.x / cs) != n_draft))
    atomicOr(err, OPTR_DEVERR_CU_NEW);
  const int c0 = __ldcg(cu + b), c1 = __ldcg(cu + b + 1);
  if (c0 < 0 || c1 < c0 || c1 > n_draft) {  // the same for the whole cluster
    if (rank == 0 && tid == 0) {
      accepted[b] = -1;
      atomicOr(err, OPTR_DEVERR_CU_NEW);
    }
    return;
  }
  const int n = c1 - c0;
  const float* e = noise + (size_t)b * V;
  const int n_vec = V / kVec;
  const int lo = (int)((long long)n_vec * rank / cs), hi = (int)((long long)n_vec * (rank + 1) / cs);
  // first rejected draft: one lane per draft, 32 at a time
  if (warp == 0) {
    int a = n, x_a = -1;
    for (int i0 = 0; i0 < n; i0 += 32) {
      const int i = i0 + lane;
      bool rej = false;
      int x = 0;
      if (i < n) {
        x = __ldcg(drafts + c0 + i);
        rej = true;
        if (x >= 0 && x < V) {
          const float p = prob(__ldcg(tp + ((size_t)c0 + b + i) * V + x));
          const float q = dp ? prob(__ldcg(dp + ((size_t)c0 + i) * V + x)) : 1.f;
          rej = !(__fmul_rn(__ldcg(u + c0 + i), q) < p);
        }
      }
      const unsigned m = __ballot_sync(0xffffffffu, rej);
      if (m) {
        a = i0 + __ffs(m) - 1;
        x_a = __shfl_sync(0xffffffffu, x, __ffs(m) - 1);
        break;
      }
    }
    if (lane == 0) {
      head[0] = a;
      head[1] = x_a;
    }
  } else if (warp == 1 && rank == 0) {
    // drafts out of range, also those that no acceptance reaches
    for (int i = lane; i < n; i += 32) {
      const int x = __ldcg(drafts + c0 + i);
      if (x < 0 || x >= V) atomicOr(err, OPTR_DEVERR_TOKEN);
    }
  }
  __syncthreads();
  const int a = head[0];
  const T* p = tp + ((size_t)c0 + b + a) * V;
  const T* q = dp && a < n ? dp + ((size_t)c0 + a) * V : nullptr;
  const int cut = !dp && a < n ? head[1] : -1;  // a draft without probabilities: q is 1 there
  // pass 0: the residual.  Where it is zero everywhere (p <= q throughout, to
  // rounding) pass 1 draws from p.
  unsigned long long all = 0;
  for (int pass = 0; pass < 2; ++pass) {
    float top = -1.f;
    int at = 0;
    const bool less = q && pass == 0;
    // two batches in registers: one is loaded while the other is looked at
    float rr[2][kUnroll][kVec], zz[2][kUnroll][kVec], yy[2][kUnroll][kVec];
    auto load = [&](int base, float (&r)[kUnroll][kVec], float (&z)[kUnroll][kVec],
                    float (&y)[kUnroll][kVec]) {
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        const size_t v = (size_t)min(base + tid + j * kVerifyThreads, hi - 1) * kVec;
        load_vec(p + v, r[j]);
        load_vec(e + v, z[j]);
        if (less) load_vec(q + v, y[j]);
      }
    };
    auto look = [&](int base, float (&r)[kUnroll][kVec], float (&z)[kUnroll][kVec],
                    float (&y)[kUnroll][kVec]) {
      const int v0 = base + tid;
      // approximate quotients choose whom to divide: those that may reach the
      // warp's largest so far
      float m = fmaxf(top, 0.f);
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        const int v = v0 + j * kVerifyThreads;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          float x = r[j][i];
          if (less) x = fmaxf(__fsub_rn(x, y[j][i]), 0.f);
          if (pass == 0 && v * kVec + i == cut) x = 0.f;
          r[j][i] = v < hi ? x : -1.f;
          y[j][i] = __fdividef(r[j][i], z[j][i]);
          m = fmaxf(m, y[j][i]);
        }
      }
      m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
      // The approximation is within 2 ulp; divisors past kFar may lie outside its range:
      // divide all there.  (Its documented range begins at 2^-126.  Below, it was within
      // 2 ulp too for every subnormal divisor, each with 256 dividends.)
      constexpr float kFar = 1e30f;
      const float least = m < 1.f / kFar ? 0.f : fminf(m, kFar) * 0.99999f;
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          if (!(y[j][i] < least) || !(z[j][i] < kFar)) {
            const float w = r[j][i] >= 0.f ? __fdiv_rn(r[j][i], z[j][i]) : -1.f;
            if (w > top) {
              top = w;
              at = (v0 + j * kVerifyThreads) * kVec + i;
            }
          }
        }
      }
    };
    constexpr int kBatch = kVerifyThreads * kUnroll;
    if (lo < hi) load(lo, rr[0], zz[0], yy[0]);
    for (int base = lo; base < hi; base += 2 * kBatch) {
      if (base + kBatch < hi) load(base + kBatch, rr[1], zz[1], yy[1]);
      look(base, rr[0], zz[0], yy[0]);
      if (base + 2 * kBatch < hi) load(base + 2 * kBatch, rr[0], zz[0], yy[0]);
      if (base + kBatch < hi) look(base + kBatch, rr[1], zz[1], yy[1]);
    }
    unsigned long long c = warp_max(top >= 0.f ? candidate(top, at) : 0ull);
    if (lane == 0) wbest[warp] = c;
    __syncthreads();
    if (warp == 0) {
      c = warp_max(lane < kVerifyThreads / 32 ? wbest[lane] : 0ull);
      if (lane == 0) best[pass] = c;
    }
    __syncthreads();
    all = best[pass];
    if (cs > 1) {
      cluster_sync();
      for (int r = 0; r < cs; ++r) {
        const unsigned long long y = cluster_load(&best[pass], r);
        if (y > all) all = y;
      }
    }
    if ((uint32_t)(all >> 32) != 0u) break;  // the same in the whole cluster
  }
  if (rank == 0) {
    const int token = (int)(0xFFFFFFFFu - (unsigned)all);
    if (tid == 0) accepted[b] = a;
    for (int i = tid; i <= n; i += kVerifyThreads)
      tokens[(size_t)c0 + b + i] = i < a ? __ldcg(drafts + c0 + i) : i == a ? token : -1;
  }
  if (cs > 1) cluster_sync();  // no CTA leaves while its maximum may be read
}

template <typename T>
cudaError_t launch_verify(const optr_params* p, const void* tp, const void* dp,
                          const int32_t* drafts, const float* u, const float* noise,
                          const int32_t* cu, int n_draft, int B, int V, int32_t* accepted,
                          int32_t* tokens, cudaStream_t s) {
  // four values an access where the vocabulary and the rows' alignment admit it
  // (16 sequences, 131072 tokens: 10.0 us, 11.4 with one value an access)
  const bool wide = V % 4 == 0 && aligned(tp, 4 * sizeof(T)) && aligned(dp, 4 * sizeof(T)) &&
                    aligned(noise, 16);
  // CTAs per sequence: about kPerSm per SM in all, a round of loads each at least
  // (128 ragged sequences: 29.0 us with 2 an SM, 37.8 with 1; with 4, more than fit, 34)
  constexpr int kPerSm = 2;
  int cs = 8;
  while (cs > 1 && ((long long)B * cs > (long long)kPerSm * p->num_sms ||
                    (long long)cs * kVerifyThreads * 8 > 2LL * V))
    cs >>= 1;
  auto fn = wide ? verify_kernel<T, 4> : verify_kernel<T, 1>;
  return launch_pdl_cluster(fn, dim3((unsigned)B * cs), dim3(kVerifyThreads), cs, 0, s,
                            (const T*)tp, (const T*)dp, drafts, u, noise, cu, n_draft, V, cs,
                            accepted, tokens, p->err);
}

}  // namespace
}  // namespace optr

extern "C" optr_status optr_verify_drafts(const optr_params* p, const void* target_probs,
                                          const void* draft_probs, int probs_dtype,
                                          const int32_t* drafts, const float* uniform,
                                          const float* noise, const int32_t* cu_draft,
                                          int n_draft, int B, int vocab, int32_t* accepted,
                                          int32_t* tokens, cudaStream_t stream) {
  using namespace optr;
  if (!p || n_draft < 0 || B <= 0 || vocab <= 0) return OPTR_ERR_INVALID_ARG;
  if (!target_probs || !noise || !cu_draft || !accepted || !tokens ||
      (n_draft > 0 && (!drafts || !uniform)))
    return OPTR_ERR_INVALID_ARG;
  if (probs_dtype != OPTR_PROBS_F32 && probs_dtype != OPTR_PROBS_BF16)
    return OPTR_ERR_UNSUPPORTED;
  const size_t size = probs_dtype == OPTR_PROBS_F32 ? 4 : 2;
  if (!aligned(target_probs, size) || !aligned(draft_probs, size) || !aligned(noise, 4))
    return OPTR_ERR_INVALID_ARG;
  if (B > (1 << 24) || (long long)n_draft + B > 0x7fffffffLL || vocab > (1 << 30))
    return OPTR_ERR_OUT_OF_RANGE;
  auto fn = probs_dtype == OPTR_PROBS_F32 ? launch_verify<float> : launch_verify<__nv_bfloat16>;
  return cuda_status(fn(p, target_probs, draft_probs, drafts, uniform, noise, cu_draft, n_draft, B,
                        vocab, accepted, tokens, stream));
}
