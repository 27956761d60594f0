// Attention weights of a decode step's few tokens, summed by position ("optr_kv_score").
//
// With one to kFewTok tokens a (sequence, KV head) the keys are read once: their logits, 16
// bytes a token and position, are kept for the second pass.  few_cluster_kernel does
// all in one launch: a cluster of CTAs takes a (sequence, KV head), each CTA a range of
// its pages and window rows; it rotates the queries (as the decode does), keeps the
// logits in shared memory (in the workspace where they do not fit), and maxima and sums
// meet across the cluster.  16 x 1 over 8192: 29.5 us, 1.7 TB/s; of that some 9 us are the
// products and what brings the codes to them, 7 us the rest of the page loop, 8 us the weights
// and 6 us the launch and the rotation, and 24 of 152 SMs have no (sequence, KV head).  One
// token over 1024: 8.8 us, the host's time of a call.
//
// Long contexts of so few or so many (sequence, KV head)s that many SMs would idle take three
// launches instead (clusters()): few_query_kernel, few_logit_kernel, in which all steps of
// all (sequence, KV head)s stand in one line that is cut into equal ranges, one a warp, and
// few_sum_kernel, which joins the warps' maxima and sums and adds the weights up.
//
// A page's logits are the decode's (decode_tc.cu): m16n8k16 products of the codes, as the
// fp16 numbers 1024 + code 2^pos that their bits make, with the four query heads in fp16
// hi and lo parts (eight columns), one accumulator a scale.  Window keys are bf16 as they
// are, 16 rows a step, which counts as four pages in the line.
#include <type_traits>

#include "cluster.cuh"
#include "qrot.cuh"
#include "score.cuh"

#include <algorithm>

namespace optr {
namespace {

constexpr int kWarps = 16;
constexpr int kStages = 6;         // pages on the way to a warp, in pairs
constexpr int kHalfRec = 768;      // a page's key codes and pairs
constexpr int kWinCost = 4;
constexpr int kWinRows = 16;
// words of a token's query: fragments, offsets, inverse prescales, sums, <q, mu>
constexpr int kFrag = 0, kOff = 512, kInv = 544, kSum = 548, kMu = 564, kQueryWords = 576;

struct Steps {
  __device__ __forceinline__ static int pages(int n_int) { return (n_int + kPage - 1) / kPage; }
  __device__ __forceinline__ static int of(const ScoreSeq& s) {
    return pages(s.n_int) + kWinCost * ((s.n_win + kWinRows - 1) / kWinRows);
  }
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Workspace of the three launches: queries [segments][max_new][kQueryWords], partials [W + segments][16]
// {maximum, sum}, logits [segments][positions][max_new][4].
struct FewArgs {
  ScoreArgs A;
  uint32_t* query;
  float2* part;
  float4* logits;
  int positions, W;
  float qscale;
};
__device__ __forceinline__ uint32_t* few_query(const FewArgs& F, int seg, int i) {
  return F.query + ((size_t)seg * F.A.max_new + i) * kQueryWords;
}

__global__ void __launch_bounds__(kQrotThreads) few_query_kernel(const __grid_constant__ FewArgs F) {
  __shared__ QrotSmem sm;
  const ScoreArgs& A = F.A;
  const int seg = blockIdx.x, b = seg / A.h_kv, h = seg % A.h_kv, tid = threadIdx.x;
  float rv[32];
  load_rotation_slice(A.R_k, h, rv);
  pdl_wait();
  pdl_trigger();
  if (seg == 0 && tid < 32) report_sequences(A);
  const ScoreSeq s = score_seq(A, b);
  if (Steps::of(s) == 0) return;
  for (int i = 0; i < s.rows; ++i) {
    const __nv_bfloat16* q = A.q + (((size_t)s.c0 + i) * A.h_kv + h) * (4 * kD);
    uint32_t* out = few_query(F, seg, i);
    rotate_query(sm, q, rv, F.qscale, nullptr, reinterpret_cast<float*>(out + kSum), out + kFrag,
                 reinterpret_cast<float*>(out + kOff), reinterpret_cast<float*>(out + kInv));
    if (A.win.win && tid < 128) {  // head tid / 32
      float d = 0.f;
      for (int k = tid & 31; k < kD; k += 32)
        d = fmaf(__bfloat162float(q[(tid >> 5) * kD + k]), __ldg(A.mu + (size_t)h * kD + k), d);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
      if ((tid & 31) == 0) reinterpret_cast<float*>(out + kMu)[tid >> 5] = d * F.qscale;
    }
    __syncthreads();
  }
}

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// d = a b + c
__device__ __forceinline__ void mma_f16_from(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                             uint32_t b0, uint32_t b1, const float (&c)[4]) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%10,%11,%12,%13};\n"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int pos>
__device__ __forceinline__ uint32_t field(uint32_t x) {  // 1024 + code 2^pos of either half
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(y) : "r"(x), "n"(0x00030003u << pos), "r"(0x64006400u));
  return y;
}
// The codes of a word whose halves hold a byte of group 2 j (low) and 2 j + 1 (high), as A
// registers by group parity (code_pos says where each stands).
__device__ __forceinline__ void fields(uint32_t y, uint32_t (&out)[2][4]) {
  const uint32_t l = y << 4, r = y >> 6;
  out[0][0] = field<code_pos(0, 0)>(l);
  out[0][1] = field<code_pos(0, 1)>(l);
  out[0][2] = field<code_pos(0, 2)>(y);
  out[0][3] = field<code_pos(0, 3)>(y);
  out[1][0] = field<code_pos(1, 0)>(y);
  out[1][1] = field<code_pos(1, 1)>(r);
  out[1][2] = field<code_pos(1, 2)>(r);
  out[1][3] = field<code_pos(1, 3)>(r);
}

__device__ __forceinline__ float low_half(uint32_t x) {
  return __low2float(*reinterpret_cast<const __half2*>(&x));
}

// A token's query in shared memory: by group the lanes' fragments, then as in the
// workspace, with the min terms' fragment ready.
struct FewQuery {
  uint4 frag[kGroups][32];
  float off[32];
  uint32_t min[32];
  float inv[4], mu[4];
};

// A token's query as a lane has it: B fragments of its column, what the products start
// from, the min terms' B fragment, and the inverse prescale of head lane % 4.
template <bool kCompact>
struct Query {
  uint4 frag[kGroups];
  float start[kGroups][4];
  uint32_t min;
  float inv;

  __device__ __forceinline__ void load(const uint32_t* w) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int G = 0; G < kGroups; ++G)
      frag[G] = __ldcg(reinterpret_cast<const uint4*>(w + kFrag + lane * 16) + G);
    const float4* o = reinterpret_cast<const float4*>(w + kOff + c * 8);
    const float4 a = __ldcg(o), b = __ldcg(o + 1);
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int G = 0; G < kGroups; ++G) start[G][0] = start[G][2] = -x[2 * G], start[G][1] = start[G][3] = -x[2 * G + 1];
    // column g of the min terms' product: head g / 2, hi or lo part of group c's sum
    const float s = __uint_as_float(__ldcg(w + kSum + (g >> 1) * kGroups + c));
    const float hi = __uint_as_float(__float_as_uint(s) & 0xffffe000u);
    const uint32_t part = __half_as_ushort(__float2half_rn(g & 1 ? s - hi : hi));
    min = part << 16;
    inv = __uint_as_float(__ldcg(w + kInv + c));
  }
  // of shared memory
  __device__ __forceinline__ void load(const FewQuery& w) {
    const int lane = threadIdx.x & 31, c = lane & 3;
    const float4 *o = reinterpret_cast<const float4*>(w.off + c * 8), a = o[0], b = o[1];
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int G = 0; G < kGroups; ++G) {
      frag[G] = w.frag[G][lane];
      start[G][0] = start[G][2] = -x[2 * G], start[G][1] = start[G][3] = -x[2 * G + 1];
    }
    min = w.min[lane];
    inv = w.inv[c];
  }
};

// A page's codes and pairs as a lane has them: tokens g and g + 8.
template <bool kCompact>
struct Page {
  uint32_t f[2][2][2][4];  // [row][groups 2 j ..][parity][code]
  uint32_t w0, w1;         // the min terms' A registers
  uint4 m0, m1;            // four groups' pairs (the compact record: w0, w1 are the ones)

  __device__ __forceinline__ void load(const uint8_t* st) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const uint2 k0 = *reinterpret_cast<const uint2*>(st + g * 32 + 8 * c);
    const uint2 k1 = *reinterpret_cast<const uint2*>(st + (g + 8) * 32 + 8 * c);
    fields(__byte_perm(k0.x, k0.y, 0x5410), f[0][0]);
    fields(__byte_perm(k0.x, k0.y, 0x7632), f[0][1]);
    fields(__byte_perm(k1.x, k1.y, 0x5410), f[1][0]);
    fields(__byte_perm(k1.x, k1.y, 0x7632), f[1][1]);
    constexpr int ms = meta_stride(kCompact);
    w0 = *reinterpret_cast<const uint32_t*>(st + 512 + g * ms + (kCompact ? 0 : 4 * c));
    w1 = *reinterpret_cast<const uint32_t*>(st + 512 + (g + 8) * ms + (kCompact ? 0 : 4 * c));
    if constexpr (!kCompact) {
      m0 = *reinterpret_cast<const uint4*>(st + 512 + g * ms);
      m1 = *reinterpret_cast<const uint4*>(st + 512 + (g + 8) * ms);
    }
  }

  // logits of tokens g, g + 8, head c
  __device__ __forceinline__ float2 logits(const Query<kCompact>& q) const {
    // an accumulator a group, the compact record's too: in one for all, which starts from
    // four offsets, a logit is off ten times as far
    float s[kGroups][4];
#pragma unroll
    for (int G = 0; G < kGroups; ++G) {
      const uint32_t (&a)[4] = f[0][G >> 1][G & 1];
      const uint32_t (&b)[4] = f[1][G >> 1][G & 1];
      mma_f16_from(s[G], a[0], b[0], a[1], b[1], q.frag[G].x, q.frag[G].y, q.start[G]);
      mma_f16(s[G], a[2], b[2], a[3], b[3], q.frag[G].z, q.frag[G].w);
    }
    float u[4] = {0.f, 0.f, 0.f, 0.f}, t0, t1;
    mma_f16(u, w0, w1, 0u, 0u, q.min, 0u);
    if constexpr (kCompact) {
      t0 = t1 = 0.f;
#pragma unroll
      for (int G = 0; G < kGroups; ++G) {
        t0 += s[G][0] + s[G][1];
        t1 += s[G][2] + s[G][3];
      }
      t0 *= low_half(w0);
      t1 *= low_half(w1);
    } else {
      const uint32_t x[4] = {m0.x, m0.y, m0.z, m0.w}, y[4] = {m1.x, m1.y, m1.z, m1.w};
      t0 = t1 = 0.f;
#pragma unroll
      for (int G = 0; G < kGroups; ++G) {
        t0 = fmaf(low_half(x[G]), s[G][0] + s[G][1], t0);
        t1 = fmaf(low_half(y[G]), s[G][2] + s[G][3], t1);
      }
    }
    return make_float2(fmaf(q.inv, t0, u[0] + u[1]), fmaf(q.inv, t1, u[2] + u[3]));
  }
};

// Products of 16 window rows' keys (rows g and g + 8, channels 32 e + 8 c ..) with the four
// heads of a query (lanes whose column is a head's: `has`), head c of rows g and g + 8.
__device__ __forceinline__ float2 window_logits(const uint4 (&a)[4], const uint4 (&b)[4], const __nv_bfloat16* qr,
                                                bool has) {
  // (a sum of its own for each step, since a product rounds at its largest term: the
  // key mean may make one channel's far larger than the logit)
  float d0 = 0.f, d1 = 0.f;
  // column g: head g / 2 of the even ones, nothing of the odd ones; the places of
  // the inner dimension are permuted alike in both operands
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (has) x = __ldcg(reinterpret_cast<const uint4*>(qr + 32 * s));
    float d[4] = {0.f, 0.f, 0.f, 0.f}, e[4] = {0.f, 0.f, 0.f, 0.f};
    mma_bf16(d, a[s].x, b[s].x, a[s].y, b[s].y, x.x, x.y);
    mma_bf16(e, a[s].z, b[s].z, a[s].w, b[s].w, x.z, x.w);
    d0 += d[0] + e[0];
    d1 += d[2] + e[2];
  }
  return make_float2(d0, d1);
}

template <bool kCompact, int kTokens>
__global__ void __launch_bounds__(kWarps * 32, 1) few_logit_kernel(const __grid_constant__ FewArgs F) {
  extern __shared__ __align__(16) unsigned char dsm_[];
  const ScoreArgs& A = F.A;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  uint8_t* stage = dsm_ + (size_t)warp * kStages * kHalfRec;
  const int w = warp * gridDim.x + blockIdx.x;  // neighbours' ranges on different SMs
  pdl_wait();
  pdl_trigger();
  ScoreFinder<Steps> next;
  next.start(A, w, F.W);
  while (next.f < next.f1) {
    ScorePiece p;
    next.next(A, p);
    if (p.t1 <= p.t0) break;
    const int pages = Steps::pages(p.n_int), last = min(p.t1, pages);
    const int32_t* table = A.bt + (size_t)p.b * A.max_pages + A.sink / kPage;
    // lane: the physical page of base + lane
    int base = p.t0, phys = -1;
    auto resolve = [&](int from) {
      base = from;
      phys = -1;
      if (from + lane < last) {
        phys = __ldcg(table + from + lane);
        if (phys < 0 || phys >= A.num_pages) {
          phys = -1;
          atomicOr(A.err, OPTR_DEVERR_PAGE_ID);
        }
      }
    };
    resolve(p.t0);
    uint32_t bad = 0;  // stages of pages that are not to be read
    auto issue = [&](int page, int s) {
      if (page < last) {
        if (page - base == 32) resolve(page);
        const int x = __shfl_sync(0xffffffffu, phys, page - base);
        bad = x < 0 ? bad | 1u << s : bad & ~(1u << s);
        const uint8_t* src = A.pool + ((size_t)max(x, 0) * A.h_kv + p.h) * chunk_bytes(kCompact) + 16 * lane;
        uint8_t* dst = stage + s * kHalfRec + 16 * lane;
        cp_async16_zfill(dst, src + OPTR_K_CODES_OFFSET, x >= 0);
        if (lane < meta_stride(kCompact)) cp_async16_zfill(dst + 512, src + OPTR_K_META_OFFSET, x >= 0);
      }
    };
    Query<kCompact> q;
    if (kTokens == 1 && p.t0 < pages) q.load(few_query(F, p.seg, 0));
    float m[kTokens], l[kTokens];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) m[i] = -1e30f, l[i] = 0.f;
    float* out = reinterpret_cast<float*>(F.logits) + (size_t)p.seg * F.positions * A.max_new * 4 + c;
    // two logits of token i, at positions that count if they are seen
    auto take = [&](int i, int pos0, int pos1, bool in0, bool in1, float x0, float x1) {
      const int seen = p.pos0 + i;
      x0 = in0 && pos0 <= seen ? x0 : -INFINITY;
      x1 = in1 && pos1 <= seen ? x1 : -INFINITY;
      if (in0) out[((size_t)pos0 * A.max_new + i) * 4] = x0;
      if (in1) out[((size_t)pos1 * A.max_new + i) * 4] = x1;
      const float mn = fmaxf(m[i], fmaxf(x0, x1));
      l[i] = fmaf(l[i], ex2(m[i] - mn), ex2(x0 - mn) + ex2(x1 - mn));
      m[i] = mn;
    };
    constexpr int kPairs = kStages / 2;
#pragma unroll
    for (int s = 0; s < kPairs - 1; ++s) {
      issue(p.t0 + 2 * s, 2 * s);
      issue(p.t0 + 2 * s + 1, 2 * s + 1);
      cp_async_commit();
    }
    int at = 0;  // the pair's stages
#pragma unroll 1
    for (int page = p.t0; page < last; page += 2) {
      const int to = at == 0 ? kPairs - 1 : at - 1;
      issue(page + 2 * (kPairs - 1), 2 * to);
      issue(page + 2 * (kPairs - 1) + 1, 2 * to + 1);
      cp_async_commit();
      cp_async_wait<kPairs - 1>();
      __syncwarp();
      Page<kCompact> x[2];
      const int pairs = page + 1 < last ? 2 : 1;
#pragma unroll
      for (int e = 0; e < 2; ++e) x[e].load(stage + (2 * at + e) * kHalfRec);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kTokens; ++i) {
        if (i >= p.rows) break;
        if (kTokens > 1) q.load(few_query(F, p.seg, i));
        float2 y[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) y[e] = x[e].logits(q);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int k = kPage * (page + e) + g;  // of the INT2 keys
          const bool ok = !(bad >> (2 * at + e) & 1);
          const bool in0 = e < pairs && k < p.n_int, in1 = e < pairs && k + 8 < p.n_int;
          take(i, A.sink + k, A.sink + k + 8, in0, in1, ok ? y[e].x : -INFINITY, ok ? y[e].y : -INFINITY);
        }
      }
      at = at + 1 == kPairs ? 0 : at + 1;
    }
    cp_async_wait<0>();
    // window rows, 16 a step: the warp that has a step's first unit
    const int first = max(0, p.t0 - pages);
    for (int u = (first + kWinCost - 1) / kWinCost; pages + kWinCost * u < p.t1; ++u) {
      const int i0 = kWinRows * u + g, i1 = i0 + 8;
      const bool in0 = i0 < p.n_win, in1 = i1 < p.n_win;
      const int pos0 = win_pos(in0 ? i0 : 0, p.n, A.sink, A.recent), pos1 = win_pos(in1 ? i1 : 0, p.n, A.sink, A.recent);
      const __nv_bfloat16* rows = A.win.win + (((size_t)p.slot * A.h_kv + p.h) * 2) * (A.sink + A.recent) * kD + 8 * c;
      const __nv_bfloat16 *r0 = rows + (size_t)win_row(pos0, A.sink, A.recent) * kD,
                          *r1 = rows + (size_t)win_row(pos1, A.sink, A.recent) * kD;
      uint4 a[4], b[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        a[s] = __ldcg(reinterpret_cast<const uint4*>(r0 + 32 * s));
        b[s] = __ldcg(reinterpret_cast<const uint4*>(r1 + 32 * s));
      }
      for (int i = 0; i < p.rows; ++i) {
        const __nv_bfloat16* qr = A.q + ((((size_t)p.c0 + i) * A.h_kv + p.h) * 4 + (g >> 1)) * kD + 8 * c;
        const float2 d = window_logits(a, b, qr, !(g & 1));
        const float mu = __uint_as_float(__ldcg(few_query(F, p.seg, i) + kMu + c));
        const float x0 = fmaf(d.x, F.qscale, -mu), x1 = fmaf(d.y, F.qscale, -mu);
#pragma unroll
        for (int t = 0; t < kTokens; ++t)
          if (t == i) take(t, pos0, pos1, in0, in1, x0, x1);
      }
    }
    // over the lanes of a head
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, m[i], o), ol = __shfl_xor_sync(0xffffffffu, l[i], o);
        const float mn = fmaxf(m[i], om);
        l[i] = l[i] * ex2(m[i] - mn) + ol * ex2(om - mn);
        m[i] = mn;
      }
      if (lane < 4) F.part[((size_t)w + p.seg) * (4 * kFewTok) + 4 * i + c] = make_float2(m[i], l[i]);
    }
  }
}

constexpr int kSumThreads = 256, kSumEach = 4;

// CTA (x, seg): 1024 positions' weights.
__global__ void __launch_bounds__(kSumThreads) few_sum_kernel(const __grid_constant__ FewArgs F) {
  __shared__ long long sum[kSumThreads / 32];
  __shared__ float2 meet[16][4 * kFewTok];
  __shared__ float ref[4 * kFewTok];
  const ScoreArgs& A = F.A;
  const int seg = blockIdx.y, b = seg / A.h_kv, h = seg % A.h_kv, tid = threadIdx.x;
  pdl_wait();
  pdl_trigger();
  const ScoreSeq s = score_seq(A, b);
  const int pos0 = kSumThreads * kSumEach * blockIdx.x;
  if (pos0 >= s.n || s.rows == 0) return;
  int w0, w1;
  workers_of<Steps>(A, b, h, F.W, sum, w0, w1);
  float m = -INFINITY, l = 0.f;
  auto join = [&](float2 x) {
    if (x.y == 0.f) return;
    const float mn = fmaxf(m, x.x);
    l = l * ex2(m - mn) + x.y * ex2(x.x - mn);
    m = mn;
  };
  const int col = tid & 15, split = tid >> 4;
  if (col < 4 * s.rows) {
#pragma unroll 4
    for (int w = w0 + split; w <= w1; w += kSumThreads / 16)
      join(__ldcg(F.part + ((size_t)w + seg) * (4 * kFewTok) + col));
  }
  meet[split][col] = make_float2(m, l);
  __syncthreads();
  if (tid < 16) {
    m = -INFINITY, l = 0.f;
    for (int i = 0; i < kSumThreads / 16; ++i) join(meet[i][tid]);
    ref[tid] = l > 0.f ? -(m + log2f(l)) : -INFINITY;
  }
  __syncthreads();
  const int end = int2_end(s.n, A.sink, A.recent);
  const float4* logits = F.logits + (size_t)seg * F.positions * A.max_new;
  float* score = A.score + (size_t)seg * A.n_score;
#pragma unroll
  for (int e = 0; e < kSumEach; ++e) {
    const int pos = pos0 + kSumThreads * e + tid;
    // (window positions of a slot out of range have no logits)
    if (pos >= s.n || (s.n_win == 0 && (pos < A.sink || pos >= end))) continue;
    float x = 0.f;
    for (int i = 0; i < s.rows; ++i) {
      const float4 y = __ldcg(logits + (size_t)pos * A.max_new + i);
      x += (ex2(y.x + ref[4 * i]) + ex2(y.y + ref[4 * i + 1])) + (ex2(y.z + ref[4 * i + 2]) + ex2(y.w + ref[4 * i + 3]));
    }
    score[pos] = __ldcg(score + pos) + x;
  }
}

// ------------------------------------------------------- a cluster a (sequence, KV head)

constexpr int kOneStages = 6;

// CTA rank r of a cluster of cs: pages P (r) .. P (r + 1) of the INT2 keys and steps
// of 16 window rows alike, by place: place 16 x + t is token t of the x-th.
struct OneSmem {
  union {
    QrotSmem rot;
    float4 logits[1];  // [tokens][places]
  };
};
struct OneFixed {
  FewQuery query[kFewTok];
  uint32_t frag[512];
  float sum[16];
  float top[kWarps][4 * kFewTok], part[kWarps][4 * kFewTok];
  float2 mine[4 * kFewTok];
  float ref[4 * kFewTok];
  alignas(16) uint8_t stage[kWarps][kOneStages][kHalfRec];
};

// kSpill: the logits lie in the workspace, [CTA][token][place].
template <bool kCompact, int kTokens, bool kSpill>
__global__ void __launch_bounds__(kWarps * 32, 1)
few_cluster_kernel(const __grid_constant__ ScoreArgs A, int log_cs, int places, float4* spill, float qscale) {
  extern __shared__ __align__(16) unsigned char dsm_[];
  OneFixed& S = *reinterpret_cast<OneFixed*>(dsm_);
  OneSmem& U = *reinterpret_cast<OneSmem*>(dsm_ + sizeof(OneFixed));
  const int cs = 1 << log_cs, rank = cs > 1 ? cluster_rank_of() : 0;
  const int seg = blockIdx.x >> log_cs, b = seg / A.h_kv, h = seg % A.h_kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  float rv[32];
  load_rotation_slice(A.R_k, h, rv);
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && warp == 0) report_sequences(A);
  const ScoreSeq s = score_seq(A, b);
  if (Steps::of(s) == 0) return;  // the whole cluster
  const int all = Steps::pages(s.n_int), steps = (s.n_win + kWinRows - 1) / kWinRows;
  const int P0 = all * rank >> log_cs, P1 = all * (rank + 1) >> log_cs;
  const int U0 = steps * rank >> log_cs, U1 = steps * (rank + 1) >> log_cs;
  // this warp's pages
  const int p0 = P0 + ((P1 - P0) * warp / kWarps), last = P0 + ((P1 - P0) * (warp + 1) / kWarps);
  const int32_t* table = A.bt + (size_t)b * A.max_pages + A.sink / kPage;
  // lane: the physical page of base + lane
  int base = p0, phys = -1;
  auto resolve = [&](int from) {
    base = from;
    phys = -1;
    if (from + lane < last) {
      phys = __ldcg(table + from + lane);
      if (phys < 0 || phys >= A.num_pages) {
        phys = -1;
        atomicOr(A.err, OPTR_DEVERR_PAGE_ID);
      }
    }
  };
  resolve(p0);
  uint32_t bad = 0;  // stages of pages that are not to be read
  uint8_t* stage = S.stage[warp][0];
  auto issue = [&](int page, int st) {
    if (page < last) {
      if (page - base == 32) resolve(page);
      const int x = __shfl_sync(0xffffffffu, phys, page - base);
      bad = x < 0 ? bad | 1u << st : bad & ~(1u << st);
      const uint8_t* src = A.pool + ((size_t)max(x, 0) * A.h_kv + h) * chunk_bytes(kCompact) + 16 * lane;
      uint8_t* dst = stage + st * kHalfRec + 16 * lane;
      cp_async16_zfill(dst, src + OPTR_K_CODES_OFFSET, x >= 0);
      if (lane < meta_stride(kCompact)) cp_async16_zfill(dst + 512, src + OPTR_K_META_OFFSET, x >= 0);
    }
  };
  constexpr int kPairs = kOneStages / 2;
#pragma unroll
  for (int e = 0; e < kPairs - 1; ++e) {
    issue(p0 + 2 * e, 2 * e);
    issue(p0 + 2 * e + 1, 2 * e + 1);
    cp_async_commit();
  }
  float* score = A.score + (size_t)seg * A.n_score;
  // (the sums so far, a line of 32 a thread)
  if (32 * tid < kPage * (P1 - P0))
    asm volatile("prefetch.global.L2 [%0];" ::"l"(score + min(A.sink + kPage * P0 + 32 * tid, s.n - 1)));
  // the tokens' queries, while the first pages are on their way
#pragma unroll 1
  for (int i = 0; i < s.rows; ++i) {
    const __nv_bfloat16* q = A.q + (((size_t)s.c0 + i) * A.h_kv + h) * (4 * kD);
    FewQuery& Q = S.query[i];
    rotate_query(U.rot, q, rv, qscale, nullptr, S.sum, S.frag, Q.off, Q.inv);
    __syncthreads();
    // [lane][group][word] to [group][lane][word]
    reinterpret_cast<uint32_t*>(Q.frag)[(tid >> 2 & 3) * 128 + (tid >> 4) * 4 + (tid & 3)] = S.frag[tid];
    if (warp == 0) {
      // column g of the min terms' product: head g / 2, hi or lo part of group c's sum
      const float x = S.sum[(g >> 1) * kGroups + c];
      const float hi = __uint_as_float(__float_as_uint(x) & 0xffffe000u);
      Q.min[lane] = (uint32_t)__half_as_ushort(__float2half_rn(g & 1 ? x - hi : hi)) << 16;
    }
    if (A.win.win && tid < 128) {  // head tid / 32
      float d = 0.f;
      for (int k = lane; k < kD; k += 32)
        d = fmaf(__bfloat162float(q[warp * kD + k]), __ldg(A.mu + (size_t)h * kD + k), d);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
      if (lane == 0) Q.mu[warp] = d * qscale;
    }
  }
  __syncthreads();
  float m[kTokens];
#pragma unroll
  for (int i = 0; i < kTokens; ++i) m[i] = -1e30f;
  float4* const stored = kSpill ? spill + (size_t)blockIdx.x * A.max_new * places : U.logits;
  float* logits = reinterpret_cast<float*>(stored) + c;
  Query<kCompact> q;
  if (kTokens == 1) q.load(S.query[0]);
  int at = 0;  // the pair's stages
#pragma unroll 1
  for (int page = p0; page < last; page += 2) {
    const int to = at == 0 ? kPairs - 1 : at - 1;
    issue(page + 2 * (kPairs - 1), 2 * to);
    issue(page + 2 * (kPairs - 1) + 1, 2 * to + 1);
    cp_async_commit();
    cp_async_wait<kPairs - 1>();
    __syncwarp();
    Page<kCompact> x[kTokens > 1 ? 2 : 1];
    if (kTokens > 1) {
#pragma unroll
      for (int e = 0; e < 2; ++e) x[kTokens > 1 ? e : 0].load(stage + (2 * at + e) * kHalfRec);
    }
    const bool whole = !(bad >> (2 * at) & 3) && kPage * (page + 2) <= s.n_int && page + 1 < last;
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
      if (i >= s.rows) break;
      if (kTokens > 1) q.load(S.query[i]);
      float2 y[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (kTokens == 1) x[0].load(stage + (2 * at + e) * kHalfRec);
        y[e] = x[kTokens > 1 ? e : 0].logits(q);
      }
      float* out = logits + ((size_t)i * places + kPage * (page - P0) + g) * 4;
      // the last page, one that is not to be read, keys that this token does not see
      const int lim = min(s.n_int, s.pos0 + i + 1 - A.sink);
      if (!whole || kPage * (page + 2) > lim) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int k = kPage * (page + e) + g;
          const bool ok = !(bad >> (2 * at + e) & 1);
          if (!ok || k >= lim) y[e].x = -INFINITY;
          if (!ok || k + 8 >= lim) y[e].y = -INFINITY;
        }
      }
      out[0] = y[0].x;
      out[32] = y[0].y;
      m[i] = fmaxf(m[i], fmaxf(y[0].x, y[0].y));
      if (page + 1 < last) {
        out[64] = y[1].x;
        out[96] = y[1].y;
        m[i] = fmaxf(m[i], fmaxf(y[1].x, y[1].y));
      }
    }
    __syncwarp();  // the stages are free
    at = at + 1 == kPairs ? 0 : at + 1;
  }
  cp_async_wait<0>();
  const int w_place = kPage * (P1 - P0);  // of the first window row
  for (int u = U0 + warp; u < U1; u += kWarps) {
    const int i0 = kWinRows * u + g, i1 = i0 + 8;
    const bool in0 = i0 < s.n_win, in1 = i1 < s.n_win;
    const int pos0 = win_pos(in0 ? i0 : 0, s.n, A.sink, A.recent), pos1 = win_pos(in1 ? i1 : 0, s.n, A.sink, A.recent);
    const __nv_bfloat16* rows = A.win.win + (((size_t)s.slot * A.h_kv + h) * 2) * (A.sink + A.recent) * kD + 8 * c;
    const __nv_bfloat16 *r0 = rows + (size_t)win_row(pos0, A.sink, A.recent) * kD,
                        *r1 = rows + (size_t)win_row(pos1, A.sink, A.recent) * kD;
    uint4 k0[4], k1[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      k0[e] = __ldcg(reinterpret_cast<const uint4*>(r0 + 32 * e));
      k1[e] = __ldcg(reinterpret_cast<const uint4*>(r1 + 32 * e));
    }
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
      if (i >= s.rows) break;
      const __nv_bfloat16* qr = A.q + ((((size_t)s.c0 + i) * A.h_kv + h) * 4 + (g >> 1)) * kD + 8 * c;
      const float2 d = window_logits(k0, k1, qr, !(g & 1));
      const int seen = s.pos0 + i;
      const float x0 = in0 && pos0 <= seen ? fmaf(d.x, qscale, -S.query[i].mu[c]) : -INFINITY;
      const float x1 = in1 && pos1 <= seen ? fmaf(d.y, qscale, -S.query[i].mu[c]) : -INFINITY;
      float* out = logits + ((size_t)i * places + w_place + kWinRows * (u - U0) + g) * 4;
      out[0] = x0;
      out[32] = x1;
      m[i] = fmaxf(m[i], fmaxf(x0, x1));
    }
  }
  // the CTA's maxima, its sums over those, and the cluster's of both
  const int cols = 4 * s.rows;
#pragma unroll
  for (int i = 0; i < kTokens; ++i) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) m[i] = fmaxf(m[i], __shfl_xor_sync(0xffffffffu, m[i], o));
    if (lane < 4) S.top[warp][4 * i + c] = m[i];
  }
  __syncthreads();
  auto over_warps = [&](const float (&x)[kWarps][4 * kFewTok], int col, auto join) {
    float y = x[lane % kWarps][col];
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) y = join(y, __shfl_xor_sync(0xffffffffu, y, o));
    return y;
  };
  const int n_int = min(kPage * (P1 - P0), s.n_int - kPage * P0), n_win = max(0, min(kWinRows * (U1 - U0), s.n_win - kWinRows * U0));
  const int n_all = n_int + n_win;
  for (int i = 0; i < s.rows; ++i) {
    float top[4], l[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      top[j] = over_warps(S.top, 4 * i + j, [](float x, float y) { return fmaxf(x, y); });
    const float4* x = stored + (size_t)i * places;
#pragma unroll 8
    for (int k = tid; k < n_all; k += kWarps * 32) {
      const float4 y = x[k < n_int ? k : k - n_int + w_place];
      l[0] += ex2(y.x - top[0]);
      l[1] += ex2(y.y - top[1]);
      l[2] += ex2(y.z - top[2]);
      l[3] += ex2(y.w - top[3]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) l[j] += __shfl_xor_sync(0xffffffffu, l[j], o);
      if (lane == j) {
        S.part[warp][4 * i + j] = l[j];
        if (warp == 0) S.mine[4 * i + j].x = top[j];
      }
    }
  }
  __syncthreads();
  if (tid < cols) {
    float l = 0.f;
    for (int i = 0; i < kWarps; ++i) l += S.part[i][tid];
    S.mine[tid].y = l;
  }
  // the sums so far, kEach positions of a thread at a time: on their way before they are wanted
  constexpr int kEach = 8;
  float old[kEach];
  auto pos_of = [&](int k) {
    return k < n_int ? A.sink + kPage * P0 + k : win_pos(kWinRows * U0 + k - n_int, s.n, A.sink, A.recent);
  };
  auto fetch = [&](int k0) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int k = k0 + e * kWarps * 32;
      old[e] = k < n_all ? __ldcg(score + pos_of(k)) : 0.f;
    }
  };
  fetch(tid);
  if (cs > 1) cluster_barrier(); else __syncthreads();
  if (tid < cols) {
    float2 y[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      y[r] = make_float2(-1e30f, 0.f);
      if (r < cs) {
        if (cs > 1) {
          const unsigned long long z = cluster_ld64(&S.mine[tid], r);
          y[r] = make_float2(__uint_as_float((uint32_t)z), __uint_as_float((uint32_t)(z >> 32)));
        } else {
          y[r] = S.mine[tid];
        }
      }
    }
    float top = -1e30f, l = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) top = fmaxf(top, y[r].x);
#pragma unroll
    for (int r = 0; r < 8; ++r) l += y[r].y * ex2(y[r].x - top);
    S.ref[tid] = l > 0.f ? -(top + log2f(l)) : -INFINITY;
  }
  __syncthreads();
  if (cs > 1) cluster_arrive();  // no CTA leaves while its shared memory may be read
  for (int k0 = tid; k0 < n_all; k0 += kEach * kWarps * 32) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int k = k0 + e * kWarps * 32;
      if (k >= n_all) break;
      const int place = k < n_int ? k : k - n_int + w_place;
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < kTokens; ++i) {
        if (i >= s.rows) break;
        const float4 y = stored[(size_t)i * places + place], r = *reinterpret_cast<const float4*>(S.ref + 4 * i);
        x += (ex2(y.x + r.x) + ex2(y.y + r.y)) + (ex2(y.z + r.z) + ex2(y.w + r.w));
      }
      score[pos_of(k)] = old[e] + x;
    }
    fetch(k0 + kEach * kWarps * 32);
  }
  if (cs > 1) cluster_wait();
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

template <int kTokens>
cudaError_t launch_logits(const optr_params* p, const FewArgs& F, cudaStream_t s) {
  auto fn = F.A.compact ? few_logit_kernel<true, kTokens> : few_logit_kernel<false, kTokens>;
  const size_t smem = (size_t)kWarps * kStages * kHalfRec;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(fn), smem);
  return e != cudaSuccess ? e : launch_pdl(fn, dim3(p->num_sms), dim3(kWarps * 32), smem, s, F);
}

// The cluster kernel's launch: log2 of the CTAs of a (sequence, KV head), places of a CTA,
// and whether their logits fit shared memory.
struct Clusters {
  int log_cs, places;
  size_t smem;
  bool spill, use;
};
Clusters clusters(const optr_params* p, int B, int max_new, int max_pages) {
  Clusters c;
  const long long segs = (long long)B * p->cfg.h_kv;
  // as many as are resident at once: at one CTA an SM, 152 SMs take 152 CTAs in clusters of 2, 144
  // of 4 and 120 of 8
  const int most[4] = {p->num_sms, p->num_sms, p->num_sms * 15 / 16, p->num_sms * 3 / 4};
  c.log_cs = 0;
  while (c.log_cs < 3 && (segs << (c.log_cs + 1)) <= most[c.log_cs + 1]) ++c.log_cs;
  const int units = (max_pages + 2) / (1 << c.log_cs) + 3;
  c.places = units * kPage;
  c.smem = sizeof(OneFixed) + std::max(sizeof(QrotSmem), (size_t)c.places * max_new * sizeof(float4));
  c.spill = c.smem > 227 * 1024;
  if (c.spill) c.smem = sizeof(OneFixed) + sizeof(QrotSmem);
  // long contexts that leave many SMs idle are cut evenly instead (few_logit_kernel: 4 x 1 over
  // 131072 with 64 CTAs 203 us, evenly 146)
  const long long ctas = segs << c.log_cs, rounds = (ctas + p->num_sms - 1) / p->num_sms;
  c.use = !c.spill || ctas * 10 >= rounds * p->num_sms * 7;
  return c;
}

template <int kTokens>
cudaError_t launch_cluster(const ScoreArgs& A, const Clusters& c, float4* spill, cudaStream_t s) {
  auto fn = A.compact ? c.spill ? few_cluster_kernel<true, kTokens, true> : few_cluster_kernel<true, kTokens, false>
                      : c.spill ? few_cluster_kernel<false, kTokens, true> : few_cluster_kernel<false, kTokens, false>;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(fn), c.smem);
  return e != cudaSuccess ? e : launch_pdl_cluster(fn, dim3((unsigned)(A.B * A.h_kv) << c.log_cs), dim3(kWarps * 32),
                                                   1 << c.log_cs, c.smem, s, A, c.log_cs, c.places, spill, kLogit);
}

}  // namespace

// Few tokens' logits: of all positions at most, and of a page's.
constexpr size_t kMostLogits = 256ull << 20;
size_t page_logits(int max_new) { return (size_t)kPage * max_new * sizeof(float4); }

FewLayout few_layout(const optr_params* p, int B, int max_new, int max_pages) {
  FewLayout l;
  const size_t segs = (size_t)B * p->cfg.h_kv;
  l.W = p->num_sms * kWarps;
  l.part = round_up(segs * max_new * kQueryWords * sizeof(uint32_t));
  l.logits = l.part + round_up((segs + l.W) * 4 * kFewTok * sizeof(float2));
  // A cluster has up to two pages and three for each of its CTAs beside (clusters()), and more
  // than one CTA only while all fit the SMs.  Calls of more positions are not of few tokens: the size is
  // that of the largest smaller call which is.
  const size_t page = page_logits(max_new);
  const size_t logits = (size_t)max_pages > kMostLogits / (segs * page) ? kMostLogits : segs * max_pages * page;
  l.total = l.logits + round_up(logits + (5 * segs + 3 * (size_t)p->num_sms) * page);
  return l;
}

// Few tokens, and logits within kMostLogits.
bool few_tokens(const optr_params* p, int B, int max_new, int max_pages) {
  return max_new <= kFewTok && (size_t)max_pages <= kMostLogits / ((size_t)B * p->cfg.h_kv * page_logits(max_new));
}

cudaError_t launch_score_few(const optr_params* p, const ScoreArgs& A, uint8_t* ws, cudaStream_t s) {
  const FewLayout l = few_layout(p, A.B, A.max_new, A.max_pages);
  const Clusters c = clusters(p, A.B, A.max_new, A.max_pages);
  if (c.use) {
    float4* spill = (float4*)(ws + l.logits);
    return A.max_new == 1 ? launch_cluster<1>(A, c, spill, s) : launch_cluster<kFewTok>(A, c, spill, s);
  }
  const FewArgs F{A, (uint32_t*)ws, (float2*)(ws + l.part), (float4*)(ws + l.logits), A.max_pages * kPage, l.W,
                  kLogit};
  const unsigned segs = (unsigned)A.B * A.h_kv;
  cudaError_t e = launch_pdl(few_query_kernel, dim3(segs), dim3(kQrotThreads), 0, s, F);
  if (e == cudaSuccess) e = A.max_new == 1 ? launch_logits<1>(p, F, s) : launch_logits<kFewTok>(p, F, s);
  const int n = std::min(F.positions, A.n_score), each = kSumThreads * kSumEach;
  if (e == cudaSuccess)
    e = launch_pdl(few_sum_kernel, dim3((n + each - 1) / each, segs), dim3(kSumThreads), 0, s, F);
  return e;
}

}  // namespace optr
