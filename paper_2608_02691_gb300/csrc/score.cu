// Attention weights of the new tokens, summed by position (include/optr.h,
// "optr_kv_score"): score[s] += sum over tokens i and heads of softmax(l_i)(s).
//
// The sum over rows needs each row's normaliser first, and the logits are too many to
// be kept (a row of 32768 floats for each of 64 tokens x 4 heads), so they are computed
// twice: query_kernel rotates the queries, logit_kernel<false> finds each row's maximum
// and sum by CTA, logit_kernel<true> joins those, computes the logits again and adds
// exp2(l - lse) up.
//
// Layout.  A tile is 128 keys times the block's columns (64 tokens x 4 heads at most):
// D[key][column] = K Q^T on the tensor core, K in tensor memory (written there by the
// warps that dequantize: a lane has a key), Q in shared memory for a whole piece.  A
// thread of the epilogue has one key: the sum over rows, which the second pass wants,
// is a sum along its registers, and the sum over keys of the first pass is kept per
// column in registers too and meets the other lanes' once a piece.
//
// Bound.  A tile's products: 1.3 us at 256 columns (two products); with 32 columns the
// records' and the keys' way, 0.7 us.
// 2 x 64 tokens over some 32000 positions take 137 us: 70 and 65 for the two passes (26
// tiles an SM each, the tensor pipe 50% busy; without exponentials 66 and 61, without half
// of the products 60 and 58), the rest the query kernel and the launches.  What is left
// lies between the tiles: starts, the query operand's 128 KB, and the few SMs whose
// range goes over a segment's end and waits for the next one's operand.
//
// References.  A sum over keys needs none as long as 2^l neither overflows nor vanishes, and
// |l| <= max |k| * sum |q| holds for every tile of ordinary inputs: then the reference is 0
// and no maximum is looked for (70 us; with one for each column 95).  A sum over reference 0
// may be as small as 2^-118, beside which a later tile's terms below 2^-126 are nothing to a
// float and yet count: where a tile that gets a look lies 2^20 and more below a reference, such
// sums are brought near 1, their references with them.  So are all before those of warps and CTAs
// are joined.
//
// Rounding.  The sums are float32, and a weight moves by what its logit does: rounding
// queries or keys to 16 bits would move it by some 3e-4.  So queries go in as fp16 hi + lo
// parts (22 bits, over a power of two by block), and keys without a rounding.  With one
// pair a slot the codes are the operand, as subnormal numbers, code 2^-16 (lower bits cost
// the sums precision: products are aligned as if their operands were normal), and scale
// and minimum are the epilogue's.  With four pairs a value is (code - 1) scale, four numbers
// of a group that fp16 holds (over a power of two by key; the codes pick among them by byte
// permutes), plus minimum + scale of its group, which meets the query's sum over the group in one
// step more, both as hi + lo.  Window keys and their queries are bf16 as they are, one product.
#include "cluster.cuh"
#include "f32x2.cuh"
#include "score.cuh"
#include "tc05.cuh"

#include <algorithm>
#include <type_traits>

namespace optr {
namespace {

// ------------------------------------------------------------- queries

// Place of a channel in a key row: word w of a slot's codes has, by byte, the four
// groups' channels 4 w .. 4 w + 3.  Codes that go in as they are: a register has the same
// two bits of either half of the word.
__host__ __device__ constexpr int key_place(int channel, bool codes) {
  const int w = (channel >> 2) & 7, G = channel >> 5, e = channel & 3;
  return codes ? 16 * w + 2 * (4 * (G & 1) + e) + (G >> 1) : 16 * w + 4 * G + e;
}

// Element (n, k) of an operand of n columns, K-major without swizzle: core matrices of
// 8 columns x 8 of k (128 B), 128 B apart along k and 2048 B along n.
__device__ __forceinline__ int operand_offset(int n, int k) {
  return (n / 8) * 2048 + (k / 8) * 128 + (n % 8) * 16 + (k % 8) * 2;
}

// An operand of 16 inner elements: two core matrices, 128 B apart, of 8 columns each; the
// first element of column n (the ninth is 128 B on).
__device__ __forceinline__ int ext_offset(int n) { return (n / 8) * 256 + (n % 8) * 16; }

constexpr int kRotThreads = 256;
constexpr int kRotCols = 32;  // columns of a CTA: 8 tokens

// CTA (x, seg): columns 32 x .. of the segment's block, rotated.  The queries are bf16, so
// products with three bf16 parts of the rotation's elements are as good as float32's:
// m16n8k16, a warp has 16 channels of the 32 columns.  The rotation comes into shared
// memory whole, before what the call waits for: its 128 rows' latencies are one.
constexpr int kRotPad = kD + 4, kQueryPad = kD + 8;  // rows in different banks
struct QuerySmem {
  float R[kD][kRotPad];
  __nv_bfloat16 q[kRotCols][kQueryPad];
  // of the columns: by warp the largest element, the sum and the sum of magnitudes; <q, mu>
  float top[8][kRotCols], sum[8][kRotCols], size[8][kRotCols], dot[kRotCols], given[kRotCols];
  float most[3];  // the CTA's largest element, and sums of magnitudes, rotated and as given
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The bf16 parts of two numbers: their rounded values are taken off x and y.
__device__ __forceinline__ uint32_t bf16_part(float& x, float& y) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  x -= __uint_as_float(r << 16);
  y -= __uint_as_float(r & 0xffff0000u);
  return r;
}

// Over the warp's lanes, of 16 values each: value lane / 2 (in both lanes).
template <typename Join>
__device__ __forceinline__ float over_lanes(float (&x)[16], Join join) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 1; o >>= 1) {
    const bool upper = lane & o;
#pragma unroll
    for (int j = 0; j < o / 2; ++j) {
      const float mine = upper ? x[j + o / 2] : x[j], other = upper ? x[j] : x[j + o / 2];
      x[j] = join(mine, __shfl_xor_sync(0xffffffffu, other, o));
    }
  }
  return join(x[0], __shfl_xor_sync(0xffffffffu, x[0], 1));
}

__global__ void __launch_bounds__(kRotThreads) query_kernel(const __grid_constant__ ScoreArgs A) {
  extern __shared__ __align__(1024) unsigned char dsm_[];
  QuerySmem& S = *reinterpret_cast<QuerySmem*>(dsm_);
  const int seg = blockIdx.y, b = seg / A.h_kv, h = seg % A.h_kv, tid = threadIdx.x;
  const int warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  for (int i = tid; i < kD * kD / 4; i += kRotThreads)
    cp_async16(&S.R[i / (kD / 4)][4 * (i % (kD / 4))], A.R_k + (size_t)h * kD * kD + 4 * i);
  cp_async_commit();
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && seg == 0 && A.t0 == 0 && tid < 32) report_sequences(A);
  const ScoreSeq s = score_seq(A, b);
  const int c0 = kRotCols * blockIdx.x, N = (4 * s.rows + 15) / 16 * 16;
  if (seq_tiles(s) == 0) {  // the whole cluster
    cp_async_wait<0>();
    return;
  }
  const bool win = A.win.win != nullptr;
  uint8_t* out = qop_of(A, seg);
  if (c0 < N) {
    for (int i = tid; i < kRotCols * kD / 8; i += kRotThreads) {
      const int n = i / (kD / 8), x = 8 * (i % (kD / 8)), tok = (c0 + n) / 4;
      uint4 y = make_uint4(0u, 0u, 0u, 0u);
      if (tok < s.rows)
        y = __ldcg(reinterpret_cast<const uint4*>(
            A.q + (((size_t)s.c0 + A.t0 + tok) * A.h_kv + h) * (4 * kD) + (n & 3) * kD + x));
      *reinterpret_cast<uint4*>(&S.q[n][x]) = y;
      if (win && c0 + n < N)
        *reinterpret_cast<uint4*>(out + (size_t)A.cols * 512 + operand_offset(c0 + n, x)) = y;
    }
  }
  cp_async_wait<0>();
  __syncthreads();
  float acc[2][2][4] = {};  // columns 16 i + g, + 8; channels 16 warp + 8 j + 2 c, + 1
  if (c0 < N) {
#pragma unroll 2
    for (int k = 0; k < kD; k += 16) {
      uint32_t a[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          a[i][e] = *reinterpret_cast<const uint32_t*>(&S.q[16 * i + g + 8 * (e & 1)][k + 2 * c + 8 * (e >> 1)]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int n = 16 * warp + 8 * j + g;
        float x[4] = {S.R[k + 2 * c][n], S.R[k + 2 * c + 1][n], S.R[k + 2 * c + 8][n], S.R[k + 2 * c + 9][n]};
#pragma unroll
        for (int part = 0; part < 3; ++part) {
          const uint32_t b0 = bf16_part(x[0], x[1]), b1 = bf16_part(x[2], x[3]);
          mma_bf16(acc[0][j], a[0], b0, b1);
          mma_bf16(acc[1][j], a[1], b0, b1);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float x[4] = {acc[i][0][2 * e], acc[i][0][2 * e + 1], acc[i][1][2 * e], acc[i][1][2 * e + 1]};
        float m = fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3])));
        float t = (x[0] + x[1]) + (x[2] + x[3]), l = (fabsf(x[0]) + fabsf(x[1])) + (fabsf(x[2]) + fabsf(x[3]));
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
          t += __shfl_xor_sync(0xffffffffu, t, o);
          l += __shfl_xor_sync(0xffffffffu, l, o);
        }
        if (c == 0) {
          const int n = 16 * i + 8 * e + g;
          S.top[warp][n] = m;
          S.sum[warp][n] = t;
          S.size[warp][n] = l;
        }
      }
    // <q, mu>: eight lanes a column
    float d = 0.f, l = 0.f;
#pragma unroll
    for (int x = 8 * (lane & 7); x < kD; x += 64) {
      const uint4 y = *reinterpret_cast<const uint4*>(&S.q[tid >> 3][x]);
      const float4* mu = reinterpret_cast<const float4*>(A.mu + (size_t)h * kD + x);
      const float4 m0 = __ldg(mu), m1 = __ldg(mu + 1);
      const uint32_t word[4] = {y.x, y.y, y.z, y.w};
      const float m[8] = {m0.x, m0.y, m0.z, m0.w, m1.x, m1.y, m1.z, m1.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = __uint_as_float(word[e] << 16), b = __uint_as_float(word[e] & 0xffff0000u);
        d = fmaf(a, m[2 * e], d);
        d = fmaf(b, m[2 * e + 1], d);
        l += fabsf(a) + fabsf(b);
      }
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      d += __shfl_xor_sync(0xffffffffu, d, o);
      l += __shfl_xor_sync(0xffffffffu, l, o);
    }
    if ((lane & 7) == 0) S.dot[tid >> 3] = d, S.given[tid >> 3] = l;
  }
  __syncthreads();
  auto warps = [&](const float (&x)[8][kRotCols], int n) {
    return ((x[0][n] + x[1][n]) + (x[2][n] + x[3][n])) + ((x[4][n] + x[5][n]) + (x[6][n] + x[7][n]));
  };
  if (tid < 32) {
    float m = 0.f, l = 0.f, given = 0.f;
    if (c0 < N) {
      given = S.given[lane];
      for (int w = 0; w < 8; ++w) m = fmaxf(m, S.top[w][lane]);
      l = warps(S.size, lane);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      l = fmaxf(l, __shfl_xor_sync(0xffffffffu, l, o));
      given = fmaxf(given, __shfl_xor_sync(0xffffffffu, given, o));
    }
    if (lane == 0) S.most[0] = m, S.most[1] = l, S.most[2] = given;
  }
  const int cs = gridDim.x;  // a cluster has the block's columns
  if (cs > 1) cluster_barrier(); else __syncthreads();
  float m = S.most[0], l = S.most[1], given = S.most[2];
  if (cs > 1) {
    const int r = lane % cs;  // a CTA a lane
    m = __uint_as_float(cluster_ld32(&S.most[0], r));
    l = __uint_as_float(cluster_ld32(&S.most[1], r));
    given = __uint_as_float(cluster_ld32(&S.most[2], r));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      l = fmaxf(l, __shfl_xor_sync(0xffffffffu, l, o));
      given = fmaxf(given, __shfl_xor_sync(0xffffffffu, given, o));
    }
    cluster_arrive();  // no CTA leaves while its shared memory may be read
  }
  if (c0 < N) {
    // The block's largest at 2^13 .. 2^14: an element has 22 bits down to 2^-17 of that, and
    // below it is known to 2^-38 of the largest.
    const int E = m > 0.f ? max(-100, min(100, 13 - ((int)(__float_as_uint(m) >> 23) - 127))) : 0;
    float* line = reinterpret_cast<float*>(out + qop_lines(A.cols, win, A.compact));
    const float up = __uint_as_float((uint32_t)(127 + E) << 23);
    __half* stage = reinterpret_cast<__half*>(S.R);  // the rotation has been used
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int n = 16 * i + 8 * e + g;
          const int ch = 16 * warp + 8 * j + 2 * c;
          const float x = acc[i][j][2 * e] * up, y = acc[i][j][2 * e + 1] * up;
          const __half2 hi = __floats2half2_rn(x, y);
          const float2 z = __half22float2(hi);
          const __half2 lo = __floats2half2_rn(x - z.x, y - z.y);
          __half* at = stage + operand_offset(n, key_place(ch, A.compact)) / 2;
          if (A.compact) {  // (the second channel's place is two on)
            at[0] = __low2half(hi), at[2] = __high2half(hi);
            at += kRotCols * kD;
            at[0] = __low2half(lo), at[2] = __high2half(lo);
          } else {
            *reinterpret_cast<__half2*>(at) = hi;
            *reinterpret_cast<__half2*>(at + kRotCols * kD) = lo;
          }
        }
    __syncthreads();
    // (as they lie in memory: eight columns are 2 KB)
    for (int i = tid; i < min(kRotCols, N - c0) / 8 * 128; i += kRotThreads) {
      uint4* to = reinterpret_cast<uint4*>(out + (size_t)c0 * 256) + i;
      to[0] = reinterpret_cast<const uint4*>(stage)[i];
      to[A.cols * 16] = reinterpret_cast<const uint4*>(stage + kRotCols * kD)[i];
    }
    // Beside four pairs a slot: the groups' sums, over 2^5 (32 channels), as the parts that meet
    // a key's minima: hi, lo, hi
    if (!A.compact && tid < 128 && c0 + lane < N) {
      const int n = c0 + lane;
      const float x = (S.sum[2 * warp][lane] + S.sum[2 * warp + 1][lane]) * (up * 0x1p-5f);
      const __half hi = __float2half_rn(x), lo = __float2half_rn(x - __half2float(hi));
      __half* at = reinterpret_cast<__half*>(out + (size_t)A.cols * (win ? 768 : 512) + ext_offset(n)) + warp;
      at[0] = hi, at[4] = lo, at[64] = hi, at[68] = __float2half_rn(0.f);
    }
    if (tid < kRotCols && c0 + tid < N) {
      line[c0 + tid] = kLogit * S.dot[tid];
      line[A.cols + c0 + tid] = kLogit * warps(S.sum, tid);
    }
    if (blockIdx.x == 0 && tid == 0)
      *reinterpret_cast<float4*>(line + 2 * A.cols) =
          make_float4(__uint_as_float((uint32_t)(127 - E) << 23) * (A.compact ? 0x1p16f * kLogit : kLogit), kLogit * l, kLogit * given, 0.f);
  }
  if (cs > 1) cluster_wait();
}

// -------------------------------------------------------------- logits

// Warps: two epilogue groups of four, four that write keys, one each for the copies, the
// products and the pieces.  Registers a thread after the split, of the launch's.
// kNarrow: blocks of 16 tokens at most.  A tile of theirs is bound by its keys' way into tensor
// memory, so two groups write keys, in tiles of their parity, and four tiles of keys
// stand there (16 x 8 over 8192: 123 -> 119 us).  A group skips the phases of a record buffer
// that the other takes, so that a phase may not be taken for the next but one: by when a
// group waits for the tile eight behind, the products of the sixth before it are done, so
// that tile's records have been there.
template <bool kNarrow>
struct Roles {
  static constexpr int kThreads = kNarrow ? 640 : 512;
  static constexpr int kKeyWarp = 8, kKeyGroups = kNarrow ? 2 : 1, kCopyWarp = kKeyWarp + 4 * kKeyGroups;
  static constexpr int kMmaWarp = kCopyWarp + 1, kPlanWarp = kCopyWarp + 2;
  static constexpr int kConsumers = kCopyWarp + 2;  // warps that take the pieces
  static constexpr int kLaunch = kNarrow ? 96 : 128, kEpi = kNarrow ? 136 : 208;
  static constexpr int kKey = kNarrow ? 72 : 56, kIssue = kNarrow ? 64 : 40;
  static_assert(2 * kEpi + kKeyGroups * kKey + kIssue <= kThreads / 128 * kLaunch, "registers of the launch");
  static constexpr int kCols = kNarrow ? 64 : 128;  // columns of a D
};
constexpr uint32_t kTmemCols = 512, kColD = 0;
// D[d] at kCols d, then the tiles of keys: 64 columns, and 8 for the minima of four pairs a
// slot (with two such tiles and D of 128 columns there is no room for a third D).
template <bool kCompact, bool kNarrow>
struct Tmem {
  static constexpr int kDs = kCompact || kNarrow ? 3 : 2, kKs = kNarrow ? 4 : 2;
  static constexpr uint32_t kDCols = Roles<kNarrow>::kCols, kColK = kDCols * kDs, kKeyCols = kCompact ? 64u : 80u;
  static_assert(kColK + kKs * kKeyCols <= kTmemCols, "tensor memory");
};
constexpr int kPieces = 3;     // pieces found ahead
constexpr float kSlack = 60.f; // a column's logits may pass its reference by 2^60

template <bool kCompact, bool kNarrow>
struct Smem {
  static constexpr int kCols = kNarrow ? kBlockCols / 4 : kBlockCols;
    static constexpr int kRaw = kNarrow ? 8 : kCompact ? 3 : 2;  // tiles of records on the way
  static_assert(!kNarrow || kRaw >= 8, "see Roles");
  uint8_t q[3][kCols * 256];    // hi, lo, as given
  uint8_t raw[kRaw][kKeys / kPage][512 + 16 * meta_stride(kCompact)];  // a page's key codes and pairs
  alignas(16) float off[kCols], sum[kCompact ? kCols : 4];
  alignas(16) uint8_t ext[kCompact ? 16 : kCols * 32];  // the groups' sums
  float4 block;  // the block's factor, and its largest sums of magnitudes
  // minus the columns' references: pass 0 by warp, pass 1 the normalisers
  alignas(16) float ref[8][kKeys];
  float meet[8][kKeys];              // pass 0: the warps' sums of a piece (and, on the way, factors)
  // A key's largest value, or its pair, and whether it counts.  Read between a tile's
  // logits and its last D being free; written for tile t + kRing once the products of
  // t + kRing less the tiles of keys are done, which waited for the Ds before their own.
  static constexpr int kRing = kCompact || kNarrow ? 8 : 4;
  uint32_t scale[kRing][kKeys];
  uint32_t counts[kRing][4];
  uint32_t pages[kRaw];              // a raw tile's pages that are in range
  ScorePiece piece[kPieces];
  uint64_t raw_full[kRaw], raw_empty[kRaw], k_full[4], k_empty[4];
  uint64_t d_full[3][2], d_empty[3];  // by D and the epilogue group that takes it
  uint64_t piece_full[kPieces], piece_empty[kPieces], q_full, q_empty, drained;
  // a piece's meeting of a group's warps (pass 0), and normalisers (pass 1, of all)
  uint64_t meet_full[2], meet_empty[2];
  uint32_t tmem;
  int abort;
};

static_assert(sizeof(Smem<false, false>) <= 232448 && sizeof(Smem<true, false>) <= 232448 &&
                  sizeof(Smem<false, true>) <= 232448, "shared memory of a CTA");

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half(float a, float b) {  // a in the low half
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ float2 unpack_half(uint32_t x) {
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}

// Registers that a load from tensor memory fills: what uses them stays behind the wait
// before this.
template <int n>
__device__ __forceinline__ void loaded(uint32_t (&x)[n]) {
#pragma unroll
  for (int i = 0; i < n; ++i) asm volatile("" : "+r"(x[i]));
}

// The power of two that a key is divided by, of its largest value's bits.
__device__ __forceinline__ int key_power(uint32_t top) { return min(max((int)(top >> 23) - 126, -60), 60); }

// Largest of x over the warp (x is not NaN).
__device__ __forceinline__ float warp_largest(float x) {
  const int i = __float_as_int(x);
  const int y = __reduce_max_sync(0xffffffffu, i ^ ((i >> 31) & 0x7fffffff));
  return __int_as_float(y ^ ((y >> 31) & 0x7fffffff));
}

template <bool kSum, bool kCompact, bool kNarrow>
__global__ void __launch_bounds__(Roles<kNarrow>::kThreads, 1) logit_kernel(const __grid_constant__ ScoreArgs A) {
  extern __shared__ __align__(1024) unsigned char dsm_[];
  using Tmem = Tmem<kCompact, kNarrow>;
  using Roles = Roles<kNarrow>;
  constexpr int kDs = Tmem::kDs;
  constexpr uint32_t kKs = Tmem::kKs;
  constexpr int kKeyWarp = Roles::kKeyWarp, kCopyWarp = Roles::kCopyWarp, kMmaWarp = Roles::kMmaWarp;
  constexpr int kPlanWarp = Roles::kPlanWarp, kCols = Roles::kCols;
  using Smem = Smem<kCompact, kNarrow>;
  Smem& S = *reinterpret_cast<Smem*>(dsm_);
  constexpr uint32_t kRing = Smem::kRing;
  constexpr int kRaw = Smem::kRaw;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) {
    for (int i = 0; i < kRaw; ++i) {
      tc05::bar_init(&S.raw_full[i], kNarrow ? 33 : 1);  // (the lanes' copies, and the tile's pages)
      tc05::bar_init(&S.raw_empty[i], 4);
    }
    for (int i = 0; i < 4; ++i) {
      tc05::bar_init(&S.k_full[i], 4);
      tc05::bar_init(&S.k_empty[i], 1);
    }
    for (int i = 0; i < 3; ++i) {
      tc05::bar_init(&S.d_empty[i], 4);
      for (int e = 0; e < 2; ++e) tc05::bar_init(&S.d_full[i][e], 1);
    }
    for (int i = 0; i < kPieces; ++i) {
      tc05::bar_init(&S.piece_full[i], 1);
      tc05::bar_init(&S.piece_empty[i], Roles::kConsumers);
    }
    tc05::bar_init(&S.q_full, 1);
    tc05::bar_init(&S.q_empty, 9);  // the products, and the epilogue's warps
    tc05::bar_init(&S.drained, 1);
    for (int i = 0; i < 2; ++i) {
      tc05::bar_init(&S.meet_full[i], kSum ? 8 : 4);
      tc05::bar_init(&S.meet_empty[i], kSum ? 8 : 4);
    }
    S.abort = 0;
    tc05::bar_init_fence();
  }
  if (warp == kMmaWarp) tc05::tmem_alloc(&S.tmem, kTmemCols);
  pdl_wait();
  pdl_trigger();
  tc05::fence_before();
  __syncthreads();
  tc05::fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, S.tmem, 0);
  volatile int* abort = &S.abort;
  const int w = blockIdx.x;
  bool dead = false;
  auto wait = [&](uint64_t* bar, uint32_t phase) {
    if (!__all_sync(0xffffffffu, tc05::bar_wait_spin(bar, phase & 1, abort))) dead = true;
    tc05::fence_after();
    return !dead;
  };
  auto arrive = [&](uint64_t* bar) {  // the warp
    __syncwarp();
    if (lane == 0) tc05::bar_arrive(bar);
  };
  auto next_piece = [&](uint32_t n, ScorePiece& p) {
    const uint32_t i = n % kPieces;
    if (dead || !wait(&S.piece_full[i], n / kPieces)) return false;
    p = S.piece[i];
    arrive(&S.piece_empty[i]);
    return p.t1 > p.t0;
  };
  const bool win = A.win.win != nullptr;
  if (warp < kKeyWarp) {
    // ------------------------------------------------------------ epilogue
    // Columns beyond 128 have a D of their own.  Maxima and sums: group g takes its D
    // (pair), or the tiles of its parity; weights: the tiles of its parity, both D.
    tc05::reg_inc<Roles::kEpi>();
    const int g = warp >> 2, key = 32 * (warp & 3) + lane;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    uint32_t phases = 0, nk = 0, nu = 0;  // of d_full[.][g], by bit; key tiles and Ds of the CTA
    ScorePiece p;
    for (uint32_t n = 0; next_piece(n, p); ++n) {
      const int tiles = p.t1 - p.t0, cols = p.cols();
      const bool pair = !kNarrow && cols > kKeys;
      if constexpr (kSum) {
        // minus the columns' normalisers, from the parts of the CTAs that had keys of the segment
        arrive(&S.meet_empty[0]);  // (the piece before has been read)
        if (!wait(&S.meet_empty[0], n)) break;
        const int col = tid;
        float m = -INFINITY, l = 0.f;
        auto join = [&](float2 x) {
          const float mn = fmaxf(m, x.x);
          if (x.y > 0.f) l = l * ex2(m - mn) + x.y * ex2(x.x - mn), m = mn;
        };
        if (col < cols) {
          const int halves = pair ? 1 : 2;  // both groups' parts where they share the columns
#pragma unroll 1
          for (int i0 = 0; i0 < halves * (p.w1 - p.w0 + 1); i0 += 8) {
            float2 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int j = i0 + i, w = p.w0 + (pair ? j : j >> 1);
              x[i] = w <= p.w1 ? __ldcg(score_part(A, w, p.seg) + (pair ? 0 : (j & 1) * kKeys) + col)
                               : make_float2(0.f, 0.f);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) join(x[i]);
          }
        }
        S.ref[0][col] = l > 0.f ? -(m + log2f(l)) : -INFINITY;
        arrive(&S.meet_full[0]);
        if (!wait(&S.meet_full[0], n)) break;
      }
      if (!wait(&S.q_full, n)) break;
      float* ref = kSum ? S.ref[0] : S.ref[warp];
      const int cbase = !kSum && pair ? kKeys * g : 0;  // first column of the group's
      const float factor = S.block.x;
      float acc[kSum ? 1 : kCols];
      // what they may pass it by unseen: a group's sum over the piece stays below 2^126
      const float most = 119.f - (32 - __clz(tiles));
      uint32_t known = 0;     // bit c: column 16 c + lane / 2 has keys in its sum, or is none
      float least = 0.f;      // no reference has been lower
      bool unseen = false, near = false;  // sums of unseen logits: there are, have been brought near 1
      if constexpr (!kSum) {
#pragma unroll
        for (int c = 0; c < kCols; ++c) acc[c] = 0.f;
#pragma unroll
        for (int c = 0; c < kCols / 32; ++c) ref[32 * c + lane] = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) known |= (cbase + 16 * c + (lane >> 1) >= cols ? 1u : 0u) << c;
        __syncwarp();
      }
      for (int t = 0; t < tiles; ++t) {
        if ((kSum || !pair) && (t & 1) != g) continue;
        const int tile = p.t0 + t;
        const bool exact = tile >= p.I();  // a window tile
        float scale = 0.f, low = 0.f, old = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        int first = 0;                   // the first column that sees the key
        float* at = nullptr;
        bool begun = false;
#pragma unroll 1
        for (int d = kSum || !pair ? 0 : g; d < (pair && (kSum || g == 1) ? 2 : 1); ++d) {
          const uint32_t D = (nu + (pair ? 2 * t + d : t)) % kDs;
          if (!wait(&S.d_full[D][g], phases >> D & 1)) break;
          phases ^= 1u << D;
          if (!begun) {
            begun = true;
            const uint32_t r = (nk + t) % kRing, word = S.scale[r][key];
            if (exact) {
              low = __uint_as_float(word);
            } else if (kCompact) {
              const float2 y = unpack_half(word);
              scale = y.x * factor, low = y.y;
            } else {
              scale = __uint_as_float((uint32_t)(127 + key_power(word)) << 23) * factor;
              low = __uint_as_float(word);
            }
            const int i = kKeys * (exact ? tile - p.I() : tile) + key;
            const int pos = exact ? win_pos(i, p.n, A.sink, A.recent) : A.sink + i;
            if (S.counts[r][warp & 3] >> lane & 1) {
              const int tok = pos - p.pos0 - A.t0;
              first = tok > 0 ? 4 * tok : 0;
              if (kSum) {
                at = A.score + (size_t)p.seg * A.n_score + pos;
                old = __ldcg(at);
              }
            } else {
              first = 1 << 20;
            }
          }
          const uint32_t tD = tmem + lanes + kColD + Tmem::kDCols * D;
          const int c_lo = kSum ? kKeys * d : cbase;    // the columns' place in the block
          const int n_cols = min(kKeys, cols - c_lo);
          const bool masked = __any_sync(0xffffffffu, first > c_lo);
          auto free_d = [&]() {
            tc05::fence_before();
            arrive(&S.d_empty[D]);
          };
          // logits of 16 columns, over their references.  What a tile is stands in the
          // type, since branches within made this loop half as long again: it has to
          // stay small in the instruction cache.
          auto logits = [&](int c, const uint32_t* x, float (&y)[16], auto exact_tile, auto masked_tile) {
            const float* r = kSum ? S.ref[0] + c_lo + 16 * c : ref + 16 * c;
            const float2 scale2 = make_float2(scale, scale), low2 = make_float2(low, low);
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
              const float4 m = *reinterpret_cast<const float4*>(r + j);
              if constexpr (decltype(exact_tile)::value) {
                const float4 o = *reinterpret_cast<const float4*>(&S.off[c_lo + 16 * c + j]);
                y[j] = fmaf(__uint_as_float(x[j]), kLogit, m.x - o.x);
                y[j + 1] = fmaf(__uint_as_float(x[j + 1]), kLogit, m.y - o.y);
                y[j + 2] = fmaf(__uint_as_float(x[j + 2]), kLogit, m.z - o.z);
                y[j + 3] = fmaf(__uint_as_float(x[j + 3]), kLogit, m.w - o.w);
              } else {
                float2 m0 = make_float2(m.x, m.y), m1 = make_float2(m.z, m.w);
                if constexpr (kCompact) {
                  const float4 q = *reinterpret_cast<const float4*>(&S.sum[c_lo + 16 * c + j]);
                  m0 = fma2(make_float2(q.x, q.y), low2, m0);
                  m1 = fma2(make_float2(q.z, q.w), low2, m1);
                }
                m0 = fma2(make_float2(__uint_as_float(x[j]), __uint_as_float(x[j + 1])), scale2, m0);
                m1 = fma2(make_float2(__uint_as_float(x[j + 2]), __uint_as_float(x[j + 3])), scale2, m1);
                y[j] = m0.x, y[j + 1] = m0.y, y[j + 2] = m1.x, y[j + 3] = m1.y;
              }
            }
            if constexpr (decltype(masked_tile)::value) {
              const int k = first - c_lo - 16 * c;
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (j < k) y[j] = -INFINITY;
            }
          };
          auto by_tile = [&](auto f) {
            if (exact)
              f(std::true_type{}, std::true_type{});
            else if (masked)
              f(std::false_type{}, std::true_type{});
            else
              f(std::false_type{}, std::false_type{});
          };
          if constexpr (kSum) {
            // all of D first: the next products may start
            uint32_t x[kCols / 32][32];
#pragma unroll
            for (int c = 0; c < kCols / 32; ++c)
              if (32 * c < n_cols) tc05::tmem_ld32(tD + 32 * c, x[c]);
            tc05::tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < kCols / 32; ++c) loaded(x[c]);
            free_d();
            by_tile([&](auto exact_tile, auto masked_tile) {
#pragma unroll
              for (int c = 0; c < kCols / 16; ++c) {
                if (16 * c >= n_cols) break;
                float y[16];
                logits(c, x[c / 2] + 16 * (c & 1), y, exact_tile, masked_tile);
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                  sum.x += ex2(y[j]);
                  sum.y += ex2(y[j + 1]);
                  sum.z += ex2(y[j + 2]);
                  sum.w += ex2(y[j + 3]);
                }
              }
            });
          } else {
            // References are 0 as long as no logit lies far from it: that none can, of keys whose
            // values are top at most, the queries' sums of magnitudes say.  Else columns that
            // have no keys yet, and such whose logits pass their reference by far, take the warp's
            // largest.
            const float top = exact || !kCompact ? low : fmaxf(fabsf(low), fabsf(fmaf(3.f, scale / factor, low)));
            const float size = exact ? S.block.z : S.block.y;
            if (!__any_sync(0xffffffffu, (masked && known != 0xffu) || (first < cols && !(size * top <= least + most)))) {
              known = 0xffu;
              unseen = true;
            } else {
              float* by = S.meet[warp];  // by what a column's sum shrinks, twice (2^-m may be 0)
              bool shrink = false, deep = false;
#pragma unroll 1
              for (int c = 0; c < kCols / 16; ++c) {
                if (16 * c >= n_cols) break;
                uint32_t x[16];
                tc05::tmem_ld16(tD + 16 * c, x);
                tc05::tmem_wait_ld();
                loaded(x);
                float y[16];
                if (exact)
                  logits(c, x, y, std::true_type{}, std::true_type{});
                else
                  logits(c, x, y, std::false_type{}, std::true_type{});
                // (column 16 c + lane / 2)
                const float m = over_lanes(y, [](float a, float b) { return fmaxf(a, b); });
                const bool fresh = !(known >> c & 1);
                const bool moves = m > (fresh ? -INFINITY : kSlack);
                if (moves) {
                  known |= 1u << c;
                  least = fminf(least, m - ref[16 * c + (lane >> 1)]);
                }
                __syncwarp();
                if (lane & 1) {
                  if (moves) ref[16 * c + (lane >> 1)] -= m;
                  by[16 * c + (lane >> 1)] = moves && !fresh ? ex2(-0.5f * m) : 1.f;
                }
                shrink |= moves && !fresh;
                deep |= !fresh && m < -20.f && m > -INFINITY;
              }
              __syncwarp();
              if (unseen && !near && __any_sync(0xffffffffu, deep)) {
                // (all columns have keys, and those that move a sum near 1: not needed again)
                near = shrink = true;
#pragma unroll
                for (int c = 0; c < kCols; c += 32) {
                  if (c >= n_cols) break;
                  uint32_t largest = 0u;
#pragma unroll
                  for (int j = 0; j < 32; ++j) {
                    const uint32_t x = __reduce_max_sync(0xffffffffu, __float_as_uint(acc[c + j]));
                    if (lane == j) largest = x;
                  }
                  if (c + lane < n_cols && by[c + lane] == 1.f) {
                    const float e = (float)(largest >> 23) - 127.f;
                    by[c + lane] = ex2(-0.5f * e);
                    ref[c + lane] -= e;
                    least = fminf(least, -ref[c + lane]);
                  }
                }
              }
              least = -warp_largest(-least);
              __syncwarp();
              if (__any_sync(0xffffffffu, shrink)) {
#pragma unroll
                for (int c = 0; c < kCols; c += 4) {
                  if (c >= n_cols) break;
                  const float4 f = *reinterpret_cast<const float4*>(by + c);
                  acc[c] *= f.x, acc[c + 1] *= f.y, acc[c + 2] *= f.z, acc[c + 3] *= f.w;
                  acc[c] *= f.x, acc[c + 1] *= f.y, acc[c + 2] *= f.z, acc[c + 3] *= f.w;
                }
                __syncwarp();
              }
            }
            by_tile([&](auto exact_tile, auto masked_tile) {
#pragma unroll
              for (int c = 0; c < kCols / 16; ++c) {
                if (16 * c >= n_cols) break;
                uint32_t x[16];
                tc05::tmem_ld16(tD + 16 * c, x);
                tc05::tmem_wait_ld();
                loaded(x);
                if (16 * (c + 1) >= n_cols) free_d();
                float y[16];
                logits(c, x, y, exact_tile, masked_tile);
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[16 * c + j] += ex2(y[j]);
              }
            });
          }
        }
        if (dead) break;
        if (kSum && at) *at = old + ((sum.x + sum.y) + (sum.z + sum.w));
      }
      if (dead) break;
      nk += tiles;
      nu += pair ? 2 * tiles : tiles;
      if constexpr (!kSum) {
        // over the warp's keys: 32 columns a time, each lane ends with one's sum
#pragma unroll
        for (int c = 0; c < kCols / 32; ++c) {
          float* a = acc + 32 * c;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) {
            const bool upper = lane & o;
#pragma unroll
            for (int j = 0; j < o; ++j) {
              const float mine = upper ? a[j + o] : a[j], other = upper ? a[j] : a[j + o];
              a[j] = mine + __shfl_xor_sync(0xffffffffu, other, o);
            }
          }
          S.meet[warp][32 * c + lane] = a[0];
        }
        __syncwarp();
        // over the group's warps
        arrive(&S.meet_full[g]);
        if (!wait(&S.meet_full[g], n)) break;
        float m = -INFINITY, l = 0.f;
        if (key < kCols) {
          // (a sum is y 2^e over its reference)
          float y[4], e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = __float_as_uint(S.meet[4 * g + i][key]);
            y[i] = __uint_as_float((x & 0x7fffffu) | 0x3f800000u);
            e[i] = (float)((int)(x >> 23) - 127);
            if (x < 1u << 23) y[i] = 0.f;  // none
            if (y[i] > 0.f) m = fmaxf(m, e[i] - S.ref[4 * g + i][key]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (y[i] > 0.f) l += y[i] * ex2((-S.ref[4 * g + i][key] - m) + e[i]);
          score_part(A, w, p.seg)[kKeys * g + key] = make_float2(m, l);
        }
        arrive(&S.meet_empty[g]);
        if (!wait(&S.meet_empty[g], n)) break;
      }
      arrive(&S.q_empty);
    }
  } else if (warp < kCopyWarp) {
    // --------------------------------------------------------------- keys
    // Thread = key.  A's row in tensor memory: 64 columns of its codes as they are, its four groups'
    // (code - 1) scale with 8 of their minima's parts beside, or a window key's bf16.
    tc05::reg_dec<Roles::kKey>();
    constexpr int ms = meta_stride(kCompact);
    const int quarter = warp & 3, key = tid & 127;
    const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
    uint32_t nk = 0, raws = 0;
    ScorePiece p;
    for (uint32_t n = 0; next_piece(n, p); ++n) {
      for (int tile = p.t0; tile < p.t1; ++tile, ++nk) {
        if (Roles::kKeyGroups > 1 && (nk & 1) != (uint32_t)((warp - kKeyWarp) >> 2)) {  // the other group's
          raws += tile < p.I();
          continue;
        }
        const uint32_t s = nk % kKs, tK = tmem + lanes + Tmem::kColK + Tmem::kKeyCols * s;
        bool ok;
        uint32_t scale = 0u;
        if (tile < p.I()) {
          const uint32_t r = raws % kRaw;
          if (!wait(&S.raw_full[r], raws / kRaw)) break;
          ++raws;
          ok = kKeys * tile + key < p.n_int && (S.pages[r] >> (key / kPage) & 1);
          const uint8_t* raw = S.raw[r][key / kPage];
          const int slot = key % kPage;
          [[maybe_unused]] uint32_t value[4][2], least[2][4];  // of each group; minima's parts
          if constexpr (kCompact) {
            scale = *reinterpret_cast<const uint32_t*>(raw + 512 + ms * slot);
          } else {
            const uint4 mm = *reinterpret_cast<const uint4*>(raw + 512 + ms * slot);
            // over a power of two above the largest
            const uint32_t pairs[4] = {mm.x, mm.y, mm.z, mm.w};
            float top = 0.f;
#pragma unroll
            for (int G = 0; G < 4; ++G) {
              const float2 y = unpack_half(pairs[G]);
              top = fmaxf(top, fmaxf(fabsf(y.y), fabsf(fmaf(3.f, y.x, y.y))));
            }
            scale = __float_as_uint(top);
            const float down = __uint_as_float((uint32_t)(127 - key_power(scale)) << 23);
            // a value is (code - 1) scale, which fp16 holds, and the rest of its group's
            float x[4];
#pragma unroll
            for (int G = 0; G < 4; ++G) {
              const float2 y = unpack_half(pairs[G]);
              const float sc = y.x * down;
              value[G][0] = pack_half(-sc, 0.f);
              value[G][1] = pack_half(sc, 2.f * sc);
              x[G] = (y.x + y.y) * down * 32.f;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              least[0][i] = least[0][2 + i] = pack_half(x[2 * i], x[2 * i + 1]);
              const float2 z = unpack_half(least[0][i]);
              least[1][i] = pack_half(x[2 * i] - z.x, x[2 * i + 1] - z.y);
              least[1][2 + i] = 0u;
            }
          }
          if (nk >= kKs && !wait(&S.k_empty[s], nk / kKs - 1)) break;
#pragma unroll
          for (int part = 0; part < 4; ++part) {
            const uint2 word = *reinterpret_cast<const uint2*>(raw + 32 * slot + 8 * part);
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              const uint32_t x = v ? word.y : word.x;
              uint32_t y[8];
              if constexpr (kCompact) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = (e < 4 ? x << (8 - 2 * e) : x >> (2 * e - 8)) & 0x03000300u;
                tc05::tmem_st8(tK + 16 * part + 8 * v, y);
              } else {
                uint32_t pick[8];  // by group and half of its byte
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  // code c of a byte picks bytes 2 c and 2 c + 1 of its group's values
                  const uint32_t a = (x >> (4 * e) & 0x03030303u) * 0x22u + 0x10101010u;
                  const uint32_t b = (x >> (4 * e + 2) & 0x03030303u) * 0x22u + 0x10101010u;
                  pick[e] = __byte_perm(a, b, 0x5140);
                  pick[4 + e] = __byte_perm(a, b, 0x7362);
                  pick[2 + e] = pick[e] >> 16;
                  pick[6 + e] = pick[4 + e] >> 16;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __byte_perm(value[e / 2][0], value[e / 2][1], pick[e]);
                tc05::tmem_st8(tK + 16 * part + 8 * v, y);
              }
            }
          }
          if constexpr (!kCompact) {
            const uint32_t y[8] = {least[0][0], least[0][1], least[0][2], least[0][3],
                                   least[1][0], least[1][1], least[1][2], least[1][3]};
            tc05::tmem_st8(tK + 64, y);
          }
          arrive(&S.raw_empty[r]);
        } else {
          const int i = kKeys * (tile - p.I()) + key;
          if (nk >= kKs && !wait(&S.k_empty[s], nk / kKs - 1)) break;
          const uint4* src = nullptr;
          ok = i < p.n_win;
          if (ok) {
            const int row = win_row(win_pos(i, p.n, A.sink, A.recent), A.sink, A.recent);
            src = reinterpret_cast<const uint4*>(
                A.win.win + ((((size_t)p.slot * A.h_kv + p.h) * 2) * (A.sink + A.recent) + row) * kD);
          }
          float top = 0.f;  // of the centered key
#pragma unroll 1
          for (int part = 0; part < 2; ++part) {
            uint4 x[8];  // all on their way at once
#pragma unroll
            for (int v = 0; v < 8; ++v) x[v] = src ? __ldcg(src + 8 * part + v) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int v = 0; v < 8; v += 2) {
              const uint32_t y[8] = {x[v].x, x[v].y, x[v].z, x[v].w, x[v + 1].x, x[v + 1].y, x[v + 1].z, x[v + 1].w};
              tc05::tmem_st8(tK + 32 * part + 4 * v, y);
              if (!kSum) {
                const float2* mu = reinterpret_cast<const float2*>(A.mu + (size_t)p.h * kD + 64 * part + 8 * v);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const float2 m = __ldg(mu + e);
                  top = fmaxf(top, fmaxf(fabsf(__uint_as_float(y[e] << 16) - m.x),
                                         fabsf(__uint_as_float(y[e] & 0xffff0000u) - m.y)));
                }
              }
            }
          }
          scale = __float_as_uint(top);
        }
        S.scale[nk % kRing][key] = scale;
        const uint32_t counts = __ballot_sync(0xffffffffu, ok);
        if (lane == 0) S.counts[nk % kRing][quarter] = counts;
        tc05::tmem_wait_st();
        tc05::fence_before();
        arrive(&S.k_full[s]);
      }
      if (dead) break;
    }
  } else {
    tc05::reg_dec<Roles::kIssue>();
    if (warp == kCopyWarp) {
      // ------------------------------------------------------------- copies
      uint32_t raws = 0, nq = 0;
      ScorePiece p;
      for (uint32_t n = 0; next_piece(n, p); ++n) {
        if (n > 0 && !wait(&S.q_empty, n - 1)) break;
        const uint32_t bytes = (uint32_t)(p.N() + 7) / 8 * 2048, line = (uint32_t)p.N() * 4;
        if (lane == 0) {
          const uint8_t* src = qop_of(A, p.seg);
          const int all = win ? 3 : 2, kinds = p.t1 > p.I() ? 3 : 2;  // as given for window tiles
          const uint32_t ext = kCompact ? 0u : (uint32_t)(p.N() + 7) / 8 * 256;
          tc05::bar_arrive_expect_tx(&S.q_full, kinds * bytes + ext + (1 + kCompact) * line + 16);
          for (int i = 0; i < kinds; ++i) tc05::bulk_g2s(S.q[i], src + (size_t)A.cols * 256 * i, bytes, &S.q_full);
          if (!kCompact) tc05::bulk_g2s(S.ext, src + (size_t)A.cols * 256 * all, ext, &S.q_full);
          const uint8_t* c = src + qop_lines(A.cols, win, kCompact);
          tc05::bulk_g2s(S.off, c, line, &S.q_full);
          if (kCompact) tc05::bulk_g2s(S.sum, c + (size_t)A.cols * 4, line, &S.q_full);
          tc05::bulk_g2s(&S.block, c + (size_t)A.cols * 8, 16, &S.q_full);
        }
        __syncwarp();
        ++nq;
        // lane: page of the tile, codes (0 .. 7) or pairs (8 .. 15); entries a tile ahead
        auto request = [&](int tile) {
          const int i = kKeys * tile + kPage * (lane & 7);
          return tile < min(p.t1, p.I()) && lane < 16 && i < p.n_int
                     ? __ldcg(A.bt + (size_t)p.b * A.max_pages + (A.sink + i) / kPage) : -1;
        };
        int page = request(p.t0);
        for (int tile = p.t0; tile < min(p.t1, p.I()); ++tile, ++raws) {
          const uint32_t r = raws % kRaw;
          const int ahead = request(tile + 1);
          if (raws >= kRaw && !wait(&S.raw_empty[r], raws / kRaw - 1)) break;
          const bool in = page >= 0 && page < A.num_pages;
          const uint32_t pages = __ballot_sync(0xffffffffu, in) & 0xffu;
          constexpr int kLanes = meta_stride(kCompact);  // 16-byte pieces of a page's pairs
          if (lane == 0) {
            S.pages[r] = pages;
            if (kNarrow)
              tc05::bar_arrive(&S.raw_full[r]);
            else
              tc05::bar_arrive_expect_tx(&S.raw_full[r], __popc(pages) * (512u + 16u * kLanes));
          }
          if (!in && lane < 8 && kKeys * tile + kPage * lane < p.n_int) atomicOr(A.err, OPTR_DEVERR_PAGE_ID);
          __syncwarp();
          if constexpr (kNarrow) {
            // Plain asynchronous copies.  As bulk copies, 16 small ones a tile, they take 0.8 us: more
            // than all else of a narrow tile (16 x 8 over 8192: 119 us, so 100), less than a wide one
            // (16 x 32: 164 us, so 172).
            auto copy = [&](int x, uint32_t to, uint32_t from) {
              const int phys = __shfl_sync(0xffffffffu, page, x);
              const bool ok = pages >> x & 1;
              cp_async16_zfill(S.raw[r][x] + to,
                               A.pool + ((size_t)(ok ? phys : 0) * A.h_kv + p.h) * chunk_bytes(kCompact) + from, ok);
            };
#pragma unroll
            for (int x = 0; x < 8; ++x) copy(x, 16 * lane, OPTR_K_CODES_OFFSET + 16 * lane);
#pragma unroll
            for (int x = 0; x < 8 * kLanes / 32; ++x)
              copy(x * (32 / kLanes) + lane / kLanes, 512 + 16 * (lane % kLanes),
                   OPTR_K_META_OFFSET + 16 * (lane % kLanes));
            tc05::bar_arrive_copies(&S.raw_full[r]);
          } else if (in) {
            const uint8_t* src = A.pool + ((size_t)page * A.h_kv + p.h) * chunk_bytes(kCompact);
            const bool codes = lane < 8;
            tc05::bulk_g2s(S.raw[r][lane & 7] + (codes ? 0 : 512),
                           src + (codes ? OPTR_K_CODES_OFFSET : OPTR_K_META_OFFSET), codes ? 512u : 16u * kLanes,
                           &S.raw_full[r]);
          }
          __syncwarp();
          page = ahead;
        }
        if (dead) break;
      }
      // copies in flight land before the CTA exits
      if (nq) tc05::bar_wait_drain(&S.q_full, (nq - 1) & 1);
      if (kNarrow) cp_async_commit(), cp_async_wait<0>();
      for (uint32_t x = raws > kRaw ? raws - kRaw : 0; x < raws; ++x)
        tc05::bar_wait_drain(&S.raw_full[x % kRaw], x / kRaw & 1);
      __syncwarp();
    } else if (warp == kMmaWarp) {
      // ----------------------------------------------------------- products
      const uint32_t sq = tc05::smem_addr(S.q[0]), ext = tc05::smem_addr(S.ext);
      uint32_t nk = 0, nu = 0;
      bool used = false;
      ScorePiece p;
      for (uint32_t n = 0; next_piece(n, p); ++n) {
        const int N = p.N();
        const bool pair = !kNarrow && p.cols() > kKeys;
        if (!wait(&S.q_full, n)) break;
        used = true;
        for (int t = 0; t < p.t1 - p.t0; ++t, ++nk) {
          const uint32_t s = nk % kKs, a = tmem + Tmem::kColK + Tmem::kKeyCols * s;
          const bool exact = p.t0 + t >= p.I();
          if (!wait(&S.k_full[s], nk / kKs)) break;
          for (int d = 0; d < (pair ? 2 : 1); ++d) {
            const uint32_t D = nu % kDs;
            const uint32_t id = tc05::idesc_f16(128, pair && d ? N - kKeys : min(N, kKeys));
            if (nu >= kDs && !wait(&S.d_empty[D], nu / kDs - 1)) break;
            ++nu;
            const uint32_t out = tmem + kColD + Tmem::kDCols * D, b = sq + (uint32_t)d * (kKeys * 256);
            constexpr uint32_t kPart = Smem::kCols * 256;
            if (exact) {
              tc05::mma128_ts<16>(out, a, tc05::smem_desc(b + 2 * kPart, 128, 2048), id | tc05::kIdescBf16, 0);
            } else if (kCompact) {
              tc05::mma128_ts<16>(out, a, tc05::smem_desc(b + kPart, 128, 2048), id, 0);
              tc05::mma128_ts<16>(out, a, tc05::smem_desc(b, 128, 2048), id, 1);
            } else {
              // the small parts first: half of the steps round at the sum's size
              tc05::mma128_ts<16>(out, a, tc05::smem_desc(b + kPart, 128, 2048), id, 0);
              tc05::mma16_ts(out, a + 64, tc05::smem_desc(ext + (uint32_t)d * (kKeys * 32), 128, 256), id, 1);
              tc05::mma128_ts<16>(out, a, tc05::smem_desc(b, 128, 2048), id, 1);
            }
            tc05::mma_commit_warp(&S.d_full[D][kSum || !pair ? t & 1 : d]);
          }
          if (dead) break;
          tc05::mma_commit_warp(&S.k_empty[s]);
        }
        if (dead) break;
        tc05::mma_commit_warp(&S.q_empty);
      }
      if (used) {  // the tensor core is done with tensor memory before it is freed
        tc05::mma_commit_warp(&S.drained);
        tc05::bar_wait_drain(&S.drained, 0);
      }
      __syncwarp();
    } else if (warp == kPlanWarp) {
      // ------------------------------------------------------------- pieces
      ScoreFinder<Tiles> next;
      next.start(A, w, A.W);
      bool more = true;
      for (uint32_t n = 0; more; ++n) {
        const uint32_t i = n % kPieces;
        ScorePiece p;
        p.t0 = p.t1 = 0;
        if (next.f < next.f1) next.next(A, p);
        if (kSum) next.workers(A, p);
        more = p.t1 > p.t0;
        if (n >= kPieces && !wait(&S.piece_empty[i], n / kPieces - 1)) break;
        if (lane == 0) {
          S.piece[i] = p;
          tc05::bar_arrive(&S.piece_full[i]);
        }
        __syncwarp();
      }
    }
  }

  tc05::fence_before();
  __syncthreads();
  if (S.abort && tid == 0) atomicOr(A.err, OPTR_DEVERR_TIMEOUT);
  if (warp == kMmaWarp) {
    tc05::fence_after();
    tc05::tmem_dealloc(tmem, kTmemCols);
  }
}

// ---------------------------------------------------------------- host

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

struct ScoreLayout {
  size_t part, total;
  int cols, W;
};

ScoreLayout score_layout(const optr_params* p, int B, int max_new) {
  ScoreLayout l;
  l.cols = (4 * std::min(max_new, kTok) + 15) / 16 * 16;
  l.W = p->num_sms;
  const size_t segs = (size_t)B * p->cfg.h_kv;
  l.part = round_up(segs * qop_bytes(l.cols, p->cfg.sink + p->cfg.recent > 0, p->cfg.group == 4 * kG));
  l.total = l.part + round_up((segs + l.W) * 2 * kKeys * sizeof(float2));
  return l;
}

}  // namespace
}  // namespace optr

using namespace optr;

extern "C" size_t optr_kv_score_workspace_size(const optr_params* p, int n_tok, int B, int max_new,
                                               int max_pages) {
  if (!p || n_tok < 0 || B <= 0 || max_new <= 0 || max_pages <= 0) return 0;
  // (it holds every smaller call's work, whichever form that takes)
  return std::max(score_layout(p, B, max_new).total,
                  few_layout(p, B, std::min(max_new, kFewTok), max_pages).total);
}

extern "C" optr_status optr_kv_score_win(const optr_params* p, const void* q, int n_tok,
                                         const int32_t* cu_new, const int32_t* pos0, int max_new,
                                         const int32_t* block_table, int B, int max_pages,
                                         const uint8_t* pool, int num_pages, const void* win,
                                         const int32_t* win_slot, int n_slots, float* score, int n_score,
                                         void* workspace, size_t ws_bytes, cudaStream_t stream) {
  if (!p || n_tok < 0 || B <= 0 || max_pages <= 0 || num_pages <= 0 || max_new <= 0 || n_score <= 0)
    return OPTR_ERR_INVALID_ARG;
  if (n_tok == 0) return OPTR_OK;
  if (!q || !cu_new || !pos0 || !block_table || !pool || !score || !aligned(q, 16) || !aligned(pool, 16) ||
      !aligned(score, 4))
    return OPTR_ERR_INVALID_ARG;
  WinArgs w{nullptr, nullptr, 0};
  if (p->cfg.sink + p->cfg.recent > 0) {
    if (!win || !win_slot || n_slots <= 0 || !aligned(win, 16)) return OPTR_ERR_INVALID_ARG;
    w = WinArgs{(__nv_bfloat16*)const_cast<void*>(win), win_slot, n_slots};
  }
  if ((long long)B * p->cfg.h_kv > 65535 || (long long)max_pages * kPage > (1LL << 30) || n_tok > (1 << 24))
    return OPTR_ERR_OUT_OF_RANGE;
  const ScoreLayout l = score_layout(p, B, max_new);
  if (!workspace || ws_bytes < optr_kv_score_workspace_size(p, n_tok, B, max_new, max_pages) || !aligned(workspace, 256)) return OPTR_ERR_WORKSPACE;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  ScoreArgs A{static_cast<const __nv_bfloat16*>(q), n_tok, cu_new, pos0, max_new, 0, block_table, B, max_pages,
              pool, num_pages, w, p->cfg.sink, p->cfg.recent, p->cfg.h_kv, p->cfg.group == 4 * kG, p->R_k, p->mu,
              score, n_score, p->err, l.cols, ws, (float2*)(ws + l.part), l.W};
  if (few_tokens(p, B, max_new, max_pages)) return cuda_status(launch_score_few(p, A, ws, stream));
  const bool narrow = l.cols <= Smem<false, true>::kCols;
  auto first = A.compact ? logit_kernel<false, true, false> : logit_kernel<false, false, false>;
  auto second = A.compact ? logit_kernel<true, true, false> : logit_kernel<true, false, false>;
  const int threads = narrow ? Roles<true>::kThreads : Roles<false>::kThreads;
  size_t smem = A.compact ? sizeof(Smem<true, false>) : sizeof(Smem<false, false>);
  if (narrow) {
    first = A.compact ? logit_kernel<false, true, true> : logit_kernel<false, false, true>;
    second = A.compact ? logit_kernel<true, true, true> : logit_kernel<true, false, true>;
    smem = A.compact ? sizeof(Smem<true, true>) : sizeof(Smem<false, true>);
  }
  if (ensure_dynamic_smem(reinterpret_cast<const void*>(query_kernel), sizeof(QuerySmem)) != cudaSuccess ||
      ensure_dynamic_smem(reinterpret_cast<const void*>(first), smem) != cudaSuccess ||
      ensure_dynamic_smem(reinterpret_cast<const void*>(second), smem) != cudaSuccess)
    return OPTR_ERR_CUDA;
  const unsigned segs = (unsigned)B * p->cfg.h_kv;
  // a block of tokens a time, in stream order: the sums do not depend on chance
  cudaError_t e = cudaSuccess;
  const int most = std::min(max_new, n_tok);  // no sequence has more
  for (A.t0 = 0; A.t0 < most && e == cudaSuccess; A.t0 += kTok) {
    const int parts = (l.cols + kRotCols - 1) / kRotCols;
    e = launch_pdl_cluster(query_kernel, dim3(parts, segs), dim3(kRotThreads), parts, sizeof(QuerySmem), stream, A);
    if (e == cudaSuccess) e = launch_pdl(first, dim3(l.W), dim3(threads), smem, stream, A);
    if (e == cudaSuccess) e = launch_pdl(second, dim3(l.W), dim3(threads), smem, stream, A);
  }
  return cuda_status(e);
}

extern "C" optr_status optr_kv_score(const optr_params* p, const void* q, int n_tok, const int32_t* cu_new,
                                     const int32_t* pos0, int max_new, const int32_t* block_table, int B,
                                     int max_pages, const uint8_t* pool, int num_pages, float* score,
                                     int n_score, void* workspace, size_t ws_bytes, cudaStream_t stream) {
  if (p && (p->cfg.sink > 0 || p->cfg.recent > 0)) return OPTR_ERR_INVALID_ARG;
  return optr_kv_score_win(p, q, n_tok, cu_new, pos0, max_new, block_table, B, max_pages, pool, num_pages,
                           nullptr, nullptr, 0, score, n_score, workspace, ws_bytes, stream);
}
