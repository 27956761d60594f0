// Attention of a chunk of new tokens over the paged INT2 cache
// (include/optr.h, "optr_chunk_attention").
//
// Two launches: chunk_kernel attends, chunk_combine_kernel joins the segments
// that more than one CTA worked on.
//
// Work.  A query block is 64 new tokens of one sequence with the 4 query heads
// of one KV head: 256 rows, two tensor-core tiles of 32 tokens x 4 heads.  It
// goes over its keys in tiles of 128: the cached INT2 positions, the windows'
// rows, then the chunk's own tokens up to its diagonal.  All tiles of all
// (sequence, KV head, query block) segments are put into one line that is cut
// into equal ranges, one per SM: a long context of one sequence, a ragged batch
// and a causal prompt (whose blocks see between one tile and all) fill the GPU
// alike, and a CTA leaves at most two partial results.  A block of 32 tokens or
// fewer is one query tile, whose key tiles the two softmax groups take in turn.
//
// Bound.  Chunk tokens (bf16): the tensor cores; an 8192-token prompt of 32 heads
// takes 408 us, 1.35 PFLOP/s.  INT2 tiles: the chain of a tile, no one part of it.
// A 128-key tile is 64 KB of fp16 operands written (two warpgroups, from the
// records' 12 KB) and 96 KB read per query tile by its two products, 1.4 us for
// one query tile and 2.0 us for two; 2048 tokens over 32768 take 885 us, 16 x 5 over
// 8192 80 us and 8 over 131072 77 us, the records alone at 1.3 TB/s.  Of up to 8 new
// tokens all rows lie in one quarter of the query tile, so one warp of each softmax
// group has them all.
//
// A row's softmax runs over the tiles with a running maximum m and sum l
// (float32, log2 domain); O and m, l of different ranges merge exactly.
// The INT2 keys and values live in their rotated bases, all others in the
// model's.  Keys: the query operand changes with the tile's kind (q R_k in fp16,
// scaled by a power of two per row; q itself in bf16, and the constant <q, mu>
// taken off).  Values: O is normalised and multiplied by R_v^T once, after the
// last INT2 tile, and the other tiles go on from there.
//
// Both operands of a product have one type: fp16 where the keys and values are
// dequantized (their codes, scales and minima are fp16, and 11 bits of the query,
// the weights and the normalised O lose less than 8), bf16 where they are given so.
// Of R_v^T the fp16 part alone is taken: its lo part would cost a product more at
// a segment's end for 2^-12 of an element, under the output's 2^-9.
#include "append_common.cuh"
#include "chunk.cuh"
#include "dequant.cuh"
#include "f32x2.cuh"
#include "tc05.cuh"
#include "tmap.cuh"

#include <algorithm>

namespace optr {
namespace {

// ----------------------------------------------------------- attention

// Warpgroups: two of softmax, two of keys and values, one of two TMA warps, the
// MMA warp and the one that finds the CTA's pieces.  Registers a thread after the
// split, of the launch's 640 x 96.
constexpr int kDeqWarp = 8, kTmaWarp = 16, kMmaWarp = 18, kPlanWarp = 19;
constexpr int kThreads = 640;
constexpr int kRegLaunch = 96, kRegSoftmax = 128, kRegDeq = 72, kRegIssue = 72;
static_assert(2 * kRegSoftmax + 2 * kRegDeq + kRegIssue <= 5 * kRegLaunch, "registers of the launch");
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256;  // S[g] (and P[g]) at 128 g, O[g] at 256 + 128 g
constexpr int kRing = 2;
constexpr uint32_t kHalf = kTile * 128;      // 64 channels of 128 rows
constexpr uint32_t kOperand = 2 * kHalf;     // 128 x 128 of 16 bits
constexpr int kPieces = 3;       // pieces found ahead
constexpr float kSlack = 8.f;  // a row's maximum may grow by 2^8 before O is rescaled
// The largest weight stands at 2^kLift, with the slack at 2^15 at most, inside fp16:
// weights count down to 2^-32 of it, and a million keys below that weigh 2^-12.
constexpr float kLift = 7.f;

struct Smem {
  uint8_t q[2][kOperand];            // the query operand, by tile
  uint8_t k[kRing][kOperand];        // keys by tile
  uint8_t v[kRing][kOperand];        // values by tile; R_v^T
  uint8_t raw[2][8][kChunk];         // records of a tile's pages, as in the pool
  // INT2 tiles: keys whose page is in range.  Read between the tile's logits
  // and its probabilities: by when K of tile t + 4 may be written, the logits of
  // t + 2 are done, so the probabilities of t + 1.
  alignas(16) uint32_t mask[4][4];
  // what the first softmax group tells the second of a query tile that they
  // share, and the second the first of its part of the output
  float scale[128], off[128];
  float2 ml[128];
  Piece piece[kPieces];
  // dequantized, brought by TMA, free again; v_full also after v_tma, once the
  // rows that do not count are cleared
  uint64_t k_full[kRing], k_tma[kRing], k_empty[kRing];
  uint64_t v_full[kRing], v_tma[kRing], v_empty[kRing];
  uint64_t k_grant[2][kRing], v_grant[2][kRing];  // a slot is the dequantizing group's
  uint64_t raw_full[2], raw_empty[2], second_ready, joined;
  uint64_t piece_full[kPieces], piece_empty[kPieces];
  uint64_t s_full[2], p_ready[2], o_full[2], q_ready[2], q_full, q_empty, drained;
  uint32_t tmem;
  int abort;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <bool kBf16>
__device__ __forceinline__ uint32_t pack16(float a, float b) {  // a in the low half
  uint32_t r;
  if (kBf16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// 32 bytes of a row, in one piece where the rows are aligned so: a thread
// writes its own row, so every store of the warp touches 32 lines.
__device__ __forceinline__ void store32(void* p, const uint32_t (&y)[8], bool whole) {
  if (whole) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(y[0]), "r"(y[1]),
                 "r"(y[2]), "r"(y[3]), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7]) : "memory");
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(y[0], y[1], y[2], y[3]);
    static_cast<uint4*>(p)[1] = make_uint4(y[4], y[5], y[6], y[7]);
  }
}

// One row of a logit tile: S (128 columns of tensor memory at tS) becomes P =
// 2^(S scale - off - m) in 16 bits over its first 64 columns; m, l and O are
// brought along.  Bits of `mask` and the first `lim` columns count.  l sums the weights
// before they are rounded (each by up to 2^-11 of it in fp16, 2^-8 in bf16, to either side).
template <bool kBf16>
__device__ __forceinline__ void softmax_tile(uint32_t tS, uint32_t tO, float scale, float off,
                                             uint4 mask, int lim, bool fresh, float& m, float& l) {
  const bool whole = __all_sync(0xffffffffu, lim >= kTile) &&
                     (mask.x & mask.y & mask.z & mask.w) == 0xffffffffu;
  // chunk c of the row, the columns that do not count at -infinity
  auto load = [&](int c, uint32_t (&s)[32]) {
    tc05::tmem_ld32(tS + 32 * c, s);
    tc05::tmem_wait_ld();
    if (!whole) {
      const int n = lim - 32 * c;
      const uint32_t word = c == 0 ? mask.x : c == 1 ? mask.y : c == 2 ? mask.z : mask.w;
      const uint32_t k = word & (n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u);
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (!(k >> j & 1)) s[j] = 0xff800000u;
    }
  };
  float x[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    uint32_t s[32];
    load(c, s);
#pragma unroll
    for (int j = 0; j < 32; j += 8)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = fmaxf(x[i], fmaxf(__uint_as_float(s[j + i]), __uint_as_float(s[j + 4 + i])));
  }
  const float t = fmaf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), scale, -off) - kLift;
  if (fresh) {
    m = fmaxf(m, t);
  } else if (__any_sync(0xffffffffu, t > m + kSlack)) {
    const float mn = t > m + kSlack ? t : m, al = ex2(m - mn);
    m = mn;
    l *= al;
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
      uint32_t o[32];
      tc05::tmem_ld32(tO + 32 * c, o);
      tc05::tmem_wait_ld();
#pragma unroll
      for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * al);
      tc05::tmem_st32(tO + 32 * c, o);
    }
  }
  const float2 scale2 = make_float2(scale, scale), sub2 = make_float2(-(off + m), -(off + m));
  float2 sum[2] = {};
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    uint32_t s[32], p[16];
    load(c, s);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float2 y = fma2(make_float2(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1])),
                            scale2, sub2);
      const float2 e = make_float2(ex2(y.x), ex2(y.y));
      sum[j & 1] = add2(sum[j & 1], e);
      p[j] = pack16<kBf16>(e.x, e.y);
    }
    tc05::tmem_st16(tS + 16 * c, p);
  }
  const float2 total = add2(sum[0], sum[1]);
  l += total.x + total.y;
  tc05::tmem_wait_st();
}

// One row of the rotated queries (128 columns of tensor memory at tS) as the
// INT2 tiles' query operand: fp16 over a power of two >= its largest value, so
// that no query leaves fp16's range.  The logit of an INT2 key is then
// S scale - off, in the units of the other keys' <q, k>: -off carries <q, mu>,
// which centering took from the keys.
__device__ __forceinline__ void rotated_query(uint32_t tS, uint8_t* q, int row, const float* muR,
                                              float& scale, float& off) {
  float top = 0.f, dot = 0.f;
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    uint32_t s[32];
    tc05::tmem_ld32(tS + 32 * c, s);
    tc05::tmem_wait_ld();
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      top = fmaxf(top, fabsf(__uint_as_float(s[k])));
      dot = fmaf(__uint_as_float(s[k]), __ldg(muR + row_channel(k) + 8 * c), dot);
    }
  }
  const int E = min(max((int)(__float_as_uint(top) >> 23) - 126, -120), 120);
  const float down = __uint_as_float((uint32_t)(127 - E) << 23);
  scale = __uint_as_float((uint32_t)(127 + E) << 23) * kLogit;
  off = -dot * kLogit;
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    uint32_t s[32];
    tc05::tmem_ld32(tS + 32 * c, s);
    tc05::tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        y[e] = pack16<false>(__uint_as_float(s[8 * i + 2 * e]) * down,
                             __uint_as_float(s[8 * i + 2 * e + 1]) * down);
      const int piece = 4 * (c & 1) + i;  // of the channel half c / 2
      *reinterpret_cast<uint4*>(q + (c >> 1) * kHalf + row * 128 + ((piece ^ (row & 7)) << 4)) =
          make_uint4(y[0], y[1], y[2], y[3]);
    }
  }
}

__global__ void __launch_bounds__(kThreads, 1)
chunk_kernel(const __grid_constant__ CUtensorMap tm_q,
             const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
             const __grid_constant__ CUtensorMap tm_win, const __grid_constant__ ChunkArgs A) {
  extern __shared__ __align__(1024) unsigned char dsm_[];
  Smem& S = *reinterpret_cast<Smem*>(dsm_);
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // uniform, as the compiler sees it
  if (tid == 0) {
    for (int s = 0; s < kRing; ++s) {
      tc05::bar_init(&S.k_full[s], 128);
      tc05::bar_init(&S.k_tma[s], 1);
      tc05::bar_init(&S.k_empty[s], 1);
      tc05::bar_init(&S.v_full[s], 128);
      tc05::bar_init(&S.v_tma[s], 1);
      tc05::bar_init(&S.v_empty[s], 1);
      for (int g = 0; g < 2; ++g) {
        tc05::bar_init(&S.k_grant[g][s], 1);
        tc05::bar_init(&S.v_grant[g][s], 1);
      }
    }
    for (int i = 0; i < kPieces; ++i) {
      tc05::bar_init(&S.piece_full[i], 1);
      tc05::bar_init(&S.piece_empty[i], kPlanWarp);
    }
    for (int g = 0; g < 2; ++g) {
      tc05::bar_init(&S.s_full[g], 1);
      tc05::bar_init(&S.p_ready[g], 4);
      tc05::bar_init(&S.o_full[g], 1);
      tc05::bar_init(&S.q_ready[g], 4);
      tc05::bar_init(&S.raw_full[g], 1);
      tc05::bar_init(&S.raw_empty[g], 4);
    }
    tc05::bar_init(&S.second_ready, 4);
    tc05::bar_init(&S.joined, 4);
    tc05::bar_init(&S.q_full, 1);
    tc05::bar_init(&S.q_empty, 1);
    tc05::bar_init(&S.drained, 1);
    S.abort = (tc05::smem_addr(S.q[0]) & 1023u) != 0;  // the swizzle's alignment
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
  // the CTA's n-th piece, as every warp but the finder's takes it; false after the last
  auto next_piece = [&](uint32_t n, Piece& p) {
    const uint32_t i = n % kPieces;
    if (dead || !wait(&S.piece_full[i], n / kPieces)) return false;
    p = S.piece[i];
    arrive(&S.piece_empty[i]);
    return p.t1 > p.t0;
  };
  if (warp < kDeqWarp)
    tc05::reg_inc<kRegSoftmax>();
  else if (warp < kTmaWarp)
    tc05::reg_dec<kRegDeq>();
  else
    tc05::reg_dec<kRegIssue>();
  if (warp < kDeqWarp) {
    // ------------------------------------------------------------- softmax
    const int g = warp >> 2, row = 32 * (warp & 3) + lane;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t tS = tmem + lanes + kColS + 128u * g, tO = tmem + lanes + kColO + 128u * g;
    uint32_t nk = 0, ns = 0, no = 0, nj = 0;  // key tiles of the CTA; S, O and joining phases
    auto ready = [&]() {  // the warp's rows of P are in tensor memory
      tc05::fence_before();
      arrive(&S.p_ready[g]);
    };
    Piece p;
    for (uint32_t n = 0; next_piece(n, p); ++n) {
      const int all_tiles = p.t1 - p.t0, nint = p.int_tiles();
      const uint32_t base = nk + (nint > 0);
      nk = base + all_tiles;
      // The groups have a query tile each, or alternate key tiles of the one
      const bool pair = p.q_tiles() == 2;
      const int stride = pair ? 1 : 2, from = pair ? 0 : g;
      const int ints = pair ? nint : (nint + 1 - g) / 2;
      const int tiles = pair ? all_tiles : (all_tiles + 1 - g) / 2;
      const int i = p.qb * kQTok + (pair ? 32 * g : 0) + (row >> 2), j = row & 3;
      const bool valid = i < p.n_new;
      // A warp without a row only keeps the others' phases: what its rows of S, P
      // and O hold stays in them.
      const bool rows = __any_sync(0xffffffffu, valid);
      const size_t at = ((size_t)p.c0 + i) * 4 * A.h_kv + 4 * p.h + j;
      float scale = 0.f, off = 0.f, m = -1e30f, l = 0.f;
      if (nint > 0 && (pair || g == 0)) {
        if (!wait(&S.s_full[g], ns++)) break;
        if (rows) rotated_query(tS, S.q[g], row, A.muR + p.h * kD, scale, off);
        if (!pair) {
          S.scale[row] = scale;
          S.off[row] = off;
        }
        tc05::fence_before();
        tc05::fence_proxy_async();
        arrive(&S.q_ready[g]);
      }
      bool fresh = true;
      for (int k = 0; k < ints; ++k) {
        const int t = from + stride * k;
        if (!wait(&S.s_full[g], ns++)) break;
        if (fresh && !pair) {  // (the first group wrote them before these logits)
          scale = S.scale[row];
          off = S.off[row];
        }
        const uint4 mask = *reinterpret_cast<const uint4*>(S.mask[(base + t) % 4]);
        if (rows)
          softmax_tile<false>(tS, tO, scale, off, mask, p.n_int - kTile * (p.t0 + t), fresh, m,
                              l);
        fresh = false;
        ready();
      }
      if (dead) break;
      if (ints > 0) {
        // O / l into the model's basis: the A operand of the product with 64
        // R_v^T takes P's place, in fp16; where a row lies too low in fp16's range
        // (a mean over many keys, or small values) over a power of two 2^E > its largest
        if (!wait(&S.o_full[g], no++)) break;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        float down = inv;
        int E = 0;
#pragma unroll 1
        for (int pass = 0; pass < 2 && rows; ++pass) {
          __half2 x = __float2half2_rn(0.f);
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            uint32_t o[32], a[16];
            tc05::tmem_ld32(tO + 32 * c, o);
            tc05::tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              a[e] = pack16<false>(__uint_as_float(o[2 * e]) * down, __uint_as_float(o[2 * e + 1]) * down);
              x = __hmax2(x, __habs2(*reinterpret_cast<const __half2*>(&a[e])));
            }
            tc05::tmem_st16(tS + 16 * c, a);
          }
          tc05::tmem_wait_st();
          const float top = fmaxf(__low2float(x), __high2float(x));
          // from 2^-10 on fp16's steps of 2^-24 are at most 2^-14 of the row's largest
          if (pass == 1 || !__any_sync(0xffffffffu, valid && top < 0x1p-10f)) break;
          E = max((int)(__float_as_uint(top) >> 23) - 126, -24);
          down = inv * __uint_as_float((uint32_t)(127 - E) << 23);
        }
        if (l > 0.f) {  // O is now 2^(6 - E) of weight 2^m l / 2^(6 - E)
          m += __log2f(l) - (float)(6 - E);
          l = __uint_as_float((uint32_t)(133 - E) << 23);
        }
        ready();
      }
      for (int k = ints; k < tiles; ++k) {
        if (!wait(&S.s_full[g], ns++)) break;
        // window rows as far as they are filled; own tiles causally
        const int tile = p.t0 + from + stride * k - p.I;
        const int lim = tile < p.Wt ? p.n_win - kTile * tile : i + 1 - kTile * (tile - p.Wt);
        if (rows)
          softmax_tile<true>(tS, tO, kLogit, 0.f, make_uint4(~0u, ~0u, ~0u, ~0u), lim, fresh, m, l);
        fresh = false;
        ready();
      }
      if (dead || (tiles > 0 && !wait(&S.o_full[g], no++))) break;
      // The groups' parts of one query tile meet: the second's output is in the
      // same lanes of tensor memory
      float u = 1.f, v = 0.f;
      const bool join = !pair && all_tiles > 1;
      if (join && g == 1) {
        S.ml[row] = make_float2(m, l);
        tc05::fence_before();
        arrive(&S.second_ready);
        if (!wait(&S.joined, nj++)) break;
        continue;
      }
      if (!pair && g == 1) continue;
      if (join) {
        if (!wait(&S.second_ready, nj++)) break;
        const float2 o = S.ml[row];
        const float mn = fmaxf(m, o.x);
        u = ex2(m - mn);
        v = ex2(o.x - mn);
        l = l * u + o.y * v;
        m = mn;
      }
      auto output = [&](int c, uint32_t (&o)[32]) {
        tc05::tmem_ld32(tO + 32 * c, o);
        tc05::tmem_wait_ld();
        if (join) {
          uint32_t x[32];
          tc05::tmem_ld32(tO + 128 + 32 * c, x);
          tc05::tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e)
            o[e] = __float_as_uint(__uint_as_float(o[e]) * u + __uint_as_float(x[e]) * v);
        }
      };
      if (all_tiles == p.total) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll 1
        for (int c = 0; c < 4 && rows; ++c) {
          uint32_t o[32];
          output(c, o);
          if (valid)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              uint32_t y[8];
#pragma unroll
              for (int z = 0; z < 8; ++z)
                y[z] = pack16<true>(__uint_as_float(o[16 * e + 2 * z]) * inv,
                                    __uint_as_float(o[16 * e + 2 * z + 1]) * inv);
              store32(A.out + at * kD + 32 * c + 16 * e, y, A.out32);
            }
        }
      } else {
        float* part = part_of(A, w, p.t0 > 0);
        const int r = 128 * g + row;
#pragma unroll 1
        for (int c = 0; c < 4 && rows; ++c) {
          uint32_t o[32];
          output(c, o);
          if (valid)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              reinterpret_cast<uint4*>(part)[(size_t)(8 * c + e) * A.rows + r] =
                  make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        }
        if (valid) {
          part[(size_t)A.rows * kD + r] = m;
          part[(size_t)A.rows * (kD + 1) + r] = l;
        }
      }
      tc05::fence_before();
      if (join) arrive(&S.joined);
    }
  } else if (warp < kTmaWarp) {
    // --------------------------------------------------- keys and values
    // The groups take alternate INT2 tiles, thread = key, in slots that the TMA
    // warps grant them; of the tiles that TMA brings, the group of the slot clears
    // the values that do not count (0 times what lies there need not be 0).
    const int g = (warp - kDeqWarp) >> 2, quarter = warp & 3, key = tid & 127;
    const int ms = meta_stride(A.compact);
    uint32_t nk = 0, nv = 0, nt = 0, raws = 0, tma = 0, grants[2][kRing] = {};
    uint32_t past = 0;  // whether a key or value left fp16's range
    Piece p;
    for (uint32_t n = 0; next_piece(n, p); ++n) {
      const int nint = p.int_tiles(), nother = p.t1 - p.t0 - nint;
      if (nint > 0) {  // R_k's parts: one entry of each ring, brought by TMA
        if (nv % kRing == g) {
          if (!wait(&S.v_tma[g], tma++)) break;
          tc05::bar_arrive(&S.v_full[g]);
        }
        ++nk, ++nv;
      }
      auto request = [&](int t) {
        const int pos = (p.t0 + t) * kTile + key;
        return t < nint && pos < p.n_int
                   ? __ldcg(A.bt + (size_t)p.b * A.max_pages + (A.sink + pos) / kPage) : -1;
      };
      const int t0 = (int)((nt ^ g) & 1);  // the group's first tile of the piece
      int page = request(t0);
      for (int t = 0; t < nint; ++t, ++nk, ++nv, ++nt) {
        if (t % 2 != t0) continue;
        const bool inside = (p.t0 + t) * kTile + key < p.n_int;
        const bool ok = inside && page >= 0 && page < A.num_pages;
        if (inside && !ok) atomicOr(A.err, OPTR_DEVERR_PAGE_ID);
        page = request(t + 2);
        const uint32_t bits = __ballot_sync(0xffffffffu, ok || !inside);
        if (!wait(&S.raw_full[g], raws++)) break;
        // Codes and metadata of both kinds, so that the buffer is free at once.  The
        // halves are read in an order that keeps eight lanes' pieces, 32 B apart,
        // in different banks.
        const uint8_t* raw = S.raw[g][key / kPage];
        const int slot = key % kPage, second = key >> 2 & 1;
        uint4 c[2][2], mm[2];
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
          const uint8_t* x = raw + (kind ? OPTR_V_CODES_OFFSET : OPTR_K_CODES_OFFSET) + 32 * slot;
          const uint4 a = *reinterpret_cast<const uint4*>(x + 16 * second);
          const uint4 b = *reinterpret_cast<const uint4*>(x + 16 * (1 - second));
          c[kind][0] = second ? b : a;
          c[kind][1] = second ? a : b;
          const uint8_t* y = raw + (kind ? vmeta_offset(A.compact) : OPTR_K_META_OFFSET) + ms * slot;
          mm[kind] = make_uint4(0u, 0u, 0u, 0u);  // a row of zeros where the key does not count
          if (ok) {
            if (A.compact)
              mm[kind].x = mm[kind].y = mm[kind].z = mm[kind].w = *reinterpret_cast<const uint32_t*>(y);
            else
              mm[kind] = *reinterpret_cast<const uint4*>(y);
          }
        }
        arrive(&S.raw_empty[g]);
#pragma unroll 1
        for (int kind = 0; kind < 2; ++kind) {
          const uint32_t st = (kind ? nv : nk) % kRing;
          if (!wait(kind ? &S.v_grant[g][st] : &S.k_grant[g][st], grants[kind][st]++)) break;
          if (!kind && lane == 0) S.mask[nk % 4][quarter] = bits;
          uint8_t* dst = (kind ? S.v[st] : S.k[st]) + key * 128;
          const uint4 m = kind ? mm[1] : mm[0];
          const SlotMeta sm = slot_meta(m.x, m.y, m.z, m.w);
          note_range(sm, past);
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            const uint4 y = kind ? (half ? c[1][1] : c[1][0]) : (half ? c[0][1] : c[0][0]);
            const uint32_t word[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t x[8];
              dequant_word(word[i], sm, x);
              *reinterpret_cast<uint4*>(dst + half * kHalf + (((2 * i) ^ (key & 7)) << 4)) =
                  make_uint4(x[0], x[1], x[2], x[3]);
              *reinterpret_cast<uint4*>(dst + half * kHalf + (((2 * i + 1) ^ (key & 7)) << 4)) =
                  make_uint4(x[4], x[5], x[6], x[7]);
            }
          }
          tc05::fence_proxy_async();
          tc05::bar_arrive(kind ? &S.v_full[st] : &S.k_full[st]);
        }
        if (dead) break;
      }
      if (dead) break;
      nk += nother;
      for (int t = nint > 0 ? -1 : 0; t < nother; ++t, ++nv) {  // -1: R_v^T
        const int st = nv % kRing;
        if (st != g) continue;
        if (!wait(&S.v_tma[st], tma++)) break;
        const int tile = p.t0 + nint + t - p.I;
        const int count = tile < p.Wt ? p.n_win - kTile * tile : p.n_new - kTile * (tile - p.Wt);
        if (t >= 0 && count < kTile) {
          if (key >= count) {
            uint8_t* r = S.v[st] + key * 128;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              *reinterpret_cast<uint4*>(r + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
              *reinterpret_cast<uint4*>(r + kHalf + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
            }
          }
          tc05::fence_proxy_async();
        }
        tc05::bar_arrive(&S.v_full[st]);
      }
    }
    if (any_past_range(past)) atomicOr(A.err, OPTR_DEVERR_FP16_RANGE);
  } else if (warp == kTmaWarp || warp == kTmaWarp + 1) {
    // ------------------------------------------------------------ TMA
    // One warp for the queries, records, keys and R_k, one for the values and
    // R_v^T.  They alone wait for the ring's slots, every phase in turn, and grant
    // the dequantizing groups theirs: a wait tells a phase from the next but not
    // from the next but one, and whoever waited for some of the phases only could
    // miss two.
    const bool values = warp != kTmaWarp;
    uint64_t* const empty = values ? S.v_empty : S.k_empty;
    uint64_t* const full = values ? S.v_tma : S.k_tma;
    uint32_t step = 0, nq = 0, nt = 0, fetched = 0, pending[kRing] = {0, 0};
    auto load_q = [&](const Piece& p) {
      if (values || dead || (nq > 0 && !wait(&S.q_empty, nq - 1))) return;
      if (lane == 0) {
        const int tiles = p.q_tiles();
        tc05::bar_arrive_expect_tx(&S.q_full, tiles * kOperand);
        for (int g = 0; g < tiles; ++g)
          for (int c = 0; c < 2; ++c)
            tc05::tma_load_3d(S.q[g] + c * kHalf, &tm_q, 64 * c, 4 * p.h,
                              p.c0 + p.qb * kQTok + 32 * g, &S.q_full);
      }
      ++nq;
    };
    auto free_slot = [&]() {
      return !dead && (step < kRing || wait(&empty[step % kRing], step / kRing - 1));
    };
    auto bring = [&](const uint16_t* operand) {  // a 32 KB operand into the ring
      if (!free_slot()) return;
      const int st = step++ % kRing;
      if (lane == 0) {
        tc05::bar_arrive_expect_tx(&full[st], kOperand);
        tc05::bulk_g2s(values ? S.v[st] : S.k[st], operand, kOperand, &full[st]);
      }
      __syncwarp();
      ++pending[st];
    };
    Piece p;
    for (uint32_t n = 0; next_piece(n, p); ++n) {
      const int nint = p.int_tiles(), nother = p.t1 - p.t0 - nint;
      if (nint > 0) {
        load_q(p);
        // hi and lo of R_k
        bring(A.Rk_query + (size_t)p.h * kRT5Halves + (values ? kD * kD : 0));
        // INT2 tiles: records two tiles ahead, the pages' entries three; lane = page
        auto request = [&](int t) {
          const int pos = (p.t0 + t) * kTile + kPage * lane;
          return t < nint && lane < 8 && pos < p.n_int
                     ? __ldcg(A.bt + (size_t)p.b * A.max_pages + (A.sink + pos) / kPage) : -1;
        };
        auto fetch = [&](int t, int page) {
          if (t >= nint || dead) return;
          const uint32_t x = nt + t, g = x & 1, bytes = chunk_bytes(A.compact);
          if (x >= 2 && !wait(&S.raw_empty[g], x / 2 - 1)) return;
          const bool in = page >= 0 && page < A.num_pages;
          const uint32_t copies = __popc(__ballot_sync(0xffffffffu, in));
          if (lane == 0) tc05::bar_arrive_expect_tx(&S.raw_full[g], copies * bytes);
          __syncwarp();
          if (in)
            tc05::bulk_g2s(S.raw[g][lane], A.pool + ((size_t)page * A.h_kv + p.h) * bytes, bytes,
                           &S.raw_full[g]);
          __syncwarp();
          fetched = x + 1;
        };
        int page = -1;
        if (!values) {
          const int e0 = request(0), e1 = request(1);
          page = request(2);
          fetch(0, e0);
          fetch(1, e1);
        }
        for (int t = 0; t < nint && free_slot(); ++t, ++step) {
          const uint32_t g = (nt + t) & 1;
          arrive(values ? &S.v_grant[g][step % kRing] : &S.k_grant[g][step % kRing]);
          if (!values) {
            fetch(t + 2, page);
            page = request(t + 3);
          }
        }
        nt += nint;
        if (values) bring(A.Rv_back + (size_t)p.h * kRT5Halves);  // hi of 64 R_v^T
      }
      for (int t = 0; t < nother && free_slot(); ++t) {
        const int st = step++ % kRing, tile = p.t0 + nint + t - p.I;
        if (lane == 0) {
          tc05::bar_arrive_expect_tx(&full[st], kOperand);
          for (int c = 0; c < 2; ++c) {
            uint8_t* dst = (values ? S.v[st] : S.k[st]) + c * kHalf;
            if (tile < p.Wt)
              tc05::tma_load_3d(dst, &tm_win, 64 * c, 0,
                                ((p.slot * A.h_kv + p.h) * 2 + values) * (A.sink + A.recent) +
                                    kTile * tile, &full[st]);
            else
              tc05::tma_load_3d(dst, values ? &tm_v : &tm_k, 64 * c, p.h,
                                p.c0 + kTile * (tile - p.Wt), &full[st]);
          }
        }
        __syncwarp();
        ++pending[st];
        if (t == 0) load_q(p);
      }
    }
    // copies in flight land before the CTA exits (after an abort nobody else
    // waits for them)
    for (int s = 0; s < kRing; ++s)
      if (pending[s]) tc05::bar_wait_drain(&full[s], (pending[s] - 1) & 1);
    if (nq) tc05::bar_wait_drain(&S.q_full, (nq - 1) & 1);
    for (uint32_t x = fetched > 2 ? fetched - 2 : 0; x < fetched; ++x)
      tc05::bar_wait_drain(&S.raw_full[x & 1], x / 2 & 1);
    __syncwarp();
  } else if (warp == kPlanWarp) {
    // ---------------------------------------------------------- pieces
    find_pieces<kPieces>(A, w, S.piece, S.piece_full, S.piece_empty, abort);
  } else {
    // ------------------------------------------------------------ MMA
    constexpr uint32_t kId = tc05::idesc_f16(128, 128);
    const uint32_t sq = tc05::smem_addr(S.q[0]), sk = tc05::smem_addr(S.k[0]),
                   sv = tc05::smem_addr(S.v[0]);
    uint32_t nk = 0, nv = 0, nq = 0, np[2] = {0, 0}, nr[2] = {0, 0}, kd[kRing] = {0, 0}, kt[kRing] = {0, 0};
    bool used = false;
    auto wait_k = [&](int phase) {  // keys of tile nk, dequantized or by TMA
      const uint32_t st = nk % kRing;
      return phase ? wait(&S.k_tma[st], kt[st]++) : wait(&S.k_full[st], kd[st]++);
    };
    // S[g] = query tile t times key tile nk
    auto qk = [&](int t, int g, uint32_t type) {
      const uint32_t a = sq + t * kOperand, b = sk + nk % kRing * kOperand;
      tc05::mma128_ss<2, 2, true, true>(tmem + kColS + 128u * g, tc05::smem_desc_sw128(a, 16),
                                        tc05::smem_desc_sw128(b, 16), kId | type, 0);
      tc05::mma_commit_warp(&S.s_full[g]);
    };
    Piece p;
    for (uint32_t n = 0; next_piece(n, p); ++n) {
      const int all_tiles = p.t1 - p.t0, nint = p.int_tiles();
      // Tile u is for both groups (each its query tile), or for group u % 2; the
      // logits of the next one of a group follow its product with the values.
      const bool pair = p.q_tiles() == 2;
      const int ahead = pair ? 1 : 2;
      auto first_of = [&](int u) { return pair ? 0 : u & 1; };
      auto last_of = [&](int u) { return pair ? 1 : u & 1; };
      bool add[2] = {false, false};
      used = true;
      for (int phase = 0; phase < 2 && !dead; ++phase) {
        const int u0 = phase ? nint : 0, u1 = phase ? all_tiles : nint;
        if (u0 == u1) continue;
        const uint32_t type = phase ? tc05::kIdescBf16 : 0u;
        if (!wait(&S.q_full, nq++)) break;
        if (!phase) {  // q R_k, bf16 hi + lo, by way of S
          if (!wait_k(1) || !wait(&S.v_full[nv % kRing], nv / kRing)) break;
          for (int g = 0; g < (pair ? 2 : 1); ++g) {
            const uint32_t a = sq + g * kOperand;
            for (int part = 0; part < 2; ++part) {
              const uint32_t b = part ? sv + nv % kRing * kOperand : sk + nk % kRing * kOperand;
              tc05::mma128_ss<2, 16, true, false>(tmem + kColS + 128u * g, tc05::smem_desc_sw128(a, 16),
                                                  tc05::smem_desc(b, 128, 2048),
                                                  kId | tc05::kIdescBf16, part);
            }
            tc05::mma_commit_warp(&S.s_full[g]);
          }
          tc05::mma_commit_warp(&S.k_empty[nk++ % kRing]);
          tc05::mma_commit_warp(&S.v_empty[nv++ % kRing]);
        }
        for (int u = u0; u < min(u0 + ahead, u1); ++u) {
          if (!wait_k(phase)) break;
          for (int g = first_of(u); g <= last_of(u); ++g) {
            const int t = pair ? g : 0;
            if (!phase && u == u0 && !wait(&S.q_ready[t], nr[t]++)) break;
            qk(t, g, type);
          }
          tc05::mma_commit_warp(&S.k_empty[nk++ % kRing]);
        }
        if (u1 - u0 <= ahead) tc05::mma_commit_warp(&S.q_empty);
        for (int u = u0; u < u1 && !dead; ++u) {
          if (!wait(&S.v_full[nv % kRing], nv / kRing)) break;
          const uint32_t b = sv + nv % kRing * kOperand;
          const bool more = u + ahead < u1;
          for (int g = first_of(u); g <= last_of(u); ++g) {
            if (!wait(&S.p_ready[g], np[g]++)) break;
            tc05::mma128_ts<128>(tmem + kColO + 128u * g, tmem + kColS + 128u * g,
                                 tc05::smem_desc_sw128(b, kHalf), kId | type | tc05::kIdescMajorMnB,
                                 add[g]);
            add[g] = true;
            if (!more) tc05::mma_commit_warp(&S.o_full[g]);
            if (g == last_of(u)) tc05::mma_commit_warp(&S.v_empty[nv % kRing]);
            if (more) {
              if (g == first_of(u) && !wait_k(phase)) break;
              qk(pair ? g : 0, g, type);
            }
          }
          ++nv;
          if (more) tc05::mma_commit_warp(&S.k_empty[nk++ % kRing]);
          if (u + ahead + 1 == u1) tc05::mma_commit_warp(&S.q_empty);
        }
        if (dead || phase) continue;
        // O R_v^T of the groups that have INT2 tiles
        if (!wait(&S.v_full[nv % kRing], nv / kRing)) break;
        for (int g = 0; g < (pair ? 2 : min(nint, 2)); ++g) {
          if (!wait(&S.p_ready[g], np[g]++)) break;
          const uint32_t b = sv + nv % kRing * kOperand;
          tc05::mma128_ts<16>(tmem + kColO + 128u * g, tmem + kColS + 128u * g,
                              tc05::smem_desc(b, 128, 2048), kId, 0);
          // the group has no tile after these
          if (pair ? nint == all_tiles : (all_tiles + 1 - g) / 2 == (nint + 1 - g) / 2)
            tc05::mma_commit_warp(&S.o_full[g]);
        }
        tc05::mma_commit_warp(&S.v_empty[nv++ % kRing]);
      }
    }
    if (used) {  // the tensor core is done with tensor memory before it is freed
      tc05::mma_commit_warp(&S.drained);
      tc05::bar_wait_drain(&S.drained, 0);
    }
    __syncwarp();
  }

  tc05::fence_before();
  __syncthreads();
  if (S.abort && tid == 0) atomicOr(A.err, OPTR_DEVERR_TIMEOUT);
  if (warp == kMmaWarp) {
    tc05::fence_after();
    tc05::tmem_dealloc(tmem, kTmemCols);
  }
}

// ------------------------------------------------------------- combine

// Zero rows t0 .. t1-1, by a whole CTA of 256.  Where the offsets fall somewhere,
// the rows of a sequence that is in order may be among these and stay.  A function
// of its own, so that the calls that have no such rows do not carry its registers
// (16 x 5 over 8192: 80.0 us, 81.1 inlined).
__device__ __noinline__ void clear_rows(const ChunkArgs& A, int t0, int t1) {
  auto any = [&](auto test) {  // of the sequences
    int found = 0;
    for (int b = threadIdx.x; b < A.B; b += 256) found |= test(b);
    return __syncthreads_or(found);
  };
  const bool fall = any([&](int b) { return __ldcg(A.cu + b + 1) < __ldcg(A.cu + b); });
  const int n = A.h_kv * 4 * kD / 8;
  for (int t = t0; t < t1; ++t) {
    if (fall && any([&](int b) {
          const SeqWork x = seq_work(A, b);
          return x.c0 <= t && t < x.c0 + x.n_new;
        }))
      continue;
    uint4* o = reinterpret_cast<uint4*>(A.out) + (size_t)t * n;
    for (int i = threadIdx.x; i < n; i += 256) o[i] = make_uint4(0u, 0u, 0u, 0u);
  }
}

// Joins the partials of the segments that several CTAs had a part in: CTA
// (w, y) rows kRows y .. of the one that CTA w began.  A thread has 4 channels
// of a row and every kSplit-th part: a prefill's segments are of two or three
// parts and many rows (kSplit 1), those of a few tokens over a long context of
// many parts and few rows (kSplit 4).  The CTAs also clear the rows of sequences
// that were left out and those of none.
template <bool kFew>
__global__ void __launch_bounds__(256) chunk_combine_kernel(const __grid_constant__ ChunkArgs A) {
  constexpr int kSplit = kFew ? 4 : 1, kRows = 8 / kSplit;
  __shared__ float4 so[kSplit][kRows][32];
  __shared__ float2 sml[kSplit][kRows];
  const int w = blockIdx.x, tid = threadIdx.x;
  pdl_wait();
  pdl_trigger();
  const ChunkSeg* from = A.seg + w;
  const ChunkSeg seg{__ldcg(&from->F),  __ldcg(&from->end), __ldcg(&from->c0), __ldcg(&from->n_new),
                     __ldcg(&from->h), __ldcg(&from->qb),  __ldcg(&from->W),  __ldcg(&from->valid)};
  auto clear = [&](int t0, int t1) {
    if (t1 > t0) clear_rows(A, t0, t1);
  };
  const int id = w + blockIdx.y * gridDim.x, all = gridDim.x * gridDim.y;
  for (int b = id; b <= A.B; b += all) {
    const int c1 = b < A.B ? __ldcg(A.cu + b + 1) : __ldcg(A.cu);
    if (b == A.B) {
      clear(0, min(c1, A.n_tok));
    } else {
      if (b == A.B - 1) clear(max(c1, 0), A.n_tok);
      if (seq_work(A, b).bad) clear(max(0, __ldcg(A.cu + b)), min(c1, A.n_tok));
    }
  }
  const int row = tid % kRows, split = tid / kRows % kSplit, cg = tid / (kRows * kSplit);
  const int r = kRows * blockIdx.y + row;
  const int i = seg.qb * kQTok + r / 4;
  if (!seg.valid || seg.qb * kQTok + kRows * (int)blockIdx.y / 4 >= seg.n_new) return;
  const bool in = r < A.rows && i < seg.n_new;
  float M = -INFINITY, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto join = [&](float m, float l, float4 y) {
    if (l == 0.f) return;  // no part, or one whose keys were all left out
    const float mn = fmaxf(M, m), u = ex2(M - mn), v = ex2(m - mn);
    M = mn;
    L = L * u + l * v;
    o = make_float4(o.x * u + y.x * v, o.y * u + y.y * v, o.z * u + y.z * v, o.w * u + y.w * v);
  };
  constexpr int kAhead = 4;  // partials requested at a time
  for (int x0 = w + split; x0 < seg.W && seg.F * x0 / seg.W < seg.end; x0 += kAhead * kSplit) {
    float m[kAhead], l[kAhead];
    float4 y[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int x = x0 + k * kSplit;
      l[k] = 0.f;
      if (in && x < seg.W && seg.F * x / seg.W < seg.end) {
        const float* part = part_of(A, x, x != w);
        m[k] = __ldcg(part + (size_t)A.rows * kD + r);
        l[k] = __ldcg(part + (size_t)A.rows * (kD + 1) + r);
        y[k] = __ldcg(reinterpret_cast<const float4*>(part) + (size_t)cg * A.rows + r);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) join(m[k], l[k], y[k]);
  }
  if (kSplit > 1) {
    so[split][row][cg] = o;
    if (cg == 0) sml[split][row] = make_float2(M, L);
    __syncthreads();
    if (split != 0) return;
    for (int k = 1; k < kSplit; ++k) join(sml[k][row].x, sml[k][row].y, so[k][row][cg]);
  }
  if (!in) return;
  const float inv = L > 0.f ? 1.f / L : 0.f;
  const size_t at = ((size_t)seg.c0 + i) * 4 * A.h_kv + 4 * seg.h + r % 4;
  *reinterpret_cast<uint2*>(A.out + at * kD + 4 * cg) =
      make_uint2(pack16<true>(o.x * inv, o.y * inv), pack16<true>(o.z * inv, o.w * inv));
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

// Offsets of a call's workspace, bytes.
struct ChunkLayout {
  size_t part, total;
  int rows, W;
};

ChunkLayout chunk_layout(const optr_params* p, int max_new) {
  ChunkLayout l;
  l.rows = max_new > kQTok / 2 ? 256 : 128;
  l.W = p->num_sms;
  l.part = round_up(sizeof(ChunkSeg) * (size_t)l.W);
  l.total = l.part + round_up(2 * (size_t)l.W * part_floats(l.rows) * sizeof(float));
  return l;
}

}  // namespace
}  // namespace optr

using namespace optr;

extern "C" size_t optr_chunk_workspace_size(const optr_params* p, int n_tok, int B, int max_new) {
  if (!p || n_tok < 0 || B <= 0 || max_new <= 0) return 0;
  return chunk_layout(p, max_new).total;
}

extern "C" optr_status optr_chunk_attention_win(
    const optr_params* p, const void* q, const void* k, const void* v, int n_tok,
    const int32_t* cu_new, const int32_t* pos0, int max_new, const int32_t* block_table, int B,
    int max_pages, const uint8_t* pool, int num_pages, const void* win, const int32_t* win_slot,
    int n_slots, void* out, void* workspace, size_t ws_bytes, cudaStream_t stream) {
  if (!p || n_tok < 0 || B <= 0 || max_pages <= 0 || num_pages <= 0 || max_new <= 0)
    return OPTR_ERR_INVALID_ARG;
  WinArgs w{};
  if (p->cfg.sink > 0 || p->cfg.recent > 0) {
    if (!win || !win_slot || n_slots <= 0 || !aligned(win, 16)) return OPTR_ERR_INVALID_ARG;
    w = WinArgs{static_cast<__nv_bfloat16*>(const_cast<void*>(win)), win_slot, n_slots};
  }
  if (n_tok == 0) return OPTR_OK;
  if (!q || !k || !v || !cu_new || !pos0 || !block_table || !pool || !out) return OPTR_ERR_INVALID_ARG;
  if (!aligned(pool, 16) || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16))
    return OPTR_ERR_INVALID_ARG;
  for (const void* x : {q, k, v, (const void*)out}) {  // TMA reads device memory
    bool host = false;
    if (!io_pointer(x, &x, &host) || host) return OPTR_ERR_INVALID_ARG;
  }
  if ((long long)max_pages * kPage > (1LL << 30) || B > (1 << 24)) return OPTR_ERR_OUT_OF_RANGE;
  const int h_kv = p->cfg.h_kv, win_rows = p->cfg.sink + p->cfg.recent;
  // token and window rows are counted with 32 bits
  if ((long long)n_slots * h_kv * 2 * win_rows >= (1LL << 31)) return OPTR_ERR_OUT_OF_RANGE;
  const ChunkLayout l = chunk_layout(p, max_new);
  if (!workspace || ws_bytes < l.total || !aligned(workspace, 256)) return OPTR_ERR_WORKSPACE;
  char* ws = static_cast<char*>(workspace);
  const ChunkArgs A{n_tok, cu_new, pos0, max_new, block_table, B, max_pages, pool, num_pages, w,
                    p->cfg.sink, p->cfg.recent, h_kv, p->cfg.group == 4 * kG, p->Rk_query, p->Rv_back,
                    p->muR, (__nv_bfloat16*)out, p->err, (ChunkSeg*)ws, (float*)(ws + l.part),
                    l.rows, l.W, aligned(out, 32)};
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(chunk_kernel), sizeof(Smem));
  if (e != cudaSuccess) return OPTR_ERR_CUDA;
  CUtensorMap mq, mk, mv, mw;
  if (!token_rows_map(&mq, q, n_tok, 4 * h_kv, 32, 4) ||
      !token_rows_map(&mk, k, n_tok, h_kv, kTile) || !token_rows_map(&mv, v, n_tok, h_kv, kTile) ||
      !(w.win ? token_rows_map(&mw, w.win, n_slots * h_kv * 2 * win_rows, 1, kTile)
              : token_rows_map(&mw, k, n_tok, h_kv, kTile)))
    return OPTR_ERR_CUDA;
  // few rows of many parts: 8 or more for each (sequence, KV head).  8 drafts over
  // 131072 tokens: 76.8 us, 77.8 without the split; 16 x 5 over 8192, where the
  // rule says no: 80.0, 82.3 with it.
  const bool few = max_new <= 16 && (long long)B * h_kv * 8 <= l.W;
  const int per = few ? 2 : 8;  // rows of a joining CTA
  const dim3 joins(l.W, (std::min(l.rows, 4 * max_new) + per - 1) / per);
  e = launch_pdl(chunk_kernel, dim3(l.W), dim3(kThreads), sizeof(Smem), stream, mq, mk, mv, mw, A);
  if (e == cudaSuccess)
    e = launch_pdl(few ? chunk_combine_kernel<true> : chunk_combine_kernel<false>, joins, dim3(256), 0,
                   stream, A);
  return cuda_status(e);
}

extern "C" optr_status optr_chunk_attention(const optr_params* p, const void* q, const void* k,
                                            const void* v, int n_tok, const int32_t* cu_new,
                                            const int32_t* pos0, int max_new,
                                            const int32_t* block_table, int B, int max_pages,
                                            const uint8_t* pool, int num_pages, void* out,
                                            void* workspace, size_t ws_bytes, cudaStream_t stream) {
  if (p && (p->cfg.sink > 0 || p->cfg.recent > 0)) return OPTR_ERR_INVALID_ARG;
  return optr_chunk_attention_win(p, q, k, v, n_tok, cu_new, pos0, max_new, block_table, B, max_pages,
                                  pool, num_pages, nullptr, nullptr, 0, out, workspace, ws_bytes,
                                  stream);
}
