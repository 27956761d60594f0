// Chunk attention of a few new tokens per sequence (drafted tokens; up to 12):
// chunk.cu's computation with the tiles transposed, so that what is padded is
// the keys' tile (never) and not the queries' (4 to 48 rows):
//   S^T[key][row] = K Q^T,   O^T[channel][row] += V^T P^T
// with M = 128 keys or channels and N = 16, 32 or 48 rows.
//
// One CTA per SM; the pieces of its range as in chunk.cu.  Two warpgroups
// dequantize, alternate tiles, into two-deep rings of key and value tiles; two
// more take the softmax of alternate tiles, each with logits, probabilities and
// an output of its own, which meet at the piece's end.  Per tile of 128 keys 12 KB
// come in, which an SM's share of the memory's rate brings in about 530 cycles;
// its codes take about 600 issue slots of each SM quarter to dequantize, its MMAs
// about 650 cycles (the operands in shared memory, not N, set their pace).
//
// A softmax thread has one key of the tile and its logits with all rows:
// probabilities go into shared memory transposed, the rows' sums are kept per
// thread and added up at the end; a row's maximum is kept for the warpgroup and
// only looked at again when some thread's logit passes it by 2^8.
#include "append_common.cuh"
#include "chunk.cuh"
#include "dequant.cuh"
#include "f32x2.cuh"
#include "tc05.cuh"
#include "tmap.cuh"

namespace optr {
namespace {

constexpr uint32_t kHalf = kTile * 128;       // 64 channels of 128 rows, 16 bits
constexpr uint32_t kOperand = 2 * kHalf;
constexpr float kSlack = 8.f;
constexpr int kRing = 2;
constexpr int kPieces = 3;  // pieces found ahead
constexpr int kRaw = 4;     // tiles of records
// Warpgroups: two of softmax, two of keys and values, one of two TMA warps, the
// MMA warp and the one that finds the CTA's pieces.
constexpr int kDeqWarp = 8, kTmaWarp = 16, kMmaWarp = 18, kPlanWarp = 19;
constexpr int kThreads = 640;
constexpr int kRegLaunch = 96, kRegSoftmax = 128, kRegDeq = 72, kRegIssue = 72;
static_assert(2 * kRegSoftmax + 2 * kRegDeq + kRegIssue <= 5 * kRegLaunch, "registers of the launch");

template <int N>
struct Smem {
  uint8_t k[kRing][kOperand];    // keys by TMA, R_k (dequantized keys: tensor memory)
  uint8_t v[kRing][kOperand];
  uint8_t q[N * kD * 2];         // queries [row][channel or place], two halves of 64
  // probabilities [row][key] by softmax group; O [row][place] for its rotation;
  // at a piece's end both together are the second group's O, float [row][channel]
  uint8_t p[2][N * kTile * 2];
  uint8_t raw[kRaw][8][kChunk];  // records of the tiles' pages, as in the pool
  uint32_t mask[4][4];           // INT2 tiles: keys whose page is in range (as in chunk.cu)
  alignas(16) float mul[2][N], add[2][N];  // logit over the maximum = S mul + add
  float quarter[2][4][N];        // of a group's four warps
  float m[2][N], l[2][N], d[2][N], off[N], scale[N];
  Piece piece[kPieces];
  uint64_t piece_full[kPieces], piece_empty[kPieces];
  uint64_t raw_full[kRaw], raw_empty[kRaw];
  uint64_t k_full[kRing], k_tma[kRing], k_empty[kRing];
  uint64_t v_full[kRing], v_tma[kRing], v_empty[kRing];
  uint64_t k_grant[2][kRing], v_grant[2][kRing];  // a slot is the dequantizing group's
  uint64_t s_full[2], p_ready[2], o_full[2], q_raw, q_ready, q_empty;
  uint64_t first_done, second_ready, joined, drained;
  uint32_t tmem;
  int abort;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}

// The 128 threads of warpgroup g.
__device__ __forceinline__ void group_sync(int g) {
  asm volatile("bar.sync %0, 128;" ::"r"(1 + g) : "memory");
}
__device__ __forceinline__ bool group_any(int g, bool x) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %2, 0;\n"
      " barrier.cta.red.or.pred q, %1, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r) : "r"(1 + g), "r"((uint32_t)x) : "memory");
  return r != 0;
}

// Byte of element (row, i) of a [rows][128] 16-bit operand in two halves of 64
// with the 128-byte swizzle.
template <int N>
__device__ __forceinline__ uint32_t at16(int row, int i) {
  return (i >> 6) * (N * 128) + row * 128 + ((((i >> 3) & 7) ^ (row & 7)) << 4) + (i & 7) * 2;
}

__device__ __forceinline__ uint32_t pack16(float a, float b, bool bf16) {  // a in the low half
  uint32_t r;
  if (bf16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// Columns j, j + 1 of a transposed tile: the thread's element i of rows j, j + 1.
template <int N>
__device__ __forceinline__ void put_pair(uint8_t* base, int j, int i, uint32_t x) {
  *reinterpret_cast<uint16_t*>(base + at16<N>(j, i)) = (uint16_t)x;
  *reinterpret_cast<uint16_t*>(base + at16<N>(j + 1, i)) = (uint16_t)(x >> 16);
}

template <int N>
__global__ void __launch_bounds__(kThreads, 1)
chunk_small_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                   const __grid_constant__ CUtensorMap tm_win, const __nv_bfloat16* __restrict__ q_in,
                   const float* __restrict__ mu, const uint16_t* __restrict__ Rk_row,
                   const __grid_constant__ ChunkArgs A) {
  constexpr uint32_t kColK = 4 * N;                 // after S[2], O[2]: keys by slot, 64 each
  constexpr uint32_t kCols = N <= 32 ? 256 : 512;
  extern __shared__ __align__(1024) unsigned char dsm_[];
  Smem<N>& S = *reinterpret_cast<Smem<N>*>(dsm_);
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
    for (int i = 0; i < kRaw; ++i) {
      tc05::bar_init(&S.raw_full[i], 1);
      tc05::bar_init(&S.raw_empty[i], 4);
    }
    for (int i = 0; i < kPieces; ++i) {
      tc05::bar_init(&S.piece_full[i], 1);
      tc05::bar_init(&S.piece_empty[i], kPlanWarp);
    }
    for (int g = 0; g < 2; ++g) {
      tc05::bar_init(&S.s_full[g], 1);
      tc05::bar_init(&S.p_ready[g], 4);
      tc05::bar_init(&S.o_full[g], 1);
    }
    tc05::bar_init(&S.q_raw, 4);
    tc05::bar_init(&S.q_ready, 4);
    tc05::bar_init(&S.q_empty, 1);
    tc05::bar_init(&S.first_done, 4);
    tc05::bar_init(&S.second_ready, 4);
    tc05::bar_init(&S.joined, 4);
    tc05::bar_init(&S.drained, 1);
    S.abort = (tc05::smem_addr(&S) & 1023u) != 0;  // the swizzle's alignment
    tc05::bar_init_fence();
  }
  if (warp == kMmaWarp) tc05::tmem_alloc(&S.tmem, kCols);
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
    const int g = warp >> 2, quarter = warp & 3, key = tid & 127;
    const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
    const uint32_t tS = tmem + lanes + g * N, tO = tmem + lanes + 2 * N + g * N;
    uint32_t nk = 0, ns = 0, no = 0, nq = 0, nj = 0;  // key tiles; phases
    uint8_t* const P = S.p[g];
    // A warp whose wait ran out leads its group out at the next vote: the group's
    // barriers want all of it.
    Piece p;
    for (uint32_t n = 0;; ++n) {
      const bool more = next_piece(n, p);
      if (group_any(g, dead) || !more) break;
      const int all_tiles = p.t1 - p.t0, nint = p.int_tiles();
      // this group's tiles: those of its parity
      const int tiles = (all_tiles + 1 - g) / 2, ints = (nint + 1 - g) / 2;
      const int rows = 4 * p.n_new;
      const uint32_t base = nk + (nint > 0);
      nk = base + all_tiles;
      float2 l[N / 2];  // the rows' sums over the thread's keys
#pragma unroll
      for (int c = 0; c < N / 2; ++c) l[c] = make_float2(0.f, 0.f);
      bool first = true;  // no maximum yet

      // the rows' queries, as they come or as fp16 over a power of two
      auto load_q = [&](bool rotate) {
        if (nq > 0 && !wait(&S.q_empty, nq - 1)) return;
        ++nq;
#pragma unroll 4
        for (int r = quarter; r < N; r += 4) {
          uint2 x = make_uint2(0u, 0u);
          if (r < rows)
            x = __ldcg(reinterpret_cast<const uint2*>(
                    q_in + (((size_t)p.c0 + r / 4) * 4 * A.h_kv + 4 * p.h + r % 4) * kD) + lane);
          if (rotate) {
            const float a = __uint_as_float(x.x << 16), b = __uint_as_float(x.x & 0xffff0000u);
            const float c = __uint_as_float(x.y << 16), d = __uint_as_float(x.y & 0xffff0000u);
            const float4 mm = __ldg(reinterpret_cast<const float4*>(mu + p.h * kD) + lane);
            float dot = a * mm.x + b * mm.y + c * mm.z + d * mm.w;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
            const float top = warp_max(fmaxf(fmaxf(fabsf(a), fabsf(b)), fmaxf(fabsf(c), fabsf(d))));
            const int E = min(max((int)(__float_as_uint(top) >> 23) - 126, -120), 120);
            const float down = __uint_as_float((uint32_t)(127 - E) << 23);
            if (lane == 0) {
              S.scale[r] = __uint_as_float((uint32_t)(127 + E) << 23) * kLogit;
              S.off[r] = -dot * kLogit;
            }
            x = make_uint2(pack16(a * down, b * down, false), pack16(c * down, d * down, false));
          }
          *reinterpret_cast<uint2*>(S.q + at16<N>(r, 4 * lane)) = x;
        }
        tc05::fence_proxy_async();
      };
      // Eight logits of the thread's key, rows c0 .. c0 + 7, over the rows'
      // maxima; unless all the warp's keys count for all rows, bit c / 4 of `seen`
      // says whether the thread's counts for the rows of new token c / 4.
      auto logits = [&](int c0, uint32_t seen, bool all, float2 (&y)[4]) {
        uint32_t s[8];
        tc05::tmem_ld8(tS + c0, s);
        float mul[8], add[8];
        *reinterpret_cast<float4*>(mul) = *reinterpret_cast<const float4*>(&S.mul[g][c0]);
        *reinterpret_cast<float4*>(mul + 4) = *reinterpret_cast<const float4*>(&S.mul[g][c0 + 4]);
        *reinterpret_cast<float4*>(add) = *reinterpret_cast<const float4*>(&S.add[g][c0]);
        *reinterpret_cast<float4*>(add + 4) = *reinterpret_cast<const float4*>(&S.add[g][c0 + 4]);
        tc05::tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[j] = fma2(make_float2(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1])),
                      make_float2(mul[2 * j], mul[2 * j + 1]), make_float2(add[2 * j], add[2 * j + 1]));
          if (!all && !(seen >> (c0 / 4 + j / 2) & 1)) y[j] = make_float2(-INFINITY, -INFINITY);
        }
      };
      // The rows' maxima anew where a logit has left them behind (or none is
      // there yet), l and O brought along.
      auto new_maxima = [&](uint32_t seen) {
        if (group_any(g, dead)) {
          dead = true;
          return;
        }
#pragma unroll 1
        for (int c0 = 0; c0 < rows; c0 += 8) {
          float2 y[4];
          logits(c0, seen, false, y);
          float z = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float t = warp_max(j & 1 ? y[j / 2].y : y[j / 2].x);
            if (lane == j) z = t;
          }
          if (lane < 8) S.quarter[g][quarter][c0 + lane] = z;
        }
        group_sync(g);
        if (key < rows) {
          const int c = key;
          const float z = fmaxf(fmaxf(S.quarter[g][0][c], S.quarter[g][1][c]),
                                fmaxf(S.quarter[g][2][c], S.quarter[g][3][c]));
          const float d = (first && z > -INFINITY) || z > kSlack ? z : 0.f;  // the maximum's growth
          S.m[g][c] += d;
          S.d[g][c] = d;
          S.add[g][c] -= d;
        }
        group_sync(g);
        const bool was_first = first;  // then l and O are zero
        first = first && fmaxf(fmaxf(S.quarter[g][0][0], S.quarter[g][1][0]),
                               fmaxf(S.quarter[g][2][0], S.quarter[g][3][0])) == -INFINITY;
        if (was_first) return;
#pragma unroll
        for (int c = 0; c < N / 2; ++c)
          if (2 * c < rows) {
            l[c].x *= ex2(-S.d[g][2 * c]);
            l[c].y *= ex2(-S.d[g][2 * c + 1]);
          }
#pragma unroll 1
        for (int c0 = 0; c0 < rows; c0 += 8) {
          uint32_t o[8];
          tc05::tmem_ld8(tO + c0, o);
          tc05::tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int c = c0 + j;
            o[j] = __float_as_uint(__uint_as_float(o[j]) * (c < rows ? ex2(-S.d[g][c]) : 1.f));
          }
          tc05::tmem_st8(tO + c0, o);
        }
        tc05::tmem_wait_st();
      };
      // The tile's logits become probabilities, in shared memory and in l.
      auto softmax = [&](uint32_t seen, bool bf16) {
        const bool all = __all_sync(0xffffffffu, (seen & 0xffffu) == 0xffffu);
        float top = -INFINITY;
        if (!first) {
#pragma unroll 1
          for (int c0 = 0; c0 < rows; c0 += 8) {
            float2 y[4];
            logits(c0, seen, all, y);
            top = fmaxf(top, fmaxf(fmaxf(fmaxf(y[0].x, y[0].y), fmaxf(y[1].x, y[1].y)),
                                   fmaxf(fmaxf(y[2].x, y[2].y), fmaxf(y[3].x, y[3].y))));
          }
        }
        // (a warp whose wait ran out leads the group out with it)
        if (group_any(g, first || top > kSlack || dead)) {
          new_maxima(seen);
          if (dead) return;
        }
#pragma unroll
        for (int c0 = 0; c0 < N; c0 += 8)
          if (c0 < rows) {
            float2 y[4];
            logits(c0, seen, all, y);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 e = make_float2(ex2(y[j].x), ex2(y[j].y));
              l[c0 / 2 + j] = add2(l[c0 / 2 + j], e);
              put_pair<N>(P + c0 * 128, 2 * j, key, pack16(e.x, e.y, bf16));
            }
          }
        tc05::fence_before();
        tc05::fence_proxy_async();
        arrive(&S.p_ready[g]);
      };
      // l summed over the threads, into S.l[g]
      auto sum_rows = [&]() {
#pragma unroll
        for (int c = 0; c < N; ++c)
          if (c < rows) {
            float x = c & 1 ? l[c / 2].y : l[c / 2].x;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
            if (lane == 0) S.quarter[g][quarter][c] = x;
          }
        group_sync(g);
        if (key < rows)
          S.l[g][key] = (S.quarter[g][0][key] + S.quarter[g][1][key]) +
                        (S.quarter[g][2][key] + S.quarter[g][3][key]);
        group_sync(g);
      };

      if (key < N) S.m[g][key] = 0.f;
      if (nint > 0 && g == 0) {
        // q R_k, transposed: thread = place of the rotated row
        load_q(true);
        arrive(&S.q_raw);
        wait(&S.s_full[0], ns++);
        if (group_any(g, dead)) break;
#pragma unroll 1
        for (int c0 = 0; c0 < N; c0 += 8) {
          uint32_t s[8];
          tc05::tmem_ld8(tS + c0, s);
          tc05::tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 8; j += 2)
            put_pair<N>(S.q + c0 * 128, j, key,
                        pack16(__uint_as_float(s[j]) * (1.f / 64.f),
                               __uint_as_float(s[j + 1]) * (1.f / 64.f), false));
        }
        tc05::fence_before();
        tc05::fence_proxy_async();
        arrive(&S.q_ready);
      }
      for (int i = 0; i < ints; ++i) {
        wait(&S.s_full[g], ns++);
        if (i == 0) {  // (the first group wrote scale and off before these logits)
          if (key < N) {
            S.mul[g][key] = S.scale[key];
            S.add[g][key] = -S.off[key];
          }
          group_sync(g);
        }
        const int t = 2 * i + g;
        const uint32_t in = S.mask[(base + t) % 4][quarter] >> lane & 1;
        softmax(in && key < p.n_int - kTile * (p.t0 + t) ? 0xffffu : 0u, false);
        if (dead) break;  // (voted on)
      }
      if (group_any(g, dead)) break;
      if (ints > 0) {
        // O / l into the model's basis: thread = place of the rotated row
        sum_rows();
        wait(&S.o_full[g], no++);
        if (group_any(g, dead)) break;
#pragma unroll 1
        for (int c0 = 0; c0 < rows; c0 += 8) {
          uint32_t o[8];
          tc05::tmem_ld8(tO + c0, o);
          tc05::tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 8; j += 2) {
            const float L0 = c0 + j < rows ? S.l[g][c0 + j] : 0.f;
            const float L1 = c0 + j < rows ? S.l[g][c0 + j + 1] : 0.f;
            put_pair<N>(P + c0 * 128, j, key,
                        pack16(L0 > 0.f ? __fdividef(__uint_as_float(o[j]), L0) : 0.f,
                               L1 > 0.f ? __fdividef(__uint_as_float(o[j + 1]), L1) : 0.f, false));
          }
        }
        if (key < rows && S.l[g][key] > 0.f) S.m[g][key] += __log2f(S.l[g][key]) - 6.f;
#pragma unroll
        for (int c = 0; c < N / 2; ++c)  // O is now 64 of weight 2^m l / 64
          if (2 * c < rows)
            l[c] = make_float2(key == 0 && S.l[g][2 * c] > 0.f ? 64.f : 0.f,
                               key == 0 && S.l[g][2 * c + 1] > 0.f ? 64.f : 0.f);
        tc05::fence_before();
        tc05::fence_proxy_async();
        arrive(&S.p_ready[g]);
      }
      if (all_tiles > nint) {
        if (g == 0) {
          load_q(false);
          arrive(&S.q_ready);
        }
        if (key < N) {
          S.mul[g][key] = kLogit;
          S.add[g][key] = -S.m[g][key];
        }
        group_sync(g);
      }
      for (int i = ints; i < tiles; ++i) {
        wait(&S.s_full[g], ns++);
        // window rows as far as they are filled; own tokens causally
        const int tile = p.t0 + 2 * i + g - p.I;
        const bool own = tile >= p.Wt;
        const int count = own ? p.n_new : p.n_win - kTile * tile;
        softmax(key >= count ? 0u : own ? 0xffffu << key : 0xffffu, true);
        if (dead) break;  // (voted on)
      }
      if (group_any(g, dead)) break;
      if (tiles > 0) {
        sum_rows();
        wait(&S.o_full[g], no++);
      }
      if (group_any(g, dead)) break;
      // The groups' outputs meet; thread = channel.
      float* const other = reinterpret_cast<float*>(S.p[0]);
      if (all_tiles > 1) {
        if (g == 0) {
          arrive(&S.first_done);
          wait(&S.second_ready, nj);
        } else {
          wait(&S.first_done, nj);  // the first group's P is free as well
#pragma unroll 1
          for (int c0 = 0; c0 < rows; c0 += 8) {
            uint32_t o[8];
            tc05::tmem_ld8(tO + c0, o);
            tc05::tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (c0 + j < rows) other[(c0 + j) * kD + key] = __uint_as_float(o[j]);
          }
          tc05::fence_before();
          arrive(&S.second_ready);
          wait(&S.joined, nj);
        }
        ++nj;
      }
      if (g == 0) {
        const bool whole = all_tiles == p.total;
        float* part = part_of(A, w, p.t0 > 0);
#pragma unroll 1
        for (int c0 = 0; c0 < rows; c0 += 8) {
          uint32_t o[8];
          tc05::tmem_ld8(tO + c0, o);
          tc05::tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int r = c0 + j;
            if (r >= rows) continue;
            float x = __uint_as_float(o[j]), M = S.m[0][r], L = S.l[0][r];
            if (all_tiles > 1 && S.l[1][r] > 0.f) {
              const float mn = L > 0.f ? fmaxf(M, S.m[1][r]) : S.m[1][r];
              const float u = L > 0.f ? ex2(M - mn) : 0.f, v = ex2(S.m[1][r] - mn);
              x = x * u + other[r * kD + key] * v;
              L = L * u + S.l[1][r] * v;
              M = mn;
            }
            if (whole)
              A.out[(((size_t)p.c0 + r / 4) * 4 * A.h_kv + 4 * p.h + r % 4) * kD + key] =
                  __float2bfloat16_rn(L > 0.f ? __fdividef(x, L) : 0.f);
            else {
              part[(size_t)r * kD + key] = x;
              if (key == 0) {
                part[(size_t)A.rows * kD + r] = M;
                part[(size_t)A.rows * (kD + 1) + r] = L;
              }
            }
          }
        }
        tc05::fence_before();
        if (all_tiles > 1) arrive(&S.joined);
      }
      if (group_any(g, dead)) break;
    }
  } else if (warp < kTmaWarp) {
    // --------------------------------------------------- keys and values
    // The groups take alternate INT2 tiles, thread = key, in slots that the TMA
    // warps grant them; of the tiles that TMA brings, the group of the slot clears
    // the values that do not count.
    const int g = (warp - kDeqWarp) >> 2, quarter = warp & 3, key = tid & 127;
    const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
    uint32_t nk = 0, nv = 0, nt = 0, tma = 0;
    const int ms = meta_stride(A.compact);
    uint32_t gk[kRing] = {0, 0}, gv[kRing] = {0, 0};  // grants seen
    Piece p;
    for (uint32_t n = 0; next_piece(n, p); ++n) {
      const int nint = p.int_tiles(), nother = p.t1 - p.t0 - nint;
      nk += nint > 0;  // R_k
      // the group's first INT2 tile of the piece
      const int t0 = (int)((nt ^ g) & 1);
      auto request = [&](int t) {
        const int pos = (p.t0 + t) * kTile + key;
        return t < nint && pos < p.n_int
                   ? __ldcg(A.bt + (size_t)p.b * A.max_pages + (A.sink + pos) / kPage) : -1;
      };
      int page = request(t0);
      for (int t = 0; t < nint; ++t, ++nk, ++nv, ++nt) {
        if (t % 2 != t0) continue;
        const uint32_t slot = nt % kRaw;
        const bool inside = (p.t0 + t) * kTile + key < p.n_int;
        const bool ok = inside && page >= 0 && page < A.num_pages;
        if (inside && !ok) atomicOr(A.err, OPTR_DEVERR_PAGE_ID);
        page = request(t + 2);
        const uint32_t bits = __ballot_sync(0xffffffffu, ok || !inside);
        if (!wait(&S.raw_full[slot], nt / kRaw)) break;
        const uint8_t* raw = S.raw[slot][key / kPage];
        // the codes of one kind, the halves read in an order that keeps eight
        // lanes' pieces, 32 B apart, in different banks; and the metadata
        auto codes = [&](int kind, uint4 (&c)[2]) {
          const uint8_t* x = raw + (kind ? OPTR_V_CODES_OFFSET : OPTR_K_CODES_OFFSET) + 32 * (key % kPage);
          const int first = key >> 2 & 1;
          const uint4 a = *reinterpret_cast<const uint4*>(x + 16 * first);
          const uint4 b = *reinterpret_cast<const uint4*>(x + 16 * (1 - first));
          c[0] = first ? b : a;
          c[1] = first ? a : b;
        };
        auto pairs = [&](int kind) {  // zero where the key does not count: a row of zeros
          const uint8_t* x = raw + (kind ? vmeta_offset(A.compact) : OPTR_K_META_OFFSET) + ms * (key % kPage);
          uint4 mm = make_uint4(0u, 0u, 0u, 0u);
          if (ok) {
            if (A.compact)
              mm.x = mm.y = mm.z = mm.w = *reinterpret_cast<const uint32_t*>(x);
            else
              mm = *reinterpret_cast<const uint4*>(x);
          }
          return slot_meta(mm.x, mm.y, mm.z, mm.w);
        };
        if (!wait(&S.k_grant[g][nk % kRing], gk[nk % kRing]++)) break;
        if (lane == 0) S.mask[nk % 4][quarter] = bits;
        uint4 c[2];
        codes(0, c);
        const SlotMeta km = pairs(0);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t word[4] = {c[half].x, c[half].y, c[half].z, c[half].w};
          uint32_t x[32];
#pragma unroll
          for (int i = 0; i < 4; ++i) dequant_word(word[i], km, reinterpret_cast<uint32_t(&)[8]>(x[8 * i]));
          tc05::tmem_st32(tmem + lanes + kColK + 64 * (nk % kRing) + 32 * half, x);
        }
        tc05::tmem_wait_st();
        tc05::fence_before();
        tc05::bar_arrive(&S.k_full[nk % kRing]);
        if (!wait(&S.v_grant[g][nv % kRing], gv[nv % kRing]++)) break;
        codes(1, c);
        const SlotMeta vm = pairs(1);
        uint8_t* dst = S.v[nv % kRing] + key * 128;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t word[4] = {c[half].x, c[half].y, c[half].z, c[half].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t x[8];
            dequant_word(word[i], vm, x);
            *reinterpret_cast<uint4*>(dst + half * kHalf + (((2 * i) ^ (key & 7)) << 4)) =
                make_uint4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<uint4*>(dst + half * kHalf + (((2 * i + 1) ^ (key & 7)) << 4)) =
                make_uint4(x[4], x[5], x[6], x[7]);
          }
        }
        tc05::fence_proxy_async();
        tc05::bar_arrive(&S.v_full[nv % kRing]);
        arrive(&S.raw_empty[slot]);
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
          if (key >= count) {  // 0 times what lies there need not be 0
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
  } else if (warp == kTmaWarp || warp == kTmaWarp + 1) {
    // ------------------------------------------------------------ TMA
    // One warp for the records, keys and R_k, one for the values and R_v^T.  They alone wait
    // for the ring's slots, every phase in turn, and grant the dequantizing groups
    // theirs: a wait tells a phase from the next but not from the next but one,
    // and whoever waited for some of the phases only could miss two.
    const bool values = warp != kTmaWarp;
    uint64_t* const empty = values ? S.v_empty : S.k_empty;
    uint64_t* const full = values ? S.v_tma : S.k_tma;
    uint32_t step = 0, nt = 0, fetched = 0, pending[kRing] = {0, 0};
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
        if (!values) bring(Rk_row + (size_t)p.h * kD * kD);
        // INT2 tiles: records two tiles ahead, the pages' entries three
        auto request = [&](int t) {
          const int pos = (p.t0 + t) * kTile + 16 * lane;
          return t < nint && lane < 8 && pos < p.n_int
                     ? __ldcg(A.bt + (size_t)p.b * A.max_pages + (A.sink + pos) / kPage) : -1;
        };
        auto fetch = [&](int t, int page) {
          if (t >= nint || dead) return;
          const uint32_t i = nt + t, slot = i % kRaw, bytes = chunk_bytes(A.compact);
          if (i >= kRaw && !wait(&S.raw_empty[slot], i / kRaw - 1)) return;
          const bool in = page >= 0 && page < A.num_pages;
          const uint32_t copies = __popc(__ballot_sync(0xffffffffu, in));
          if (lane == 0) tc05::bar_arrive_expect_tx(&S.raw_full[slot], copies * bytes);
          __syncwarp();
          if (in)
            tc05::bulk_g2s(S.raw[slot][lane], A.pool + ((size_t)page * A.h_kv + p.h) * bytes, bytes,
                           &S.raw_full[slot]);
          __syncwarp();
          fetched = i + 1;
        };
        int page = -1;
        if (!values) {
          const int e0 = request(0), e1 = request(1);
          page = request(2);
          fetch(0, e0);
          fetch(1, e1);
        }
        for (int t = 0; t < nint; ++t, ++step) {
          if (!values) {
            fetch(t + 2, page);
            page = request(t + 3);
          }
          if (!free_slot()) break;
          const uint32_t g = (nt + t) & 1;
          arrive(values ? &S.v_grant[g][step % kRing] : &S.k_grant[g][step % kRing]);
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
      }
    }
    // copies in flight land before the CTA exits
    for (int s = 0; s < kRing; ++s)
      if (pending[s]) tc05::bar_wait_drain(&full[s], (pending[s] - 1) & 1);
    for (uint32_t i = fetched > kRaw ? fetched - kRaw : 0; i < fetched; ++i)
      tc05::bar_wait_drain(&S.raw_full[i % kRaw], i / kRaw & 1);
    __syncwarp();
  } else if (warp == kPlanWarp) {
    // ---------------------------------------------------------- pieces
    find_pieces<kPieces>(A, w, S.piece, S.piece_full, S.piece_empty, abort);
  } else {
    // ------------------------------------------------------------ MMA
    const uint32_t sq = tc05::smem_addr(S.q), sp = tc05::smem_addr(S.p[0]),
                   sk = tc05::smem_addr(S.k[0]), sv = tc05::smem_addr(S.v[0]);
    uint32_t nk = 0, nv = 0, nr = 0, nw = 0, np[2] = {0, 0}, kd[kRing] = {0, 0}, kt[kRing] = {0, 0};
    bool used = false;
    auto wait_k = [&](bool tma) {  // key tile nk, by TMA or dequantized
      const uint32_t st = nk % kRing;
      return tma ? wait(&S.k_tma[st], kt[st]++) : wait(&S.k_full[st], kd[st]++);
    };
    auto rows_desc = [&](uint32_t b, int ks) {  // operand of N rows, 128 of its inner dimension
      return tc05::smem_desc_sw128(b + (ks >> 2) * (N * 128) + (ks & 3) * 32, 16);
    };
    Piece p;
    for (uint32_t n = 0; next_piece(n, p); ++n) {
      const int all_tiles = p.t1 - p.t0, nint = p.int_tiles();
      const uint32_t id = tc05::idesc_f16(128, (4 * p.n_new + 15) / 16 * 16);
      used = true;
      bool add[2] = {false, false};
      auto qk = [&](int s, uint32_t type) {
        const uint32_t a = sk + nk % kRing * kOperand, t = tmem + kColK + nk % kRing * 64;
        if (type) {
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            tc05::mma_ss_warp(tmem + s * N,
                              tc05::smem_desc_sw128(a + (ks >> 2) * kHalf + (ks & 3) * 32, 16),
                              rows_desc(sq, ks), id | type, ks != 0);
        } else {
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            tc05::mma_ts_warp(tmem + s * N, t + 8 * ks, rows_desc(sq, ks), id, ks != 0);
        }
        tc05::mma_commit_warp(&S.s_full[s]);
        tc05::mma_commit_warp(&S.k_empty[nk++ % kRing]);
      };
      for (int phase = 0; phase < 2 && !dead; ++phase) {
        const int u0 = phase ? nint : 0, u1 = phase ? all_tiles : nint;
        if (u0 == u1) continue;
        const uint32_t type = phase ? tc05::kIdescBf16 : 0u;
        if (!phase) {  // q R_k, by way of the first group's S
          if (!wait(&S.q_raw, nw++) || !wait_k(true)) break;
          const uint32_t a = sk + nk % kRing * kOperand;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            tc05::mma_ss_warp(tmem, tc05::smem_desc(a + ks * 256, 128, 2048), rows_desc(sq, ks),
                              tc05::idesc_f16(128, N), ks != 0);
          tc05::mma_commit_warp(&S.s_full[0]);
          tc05::mma_commit_warp(&S.k_empty[nk++ % kRing]);
        }
        if (!wait(&S.q_ready, nr++)) break;
        for (int u = u0; u < min(u0 + 2, u1); ++u) {
          if (!wait_k(phase)) break;
          qk(u & 1, type);
        }
        if (dead) break;
        // S and P of a group are free for tile u + 2 once tile u's product with
        // the values is done, which the tensor core's order sees to
        if (u1 - u0 <= 2) tc05::mma_commit_warp(&S.q_empty);
        for (int u = u0; u < u1; ++u) {
          const int s = u & 1;
          if (!wait(&S.v_full[nv % kRing], nv / kRing) || !wait(&S.p_ready[s], np[s]++)) break;
          const uint32_t a = sv + nv % kRing * kOperand;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            tc05::mma_ss_warp(tmem + (2 + s) * N, tc05::smem_desc_sw128(a + ks * 2048, kHalf),
                              rows_desc(sp + s * (N * kTile * 2), ks),
                              id | type | tc05::kIdescMajorMnA, add[s] || ks != 0);
          add[s] = true;
          tc05::mma_commit_warp(&S.v_empty[nv++ % kRing]);
          if (u + 2 >= u1) tc05::mma_commit_warp(&S.o_full[s]);
          if (u + 2 < u1) {
            if (!wait_k(phase)) break;
            qk(s, type);
            if (u + 3 == u1) tc05::mma_commit_warp(&S.q_empty);
          }
        }
        if (dead || phase) continue;
        // O R_v^T of the groups that have INT2 tiles
        if (!wait(&S.v_full[nv % kRing], nv / kRing)) break;
        for (int s = 0; s < min(nint, 2); ++s) {
          if (!wait(&S.p_ready[s], np[s]++)) break;
          const uint32_t a = sv + nv % kRing * kOperand;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            tc05::mma_ss_warp(tmem + (2 + s) * N, tc05::smem_desc(a + ks * 256, 128, 2048),
                              rows_desc(sp + s * (N * kTile * 2), ks), id, ks != 0);
          // the group has no tile after these
          if ((all_tiles + 1 - s) / 2 == (nint + 1 - s) / 2) tc05::mma_commit_warp(&S.o_full[s]);
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
    tc05::tmem_dealloc(tmem, kCols);
  }
}

template <int N>
cudaError_t launch_n(const optr_params* p, const ChunkArgs& A, const __nv_bfloat16* q,
                     const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mw,
                     cudaStream_t s) {
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(chunk_small_kernel<N>),
                                      sizeof(Smem<N>));
  if (e != cudaSuccess) return e;
  return launch_pdl(chunk_small_kernel<N>, dim3(A.W), dim3(kThreads), sizeof(Smem<N>), s, mk, mv, mw,
                    q, (const float*)p->mu, (const uint16_t*)p->Rk_row, A);
}

}  // namespace

int chunk_small_rows(int max_new) { return max_new <= 12 ? (4 * max_new + 15) / 16 * 16 : 0; }

cudaError_t launch_chunk_small(const optr_params* p, const ChunkArgs& A, const __nv_bfloat16* q,
                               const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mw,
                               cudaStream_t s) {
  switch (A.rows) {
    case 16: return launch_n<16>(p, A, q, mk, mv, mw, s);
    case 32: return launch_n<32>(p, A, q, mk, mv, mw, s);
    default: return launch_n<48>(p, A, q, mk, mv, mw, s);
  }
}

}  // namespace optr
