// Chunk attention of a few new tokens per sequence (drafted tokens; up to 16):
// chunk.cu's computation with the tiles transposed, so that what is padded is
// the keys' tile (never) and not the queries' (4 to 64 rows):
//   S^T[key][row] = K Q^T,   O^T[channel][row] += V^T P^T
// with M = 128 keys or channels and N = 16 .. 64 rows.
//
// Bound by what it takes to dequantize: per tile of 128 keys 12 KB come in, which
// an SM's share of the memory's rate brings in about 530 cycles, and its 2 x 128 x
// 128 codes take about as many issue slots of each SM quarter; N rows' softmax
// adds N / 32 of 128 threads' exponentials.  So all warps do the same work, and
// the tensor core's is nearly free.  A CTA is 2 to 4 warpgroups, each a worker
// with a range of tiles, queries and accumulators of its own (chunk.cuh's line of
// tiles is cut into equal ranges, one per warpgroup): while one waits for its MMA
// or its loads the others dequantize.
//
// Thread = key of the tile.  Its record is in registers a tile ahead.  The key goes
// into tensor memory as a row of the A operand, the value into a row of shared
// memory (V^T is that tile read along its other dimension).  The thread then holds
// its key's logits with all rows: probabilities go into shared memory transposed, where
// the rows' sums are taken; a row's maximum is kept for the warpgroup and only
// looked at again when some thread's logit passes it by 2^8.
#include "append_common.cuh"
#include "chunk.cuh"
#include "dequant.cuh"
#include "tc05.cuh"
#include "tmap.cuh"

namespace optr {
namespace {

constexpr uint32_t kBuf = kTile * kD * 2;  // 128 x 128 of 16 bits
constexpr float kSlack = 8.f;

// Warpgroups per CTA for up to N rows: what tensor memory (64 + 2 N columns each)
// and registers admit.
__host__ __device__ constexpr int groups_for(int N) { return N <= 32 ? 4 : N <= 48 ? 3 : 2; }

template <int N>
struct GroupSmem {
  alignas(1024) uint8_t v[kBuf];  // values; keys brought by TMA; operands of the rotations
  uint8_t q[N * kD * 2];      // queries [row][channel or place], two halves of 64
  uint8_t p[N * kTile * 2];   // probabilities [row][key]; O [row][place] for its rotation
  alignas(16) float2 ms[N];   // logit = S x + y: {x, y}, y = -(offset + maximum)
  float quarter[4][N];        // of the four warps
  float m[N], l[N], d[N], off[N], scale[N];
  Piece piece;
};

template <int N>
struct Smem {
  GroupSmem<N> g[groups_for(N)];
  uint64_t s_done[4], o_done[4], t_done[4], drained[4];
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

// A key's record of one kind, as read: codes and {scale, min} words.
struct Record {
  uint4 c[2], m;
};

template <int N>
__global__ void __launch_bounds__(128 * groups_for(N), 1)
chunk_small_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                   const __grid_constant__ CUtensorMap tm_win, const __nv_bfloat16* __restrict__ q_in,
                   const float* __restrict__ mu, const uint16_t* __restrict__ Rk_row,
                   const __grid_constant__ ChunkArgs A) {
  constexpr int kGroupsN = groups_for(N);
  constexpr uint32_t kCols = 64 + 2 * N;  // K | S | O
  extern __shared__ __align__(1024) unsigned char dsm_[];
  Smem<N>& S = *reinterpret_cast<Smem<N>*>(dsm_);
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int g = warp >> 2, quarter = warp & 3, key = tid & 127;
  GroupSmem<N>& G = S.g[g];
  if (tid == 0) {
    for (int i = 0; i < 4; ++i) {
      tc05::bar_init(&S.s_done[i], 1);
      tc05::bar_init(&S.o_done[i], 1);
      tc05::bar_init(&S.t_done[i], 1);
      tc05::bar_init(&S.drained[i], 1);
    }
    S.abort = (tc05::smem_addr(&S) & 1023u) != 0;  // the swizzle's alignment
    tc05::bar_init_fence();
  }
  if (warp == 0) tc05::tmem_alloc(&S.tmem, 512);
  pdl_wait();
  pdl_trigger();
  tc05::fence_before();
  __syncthreads();
  tc05::fence_after();
  const uint32_t base = S.tmem + kCols * g;
  const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
  const uint32_t tK = base, tS = base + 64, tO = base + 64 + N;
  volatile int* abort = &S.abort;
  const int w = g * gridDim.x + blockIdx.x;  // (few workers have work: of different SMs)

  if (w == 0 && quarter == 0) report_sequences(A);
  PieceFinder next;  // the group's first warp's
  if (quarter == 0) next.start(A, w);
  ChunkSeg seg{};
  uint32_t ns = 0, no = 0, nt = 0, brought = 0;  // phases of s_done, o_done, t_done
  bool dead = false, used = false;
  auto wait = [&](uint64_t* bar, uint32_t phase) {
    if (!__all_sync(0xffffffffu, tc05::bar_wait_spin(bar, phase & 1, abort))) dead = true;
    tc05::fence_after();
  };
  const uint32_t sv = tc05::smem_addr(G.v), sq = tc05::smem_addr(G.q), sp = tc05::smem_addr(G.p);

  constexpr int kPerRow = N == 16 ? 8 : N == 32 ? 4 : 2;  // threads per row's sum
  const int lrow = key / kPerRow, lpart = key % kPerRow;
  while (true) {
    if (quarter == 0) {
      Piece x;
      x.t0 = x.t1 = 0;
      while (next.f < next.f1 && x.t1 == x.t0) next.next(A, x);
      if (x.t1 > 0 && x.t0 == 0 && x.t1 < x.total)
        seg = ChunkSeg{next.F, next.f_seg + kBegin + x.total, x.c0, x.n_new, x.h, x.qb, next.W, 1};
      if (lane == 0) G.piece = x;
    }
    group_sync(g);
    const Piece p = G.piece;
    if (p.t1 == p.t0) break;
    used = true;
    const int nint = p.int_tiles();
    const int rows = 4 * p.n_new, nc = (rows + 15) / 16;  // rows, in chunks of 16
    const uint32_t id = tc05::idesc_f16(128, 16 * nc);
    float l = 0.f;      // sum of row `lrow`'s probabilities over the thread's share of the keys
    bool fresh = true;  // nothing in O yet
    bool first = true;  // no maximum yet

    // queries of the rows, as they come or as fp16 over a power of two
    auto load_q = [&](bool rotate) {
      for (int r = quarter; r < 16 * nc; r += 4) {
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
            G.scale[r] = __uint_as_float((uint32_t)(127 + E) << 23) * kLogit;
            G.off[r] = -dot * kLogit;
          }
          const __half2 u = __floats2half2_rn(a * down, b * down), v = __floats2half2_rn(c * down, d * down);
          x = make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
        }
        *reinterpret_cast<uint2*>(G.q + at16<N>(r, 4 * lane)) = x;
      }
    };
    // 32 KB of an operand or a tile into v, two halves
    auto bring = [&](const uint16_t* operand) {
      ++brought;
      if (key == 0) {
        tc05::bar_arrive_expect_tx(&S.t_done[g], kBuf);
        tc05::bulk_g2s(G.v, operand, kBuf, &S.t_done[g]);
      }
    };
    auto bring_tile = [&](int tile, int kind) {
      ++brought;
      if (key == 0) {
        tc05::bar_arrive_expect_tx(&S.t_done[g], kBuf);
        for (int c = 0; c < 2; ++c) {
          uint8_t* dst = G.v + c * (kBuf / 2);
          if (tile < p.Wt)
            tc05::tma_load_3d(dst, &tm_win, 64 * c, 0,
                              ((p.slot * A.h_kv + p.h) * 2 + kind) * (A.sink + A.recent) + kTile * tile,
                              &S.t_done[g]);
          else
            tc05::tma_load_3d(dst, kind ? &tm_v : &tm_k, 64 * c, p.h, p.c0 + kTile * (tile - p.Wt),
                              &S.t_done[g]);
        }
      }
    };
    // D (+)= A B^T by warp 0 of the group, after what all threads wrote
    enum { kKeysTmem, kKeysSmem, kValues, kOperandSmem };
    auto product = [&](int what, uint32_t d, uint32_t b, uint32_t type, bool add, uint64_t* bar) {
      tc05::fence_before();
      tc05::fence_proxy_async();
      group_sync(g);
      if (quarter == 0) {
        tc05::fence_after();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          const uint64_t db = tc05::smem_desc_sw128(b + (ks >> 2) * (N * 128) + (ks & 3) * 32, 16);
          const uint32_t acc = add || ks != 0;
          if (what == kKeysTmem) {
            tc05::mma_ts_warp(d, tK + 8u * ks, db, id | type, acc);
          } else {
            const uint64_t da =
                what == kKeysSmem ? tc05::smem_desc_sw128(sv + (ks >> 2) * (kBuf / 2) + (ks & 3) * 32, 16)
                : what == kValues ? tc05::smem_desc_sw128(sv + ks * 2048, kBuf / 2)
                                  : tc05::smem_desc(sv + ks * 256, 128, 2048);
            tc05::mma_ss_warp(d, da, db, id | type | (what == kValues ? tc05::kIdescMajorMnA : 0u), acc);
          }
        }
        tc05::mma_commit_warp(bar);
      }
    };
    // Adds the tile's probabilities, as they stand in shared memory, to l.
    auto add_rows = [&](bool bf16) {
      if (lrow >= 16 * nc) return;
#pragma unroll
      for (int i = 0; i < 16 / kPerRow; ++i) {
        const int k = 8 * (lpart + kPerRow * i);
        const uint4 x = *reinterpret_cast<const uint4*>(G.p + at16<N>(lrow, k));
        const uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 y = bf16 ? make_float2(__uint_as_float(word[e] << 16),
                                              __uint_as_float(word[e] & 0xffff0000u))
                                : __half22float2(*reinterpret_cast<const __half2*>(&word[e]));
          l += y.x + y.y;
        }
      }
    };
    // l summed over a row's threads, into G.l
    auto sum_rows = [&]() {
      float x = l;
#pragma unroll
      for (int o = 1; o < kPerRow; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      if (lpart == 0 && lrow < N) G.l[lrow] = x;
      group_sync(g);
    };
    // The tile's probabilities, from its logits, under the maxima as they are;
    // returns the largest logit over its row's maximum.  Bit c / 4 of `seen`
    // says whether the thread's key counts for the rows of new token c / 4.
    auto probabilities = [&](uint32_t seen, bool bf16) {
      float top = -INFINITY;
#pragma unroll 1
      for (int c0 = 0; c0 < 16 * nc; c0 += 16) {
        uint32_t s[16];
        tc05::tmem_ld16(tS + lanes + c0, s);
        tc05::tmem_wait_ld();
        const uint32_t bits = seen >> (c0 >> 2);
        uint8_t* row = G.p + c0 * 128;
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          const float4 x = *reinterpret_cast<const float4*>(&G.ms[c0 + j]);
          const bool in = bits >> (j >> 2) & 1;
          const float y0 = in ? fmaf(__uint_as_float(s[j]), x.x, x.y) : -INFINITY;
          const float y1 = in ? fmaf(__uint_as_float(s[j + 1]), x.z, x.w) : -INFINITY;
          top = fmaxf(top, fmaxf(y0, y1));
          const uint32_t e = pack16(ex2(y0), ex2(y1), bf16);
          *reinterpret_cast<uint16_t*>(row + at16<N>(j, key)) = (uint16_t)e;
          *reinterpret_cast<uint16_t*>(row + at16<N>(j + 1, key)) = (uint16_t)(e >> 16);
        }
      }
      return top;
    };
    auto softmax = [&](uint32_t seen, bool bf16) {
      const float top = probabilities(seen, bf16);
      // (a warp whose wait ran out leads the group out with it)
      if (!group_any(g, first || top > kSlack || dead)) return;
      if (group_any(g, dead)) {
        dead = true;
        return;
      }
      // maxima anew
#pragma unroll 1
      for (int c0 = 0; c0 < 16 * nc; c0 += 16) {
        uint32_t s[16];
        tc05::tmem_ld16(tS + lanes + c0, s);
        tc05::tmem_wait_ld();
        float z = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float2 x = G.ms[c0 + j];
          const float y = seen >> ((c0 + j) >> 2) & 1 ? fmaf(__uint_as_float(s[j]), x.x, x.y) : -INFINITY;
          const float t = warp_max(y);
          if (lane == j) z = t;
        }
        if (lane < 16) G.quarter[quarter][c0 + lane] = z;
      }
      group_sync(g);
      for (int c = key; c < 16 * nc; c += 128) {
        const float z = fmaxf(fmaxf(G.quarter[0][c], G.quarter[1][c]),
                              fmaxf(G.quarter[2][c], G.quarter[3][c]));
        const float d = (first && z > -INFINITY) || z > kSlack ? z : 0.f;  // the maximum's growth
        G.m[c] += d;
        G.d[c] = d;
        G.ms[c].y -= d;
      }
      group_sync(g);
      const bool was_first = first;  // then l and O are zero
      first = first && fmaxf(fmaxf(G.quarter[0][0], G.quarter[1][0]),
                             fmaxf(G.quarter[2][0], G.quarter[3][0])) == -INFINITY;
      if (!was_first) {
        if (lrow < 16 * nc) l *= ex2(-G.d[lrow]);
#pragma unroll 1
        for (int c0 = 0; c0 < 16 * nc; c0 += 16) {
          uint32_t o[16];
          tc05::tmem_ld16(tO + lanes + c0, o);
          tc05::tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * ex2(-G.d[c0 + j]));
          tc05::tmem_st16(tO + lanes + c0, o);
        }
        tc05::tmem_wait_st();
      }
      probabilities(seen, bf16);
    };

    if (nint > 0) {
      // q R_k, transposed: thread = place of the rotated row
      bring(Rk_row + (size_t)p.h * kD * kD);
      load_q(true);
      wait(&S.t_done[g], nt++);
      product(kOperandSmem, tS, sq, 0u, false, &S.s_done[g]);
      wait(&S.s_done[g], ns++);
      if (group_any(g, dead)) break;
#pragma unroll 1
      for (int c0 = 0; c0 < 16 * nc; c0 += 16) {
        uint32_t s[16];
        tc05::tmem_ld16(tS + lanes + c0, s);
        tc05::tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          const uint32_t e = pack16(__uint_as_float(s[j]) * (1.f / 64.f),
                                    __uint_as_float(s[j + 1]) * (1.f / 64.f), false);
          *reinterpret_cast<uint16_t*>(G.q + c0 * 128 + at16<N>(j, key)) = (uint16_t)e;
          *reinterpret_cast<uint16_t*>(G.q + c0 * 128 + at16<N>(j + 1, key)) = (uint16_t)(e >> 16);
        }
      }
      for (int c = key; c < 16 * nc; c += 128) {
        G.m[c] = 0.f;
        G.ms[c] = make_float2(G.scale[c], -G.off[c]);
      }
      // INT2 tiles
      const int ms = meta_stride(A.compact);
      auto request = [&](int t) {
        const int n = t * kTile + key;
        return n < p.n_int && t < p.t1
                   ? __ldcg(A.bt + (size_t)p.b * A.max_pages + (A.sink + n) / kPage) : -1;
      };
      // whether the key of tile t counts, by its page
      auto counts = [&](int t, int page) {
        if (!(t * kTile + key < p.n_int && t < p.t1)) return false;
        if (page >= 0 && page < A.num_pages) return true;
        atomicOr(A.err, OPTR_DEVERR_PAGE_ID);
        return false;
      };
      auto fetch = [&](Record& r, bool ok, int page, int kind) {
        r.m = make_uint4(0u, 0u, 0u, 0u);  // a row of zeros where the key does not count
        if (!ok) return;
        const uint8_t* x = A.pool + ((size_t)page * A.h_kv + p.h) * chunk_bytes(A.compact);
        const int slot = key % kPage;  // (sink is a multiple of 16)
        const uint4* c = reinterpret_cast<const uint4*>(
            x + (kind ? OPTR_V_CODES_OFFSET : OPTR_K_CODES_OFFSET) + 32 * slot);
        const uint8_t* m = x + (kind ? vmeta_offset(A.compact) : OPTR_K_META_OFFSET) + ms * slot;
        r.c[0] = __ldcg(c);
        r.c[1] = __ldcg(c + 1);
        if (A.compact)
          r.m.x = r.m.y = r.m.z = r.m.w = __ldcg(reinterpret_cast<const uint32_t*>(m));
        else
          r.m = __ldcg(reinterpret_cast<const uint4*>(m));
      };
      Record rk{}, rv{};
      int page = request(p.t0);
      bool ok = counts(p.t0, page);
      fetch(rk, ok, page, 0);
      fetch(rv, ok, page, 1);
      page = request(p.t0 + 1);
      for (int t = p.t0; t < p.t0 + nint; ++t) {
        const bool okn = counts(t + 1, page);
        const SlotMeta km = slot_meta(rk.m.x, rk.m.y, rk.m.z, rk.m.w);
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          const uint4 c = half ? rk.c[1] : rk.c[0];
          const uint32_t word[4] = {c.x, c.y, c.z, c.w};
          uint32_t x[32];
#pragma unroll
          for (int i = 0; i < 4; ++i) dequant_word(word[i], km, reinterpret_cast<uint32_t(&)[8]>(x[8 * i]));
          tc05::tmem_st32(tK + lanes + 32 * half, x);
        }
        fetch(rk, okn, page, 0);
        tc05::tmem_wait_st();
        product(kKeysTmem, tS, sq, 0u, false, &S.s_done[g]);
        // the last tile's values and probabilities are done with
        if (!fresh) wait(&S.o_done[g], no++);
        const SlotMeta vm = slot_meta(rv.m.x, rv.m.y, rv.m.z, rv.m.w);
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          const uint4 c = half ? rv.c[1] : rv.c[0];
          const uint32_t word[4] = {c.x, c.y, c.z, c.w};
          uint8_t* dst = G.v + half * (kBuf / 2) + key * 128;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t x[8];
            dequant_word(word[i], vm, x);
            *reinterpret_cast<uint4*>(dst + (((2 * i) ^ (key & 7)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<uint4*>(dst + (((2 * i + 1) ^ (key & 7)) << 4)) =
                make_uint4(x[4], x[5], x[6], x[7]);
          }
        }
        fetch(rv, okn, page, 1);
        page = request(t + 2);
        wait(&S.s_done[g], ns++);
        softmax(ok ? 0xffffu : 0u, false);
        if (dead) break;
        product(kValues, tO, sp, 0u, !fresh, &S.o_done[g]);
        add_rows(false);
        fresh = false;
        ok = okn;
      }
      if (dead) break;
      // O / l into the model's basis: thread = place of the rotated row
      wait(&S.o_done[g], no++);
      if (group_any(g, dead)) break;
      bring(A.Rv_back + (size_t)p.h * kRT5Halves);
      sum_rows();
#pragma unroll 1
      for (int c0 = 0; c0 < 16 * nc; c0 += 16) {
        uint32_t o[16];
        tc05::tmem_ld16(tO + lanes + c0, o);
        tc05::tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          const float L0 = G.l[c0 + j], L1 = G.l[c0 + j + 1];
          const uint32_t e = pack16(L0 > 0.f ? __fdividef(__uint_as_float(o[j]), L0) : 0.f,
                                    L1 > 0.f ? __fdividef(__uint_as_float(o[j + 1]), L1) : 0.f, false);
          *reinterpret_cast<uint16_t*>(G.p + c0 * 128 + at16<N>(j, key)) = (uint16_t)e;
          *reinterpret_cast<uint16_t*>(G.p + c0 * 128 + at16<N>(j + 1, key)) = (uint16_t)(e >> 16);
        }
      }
      if (lrow < N)  // O is now 64 of weight 2^m l / 64
        l = lpart == 0 && G.l[lrow] > 0.f ? 64.f : 0.f;
      for (int c = key; c < 16 * nc; c += 128)
        if (G.l[c] > 0.f) G.m[c] += __log2f(G.l[c]) - 6.f;
      wait(&S.t_done[g], nt++);
      product(kOperandSmem, tO, sp, 0u, false, &S.o_done[g]);
    } else {
      for (int c = key; c < 16 * nc; c += 128) G.m[c] = 0.f;
    }

    // the windows' rows and the chunk's own
    const int nother = p.t1 - p.t0 - nint;
    if (nother > 0) {
      load_q(false);
      for (int c = key; c < 16 * nc; c += 128) G.ms[c] = make_float2(kLogit, -G.m[c]);
    }
    for (int t = 0; t < nother; ++t) {
      const int tile = p.t0 + nint + t - p.I;
      const bool own = tile >= p.Wt;
      const int count = own ? p.n_new : p.n_win - kTile * tile;
      if (!fresh) wait(&S.o_done[g], no++);
      bring_tile(tile, 0);
      wait(&S.t_done[g], nt++);
      product(kKeysSmem, tS, sq, tc05::kIdescBf16, false, &S.s_done[g]);
      wait(&S.s_done[g], ns++);
      bring_tile(tile, 1);
      softmax(key >= count ? 0u : own ? 0xffffu << key : 0xffffu, true);
      if (dead) break;
      wait(&S.t_done[g], nt++);
      if (key >= count) {  // 0 times what lies there need not be 0
        uint8_t* r = G.v + key * 128;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          *reinterpret_cast<uint4*>(r + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
          *reinterpret_cast<uint4*>(r + kBuf / 2 + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
        }
      }
      product(kValues, tO, sp, tc05::kIdescBf16, !fresh, &S.o_done[g]);
      add_rows(true);
      fresh = false;
    }
    if (dead) break;
    wait(&S.o_done[g], no++);
    if (group_any(g, dead)) break;
    // thread = channel
    sum_rows();
    const bool whole = p.t1 - p.t0 == p.total;
    float* part = part_of(A, w, p.t0 > 0);
#pragma unroll 1
    for (int c0 = 0; c0 < 16 * nc; c0 += 16) {
      uint32_t o[16];
      tc05::tmem_ld16(tO + lanes + c0, o);
      tc05::tmem_wait_ld();
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int r = c0 + j;
        if (r >= rows) continue;
        const float x = __uint_as_float(o[j]), L = G.l[r];
        if (whole)
          A.out[(((size_t)p.c0 + r / 4) * 4 * A.h_kv + 4 * p.h + r % 4) * kD + key] =
              __float2bfloat16_rn(L > 0.f ? __fdividef(x, L) : 0.f);
        else
          part[(size_t)r * kD + key] = x;
      }
    }
    if (!whole)
      for (int r = key; r < rows; r += 128) {
        part[(size_t)A.rows * kD + r] = G.m[r];
        part[(size_t)A.rows * (kD + 1) + r] = G.l[r];
      }
    tc05::fence_before();
    group_sync(g);
  }
  if (key == 0) A.seg[w] = seg;
  // what was issued ends before shared and tensor memory are given back
  if (key == 0 && brought > 0) tc05::bar_wait_drain(&S.t_done[g], (brought - 1) & 1);
  __syncwarp();
  if (quarter == 0 && used) {
    tc05::mma_commit_warp(&S.drained[g]);
    tc05::bar_wait_drain(&S.drained[g], 0);
  }
  tc05::fence_before();
  __syncthreads();
  if (S.abort && tid == 0) atomicOr(A.err, OPTR_DEVERR_TIMEOUT);
  if (warp == 0) {
    tc05::fence_after();
    tc05::tmem_dealloc(S.tmem, 512);
  }
}

template <int N>
cudaError_t launch_n(const optr_params* p, const ChunkArgs& A, const __nv_bfloat16* q,
                     const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mw,
                     cudaStream_t s) {
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(chunk_small_kernel<N>),
                                      sizeof(Smem<N>));
  if (e != cudaSuccess) return e;
  return launch_pdl(chunk_small_kernel<N>, dim3(p->num_sms), dim3(128 * groups_for(N)),
                    sizeof(Smem<N>), s, mk, mv, mw, q, (const float*)p->mu,
                    (const uint16_t*)p->Rk_row, A);
}

}  // namespace

int chunk_small_rows(int max_new) { return max_new <= 16 ? (4 * max_new + 15) / 16 * 16 : 0; }
int chunk_small_groups(int rows) { return groups_for(rows); }

cudaError_t launch_chunk_small(const optr_params* p, const ChunkArgs& A, const __nv_bfloat16* q,
                               const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mw,
                               cudaStream_t s) {
  switch (A.rows) {
    case 16: return launch_n<16>(p, A, q, mk, mv, mw, s);
    case 32: return launch_n<32>(p, A, q, mk, mv, mw, s);
    case 48: return launch_n<48>(p, A, q, mk, mv, mw, s);
    default: return launch_n<64>(p, A, q, mk, mv, mw, s);
  }
}

}  // namespace optr
