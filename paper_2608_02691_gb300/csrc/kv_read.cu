// Cache read-back (include/optr.h, "optr_kv_read"): the INT2 records of given
// positions as bf16 rows in the model's basis,
//   k = khat R_k^T + mu,   v = vhat R_v^T.
//
// The mirror of the tcgen05 cache write (append_tc05.cu): per KV head and kind
// a product Y[tok][128] = Z[tok][128] R^T[128][128] of 128-token tiles, Z the
// dequantized rows (exact codes, scales and minima, rounded once to fp16;
// dequant.cuh), R^T as fp16 hi + lo parts of 64 R^T, which keep ~22 bits of it
// under a float32 accumulator.
//
// One CTA per SM works on one (KV head, kind) and loops over its tiles:
//   8 converter warps  two groups of 4 take alternate tiles, a thread per row:
//                   table entry requested four of the group's tiles ahead,
//                   record copied to shared memory three ahead, then 128 values
//                   into tensor memory (A operand);
//   MMA warp        issues a tile's 16 tcgen05.mma;
//   8 epilogue warps  two groups likewise: accumulator rows back, mu, bf16,
//                   into a swizzled shared-memory tile that two TMA copies
//                   store.
// Bound by memory: 96 B (G = 32) or 72 B read and 512 B written per token and
// KV head.  16 x 8192 tokens of 8 KV heads take 127 us (124 to 129 from box to box),
// 5.0 TB/s, 74% of a copy's rate; 144 with the records a tile ahead in registers, 3
// more with whole tiles stored at a time.  777 tokens take 7.5 to 8.7 us, all latency.
#include "append_common.cuh"
#include "decode_common.cuh"
#include "dequant.cuh"
#include "f32x2.cuh"
#include "tc05.cuh"
#include "tmap.cuh"

namespace optr {
namespace {

constexpr int kRows = 128;
constexpr int kCuCache = 512;
constexpr int kConvWarps = 8, kEpiWarps = 8;
constexpr int kEpiWarp = kConvWarps, kMmaWarp = kConvWarps + kEpiWarps;
constexpr int kThreads = (kMmaWarp + 1) * 32;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColD = 0, kColA = 256;  // D[g] at 128 g, A[g] at 256 + 64 g
constexpr uint32_t kTileBytes = kRows * kD * 2;
constexpr int kAhead = 4;  // tiles whose records a converter group has in flight

struct Smem {
  uint16_t b[2][kD * kD];
  // output rows, bf16: [channel half][row][128 B], TMA 128-byte swizzle
  uint8_t stage[2][kTileBytes];
  // records as read, of the group's next tiles: codes (2 x 16 B), {scale, min} words
  uint4 raw[2][kAhead][3][kRows];
  alignas(16) float add[kD];  // mu (keys) or 0 (values)
  int cu[kCuCache + 1];
  int p0[kCuCache];
  uint64_t aready[2], adone[2], dready[2], dfree[2];
  uint32_t tmem;
  int abort;
};

__device__ __forceinline__ void group_sync(int id) {
  asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory");
}

// group_sync, and whether x held in any thread of the group.
__device__ __forceinline__ bool group_any(int id, bool x) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %2, 0;\n"
      " barrier.cta.red.or.pred q, %1, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r) : "r"(id), "r"((uint32_t)x) : "memory");
  return r != 0;
}

__device__ __forceinline__ void tma_store_3d(const void* tmap, int c0, int c1, int c2,
                                             const void* src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
               ::"l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2),
                 "r"(tc05::smem_addr(src))
               : "memory");
}

template <bool kG128>
__global__ void __launch_bounds__(kThreads, 1)
kv_read_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
               int n_tok, const int32_t* __restrict__ cu_read, const int32_t* __restrict__ pos0,
               const int32_t* __restrict__ bt, int B, int max_pages,
               const uint8_t* __restrict__ pool, int num_pages, int h_kv,
               const uint16_t* __restrict__ Rk_back, const uint16_t* __restrict__ Rv_back,
               const float* __restrict__ mu, unsigned* err) {
  extern __shared__ __align__(1024) unsigned char dsm_[];
  Smem& S = *reinterpret_cast<Smem*>(dsm_);
  const int h = blockIdx.y, kind = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int tiles = (n_tok + kRows - 1) / kRows;
  const int my_tiles =
      tiles > (int)blockIdx.x ? (tiles - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0;

  {
    const uint4* src = reinterpret_cast<const uint4*>(kind ? Rv_back : Rk_back) +
                       (size_t)h * (2 * kD * kD * 2 / 16);
    uint4* dst = reinterpret_cast<uint4*>(&S.b[0][0]);
    for (int i = tid; i < 2 * kD * kD * 2 / 16; i += kThreads) cp_async16_zfill(dst + i, src + i, true);
    cp_async_commit();
  }
  if (tid < kD) S.add[tid] = kind ? 0.f : __ldg(mu + h * kD + tid);
  if (tid == 0) {
    for (int g = 0; g < 2; ++g) {
      tc05::bar_init(&S.aready[g], 128);
      tc05::bar_init(&S.adone[g], 1);
      tc05::bar_init(&S.dready[g], 1);
      tc05::bar_init(&S.dfree[g], 128);
    }
    S.abort = (tc05::smem_addr(S.stage[0]) & 1023u) != 0;  // the swizzle's alignment
    tc05::bar_init_fence();
  }
  if (warp == kMmaWarp) tc05::tmem_alloc(&S.tmem, kTmemCols);
  pdl_wait();
  pdl_trigger();
  const bool cached = B <= kCuCache;
  if (cached) {
    for (int i = tid; i <= B; i += kThreads) S.cu[i] = __ldcg(cu_read + i);
    for (int i = tid; i < B; i += kThreads) S.p0[i] = __ldcg(pos0 + i);
  }
  cp_async_wait<0>();
  tc05::fence_proxy_async();
  tc05::fence_before();
  __syncthreads();
  tc05::fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, S.tmem, 0);
  volatile int* abort = &S.abort;

  if (warp < kConvWarps) {
    // -------------------------------------------------------- converters
    const int g = warp >> 2, q = warp & 3, row = 32 * q + lane;
    const uint32_t tA = tmem + ((uint32_t)(32 * q) << 16) + kColA + 64u * g;
    auto cu = [&](int b) { return cached ? S.cu[b] : __ldcg(cu_read + b); };
    // A tile's page entry is requested one tile of the group before its
    // records are. The group's tokens only rise, so the sequence is searched
    // once and then followed.
    int lo = 0, page = 0, slot = 0;  // page is left as loaded: a test here would wait for it
    bool have = false, found = false;
    auto request = [&](int i) {
      have = false;
      const int tok = ((int)blockIdx.x + i * (int)gridDim.x) * kRows + row;
      if (i >= my_tiles || tok >= n_tok) return;
      if (!found) {
        found = true;
        int hi = B;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (cu(mid) <= tok) lo = mid; else hi = mid;
        }
      }
      while (lo + 1 < B && cu(lo + 1) <= tok) ++lo;
      const int c0 = cu(lo);
      if (!(c0 <= tok && tok < cu(lo + 1))) {
        atomicOr(err, OPTR_DEVERR_CU_NEW);
        return;
      }
      const long long pos = (long long)(cached ? S.p0[lo] : __ldcg(pos0 + lo)) + (tok - c0);
      if (pos < 0 || pos >= (long long)max_pages * kPage) {
        atomicOr(err, OPTR_DEVERR_POSITION);
        return;
      }
      have = true;
      slot = (int)pos % kPage;
      page = __ldcg(bt + (size_t)lo * max_pages + (int)pos / kPage);
    };
    uint32_t words = 0;  // G = 128: which of its 16 bytes of {scale, min} a tile's row has
    // Copies into shared memory keep their loads in flight without registers;
    // a thread reads back what it copied itself, so its own wait is enough.
    auto fetch = [&](int at) {
      uint4(*raw)[kRows] = S.raw[g][at];
      const bool ok = have && (unsigned)page < (unsigned)num_pages;
      if (have && !ok) atomicOr(err, OPTR_DEVERR_PAGE_ID);
      const uint8_t* rec = pool + (ok ? ((size_t)page * h_kv + h) * chunk_bytes(kG128) : 0);
      const int s = ok ? slot : 0;
      const uint8_t* c = rec + (kind ? OPTR_V_CODES_OFFSET : OPTR_K_CODES_OFFSET) + s * 32;
      const uint8_t* m = rec + (kind ? vmeta_offset(kG128) : OPTR_K_META_OFFSET) +
                         (kG128 ? s & ~3 : s) * meta_stride(kG128);  // 16 bytes at least
      cp_async16_zfill(&raw[0][row], c, ok);
      cp_async16_zfill(&raw[1][row], c + 16, ok);
      cp_async16_zfill(&raw[2][row], m, ok);
      cp_async_commit();
      words = words << 2 | (uint32_t)(s & 3);
    };
    uint32_t past = 0;  // whether a value left fp16's range
    request(g);
    for (int k = 0; k < kAhead - 1; ++k) {
      fetch(k);
      request(g + 2 * (k + 1));
    }
#pragma unroll 1
    for (int i = g, k = 0; i < my_tiles; i += 2, ++k) {
      fetch((k + kAhead - 1) % kAhead);
      request(i + 2 * kAhead);
      cp_async_wait<kAhead - 1>();
      const uint4(*raw)[kRows] = S.raw[g][k % kAhead];
      const uint4 c0 = raw[0][row], c1 = raw[1][row];
      uint4 mw;
      if (kG128)
        mw.x = mw.y = mw.z = mw.w =
            reinterpret_cast<const uint32_t*>(&raw[2][row])[words >> (2 * (kAhead - 1)) & 3u];
      else
        mw = raw[2][row];
      const SlotMeta m = slot_meta(mw.x, mw.y, mw.z, mw.w);
      note_range(m, past);
      const uint32_t word[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
      if (k > 0 && !__all_sync(0xffffffffu, tc05::bar_wait(&S.adone[g], (k - 1) & 1, abort))) break;
      tc05::fence_after();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t a[32];
#pragma unroll
        for (int w = 0; w < 4; ++w)
          dequant_word(word[4 * half + w], m, reinterpret_cast<uint32_t(&)[8]>(a[8 * w]));
        tc05::tmem_st32(tA + 32u * half, a);
      }
      tc05::tmem_wait_st();
      tc05::fence_before();
      tc05::bar_arrive(&S.aready[g]);
    }
    cp_async_wait<0>();
    if (any_past_range(past)) atomicOr(err, OPTR_DEVERR_FP16_RANGE);
  } else if (warp == kMmaWarp) {
    // --------------------------------------------------------------- MMA
    int last = -1;
    const uint32_t b0 = tc05::smem_addr(&S.b[0][0]);
    for (int i = 0; i < my_tiles; ++i) {
      const int g = i & 1, k = i >> 1;
      if (!__all_sync(0xffffffffu, tc05::bar_wait(&S.aready[g], k & 1, abort))) break;
      if (k > 0 && !__all_sync(0xffffffffu, tc05::bar_wait(&S.dfree[g], (k - 1) & 1, abort))) break;
      tc05::fence_after();
      const uint32_t d = tmem + kColD + 128u * g, a = tmem + kColA + 64u * g;
      for (int term = 0; term < 2; ++term)
        tc05::mma128_ts<16>(d, a, tc05::smem_desc(b0 + term * kD * kD * 2, 128, 2048),
                            tc05::idesc_f16(128, 128), term);
      tc05::mma_commit_warp(&S.dready[g]);
      tc05::mma_commit_warp(&S.adone[g]);
      last = i;
    }
    if (last >= 0) {  // the tensor core is done with tensor memory before it is freed
      tc05::bar_wait_drain(&S.dready[last & 1], (last >> 1) & 1);
      tc05::bar_wait_drain(&S.adone[last & 1], (last >> 1) & 1);
    }
  } else {
    // ---------------------------------------------------------- epilogue
    const int g = (warp - kEpiWarp) >> 2, q = warp & 3, row = 32 * q + lane;
    const uint32_t tD = tmem + ((uint32_t)(32 * q) << 16) + kColD + 128u * g;
    const bool leader = q == 0 && lane == 0;
    const CUtensorMap* tmap = kind ? &tmap_v : &tmap_k;
    bool left = false;
    for (int i = g, k = 0; i < my_tiles && !left; i += 2, ++k) {
      const bool ok = __all_sync(0xffffffffu, tc05::bar_wait(&S.dready[g], k & 1, abort));
      tc05::fence_after();
      // a channel half at a time: the other half's copy may still be reading
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint8_t* out = S.stage[g] + half * (kTileBytes / 2);
        if (leader) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        group_sync(1 + g);
        if (ok) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t d[32];
            tc05::tmem_ld32(tD + 64u * half + 32u * c, d);
            tc05::tmem_wait_ld();
            if (half == 1 && c == 1) {
              tc05::fence_before();
              tc05::bar_arrive(&S.dfree[g]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t y[4];
#pragma unroll
              for (int e = 0; e < 4; e += 2) {
                const float4 add =
                    *reinterpret_cast<const float4*>(&S.add[64 * half + 32 * c + 8 * j + 2 * e]);
                const uint32_t* x = &d[8 * j + 2 * e];
                const float2 inv = make_float2(1.f / 64.f, 1.f / 64.f);
                const float2 lo = fma2(make_float2(__uint_as_float(x[0]), __uint_as_float(x[1])),
                                       inv, make_float2(add.x, add.y));
                const float2 hi = fma2(make_float2(__uint_as_float(x[2]), __uint_as_float(x[3])),
                                       inv, make_float2(add.z, add.w));
                const __nv_bfloat162 zl = __floats2bfloat162_rn(lo.x, lo.y);
                const __nv_bfloat162 zh = __floats2bfloat162_rn(hi.x, hi.y);
                y[e] = *reinterpret_cast<const uint32_t*>(&zl);
                y[e + 1] = *reinterpret_cast<const uint32_t*>(&zh);
              }
              *reinterpret_cast<uint4*>(out + row * 128 + (((4 * c + j) ^ (row & 7)) << 4)) =
                  make_uint4(y[0], y[1], y[2], y[3]);
            }
          }
          tc05::fence_proxy_async();
        }
        if (group_any(1 + g, !ok)) {  // the group leaves together
          left = true;
          break;
        }
        if (leader) {
          const int tok0 = ((int)blockIdx.x + i * (int)gridDim.x) * kRows;
          tma_store_3d(tmap, 64 * half, h, tok0, out);
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
      }
    }
    if (leader) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }

  tc05::fence_before();
  __syncthreads();
  if (S.abort && tid == 0) atomicOr(err, OPTR_DEVERR_TIMEOUT);
  if (warp == kMmaWarp) {
    tc05::fence_after();
    tc05::tmem_dealloc(tmem, kTmemCols);
  }
}

}  // namespace
}  // namespace optr

extern "C" optr_status optr_kv_read(const optr_params* p, int n_tok, const int32_t* cu_read,
                                    const int32_t* pos0, const int32_t* block_table, int B,
                                    int max_pages, const uint8_t* pool, int num_pages, void* k,
                                    void* v, cudaStream_t stream) {
  using namespace optr;
  if (!p || n_tok < 0 || B <= 0 || max_pages <= 0 || num_pages <= 0) return OPTR_ERR_INVALID_ARG;
  if (n_tok == 0) return OPTR_OK;
  if (!cu_read || !pos0 || !block_table || !pool || !k || !v) return OPTR_ERR_INVALID_ARG;
  if (!aligned(pool, 16) || !aligned(k, 16) || !aligned(v, 16)) return OPTR_ERR_INVALID_ARG;
  const void *kd = nullptr, *vd = nullptr;
  bool k_host = false, v_host = false;
  // the rows are stored by TMA: device memory only
  if (!io_pointer(k, &kd, &k_host) || !io_pointer(v, &vd, &v_host) || k_host || v_host)
    return OPTR_ERR_INVALID_ARG;
  if ((long long)max_pages * kPage > (1LL << 30)) return OPTR_ERR_OUT_OF_RANGE;
  const int h_kv = p->cfg.h_kv;
  auto fn = p->cfg.group == 4 * kG ? kv_read_kernel<true> : kv_read_kernel<false>;
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(fn), sizeof(Smem));
  if (e != cudaSuccess) return OPTR_ERR_CUDA;
  CUtensorMap mk, mv;
  if (!token_rows_map(&mk, kd, n_tok, h_kv, kRows) || !token_rows_map(&mv, vd, n_tok, h_kv, kRows))
    return OPTR_ERR_CUDA;
  const int tiles = (n_tok + kRows - 1) / kRows;
  const int per = max(1, min(tiles, p->num_sms / (2 * h_kv)));
  return cuda_status(launch_pdl(fn, dim3(per, h_kv, 2), dim3(kThreads), sizeof(Smem), stream, mk, mv,
                                n_tok, cu_read, pos0, block_table, B, max_pages, pool, num_pages,
                                h_kv, (const uint16_t*)p->Rk_back, (const uint16_t*)p->Rv_back,
                                (const float*)p->mu, p->err));
}
