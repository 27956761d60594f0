// Attention of a chunk of new tokens over the paged INT2 cache
// (include/optr.h, "optr_chunk_attention").
#include "append_common.cuh"
#include "optr_internal.cuh"

namespace optr {
namespace {

constexpr int kKeys = 16;  // keys per tile: one page

struct ChunkArgs {
  const __nv_bfloat16 *q, *k, *v;
  int n_tok;
  const int32_t *cu, *pos0;
  int max_new;
  const int32_t* bt;
  int B, max_pages;
  const uint8_t* pool;
  int num_pages;
  WinArgs win;
  int sink, recent, h_kv, fold_v, compact;
  const float *R_k, *R_vT, *mu;
  __nv_bfloat16* out;
  unsigned* err;
};

// A block per (new token, KV head): thread = channel, warp = query head.
__global__ void __launch_bounds__(128) chunk_simple_kernel(const ChunkArgs A) {
  __shared__ float qx[4][kD], qr[4][kD], K[kKeys][kD + 1], V[kKeys][kD], P[4][kKeys], alpha[4], L[4];
  const int t = blockIdx.x, h = blockIdx.y, c = threadIdx.x, w = c >> 5, lane = c & 31;
  pdl_wait();
  pdl_trigger();
  const float scale = 1.44269504f * 0.08838834764831845f;
  const int b = find_seq(A.cu, A.B, t);
  const int c0 = __ldcg(A.cu + b), c1 = __ldcg(A.cu + b + 1), n = __ldcg(A.pos0 + b);
  __nv_bfloat16* out = A.out + ((size_t)t * 4 * A.h_kv + 4 * h) * kD;
  unsigned bad = 0;
  if (!(c0 <= t && t < c1 && c0 >= 0 && c1 <= A.n_tok && c1 - c0 <= A.max_new)) bad = OPTR_DEVERR_CU_NEW;
  if (n < 0 || n > A.max_pages * kPage) bad = OPTR_DEVERR_SEQ_LEN;
  if (bad) {
    if (c == 0) atomicOr(A.err, bad);
    for (int j = 0; j < 4; ++j) out[j * kD + c] = __float2bfloat16(0.f);
    return;
  }
  for (int j = 0; j < 4; ++j)
    qx[j][c] = scale * __bfloat162float(A.q[((size_t)t * 4 * A.h_kv + 4 * h + j) * kD + c]);
  __syncthreads();
  float r[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < kD; ++i) {
    const float x = A.R_k[((size_t)h * kD + i) * kD + c];
    for (int j = 0; j < 4; ++j) r[j] = fmaf(qx[j][i], x, r[j]);
  }
  for (int j = 0; j < 4; ++j) qr[j][c] = r[j];
  float acc[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;

  // one tile of `cnt` keys in K and V, logits with the queries Q
  auto tile = [&](const float (*Q)[kD], int cnt) {
    __syncthreads();
    const int s = lane & 15, half = lane >> 4;
    float x = 0.f;
    for (int i = 64 * half; i < 64 * half + 64; ++i) x = fmaf(Q[w][i], K[s][i], x);
    x += __shfl_xor_sync(0xffffffffu, x, 16);
    if (s >= cnt) x = -INFINITY;
    float mx = x;
    for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float mn = fmaxf(m, mx);
    const float al = m == -INFINITY ? 0.f : exp2f(m - mn);
    const float p = mn == -INFINITY ? 0.f : exp2f(x - mn);
    float sum = p;
    for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    l = l * al + sum;
    m = mn;
    if (half == 0) P[w][s] = p;
    if (lane == 0) alpha[w] = al;
    __syncthreads();
    for (int j = 0; j < 4; ++j) {
      acc[j] *= alpha[j];
      for (int s2 = 0; s2 < cnt; ++s2) acc[j] = fmaf(P[j][s2], V[s2][c], acc[j]);
    }
    __syncthreads();
  };

  // cached INT2 positions
  const int e = int2_end(n, A.sink, A.recent);
  const int ms = meta_stride(A.compact), g = A.compact ? 0 : c >> 5;
  const int byte = 4 * (c % 32 / 4) + c / 32, bit = 2 * (c % 4);
  for (int s0 = A.sink; s0 < min(e, n); s0 += kKeys) {
    const int page = __ldcg(A.bt + (size_t)b * A.max_pages + s0 / kPage);
    if (page < 0 || page >= A.num_pages) {
      if (c == 0) atomicOr(A.err, OPTR_DEVERR_PAGE_ID);
      continue;
    }
    const uint8_t* rec = A.pool + ((size_t)page * A.h_kv + h) * chunk_bytes(A.compact);
    const int cnt = min(kKeys, min(e, n) - s0);
    for (int s = 0; s < kKeys; ++s) {
      const __half2 mk = *reinterpret_cast<const __half2*>(rec + OPTR_K_META_OFFSET + s * ms + 4 * g);
      const __half2 mv = *reinterpret_cast<const __half2*>(rec + vmeta_offset(A.compact) + s * ms + 4 * g);
      const int ck = rec[OPTR_K_CODES_OFFSET + 32 * s + byte] >> bit & 3;
      const int cv = rec[OPTR_V_CODES_OFFSET + 32 * s + byte] >> bit & 3;
      K[s][c] = s < cnt ? ck * __low2float(mk) + __high2float(mk) : 0.f;
      V[s][c] = s < cnt ? cv * __low2float(mv) + __high2float(mv) : 0.f;
    }
    tile(qr, cnt);
  }
  if (!A.fold_v) {  // the INT2 part into the model's basis
    for (int j = 0; j < 4; ++j) K[j][c] = acc[j];
    __syncthreads();
    for (int j = 0; j < 4; ++j) acc[j] = 0.f;
    for (int i = 0; i < kD; ++i) {
      const float x = A.R_vT[((size_t)h * kD + i) * kD + c];
      for (int j = 0; j < 4; ++j) acc[j] = fmaf(K[j][i], x, acc[j]);
    }
    __syncthreads();
  }
  const float mu = A.mu[h * kD + c];
  // the past's windows: the store's rows, all of them once n >= sink + recent
  if (A.win.win) {
    const int rows = A.sink + A.recent, slot = __ldcg(A.win.slot + b);
    if (slot < 0 || slot >= A.win.n_slots) {
      if (c == 0) atomicOr(A.err, OPTR_DEVERR_WIN_SLOT);
    } else {
      const __nv_bfloat16* wk = A.win.win + ((size_t)slot * A.h_kv + h) * 2 * rows * kD;
      const int have = min(n, rows);
      for (int s0 = 0; s0 < have; s0 += kKeys) {
        const int cnt = min(kKeys, have - s0);
        for (int s = 0; s < kKeys; ++s) {
          K[s][c] = s < cnt ? __bfloat162float(wk[(size_t)(s0 + s) * kD + c]) - mu : 0.f;
          V[s][c] = s < cnt ? __bfloat162float(wk[(size_t)(rows + s0 + s) * kD + c]) : 0.f;
        }
        tile(qx, cnt);
      }
    }
  }
  for (int s0 = c0; s0 <= t; s0 += kKeys) {
    const int cnt = min(kKeys, t + 1 - s0);
    for (int s = 0; s < kKeys; ++s) {
      const size_t at = ((size_t)(s0 + s) * A.h_kv + h) * kD + c;
      K[s][c] = s < cnt ? __bfloat162float(A.k[at]) - mu : 0.f;
      V[s][c] = s < cnt ? __bfloat162float(A.v[at]) : 0.f;
    }
    tile(qx, cnt);
  }
  if (lane == 0) L[w] = l;
  __syncthreads();
  for (int j = 0; j < 4; ++j) out[j * kD + c] = __float2bfloat16(acc[j] / L[j]);
}

}  // namespace
}  // namespace optr

using namespace optr;

extern "C" size_t optr_chunk_workspace_size(const optr_params* p, int n_tok, int B, int max_new) {
  if (!p || n_tok < 0 || B <= 0 || max_new <= 0) return 0;
  return 256;
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
  const void* dev[4] = {q, k, v, out};
  for (const void*& x : dev) {
    bool host = false;
    if (!io_pointer(x, &x, &host) || host) return OPTR_ERR_INVALID_ARG;
  }
  if ((long long)max_pages * kPage > (1LL << 30) || B > (1 << 24)) return OPTR_ERR_OUT_OF_RANGE;
  if (!workspace || ws_bytes < optr_chunk_workspace_size(p, n_tok, B, max_new) || !aligned(workspace, 256))
    return OPTR_ERR_WORKSPACE;
  const ChunkArgs A{(const __nv_bfloat16*)q, (const __nv_bfloat16*)k, (const __nv_bfloat16*)v, n_tok,
                    cu_new, pos0, max_new, block_table, B, max_pages, pool, num_pages, w,
                    p->cfg.sink, p->cfg.recent, p->cfg.h_kv, p->fold_v, p->cfg.group == 4 * kG,
                    p->R_k, p->R_vT, p->mu, (__nv_bfloat16*)out, p->err};
  return cuda_status(launch_pdl(chunk_simple_kernel, dim3(n_tok, p->cfg.h_kv), dim3(128), 0, stream, A));
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
