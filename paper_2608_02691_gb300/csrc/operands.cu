// Tensor-core operands of the rotations, built once per params on the device
// (optr_params_create).
#include "dequant.cuh"
#include "optr_internal.cuh"

namespace optr {
namespace {

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&x);
}

// fp16 hi and lo parts of 64 x at element (n, k) of a tcgen05 B operand: K-major
// without swizzle, core matrices of 8 columns n x 8 inner indices k, 128 B apart
// along k (LBO) and 2048 B along n (SBO); 32 KB a part.
__device__ __forceinline__ void put_tc05(uint16_t* out, int n, int k, float x) {
  const int off = ((n / 8) * 2048 + (k / 8) * 128 + (n % 8) * 16 + (k % 8) * 2) / 2;
  const __half hi = __float2half_rn(x * 64.0f);
  out[off] = __half_as_ushort(hi);
  out[kD * kD + off] = __half_as_ushort(__float2half_rn(x * 64.0f - __half2float(hi)));
}

// z R (forward, the cache write) and z R^T with the inner index in the order
// of dequantized rows (back), of one head and kind per block.
__global__ void tc05_operands_kernel(const float* R_k, const float* R_v, uint16_t* k_fwd,
                                     uint16_t* v_fwd, uint16_t* k_back, uint16_t* v_back) {
  const int h = blockIdx.x;
  const float* R = (blockIdx.y ? R_v : R_k) + (size_t)h * kD * kD;
  uint16_t* fwd = (blockIdx.y ? v_fwd : k_fwd) + (size_t)h * kRT5Halves;
  uint16_t* back = (blockIdx.y ? v_back : k_back) + (size_t)h * kRT5Halves;
  for (int i = threadIdx.x; i < kD * kD; i += blockDim.x) {
    const int n = i / kD, k = i % kD;
    put_tc05(fwd, n, k, R[k * kD + n]);
    put_tc05(back, n, k, R[n * kD + row_channel(k)]);
  }
}

// mma.sync B fragments of R_k (bf16 hi + lo, 17 bits of it), columns in the
// order of dequantized rows: [head][column tile pair w][k step][tile][lane]
// {hi b0, hi b1, lo b0, lo b1}.
__global__ void rk_fragments_kernel(const float* R_k, uint4* out) {
  const int h = blockIdx.x;
  for (int i = threadIdx.x; i < 8 * 8 * 2 * 32; i += blockDim.x) {
    const int lane = i & 31, nt = (i >> 5) & 1, ks = (i >> 6) & 7, w = i >> 9;
    const int c = row_channel(8 * (2 * w + nt) + lane / 4);
    float x[4], lo[4];
    for (int j = 0; j < 4; ++j) {
      const int k = 16 * ks + 2 * (lane % 4) + (j & 1) + 8 * (j >> 1);
      x[j] = R_k[((size_t)h * kD + k) * kD + c];
      lo[j] = x[j] - __bfloat162float(__float2bfloat16_rn(x[j]));
    }
    out[(size_t)h * 4096 + i] = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]),
                                           bf16_pair(lo[0], lo[1]), bf16_pair(lo[2], lo[3]));
  }
}

}  // namespace

cudaError_t build_operands(optr_params* p) {
  const int H = p->cfg.h_kv;
  const size_t bytes = sizeof(uint16_t) * (size_t)H * kRT5Halves;
  cudaError_t e = cudaSuccess;
  for (uint16_t** x : {&p->Rk_t5, &p->Rv_t5, &p->Rk_back, &p->Rv_back})
    if (e == cudaSuccess) e = cudaMalloc(x, bytes);
  if (e == cudaSuccess) e = cudaMalloc(&p->Rk_frag, sizeof(uint4) * 4096 * (size_t)H);
  if (e != cudaSuccess) return e;
  tc05_operands_kernel<<<dim3(H, 2), 256>>>(p->R_k, p->R_v, p->Rk_t5, p->Rv_t5, p->Rk_back,
                                            p->Rv_back);
  rk_fragments_kernel<<<H, 256>>>(p->R_k, p->Rk_frag);
  e = cudaGetLastError();
  return e == cudaSuccess ? cudaStreamSynchronize(nullptr) : e;
}

}  // namespace optr
