// Tensor-core operands of the rotations, built once per params on the device
// (optr_params_create).
#include "dequant.cuh"
#include "optr_internal.cuh"

namespace optr {
namespace {

// Element (n, k) of a tcgen05 B operand, K-major without swizzle: core matrices
// of 8 columns n x 8 inner indices k, 128 B apart along k (LBO) and 2048 B along
// n (SBO), 32 KB.
__device__ __forceinline__ int tc05_offset(int n, int k) {
  return ((n / 8) * 2048 + (k / 8) * 128 + (n % 8) * 16 + (k % 8) * 2) / 2;
}

// fp16 hi and lo parts of 64 x.
__device__ __forceinline__ void put_tc05(uint16_t* out, int n, int k, float x) {
  const int off = tc05_offset(n, k);
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

// R_k as bf16 hi + lo (17 bits of it) in the same layout, columns in the order
// of dequantized rows: queries are rotated as they come, in bf16.
__global__ void query_operand_kernel(const float* R_k, uint16_t* out) {
  const int h = blockIdx.x;
  for (int i = threadIdx.x; i < kD * kD; i += blockDim.x) {
    const int n = i / kD, k = i % kD;
    const float x = R_k[((size_t)h * kD + k) * kD + row_channel(n)];
    const __nv_bfloat16 hi = __float2bfloat16_rn(x);
    uint16_t* o = out + (size_t)h * kRT5Halves + tc05_offset(n, k);
    o[0] = __bfloat16_as_ushort(hi);
    o[kD * kD] = __bfloat16_as_ushort(__float2bfloat16_rn(x - __bfloat162float(hi)));
  }
}

}  // namespace

cudaError_t build_operands(optr_params* p) {
  const int H = p->cfg.h_kv;
  const size_t bytes = sizeof(uint16_t) * (size_t)H * kRT5Halves;
  cudaError_t e = cudaSuccess;
  for (uint16_t** x : {&p->Rk_t5, &p->Rv_t5, &p->Rk_back, &p->Rv_back, &p->Rk_query})
    if (e == cudaSuccess) e = cudaMalloc(x, bytes);
  if (e != cudaSuccess) return e;
  tc05_operands_kernel<<<dim3(H, 2), 256>>>(p->R_k, p->R_v, p->Rk_t5, p->Rv_t5, p->Rk_back,
                                            p->Rv_back);
  query_operand_kernel<<<H, 256>>>(p->R_k, p->Rk_query);
  e = cudaGetLastError();
  return e == cudaSuccess ? cudaStreamSynchronize(nullptr) : e;
}

}  // namespace optr
