// gfx950 matrix product of e4m3 activations and weights with a scale for each block of 128:
//   y[m, n] = sum_b xs[m, b] ws[n / 128, b] sum_{k in block b} xq[m, k] wq[n, k].
// The inner sum is one matrix instruction of K = 128 (v_mfma_f32_16x16x128_f8f6f4) that starts from
// zero; its fp32 result is added to the fp32 accumulator times the product of the two scales.
#include "af_device.h"
#include "af_fp8.h"

namespace af {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// D[i][j] = sum_k A[i][k] B[j][k]: lane l holds bytes k = 32 (l / 16) .. +31 of row i = l % 16 of A and of
// row j = l % 16 of B, and receives D[4 (l / 16) + e][l % 16], e = 0..3.
__device__ __forceinline__ f32x4 mma_fp8(i32x8 a, i32x8 b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}

__device__ __forceinline__ void store4(float* p, const float* v, int n) {
  if (n >= 4) __builtin_memcpy(p, v, 16);
  else
    for (int e = 0; e < n; ++e) p[e] = v[e];
}
__device__ __forceinline__ void store4(bf16* p, const float* v, int n) {
  bf16 t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = from_f<bf16>(v[e]);
  if (n >= 4) __builtin_memcpy(p, t, 8);
  else
    for (int e = 0; e < n; ++e) p[e] = t[e];
}

// One wave per 16 x 16 outputs, operands straight from memory.  The weights are the first operand, so
// that a lane holds four consecutive columns of one row.
template <typename O>
__global__ __launch_bounds__(64) void gemm_fp8_kernel(Fp8GemmArgs a) {
  const int lane = threadIdx.x, lr = lane & 15, lg = lane >> 4;
  const int n_mt = (a.M + 15) >> 4;
  const int mt = blockIdx.x % n_mt, nt = blockIdx.x / n_mt;
  const int m = min(mt * 16 + lr, a.M - 1), n = min(nt * 16 + lr, a.N - 1);  // past the end: a valid row, never stored
  const uint8_t* xp = (const uint8_t*)a.xq + (size_t)m * a.K;
  const uint8_t* wp = (const uint8_t*)a.wq + (size_t)n * a.K;
  const float* xs = a.xs + (size_t)m * a.kb;
  const float* ws = a.ws + (size_t)(nt * 16 / FP8_BLOCK) * a.kb;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int b = 0; b < a.kb; ++b) {
    uint4 xv[2], wv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = b * FP8_BLOCK + lg * 32 + 16 * h;  // K % 16 == 0: a chunk is wholly inside or outside
      xv[h] = k < a.K ? *(const uint4*)(xp + k) : zero4();
      wv[h] = k < a.K ? *(const uint4*)(wp + k) : zero4();
    }
    i32x8 xf, wf;
    __builtin_memcpy(&xf, xv, 32);
    __builtin_memcpy(&wf, wv, 32);
    const f32x4 d = mma_fp8(wf, xf);
    const float s = xs[b] * ws[b];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = fmaf(d[e], s, acc[e]);
  }
  const int mo = mt * 16 + lr, no = nt * 16 + lg * 4;
  if (mo < a.M && no < a.N) store4((O*)a.y + (size_t)mo * a.N + no, acc, a.N - no);
}

hipError_t launch_gemm_fp8(int out_dtype, const Fp8GemmArgs& a, hipStream_t s) {
  const long tiles = (long)((a.M + 15) / 16) * ((a.N + 15) / 16);
  if (out_dtype == AF_BF16)
    hipLaunchKernelGGL(gemm_fp8_kernel<bf16>, dim3((unsigned)tiles), dim3(64), 0, s, a);
  else
    hipLaunchKernelGGL(gemm_fp8_kernel<float>, dim3((unsigned)tiles), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace af
