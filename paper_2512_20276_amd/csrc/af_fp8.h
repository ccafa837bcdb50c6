// Declarations shared by the 8-bit operators and the sampler (af_fp8.hip, af_gemm_fp8.hip,
// af_sample.hip) and their entry points (af_ops.cpp).
#pragma once

#include "af_internal.h"

namespace af {

constexpr int FP8_BLOCK = 128;        // columns (and, for weights, rows) that share a scale
constexpr float FP8_MAX = 448.f;      // largest finite e4m3 value
constexpr float FP8_MIN_SCALE = 1.1754943508222875e-38f;  // 2^-126: the scale of an all-zero block

inline int fp8_blocks(int n) { return n / FP8_BLOCK + (n % FP8_BLOCK != 0); }

// h = x + resid (stored in resid_out; without resid h = x and nothing is stored), then the RMSNorm of h
// in e4m3 with a scale for every 128 columns of a row.
hipError_t launch_add_rmsnorm_fp8(int dtype, const void* x, const void* resid, const void* g, void* resid_out,
                                  void* q, float* scales, int M, int D, float eps, hipStream_t s);
// x [M, K] in e4m3 with a scale for every block of block_rows (1 or 128) x 128.
hipError_t launch_quantize_fp8(int dtype, const void* x, void* q, float* scales, int M, int K, int block_rows,
                               hipStream_t s);

struct Fp8GemmArgs {
  const void* xq;    // [M, K] e4m3
  const float* xs;   // [M, kb]
  const void* wq;    // [N, K] e4m3
  const float* ws;   // [nb, kb]
  void* y;           // [M, N]
  int M, N, K, kb;   // kb: blocks of 128 columns, the last one partial where K % 128 != 0
};
constexpr int FP8_MAX_K = 1 << 22;  // the largest tile's 288 rows take less than 2^31 bytes, so offsets in it fit 32 bits
// Index of the kernel that a product of these sizes takes (in the lists of af_gemm_fp8.hip).
int gemm_fp8_plan(int out_dtype, int M, int N, int K);
hipError_t launch_gemm_fp8(int out_dtype, const Fp8GemmArgs& a, hipStream_t s);

struct SampleArgs {
  const void* logits;  // [rows, V]
  int V;
  const float* temperature;  // [rows] each, or null: off
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniforms;
  int32_t* tokens;
};
constexpr int SAMPLE_MAX_V = 1 << 22;  // the sums of V weights of up to 2^40 stay below 2^62
hipError_t launch_sample(int dtype, const SampleArgs& a, int n_rows, hipStream_t s);

}  // namespace af
