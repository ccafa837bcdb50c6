// gfx950 kernels that write 8-bit floating point (e4m3) with fp32 scales: RMSNorm with the residual's
// addition, and the quantisation of given rows and weights.
//
// A block of values v is stored as q = e4m3(v / s) with s = max(max |v| / 448, 2^-126), rounded to
// nearest even: the largest magnitude lands on 448, the largest e4m3 value, and the floor keeps the
// division defined for a block of zeros.  A block that holds an infinity or a NaN gets s = NaN and
// q = NaN throughout, so that nothing computed from it looks finite.
#include "af_device.h"
#include "af_fp8.h"

namespace af {

constexpr unsigned INF_BITS = 0x7f800000u;

__device__ __forceinline__ unsigned abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The scale of a block from its largest |v|, as bits: of the magnitudes' bits as integers NaN is the
// largest and infinity the next, so one integer maximum finds either.
__device__ __forceinline__ float scale_of(unsigned largest) {
  if (largest >= INF_BITS) return __uint_as_float(0x7fc00000u);
  return fmaxf(__uint_as_float(largest) / FP8_MAX, FP8_MIN_SCALE);
}

// Maximum over the 16 lanes (of 8 values each) that hold one block of 128.
__device__ __forceinline__ unsigned max16(unsigned m) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, o));
  return m;
}

// Eight values as e4m3, in order.
__device__ __forceinline__ uint2 pack8(const float* v, float s) {
  float t[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = v[e] / s;
  uint2 r;
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], hi, true);
  r.x = (unsigned)lo;
  r.y = (unsigned)hi;
  return r;
}

// Eight consecutive elements of a row of which n (1..8, or fewer: none) exist; the rest are zeros.
// Whole chunks move in 16-byte accesses at any alignment that the element type allows.
template <typename T>
__device__ __forceinline__ void load_chunk(const T* p, int n, T* v) {
  if (n >= 8) {
    __builtin_memcpy(v, p, 8 * sizeof(T));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : from_f<T>(0.f);
  }
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* p, int n, const T* v) {
  if (n >= 8) {
    __builtin_memcpy(p, v, 8 * sizeof(T));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = v[e];
  }
}
__device__ __forceinline__ void store_q(uint8_t* p, int n, uint2 q) {
  if (n >= 8) {
    __builtin_memcpy(p, &q, 8);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = (uint8_t)((e < 4 ? q.x >> (8 * e) : q.y >> (8 * (e - 4))) & 255u);
  }
}

// ------------------------------------------------------------------ residual + RMSNorm -> e4m3
// One workgroup per row; 16 consecutive threads hold one block of 128 columns.
constexpr int NORM8_THREADS = 512;

template <typename T>
__global__ __launch_bounds__(NORM8_THREADS) void add_rmsnorm_fp8_kernel(const T* x, const T* resid,
                                                                      const T* __restrict__ g, T* resid_out,
                                                                      uint8_t* __restrict__ q,
                                                                      float* __restrict__ scales, int D, int kb,
                                                                      float eps) {
  __shared__ float red[NORM8_THREADS / 64];
  const size_t row = blockIdx.x;
  const T* xr = x + row * D;
  const T* rr = resid ? resid + row * D : nullptr;
  T* hr = resid ? resid_out + row * D : nullptr;
  const int n_ch = kb * 16;  // chunks of 8 columns, whole blocks of them
  float ss = 0.f;
  for (int c = threadIdx.x; c < n_ch; c += NORM8_THREADS) {
    const int n = D - 8 * c;
    T v[8];
    load_chunk(xr + 8 * c, n, v);
    if (resid) {
      T r[8];
      load_chunk(rr + 8 * c, n, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = from_f<T>(to_f(v[e]) + to_f(r[e]));
      store_chunk(hr + 8 * c, n, v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(to_f(v[e]), to_f(v[e]), ss);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  float tot = red[0];
#pragma unroll
  for (int w = 1; w < NORM8_THREADS / 64; ++w) tot += red[w];
  const float inv = 1.0f / sqrtf(tot / (float)D + eps);
  const T* src = resid ? hr : xr;  // each thread reads back what it wrote
  for (int c = threadIdx.x; c < n_ch; c += NORM8_THREADS) {
    const int n = D - 8 * c;
    T v[8], gv[8];
    load_chunk(src + 8 * c, n, v);
    load_chunk(g + 8 * c, n, gv);
    float y[8];
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = to_f(v[e]) * inv * to_f(gv[e]);
      if (e < n) m = max(m, abs_bits(y[e]));
      else y[e] = 0.f;
    }
    const float s = scale_of(max16(m));
    if (n > 0) store_q(q + row * D + 8 * c, n, pack8(y, s));
    if ((c & 15) == 0) scales[row * kb + (c >> 4)] = s;
  }
}

hipError_t launch_add_rmsnorm_fp8(int dtype, const void* x, const void* resid, const void* g, void* resid_out,
                                  void* q, float* scales, int M, int D, float eps, hipStream_t s) {
  const int kb = fp8_blocks(D);
  if (dtype == AF_BF16)
    hipLaunchKernelGGL(add_rmsnorm_fp8_kernel<bf16>, dim3(M), dim3(NORM8_THREADS), 0, s, (const bf16*)x,
                       (const bf16*)resid, (const bf16*)g, (bf16*)resid_out, (uint8_t*)q, scales, D, kb, eps);
  else
    hipLaunchKernelGGL(add_rmsnorm_fp8_kernel<float>, dim3(M), dim3(NORM8_THREADS), 0, s, (const float*)x,
                       (const float*)resid, (const float*)g, (float*)resid_out, (uint8_t*)q, scales, D, kb, eps);
  return hipGetLastError();
}

// ------------------------------------------------------------------ quantisation
// Blocks of 1 x 128: 16 threads each, blocks in row-major order.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, uint8_t* __restrict__ q,
                                                            float* __restrict__ scales, long n_blocks, int K,
                                                            int kb) {
  const long b = (long)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (b >= n_blocks) return;  // all 16 threads of a block leave together
  const long row = b / kb;
  const int k0 = (int)(b - row * kb) * FP8_BLOCK + 8 * (threadIdx.x & 15), n = K - k0;
  T v[8];
  load_chunk(x + row * K + k0, n, v);
  float f[8];
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    f[e] = to_f(v[e]);
    m = max(m, abs_bits(f[e]));
  }
  const float s = scale_of(max16(m));
  if (n > 0) store_q(q + row * K + k0, n, pack8(f, s));
  if ((threadIdx.x & 15) == 0) scales[b] = s;
}

// Blocks of 128 x 128: one workgroup each, 16 threads a row, 8 rows a thread, all in registers
// between the maximum and the rounding.
template <typename T>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const T* __restrict__ x, uint8_t* __restrict__ q,
                                                              float* __restrict__ scales, int M, int K, int kb) {
  __shared__ unsigned red[4];
  const int bm = blockIdx.x / kb, bk = blockIdx.x % kb;
  const int k0 = bk * FP8_BLOCK + 8 * (threadIdx.x & 15), n = K - k0, r0 = bm * FP8_BLOCK + (threadIdx.x >> 4);
  T v[8][8];
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    load_chunk(x + (size_t)(r < M ? r : 0) * K + (n > 0 ? k0 : 0), r < M ? n : 0, v[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, abs_bits(to_f(v[i][e])));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, o));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  const float s = scale_of(max(max(red[0], red[1]), max(red[2], red[3])));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (r >= M || n <= 0) continue;
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = to_f(v[i][e]);
    store_q(q + (size_t)r * K + k0, n, pack8(f, s));
  }
  if (threadIdx.x == 0) scales[blockIdx.x] = s;
}

template <typename T>
static hipError_t quantize_launch(const T* x, uint8_t* q, float* scales, int M, int K, int block_rows, hipStream_t s) {
  const int kb = fp8_blocks(K);
  if (block_rows == 1) {
    const long nb = (long)M * kb;
    hipLaunchKernelGGL(quantize_rows_kernel<T>, dim3((unsigned)((nb + 15) / 16)), dim3(256), 0, s, x, q, scales, nb, K,
                       kb);
  } else {
    hipLaunchKernelGGL(quantize_blocks_kernel<T>, dim3((unsigned)(fp8_blocks(M) * kb)), dim3(256), 0, s, x, q, scales,
                       M, K, kb);
  }
  return hipGetLastError();
}

hipError_t launch_quantize_fp8(int dtype, const void* x, void* q, float* scales, int M, int K, int block_rows,
                               hipStream_t s) {
  return dtype == AF_BF16 ? quantize_launch((const bf16*)x, (uint8_t*)q, scales, M, K, block_rows, s)
                          : quantize_launch((const float*)x, (uint8_t*)q, scales, M, K, block_rows, s);
}

}  // namespace af
