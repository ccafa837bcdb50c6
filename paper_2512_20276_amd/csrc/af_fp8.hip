// gfx950 kernels that write 8-bit floating point (e4m3) with fp32 scales: RMSNorm with the residual's
// addition, and the quantisation of given rows and weights.
//
// A block of values v is stored as q = e4m3(v / s) with s = max(max |v| / 448, 2^-126), rounded to
// nearest even: the largest magnitude lands on 448, the largest e4m3 value, and the floor keeps the
// division defined for a block of zeros.  A block that holds an infinity or a NaN gets s = NaN and
// q = NaN throughout, so that nothing computed from it looks finite.  The quotient is the one that rounding
// v / s to fp32 gives, from a reciprocal that the block's elements share: bf16 elements over a bf16 maximum
// often lie midway between two e4m3 values, where an ulp decides (v times the reciprocal instruction's 1 / s
// alone took the other value for 1.3 to 1.7 in 10^3 of bf16 elements).  (With the division itself, ten
// instructions an element, 22016 x 4096 weights took 59.5 us, bound by them; so 54.5.)
//
// Every kernel here reads its input once, in 16-byte accesses, and is bound by memory: what it holds of a
// block or a row stays in registers between the maximum, or the norm, and the rounding.
#include "af_device.h"
#include "af_fp8.h"

namespace af {

constexpr unsigned INF_BITS = 0x7f800000u;

__device__ __forceinline__ unsigned abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The scale of a block from its largest |v|, as bits: of the magnitudes' bits as integers NaN is the
// largest and infinity the next, so one integer maximum finds either.  The division by 448 is a product with 1 / 448
// and its correction: the rounded quotient for every magnitude that keeps it at 2^-126 or more.
__device__ __forceinline__ float scale_of(unsigned largest) {
  if (largest >= INF_BITS) return __uint_as_float(0x7fc00000u);
  const float m = __uint_as_float(largest), q = m * (1.0f / FP8_MAX);
  return fmaxf(fmaf(-fmaf(q, FP8_MAX, -m), 1.0f / FP8_MAX, q), FP8_MIN_SCALE);
}

// The lane's value rotated by N places within its row of 16 lanes.
template <int N>
__device__ __forceinline__ unsigned ror16(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xf, 0xf, false);
}
// Maximum over the 16 lanes (of 8 values each) that hold one block of 128.
__device__ __forceinline__ unsigned max16(unsigned m) {
  m = max(m, ror16<8>(m));
  m = max(m, ror16<4>(m));
  m = max(m, ror16<2>(m));
  return max(m, ror16<1>(m));
}
// Sum over the wave, in one order (every kernel that normalises a row takes the same).
__device__ __forceinline__ float wave_sum(float v) {
  v += __uint_as_float(ror16<8>(__float_as_uint(v)));
  v += __uint_as_float(ror16<4>(__float_as_uint(v)));
  v += __uint_as_float(ror16<2>(__float_as_uint(v)));
  v += __uint_as_float(ror16<1>(__float_as_uint(v)));
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Eight values over the scale s, as e4m3, in order.  With r = 1 / s and q = v r, each rounded, q - (q s - v) r is
// v / s rounded: the remainder q s - v has no rounding error while its last place, 2^-57 of s for the smallest
// quotient that does not become 0, is a multiple of 2^-149.  Blocks of a smaller scale are taken 2^64 times as large.
// The reciprocal instruction and one Newton step give the rounded 1 / s for all 2^23 significands.  (The remainder's
// sign as it is keeps that of -0.)
__device__ __forceinline__ uint2 pack8(const float* v, float s) {
  const float up = s < 0x1p-92f ? 0x1p64f : 1.0f;  // (as a branch 2264 x 4096 norms took 0.3 us more)
  s *= up;
  float r = __builtin_amdgcn_rcpf(s);
  r = fmaf(fmaf(-s, r, 1.0f), r, r);
  float a[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float w = v[e] * up, q = w * r;
    a[e] = fmaf(-fmaf(q, s, -w), r, q);
  }
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(a[0], a[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(a[2], a[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(a[4], a[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(a[6], a[7], hi, true);
  return make_uint2((unsigned)lo, (unsigned)hi);
}

// Eight elements in their words, for rows that are held for long: in an array of bf16, whose last chunk of a row is
// filled one by one, each has a register of its own.
template <typename T>
struct Eight {
  unsigned w[2 * sizeof(T)];
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
};
__device__ __forceinline__ Eight<float> eight_of(const float* v, float) {
  Eight<float> r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.w[e] = __float_as_uint(v[e]);
  return r;
}
__device__ __forceinline__ Eight<bf16> eight_of(const float* v, bf16) {
  Eight<bf16> r;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bf16 t[2] = {from_f<bf16>(v[2 * e]), from_f<bf16>(v[2 * e + 1])};
    __builtin_memcpy(&r.w[e], t, 4);
  }
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
__device__ __forceinline__ void load_chunk(const T* p, int n, Eight<T>& v) {
  if (n >= 8) {
    __builtin_memcpy(v.w, p, 8 * sizeof(T));
  } else {
    T t[8];
    load_chunk(p, n, t);
    __builtin_memcpy(v.w, t, 8 * sizeof(T));
#pragma unroll
    for (int e = 0; e < (int)(2 * sizeof(T)); ++e) asm volatile("" : "+v"(v.w[e]));  // words from here on
  }
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* p, int n, const Eight<T>& v) {
  if (n >= 8) {
    __builtin_memcpy(p, v.w, 8 * sizeof(T));
  } else {
    T t[8];
    __builtin_memcpy(t, v.w, 8 * sizeof(T));
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = t[e];
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
// WAVES waves to a row: one (rows of up to 512 columns, four rows a workgroup) or eight, CPL chunks of 8
// columns a thread, 16 consecutive lanes to a block of 128 columns.  The row stays in registers; a workgroup
// that has another row to do requests it before it waits for this one's sum.  CPL = 0: longer rows, whose
// second pass reads back what the thread itself wrote (or the input).
// A row is added up in one order, whatever the number of rows.  Where the sum of squares leaves fp32's range it is
// taken again of the row times a power of two.  Three chunks a thread are kept to 128 registers, for two workgroups a
// CU (2264 x 11008 bf16 50.7 us, with 135 registers 60.2).
template <typename T, int WAVES, int CPL>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES, CPL == 3 ? 4 : 1) void add_rmsnorm_fp8_kernel(
    const T* x, const T* resid, const T* __restrict__ g, T* resid_out, uint8_t* __restrict__ q,
    float* __restrict__ scales, int M, int D, int kb, float eps) {
  constexpr int RPW = WAVES == 1 ? 4 : 1;  // rows of a workgroup at a time
  __shared__ float red[3][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c0 = WAVES == 1 ? lane : (int)threadIdx.x;
  constexpr int STEP = 64 * WAVES;
  const int n_ch = kb * 16;  // chunks of 8 columns, whole blocks of them

  auto quantize = [&](size_t row, int c, const Eight<T>& h, const Eight<T>& gv, float inv) {
    const int n = D - 8 * c;
    float y[8];
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = h[e] * inv * gv[e];  // (past the end 0, or NaN as the whole row)
      m = max(m, abs_bits(y[e]));
    }
    const float s = scale_of(max16(m));
    if (n > 0) store_q(q + row * D + 8 * c, n, pack8(y, s));
    if ((c & 15) == 0) scales[row * kb + (c >> 4)] = s;
  };
  // h + r, rounded as it is stored
  auto add = [](Eight<T>& h, const Eight<T>& r) {
    float t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = h[e] + r[e];
    h = eight_of(t, T());
  };
  // the row's sum, from this thread's part of it
  auto row_sum = [&](float ss, int set) {
    ss = wave_sum(ss);
    if constexpr (WAVES > 1) {
      if (lane == 0) red[set][wave] = ss;
      __syncthreads();
      ss = red[set][0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) ss += red[set][w];
    }
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(ss)));  // (the same in every lane)
  };
  // 1 / the root of the mean square and eps, from this thread's part of the sum; scaled(f): the same part of the
  // squares of the row times f.  A sum of 2^128 or more has an element of 2^48, so that of 2^-84 times the row has all
  // that counts; one below 2^-96 has no element of 2^-48, and 2^100 times the row is exact.  (Set 2 is free again by the
  // barrier of the next row's first sum.)
  auto norm_of = [&](float ss, int turn, auto scaled) {
    ss = row_sum(ss, turn);
    float f = 1.0f, e = eps;
    if (ss > 3.402823466e38f) f = 0x1p-84f;  // (or an element is infinite: the second sum is, too)
    else if (ss < 0x1p-96f && eps < 0x1p-110f) f = 0x1p100f;
    if (f != 1.0f) {
      ss = row_sum(scaled(f), 2);
      e = eps * f * f;
    }
    return f * (1.0f / sqrtf(ss / (float)D + e));
  };

  if constexpr (CPL > 0) {
    Eight<T> h[CPL], r[CPL], gv[CPL];
    const size_t step = (size_t)gridDim.x * RPW;
    size_t row = (size_t)blockIdx.x * RPW + (WAVES == 1 ? wave : 0);
    auto load = [&](size_t row) {
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const int c = c0 + STEP * i, n = row < (size_t)M ? D - 8 * c : 0;
        load_chunk(x + row * D + 8 * c, n, h[i]);
        if (resid) load_chunk(resid + row * D + 8 * c, n, r[i]);
      }
    };
    load(row);
#pragma unroll
    for (int i = 0; i < CPL; ++i) load_chunk(g + 8 * (c0 + STEP * i), D - 8 * (c0 + STEP * i), gv[i]);
    for (int turn = 0; row < (size_t)M; row += step, turn ^= 1) {  // a wave's rows are the same for all its lanes
      Eight<T> v[CPL];
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const int c = c0 + STEP * i, n = D - 8 * c;
        v[i] = h[i];
        if (resid) {
          add(v[i], r[i]);
          if (n > 0) store_chunk(resid_out + row * D + 8 * c, n, v[i]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss);
      }
      load(row + step);
      const float inv = norm_of(ss, turn, [&](float f) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < CPL; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fmaf(v[i][e] * f, v[i][e] * f, s);
        return s;
      });
#pragma unroll
      for (int i = 0; i < CPL; ++i)
        if (c0 + STEP * i < n_ch) quantize(row, c0 + STEP * i, v[i], gv[i], inv);
    }
  } else {
    const size_t row = blockIdx.x;
    const T* xr = x + row * D;
    T* hr = resid ? resid_out + row * D : nullptr;
    float ss = 0.f;
    for (int c = c0; c < n_ch; c += STEP) {
      const int n = D - 8 * c;
      Eight<T> h;
      load_chunk(xr + 8 * c, n, h);
      if (resid) {
        Eight<T> r;
        load_chunk(resid + row * D + 8 * c, n, r);
        add(h, r);
        store_chunk(hr + 8 * c, n, h);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(h[e], h[e], ss);
    }
    const T* src = resid ? hr : xr;
    const float inv = norm_of(ss, 0, [&](float f) {
      float s = 0.f;
      for (int c = c0; c < n_ch; c += STEP) {
        Eight<T> h;
        load_chunk(src + 8 * c, D - 8 * c, h);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(h[e] * f, h[e] * f, s);
      }
      return s;
    });
    for (int c = c0; c < n_ch; c += STEP) {
      Eight<T> h, gv;
      load_chunk(src + 8 * c, D - 8 * c, h);
      load_chunk(g + 8 * c, D - 8 * c, gv);
      quantize(row, c, h, gv, inv);
    }
  }
}

// Workgroups of eight waves, three a CU (2264 x 4096 bf16: 14.1 us; two and four 14.4, one row each 14.7).
constexpr int NORM8_WGS = 768;

template <typename T>
static hipError_t norm_launch(const T* x, const T* resid, const T* g, T* resid_out, uint8_t* q, float* scales, int M,
                              int D, float eps, hipStream_t s) {
  const int kb = fp8_blocks(D);
  const dim3 few((unsigned)std::min((M + 3) / 4, 2 * NORM8_WGS)), some((unsigned)std::min(M, NORM8_WGS)), all((unsigned)M);
  if (D <= 512)
    hipLaunchKernelGGL((add_rmsnorm_fp8_kernel<T, 1, 1>), few, dim3(256), 0, s, x, resid, g, resid_out, q, scales, M, D, kb, eps);
  else if (D <= 4096)
    hipLaunchKernelGGL((add_rmsnorm_fp8_kernel<T, 8, 1>), some, dim3(512), 0, s, x, resid, g, resid_out, q, scales, M, D, kb, eps);
  else if (D <= 12288)
    hipLaunchKernelGGL((add_rmsnorm_fp8_kernel<T, 8, 3>), some, dim3(512), 0, s, x, resid, g, resid_out, q, scales, M, D, kb, eps);
  else
    hipLaunchKernelGGL((add_rmsnorm_fp8_kernel<T, 8, 0>), all, dim3(512), 0, s, x, resid, g, resid_out, q, scales, M, D, kb, eps);
  return hipGetLastError();
}

hipError_t launch_add_rmsnorm_fp8(int dtype, const void* x, const void* resid, const void* g, void* resid_out,
                                  void* q, float* scales, int M, int D, float eps, hipStream_t s) {
  return dtype == AF_BF16 ? norm_launch((const bf16*)x, (const bf16*)resid, (const bf16*)g, (bf16*)resid_out,
                                        (uint8_t*)q, scales, M, D, eps, s)
                          : norm_launch((const float*)x, (const float*)resid, (const float*)g, (float*)resid_out,
                                        (uint8_t*)q, scales, M, D, eps, s);
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
