// gfx950 kernel that draws a token per row of logits with temperature, top-k, top-p and min-p.
//
// Order the tokens by logit, descending, equal ones by index.  With w_i = exp((z_i - max z) / T) the
// kept set is a prefix of that order: its first k tokens; of these the shortest prefix whose weight is
// at least p of theirs; of these the ones with w_i >= min_p (the first token always stays).  The token
// drawn is the lowest index i at which the kept weight of the indices up to i exceeds u times all of it.
//
// The weights are summed as integers, w_i * 2^40 rounded: such sums are the same in any order, so the
// token does not depend on how a row is split over threads, and the weights are computed in 64 bits, so
// that a sum over a long vocabulary still tells neighbouring tokens apart (an fp32 sum of 32000 weights
// is off by more than the share of most of them).  Tokens below 2^-41 of the top one weigh nothing.
#include "af_device.h"
#include "af_fp8.h"

namespace af {

constexpr int SAMPLE_THREADS = 1024;
typedef unsigned long long u64;

// Keys in the order of the logits: 0 for a token that cannot be drawn (-inf, NaN), else larger for a
// larger logit; -0 and 0 are equal.
__device__ __forceinline__ unsigned key_of(float z) {
  if (!(z > -INFINITY)) return 0;
  const unsigned b = __float_as_uint(z + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// exp((z - top) / T) in units of 2^-40; 2^40 for the top logit itself, also where that is infinite.
__device__ __forceinline__ double weight_of(float z, float top, double inv_t) {
  if (z == top) return 1.0;
  const double a = ((double)z - (double)top) * inv_t;
  return a > -29.0 ? exp(a) : 0.0;  // e^-29 < 2^-41
}
constexpr double ONE = 1099511627776.0;  // 2^40
__device__ __forceinline__ u64 units(double w) { return (u64)rint(w * ONE); }

template <typename V>
__device__ __forceinline__ V block_sum(V v, V* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  V t = 0;
  for (int w = 0; w < SAMPLE_THREADS / 64; ++w) t += red[w];
  return t;
}
// Sum over the threads before this one.
__device__ __forceinline__ u64 block_before(u64 v, u64* red) {
  u64 x = v;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 t = __shfl_up(x, o);
    if (lane >= o) x += t;
  }
  __syncthreads();
  if (lane == 63) red[wave] = x;
  __syncthreads();
  u64 base = 0;
  for (int w = 0; w < wave; ++w) base += red[w];
  return base + x - v;
}

template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(SampleArgs a) {
  __shared__ u64 red[16];
  __shared__ u64 hist[256];
  __shared__ unsigned s_key;
  __shared__ u64 s_left;
  const int row = blockIdx.x, tid = threadIdx.x, V = a.V;
  const T* z = (const T*)a.logits + (size_t)row * V;
  const float temp = a.temperature ? a.temperature[row] : 1.f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.f;
  const float min_in = a.min_p ? a.min_p[row] : 0.f, min_p = min_in > 0.f ? fminf(min_in, 1.f) : 0.f;

  // ---- the first largest logit
  unsigned best = 0;
  int at = 0x7fffffff, n_valid = 0;
  for (int i = tid; i < V; i += SAMPLE_THREADS) {
    const unsigned k = key_of(to_f(z[i]));
    n_valid += k != 0;
    if (k > best) {
      best = k;
      at = i;
    }
  }
  u64 top1 = ((u64)best << 32) | (unsigned)~at;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top1 = max(top1, (u64)__shfl_xor(top1, o));
  if ((tid & 63) == 0) red[tid >> 6] = top1;
  __syncthreads();
  for (int w = 0; w < 16; ++w) top1 = max(top1, red[w]);
  const unsigned top_key = (unsigned)(top1 >> 32);
  n_valid = block_sum(n_valid, (int*)red);
  if (top_key == 0 || !(temp > 0.f)) {
    if (tid == 0) a.tokens[row] = top_key == 0 ? 0 : (int)~(unsigned)top1;
    return;
  }
  const float top = value_of(top_key);
  const double inv_t = 1.0 / (double)temp;

  // kept: keys above `cut`, and the first `ties` tokens of key `cut`
  unsigned cut = 1;
  u64 ties = ~0ull;
  // Finds the key at which the running total over the order (of token counts or weights) reaches
  // `want` (1 .. total), and the total of the keys above it.
  auto search = [&](auto amount, u64 want) {
    unsigned prefix = 0;
    u64 left = want;
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = tid; i < V; i += SAMPLE_THREADS) {
        const float v = to_f(z[i]);
        const unsigned k = key_of(v);
        if (k >= cut && k != 0 && (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))))
          atomicAdd(&hist[(k >> shift) & 255], amount(v));
      }
      __syncthreads();
      if (tid == 0) {
        int d = 255;
        u64 l = left;
        for (; d > 0 && hist[d] < l; --d) l -= hist[d];
        s_key = prefix | ((unsigned)d << shift);
        s_left = l;
      }
      __syncthreads();
      prefix = s_key;
      left = s_left;
    }
    cut = prefix;
    return left;
  };
  if (top_k > 0 && top_k < n_valid) ties = search([](float) { return (u64)1; }, (u64)top_k);
  if (top_p < 1.f) {
    u64 above = 0, tied = 0;
    for (int i = tid; i < V; i += SAMPLE_THREADS) {
      const float v = to_f(z[i]);
      const unsigned k = key_of(v);
      if (k > cut) above += units(weight_of(v, top, inv_t));
      tied += k == cut;
    }
    above = block_sum(above, red);
    tied = block_sum(tied, red);
    const u64 each = units(weight_of(value_of(cut), top, inv_t));
    const u64 all = above + min(ties, tied) * each;
    // the first token from which on the weight before it is p of all or more stays out
    const double want_f = ceil((double)fmaxf(top_p, 0.f) * (double)all);
    const u64 want = max((u64)1, min(all, (u64)want_f));
    if (want <= above) {
      const u64 left = search([&](float v) { return units(weight_of(v, top, inv_t)); }, want);
      const u64 w = units(weight_of(value_of(cut), top, inv_t));
      ties = w ? (left + w - 1) / w : 1;
    } else if (each) {
      ties = min(ties, (want - above + each - 1) / each);
    }
  }

  // ---- the draw: contiguous runs of indices per thread
  const int per = (V + SAMPLE_THREADS - 1) / SAMPLE_THREADS, lo = min(V, tid * per), hi = min(V, lo + per);
  u64 mine = 0;
  for (int i = lo; i < hi; ++i) mine += key_of(to_f(z[i])) == cut;
  const u64 tie0 = block_before(mine, red);
  auto kept = [&](int i, u64& tie) {
    const float v = to_f(z[i]);
    const unsigned k = key_of(v);
    bool in = k > cut;
    if (k == cut) in = tie++ < ties;
    const double w = weight_of(v, top, inv_t);
    return in && k != 0 && (w >= (double)min_p || k == top_key) ? units(w) : (u64)0;
  };
  u64 sum = 0, tie = tie0;
  for (int i = lo; i < hi; ++i) sum += kept(i, tie);
  const u64 before = block_before(sum, red);
  const u64 total = block_sum(sum, red);
  const float u = a.uniforms[row];
  u64 target = u > 0.f ? (u64)((double)u * (double)total) : 0;
  target = min(target, total - 1);
  if (target >= before && target < before + sum) {
    u64 c = before;
    tie = tie0;
    int i = lo;
    for (; i < hi; ++i) {
      c += kept(i, tie);
      if (c > target) break;
    }
    a.tokens[row] = i;
  }
}

hipError_t launch_sample(int dtype, const SampleArgs& a, int n_rows, hipStream_t s) {
  if (dtype == AF_BF16)
    hipLaunchKernelGGL(sample_kernel<bf16>, dim3(n_rows), dim3(SAMPLE_THREADS), 0, s, a);
  else
    hipLaunchKernelGGL(sample_kernel<float>, dim3(n_rows), dim3(SAMPLE_THREADS), 0, s, a);
  return hipGetLastError();
}

}  // namespace af
