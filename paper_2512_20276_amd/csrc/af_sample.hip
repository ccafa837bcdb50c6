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
//
// One workgroup of 1024 threads per row, which holds up to 32768 logits in registers, so that a row is
// read once (longer ones are read again, from L2, in every pass).  Nothing is sorted:
//  - top-k of up to 1024: 1024 threads hold a maximum each; the k-th largest of those is a bound that at
//    least k tokens reach and hardly more do.  A histogram of the maxima gives it, the tokens past it
//    (some 50 to 70 for k = 50) meet in LDS, and everything else happens among them.
//  - otherwise a cut is found by a histogram of counts or weights over the distance from the top, in
//    bins of 1/128 of that distance, then again within the bin that holds the cut until it is one value.
#include "af_device.h"
#include "af_fp8.h"

namespace af {

constexpr int SAMPLE_THREADS = 1024;
constexpr int SAMPLE_WAVES = SAMPLE_THREADS / 64;
constexpr int SAMPLE_PER = 32;                            // logits of a thread in registers
constexpr int SAMPLE_TILE = SAMPLE_THREADS * SAMPLE_PER;  // logits of a workgroup in registers
constexpr int SAMPLE_BINS = 4 * SAMPLE_THREADS;
constexpr int SAMPLE_EXP = 64;                            // entries of the table of powers of two
typedef unsigned long long u64;

// ------------------------------------------------------------------ keys
// Logits are taken as they come but for NaN (-inf) and -0 (0).  Keys are in their order; a larger logit
// has a larger key, -inf has key LOWEST - 1.
constexpr unsigned LOWEST = 0x00800000u;
__device__ __forceinline__ float clean(float z) { return fmaxf(z, -INFINITY) + 0.f; }
__device__ __forceinline__ unsigned key_of(float z) {
  const unsigned b = __float_as_uint(z);
  return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// Bin of a distance d >= 0 between keys: 128 to an octave.
__device__ __forceinline__ int bin_of(unsigned d) {
  const int b = (int)(__float_as_uint((float)d) >> 16) - (127 << 7);
  return d == 0 ? 0 : b;  // d = 1: bin 0 too
}
// A distance that no element of bins 0 .. b exceeds (the conversion may have rounded it down).
__device__ __forceinline__ unsigned reach_of(int b) {
  const float f = __uint_as_float(((unsigned)(b + (127 << 7)) << 16) | 0xffffu);
  return f >= 4294966784.f ? 0xffffffffu : (unsigned)(f * 1.0000005f) + 1u;
}

// ------------------------------------------------------------------ sums over lanes
// The lane's value moved by a DPP control; lanes without a source, or in rows masked out, get 0.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ u64 dpp64(u64 v) {
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)v, CTRL, ROWS, 0xf, false);
  const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(v >> 32), CTRL, ROWS, 0xf, false);
  return ((u64)hi << 32) | lo;
}
// Inclusive sums over the 16 lanes of a row, and over the wave.
__device__ __forceinline__ u64 row_scan(u64 v) {
  v += dpp64<0x111>(v);
  v += dpp64<0x112>(v);
  v += dpp64<0x114>(v);
  return v + dpp64<0x118>(v);
}
__device__ __forceinline__ u64 wave_scan(u64 v) {
  v = row_scan(v);
  v += dpp64<0x142, 0xa>(v);  // the last lane of rows 0 and 2 to rows 1 and 3
  return v + dpp64<0x143, 0xc>(v);  // the last lane of row 1 to rows 2 and 3
}
__device__ __forceinline__ u64 readlane64(u64 v, int lane) {
  return ((u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(v >> 32), lane) << 32) |
         (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, lane);
}

struct SampleLds {
  u64 hist[SAMPLE_BINS];
  u64 cand[SAMPLE_THREADS];
  double exp2[SAMPLE_EXP];
  u64 red[2][SAMPLE_WAVES];
  float redf[SAMPLE_WAVES];
  u64 left, tile_total[SAMPLE_MAX_V / SAMPLE_TILE];
  unsigned lo, hi;
  int bin, n, at;
};

// Sum over the threads before this one, and over all.  (turn: which of two sets of sums in LDS; a set is
// free for the call after next, since every call has a barrier.)
__device__ __forceinline__ u64 block_scan(u64 v, SampleLds& l, int turn, u64* total) {
  const u64 x = wave_scan(v);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 63) l.red[turn][wave] = x;
  __syncthreads();
  u64 before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < SAMPLE_WAVES; ++w) {
    const u64 t = l.red[turn][w];
    all += t;
    before += w < wave ? t : 0;
  }
  *total = all;
  return before + x - v;
}

// exp((z - top) / T) in units of 2^-40: c = log2(e) / T, powers of two from a table and a polynomial,
// 2^a = 2^(j / 64) 2^r with |r| <= 1/128, off by less than 1e-13 of itself.
struct Weigh {
  double top, c;
  const double* table;
  __device__ __forceinline__ u64 operator()(float z) const {
    const double a = ((double)z - top) * c;
    if (!(a > -41.5)) return (double)z == top ? (u64)1 << 40 : 0;  // also where both are infinite, or c is
    const double j = rint(a * 64.0), r = fma(j, -1.0 / 64.0, a);
    const int n = (int)j;
    // exp(r ln 2) - 1 to the fourth power
    double p = fma(r, 9.618129107628477e-3, 5.550410866482158e-2);
    p = fma(r, p, 2.402265069591007e-1);
    p = fma(r, p, 6.931471805599453e-1);
    const double t = table[n & 63];
    const double w = ldexp(fma(t * r, p, t), 40 + (n >> 6));
    return (u64)__double_as_longlong(w + 4503599627370496.0) & 0xfffffffffffffULL;  // + 2^52: rounded to a whole number
  }
};

// ONE: the row fits the registers of the workgroup.
template <typename T, bool ONE>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(SampleArgs a) {
  constexpr int VEC = 16 / sizeof(T), U = SAMPLE_PER / VEC;  // logits of a load, loads of a thread and tile
  __shared__ SampleLds l;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V;
  const T* zr = (const T*)a.logits + (size_t)row * V;
  const float temp = a.temperature ? a.temperature[row] : 1.f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.f;
  const float min_in = a.min_p ? a.min_p[row] : 0.f;
  const u64 least = min_in > 0.f ? (u64)ceil((double)fminf(min_in, 1.f) * 1099511627776.0) : 0;
  const int n_tiles = ONE ? 1 : (V + SAMPLE_TILE - 1) / SAMPLE_TILE;
  if (tid < SAMPLE_EXP) l.exp2[tid] = exp2((double)tid * (1.0 / SAMPLE_EXP));

  // ---- the row: element e of load u of a thread is logit tile * TILE + VEC (1024 u + tid) + e
  float z[SAMPLE_PER];
  auto load_tile = [&](int tile) {
    const int base = tile * SAMPLE_TILE + VEC * tid;
    T raw[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = base + VEC * SAMPLE_THREADS * u;
      if (i + VEC <= V) {
        __builtin_memcpy(raw[u], zr + i, 16);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) raw[u][e] = i + e < V ? zr[i + e] : from_f<T>(-INFINITY);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < VEC; ++e) z[u * VEC + e] = clean(to_f(raw[u][e]));
  };
  auto index_of = [&](int tile, int q) { return tile * SAMPLE_TILE + VEC * (SAMPLE_THREADS * (q / VEC) + tid) + q % VEC; };
  // The logit, as a value that the compiler knows nothing of: what a pass computes from it is not kept in
  // registers for the next pass, which has no room for it.
  auto fresh = [&](auto q) {
    asm volatile("" : "+v"(z[q]));
    return z[q];
  };
  // f(logit, tile, its number in the thread) for every logit of the thread
  auto each = [&](auto f) {
    for (int tile = 0; tile < n_tiles; ++tile) {
      if constexpr (!ONE) load_tile(tile);
      static_for<0, SAMPLE_PER>([&](auto q) {
        f(fresh(q), tile, (int)decltype(q)::value);
        __builtin_amdgcn_sched_barrier(0);
      });
    }
  };
  if constexpr (ONE) load_tile(0);

  // ---- the largest logit
  float mine = -INFINITY;
  each([&](float v, int, int) { mine = fmaxf(mine, v); });
  float top = mine;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if (lane == 0) l.redf[wave] = top;
  if (tid == 0) {
    l.n = 0;
    l.at = 0x7fffffff;
  }
#pragma unroll
  for (int i = 0; i < SAMPLE_BINS / SAMPLE_THREADS; ++i) l.hist[tid + SAMPLE_THREADS * i] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SAMPLE_WAVES; ++w) top = fmaxf(top, l.redf[w]);
  if (top == -INFINITY) {
    if (tid == 0) a.tokens[row] = 0;
    return;
  }
  if (!(temp > 0.f)) {  // the greedy token
    int at = 0x7fffffff;
    if (mine == top) each([&](float v, int tile, int q) { at = min(at, v == top ? index_of(tile, q) : 0x7fffffff); });
    if (at != 0x7fffffff) atomicMin(&l.at, at);
    __syncthreads();
    if (tid == 0) a.tokens[row] = l.at;
    return;
  }
  const unsigned top_key = key_of(top);
  const Weigh weigh{(double)top, 1.4426950408889634 / (double)temp, l.exp2};
  const float u_in = a.uniforms[row];
  const double u = u_in > 0.f ? (double)u_in : 0.0;
  auto target_of = [&](u64 total) { return min((u64)fmin(u * (double)total, 9.0e18), total - 1); };
  // the weight that the kept prefix of a total has to reach
  auto want_of = [&](u64 total) {
    return max((u64)1, min(total, (u64)ceil((double)fmaxf(top_p, 0.f) * (double)total)));
  };
  // The bin in which the running sum over the bins reaches `want`: l.bin, with what is wanted of it in l.left.
  // False where all bins together do not.
  auto find_bin = [&](u64 want, int turn) {
    u64 b[4], total;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = l.hist[4 * tid + i];
    u64 before = block_scan(b[0] + b[1] + b[2] + b[3], l, turn, &total);
    if (total < want) return false;  // the same for all threads
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (before < want && want <= before + b[i]) {
        l.bin = 4 * tid + i;
        l.left = want - before;
      }
      before += b[i];
    }
    __syncthreads();
    return true;
  };

  // ---- few of the top: among the tokens that may be
  if (top_k > 0 && top_k <= SAMPLE_THREADS) {
    if (mine > -INFINITY) atomicAdd(&l.hist[bin_of(top_key - key_of(mine))], (u64)1);
    __syncthreads();
    unsigned low = LOWEST;
    if (find_bin((u64)top_k, 0)) low = top_key - min(reach_of(l.bin), top_key - LOWEST);
    const float bound = value_of(low);  // with fewer maxima than k every token
    if (mine >= bound)
      each([&](float v, int tile, int q) {
        if (v >= bound) {
          const int at = atomicAdd(&l.n, 1);
          if (at < SAMPLE_THREADS) l.cand[at] = ((u64)key_of(v) << 32) | (unsigned)~index_of(tile, q);
        }
      });
    __syncthreads();
    const int n = l.n;
    if (n <= SAMPLE_THREADS) {
      // order them: a token's place is the number of larger (key, ~index)
      u64* const sorted = l.hist;                    // [1024]
      u64* const weight = l.hist + SAMPLE_THREADS;   // [1024]
      if (tid < n) {
        const u64 c = l.cand[tid];
        int place = 0;
        for (int j = 0; j < n; ++j) place += l.cand[j] > c;
        sorted[place] = c;
      }
      __syncthreads();
      const bool in = tid < min(n, top_k);
      const u64 c = in ? sorted[tid] : 0;
      u64 w = in ? weigh(value_of((unsigned)(c >> 32))) : 0, total;
      const u64 before = block_scan(w, l, 1, &total);
      if (tid > 0 && ((top_p < 1.f && before >= want_of(total)) || w < least)) w = 0;
      if (in) weight[tid] = w;
      block_scan(w, l, 0, &total);  // (its barrier: the weights are written)
      const u64 target = target_of(total);
      if (w > 0) {
        u64 sum = 0;  // of the kept tokens of a lower index
        const int m = min(n, top_k);
        for (int j = 0; j < m; ++j) sum += (unsigned)sorted[j] > (unsigned)c ? weight[j] : 0;
        if (sum <= target && target < sum + w) a.tokens[row] = (int)~(unsigned)c;
      }
      return;
    }
    // more equal tokens than places: the long way
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SAMPLE_BINS / SAMPLE_THREADS; ++i) l.hist[tid + SAMPLE_THREADS * i] = 0;
    __syncthreads();
  }

  // ---- cuts: kept are the keys above `cut` and the first `ties` tokens of key `cut`
  unsigned cut = LOWEST - 1;
  u64 ties = ~0ull;
  // Moves the cut to where the running sum of `amount` over the tokens above the old cut reaches `want`;
  // returns what is wanted of the tokens at it.  l.hist holds the first histogram (see bin_of).
  auto narrow = [&](u64 want, auto amount) {
    unsigned lo = cut + 1, hi = top_key;
    int shift = -1;
    for (;;) {
      find_bin(want, 0);
      want = l.left;
      const int bin = l.bin;
      auto in_bin = [&](unsigned k) { return (shift < 0 ? bin_of(top_key - k) : (int)((hi - k) >> shift)) == bin; };
      // the range of the keys in the bin
      unsigned kl = 0xffffffffu, kh = 0;
      each([&](float v, int, int) {
        const unsigned k = key_of(v);
        if (k >= lo && k <= hi && in_bin(k)) {
          kl = min(kl, k);
          kh = max(kh, k);
        }
      });
      if (tid == 0) {
        l.lo = 0xffffffffu;
        l.hi = 0;
      }
      __syncthreads();  // every thread has read l.bin and its bins
#pragma unroll
      for (int i = 0; i < SAMPLE_BINS / SAMPLE_THREADS; ++i) l.hist[tid + SAMPLE_THREADS * i] = 0;
      if (kh) {
        atomicMin(&l.lo, kl);
        atomicMax(&l.hi, kh);
      }
      __syncthreads();
      lo = l.lo;
      hi = l.hi;
      if (lo == hi) break;
      shift = 0;
      while ((hi - lo) >> shift >= (unsigned)SAMPLE_BINS) ++shift;
      each([&](float v, int, int) {
        const unsigned k = key_of(v);
        if (k >= lo && k <= hi) atomicAdd(&l.hist[(hi - k) >> shift], amount(v));
      });
      __syncthreads();
    }
    cut = lo;
    return want;
  };
  if (top_k > 0) {
    each([&](float v, int, int) {
      if (v > -INFINITY) atomicAdd(&l.hist[bin_of(top_key - key_of(v))], (u64)1);
    });
    __syncthreads();
    u64 valid = 0, b = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) b += l.hist[4 * tid + i];
    block_scan(b, l, 1, &valid);
    if ((u64)top_k < valid) {
      ties = narrow((u64)top_k, [](float) { return (u64)1; });
    } else {
      __syncthreads();  // the bins have been read
#pragma unroll
      for (int i = 0; i < SAMPLE_BINS / SAMPLE_THREADS; ++i) l.hist[tid + SAMPLE_THREADS * i] = 0;
      __syncthreads();
    }
  }
  if (top_p < 1.f) {
    const float cut_v = value_of(cut);
    u64 sum = 0, tied = 0, above, n_tied;
    each([&](float v, int, int) {
      if (v > cut_v) {
        const u64 w = weigh(v);
        sum += w;
        if (w) atomicAdd(&l.hist[bin_of(top_key - key_of(v))], w);
      }
      tied += v == cut_v;
    });
    block_scan(sum, l, 0, &above);
    block_scan(tied, l, 1, &n_tied);
    const u64 at_cut = cut >= LOWEST ? weigh(cut_v) : 0, want = want_of(above + min(ties, n_tied) * at_cut);
    if (want <= above) {
      const u64 left = narrow(want, weigh), w = weigh(value_of(cut));
      ties = (left + w - 1) / w;
    } else {
      ties = min(ties, (want - above + at_cut - 1) / at_cut);
    }
  }

  // ---- the last index of a token at the cut that is kept
  const float cut_v = value_of(cut);
  // Finds the thread's part of a running sum in index order: with amount(value, index), the first index at
  // which the sum exceeds what target_of_total(total) says (l.at), if it does.
  auto locate = [&](auto amount, auto target_of_total) {
    u64 total = 0;
    int tile = 0;
    u64 target = 0;
    if constexpr (!ONE) {
      for (int t = 0; t < n_tiles; ++t) {
        load_tile(t);
        u64 s = 0, all;
        static_for<0, SAMPLE_PER>([&](auto q) {
          s += amount(fresh(q), index_of(t, q));
          __builtin_amdgcn_sched_barrier(0);
        });
        block_scan(s, l, t & 1, &all);
        if (tid == 0) l.tile_total[t] = all;
        total += all;
      }
      __syncthreads();
      target = target_of_total(total);
      u64 sum = 0;
      for (tile = 0; tile < n_tiles - 1; ++tile) {
        if (target < sum + l.tile_total[tile]) break;
        sum += l.tile_total[tile];
      }
      target -= min(target, sum);
      load_tile(tile);
    }
    // sums of 16 threads and one load: U x 64 of them, in index order
    u64 part[U];
    static_for<0, U>([&](auto u_c) {
      constexpr int Q = decltype(u_c)::value * VEC;
      u64 s = 0;
      static_for<Q, Q + VEC>([&](auto q) {
        s += amount(fresh(q), index_of(tile, q));
        __builtin_amdgcn_sched_barrier(0);
      });
      part[u_c] = s;
      s = row_scan(s);
      if ((lane & 15) == 15) l.cand[decltype(u_c)::value * 64 + (tid >> 4)] = s;
    });
    __syncthreads();
    u64 all;
    const u64 v = tid < U * 64 ? l.cand[tid] : 0;
    const u64 before = block_scan(v, l, 0, &all);
    if constexpr (ONE) target = target_of_total(all);
    if (before <= target && target < before + v) {
      l.bin = tid;
      l.left = target - before;
    }
    __syncthreads();
    if (target < all) {
      const int bin = l.bin;
      if ((tid >> 4) == (bin & 63)) {
        u64 left = l.left;
        static_for<0, U>([&](auto u_c) {
          constexpr int Q = decltype(u_c)::value * VEC;
          if ((bin >> 6) != decltype(u_c)::value) return;
          const u64 s = part[u_c], upto = row_scan(s);
          if (upto - s <= left && left < upto) {
            u64 c = upto - s;
            int at = 0x7fffffff;
            static_for<Q, Q + VEC>([&](auto q) {
              c += amount(fresh(q), index_of(tile, q));
              if (c > left) at = min(at, index_of(tile, q));
            });
            l.at = at;
          }
        });
      }
    }
    __syncthreads();
  };
  int last = V;
  if (ties != ~0ull) {
    // the ties-th token of key `cut` (all of them where there are no more)
    if (tid == 0) l.at = V;
    locate([&](float v, int) { return (u64)(v == cut_v); }, [&](u64) { return ties - 1; });
    last = l.at;
  }
  // ---- the draw
  locate(
      [&](float v, int i) {
        const u64 w = v > cut_v || (v == cut_v && v > -INFINITY && i <= last) ? weigh(v) : 0;
        return w >= least || v == top ? w : (u64)0;
      },
      [&](u64 total) { return target_of(total); });
  if (tid == 0) a.tokens[row] = l.at;
}

template <typename T>
static hipError_t sample_launch(const SampleArgs& a, int n_rows, hipStream_t s) {
  if (a.V <= SAMPLE_TILE)
    hipLaunchKernelGGL((sample_kernel<T, true>), dim3(n_rows), dim3(SAMPLE_THREADS), 0, s, a);
  else
    hipLaunchKernelGGL((sample_kernel<T, false>), dim3(n_rows), dim3(SAMPLE_THREADS), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_sample(int dtype, const SampleArgs& a, int n_rows, hipStream_t s) {
  return dtype == AF_BF16 ? sample_launch<bf16>(a, n_rows, s) : sample_launch<float>(a, n_rows, s);
}

}  // namespace af
