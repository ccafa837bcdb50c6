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
// One workgroup of 1024 threads per row, which keeps a row of up to 32768 logits in LDS, so that memory
// is read once (longer ones are read again in every pass, 32 to 48 KB of a row under way at a time).  Passes are
// loops over chunks of 16 bytes a thread: with the row in registers they were unrolled 32 times, and
// fetching those instructions took longer than executing them (64 rows of 32000 fp32 logits, top_p alone:
// 45.6 us, as loops 36.5).
// Nothing is sorted:
//  - top-k of up to 1024: 1024 threads hold a maximum each; the k-th largest of those is a bound that at
//    least k tokens reach and hardly more do.  A histogram of the maxima gives it, the tokens past it
//    (some 50 to 70 for k = 50) meet in LDS, and everything else happens among them.
//  - otherwise a cut is found by a histogram: of weights (top-p) over the weight's logarithm, of counts
//    (top-k) over the distance from the top logit in bins of 1/128 or 1/256 of it; the tokens of the bin that
//    holds the cut are put into order where they are few, else the bin is divided again.  (Weights over
//    the distance too met in few bins, where those below 0 are far from any above it: 64 x 32000 fp32
//    with settings of every kind 47.4 us, so 36.1.)
//  - bf16 logits have few values: the weight of each is computed once into a table in LDS, the cut of top-p
//    is found by counting values, and the draw adds up weights that it reads, two tokens an instruction
//    up to there (256 rows of 131072, top_p alone: 177 us with weights computed token by token, 65 so).
// Bound: with top_k, reading the row and the chain of some ten barriers (64 x 32000 fp32, k = 50: 12 us;
// the read alone is 1.6 us over the whole card, but 64 of 256 CUs have a row); else, for fp32, the 64-bit
// weights, some 25 instructions a token and pass on the one CU that has the row (64 x 32000: 14 us with
// temperature alone, 33 with top_p), for bf16 the passes' accesses to LDS, a token each (256 x 131072:
// 41 us with temperature alone, of which 30 are two passes that only compare; 65 with top_p).  A row stays
// on one CU, since sharing it needs a wait between workgroups and these calls come behind a projection that
// costs more.

#include "af_device.h"
#include "af_fp8.h"

namespace af {

constexpr int SAMPLE_THREADS = 1024;
constexpr int SAMPLE_WAVES = SAMPLE_THREADS / 64;
constexpr int SAMPLE_HELD = 32768;                        // logits of a row that is kept in LDS
constexpr int SAMPLE_FEW = 256;                           // tokens of a bin that are put into order
constexpr int SAMPLE_SPAN = 15 * 128;                     // bf16 magnitudes with a weight in LDS
constexpr int SAMPLE_EXP = 64;                            // entries of the table of powers of two
typedef unsigned long long u64;
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------ keys
// Logits are taken as they come but for NaN (-inf) and -0 (0).  Keys are in their order; a larger logit
// has a larger key, -inf has key LOWEST - 1.
constexpr unsigned LOWEST = 0x00800000u;
__device__ __forceinline__ float clean(float z) { return fmaxf(z + 0.f, -INFINITY); }
__device__ __forceinline__ unsigned key_of(float z) {
  const unsigned b = __float_as_uint(z);
  return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// Bins of a distance d >= 0 between keys, 2^BITS to an octave from 2^16 on (the bits behind the leading
// one); nearer ones share bin 0.  BINS of them in all.
template <int BITS>
struct Bins {
  static constexpr int BINS = 16 << BITS;
  static __device__ __forceinline__ int of(unsigned d) {
    d = max(d, 0x10000u);
    const int z = __clz((int)d);
    return (int)(d << z >> (31 - BITS)) + ((15 - z) << BITS) - (1 << BITS);
  }
  // The smallest and the largest distance of a bin.
  static __device__ __forceinline__ unsigned first(int bin) {
    return bin == 0 ? 0u : ((1u << BITS) + (bin & ((1 << BITS) - 1))) << ((bin >> BITS) + 16 - BITS);
  }
  static __device__ __forceinline__ unsigned last(int bin) { return bin >= BINS - 1 ? 0xffffffffu : first(bin + 1) - 1u; }
};

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

// The row (or nothing), the histogram, and for bf16 the values' weights and counts, in as many copies, by
// lane, as there is room for: equal tokens that meet in one instruction are added one after the other.
template <int ROW_BYTES, int BINS, int SLOTS, int COPIES>
struct SampleLds {
  uint4 tile[ROW_BYTES / 16 + 1];
  u64 hist[BINS];
  u64 table[SLOTS + 1];
  unsigned count[SLOTS * COPIES + 1];
  u64 mixed[2];
  u64 cand[SAMPLE_THREADS];
  double exp2[SAMPLE_EXP];
  u64 part[SAMPLE_WAVES], red[2][SAMPLE_WAVES];
  float redf[SAMPLE_WAVES];
  u64 left;
  unsigned lo, hi;
  int bin, n, at;
};

// Largest of the 16 lanes of a row, in all of them.
template <int N>
__device__ __forceinline__ float rorf(float v) {
  return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + N, 0xf, 0xf, false));
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, rorf<8>(v));
  v = fmaxf(v, rorf<4>(v));
  v = fmaxf(v, rorf<2>(v));
  return fmaxf(v, rorf<1>(v));
}
__device__ __forceinline__ float lane_of(float v, int lane) {
  return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}

// Sum over the threads before this one, and over all.  (turn: which of two sets of sums in LDS; a set is
// free for the call after next, since every call has a barrier.)
template <class L>
__device__ __forceinline__ u64 block_scan(u64 v, L& l, int turn, u64* total) {
  static_assert(SAMPLE_WAVES == 16, "a row of lanes adds the waves up");
  const u64 x = wave_scan(v);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((threadIdx.x & 63) == 63) l.red[turn][wave] = x;
  __syncthreads();
  const u64 upto = row_scan(l.red[turn][threadIdx.x & 15]);
  *total = readlane64(upto, 15);
  return x - v + (wave > 0 ? readlane64(upto, wave - 1) : 0);
}

// 2^(40 + i / 64)
__device__ const double EXP2_TABLE[SAMPLE_EXP] = {
    1099511627776.0, 1111484524408.0237, 1123587797336.3408, 1135822866265.7363,
    1148191166360.5662, 1160694148413.102, 1173333279013.7073, 1186110040722.8672,
    1199025932245.0925, 1212082468604.716, 1225281181323.604, 1238623618600.8022,
    1252111345494.1387, 1265745944103.804, 1279529013757.93, 1293462171200.1902,
    1307547050779.4426, 1321785304641.4373, 1336178602922.612, 1350728633945.9978,
    1365437104419.2583, 1380305739634.8853, 1395336283672.5735, 1410530499603.8008,
    1425890169698.6345, 1441417095634.7908, 1457113098708.9692, 1472980020050.4907,
    1489019720837.26, 1505234082514.08, 1521625007013.345, 1538194416978.134,
    1554944255987.7375, 1571876488785.6365, 1588993101509.9658, 1606296101926.4866,
    1623787519664.0955, 1641469406452.899, 1659343836364.8796, 1677412906057.1829,
    1695678735018.0535, 1714143465815.4507, 1732809264348.3684, 1751678320100.8945,
    1770752846399.0352, 1790035080670.3372, 1809527284706.3352, 1829231744927.8591,
    1849150772653.2297, 1869286704369.3738, 1889641902005.8923, 1910218753212.1138,
    1931019671637.163, 1952047097213.0808, 1973303496441.0256, 1994791362680.5928,
    2016513216442.283, 2038471605683.1575, 2060669106105.7107, 2083108321459.9976,
    2105791883849.0532, 2128722454037.6345, 2151902721764.3281, 2175335406057.0527,
};

// exp((z - top) / T) in units of 2^-40, c = 64 log2(e) / T: 2^(a / 64) for a = (z - top) c is a power of two
// times a table's 2^(i / 64) times 2^(r / 64) with |r| <= 1/2 from a polynomial, off by less than 1e-13 of
// itself.  z and top are not +inf.  Adding 1.5 * 2^52 rounds a to a whole number, which then stands in the sum's low word.
struct Weigh {
  double top, c;
  const double* table;
  // a, with its nearest whole number in the low word of m
  __device__ __forceinline__ double steps(float z, double* m) const {
    const double a = fmax(((double)z - top) * c, -3000.0);  // below 2^-46; -inf ends there too, also where c is 0
    *m = a + 6755399441055744.0;
    return a;
  }
  // How many steps of 1/64 of an octave the weight is below the top's: 0 .. 3000, none fewer for a smaller z.
  __device__ __forceinline__ int below(float z) const {
    double m;
    steps(z, &m);
    return -(int)(unsigned)(u64)__double_as_longlong(m);
  }
  __device__ __forceinline__ u64 operator()(float z) const {
    int j;
    return at(z, &j);
  }
  __device__ __forceinline__ u64 at(float z, int* steps_below) const {
    double m;
    const double a = steps(z, &m), r = a - (m - 6755399441055744.0);
    const int j = (int)(unsigned)(u64)__double_as_longlong(m);
    *steps_below = -j;
    double p = fma(r, 5.732851688640402e-10, 2.1173137155464776e-07);
    p = fma(r, p, 5.86490495505617e-05);
    p = fma(r, p, 0.010830424696249145);
    const double t = table[j & (SAMPLE_EXP - 1)];
    // the power of two goes to the exponent; adding 2^52 rounds to a whole number in the low bits
    const double w = __longlong_as_double(__double_as_longlong(fma(t * r, p, t)) + ((long long)(j >> 6) << 52));
    return (u64)__double_as_longlong(w + 4503599627370496.0) & 0xfffffffffffffULL;
  }
};

// HELD: the row is kept in LDS.
template <typename T, bool HELD>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(SampleArgs a) {
  constexpr int VEC = 16 / sizeof(T);                        // logits of a chunk
  constexpr bool TABLE = sizeof(T) == 2, CLEAN = HELD && !TABLE;  // CLEAN: the row in LDS is clean already
  using B = Bins<HELD || TABLE ? 7 : 8>;
  constexpr int OWN = B::BINS / SAMPLE_THREADS;              // bins of a thread
  constexpr int STEPS = B::BINS > 3000 ? 0 : 1;              // steps of a bin, as a power of two
  constexpr int COPIES = HELD ? 2 : 4;                       // of the counts
  constexpr int NEAR = SAMPLE_SPAN + 1, FAR = 2 * SAMPLE_SPAN + 2, SLOTS = FAR + 1;
  constexpr int OWN_S = (SLOTS + SAMPLE_THREADS - 1) / SAMPLE_THREADS;
  // chunks requested before the one in hand is used (131072 logits, k = 50: fp32 23.3 us with one, 19.5 with two, 20.8 with
  // four; bf16 29.9, 31.7 and, with spilt registers, 34.2)
  constexpr int AHEAD = HELD ? 0 : TABLE ? 1 : 2;
  __shared__ SampleLds<HELD ? SAMPLE_HELD * (int)sizeof(T) : 0, B::BINS, TABLE ? SLOTS : 0, COPIES> l;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, V = a.V;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const T* zr = (const T*)a.logits + (size_t)row * V;
  const float temp = a.temperature ? a.temperature[row] : 1.f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.f;
  const float min_in = a.min_p ? a.min_p[row] : 0.f;
  const float u_in = a.uniforms[row];
  asm volatile("" ::: "memory");  // all settings are requested here, before the row
  const u64 least = min_in > 0.f ? (u64)ceil((double)fminf(min_in, 1.f) * 1099511627776.0) : 0;
  const double power = EXP2_TABLE[tid & (SAMPLE_EXP - 1)];

  // ---- the row.  The waves' runs of `rounds` x 64 chunks follow one another; round u of a lane is the logits
  // from run + (64 u + lane) VEC on.
  const int rounds = (V + SAMPLE_THREADS * VEC - 1) / (SAMPLE_THREADS * VEC), length = rounds * 64 * VEC;
  const int run = wave * length;
  // Where the largest logit is +inf, those that are share the row: they become 0, all others -inf.
  bool infinite = false;
  auto value = [&](float z) {
    return !infinite ? clean(z) : z == INFINITY ? 0.f : -INFINITY;
  };
  auto read = [&](int i, T* c) {  // a chunk; behind the end of the row: -inf
    if (i + VEC <= V) {
      __builtin_memcpy(c, zr + i, 16);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) c[e] = i + e < V ? zr[i + e] : from_f<T>(-INFINITY);
    }
  };
  // f(chunk, index of its first logit) for all of this thread's
  auto chunks = [&](auto f) {
    T c[AHEAD + 1][VEC];
    auto get = [&](int u, T* to) {
      if constexpr (HELD) __builtin_memcpy(to, &l.tile[tid + SAMPLE_THREADS * u], 16);
      else read(run + (64 * u + lane) * VEC, to);  // one past the last is behind the run, and not used
    };
    static_for<0, AHEAD>([&](auto j) { get(j, c[j]); });
#pragma unroll 1
    for (int u = 0; u < rounds; ++u) {
      get(u + AHEAD, c[AHEAD]);
      f(c[0], run + (64 * u + lane) * VEC);
      static_for<0, AHEAD>([&](auto j) { __builtin_memcpy(c[j], c[j + 1], 16); });
    }
  };
  // f(four logits, index of the first)
  auto each = [&](auto f) {
    chunks([&](const T* c, int i) {
      static_for<0, VEC / 4>([&](auto g) {
        constexpr int G = 4 * decltype(g)::value;
        float v[4] = {to_f(c[G]), to_f(c[G + 1]), to_f(c[G + 2]), to_f(c[G + 3])};
        if constexpr (!CLEAN) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = clean(v[e]);
          if (infinite)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = value(v[e]);
        }
        f(v, i + G);
      });
    });
  };
  auto max4 = [](const float* v) { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])); };
  auto add_to = [&](int bin, u64 w) { atomicAdd(&l.hist[bin], w); };
  auto clear_hist = [&]() {
#pragma unroll
    for (int i = 0; i < OWN; ++i) l.hist[tid + SAMPLE_THREADS * i] = 0;
  };
  if constexpr (HELD) {  // every thread keeps and reads its own chunks
    constexpr int MOST = SAMPLE_HELD / SAMPLE_THREADS / VEC;
    T c[MOST][VEC];
    static_for<0, MOST>([&](auto u) {
      if ((int)u < rounds) read(run + (64 * (int)u + lane) * VEC, c[u]);
    });
    static_for<0, MOST>([&](auto u) {
      if (!((int)u < rounds)) return;
      if constexpr (CLEAN)
#pragma unroll
        for (int e = 0; e < VEC; ++e) c[u][e] = clean(c[u][e]);
      __builtin_memcpy(&l.tile[tid + SAMPLE_THREADS * (int)u], c[u], 16);
    });
  }
  if (tid < SAMPLE_EXP) l.exp2[tid] = power;

  // ---- the largest logit
  float mine = -INFINITY;
  chunks([&](const T* c, int) {  // (a maximum drops NaN)
#pragma unroll
    for (int e = 0; e < VEC; ++e) mine = fmaxf(mine, to_f(c[e]));
  });
  mine = clean(mine);
  float top = row_max(mine);
  top = fmaxf(fmaxf(lane_of(top, 0), lane_of(top, 16)), fmaxf(lane_of(top, 32), lane_of(top, 48)));
  if (lane == 0) l.redf[wave] = top;
  if (tid == 0) {
    l.n = 0;
    l.at = 0x7fffffff;
  }
  clear_hist();
  l.cand[tid] = 0;
  __syncthreads();
  top = lane_of(row_max(l.redf[lane & 15]), 0);
  if (top == INFINITY) {
    infinite = true;
    if constexpr (CLEAN)
      for (int u = 0; u < rounds; ++u) {
        float* c = (float*)&l.tile[tid + SAMPLE_THREADS * u];
#pragma unroll
        for (int e = 0; e < VEC; ++e) c[e] = value(c[e]);
      }
    mine = mine == INFINITY ? 0.f : -INFINITY;
    top = 0.f;
  }
  if (top == -INFINITY) {
    if (tid == 0) a.tokens[row] = 0;
    return;
  }
  if (!(temp > 0.f)) {  // the greedy token
    int at = 0x7fffffff;
    if (mine == top)
      each([&](const float* v, int i) {
#pragma unroll
        for (int e = 3; e >= 0; --e) at = v[e] == top ? min(at, i + e) : at;
      });
    if (at != 0x7fffffff) atomicMin(&l.at, at);
    __syncthreads();
    if (tid == 0) a.tokens[row] = l.at;
    return;
  }
  const unsigned top_key = key_of(top);
  const Weigh weigh{(double)top, 92.33248261893306 / (double)temp, l.exp2};
  const double u = u_in > 0.f ? (double)u_in : 0.0;
  auto target_of = [&](u64 total) { return min((u64)fmin(u * (double)total, 9.0e18), total - 1); };
  // the weight that the kept prefix of a total has to reach
  auto want_of = [&](u64 total) {
    return max((u64)1, min(total, (u64)ceil((double)fmaxf(top_p, 0.f) * (double)total)));
  };
  // Of this thread's N bins, N tid and so on, with amounts b[] and b's sum `before` them, the one in which the
  // running sum reaches `want`, if it does: l.bin, with what is wanted of it in l.left.
  auto reach = [&](auto n_c, const u64* b, u64 sum, u64 before, u64 want) {
    constexpr int N = decltype(n_c)::value;
    if (before < want && want <= before + sum) {
      int bin = N * tid;
#pragma unroll
      for (int i = 0; i < N - 1; ++i)
        if (want > before + b[i] && bin == N * tid + i) {
          before += b[i];
          ++bin;
        }
      l.bin = bin;
      l.left = want - before;
    }
    __syncthreads();
  };
  auto own_bins = [&](u64* b) {  // of the histogram, and their sum
    u64 sum = 0;
#pragma unroll
    for (int i = 0; i < OWN; ++i) sum += b[i] = l.hist[OWN * tid + i];
    return sum;
  };
  // The same over the histogram; false where all bins together do not reach it.
  auto find_bin = [&](u64 want, int turn) {
    u64 b[OWN], total;
    const u64 sum = own_bins(b), before = block_scan(sum, l, turn, &total);
    if (total < want) return false;  // the same for all threads
    reach(std::integral_constant<int, OWN>{}, b, sum, before, want);
    return true;
  };

  // Puts the n tokens of l.cand (zeros behind them) into their order, zeros behind them: a token's place is the
  // number of larger (key, ~index).
  auto sort_cand = [&](int n, u64* sorted) {
    if (tid < n) {
      const u64 c = l.cand[tid];
      int place = 0;
      for (int j0 = 0; j0 < n; j0 += 8) static_for<0, 8>([&](auto j) { place += l.cand[j0 + j] > c; });
      sorted[place] = c;
    } else {
      sorted[tid] = 0;
    }
  };

  // ---- few of the top: among the tokens that may be
  if (top_k > 0 && top_k <= SAMPLE_THREADS) {
    if (mine > -INFINITY) add_to(B::of(top_key - key_of(mine)), 1);
    __syncthreads();
    float bound = value_of(LOWEST);  // with fewer maxima than k every token
    if (find_bin((u64)top_k, 0)) bound = value_of(top_key - min(B::last(l.bin), top_key - LOWEST));
    if (mine >= bound)
      each([&](const float* v, int i) {
        if (max4(v) >= bound)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v[e] >= bound) {
              const int at = atomicAdd(&l.n, 1);
              if (at < SAMPLE_THREADS) l.cand[at] = ((u64)key_of(v[e]) << 32) | (unsigned)~(i + e);
            }
      });
    __syncthreads();
    const int n = l.n, m = min(n, top_k);
    u64* const sorted = l.hist;                   // [1024]
    u64* const weight = l.hist + SAMPLE_THREADS;  // [1024]
    // The kept tokens' share of the row: c and w of the token at place `tid` of m, the weight before it, and all.
    auto cut_weight = [&](u64 w, u64 before, u64 total) {
      return tid > 0 && ((top_p < 1.f && before >= want_of(total)) || w < least) ? 0 : w;
    };
    // Draws among them, once sorted and weight hold them all.
    auto draw = [&](u64 c, u64 w, u64 total) {
      const u64 target = target_of(total);
      u64 sum = 0;  // of the kept tokens of a lower index
      for (int j0 = 0; j0 < m; j0 += 8)
        static_for<0, 8>([&](auto j) { sum += (unsigned)sorted[j0 + j] > (unsigned)c ? weight[j0 + j] : 0; });
      if (w > 0 && sum <= target && target < sum + w) a.tokens[row] = (int)~(unsigned)c;
    };
    if (n <= 64) {  // one wave does it, without barriers
      if (wave > 0) return;
      sort_cand(n, sorted);
      __builtin_amdgcn_wave_barrier();
      const u64 c = sorted[tid];
      u64 w = tid < m ? weigh(value_of((unsigned)(c >> 32))) : 0;
      const u64 upto = wave_scan(w);
      w = cut_weight(w, upto - w, readlane64(upto, 63));
      weight[tid] = w;
      __builtin_amdgcn_wave_barrier();
      draw(c, w, readlane64(wave_scan(w), 63));
      return;
    }
    if (n <= SAMPLE_THREADS) {
      sort_cand(n, sorted);
      __syncthreads();
      const u64 c = sorted[tid];
      u64 w = tid < m ? weigh(value_of((unsigned)(c >> 32))) : 0, total;
      const u64 before = block_scan(w, l, 1, &total);
      w = cut_weight(w, before, total);
      weight[tid] = w;
      block_scan(w, l, 0, &total);  // (its barrier: the weights are written)
      draw(c, w, total);
      return;
    }
    // more equal tokens than places: the long way
    __syncthreads();
    clear_hist();
    __syncthreads();
  }

  float cut = -INFINITY;
  int last = V;
  u64 ties = 0;
  // ---- the weights of bf16 values.  A window of 15 octaves of magnitudes, down from that of the largest logit or
  // of 16 temperatures, has a slot per value, in descending order: SPAN positive ones, slot NEAR for what is nearer
  // to 0, SPAN negative ones, slot FAR for those of larger magnitude.  So a token's weight is read, not computed, and
  // the cut of top-p is found by counting.  (Slot 0 is for nothing.)
  unsigned base = 128;  // the least magnitude inside, in bf16's bits; 0 is never inside
  const float floor = top - 30.f * temp;  // weights below are 0
  auto slot_of = [&](float v) {
    const int bits = (int)__float_as_uint(v), sign = bits >> 31, at = (bits >> 16 & 0x7fff) - (int)base;
    return (unsigned)at < (unsigned)SAMPLE_SPAN ? NEAR + (at ^ ~sign) - sign : at < 0 ? NEAR : FAR;
  };
  auto value_at = [&](int slot) {
    return __uint_as_float(slot < NEAR ? (base + SAMPLE_SPAN - slot) << 16 : 0x80000000u | (base + slot - NEAR - 1) << 16);
  };
  // The slots of two tokens as they are stored; slots 0 and FAR, and SPAN in `at`, for those outside.
  auto slots_of = [&](u16x2 x, u16x2* at) {
    const u16x2 sign = (u16x2)((i16x2)x >> (i16x2)15);
    *at = __builtin_elementwise_min((x & (u16x2)0x7fff) - (u16x2)(unsigned short)base, (u16x2)(unsigned short)SAMPLE_SPAN);
    return (*at ^ ~sign) - sign + (u16x2)(unsigned short)NEAR;
  };
  // f(weight, value) for those tokens of a chunk that are outside, where that is not 0; most: the largest `at`
  auto outside = [&](const T* c, u16x2 most, auto f) {
    if (max(most[0], most[1]) < SAMPLE_SPAN) return;
    unsigned x[VEC / 2];
    __builtin_memcpy(x, c, 16);
#pragma unroll
    for (int j = 0; j < VEC / 2; ++j) {
      u16x2 at;
      slots_of(__builtin_bit_cast(u16x2, x[j]), &at);
      if (max(at[0], at[1]) < SAMPLE_SPAN) continue;
#pragma unroll 1
      for (int e = 0; e < 2; ++e) {
        const float v = clean(__uint_as_float(e ? x[j] & 0xffff0000u : x[j] << 16));
        const int slot = slot_of(v);
        if ((slot == NEAR || slot == FAR) && v >= floor) f(weigh(v), v);
      }
    }
  };
  // How many tokens of a chunk from index i on are `cut`, at indices past `after`; of bf16 values other than 0.
  auto equal = [&](const T* c, int i, int after) {
    unsigned x[4], n = 0;
    __builtin_memcpy(x, c, 16);
    const unsigned bits = __float_as_uint(cut);
#pragma unroll
    for (int j = 0; j < VEC / 2; ++j) {
      n += (x[j] << 16) == bits && i + 2 * j > after;
      n += (x[j] & 0xffff0000u) == bits && i + 2 * j + 1 > after;
    }
    return n;
  };
  if constexpr (TABLE) {
    const unsigned e = __float_as_uint(fmaxf(fabsf(top), fminf(16.f * temp, 1e38f))) >> 23;
    base = (e > 15 ? e - 14 : 1) << 7;
#pragma unroll
    for (int i = 0; i < OWN_S; ++i) {
      const int slot = tid + SAMPLE_THREADS * i;
      if (slot < SLOTS)
        l.table[slot] = slot == 0 || slot == NEAR || slot == FAR || !(value_at(slot) <= top) ? 0 : weigh(value_at(slot));
    }
    for (int i = tid; i < SLOTS * COPIES; i += SAMPLE_THREADS) l.count[i] = 0;
    if (tid < 2) l.mixed[tid] = 0;
    __syncthreads();
  }
  auto count_of = [&](int slot) {
    unsigned n = 0;
#pragma unroll
    for (int j = 0; j < COPIES; ++j) n += l.count[slot * COPIES + j];
    return n;
  };

  // ---- cuts: kept are the tokens above `cut`, and of those equal to it the ones up to index `last` (or,
  // where `ties` is set, the first `ties` ones: their last index is found further down)
  // Whether the draw can read its weights: the cut has a slot of its own, or there is none.
  auto by_slot = [&]() {
    const int slot = cut > -INFINITY ? slot_of(cut) : FAR - 1;
    return TABLE && !infinite && slot != NEAR && slot != FAR;
  };
  // The amount of a token in a cut: its weight (top-p) or 1 (top-k).  One after the other: the cut of top-k, the
  // cut of top-p, and the draw; one copy of the code for all.
#pragma unroll 1
  for (int stage = 0; stage < 3; ++stage) {
    const bool by_weight = stage > 0, drawing = stage == 2;
    if (stage == 0 ? top_k <= 0 : stage == 1 && !(top_p < 1.f)) continue;
    if (!drawing) {
      // Histograms of the amounts of the tokens with keys lo .. hi.  The first is of all above the old cut: of counts
      // by Bins of the distance from hi, of weights by steps of their logarithm, or of bf16 values one by one.  Then
      // the bin that holds the new cut, in parts of 2^shift keys.
      unsigned lo = cut == -INFINITY ? LOWEST : key_of(cut) + 1, hi = top_key;
      int shift = -1;
      u64 want = 0;  // the new cut is where their running sum, from the top, reaches this
      for (;;) {
        const float from = value_of(lo), upto = value_of(hi);
        const bool steps = !TABLE && shift < 0 && by_weight;  // bins of equal steps of the weight's logarithm
        u64 tied = 0;
        if (shift < 0 && by_weight) {
          if constexpr (TABLE) {
            u64 near = 0, far = 0;
            auto add = [&](u64 w, float v) {
              if (fabsf(v) < value_at(SAMPLE_SPAN)) near += w;
              else far += w;
            };
            if (cut == -INFINITY && !infinite) {
              chunks([&](const T* c, int) {
                u16x2 x[VEC / 2], most = 0, at;
                __builtin_memcpy(x, c, 16);
#pragma unroll
                for (int j = 0; j < VEC / 2; ++j) {
                  const u16x2 to = slots_of(x[j], &at) * (u16x2)(unsigned short)COPIES + (u16x2)(unsigned short)(lane & (COPIES - 1));
                  most = __builtin_elementwise_max(most, at);
                  atomicAdd(&l.count[to[0]], 1u);
                  atomicAdd(&l.count[to[1]], 1u);
                }
                outside(c, most, add);
              });
            } else {
              each([&](const float* v, int) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  if (!(v[e] >= from)) continue;
                  const int slot = slot_of(v[e]);
                  if (slot != NEAR && slot != FAR) atomicAdd(&l.count[slot * COPIES + (lane & (COPIES - 1))], 1u);
                  else if (v[e] >= floor) add(weigh(v[e]), v[e]);
                }
              });
            }
            if (near) atomicAdd(&l.mixed[0], near);
            if (far) atomicAdd(&l.mixed[1], far);
          } else {
            each([&](const float* v, int) {
              u64 w[4];
              int j[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = weigh.at(v[e], &j[e]);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (v[e] >= from && w[e]) add_to(j[e] >> STEPS, w[e]);
            });
          }
          if (cut > -INFINITY)
            each([&](const float* v, int i) {
#pragma unroll
              for (int e = 0; e < 4; ++e) tied += v[e] == cut && i + e <= last;
            });
        } else {
          each([&](const float* v, int) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (v[e] >= from && v[e] <= upto) {
                const u64 w = by_weight ? weigh(v[e]) : 1;
                const unsigned d = hi - key_of(v[e]);
                if (w) add_to(shift < 0 ? B::of(d) : (int)(d >> shift), w);
              }
          });
        }
        auto settle = [&](u64 above) {  // false: the cut stays, fewer of the tokens at it are kept
          u64 n_tied;
          block_scan(tied, l, 1, &n_tied);
          const u64 at_cut = by_weight ? weigh(cut) : 0;  // 0 also where nothing was cut
          want = by_weight ? want_of(above + n_tied * at_cut) : min((u64)top_k, above);
          if (want <= above) return true;
          const u64 r = (want - above + at_cut - 1) / at_cut;
          ties = r < n_tied ? r : 0;
          return false;
        };
        u64 above;
        if (TABLE && shift < 0 && by_weight) {
          __syncthreads();
          u64 b[OWN_S] = {}, all = 0;
#pragma unroll
          for (int i = 0; i < OWN_S; ++i) {
            const int slot = OWN_S * tid + i;
            if (slot > 0 && slot < SLOTS)
              b[i] = slot == NEAR ? l.mixed[0] : slot == FAR ? l.mixed[1] : count_of(slot) * l.table[slot];
            all += b[i];
          }
          const u64 before = block_scan(all, l, 0, &above);
          if (!settle(above)) break;
          reach(std::integral_constant<int, OWN_S>{}, b, all, before, want);
          want = l.left;
          const int slot = l.bin;
          if (slot != NEAR && slot != FAR) {  // one value
            cut = value_at(slot);
            const u64 w = l.table[slot], r = (want + w - 1) / w;
            last = V;
            ties = r < (u64)count_of(slot) ? r : 0;
            break;
          }
          // the keys that share the slot, divided like a bin
          const float edge = __uint_as_float(slot == FAR ? 0x80000000u | (base + SAMPLE_SPAN) << 16 : (base << 16) - 1u);
          hi = min(hi, key_of(edge));
          if (slot == NEAR) lo = max(lo, key_of(-edge));
          shift = 0;
          while ((hi - lo) >> shift >= (unsigned)B::BINS) ++shift;
          continue;
        }
        __syncthreads();
        if (shift < 0) {
          u64 b[OWN];
          const u64 all = own_bins(b), before = block_scan(all, l, 0, &above);
          if (!settle(above)) break;
          reach(std::integral_constant<int, OWN>{}, b, all, before, want);
        } else {
          find_bin(want, 0);
        }
        want = l.left;
        // the values of the bin; of steps: of about it, and then by the steps themselves
        const int bin = l.bin;
        float low, high;
        if (steps) {
          low = (float)((double)top - (double)(((bin + 1) << STEPS) + 1) / weigh.c);
          high = (float)((double)top - (double)((bin << STEPS) - 1) / weigh.c);
          low = fmaxf(low - fabsf(low) * 3e-7f, from);
          high += fabsf(high) * 3e-7f;
        } else {
          const unsigned d0 = shift < 0 ? B::first(bin) : (unsigned)bin << shift;
          const unsigned d1 = shift < 0 ? B::last(bin) : d0 + ((1u << shift) - 1u);
          const unsigned k1 = hi - d0;  // (no token has the key of -0, but 0 compares equal to it)
          low = value_of(hi - min(d1, hi - lo));
          high = value_of(k1 == 0x7fffffffu ? k1 - 1 : k1);
        }
        if (tid == 0) {
          l.n = 0;
          l.lo = 0xffffffffu;
          l.hi = 0;
        }
        l.cand[tid] = 0;
        __syncthreads();  // and every thread has read its bins
        clear_hist();
        // the tokens of the bin: how many, the range of their keys, and themselves if they are few
        unsigned kl = 0xffffffffu, kh = 0;
        each([&](const float* v, int i) {
          bool any = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) any |= v[e] >= low && v[e] <= high;
          if (!any) return;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v[e] >= low && v[e] <= high && (!steps || weigh.below(v[e]) >> STEPS == bin)) {
              const unsigned k = key_of(v[e]);
              kl = min(kl, k);
              kh = max(kh, k);
              const int at = atomicAdd(&l.n, 1);
              if (at < SAMPLE_FEW) l.cand[at] = ((u64)k << 32) | (unsigned)~(i + e);
            }
        });
        if (kh) {
          atomicMin(&l.lo, kl);
          atomicMax(&l.hi, kh);
        }
        __syncthreads();
        lo = l.lo;
        hi = l.hi;
        const int n = l.n;
        if (lo == hi) {  // one value
          cut = value_of(lo);
          const u64 w = by_weight ? weigh(cut) : 1, r = (want + w - 1) / w;
          last = V;
          ties = r < (u64)n ? r : 0;
          break;
        }
        if (n <= SAMPLE_FEW) {
          u64 *const sorted = l.hist + SAMPLE_THREADS, total;
          sort_cand(n, sorted);
          __syncthreads();
          const u64 c = sorted[tid], w = tid >= n ? 0 : by_weight ? weigh(value_of((unsigned)(c >> 32))) : 1;
          const u64 before = block_scan(w, l, 1, &total);
          sorted[tid] = 0;
          if (before < want && want <= before + w) l.left = c;
          __syncthreads();
          cut = value_of((unsigned)(l.left >> 32));
          last = (int)~(unsigned)l.left;
          break;
        }
        shift = 0;
        while ((hi - lo) >> shift >= (unsigned)B::BINS) ++shift;
      }
      if (!ties || (stage == 1 && by_slot())) continue;  // (by slots, the draw finds the last one itself)
    }
    // Along the indices, over the tokens of at least `least_v`: the first index at which the running sum of the
    // kept weights exceeds its target (the draw), or of the tokens at the cut the last that is kept.
    const float least_v = fmaxf(cut, value_of(LOWEST));
    auto amount = [&](const float* v, int i, bool counting, u64* w) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = weigh(v[e]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool at = v[e] == cut, kept = (v[e] > cut || (at && i + e <= last)) && (w[e] >= least || v[e] == top);
        w[e] = counting ? (u64)at : kept ? w[e] : 0;
      }
    };
    // first the wave's run: s, and with `ties` in a draw the number of its tokens at the cut
    u64 s = 0, total, w_cut = 0;
    unsigned n = 0;
    if (!drawing) {
      if (TABLE && !infinite && cut != 0.f)
        chunks([&](const T* c, int) { n += equal(c, 0, -1); });
      else
        each([&](const float* v, int) {
#pragma unroll
          for (int e = 0; e < 4; ++e) n += v[e] == cut;
        });
      s = n;
    } else if (by_slot()) {
      if constexpr (TABLE) {
        const int cut_slot = cut > -INFINITY ? slot_of(cut) : FAR;
        if (ties) w_cut = l.table[cut_slot] < least && cut != top ? 0 : l.table[cut_slot];
        __syncthreads();  // (the table has been read)
        for (int slot = tid; slot < SLOTS; slot += SAMPLE_THREADS)
          if (slot + (ties > 0) > cut_slot || (l.table[slot] < least && value_at(slot) != top)) l.table[slot] = 0;
        __syncthreads();
        chunks([&](const T* c, int i) {
          u16x2 x[VEC / 2], most = 0, at;
          __builtin_memcpy(x, c, 16);
#pragma unroll
          for (int j = 0; j < VEC / 2; ++j) {
            const u16x2 from = slots_of(x[j], &at);
            most = __builtin_elementwise_max(most, at);
            s += l.table[from[0]] + l.table[from[1]];
          }
          if (ties) n += equal(c, i, -1);
          outside(c, most, [&](u64 w, float v) { s += v > cut && (w >= least || v == top) ? w : 0; });
        });
        if (!ties && last < run + length && cut > -INFINITY) {  // those at the cut that are not kept
          chunks([&](const T* c, int i) { n += equal(c, i, last); });
          s -= n * l.table[cut_slot];
        }
      }
    } else if (least == 0 && cut == -INFINITY) {
      each([&](const float* v, int) {
        u64 w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = weigh(v[e]);
        s += (w[0] + w[1]) + (w[2] + w[3]);
      });
    } else if (least == 0) {
      each([&](const float* v, int i) {
        if (!(max4(v) >= least_v)) return;
        u64 w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = weigh(v[e]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s += v[e] > cut || (v[e] == cut && i + e <= last) ? w[e] : 0;
      });
    } else {
      each([&](const float* v, int i) {
        if (!(max4(v) >= least_v)) return;
        u64 w[4];
        amount(v, i, false, w);
        s += (w[0] + w[1]) + (w[2] + w[3]);
      });
    }
    const bool open = drawing && ties > 0;  // the last token at the cut that is kept has to be found
    s = wave_scan(s);
    const u64 at_cut = open ? wave_scan(n) : 0;
    if (lane == 63) {
      l.part[wave] = s;
      l.cand[wave] = at_cut;
    }
    __syncthreads();
    if (tid == 0) l.at = V;  // (every thread has read it)
    u64 run_weight = l.part[lane & 15];
    const u64 run_n = l.cand[lane & 15], before_n = row_scan(run_n) - run_n;
    if (open) run_weight += min(run_n, max(ties, before_n) - before_n) * w_cut;
    const u64 upto = row_scan(run_weight);
    total = readlane64(upto, 15);
    u64 target = drawing ? target_of(total) : ties - 1;
    if (target < total) {
      int w = 0;
      u64 base = 0;
      while (target >= readlane64(upto, w)) base = readlane64(upto, w++);
      target -= base;
      // then all threads share the run: `share` logits each, one behind the other
      const int share = (length + 4 * SAMPLE_THREADS - 1) / (4 * SAMPLE_THREADS) * 4, first = w * length + tid * share;
      bool counting = !drawing;
      auto four = [&](int i, u64* w4) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (HELD) {
            const int c = (i - w * length) / VEC;
            v[e] = to_f(((const T*)&l.tile[w * 64 + (c & 63) + SAMPLE_THREADS * (c >> 6)])[i % VEC + e]);
            if (!CLEAN) v[e] = value(v[e]);
          } else {
            v[e] = i + e < V ? value(to_f(zr[i + e])) : -INFINITY;
          }
        }
        amount(v, i, counting, w4);
        return (w4[0] + w4[1]) + (w4[2] + w4[3]);
      };
      u64 w4[4], goal = target;
      if (open) {  // is the last kept one in this run?
        const u64 n0 = readlane64(before_n, w), n1 = n0 + readlane64(run_n, w);
        last = ties >= n1 ? V : -1;
        if (ties > n0 && ties < n1) {
          counting = true;
          goal = ties - 1 - n0;
        }
      }
#pragma unroll 1
      for (;;) {
        s = 0;
        if (tid * share < length)
          for (int j = 0; j < share; j += 4) s += four(first + j, w4);
        u64 before = block_scan(s, l, counting, &total);
        if (before <= goal && goal < before + s) {
          int j = 0;
          u64 t;
          while (before + (t = four(first + j, w4)) <= goal) {
            before += t;
            j += 4;
          }
          int e = 0;
          for (; e < 3 && before + w4[e] <= goal; ++e) before += w4[e];
          l.at = first + j + e;
        }
        if (!drawing || !counting) break;
        __syncthreads();
        last = l.at;  // then the draw
        counting = false;
        goal = target;
      }
    }
    __syncthreads();
    last = l.at;
    ties = 0;
  }
  if (tid == 0) a.tokens[row] = last;
}

template <typename T>
static hipError_t sample_launch(const SampleArgs& a, int n_rows, hipStream_t s) {
  if (a.V <= SAMPLE_HELD)
    hipLaunchKernelGGL((sample_kernel<T, true>), dim3(n_rows), dim3(SAMPLE_THREADS), 0, s, a);
  else
    hipLaunchKernelGGL((sample_kernel<T, false>), dim3(n_rows), dim3(SAMPLE_THREADS), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_sample(int dtype, const SampleArgs& a, int n_rows, hipStream_t s) {
  return dtype == AF_BF16 ? sample_launch<bf16>(a, n_rows, s) : sample_launch<float>(a, n_rows, s);
}

}  // namespace af
