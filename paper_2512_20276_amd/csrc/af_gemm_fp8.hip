// gfx950 matrix product of e4m3 activations and weights with a scale for each block of 128:
//   y[m, n] = sum_b xs[m, b] ws[n / 128, b] sum_{k in block b} xq[m, k] wq[n, k].
// A block's inner sum starts from zero in the matrix cores; its fp32 result is added to the fp32
// accumulator times the product of the two scales.
//
// The 8-bit matrix instruction (v_mfma_f32_16x16x128_f8f6f4, as its narrower forms) adds the products of
// eight neighbouring k on a grid that ends 2^-13 below the largest of them and only the sums of eight in
// fp32: 1.4e-5 of the result for normal values, where products in bf16 instructions (exact for e4m3
// values) leave 1e-8.  That is 1/100 of bf16's own rounding, so a bf16 result may come from the 8-bit
// instruction; an fp32 result never does: there the operands are widened to bf16, at half the rate.  The
// kernels for few rows widen them for bf16 results as well, so the products of a row of such a result are exact
// in a small batch and not in a large one.
//
// The two scales are multiplied with each other first, once for a row of 16 results (applied one by one they
// would take four more instructions a product, beside its four fma): bits are lost where their product is below
// 2^-126, and one past fp32's range gives infinity, or NaN for a block's sum of 0.
#include <cmath>

#include "af_device.h"
#include "af_fp8.h"

namespace af {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

// One block of 128 k of 16 rows of an operand: lane l holds 32 bytes of row l % 16, in the same order of k
// in both operands (any order serves as long as it is the same): bytes 16 g .. and 64 + 16 g .. of the
// block, g = l / 16, so that the lanes of one 16-byte access cover 64 contiguous bytes of each row.
struct Frag8 {
  uint4 lo, hi;
};

// D[i][j] += sum_k A[i][k] B[j][k] from zero; lane l receives D[4 (l / 16) + e][l % 16], e = 0..3.
template <bool WIDE>
struct Fp8Mma;
template <>
struct Fp8Mma<false> {
  typedef i32x8 frag;
  __device__ __forceinline__ static frag load(const Frag8& f) {
    frag r;
    __builtin_memcpy(&r, &f, 32);
    return r;
  }
  __device__ __forceinline__ static f32x4 mma(frag a, frag b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
  }
};
template <>
struct Fp8Mma<true> {
  struct frag {
    bf16x8 v[4];
  };
  __device__ __forceinline__ static frag load(const Frag8& f) {
    const unsigned u[8] = {f.lo.x, f.lo.y, f.lo.z, f.lo.w, f.hi.x, f.hi.y, f.hi.z, f.hi.w};
    frag r;
    static_for<0, 4>([&](auto c) {
      constexpr int I = decltype(c)::value;
      const bf16x2 t0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)u[2 * I], 1.0f, false);
      const bf16x2 t1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)u[2 * I], 1.0f, true);
      const bf16x2 t2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)u[2 * I + 1], 1.0f, false);
      const bf16x2 t3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)u[2 * I + 1], 1.0f, true);
      r.v[I] = bf16x8{t0[0], t0[1], t1[0], t1[1], t2[0], t2[1], t3[0], t3[1]};
    });
    return r;
  }
  __device__ __forceinline__ static f32x4 mma(const frag& a, const frag& b) {
    f32x4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[0], b.v[0], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[1], b.v[1], d, 0, 0, 0);
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[2], b.v[2], d, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[3], b.v[3], d, 0, 0, 0);
  }
};

// The same pointer in every lane, in scalar registers.
__device__ __forceinline__ const void* uniform(const void* p) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)p);
  const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)((uintptr_t)p >> 32));
  return (const void*)(((uintptr_t)hi << 32) | lo);
}

// n (1..4) consecutive results of one row, rounded once.
__device__ __forceinline__ void store4(float* p, const float* v, int n) {
  if (n >= 4) {
    __builtin_memcpy(p, v, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) p[e] = v[e];
  }
}
__device__ __forceinline__ void store4(bf16* p, const float* v, int n) {
  bf16 t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = from_f<bf16>(v[e]);
  if (n >= 4) {
    __builtin_memcpy(p, t, 8);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) p[e] = t[e];
  }
}

// ------------------------------------------------------------------ few rows: K split over the waves
// One workgroup computes 16 RM rows x 16 CN columns; its NW waves take the blocks of K in turn, so no
// operand is used by two waves and every fragment goes from memory straight to the registers that the
// matrix instruction reads.  The weights are the first operand: a lane holds four consecutive columns of
// one row, whose activation scale is one register.  The waves' sums meet in LDS and are added in wave
// order.
template <int RM, int CN, int NW, typename O>
__global__ __launch_bounds__(64 * NW) void gemm_fp8_stream_kernel(Fp8GemmArgs a) {
  typedef Fp8Mma<true> Mm;  // bound by memory: widened operands cost nothing here
  constexpr int TILE = RM * CN * 256;  // results
  constexpr int TS = TILE / 4 + 4;     // f32x4 of one wave's sums, padded off the bank period
  __shared__ f32x4 part[NW > 1 ? (NW - 1) * TS : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int n_mt = (a.M + 16 * RM - 1) / (16 * RM), n_nt = (a.N + 16 * CN - 1) / (16 * CN);
  const int t = xcd_remap(blockIdx.x, n_mt * n_nt);
  const int m0 = t % n_mt * (16 * RM), n0 = t / n_mt * (16 * CN);
  // past the end: the last row or column again, never stored
  const uint8_t* xp[RM];
  const float* xsp[RM];
  const uint8_t* wp[CN];
  static_for<0, RM>([&](auto i) {
    const size_t m = min(m0 + 16 * (int)i + lr, a.M - 1);
    xp[i] = (const uint8_t*)a.xq + m * a.K + 16 * lg;
    xsp[i] = a.xs + m * a.kb;
  });
  static_for<0, CN>([&](auto j) { wp[j] = (const uint8_t*)a.wq + (size_t)min(n0 + 16 * (int)j + lr, a.N - 1) * a.K + 16 * lg; });
  const float* wsp = a.ws + (size_t)(n0 / FP8_BLOCK) * a.kb;
  f32x4 acc[RM][CN];
  static_for<0, RM>([&](auto i) { static_for<0, CN>([&](auto j) { acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f}; }); });

  auto block = [&](int b, auto load) {
    Frag8 wf[CN], xf[RM];
    float s[RM];
    static_for<0, CN>([&](auto j) { load(wp[j], b, wf[j]); });
    static_for<0, RM>([&](auto i) {
      load(xp[i], b, xf[i]);
      s[i] = xsp[i][b];
    });
    const float sw = wsp[b];
    typename Mm::frag w[CN];
    static_for<0, CN>([&](auto j) { w[j] = Mm::load(wf[j]); });
    static_for<0, RM>([&](auto i) {
      const typename Mm::frag x = Mm::load(xf[i]);
      const float sc = s[i] * sw;
      static_for<0, CN>([&](auto j) {
        const f32x4 d = Mm::mma(w[j], x);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(d[e], sc, acc[i][j][e]);
      });
    });
  };
  const int n_full = a.K / FP8_BLOCK;
  for (int b = wave; b < n_full; b += NW)
    block(b, [](const uint8_t* p, int b, Frag8& f) {
      f.lo = *(const uint4*)(p + (size_t)b * FP8_BLOCK);
      f.hi = *(const uint4*)(p + (size_t)b * FP8_BLOCK + 64);
    });
  if (a.kb > n_full && wave == n_full % NW) {  // the last block, partial: K % 16 == 0, so a chunk is wholly in or out
    const int left = a.K % FP8_BLOCK - 16 * lg;
    block(n_full, [left](const uint8_t* p, int b, Frag8& f) {
      f.lo = left > 0 ? *(const uint4*)(p + (size_t)b * FP8_BLOCK) : zero4();
      f.hi = left > 64 ? *(const uint4*)(p + (size_t)b * FP8_BLOCK + 64) : zero4();
    });
  }
  auto store = [&](int m, int n, const f32x4& v) {
    if (m >= a.M || n >= a.N) return;
    float r[4] = {v[0], v[1], v[2], v[3]};
    store4((O*)a.y + (size_t)m * a.N + n, r, a.N - n);
  };
  if constexpr (NW > 1) {
    // wave w adds up the results i with i % NW == w (in units of 16 x 16); every other wave parks its share
    static_for<0, RM * CN>([&](auto q) {
      constexpr int Q = decltype(q)::value;
      const int owner = Q % NW;
      if (wave != owner) part[(wave - (wave > owner)) * TS + Q * 64 + lane] = acc[Q / CN][Q % CN];
    });
    __syncthreads();
    static_for<0, RM * CN>([&](auto q) {
      constexpr int Q = decltype(q)::value;
      const int owner = Q % NW;
      if (wave != owner) return;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) v += w == owner ? acc[Q / CN][Q % CN] : part[(w - (w > owner)) * TS + Q * 64 + lane];
      store(m0 + 16 * (Q / CN) + lr, n0 + 16 * (Q % CN) + 4 * lg, v);
    });
  } else {
    static_for<0, RM * CN>([&](auto q) {
      constexpr int Q = decltype(q)::value;
      store(m0 + 16 * (Q / CN) + lr, n0 + 16 * (Q % CN) + 4 * lg, acc[Q / CN][Q % CN]);
    });
  }
}

template <int RM, int CN, int NW, typename O>
static void stream_launch(const Fp8GemmArgs& a, hipStream_t s) {
  const unsigned wg = (unsigned)((a.M + 16 * RM - 1) / (16 * RM)) * (unsigned)((a.N + 16 * CN - 1) / (16 * CN));
  hipLaunchKernelGGL((gemm_fp8_stream_kernel<RM, CN, NW, O>), dim3(wg), dim3(64 * NW), 0, s, a);
}

// ------------------------------------------------------------------ many rows: tiles staged in LDS
// A tile of BM = 16 RM WM rows x BN = 16 CN WN columns on WM x WN waves (times KG groups that take the
// blocks of a stage in turn).  A stage is KG blocks of 128 k of the tile's rows and weights, brought to
// LDS by global_load_lds NBUF - 1 stages ahead; a row's 128 bytes are one line of memory, and its
// 16-byte chunk c sits at place c ^ (row % 8), so that neither the 16 rows that an operand read touches
// nor the 8 of a load meet on a bank.
//
// What bounds it: a tile of few rows takes its operands into LDS at about 30 bytes a clock and CU (282 x 4096 x
// 11008 on 96 x 64 tiles: 32.2 us; in an earlier loop of 34.8 its loads alone took 28.0 and its products alone 27.2), so its
// time goes by the bytes of a workgroup, (BM + BN) K.  More stages under way were no faster (three of 40 KB, seven of
// 20 KB), but this loop cannot tell: the rows' scales pass through registers, whose loads the compiler waits for together
// with every load to LDS behind them, in the first and the last stage of a set of scales.  Operands loaded straight to
// registers came at half the rate (55.6 us: an access of 16 rows x 64 bytes takes half lines).  Large tiles are bound by the
// matrix cores and the scaling of their results, four fma a product, and by the last pass of the GPU over them, which is
// seldom full: 2264 x 22016 x 4096 at 2.0 PFLOP/s, the matrix cores busy 56 % of the time, 688 tiles on 256 CUs.
//
// The rows' scales come eight blocks at a time, 16 bytes a load (loaded block by block each was a request
// of its own for 4 bytes: a third of all requests to L2), through registers into LDS, turned to [block][row].
template <int RM, int CN, int WM, int WN, int KG, int NBUF>
struct TileShape {
  static constexpr int BM = 16 * RM * WM, BN = 16 * CN * WN, WAVES = WM * WN * KG, THREADS = 64 * WAVES;
  static constexpr int ROWS = BM + BN;                     // lines of a block, activations first
  static constexpr int LOADS = KG * ROWS / 8;              // 1 KB loads of a stage
  static constexpr int D = (LOADS + WAVES - 1) / WAVES;    // of one wave
  static constexpr int SB = 8, SST = SB / KG;              // blocks and stages of one set of scales
  static constexpr int SQ = (2 * BM + THREADS - 1) / THREADS;  // 16-byte scale loads of a thread
  static constexpr int STAGE = KG * ROWS * 128, SCALES = SB * BM * 4;
  static constexpr int LDS = NBUF * STAGE + 2 * SCALES;
  static constexpr int RED = (KG - 1) * BM * BN * 4;       // the groups' sums, in the same memory
  static_assert(SB % KG == 0 && SST >= 2, "a set of scales is written a stage before it is read");
  static_assert(LDS <= 160 * 1024 && RED <= 160 * 1024, "LDS");
};

// Of the L loads of a wave and stage, how many are requested by the end of product q of N: early where
// only one stage is under way at a time, else evenly.
template <int L, int N, bool EARLY>
constexpr int requested(int q) {
  const int n = q < N ? q + 1 : N;
  return EARLY ? (n * ((L + N - 1) / N) < L ? n * ((L + N - 1) / N) : L) : n * L / N;
}

template <int RM, int CN, int WM, int WN, int KG, int NBUF, bool WIDE, typename O>
__global__ __launch_bounds__(64 * WM * WN * KG, 1) void gemm_fp8_tile_kernel(Fp8GemmArgs a) {
  typedef TileShape<RM, CN, WM, WN, KG, NBUF> S;
  typedef Fp8Mma<WIDE> Mm;
  constexpr int W = S::WAVES;
  static_assert(128 % (16 * CN) == 0, "a wave's columns share their weight scales");
  __shared__ __attribute__((aligned(1024))) char smem[S::LDS > S::RED ? S::LDS : S::RED];
  float* const scales = (float*)(smem + NBUF * S::STAGE);  // [2][SB][BM]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int wm = wave % WM, wn = wave / WM % WN, kg = wave / (WM * WN);
  const int n_mt = (a.M + S::BM - 1) / S::BM, n_nt = (a.N + S::BN - 1) / S::BN;
  const int t = xcd_remap(blockIdx.x, n_mt * n_nt);
  const int m0 = t % n_mt * S::BM, n0 = t / n_mt * S::BN;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem);
  const char* xbase = (const char*)a.xq + (size_t)m0 * a.K;
  const char* wbase = (const char*)a.wq + (size_t)n0 * a.K;
  const int n_full = a.K / FP8_BLOCK, n_st = (n_full + KG - 1) / KG;

  // this wave's loads of a stage: load q brings lines 8 (q % (ROWS / 8)) .. +7 of the stage's block
  // q / (ROWS / 8); lane l fetches the chunk that belongs at place l % 8 of line l / 8.  Lines past the
  // last row or column hold it again.
  unsigned voff[S::D];
  static_for<0, S::D>([&](auto i) {
    const int q = min(wave + W * (int)i, S::LOADS - 1);
    const int line = q % (S::ROWS / 8) * 8 + (lane >> 3);
    const int chunk = (lane & 7) ^ (lane >> 3);
    const int row = line < S::BM ? min(line, a.M - 1 - m0) : min(line - S::BM, a.N - 1 - n0);
    voff[i] = (unsigned)row * (unsigned)a.K + 16 * chunk;
  });
  auto fetch = [&](int st, int buf, auto i) {
    const int q = min(wave + W * (int)i, S::LOADS - 1);
    const int b = min(st * KG + q / (S::ROWS / 8), n_full - 1);
    const char* p = (q % (S::ROWS / 8) * 8 < S::BM ? xbase : wbase) + (size_t)b * FP8_BLOCK;
    dma16(uniform(p), voff[i], lds0 + buf * S::STAGE + q * 1024);
  };
  // 16-byte piece i of this thread of the scales of blocks b0 .. b0 + 7: half of a row's
  f32x4 sreg[S::SQ];
  auto load_scales = [&](int b0) {
    static_for<0, S::SQ>([&](auto i) {
      const int it = tid + S::THREADS * (int)i, r = it % S::BM, b = b0 + 4 * (it / S::BM);
      const float* p = a.xs + (size_t)min(m0 + r, a.M - 1) * a.kb;
      if (b + 4 <= a.kb) {
        __builtin_memcpy(&sreg[i], p + b, 16);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) sreg[i][e] = p[min(b + e, a.kb - 1)];
      }
    });
  };
  auto park_scales = [&](int set) {
    static_for<0, S::SQ>([&](auto i) {
      const int it = tid + S::THREADS * (int)i, r = it % S::BM, b = 4 * (it / S::BM);
      if (it < 2 * S::BM)
#pragma unroll
        for (int e = 0; e < 4; ++e) scales[(set * S::SB + b + e) * S::BM + r] = sreg[i][e];
    });
  };

  f32x4 acc[RM][CN];
  static_for<0, RM>([&](auto i) { static_for<0, CN>([&](auto j) { acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f}; }); });
  // this lane's chunks of a line: at places lg ^ (row % 8) and (4 + lg) ^ (row % 8)
  const int c0 = (lg ^ (lr & 7)) * 16, c1 = ((4 + lg) ^ (lr & 7)) * 16;
  const float* wsp = a.ws + (size_t)min((n0 + wn * 16 * CN) / FP8_BLOCK, (a.N - 1) / FP8_BLOCK) * a.kb;
  // One block of this wave's rows and columns.  The products are issued in one order, row block by row
  // block; each is scaled and added two products later, when it is there, and operands are read ahead, the
  // weights of the first row block one product at a time, so that the first product waits for two reads.
  auto compute = [&](float sw, int buf, const float* sl, auto loads, auto issue) {
    constexpr int L = decltype(loads)::value;
    const char* xl = smem + buf * S::STAGE + (kg * S::ROWS + wm * 16 * RM + lr) * 128;
    const char* wl = smem + buf * S::STAGE + (kg * S::ROWS + S::BM + wn * 16 * CN + lr) * 128;
    auto frag = [&](const char* line) {
      Frag8 f;
      f.lo = *(const uint4*)(line + c0);
      f.hi = *(const uint4*)(line + c1);
      return f;
    };
    Frag8 xr[2], wr[CN];
    typename Mm::frag w[CN], x;
    f32x4 d[3];
    float sc[2], s_old = 0.f;
    xr[0] = frag(xl);
    wr[0] = frag(wl);
    __builtin_amdgcn_sched_barrier(0);
    static_for<1, CN>([&](auto j) { wr[j] = frag(wl + (int)j * 2048); });
    sc[0] = sl[0];
    if constexpr (RM > 1) {
      xr[1] = frag(xl + 2048);
      sc[1] = sl[16];
    }
    __builtin_amdgcn_sched_barrier(0);
    constexpr int LAG = 2;
    static_for<0, RM * CN + LAG>([&](auto q_c) {
      constexpr int Q = decltype(q_c)::value, I = Q / CN, J = Q % CN;
      if constexpr (Q < RM * CN) {
        if constexpr (I == 0) w[J] = Mm::load(wr[J]);
        if constexpr (J == 0) x = Mm::load(xr[I & 1]);
        d[Q % 3] = Mm::mma(w[J], x);
        if constexpr (J == (CN > 2 ? 2 : CN - 1) && I > 0 && I + 1 < RM) {
          xr[(I + 1) & 1] = frag(xl + (I + 1) * 2048);
          sc[(I + 1) & 1] = sl[16 * (I + 1)];
        }
      }
      if constexpr (Q >= LAG) {
        constexpr int P = Q - LAG, PI = P / CN, PJ = P % CN;
        if constexpr (PJ == 0) s_old = sc[PI & 1] * sw;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[PI][PJ][e] = fmaf(d[P % 3][e], s_old, acc[PI][PJ][e]);
      }
      static_for<requested<L, RM * CN, NBUF == 2>(Q - 1), requested<L, RM * CN, NBUF == 2>(Q)>([&](auto i) { issue(i); });
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  if (n_st > 0) {
    // weight scales of this wave's blocks of 64 stages, one a lane; waited for at once, before the wait
    // could count the loads to LDS behind it
    float wsv;
    auto next_ws = [&](int st) {
      wsv = wsp[min((st + lane) * KG + kg, a.kb - 1)];
      asm volatile("" : "+v"(wsv));
    };
    next_ws(0);
    load_scales(0);
    park_scales(0);
    static_for<0, NBUF - 1>([&](auto b) { static_for<0, S::D>([&](auto i) { fetch(min((int)b, n_st - 1), b, i); }); });
    int buf = 0;
    for (int st = 0; st < n_st; ++st) {
      // stage st has landed when at most the stages after it are on their way; past the barrier it has
      // for every wave, and nobody reads the buffer of stage st - 1 any more
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NBUF - 2) * S::D) : "memory");
      // the next set of scales: loaded in a set's first stage, written in its last, to the buffer whose
      // last readers the barrier has just let pass
      const int in_set = st % S::SST, set = st / S::SST & 1;
      if (in_set == S::SST - 1) park_scales(set ^ 1);
      if ((st & 63) == 0 && st > 0) next_ws(st);
      const int ahead = min(st + NBUF - 1, n_st - 1), into = buf == 0 ? NBUF - 1 : buf - 1;
      if (in_set == 0) load_scales((st / S::SST + 1) * S::SB);
      if (KG == 1 || st * KG + kg < n_full)
        compute(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wsv), st & 63)), buf,
                scales + (set * S::SB + in_set * KG + kg) * S::BM + wm * 16 * RM + lr,
                std::integral_constant<int, S::D>{}, [&](auto i) { fetch(ahead, into, i); });
      else  // no block left for this group: its share of the loads all the same
        static_for<0, S::D>([&](auto i) { fetch(ahead, into, i); });
      buf = buf + 1 == NBUF ? 0 : buf + 1;
    }
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  if (a.kb > n_full) {
    // the last block, partial: through registers, zeros behind K (K % 16 == 0: a chunk is in or out)
    for (int q = tid; q < S::ROWS * 8; q += S::THREADS) {
      const int line = q >> 3, chunk = q & 7;
      const int row = line < S::BM ? min(line, a.M - 1 - m0) : min(line - S::BM, a.N - 1 - n0);
      const char* p = (line < S::BM ? xbase : wbase) + (size_t)row * a.K + (size_t)n_full * FP8_BLOCK + 16 * chunk;
      *(uint4*)(smem + line * 128 + ((chunk ^ (line & 7)) * 16)) = n_full * FP8_BLOCK + 16 * chunk < a.K ? *(const uint4*)p : zero4();
    }
    for (int r = tid; r < S::BM; r += S::THREADS) scales[r] = a.xs[(size_t)min(m0 + r, a.M - 1) * a.kb + n_full];
    __syncthreads();
    if (kg == 0) compute(wsp[n_full], 0, scales + wm * 16 * RM + lr, std::integral_constant<int, 0>{}, [](auto) {});
    if constexpr (KG == 1 && CN > 1) __syncthreads();  // the results are turned in the same memory
  }
  if constexpr (KG > 1) {
    // the groups' sums meet in LDS and are added in group order
    __syncthreads();
    f32x4* part = (f32x4*)smem;
    constexpr int GS = S::BM * S::BN / 4;
    const int at = (wn * WM + wm) * (RM * CN * 64) + lane;
    if (kg > 0)
      static_for<0, RM * CN>([&](auto q) {
        part[(kg - 1) * GS + at + (int)q * 64] = acc[decltype(q)::value / CN][decltype(q)::value % CN];
      });
    __syncthreads();
    if (kg > 0) return;
    static_for<0, RM * CN>([&](auto q) {
#pragma unroll
      for (int g = 0; g < KG - 1; ++g)
        acc[decltype(q)::value / CN][decltype(q)::value % CN] += part[g * GS + at + (int)q * 64];
    });
  }
  if constexpr (CN == 1) {
    static_for<0, RM>([&](auto i) {
      const int m = m0 + (wm * RM + (int)i) * 16 + lr;
      static_for<0, CN>([&](auto j) {
        const int n = n0 + (wn * CN + (int)j) * 16 + 4 * lg;
        if (m >= a.M || n >= a.N) return;
        const float r[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        store4((O*)a.y + (size_t)m * a.N + n, r, a.N - n);
      });
    });
  } else {
    // A lane's four results of a row are a quarter or half of a line.  So the results of 16 rows are turned in LDS of
    // the wave's own, and a store takes rows of 16 CN columns: whole lines where CN = 4 (through L2, 2264 x
    // 22016 x 4096 took 205 us so and 219 with four results a store, 208 x 22016 x 128 to fp32 8.4 and 14.2).
    constexpr int PER = 16 / sizeof(O), ROW = 16 * CN, PITCH = ROW + PER;  // of a 16-byte piece, a row, and padded
    constexpr int PIECES = ROW / PER;
    static_assert(S::RED + WM * WN * 16 * PITCH * (int)sizeof(O) <= (int)sizeof(smem), "LDS");
    O* const turn = (O*)(smem + S::RED) + (wn * WM + wm) * (16 * PITCH);  // behind the sums that others still read
    const int n0w = n0 + wn * ROW;
    // Past L2 where the pieces are aligned: no line of the results is read before the next launch, which does not
    // find it in L2 (208 x 22016 x 128 to fp32 7.1 us, through L2 8.4; 282 x 22016 x 4096 1 % faster).
    const bool aligned = a.N % PER == 0 && (uintptr_t)a.y % 16 == 0;
    static_for<0, RM>([&](auto i) {
      static_for<0, CN>([&](auto j) {
        const float r[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        store4(turn + lr * PITCH + 16 * (int)j + 4 * lg, r, 4);
      });
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int p = lane; p < 16 * PIECES; p += 64) {
        const int r = p / PIECES, c = p % PIECES * PER, m = m0 + (wm * RM + (int)i) * 16 + r, n = n0w + c;
        if (m >= a.M || n >= a.N) continue;
        const uint4 v = *(const uint4*)(turn + r * PITCH + c);
        O* const to = (O*)a.y + (size_t)m * a.N + n;
        if (aligned) {
          __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, (u32x4*)to);
        } else if (n + PER <= a.N) {
          __builtin_memcpy(to, &v, 16);
        } else {
          O t[PER];
          __builtin_memcpy(t, &v, 16);
#pragma unroll
          for (int e = 0; e < PER; ++e)
            if (n + e < a.N) to[e] = t[e];
        }
      }
      __builtin_amdgcn_wave_barrier();
    });
  }
}

template <int RM, int CN, int WM, int WN, int KG, int NBUF, bool WIDE, typename O>
static void tile_launch(const Fp8GemmArgs& a, hipStream_t s) {
  typedef TileShape<RM, CN, WM, WN, KG, NBUF> S;
  const unsigned wg = (unsigned)((a.M + S::BM - 1) / S::BM) * (unsigned)((a.N + S::BN - 1) / S::BN);
  hipLaunchKernelGGL((gemm_fp8_tile_kernel<RM, CN, WM, WN, KG, NBUF, WIDE, O>), dim3(wg), dim3(S::THREADS), 0, s, a);
}

// ------------------------------------------------------------------ choice of the kernel
// What a variant takes, in us: a start, then passes of the GPU over the work (a started pass counts
// whole), stages of its K loop in each of them, and the stages and results of the whole work where
// the GPU is busy (in units of a full pass: L2 and HBM then set the pace of a stage).  Coefficients are a
// least-squares fit to 21 row counts (1..2264) of 10 weight shapes (512 x 4096 .. 32000 x 4096, K 512 ..
// 11008), for fp32 results also to 10 of 5 shapes with K 64 .. 256.  The bf16 ones were fitted before results were
// turned in LDS and stored past L2; fitted anew to all of these shapes they choose as well (2.4 % on the mean).  Against
// the fastest kernel for these 263 shapes the one of the least estimate takes 1.4 % longer on the mean for K of 512 and more
// (24 % at the worst: 16 x 12288 x 4096; fp32 results 0.6 and 16 %), and 7 % for K of 256 and less (66 %: 7 x 22016 x 144,
// 5.3 us for 3.2; fp32 2.5 and 28 %).  Measured, us, bf16 results, against the next variants:
//   rows x columns x K       taken                      others
//   7 x 32000 x 4096         16 x 32 streamed 26.4      64 x 64 30.0, 16 x 16 streamed 30.1
//   64 x 4096 x 4096         32 x 32, four groups 10.6  32 x 64 11.6, 64 x 64 13.3
//   282 x 4096 x 11008       96 x 64, two groups 32.2   64 x 64 39.0, 128 x 128 52.1
//   282 x 22016 x 4096       160 x 256 45.8             256 x 256 49.4, 160 x 128 55.7
//   1024 x 4096 x 4096       128 x 128, two groups 24.6 160 x 128 25.6, 128 x 256 29.3
//   2264 x 22016 x 4096      288 x 256 197              256 x 256 222, 128 x 256 226
// The streamed ones (K split over the waves, operands straight to registers) are for up to 32 rows: past
// that they read the activations again for every 16 or 32 columns.
struct Fp8Variant {
  int bm, bn, kg;   // tile, and blocks of K taken at once
  int slots;        // workgroups of it that the GPU runs at a time
  bool streamed;
  float start, pass, stage, busy_stage, busy;
};
static const Fp8Variant BF16_VARIANTS[] = {
    {16, 16, 8, 512, true, 2.03f, 0.00f, 0.54f, 1.09f, 0.00f},
    {16, 32, 8, 512, true, 0.00f, 2.03f, 1.01f, 1.42f, 0.00f},
    {32, 16, 8, 512, true, 0.00f, 2.34f, 0.79f, 0.72f, 0.00f},
    {32, 32, 4, 256, false, 1.32f, 1.82f, 0.53f, 0.23f, 0.44f},
    {64, 64, 2, 256, false, 1.41f, 2.09f, 0.46f, 0.18f, 0.69f},
    {64, 64, 2, 512, false, 2.86f, 0.00f, 0.61f, 0.57f, 3.16f},
    {32, 64, 4, 256, false, 1.65f, 2.41f, 0.73f, 0.40f, 0.32f},
    {96, 64, 2, 256, false, 1.42f, 2.29f, 0.58f, 0.18f, 0.86f},
    {128, 128, 2, 256, false, 2.77f, 1.64f, 0.97f, 0.56f, 3.00f},
    {160, 128, 2, 256, false, 3.37f, 1.74f, 1.04f, 0.57f, 3.08f},
    {128, 256, 1, 256, false, 4.54f, 0.00f, 0.75f, 0.18f, 8.32f},
    {160, 256, 1, 256, false, 4.42f, 0.00f, 0.93f, 0.40f, 9.03f},
    {256, 256, 1, 256, false, 2.23f, 2.95f, 1.28f, 0.29f, 15.29f},
    {288, 256, 1, 256, false, 0.00f, 5.52f, 1.43f, 0.20f, 18.28f},
};
// fp32 results: the operands widened to bf16, so twice the time in the matrix cores and more registers
// (the two largest tiles would not fit them)
static const Fp8Variant F32_VARIANTS[] = {
    {16, 16, 8, 512, true, 1.70f, 0.00f, 0.82f, 0.50f, 0.00f},
    {16, 32, 8, 512, true, 1.49f, 0.00f, 1.34f, 0.70f, 0.00f},
    {32, 16, 8, 512, true, 0.00f, 2.14f, 1.06f, 0.00f, 0.00f},
    {32, 32, 4, 256, false, 1.33f, 1.71f, 0.67f, 0.22f, 0.00f},
    {64, 64, 2, 256, false, 1.09f, 2.22f, 0.72f, 0.12f, 0.25f},
    {64, 64, 2, 512, false, 2.09f, 0.64f, 0.82f, 0.67f, 2.01f},
    {32, 64, 4, 256, false, 1.19f, 2.85f, 0.92f, 0.34f, 0.00f},
    {96, 64, 2, 256, false, 1.02f, 2.53f, 0.89f, 0.16f, 0.38f},
    {128, 128, 2, 256, false, 1.19f, 3.43f, 1.63f, 0.37f, 1.82f},
    {160, 128, 2, 256, false, 1.13f, 3.79f, 2.00f, 0.34f, 2.30f},
    {128, 256, 1, 256, false, 1.02f, 3.30f, 1.51f, 0.26f, 4.18f},
    {160, 256, 1, 256, false, 1.61f, 2.89f, 1.75f, 0.37f, 4.85f},
};

int gemm_fp8_plan(int out_dtype, int M, int N, int K) {
  const Fp8Variant* v = out_dtype == AF_BF16 ? BF16_VARIANTS : F32_VARIANTS;
  const int n = out_dtype == AF_BF16 ? (int)(sizeof(BF16_VARIANTS) / sizeof(*v)) : (int)(sizeof(F32_VARIANTS) / sizeof(*v));
  int best = -1;
  double least = 0;
  for (int i = 0; i < n; ++i) {
    const double wg = (double)((M - 1) / v[i].bm + 1) * ((N - 1) / v[i].bn + 1);
    if (v[i].streamed && (M > 32 || (v[i].bm > 16 && wg > v[i].slots))) continue;
    const double full = wg / v[i].slots, passes = std::ceil(full);
    const double stages = std::ceil((double)fp8_blocks(K) / v[i].kg);
    const double us = v[i].start + passes * (v[i].pass + stages * v[i].stage) + full * (stages * v[i].busy_stage + v[i].busy);
    if (best < 0 || us < least) {
      best = i;
      least = us;
    }
  }
  return best;
}

// Kernel i of the lists above.
template <bool WIDE, typename O>
static hipError_t launch_variant(int i, const Fp8GemmArgs& a, hipStream_t s) {
  switch (i) {
    case 0: stream_launch<1, 1, 8, O>(a, s); break;
    case 1: stream_launch<1, 2, 8, O>(a, s); break;
    case 2: stream_launch<2, 1, 8, O>(a, s); break;
    case 3: tile_launch<2, 1, 1, 2, 4, 3, WIDE, O>(a, s); break;
    case 4: tile_launch<2, 2, 2, 2, 2, 3, WIDE, O>(a, s); break;
    case 5: tile_launch<2, 2, 2, 2, 2, 2, WIDE, O>(a, s); break;
    case 6: tile_launch<2, 4, 1, 1, 4, 2, WIDE, O>(a, s); break;
    case 7: tile_launch<3, 2, 2, 2, 2, 3, WIDE, O>(a, s); break;
    case 8: tile_launch<4, 4, 2, 2, 2, 2, WIDE, O>(a, s); break;
    case 9: tile_launch<5, 4, 2, 2, 2, 2, WIDE, O>(a, s); break;
    case 10: tile_launch<4, 4, 2, 4, 1, 3, WIDE, O>(a, s); break;
    case 11: tile_launch<5, 4, 2, 4, 1, 2, WIDE, O>(a, s); break;
    default:
      if constexpr (WIDE) return hipErrorInvalidValue;
      else if (i == 12) tile_launch<8, 4, 2, 4, 1, 2, WIDE, O>(a, s);
      else if (i == 13) tile_launch<9, 4, 2, 4, 1, 2, WIDE, O>(a, s);
      else return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_gemm_fp8(int out_dtype, const Fp8GemmArgs& a, hipStream_t s) {
  const int i = gemm_fp8_plan(out_dtype, a.M, a.N, a.K);
  return out_dtype == AF_BF16 ? launch_variant<false, bf16>(i, a, s) : launch_variant<true, float>(i, a, s);
}

}  // namespace af
