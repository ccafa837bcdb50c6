// gfx950 kernels of attention over a paged cache for requests with several rows: prompts and chunks of them.
#include "af_paged_device.h"

namespace af {

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;

__device__ __forceinline__ float max_of_halves(float v) {  // of lane % 32 and lane % 32 + 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Tiles of keys of a page pool in LDS, keys and values as they lie in the pages: rows of HD elements, the 16-byte chunk c of
// row r at place c ^ turn(r) of the row.  With that the 16 rows of one access step of a key operand (the same chunk of each)
// and, in bf16, the 8 rows x 64 bytes of a value operand are spread evenly over the banks.  (A value operand in fp32 is
// neighbouring chunks of one row.)
template <typename T, int HD>
struct PageTiles {
  static constexpr int KEYS = ROW_KEYS<T>, ROW = HD * sizeof(T), CHUNKS = ROW / 16;
  static constexpr int BYTES = KEYS * ROW, STAGE = 2 * BYTES;
  static constexpr int STEP = 64 / CHUNKS;                // rows that a wave's load fills
  static constexpr int WAVE = KEYS / 4;                   // rows that a wave fills
  static constexpr int LOADS = WAVE / STEP;               // with so many loads, of keys and of values
  static_assert(8 % STEP == 0 && WAVE % 8 == 0 && PAGED_MIN_PAGE >= 8, "a load's rows lie in one page");
  __device__ __forceinline__ static int turn(int r) {
    if constexpr (sizeof(T) == 4) return r & 15;
    else if constexpr (HD == 128) return (r & 3) << 2 | (r >> 2 & 3);
    else return (r >> 1 & 1) << 2 | (r >> 2 & 3);
  }

  unsigned lds, voff[LOADS];
  int wave;
  __device__ __forceinline__ void init(char* smem, int of_wave) {
    const int lane = threadIdx.x & 63;
    wave = of_wave;
    lds = scalar((unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem);
    // row `step row` + lane / CHUNKS of the tile, its chunk (lane % CHUNKS) ^ turn(row)
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = wave * WAVE + i * STEP + lane / CHUNKS;
      voff[i] = (i * STEP % 8 + lane / CHUNKS) * ROW + (lane % CHUNKS ^ turn(r)) * 16;
    }
  }
  // Sends for the tile of keys j0 .. of key head hk; pages: of key j0 + lane
  __device__ __forceinline__ void load(const PagedAttnArgs& a, int hk, int j0, int pages, int buf) const {
    const int in_page = (1 << a.c.page_shift) - 1;
    // a wave's rows, in groups of 8 that lie in one page each
#pragma unroll
    for (int g = 0; g < WAVE / 8; ++g) {
      const int r = wave * WAVE + g * 8;
      const int page = max(__builtin_amdgcn_readlane(pages, r), 0);
      const size_t at = ((((size_t)page * a.c.n_kv_heads + hk) << a.c.page_shift) + ((j0 + r) & in_page)) * ROW;
      const unsigned dst = lds + buf * STAGE + r * ROW;
#pragma unroll
      for (int i = 0; i < 8 / STEP; ++i) {
        const int n = g * (8 / STEP) + i;
        dma16((const char*)a.c.k + at, voff[n], dst + i * STEP * ROW);
        dma16((const char*)a.c.v + at, voff[n], dst + BYTES + i * STEP * ROW);
      }
    }
  }
};
// This wave's loads are there, and every wave is done with what it read.
__device__ __forceinline__ void loaded() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// bf16.  Four waves of 32 columns each; the tiles of 64 keys go to LDS without passing registers, the next one while
// this one is worked on.  Scores, and outputs, are taken transposed as in Columns: S^T = K . Q^T and O^T = V^T . P^T on
// 32 x 32 tiles, so that a lane holds (half of) one column alone.  The probabilities are the second product's operand
// as they are: a lane has keys 8 i + 4 h + 0..3 (h = lane / 32), and the values' operand is read in that order, by
// LDS reads that transpose 4 x 16 elements.
// Outputs are scaled to a new maximum only when it passes the old one by 2^8 in some column: until then
// probabilities go up to 2^8 instead of 1, with the same relative precision.
// A probability is a bf16 head and a bf16 remainder (split_pair), as in attend_tile and in the ring's attention, so that a row is held
// to the same 2^-16 whether it is alone in its request's step or not.  The remainder's products are half as many matrix
// instructions again: 4096 rows took 156 us with one bf16 number (2^-8) and take 198.  Sums are of the unrounded ones.
//
// Tiles that every column sees whole have a loop of their own without any test of a key; tiles at an edge (the diagonal, a
// window's end, missing pages) mask scores, and clear values, in the tile's own place in LDS.
// What bounds it: a wave's 48 matrix instructions of 32 clocks for a tile, and about 330 vector instructions (32 of them
// exponentials), which the two waves of a SIMD run beside each other's matrix instructions.
//   4096 rows, 32 heads on 8 key heads: 137 GFLOP in 194 to 198 us, 708 to 694 TFLOP/s, 56 to 54 % of a large library product's
//   1274; with the remainders' products 206 GFLOP.  The matrix cores are busy 63 % of the time at the clock that the power limit
//   leaves.
// Tried with no gain (before the remainders): a wave priority for its matrix instructions; a tile's scores one turn ahead of
// its exponentials; half tiles by turns; loads spread between matrix instructions; tiles of 256 columns on eight waves (175 us
// against 163); tiles of 32 keys with three waves a SIMD (the same here, short prompts slower); the longest tiles elsewhere in
// the order.
template <int HD, bool SPLIT>
__device__ __forceinline__ void attend_tiles(const PagedAttnArgs& a, int block, char* smem, int& odd_tile) {
  typedef PageTiles<bf16, HD> L;
  constexpr int TK = L::KEYS, COLS = ROW_TILE<bf16>, KST = HD / 16, OB = HD / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ln = lane & 31, h = lane >> 5;
  const int at = quotient(block, a.n_kv_heads), hk = remainder(block, a.n_kv_heads, at);
  const RowTile<TK> t = row_tile<bf16, SPLIT>(a, at);
  if (t.b < 0) return;

  // ---- the wave's columns (those past the last one repeat it and are not stored)
  const int w0 = wave * 32;
  const int col = t.col0 + min(w0 + ln, t.cols - 1);
  const int i_row = quotient(col, a.group), row = t.r.first + i_row, head = hk * a.group.d + remainder(col, a.group, i_row);
  const int base = t.r.len - t.r.n, p = base + i_row;
  const int lowest = base + quotient(t.col0 + min(w0, t.cols - 1), a.group), highest = base + quotient(t.col0 + min(w0 + 31, t.cols - 1), a.group);
  // a scale below 0 turns the queries' sign, and one of 0 clears them, so that the largest score has the largest product
  const float sign = a.scale_log2 > 0.f ? 1.f : a.scale_log2 < 0.f ? -1.f : 0.f;
  const float sl = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);
  bf16x8 q[KST];
  {
    const bf16* src = (const bf16*)a.q + row * a.q_stride + head * HD + h * 8;
#pragma unroll
    for (int s = 0; s < KST; ++s) {
      q[s] = *(const bf16x8*)(src + s * 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) q[s][e] = (bf16)((float)q[s][e] * sign);
    }
  }

  L tiles;
  tiles.init(smem, wave);
  const int in_page = (1 << a.c.page_shift) - 1;

  // ---- LDS addresses: key ln of a block of 32, chunk 2 s + h; values 4 h + lane % 16 / 4 (and 8 further) of 16, dimensions
  // 16 (lane / 16 % 2) + 4 (lane % 4) of 32
  // (a row is as long as its places, so the chunk's bits are turned in the address itself)
  const int x = lane & 15, vr = 4 * h + (x >> 2), vc = (lane >> 4 & 1) * 2 + (x >> 1 & 1);
  int k_at = ln * L::ROW + (L::turn(ln) ^ h) * 16;
  int v_at[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) v_at[i] = L::BYTES + (vr + 8 * i) * L::ROW + (vc ^ L::turn(vr + 8 * i)) * 16 + (x & 1) * 8;

  if (tid == 0) odd_tile = 0;
  f32x16 o[OB];
#pragma unroll
  for (int c = 0; c < OB; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[c][e] = 0.f;
  float m = -INFINITY, l = 0.f;

  const bool idle = w0 >= t.cols;  // a wave without a column only loads (16 chunks of 4 rows: 64 us instead of 67)
  // ---- the tiles: in LDS by turns, tile i + 1 on its way while tile i is worked on
  const int i0 = t.from, end = t.end;
  // tiles of keys in [full_from, full_end), or before full_sinks, are seen whole by all columns
  const int full_end = min(t.lowest, a.c.cap - 1) + 1, full_from = max(t.highest, -1) - a.window + 1;
  int pages = -1, entry = -1;  // of this tile's keys; of the next one's, as the table has it
  int next = t.keys.key(i0);
  if (i0 < end) {
    pages = page_of<TK>(a.c, t.b, next);
    tiles.load(a, hk, next, pages, 0);
    if (i0 + 1 < end) entry = page_entry<TK>(a.c, t.b, t.keys.key(i0 + 1));
  }
  // Edge: some column does not see the whole tile
  const auto work = [&](auto Edge, int i, int j0, unsigned long long there, int here, int buf) {
    constexpr bool edge = decltype(Edge)::value;
    // ---- tiles that some column does not see whole: values that nobody sees, or that are not finite, become zeros, since a
    // probability of 0 does not hide an infinity or a NaN; the columns that see those that are not finite add them below
    bool odd_values = false;
    if constexpr (edge) {
      char* const Vt = smem + buf * L::STAGE + L::BYTES;
      constexpr int T = 256 / TK, N = L::CHUNKS / T;  // threads of a row, chunks of each
      const int r = tid / T;
      const bool some = (there >> r & 1) && some_see(a, t.lowest, t.highest, j0 + r);
      bool odd = false;
#pragma unroll
      for (int c = 0; c < N; ++c) {
        uint4* at16 = (uint4*)(Vt + r * L::ROW + (tid % T * N + c) * 16);
        const uint4 w = *at16;
        unsigned u[4] = {w.x, w.y, w.z, w.w};
        bool here = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool lo = (u[e] & 0x7f80u) == 0x7f80u, hi = (u[e] & 0x7f800000u) == 0x7f800000u;
          u[e] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
          here |= lo | hi;
        }
        if (!some) *at16 = zero4();
        else if (here) *at16 = make_uint4(u[0], u[1], u[2], u[3]);
        odd |= some & here;
      }
      if (odd) odd_tile = i + 1;
      __syncthreads();
      odd_values = odd_tile == i + 1;
      if (idle || none_see(a, lowest, highest, j0, TK)) return;
    }
    bf16x8 vf[2][OB];
    const auto read_v = [&](int k) {
#pragma unroll
      for (int c = 0; c < OB; ++c) {
        typedef __attribute__((address_space(3))) s16x4 lds4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(smem + (v_at[0] ^ c * 64) + k * 16 * L::ROW));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(smem + (v_at[1] ^ c * 64) + k * 16 * L::ROW));
        __builtin_memcpy(&vf[k & 1][c], &lo, 8);
        __builtin_memcpy((char*)&vf[k & 1][c] + 8, &hi, 8);
      }
    };
    f32x16 s[2];
    unsigned pf[4][4], pl[4][4];  // heads and remainders of the weights, operands of the second product
    {
      // ---- S^T = K . Q^T, four operands ahead
      bf16x8 kf[2][4];
      const auto read = [&](int g) {  // four of the 2 KST operands
#pragma unroll
        for (int c = 0; c < 4; ++c)
          kf[g & 1][c] = *(const bf16x8*)(smem + (k_at ^ (4 * g + c) % KST * 32) + (4 * g + c) / KST * 32 * L::ROW);
      };
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[b][e] = 0.f;
      read(0);
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
      static_for<0, KST / 2>([&](auto G) {
        constexpr int g = decltype(G)::value;
        if constexpr (g + 1 < KST / 2) read(g + 1);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          constexpr int b = 4 * g / KST;
          s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[g & 1][c], q[(4 * g + c) % KST], s[b], 0, 0, 0);
        }
        if constexpr (g + 1 < KST / 2) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          }
        }
      });
      if constexpr (edge) {
        // the lane's keys are 4 h on from constants: seen are those up to `last` that lie behind `left` or before `first`
        if (j0 + TK - 1 > lowest || j0 + TK > a.c.cap) {
          const int last = min(p, a.c.cap - 1) - j0 - 4 * h;
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (b * 32 + 8 * (e >> 2) + (e & 3) > last) s[b][e] = -INFINITY;
        }
        if (j0 <= max(highest, -1) - a.window && j0 + TK > a.sinks) {
          const int left = max(p, -1) - a.window - j0 - 4 * h, first = a.sinks - j0 - 4 * h;
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int k = b * 32 + 8 * (e >> 2) + (e & 3);
              if ((k <= left) & (k >= first)) s[b][e] = -INFINITY;
            }
        }
        if (there != ~0ull) {
          const unsigned long long mine = there >> (4 * h);
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (!(mine >> (b * 32 + 8 * (e >> 2) + (e & 3)) & 1)) s[b][e] = -INFINITY;
        }
      }
      read_v(0);  // in time for the products
      // ---- softmax
      float top = s[0][0];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[b][e]);
      top = max_of_halves(top);
      if (__any((top - m) * sl > 8.f)) {
        const float up = fmaxf(m, top), ref = up == -INFINITY ? 0.f : up;
        const float f = __builtin_amdgcn_exp2f((m - ref) * sl);
        l *= f;
#pragma unroll
        for (int c = 0; c < OB; ++c) o[c] *= f;
        m = up;
      }
      float sum[2] = {0.f, 0.f};
      const float off = m == -INFINITY ? 0.f : m * sl;  // no key seen yet: the probabilities come out 0
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          s[b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e], sl, -off));
          s[b][e + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e + 1], sl, -off));
          sum[0] += s[b][e];
          sum[1] += s[b][e + 1];
          const SplitPair w = split_pair(s[b][e], s[b][e + 1]);
          pf[b * 2 + (e >> 3)][e / 2 & 3] = w.head, pl[b * 2 + (e >> 3)][e / 2 & 3] = w.rest;
        }
      l += sum[0] + sum[1];
    }
    // ---- O^T += V^T . P^T
    static_for<0, 4>([&](auto K) {
      constexpr int k = decltype(K)::value;
      if constexpr (k < 3) read_v(k + 1);
#pragma unroll
      for (int c = 0; c < OB; ++c) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k & 1][c], __builtin_bit_cast(bf16x8, pf[k]), o[c], 0, 0, 0);
#pragma unroll
      for (int c = 0; c < OB; ++c) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k & 1][c], __builtin_bit_cast(bf16x8, pl[k]), o[c], 0, 0, 0);
      if constexpr (k < 3) {
#pragma unroll
        for (int c = 0; c < OB; ++c) {
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
          __builtin_amdgcn_sched_group_barrier(0x8, 2, 1);
        }
      }
    });
    if (edge && odd_values) {  // a weight above 0 times such a value is that value
#pragma unroll 1
      for (int k = 0; k < TK; ++k) {
        const int page = __builtin_amdgcn_readlane(here, k);
        if (page < 0 || !sees(a, p, j0 + k)) continue;
        const bf16* v = (const bf16*)a.c.v + ((((size_t)page * a.c.n_kv_heads + hk) << a.c.page_shift) + ((j0 + k) & in_page)) * HD + 4 * h;
#pragma unroll
        for (int c = 0; c < OB; ++c)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const bf16 w = v[32 * c + 8 * (e >> 2) + (e & 3)];
            if (not_finite(w)) o[c][e] += (float)w;
          }
      }
    }
  };
  // Takes turns: waits for tile i and sends for tile i + 1; whether all columns see tile i whole.
  int i = i0, buf = 0, j0 = 0, here = -1;
  unsigned long long there = 0;
  const auto turn = [&]() {
    j0 = next;
    loaded();  // this tile, and every wave is done with the other one
    there = __ballot(pages >= 0);
    here = pages;
    if (i + 1 < end) {
      next = t.keys.key(i + 1);
      pages = page_of_entry<TK>(a.c, next, entry);
      tiles.load(a, hk, next, pages, buf ^ 1);
      if (i + 2 < end) entry = page_entry<TK>(a.c, t.b, t.keys.key(i + 2));
    }
    return j0 + TK <= full_end && (j0 >= full_from || j0 + TK <= a.sinks) && there == ~0ull;
  };
  const auto done = [&]() {
    k_at ^= L::STAGE, v_at[0] ^= L::STAGE, v_at[1] ^= L::STAGE;
    buf ^= 1;
    ++i;
  };
  while (i < end) {
    bool whole = turn();
    if (whole) {
      do {
        if (!idle) work(std::false_type{}, i, j0, there, here, buf);
        done();
        if (i >= end) break;
        whole = turn();
      } while (whole);
      if (i >= end) break;
    }
    work(std::true_type{}, i, j0, there, here, buf);
    done();
  }

  l += __shfl_xor(l, 32);
  const bool real = w0 + ln < t.cols;
  if (!SPLIT || t.splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    // a lane has four of every eight dimensions, its other half the others: halves are exchanged so that each has eight in a row
    bf16* dst = (bf16*)a.o + row * a.o_stride + head * HD + 8 * h;
#pragma unroll
    for (int c = 0; c < OB; ++c)
#pragma unroll
      for (int b = 0; b < 4; b += 2) {
        uint2 w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (bf16)(o[c][4 * (b + i) + e] * inv);
          __builtin_memcpy(&w[i], &v, 8);
        }
        const auto x0 = __builtin_amdgcn_permlane32_swap(w[0].x, w[1].x, false, false);
        const auto x1 = __builtin_amdgcn_permlane32_swap(w[0].y, w[1].y, false, false);
        if (real) *(uint4*)(dst + 32 * c + 8 * b) = make_uint4(x0[0], x1[0], x0[1], x1[1]);
      }
    if (a.lse && h == 0 && real) a.lse[(size_t)row * a.n_heads + head] = lse_of(m * sl, l);
  } else if (real) {
    float* part = row_part(a, COLS, HD, t.part0 + t.split, hk);
#pragma unroll
    for (int c = 0; c < OB; ++c)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *(f32x4*)(part + (w0 + ln) * HD + 32 * c + 8 * b + 4 * h) = f32x4{o[c][4 * b], o[c][4 * b + 1], o[c][4 * b + 2], o[c][4 * b + 3]};
    if (h == 0) {
      part[COLS * HD + 2 * (w0 + ln)] = m * sl;
      part[COLS * HD + 2 * (w0 + ln) + 1] = l;
    }
  }
}

// fp32.  Four waves of 16 columns each, tiles of 32 keys in LDS by turns as above, products transposed on 16 x 16 tiles as in
// Columns.  A lane has keys 16 e + 4 g + 0..3 (g = lane / 16) of its column, and of a value's dimensions the chunks lane % 16
// and, in heads of 128, 16 on; so its output of group j is element i of dimension 64 (j / 4) + 16 g + 4 i + j % 4.
// The matrix instructions of this type, a sixteenth as fast as bf16's, bound it: 3000 rows, 32 heads on 8 of 128, take 668 us, 110
// TFLOP/s, 72 % of a large library product's 154; 1024 rows, where a CU has two workgroups in all, 102 us, 55 %.  With keys
// and values from memory to each wave's registers, as single rows take them, these were 971 and 145.
template <int HD, bool SPLIT>
__device__ __forceinline__ void attend_rows(const PagedAttnArgs& a, int block, char* smem) {
  typedef Columns<float, HD> C;
  typedef PageTiles<float, HD> L;
  constexpr int VJ = C::VJ, KST = C::KST, TK = L::KEYS, COLS = ROW_TILE<float>;
  static_assert(TK == 32 && COLS == 64, "four waves of 16 columns");
  const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), lr = lane & 15, lg = lane >> 4;
  const int at = quotient(block, a.n_kv_heads), hk = remainder(block, a.n_kv_heads, at);
  const RowTile<TK> t = row_tile<float, SPLIT>(a, at);
  if (t.b < 0) return;
  const int w0 = wave * 16;
  const int col = t.col0 + min(w0 + lr, t.cols - 1);  // columns past the last one repeat it
  const int i_row = quotient(col, a.group), row = t.r.first + i_row, head = hk * a.group.d + remainder(col, a.group, i_row);
  const int base = t.r.len - t.r.n, p = base + i_row;
  const int lowest = base + quotient(t.col0 + min(w0, t.cols - 1), a.group), highest = base + quotient(t.col0 + min(w0 + 15, t.cols - 1), a.group);
  const int in_page = (1 << a.c.page_shift) - 1;
  C c;
  c.clear();
  c.load_q((const float*)a.q + row * a.q_stride + head * HD);
  L tiles;
  tiles.init(smem, wave);

  const auto work = [&](int j0, int page, const char* tile) {
    // ---- S^T = K . Q^T
    f32x4 s2[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int t = 0; t < KST; ++t) {
      f32x4 kf[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) kf[h][i] = *(const f32x4*)(tile + (h * 16 + lr) * L::ROW + ((t * 8 + lg * 2 + i) ^ L::turn(lr)) * 16);
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int h = 0; h < 2; ++h) s2[h] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[h][e / 4][e % 4], c.q[t][e], s2[h], 0, 0, 0);
    }
    f32x4 v[8][VJ / 4];
    int of_page[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = (e >> 2) * 16 + lg * 4 + (e & 3);
#pragma unroll
      for (int d = 0; d < VJ / 4; ++d) v[e][d] = *(const f32x4*)(tile + L::BYTES + r * L::ROW + ((d * 16 + lr) ^ L::turn(r)) * 16);
    }
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = s2[e >> 2][e & 3] * a.scale_log2;
    // ---- masks: values that no column sees are replaced by zeros, since a probability of 0 does not hide an infinity or a NaN;
    // where only some columns see a value that is not finite the products are taken one by one
    bool one_by_one = false;
    if (!(all_see(a, lowest, highest, j0, TK) && __all(page >= 0))) {
#pragma unroll
      for (int h = 0; h < 2; ++h) of_page[h] = __shfl(page, h * 16 + lg * 4);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = j0 + (e >> 2) * 16 + lg * 4 + (e & 3);
        const bool there = of_page[e >> 2] >= 0;
        if (!there || !sees(a, p, j)) s[e] = -INFINITY;
        const bool some = there && some_see(a, lowest, highest, j);
#pragma unroll
        for (int d = 0; d < VJ; ++d) {
          if (!some) v[e][d / 4][d % 4] = 0.f;
          one_by_one |= not_finite(v[e][d / 4][d % 4]);
        }
      }
      one_by_one = __any(one_by_one);
    }
    // ---- softmax
    float top = s[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float m = fmaxf(c.m, top), ref = m == -INFINITY ? 0.f : m;  // no key seen yet: probabilities and factor come out 0
    if (__any(m > c.m)) {
      const float f = __builtin_amdgcn_exp2f(c.m - ref);
      c.l *= f;
#pragma unroll
      for (int j = 0; j < VJ; ++j) c.o[j] *= f;
      c.m = m;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[e] = __builtin_amdgcn_exp2f(s[e] - ref);
      c.l += s[e];
    }
    // ---- O^T += V^T . P^T
    if (!one_by_one) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int j = 0; j < VJ; ++j) c.o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][j / 4][j % 4], s[e], c.o[j], 0, 0, 0);
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll 1
      for (int g = 0; g < 4; ++g) {
        const int r = (e >> 2) * 16 + g * 4 + (e & 3);
        const float w = __shfl(s[e], g * 16 + lr);
        const int kp = __builtin_amdgcn_readlane(page, r);
        if (kp < 0 || !sees(a, p, j0 + r)) continue;
        const float* vrow = (const float*)a.c.v + ((((size_t)kp * a.c.n_kv_heads + hk) << a.c.page_shift) + ((j0 + r) & in_page)) * HD + lg * 16;
#pragma unroll
        for (int j = 0; j < VJ; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) c.o[j][i] += w * vrow[j / 4 * 64 + i * 4 + j % 4];
      }
  };

  int pages = -1, entry = -1;  // of this tile's keys; of the next one's, as the table has it
  int next = t.keys.key(t.from);
  if (t.from < t.end) {
    pages = page_of<TK>(a.c, t.b, next);
    tiles.load(a, hk, next, pages, 0);
    if (t.from + 1 < t.end) entry = page_entry<TK>(a.c, t.b, t.keys.key(t.from + 1));
  }
  for (int i = t.from, buf = 0; i < t.end; ++i, buf ^= 1) {
    const int j0 = next, page = pages;
    loaded();  // this tile, and every wave is done with the other one
    if (i + 1 < t.end) {
      next = t.keys.key(i + 1);
      pages = page_of_entry<TK>(a.c, next, entry);
      tiles.load(a, hk, next, pages, buf ^ 1);
      if (i + 2 < t.end) entry = page_entry<TK>(a.c, t.b, t.keys.key(i + 2));
    }
    if (w0 < t.cols && !none_see(a, lowest, highest, j0, TK)) work(j0, page, smem + buf * L::STAGE);
  }
  const float l = c.sum();
  if (w0 + lr >= t.cols) return;
  if (!SPLIT || t.splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    float* dst = (float*)a.o + row * a.o_stride + head * HD + lg * 16;
#pragma unroll
    for (int d = 0; d < VJ / 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(dst + d * 64 + i * 4) = f32x4{c.o[4 * d][i] * inv, c.o[4 * d + 1][i] * inv, c.o[4 * d + 2][i] * inv, c.o[4 * d + 3][i] * inv};
    if (a.lse && lg == 0) a.lse[(size_t)row * a.n_heads + head] = lse_of(c.m, l);
  } else {
    float* part = row_part(a, COLS, HD, t.part0 + t.split, hk);
#pragma unroll
    for (int d = 0; d < VJ / 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(part + (w0 + lr) * HD + d * 64 + lg * 16 + i * 4) = f32x4{c.o[4 * d][i], c.o[4 * d + 1][i], c.o[4 * d + 2][i], c.o[4 * d + 3][i]};
    if (lg == 0) {
      part[COLS * HD + 2 * (w0 + lr)] = c.m;
      part[COLS * HD + 2 * (w0 + lr) + 1] = l;
    }
  }
}

// Tiles of rows and single rows in one launch, the tiles first: they take the longest, and single rows, which read memory
// alone, fill the places that they leave.  (Alternating in eights, before the weights' remainders, a prompt of 4096 rows without
// any single row took 188 us instead of 159, four chunks with 28 single rows 56 instead of 45: the tiles began out of their
// order.)
// Workgroups of tiles beyond `tiles`, which are there if many keys are split, come last: most have nothing to do.
template <typename T, int HD, bool SPLIT>
__global__ __launch_bounds__(256, 2) void attend_step_kernel(PagedAttnArgs a, int tiles, int singles) {
  const int x = blockIdx.x;
  const bool single = x >= tiles && x < tiles + singles;
  const int block = single ? x - tiles : x < tiles ? x : x - singles;
  __shared__ __attribute__((aligned(1024))) char smem[2 * PageTiles<T, HD>::STAGE];
  static_assert(sizeof(SingleLds<HD>) <= sizeof(smem), "one workgroup's LDS");
  if (single) {
    attend_single<T, HD>(a, block, *(SingleLds<HD>*)smem);
  } else if constexpr (sizeof(T) == 2) {
    __shared__ int odd_tile;  // the last tile, counted from 1, that held values that are not finite
    attend_tiles<HD, SPLIT>(a, block, smem, odd_tile);
  } else {
    attend_rows<HD, SPLIT>(a, block, smem);
  }
}

template <typename T, int HD>
static void step_launch(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  const dim3 grid(p.row_grid + p.single_grid), block(256);
  if (p.row_split) hipLaunchKernelGGL((attend_step_kernel<T, HD, true>), grid, block, 0, s, a, p.tile_grid, p.single_grid);
  else hipLaunchKernelGGL((attend_step_kernel<T, HD, false>), grid, block, 0, s, a, p.tile_grid, p.single_grid);
}

hipError_t launch_paged_rows(int dtype, int head_dim, const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (dtype == AF_BF16) {
    if (head_dim == 128) step_launch<bf16, 128>(a, p, s);
    else step_launch<bf16, 64>(a, p, s);
  } else {
    if (head_dim == 128) step_launch<float, 128>(a, p, s);
    else step_launch<float, 64>(a, p, s);
  }
  return hipGetLastError();
}

}  // namespace af
