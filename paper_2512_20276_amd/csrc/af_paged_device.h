// Device code that the kernels over a paged cache share: where a request's rows and keys are, and the
// attention of 16 query columns over a tile of 32 keys that one wave holds in registers.
#pragma once

#include "af_device.h"
#include "af_paged.h"

namespace af {

constexpr int KEY_TILE = 32;
constexpr int NO_WINDOW = 0x7fffffff;

__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
// Divisors are powers of two as a rule (heads of a group, key heads), and then it is a shift.
__device__ __forceinline__ int quotient(int x, Divisor d) { return d.shift >= 0 ? x >> d.shift : x / d.d; }
__device__ __forceinline__ int remainder(int x, Divisor d, int q) { return x - q * d.d; }

// Eight elements whose address is a multiple of 16 bytes.
template <typename T>
struct Chunk8;
template <>
struct Chunk8<bf16> {
  typedef bf16x8 type;
};
template <>
struct Chunk8<float> {
  typedef f32x8 type __attribute__((aligned(16)));
};

struct Request {
  int first, n, len;  // rows [first, first + n), cache length with them
};
// Rows are cut to the packed ones and lengths to 0 and more, so that no table makes a kernel leave its buffers.
__device__ __forceinline__ Request request_at(const PagedCache& c, int b) {
  Request r{b, 1, max(c.lens[b], 0)};
  if (c.starts) {
    r.first = min(max(c.starts[b], 0), c.M);
    r.n = min(max(c.starts[b + 1], r.first), c.M) - r.first;
  }
  return r;
}

// The request that a row belongs to, -1: none.  Called by whole waves with one row.
__device__ __forceinline__ int request_of_row(const PagedCache& c, int row) {
  if (!c.starts) return row < c.n_seq ? row : -1;
  const int lane = threadIdx.x & 63;
  if (row < c.starts[0]) return -1;
  for (int b0 = 0; b0 < c.n_seq; b0 += 64) {
    const int b = b0 + lane;
    const unsigned long long past = __ballot(b < c.n_seq && c.starts[min(b, c.n_seq - 1) + 1] > row);
    if (past) return b0 + __builtin_ctzll(past);
  }
  return -1;
}

// Keys that positions lowest .. highest can see: [0, sink_end) and [lo, end), as tiles of TK keys.
// Tiles 0 .. n_sink - 1 are those of the first keys, the others lie from key tile `first` on; where the two
// would meet there are no separate first ones.
template <int TK>
struct KeyTiles {
  int n_sink, first, n;
  __device__ __forceinline__ int key(int i) const { return (i < n_sink ? i : first + i - n_sink) * TK; }
};
template <int TK>
__device__ __forceinline__ KeyTiles<TK> key_tiles(const PagedAttnArgs& a, int lowest, int highest) {
  const int end = min(highest, a.c.cap - 1) + 1;  // a position of -1 or less sees nothing
  const int lo = min(max(max(lowest, -1) - a.window + 1, 0), max(end, 0));
  KeyTiles<TK> t;
  t.first = lo / TK;
  t.n_sink = (min(a.sinks, lo) + TK - 1) / TK;
  if (t.n_sink >= t.first) t.n_sink = t.first = 0;
  t.n = end <= 0 ? 0 : t.n_sink + (end + TK - 1) / TK - t.first;
  return t;
}
// (The clamp keeps p - window within 32 bits where there is none.)
__device__ __forceinline__ bool sees(const PagedAttnArgs& a, int p, int j) {
  return j <= p && j < a.c.cap && (j > max(p, -1) - a.window || j < a.sinks);
}
// Whether some, or all, of the positions lowest .. highest see a key, or every one of n keys from j0 on.
__device__ __forceinline__ bool some_see(const PagedAttnArgs& a, int lowest, int highest, int j) {
  return j <= highest && j < a.c.cap && (j > max(lowest, -1) - a.window || j < a.sinks);
}
__device__ __forceinline__ bool all_see(const PagedAttnArgs& a, int lowest, int highest, int j0, int n) {
  return j0 + n - 1 <= lowest && j0 + n <= a.c.cap && (j0 > max(highest, -1) - a.window || j0 + n <= a.sinks);
}
// Whether none of them sees one of the n keys.
__device__ __forceinline__ bool none_see(const PagedAttnArgs& a, int lowest, int highest, int j0, int n) {
  return j0 > highest || j0 >= a.c.cap || (j0 + n - 1 <= max(lowest, -1) - a.window && j0 >= a.sinks);
}

// The table's entry for key j0 + lane % N, and the page that it means: -1 where there is none.  Apart, so that an entry
// can be on its way for a while: whatever looks at it waits for all loads before it.
template <int N>
__device__ __forceinline__ int page_entry(const PagedCache& c, int b, int j0) {
  const int at = (j0 + (int)(threadIdx.x & (N - 1))) >> c.page_shift;
  return c.table[(size_t)b * c.max_pages + min(at, c.max_pages - 1)];
}
template <int N>
__device__ __forceinline__ int page_of_entry(const PagedCache& c, int j0, int entry) {
  return j0 + (int)(threadIdx.x & (N - 1)) < c.cap && entry >= 0 && entry < c.n_pages ? entry : -1;
}
template <int N>
__device__ __forceinline__ int page_of(const PagedCache& c, int b, int j0) {
  return page_of_entry<N>(c, j0, page_entry<N>(c, b, j0));
}

// Softmax state and output of 16 columns, one for each lane % 16.  Scores are taken transposed, S^T = K . Q^T, and so is
// the output, O^T = V^T . P^T: of both a lane then holds its own column alone (four lanes share one), the
// probabilities are the product's operand as they are, and maximum, sum and scaling need no exchange but two
// steps over the four lanes.  A lane's output of group j is element i of head dimensions (4 g + i) VJ + j.
template <typename T, int HD>
struct Columns {
  static constexpr int KST = HD / 32, VJ = HD / 16;
  typedef typename Mma<T>::frag frag;
  frag q[KST];
  f32x4 o[VJ];
  float m, l;

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < VJ; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
  }
  // row: the lane's column, null: none
  __device__ __forceinline__ void load_q(const T* row) {
    const int lg = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < KST; ++s) {
      T t[8] = {};
      if (row) load8(row + s * 32 + lg * 8, t);
      __builtin_memcpy(&q[s], t, sizeof(q[s]));
    }
  }
  __device__ __forceinline__ float sum() const {  // of the four lanes' sums
    const float s = l + __shfl_xor(l, 16);
    return s + __shfl_xor(s, 32);
  }
};

__device__ __forceinline__ bool not_finite(bf16 x) { return (__builtin_bit_cast(unsigned short, x) & 0x7f80) == 0x7f80; }
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// Two weights of 0 and more as bf16 heads and bf16 remainders, low half first.  A head is the weight cut to 8 bits, so that no
// remainder is below 0, and the remainder is taken of the weight times 1 + 2^-23, so that it is above 0 where the weight is
// (above 2^-100): a value that is infinite then gives that infinity in both products.  The two hold the weight to 2^-16.
struct SplitPair {
  unsigned head, rest;
};
__device__ __forceinline__ SplitPair split_pair(float a, float b) {
  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  const unsigned ua = __float_as_uint(a), ub = __float_as_uint(b);
  constexpr float UP = 1.f + 0x1p-23f;
  bf16x2 r;
  r[0] = (bf16)__builtin_fmaf(a, UP, -__uint_as_float(ua & 0xffff0000u));
  r[1] = (bf16)__builtin_fmaf(b, UP, -__uint_as_float(ub & 0xffff0000u));
  return SplitPair{__builtin_amdgcn_perm(ub, ua, 0x07060302u), __builtin_bit_cast(unsigned, r)};
}

// One tile of keys j0 .. j0 + 31 of key head hk, whose pages the lanes hold (page_of).  p: the position of all columns.
// A lane loads 16 bytes of a key in each of KST steps, and its VJ values of eight keys: the keys 4 g .. 4 g + 3 of
// either half of the tile, whose probabilities it holds.  Values that are not seen are replaced by zeros, since a
// probability of 0 does not hide an infinity or a NaN.
// With bf16 values a probability is split into a bf16 head and a bf16 remainder (split_pair), two products, so that it keeps
// 16 bits and infinite values stay what they are: the cache's bytes bound these kernels, not the matrix instructions.
template <typename T, int HD>
__device__ __forceinline__ void attend_tile(const PagedAttnArgs& a, int hk, int j0, int page, int p, Columns<T, HD>& c) {
  typedef Columns<T, HD> C;
  typedef typename C::frag frag;
  constexpr int KST = C::KST, VJ = C::VJ, ALIGNED = VJ * sizeof(T) < 16 ? VJ * sizeof(T) : 16;  // pools are aligned to 16 bytes
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int in_page = (1 << a.c.page_shift) - 1;
  const size_t page_rows = (size_t)a.c.n_kv_heads << a.c.page_shift, head_row = (size_t)hk << a.c.page_shift;
  const T* K = (const T*)a.c.k;
  const T* V = (const T*)a.c.v;
  frag kf[2][KST];
  T v[8][VJ];
  int of_page[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int kp = max(__shfl(page, h * 16 + lr), 0);
    const T* krow = K + (kp * page_rows + head_row + ((j0 + h * 16 + lr) & in_page)) * HD + lg * 8;
#pragma unroll
    for (int s = 0; s < KST; ++s) kf[h][s] = *(const typename Chunk8<T>::type*)(krow + s * 32);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    of_page[h] = __shfl(page, h * 16 + lg * 4);
    const T* vrow = V + (max(of_page[h], 0) * page_rows + head_row + ((j0 + h * 16 + lg * 4) & in_page)) * HD + lr * VJ;
#pragma unroll
    for (int i = 0; i < 4; ++i) __builtin_memcpy(v[h * 4 + i], __builtin_assume_aligned(vrow + i * HD, ALIGNED), VJ * sizeof(T));
  }

  float s[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < KST; ++t) acc = Mma<T>::mma(kf[h][t], c.q[t], acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[h * 4 + i] = acc[i] * a.scale_log2;
  }
  const bool whole = all_see(a, p, p, j0, KEY_TILE) && __all(page >= 0);
  if (!whole) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = j0 + (e >> 2) * 16 + lg * 4 + (e & 3);
      const bool seen = of_page[e >> 2] >= 0 && sees(a, p, j);
      if (!seen) s[e] = -INFINITY;
#pragma unroll
      for (int d = 0; d < VJ; ++d)
        if (!seen) v[e][d] = from_f<T>(0.f);
    }
  }

  float top = s[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
  top = fmaxf(top, __shfl_xor(top, 16));
  top = fmaxf(top, __shfl_xor(top, 32));
  const float m = fmaxf(c.m, top);
  const float ref = m == -INFINITY ? 0.f : m;  // no key seen yet: probabilities and factor come out 0
  if (__any(m > c.m)) {
    const float f = __builtin_amdgcn_exp2f(c.m - ref);
    c.l *= f;
#pragma unroll
    for (int j = 0; j < VJ; ++j) c.o[j] *= f;
    c.m = m;
  }
  frag pf, pl;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    s[e] = __builtin_amdgcn_exp2f(s[e] - ref);
    c.l += s[e];
  }
  if constexpr (sizeof(T) == 2) {
    unsigned head[4], rest[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const SplitPair w = split_pair(s[2 * e], s[2 * e + 1]);
      head[e] = w.head, rest[e] = w.rest;
    }
    pf = __builtin_bit_cast(frag, head), pl = __builtin_bit_cast(frag, rest);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) pf[e] = s[e];
  }
#pragma unroll
  for (int j = 0; j < VJ; ++j) {
    frag vf;
#pragma unroll
    for (int e = 0; e < 8; ++e) vf[e] = v[e][j];
    c.o[j] = Mma<T>::mma(vf, pf, c.o[j]);
    if constexpr (sizeof(T) == 2) c.o[j] = Mma<T>::mma(vf, pl, c.o[j]);
  }
}

// The natural logarithm of a column's sum of exponentials from its maximum and sum in powers of two.
__device__ __forceinline__ float lse_of(float m, float l) { return (m + log2f(l)) * 0.6931471805599453f; }

// Sum and exclusive prefix of an integer over the wave's lanes: within rows of 16 lanes, then over the rows.
__device__ __forceinline__ int wave_prefix(int v, int& total) {
  int x = v;
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // from 1, 2, 4 and 8 lanes below
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15's to the row above, of rows 0 and 2
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31's to the upper half
  total = __builtin_amdgcn_readlane(x, 63);
  return x - v;
}

// The same sum of floats, in one order.
template <int CTRL, int ROWS>
__device__ __forceinline__ float plus_dpp(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_total(float x) {
  x = plus_dpp<0x118, 0xf>(plus_dpp<0x114, 0xf>(plus_dpp<0x112, 0xf>(plus_dpp<0x111, 0xf>(x))));
  x = plus_dpp<0x143, 0xc>(plus_dpp<0x142, 0xa>(x));
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 63));
}
// The largest of floats of 0 and more.
template <int CTRL, int ROWS>
__device__ __forceinline__ float max_dpp(float x) {
  return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float x) {
  x = max_dpp<0x118, 0xf>(max_dpp<0x114, 0xf>(max_dpp<0x112, 0xf>(max_dpp<0x111, 0xf>(x))));
  x = max_dpp<0x143, 0xc>(max_dpp<0x142, 0xa>(x));
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 63));
}

// ------------------------------------------------------------------ tiles of rows
// The rows of a request with several, each with the heads that share a key head, are columns: column x is head x % group
// of row x / group, so that a tile of columns spans few positions.
// A workgroup takes a part of the keys of one tile of columns.
template <int TK>
struct RowTile {
  int b;                // the request, -1: nothing to do
  Request r;
  int col0, cols;       // columns [col0, col0 + cols) of the request
  int lowest, highest;  // positions of the first and the last
  KeyTiles<TK> keys;
  int split, splits;    // the part of the tile's keys, of so many
  int from, end;        // its key tiles
  int part0;            // partial results of all tiles before this one's
};
// Where few rows meet many keys the keys are cut into parts of a length that gives about as many workgroups as the GPU
// holds at once (of SPLIT_TILES<T> key tiles at least), about the same for all requests.  Every tile of a request is given
// as many parts as its last one, whose rows see the most keys, takes; tiles that take fewer leave the others idle, and the
// last part takes what is left.  A request's last tile is begun first.
// The requests are read once by the lanes of a wave, again only where they are more than 64.
template <typename T, bool SPLIT>
struct RowTiles {
  static constexpr int TK = ROW_KEYS<T>, COLS = ROW_TILE<T>;
  Request r;
  int n, most;   // tiles of the lane's request, key tiles of its last one
  int per;       // key tiles of a part
  int parts;     // of a tile of the lane's request

  __device__ __forceinline__ void read(const PagedAttnArgs& a, int b0) {
    const int b = b0 + (threadIdx.x & 63);
    n = 0, most = 0;
    r = Request{0, 0, 0};
    if (b < a.c.n_seq) r = request_at(a.c, b);
    if (r.n > 1) {
      n = (r.n * a.group.d + COLS - 1) / COLS;
      if (SPLIT) most = key_tiles<TK>(a, r.len - min(r.n, quotient(COLS - 1, a.group) + 1), r.len - 1).n;
    }
  }
  __device__ __forceinline__ void init(const PagedAttnArgs& a) {
    per = 1 << 30;
    if (a.c.n_seq <= 64) read(a, 0);
    parts = 1;
    if constexpr (!SPLIT) return;
    // What a workgroup would take if all tiles were split; then, of the requests with longer tiles, what it takes if the
    // tiles of the others have a workgroup each, and no less than the longest of those, so that it is these that stay whole
    // and the parts are fewer than twice the places.  A split tile's parts are half a part more than its keys, on average.
    // Single rows beside them find a quarter of the places free: four chunks and 28 single rows take 58 us a call on a card that
    // takes 60 with an eighth, 71 with none, 62.5 with three eighths and 87 with half.
    float share = 0.f, longest = 0.f;  // of the tiles that are not split
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
      float work = 0.f, whole = 0.f;
      bool singles = false;
      for (int b0 = 0; b0 < a.c.n_seq; b0 += 64) {
        if (a.c.n_seq > 64) read(a, b0);
        float w = (float)n * (float)most, x = 0.5f * n;
        if ((float)most <= share) {
          longest = fmaxf(longest, (float)most);
          w = 0.f, x = (float)n;
        }
        work += wave_total(w);
        whole += wave_total(x);
        singles |= __any(r.n == 1);
      }
      const float places = singles ? ROW_GRID * 3 / 4 : ROW_GRID;
      share = work * a.c.n_kv_heads / fmaxf(places - whole * a.c.n_kv_heads, ROW_GRID / 8);
    }
    share = fmaxf(share, wave_max(longest));
    per = scalar(max((int)fminf(share, 1e9f) + 1, SPLIT_TILES<T>));  // (1e9: more than any tile has)
    cut();
  }
  __device__ __forceinline__ void cut() { parts = SPLIT ? max((most + per - 1) / per, 1) : 1; }
  // How many tiles are split.
  __device__ __forceinline__ int split_tiles(const PagedAttnArgs& a) {
    int some = 0;
    for (int b0 = 0; b0 < a.c.n_seq; b0 += 64) {
      if (a.c.n_seq > 64) read(a, b0), cut();
      int all;
      wave_prefix(parts > 1 ? n : 0, all);
      some += all;
    }
    return some;
  }
  // Workgroup `at` of a key head: its tile and part.  JOIN: tile `at` of those that are split, part 0.
  template <bool JOIN>
  __device__ __forceinline__ RowTile<TK> find(const PagedAttnArgs& a, int at) {
    RowTile<TK> t;
    t.b = -1;
    int before = 0, parts_before = 0, each = 1, length = per;
    for (int b0 = 0; b0 < a.c.n_seq; b0 += 64) {
      if (a.c.n_seq > 64) read(a, b0), cut();
      const int weight = JOIN ? (parts > 1 ? n : 0) : n * parts;
      int all, all_parts = 0;
      const int prefix = wave_prefix(weight, all), of_parts = JOIN ? wave_prefix(n * parts, all_parts) : 0;
      const unsigned long long past = __ballot(before + prefix + weight > at);
      if (past) {
        const int l = __builtin_ctzll(past);
        t.b = b0 + l;
        t.r = Request{__builtin_amdgcn_readlane(r.first, l), __builtin_amdgcn_readlane(r.n, l), __builtin_amdgcn_readlane(r.len, l)};
        each = __builtin_amdgcn_readlane(parts, l);
        if (each > 1) length = (__builtin_amdgcn_readlane(most, l) + each - 1) / each;
        const int within = at - before - __builtin_amdgcn_readlane(prefix, l);
        const int tile = JOIN || !SPLIT || each == 1 ? within : within / each;
        t.split = JOIN ? 0 : within - tile * each;
        t.part0 = JOIN ? parts_before + __builtin_amdgcn_readlane(of_parts, l) + within * each : at - t.split;
        t.col0 = (__builtin_amdgcn_readlane(n, l) - 1 - tile) * COLS;
        break;
      }
      before += all;
      parts_before += all_parts;
    }
    if (t.b < 0) return t;
    t.cols = min(COLS, t.r.n * a.group.d - t.col0);
    t.lowest = t.r.len - t.r.n + quotient(t.col0, a.group);
    t.highest = t.r.len - t.r.n + quotient(t.col0 + t.cols - 1, a.group);
    t.keys = key_tiles<TK>(a, t.lowest, t.highest);
    if constexpr (!SPLIT) {
      t.split = 0, t.splits = 1, t.from = 0, t.end = t.keys.n;
      return t;
    }
    t.splits = each == 1 ? 1 : max(min((t.keys.n + length - 1) / length, each), 1);
    t.from = t.split * length;
    t.end = t.split == t.splits - 1 ? t.keys.n : t.from + length;
    if (t.split >= t.splits) t.b = -1;
    // (starts that are not ascending give more parts than the workspace holds; no workgroup has taken those behind it)
    if (JOIN && (t.part0 < 0 || t.part0 > a.row_parts - t.splits)) t.b = -1;
    return t;
  }
};
template <typename T, bool SPLIT>
__device__ __forceinline__ RowTile<ROW_KEYS<T>> row_tile(const PagedAttnArgs& a, int at) {
  RowTiles<T, SPLIT> tiles;
  tiles.init(a);
  // Where all workgroups are on the GPU at once, two a CU, those that come second to a CU are taken in the opposite order: the
  // longest tile then shares its CU with the shortest.  us, without that and with it: two prompts of 1024 rows, 32 heads on 8,
  // 47.2 and 39, one of 2048 on 32 key heads 64 and 62, one of 1024 on 8 in fp32 118 and 100.5.
  if (!SPLIT && a.c.n_seq <= 64) {
    const int half = quotient(ROW_GRID / 2, a.n_kv_heads);
    int n;
    wave_prefix(tiles.n, n);
    if (n * a.c.n_kv_heads <= ROW_GRID && at >= half && at < n) at = half + n - 1 - at;
  }
  return tiles.template find<false>(a, at);
}
// Partial result of one part: cols x HD outputs, then a maximum and a sum for each column.
__device__ __forceinline__ float* row_part(const PagedAttnArgs& a, int cols, int hd, int part, int hk) {
  return a.parts + a.rows_at + ((size_t)part * a.c.n_kv_heads + hk) * paged_part_floats(cols, hd);
}

// ------------------------------------------------------------------ requests with a single row
// The heads that share a key head are the columns of a workgroup (16 at most; more take several), whose
// waves take the tiles of 32 keys in turn and merge in LDS.
//
// Which keys a workgroup takes is found on the device, from the lengths as they are when the kernel runs: the key
// tiles of all requests, one behind the other, are cut into a.shares equal shares (of SHARE_TILES tiles at least), and every
// key head has a workgroup for each.  A share may end within a request and hold several.  A request counts
// PIECE_TILES more than it has, before its first one, for what it costs a workgroup to begin and to end one.  What
// does not hold all of a request's tiles is left as a partial result (output, maximum, sum) for the join, and the
// workgroup of its first tile leaves the join word of which shares hold it.
// Short caches are not split (a.shares 0): a.single_waves of a workgroup's four waves take a request's key head.
//
// The cache's bytes bound it: each key and value is read once, by loads that go straight to the registers of the wave that
// needs them, and no wave waits for another before its own tiles are done.  (LDS would share nothing: the keys of a
// workgroup are its own.)  Two waves a SIMD, with registers for a tile of keys and of values each, keep 128 KB a CU on their
// way; three or four with fewer registers were slower.
//   64 requests x 283 keys x 32 key heads    295 MB, 51.1 us, 5.8 TB/s (a kernel that only reads: 5.9)
//   48 requests of 1 .. 16384 keys, 8 heads  355 MB, 69.9 us, 5.1 TB/s
//   one of 131072 keys, 8 heads              537 MB, 92.8 us, 5.8 TB/s
//   32 windows of 4096 of 32768, 8 heads     540 MB, 97.2 us, 5.6 TB/s
// More than 16 heads to a key head read its keys once for each 16 (from L2, if the workgroups run together).
constexpr int SINGLE_WAVES = 4;
constexpr int SHARE_TILES = 4;
constexpr int PIECE_TILES = 2;

__device__ __forceinline__ int single_tiles(const PagedAttnArgs& a, const Request& r, KeyTiles<KEY_TILE>& t) {
  t = key_tiles<KEY_TILE>(a, r.len - 1, r.len - 1);
  return r.n == 1 ? t.n : 0;
}
// Partial results of a share: of a request that began before it, and of one that ends behind it.
__device__ __forceinline__ float* single_part(const PagedAttnArgs& a, int hd, int share, int head_block, int head_blocks, bool ends_behind) {
  return a.parts + a.parts_at + ((size_t)(share * head_blocks + head_block) * 2 + ends_behind) * paged_part_floats(min(a.group.d, 16), hd);
}

template <int HD>
struct SingleLds {
  static constexpr int ROW = HD + 4;  // padded: columns on different banks
  float o[SINGLE_WAVES][16][ROW], m[SINGLE_WAVES][16], l[SINGLE_WAVES][16];
};

template <typename T, int HD>
__device__ __forceinline__ void attend_single(const PagedAttnArgs& a, int block, SingleLds<HD>& lds) {
  typedef Columns<T, HD> C;
  constexpr int VJ = C::VJ;
  const int tid = threadIdx.x, wave = scalar(tid >> 6), lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int waves = a.shares ? SINGLE_WAVES : a.single_waves, sub = wave / waves;  // of a request; which of the workgroup's
  const int blocks = (a.group.d + 15) / 16, head_blocks = a.c.n_kv_heads * blocks;
  const int item = block * (SINGLE_WAVES / waves) + sub, share = item / head_blocks, hb = item % head_blocks;
  const int hk = hb / blocks, col0 = hb % blocks * 16, cols = min(a.group.d - col0, 16);

  int b = share, at = 0, end = 0x7fffffff, before = 0, per = 0x7fffffff;
  if (a.shares) {
    Request r{0, 0, 0};
    KeyTiles<KEY_TILE> t;
    int n = 0, prefix = 0, all = 0, total = 0;
    const auto read = [&](int b0) {
      n = 0;
      if (b0 + lane < a.c.n_seq) {
        r = request_at(a.c, b0 + lane);
        n = single_tiles(a, r, t);
        if (n) n += PIECE_TILES;
      }
      prefix = wave_prefix(n, all);
    };
    for (int b0 = 0; b0 < a.c.n_seq; b0 += 64) {
      read(b0);
      total += all;
    }
    per = max((total + a.shares - 1) / a.shares, SHARE_TILES);
    at = share * per;
    end = min(at + per, total);
    if (at >= end) return;
    for (int b0 = 0;; b0 += 64) {
      if (a.c.n_seq > 64) read(b0);
      const unsigned long long past = __ballot(before + prefix + n > at);
      if (past) {
        const int l = __builtin_ctzll(past);
        b = b0 + l;
        before += __builtin_amdgcn_readlane(prefix, l);
        break;
      }
      before += all;
    }
  }
  for (;;) {
    const bool there = b < a.c.n_seq;  // (not so: a wave without a request, beside ones with one)
    const Request r = request_at(a.c, there ? b : 0);
    KeyTiles<KEY_TILE> t;
    const int n = there ? single_tiles(a, r, t) : 0;
    const int lead = a.shares && n ? PIECE_TILES : 0;
    const int i0 = max(at - before - lead, 0), i1 = min(end - before - lead, n), p = r.len - 1;
    const bool whole = i0 == 0 && i1 == n;
    C c;
    c.clear();
    if (i0 < i1 || !a.shares) {
      if (i0 < i1) c.load_q(lr < cols ? (const T*)a.q + r.first * a.q_stride + (hk * a.group.d + col0 + lr) * HD : nullptr);
      int i = i0 + wave % waves;
      int entry = i < i1 ? page_entry<KEY_TILE>(a.c, b, t.key(i)) : -1;
      for (; i < i1; i += waves) {
        const int page = page_of_entry<KEY_TILE>(a.c, t.key(i), entry);
        if (i + waves < i1) entry = page_entry<KEY_TILE>(a.c, b, t.key(i + waves));
        attend_tile<T, HD>(a, hk, t.key(i), page, p, c);
      }
      // ---- the waves' results, merged
      const float l = c.sum();
      if (lr < cols) {
        if (lg == 0) {
          lds.m[wave][lr] = c.m;
          lds.l[wave][lr] = l;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < VJ; ++j) lds.o[wave][lr][(lg * 4 + e) * VJ + j] = c.o[j][e];
      }
      __syncthreads();
      for (int x = tid - sub * waves * 64; x < cols * (HD / 4) && there && r.n == 1; x += waves * 64) {
        const int col = x / (HD / 4), d = x % (HD / 4) * 4;
        float m = -INFINITY, sum = 0.f;
        for (int w = sub * waves; w < (sub + 1) * waves; ++w) m = fmaxf(m, lds.m[w][col]);
        const float ref = m == -INFINITY ? 0.f : m;
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int w = sub * waves; w < (sub + 1) * waves; ++w) {
          const float f = __builtin_amdgcn_exp2f(lds.m[w][col] - ref);
          sum += f * lds.l[w][col];
          o += f * *(const f32x4*)&lds.o[w][col][d];
        }
        const int head = hk * a.group.d + col0 + col;
        if (whole) {
          const float inv = sum == 0.f ? 0.f : 1.0f / sum;
          T* dst = (T*)a.o + r.first * a.o_stride + head * HD + d;
#pragma unroll
          for (int e = 0; e < 4; ++e) dst[e] = from_f<T>(o[e] * inv);
          if (a.lse && d == 0) a.lse[(size_t)r.first * a.n_heads + head] = lse_of(m, sum);
        } else {
          float* part = single_part(a, HD, share, hb, head_blocks, i0 == 0);
          *(f32x4*)(part + col * HD + d) = o;
          if (d == 0) {
            float* ml = part + min(a.group.d, 16) * HD + 2 * col;
            ml[0] = m;
            ml[1] = sum;
          }
        }
      }
      if (i0 == 0 && hb == 0 && tid == 0 && a.shares) {  // the join's word: the first share, and how many
        int* word = (int*)a.parts + 2 * b;
        word[0] = share;
        word[1] = (before + lead + n - 1) / per - share + 1;
      }
    }
    before += n + lead;
    at = before;
    if (!a.shares || at >= end) return;
    ++b;
    __syncthreads();
  }
}

}  // namespace af
