// gfx950 kernels of a paged key-value cache: rotation of queries and keys with the write of keys and values
// to their pages, attention of requests with a single row, and the join of what was split over the keys.
#include "af_paged_device.h"

namespace af {

// ------------------------------------------------------------------ append
// One workgroup a row.  Pair (j, j + HD/2) of a head turns by position * theta^(-2j/HD): in turns, and in 64 bits until
// the whole turns are taken off, so that far positions keep their angle (an angle of 10^5 in 32 bits is off by
// 0.004).  The row's HD/2 sines and cosines are computed once, by as many threads, while the row's queries, keys
// and values are on their way, and read by all heads from LDS.  A thread rotates 8 pairs of a head at a time, two chunks
// of 16 bytes (fp32: four) whatever the type.
// It moves bytes: 2264 rows of 32 + 32 + 32 bf16 heads of 128 (111 MB read and written) take 19.0 to 21.7 us, 5.1 to 5.8
// TB/s; 282 such rows 5.3 us, of which 2.6 are the least that any launch here takes.  Loading the first heads ahead of
// the sines made the large case slower (24.0 to 26.5 us a call): the waves in flight hide that already.

template <typename T, int HD>
__global__ __launch_bounds__(256) void rope_append_kernel(AppendArgs a) {
  constexpr int HALF = HD / 2, PT = HALF / 8;  // threads of a head
  typedef typename Chunk8<T>::type V8;
  __shared__ float cs[2][HALF];
  const int row = blockIdx.x, tid = threadIdx.x;
  const int b = request_of_row(a.c, row);
  if (b < 0) return;
  const Request r = request_at(a.c, b);
  const int p = r.len - r.n + (row - r.first);
  if (tid < HALF) {
    int axis = 0;
    while (tid >= a.axis_end[axis]) ++axis;
    const int pos = a.positions ? a.positions[(size_t)row * a.n_axes + axis] : p;
    const double t = pos * a.turns[tid];
    const float f = 2.0f * (float)(t - rint(t));
    cs[0][tid] = cospif(f);
    cs[1][tid] = sinpif(f);
  }
  const PagedCache& c = a.c;
  const int at = p >> c.page_shift;
  int page = -1;
  if (p >= 0 && at < c.max_pages) page = c.table[(size_t)b * c.max_pages + at];
  const bool write = page >= 0 && page < c.n_pages;
  const size_t head_rows = (size_t)1 << c.page_shift;
  const size_t cell = ((size_t)max(page, 0) * c.n_kv_heads << c.page_shift) + (p & ((1 << c.page_shift) - 1));  // of head 0
  __syncthreads();
  const int part = tid % PT, j = part * 8;
  for (int h = tid / PT; h < a.n_heads + c.n_kv_heads; h += 256 / PT) {
    const bool key = h >= a.n_heads;
    const T* src = key ? (const T*)a.k + row * a.k_stride + (h - a.n_heads) * HD : (const T*)a.q + row * a.q_stride + h * HD;
    T* dst = key ? (T*)c.k + (cell + (h - a.n_heads) * head_rows) * HD : (T*)a.q_out + row * a.q_out_stride + h * HD;
    if (key && !write) continue;
    V8 x = *(const V8*)(src + j), y = *(const V8*)(src + HALF + j);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = to_f(x[e]), w = to_f(y[e]), co = cs[0][j + e], si = cs[1][j + e];
      x[e] = from_f<T>(u * co - w * si);
      y[e] = from_f<T>(w * co + u * si);
    }
    *(V8*)(dst + j) = x;
    *(V8*)(dst + HALF + j) = y;
  }
  if (!write) return;
  for (int i = tid; i < c.n_kv_heads * (HD / 8); i += 256) {
    const int h = i / (HD / 8), d = i % (HD / 8) * 8;
    *(V8*)((T*)c.v + (cell + h * head_rows) * HD + d) = *(const V8*)((const T*)a.v + row * a.v_stride + h * HD + d);
  }
}

hipError_t launch_rope_append(int dtype, int head_dim, const AppendArgs& a, hipStream_t s) {
  const dim3 grid(a.c.M), block(256);
  if (dtype == AF_BF16) {
    if (head_dim == 128) hipLaunchKernelGGL((rope_append_kernel<bf16, 128>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rope_append_kernel<bf16, 64>), grid, block, 0, s, a);
  } else {
    if (head_dim == 128) hipLaunchKernelGGL((rope_append_kernel<float, 128>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rope_append_kernel<float, 64>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------ requests with a single row
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void attend_single_kernel(PagedAttnArgs a) {
  __shared__ __attribute__((aligned(16))) SingleLds<HD> lds;
  attend_single<T, HD>(a, blockIdx.x, lds);
}

// ------------------------------------------------------------------ join
// A head of a request with a single row, by a workgroup: groups of threads take parts of their own, with a running
// maximum, and are joined in LDS.  The order of the sums goes by the parts' number alone.
// What it reads comes from L2 or the cache behind it and is little: it is one chain of loads (the request and its word,
// the parts' maxima and outputs, LDS, the store), 4.1 us for 48 requests of 32 heads, 5.1 for the 64 parts of one.
template <typename T, int HD>
__device__ __forceinline__ void join_single(const PagedAttnArgs& a, int b, int head) {
  constexpr int DT = HD / 4, GROUPS = 256 / DT;  // threads of a result, groups of threads
  __shared__ __attribute__((aligned(16))) float sum_o[GROUPS][HD];
  __shared__ float sum_m[GROUPS], sum_l[GROUPS];
  const int tid = threadIdx.x;
  const int2 word = *(const int2*)((const int*)a.parts + 2 * b);  // (means nothing where there are no keys)
  const Request r = request_at(a.c, b);
  KeyTiles<KEY_TILE> t;
  const int tiles = single_tiles(a, r, t);
  if (r.n != 1) return;
  T* dst = (T*)a.o + r.first * a.o_stride + head * HD;
  float* lse = a.lse ? a.lse + (size_t)r.first * a.n_heads + head : nullptr;
  if (tiles == 0) {
    if (tid < HD) dst[tid] = from_f<T>(0.f);
    if (lse && tid == 0) *lse = -INFINITY;
    return;
  }
  const int s0 = word.x, n = word.y;
  if (n == 1) return;
  const int blocks = (a.group.d + 15) / 16, head_blocks = a.c.n_kv_heads * blocks, cols = min(a.group.d, 16);
  const int hk = quotient(head, a.group), in_group = remainder(head, a.group, hk);
  const int hb = hk * blocks + in_group / 16, col = in_group % 16;
  const int g = tid / DT, d = tid % DT * 4;
  float m = -INFINITY, l = 0.f;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i0 = g; i0 < n; i0 += 4 * GROUPS) {  // four parts on their way at once
    float pm[4], pl[4];
    f32x4 po[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * GROUPS;
      const float* part = single_part(a, HD, s0 + min(i, n - 1), hb, head_blocks, i == 0);
      pm[u] = i < n ? part[cols * HD + 2 * col] : -INFINITY;
      pl[u] = part[cols * HD + 2 * col + 1];
      po[u] = *(const f32x4*)(part + col * HD + d);
    }
    const float up = fmaxf(fmaxf(fmaxf(pm[0], pm[1]), fmaxf(pm[2], pm[3])), m), ref = up == -INFINITY ? 0.f : up;
    const float f = exp2f(m - ref);
    l *= f;
    o *= f;
    m = up;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i0 + u * GROUPS >= n) break;
      const float w = exp2f(pm[u] - ref);
      l += w * pl[u];
      o += w * po[u];
    }
  }
  *(f32x4*)&sum_o[g][d] = o;
  if (d == 0) {
    sum_m[g] = m;
    sum_l[g] = l;
  }
  __syncthreads();
  if (tid >= HD) return;
#pragma unroll
  for (int w = 0; w < GROUPS; ++w) m = w ? fmaxf(m, sum_m[w]) : sum_m[0];
  const float ref = m == -INFINITY ? 0.f : m;
  float total = 0.f, out = 0.f;
#pragma unroll
  for (int w = 0; w < GROUPS; ++w) {
    const float f = exp2f(sum_m[w] - ref);
    total += f * sum_l[w];
    out += f * sum_o[w][tid];
  }
  dst[tid] = from_f<T>(total == 0.f ? 0.f : out * (1.0f / total));
  if (lse && tid == 0) *lse = lse_of(m, total);
}

// Tiles of rows that were split: a fixed number of workgroups that go on while there are any, since only the lengths tell how
// many there are.  A thread has HD / 32 outputs of a column, so that a half wave reads a part's column in one access, and
// eight parts are on their way at once.  To find a tile costs more than to join eight columns of it (about 1200 clocks of
// integers), so that a workgroup takes 32 columns of a tile at a time, in four turns, where there are more of them than
// twice the workgroups.  A prompt of 1024 rows, 32 heads on 8, in parts of two and three: 9.0 us, by eights 12.1; four chunks of 256
// rows on 2048 keys 12.4 and 15.3 for 34 MB.
constexpr int JOIN_COLS = 8;
constexpr int JOIN_GRID = 1024;
template <typename T, int HD>
__device__ __forceinline__ void join_rows(const PagedAttnArgs& a, int x, int grid) {
  constexpr int THREADS = 256 / JOIN_COLS, DT = HD / THREADS, COLS = ROW_TILE<T>, AHEAD = 8;
  RowTiles<T, true> tiles;
  tiles.init(a);
  const bool many = (long)tiles.split_tiles(a) * a.c.n_kv_heads * (COLS / JOIN_COLS) > 2 * grid;
  const int columns = many ? 4 * JOIN_COLS : JOIN_COLS, blocks = COLS / columns;  // of an item; items of a tile
  for (;; x += grid) {
    const int item = many ? x / (COLS / JOIN_COLS / 4) : x / (COLS / JOIN_COLS), tile = quotient(item, a.n_kv_heads), hk = remainder(item, a.n_kv_heads, tile);
    const RowTile<ROW_KEYS<T>> t = tiles.template find<true>(a, tile);
    if (t.b < 0) return;
    const int n = t.splits, d = threadIdx.x % THREADS * DT, col0 = (x - item * blocks) * columns;
    if (n == 1) continue;
    for (int col = col0 + threadIdx.x / THREADS; col < min(col0 + columns, t.cols); col += JOIN_COLS) {
      float m = -INFINITY, l = 0.f, o[DT] = {};
      for (int i0 = 0; i0 < n; i0 += AHEAD) {  // so many parts on their way at once
        float pm[AHEAD], pl[AHEAD], po[AHEAD][DT], up = m;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          pm[u] = -INFINITY;
          if (i0 + u >= n) continue;
          const float* part = row_part(a, COLS, HD, t.part0 + i0 + u, hk);
          pm[u] = part[COLS * HD + 2 * col];
          pl[u] = part[COLS * HD + 2 * col + 1];
          __builtin_memcpy(po[u], __builtin_assume_aligned(part + col * HD + d, DT * 4), sizeof(po[u]));
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) up = fmaxf(up, pm[u]);
        const float ref = up == -INFINITY ? 0.f : up, f = __builtin_amdgcn_exp2f(m - ref);
        l *= f;
#pragma unroll
        for (int e = 0; e < DT; ++e) o[e] *= f;
        m = up;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          if (i0 + u >= n) continue;
          const float w = __builtin_amdgcn_exp2f(pm[u] - ref);
          l += w * pl[u];
#pragma unroll
          for (int e = 0; e < DT; ++e) o[e] += w * po[u][e];
        }
      }
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      const int i_row = quotient(t.col0 + col, a.group), row = t.r.first + i_row, head = hk * a.group.d + remainder(t.col0 + col, a.group, i_row);
      T* dst = (T*)a.o + row * a.o_stride + head * HD + d;
#pragma unroll
      for (int e = 0; e < DT; ++e) dst[e] = from_f<T>(o[e] * inv);
      if (a.lse && d == 0) a.lse[(size_t)row * a.n_heads + head] = lse_of(m, l);
    }
  }
}

// The tiles' workgroups first, which take longer: four chunks and 28 single rows 7.1 us, the other way round 9.1.
template <typename T, int HD>
__global__ __launch_bounds__(256) void join_kernel(PagedAttnArgs a, int rows) {
  const int x = blockIdx.x;
  if (x < rows) join_rows<T, HD>(a, x, rows);
  else join_single<T, HD>(a, (x - rows) / a.n_heads, (x - rows) % a.n_heads);
}

// ------------------------------------------------------------------ launch
// Workgroups that the shares are to give: as many as the GPU holds at once (two a CU, 256 CUs), and up to a key head's more where
// those do not divide it (24 key heads: 528).  48 requests of up to 16384
// keys took 70.2 us with 512, more with 1024 and with 2048: the shares are equal, so more of them only add pieces, partial
// results and beginnings.
constexpr int SINGLE_GRID = 512;
// Caches of so many keys at most are not split.  Unsplit against split, us a call: 64 requests of 283 keys, 32 key heads, 54.6
// and 61.9; 8 of them 10.7 and 14.8; 64 of 512 keys, 8 key heads, 23.4 and 26.6, 8 of them 11.0 and 11.2.  At 1024 keys 8
// requests take 18.3 and 14.1, one 14.3 and 9.7; 64 that are all of that length 49.5 and 52.9, but lengths differ.
constexpr int DIRECT_KEYS = 512;
// Rows beside one of each request, at most, of a step whose tiles may be split: so many tiles take half of the GPU's places.
// (Requests with a single row take n_seq rows at most; what is left is in tiles whatever the lengths are.)  Tiles of equal
// lengths gain nothing from a split then.  One that is far longer than the others does, and is not split either: 32 heads on 8,
// 64 rows on 131072 keys take 295 us beside a prompt of 900 rows and 2750 beside one of 1036.
static long split_rows(int row_tile, int n_kv_heads, int group) {
  return ((ROW_GRID / 2 / n_kv_heads + 1L) * row_tile - 1) / group;
}

bool paged_plan(int dtype, int head_dim, int n_kv_heads, int n_heads, int n_seq, bool single, int M, int cap, PagedPlan* p) {
  const int group = n_heads / n_kv_heads;
  const long head_blocks = (long)n_kv_heads * ((group + 15) / 16);
  const long most_tiles = (cap + KEY_TILE - 1) / KEY_TILE + 1;  // of a request's keys
  long floats = 0, single_grid = 0, row_grid = 0, join_singles = 0, join_rows = 0;
  *p = PagedPlan{};
  // One request of a step of several rows is a prompt or a chunk of one; should it have a single row all the same, that
  // is not split, which saves the others the join (4 us): 131072 keys on 8 key heads then take 1.9 ms instead of 0.1.  A second
  // request, without rows, has it split.
  if (cap > DIRECT_KEYS && (single || n_seq > 1 || M == 1)) {
    const long shares = std::min((SINGLE_GRID + head_blocks - 1) / head_blocks, n_seq * (most_tiles + PIECE_TILES) / SHARE_TILES + 1);
    p->shares = (int)shares;
    single_grid = shares * head_blocks;
    join_singles = (long)n_seq * n_heads;
    p->parts_at = ((long)n_seq * 2 + 3) / 4 * 4;
    floats = p->parts_at + shares * head_blocks * 2 * paged_part_floats(std::min(group, 16), head_dim);
  } else {
    // Two or four requests' key heads in a workgroup once these alone fill the GPU twice or four times: a wave then works on
    // alone, and where fewer would leave CUs without loads on their way, four share.  283 keys, 32 key heads: 64 requests on a
    // wave each 54.6 us (four waves: 58.6), 32 on two 26.6 (30.4).  Of 100 keys, 128 on a wave each 47.3 (45.0).
    const long items = n_seq * head_blocks;
    p->single_waves = items >= 4 * SINGLE_GRID ? 1 : items >= 2 * SINGLE_GRID ? 2 : SINGLE_WAVES;
    const int each = SINGLE_WAVES / p->single_waves;
    single_grid = (items + each - 1) / each;
  }
  p->rows_at = floats;
  const int row_tile = dtype == AF_BF16 ? ROW_TILE<bf16> : ROW_TILE<float>;
  const int split_keys = dtype == AF_BF16 ? SPLIT_TILES<bf16> * ROW_KEYS<bf16> : SPLIT_TILES<float> * ROW_KEYS<float>;
  if (!single) {
    const long columns = (long)M * group, tiles = columns / row_tile + std::min(n_seq, M / 2);  // at most so many
    row_grid = tiles * n_kv_heads;
    p->tile_grid = (int)std::min(row_grid, 1L << 24);
    if (cap > split_keys && M - n_seq <= split_rows(row_tile, n_kv_heads, group)) {
      p->row_split = true;
      join_rows = std::min(tiles * n_kv_heads * (row_tile / JOIN_COLS), (long)JOIN_GRID);
      // Tiles in two parts or more have fewer than twice as many as their keys are parts long: 2 ROW_GRID in all (and a little
      // for the sum's rounding).
      const long most_parts = std::min(2L * ROW_GRID + 64, row_grid * (cap / split_keys + 2));
      floats += (most_parts + row_grid) * paged_part_floats(row_tile, head_dim);
      row_grid += most_parts;
    }
  }
  p->floats = floats;
  const long most = 1 << 24;  // of 256 work-items, a launch has fewer than 2^32
  if (single_grid + row_grid >= most || join_singles + join_rows >= most) return false;
  p->single_grid = (int)single_grid, p->row_grid = (int)row_grid;
  p->join_singles = (int)join_singles, p->join_rows = (int)join_rows;
  return true;
}

// The workspace grows with the rows up to where tiles are no longer split, and is smaller from there on; a single row of one
// request is split where several are not.
bool paged_workspace(int dtype, int head_dim, int n_kv_heads, int n_heads, int n_seq, bool single, int M, int cap, long* floats) {
  PagedPlan p;
  if (!paged_plan(dtype, head_dim, n_kv_heads, n_heads, n_seq, single, M, cap, &p)) return false;
  *floats = p.floats;
  if (single) return true;
  const int row_tile = dtype == AF_BF16 ? ROW_TILE<bf16> : ROW_TILE<float>;
  const long split = n_seq + split_rows(row_tile, n_kv_heads, n_heads / n_kv_heads);
  for (const long rows : {1L, split})
    if (rows < M && paged_plan(dtype, head_dim, n_kv_heads, n_heads, n_seq, single, (int)rows, cap, &p)) *floats = std::max(*floats, p.floats);
  return true;
}

template <typename T, int HD>
static hipError_t attention_launch(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (a.c.starts) {
    const hipError_t e = launch_paged_rows(sizeof(T) == 2 ? AF_BF16 : AF_F32, HD, a, p, s);
    if (e != hipSuccess) return e;
  } else {
    hipLaunchKernelGGL((attend_single_kernel<T, HD>), dim3(p.single_grid), dim3(256), 0, s, a);
  }
  if (p.join_singles + p.join_rows > 0)
    hipLaunchKernelGGL((join_kernel<T, HD>), dim3(p.join_singles + p.join_rows), dim3(256), 0, s, a, p.join_rows);
  return hipGetLastError();
}

hipError_t launch_attention_paged(int dtype, int head_dim, const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (dtype == AF_BF16) return head_dim == 128 ? attention_launch<bf16, 128>(a, p, s) : attention_launch<bf16, 64>(a, p, s);
  return head_dim == 128 ? attention_launch<float, 128>(a, p, s) : attention_launch<float, 64>(a, p, s);
}

}  // namespace af
