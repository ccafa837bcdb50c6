// gfx950 kernels of a paged key-value cache: rotation of queries and keys with the write of keys and values
// to their pages, attention of requests with a single row, and the join of what was split over the keys.
#include "af_paged_device.h"

namespace af {

// ------------------------------------------------------------------ append
// One workgroup a row.  Pair (j, j + HD/2) of a head turns by position * theta^(-2j/HD): in turns, and in 64 bits until
// the whole turns are taken off, so that far positions keep their angle (an angle of 10^5 in 32 bits is off by
// 0.004).  The row's HD/2 sines and cosines are computed once, by as many threads, while the row's queries, keys
// and values are on their way, and read by all heads from LDS.  A thread rotates 8 pairs of a head at a time.
template <typename T, int HD>
__global__ __launch_bounds__(256) void rope_append_kernel(AppendArgs a) {
  constexpr int HALF = HD / 2, PT = HALF / 8;  // threads of a head
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
    T x[8], y[8];
    load8(src + j, x);
    load8(src + HALF + j, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = to_f(x[e]), w = to_f(y[e]), co = cs[0][j + e], si = cs[1][j + e];
      x[e] = from_f<T>(u * co - w * si);
      y[e] = from_f<T>(w * co + u * si);
    }
    store8(dst + j, x);
    store8(dst + HALF + j, y);
  }
  if (!write) return;
  for (int i = tid; i < c.n_kv_heads * (HD / 8); i += 256) {
    const int h = i / (HD / 8), d = i % (HD / 8) * 8;
    T x[8];
    load8((const T*)a.v + row * a.v_stride + h * HD + d, x);
    store8((T*)c.v + (cell + h * head_rows) * HD + d, x);
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
// The heads that share a key head are the columns of a workgroup (16 at most; more take several), whose
// four waves take the tiles of 32 keys in turn and merge in LDS.
//
// Which keys a workgroup takes is found on the device, from the lengths as they are when the kernel runs: the key
// tiles of all requests, one behind the other, are cut into a.shares equal shares (of SHARE_TILES tiles at least), and every
// key head has a workgroup for each.  A share may end within a request and hold several.  What does not hold
// all of a request's tiles is left as a partial result (output, maximum, sum) for the join.
constexpr int SINGLE_WAVES = 4;
constexpr int SHARE_TILES = 4;
constexpr int SINGLE_GRID = 1024;  // workgroups that the shares are to give
constexpr int DIRECT_KEYS = 512;   // caches of so many keys at most are not split

struct Shares {
  int total, per;  // tiles of all requests, of a share
};
__device__ __forceinline__ int single_tiles(const PagedAttnArgs& a, int b, KeyTiles<KEY_TILE>& t) {
  const Request r = request_at(a.c, b);
  t = key_tiles<KEY_TILE>(a, r.len - 1, r.len - 1);
  return r.n == 1 ? t.n : 0;
}
// The first request with tiles past tile `at`, and the tiles before it; also their number in all.  Whole waves.
__device__ __forceinline__ int find_tile(const PagedAttnArgs& a, int at, int& before, int& total) {
  int found = -1, sum = 0;
  for (int b0 = 0; b0 < a.c.n_seq; b0 += 64) {
    const int b = b0 + (threadIdx.x & 63);
    KeyTiles<KEY_TILE> t;
    const int n = b < a.c.n_seq ? single_tiles(a, b, t) : 0;
    int all;
    const int prefix = wave_prefix(n, all);
    const unsigned long long past = __ballot(sum + prefix + n > at);
    if (found < 0 && past) {
      const int l = __builtin_ctzll(past);
      found = b0 + l;
      before = sum + __shfl(prefix, l);
    }
    sum += all;
  }
  total = sum;
  return found;
}
__device__ __forceinline__ int share_size(const PagedAttnArgs& a, int total) {
  return max((total + a.shares - 1) / a.shares, SHARE_TILES);
}
// Partial results of a share: of a request that began before it, and of one that ends behind it.
__device__ __forceinline__ float* single_part(const PagedAttnArgs& a, int hd, int share, int head_block, int head_blocks, bool ends_behind) {
  return a.parts + ((size_t)(share * head_blocks + head_block) * 2 + ends_behind) * paged_part_floats(min(a.group.d, 16), hd);
}

template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void attend_single_kernel(PagedAttnArgs a) {
  typedef Columns<T, HD> C;
  constexpr int VJ = C::VJ, ROW = HD + 4;  // padded: columns on different banks
  __shared__ __attribute__((aligned(16))) float wo[SINGLE_WAVES][16][ROW];
  __shared__ float wm[SINGLE_WAVES][16], wl[SINGLE_WAVES][16];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int blocks = (a.group.d + 15) / 16, head_blocks = a.c.n_kv_heads * blocks;
  const int hb = blockIdx.x % head_blocks, share = blockIdx.x / head_blocks;
  const int hk = hb / blocks, col0 = hb % blocks * 16, cols = min(a.group.d - col0, 16);

  int b = share, at = 0, end = 0x7fffffff, before = 0;
  if (a.shares) {
    int total;
    b = find_tile(a, 0, before, total);
    const int per = share_size(a, total);
    at = share * per;
    end = min(at + per, total);
    if (at >= end) return;
    b = find_tile(a, at, before, total);
  }
  for (;;) {
    b = __builtin_amdgcn_readfirstlane(b);
    KeyTiles<KEY_TILE> t;
    const int n = single_tiles(a, b, t);
    const Request r = request_at(a.c, b);
    if (n == 0 && (a.shares || r.n != 1)) {  // (a row without keys: the join writes it)
      if (!a.shares) return;
      ++b;
      continue;
    }
    const int i0 = at - before, i1 = min(end - before, n), p = r.len - 1;
    C c;
    c.clear();
    c.load_q(lr < cols ? (const T*)a.q + r.first * a.q_stride + (hk * a.group.d + col0 + lr) * HD : nullptr);
    int i = i0 + wave;
    int page = i < i1 ? page_of<KEY_TILE>(a.c, b, t.key(i)) : -1;
    for (; i < i1; i += SINGLE_WAVES) {
      const int now = page;
      if (i + SINGLE_WAVES < i1) page = page_of<KEY_TILE>(a.c, b, t.key(i + SINGLE_WAVES));
      attend_tile<T, HD, false>(a, hk, t.key(i), now, p, p, p, c);
    }
    // ---- the waves' results, merged
    const float l = c.sum();
    if (lr < cols) {
      if (lg == 0) {
        wm[wave][lr] = c.m;
        wl[wave][lr] = l;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < VJ; ++j) wo[wave][lr][(lg * 4 + e) * VJ + j] = c.o[j][e];
    }
    __syncthreads();
    const bool whole = i0 == 0 && i1 == n;
    for (int x = tid; x < cols * (HD / 4); x += 256) {
      const int col = x / (HD / 4), d = x % (HD / 4) * 4;
      float m = wm[0][col], sum = 0.f;
#pragma unroll
      for (int w = 1; w < SINGLE_WAVES; ++w) m = fmaxf(m, wm[w][col]);
      const float ref = m == -INFINITY ? 0.f : m;
      f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < SINGLE_WAVES; ++w) {
        const float f = exp2f(wm[w][col] - ref);
        sum += f * wl[w][col];
        o += f * *(const f32x4*)&wo[w][col][d];
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
          part[min(a.group.d, 16) * HD + 2 * col] = m;
          part[min(a.group.d, 16) * HD + 2 * col + 1] = sum;
        }
      }
    }
    before += n;
    at = before;
    if (!a.shares || at >= end) return;
    ++b;
    __syncthreads();
  }
}

// ------------------------------------------------------------------ join
// A head of a request with a single row, by a workgroup: maximum and sum over the parts by all threads, then the outputs
// by groups of threads, each with parts of its own.  The order of the sums goes by the parts' number alone.
template <typename T, int HD>
__device__ __forceinline__ void join_single(const PagedAttnArgs& a, int b, int head) {
  constexpr int DT = HD / 4, GROUPS = 256 / DT;  // threads of a result, groups of threads
  __shared__ __attribute__((aligned(16))) float sum_o[GROUPS][HD];
  __shared__ float red[2][4];
  const int tid = threadIdx.x, wave = tid >> 6;
  const Request r = request_at(a.c, b);
  KeyTiles<KEY_TILE> t;
  const int tiles = single_tiles(a, b, t);
  if (r.n != 1) return;
  T* dst = (T*)a.o + r.first * a.o_stride + head * HD;
  float* lse = a.lse ? a.lse + (size_t)r.first * a.n_heads + head : nullptr;
  if (tiles == 0) {
    if (tid < HD) dst[tid] = from_f<T>(0.f);
    if (lse && tid == 0) *lse = -INFINITY;
    return;
  }
  int total, before = 0;
  for (int b0 = 0, sum = 0; b0 < a.c.n_seq; b0 += 64) {
    const int x = b0 + (tid & 63);
    int all;
    const int prefix = wave_prefix(x < a.c.n_seq ? single_tiles(a, x, t) : 0, all);
    if (b >= b0 && b < b0 + 64) before = sum + __shfl(prefix, b - b0);
    total = sum += all;
  }
  const int per = share_size(a, total), s0 = before / per, n = (before + tiles - 1) / per - s0 + 1;
  if (n == 1) return;
  const int blocks = (a.group.d + 15) / 16, head_blocks = a.c.n_kv_heads * blocks, cols = min(a.group.d, 16);
  const int hb = head / a.group.d * blocks + head % a.group.d / 16, col = head % a.group.d % 16;
  const auto part = [&](int i) { return single_part(a, HD, s0 + i, hb, head_blocks, i == 0); };
  const int ml = cols * HD + 2 * col;
  float m = -INFINITY;
  for (int i = tid; i < n; i += 256) m = fmaxf(m, part(i)[ml]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  if ((tid & 63) == 0) red[0][wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  for (int i = tid; i < n; i += 256) l += part(i)[ml + 1] * exp2f(part(i)[ml] - ref);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
  if ((tid & 63) == 0) red[1][wave] = l;
  const int g = tid / DT, d = tid % DT * 4;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = g; i < n; i += GROUPS) o += exp2f(part(i)[ml] - ref) * *(const f32x4*)(part(i) + col * HD + d);
  *(f32x4*)&sum_o[g][d] = o;
  __syncthreads();
  l = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  if (tid < HD) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < GROUPS; ++w) s += sum_o[w][tid];
    dst[tid] = from_f<T>(l == 0.f ? 0.f : s * (1.0f / l));
    if (lse && tid == 0) *lse = lse_of(m, l);
  }
}

// 16 columns of a tile of rows, by a workgroup: 16 threads a column.
template <typename T, int HD>
__device__ __forceinline__ void join_rows(const PagedAttnArgs& a, int item, int col_block) {
  constexpr int DT = HD / 16;
  const RowTile<ROW_KEYS<T>> t = row_tile<ROW_KEYS<T>, ROW_TILE<T>>(a, item / a.c.n_kv_heads);
  if (t.b < 0 || t.split > 0) return;
  const int n = t.splits;
  const int col = col_block * 16 + threadIdx.x / 16, d = threadIdx.x % 16 * DT;
  if (n == 1 || col >= t.cols) return;
  const int hk = item % a.c.n_kv_heads;
  float m = -INFINITY, l = 0.f;
  for (int i = 0; i < n; ++i) m = fmaxf(m, row_part(a, ROW_TILE<T>, HD, t.n, item, i)[ROW_TILE<T> * HD + 2 * col]);
  const float ref = m == -INFINITY ? 0.f : m;
  float o[DT] = {};
  for (int i = 0; i < n; ++i) {
    const float* part = row_part(a, ROW_TILE<T>, HD, t.n, item, i);
    const float f = exp2f(part[ROW_TILE<T> * HD + 2 * col] - ref);
    l += f * part[ROW_TILE<T> * HD + 2 * col + 1];
#pragma unroll
    for (int e = 0; e < DT; ++e) o[e] += f * part[col * HD + d + e];
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const int row = t.r.first + (t.col0 + col) / a.group.d, head = hk * a.group.d + (t.col0 + col) % a.group.d;
  T* dst = (T*)a.o + row * a.o_stride + head * HD + d;
#pragma unroll
  for (int e = 0; e < DT; ++e) dst[e] = from_f<T>(o[e] * inv);
  if (a.lse && d == 0) a.lse[(size_t)row * a.n_heads + head] = lse_of(m, l);
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void join_kernel(PagedAttnArgs a, int singles) {
  const int i = blockIdx.x;
  if (i < singles) {
    join_single<T, HD>(a, i / a.n_heads, i % a.n_heads);
  } else {
    const int blocks = ROW_TILE<T> / 16;
    join_rows<T, HD>(a, (i - singles) / blocks, (i - singles) % blocks);
  }
}

// ------------------------------------------------------------------ launch
bool paged_plan(int dtype, int head_dim, int n_kv_heads, int n_heads, int n_seq, bool single, int M, int cap, PagedPlan* p) {
  const int group = n_heads / n_kv_heads;
  const long head_blocks = (long)n_kv_heads * ((group + 15) / 16);
  const long most_tiles = (cap + KEY_TILE - 1) / KEY_TILE + 1;  // of a request's keys
  long floats = 0, single_grid = n_seq * head_blocks, row_grid = 0, join_singles = 0, join_rows = 0;
  *p = PagedPlan{};
  if (cap > DIRECT_KEYS) {
    const long shares = std::min((SINGLE_GRID + head_blocks - 1) / head_blocks, n_seq * most_tiles / SHARE_TILES + 1);
    p->shares = (int)shares;
    single_grid = shares * head_blocks;
    join_singles = (long)n_seq * n_heads;
    floats = shares * head_blocks * 2 * paged_part_floats(std::min(group, 16), head_dim);
  }
  p->rows_at = floats;
  p->row_splits = 1;
  const int row_tile = dtype == AF_BF16 ? ROW_TILE<bf16> : ROW_TILE<float>;
  if (!single) {
    const long columns = (long)M * group, tiles = columns / row_tile + std::min(n_seq, M / 2);  // at most so many
    row_grid = tiles * n_kv_heads;
    const long splits = std::min((long)cap / SPLIT_KEYS + 1, (long)ROW_GRID);
    // requests with a single row take n_seq rows at most; what is left may fill the GPU whatever the lengths are
    const long sure = (long)std::max(M - n_seq, 0) * group / row_tile * n_kv_heads;
    if (splits > 1 && sure <= ROW_GRID / 2) {
      p->row_splits = (int)splits;
      join_rows = tiles * n_kv_heads * (row_tile / 16);
      floats += std::min((long)ROW_GRID, row_grid * splits) * paged_part_floats(row_tile, head_dim);
      row_grid = std::max(row_grid, (long)ROW_GRID);
    }
  }
  p->floats = floats;
  const long most = 1 << 24;  // of 256 work-items, a launch has fewer than 2^32
  if (single_grid >= most || row_grid >= most || join_singles + join_rows >= most) return false;
  p->single_grid = (int)single_grid, p->row_grid = (int)row_grid;
  p->join_singles = (int)join_singles, p->join_rows = (int)join_rows;
  return true;
}

template <typename T, int HD>
static hipError_t attention_launch(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (p.row_grid > 0) {
    hipError_t e = launch_paged_rows(sizeof(T) == 2 ? AF_BF16 : AF_F32, HD, a, p.row_grid, s);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((attend_single_kernel<T, HD>), dim3(p.single_grid), dim3(256), 0, s, a);
  if (p.join_singles + p.join_rows > 0)
    hipLaunchKernelGGL((join_kernel<T, HD>), dim3(p.join_singles + p.join_rows), dim3(256), 0, s, a, p.join_singles);
  return hipGetLastError();
}

hipError_t launch_attention_paged(int dtype, int head_dim, const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (dtype == AF_BF16) return head_dim == 128 ? attention_launch<bf16, 128>(a, p, s) : attention_launch<bf16, 64>(a, p, s);
  return head_dim == 128 ? attention_launch<float, 128>(a, p, s) : attention_launch<float, 64>(a, p, s);
}

}  // namespace af
