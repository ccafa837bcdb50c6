// gfx950 kernels of attention over a paged cache for requests with several rows: prompts and chunks of them.
#include "af_paged_device.h"

namespace af {

// Four waves, 16 columns each.
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void attend_rows_kernel(PagedAttnArgs a) {
  typedef Columns<T, HD> C;
  constexpr int VJ = C::VJ;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lg = lane >> 4;
  const int hk = blockIdx.x % a.c.n_kv_heads;
  RowTiles at = row_tiles(a, 0x7fffffff);
  if (at.n == 0) return;
  const int split = blockIdx.x / a.c.n_kv_heads / at.n, item = blockIdx.x / a.c.n_kv_heads % at.n;
  at = row_tiles(a, item);
  const RowTile t = row_tile(a, at);
  if (split >= t.splits) return;
  const int w0 = wave * 16;
  if (w0 >= t.cols) return;
  const int col = t.col0 + min(w0 + lr, t.cols - 1);  // columns past the last one repeat it
  const int row = t.r.first + col / a.group, head = hk * a.group + col % a.group;
  const int base = t.r.len - t.r.n, p = base + col / a.group;
  const int lowest = base + (t.col0 + w0) / a.group, highest = base + (t.col0 + min(w0 + 15, t.cols - 1)) / a.group;
  C c;
  c.clear();
  c.load_q((const T*)a.q + row * a.q_stride + head * HD);
  const int end = min((split + 1) * t.per, t.keys.n);
  for (int i = split * t.per; i < end; ++i) {
    const int j0 = t.keys.key(i);
    if (j0 > highest || (j0 + KEY_TILE - 1 <= max(lowest, -1) - a.window && j0 >= a.sinks)) continue;
    attend_tile<T, HD, true>(a, hk, j0, page_of(a.c, at.b, j0), p, lowest, highest, c);
  }
  const float l = c.sum();
  if (w0 + lr >= t.cols) return;
  if (t.splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    T* dst = (T*)a.o + row * a.o_stride + head * HD + lg * 4 * VJ;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < VJ; ++j) dst[e * VJ + j] = from_f<T>(c.o[j][e] * inv);
    if (a.lse && lg == 0) a.lse[(size_t)row * a.n_heads + head] = lse_of(c.m, l);
  } else {
    float* part = row_part(a, HD, at.n, item * a.c.n_kv_heads + hk, split);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < VJ; ++j) part[(w0 + lr) * HD + (lg * 4 + e) * VJ + j] = c.o[j][e];
    if (lg == 0) {
      part[a.row_tile * HD + 2 * (w0 + lr)] = c.m;
      part[a.row_tile * HD + 2 * (w0 + lr) + 1] = l;
    }
  }
}

hipError_t launch_paged_rows(int dtype, int head_dim, const PagedAttnArgs& a, int grid, hipStream_t s) {
  if (dtype == AF_BF16) {
    if (head_dim == 128) hipLaunchKernelGGL((attend_rows_kernel<bf16, 128>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attend_rows_kernel<bf16, 64>), dim3(grid), dim3(256), 0, s, a);
  } else {
    if (head_dim == 128) hipLaunchKernelGGL((attend_rows_kernel<float, 128>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attend_rows_kernel<float, 64>), dim3(grid), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace af
