// Declarations shared by the operators of a paged key-value cache (af_paged.hip, af_paged_rows.hip)
// and their entry points (af_paged_ops.cpp).
#pragma once

#include "af_internal.h"

namespace af {

// The cache and the step's requests, as the kernels read them.
struct PagedCache {
  void* k;               // [n_pages][n_kv_heads][page_size][head_dim]
  void* v;
  const int32_t* table;  // [n_seq][max_pages]
  const int32_t* lens;   // [n_seq]
  const int32_t* starts; // [n_seq + 1], or null: row b is request b's
  int n_pages, page_shift, n_kv_heads, n_seq, max_pages;
  int cap;               // max_pages * page_size, at most PAGED_MAX_KEYS
  int M;                 // rows
};
constexpr int PAGED_MAX_KEYS = 1 << 30;  // a tile's key numbers, past its last one, fit 32 bits
constexpr int PAGED_MIN_PAGE = 8;        // a lane's four neighbouring keys lie in one page
constexpr int PAGED_MAX_AXES = 3;

struct AppendArgs {
  PagedCache c;
  const void *q, *k, *v;
  void* q_out;
  long q_stride, k_stride, v_stride, q_out_stride;  // elements between rows
  const int32_t* positions;                         // [M][n_axes], or null: cache positions
  int n_axes, n_heads;
  int axis_end[PAGED_MAX_AXES];  // pairs [axis_end[a - 1], axis_end[a]) turn with axis a
  double turns[64];              // theta^(-2j / head_dim) / (2 pi): turns of pair j per position
};
hipError_t launch_rope_append(int dtype, int head_dim, const AppendArgs& a, hipStream_t s);

struct Divisor {
  int d, shift;  // shift < 0: no power of two
};
inline Divisor divisor(int d) { return Divisor{d, (d & (d - 1)) == 0 ? __builtin_ctz(d) : -1}; }

struct PagedAttnArgs {
  PagedCache c;
  const void* q;
  void* o;
  float* lse;  // [M][n_heads] or null
  long q_stride, o_stride;
  int n_heads;
  Divisor group, n_kv_heads;  // heads that share a key head; key heads
  float scale_log2;    // scale * log2(e)
  int window, sinks;   // window INT_MAX: none
  float* parts;        // what is left for the join, and partial results of what is split over the keys
  long parts_at, rows_at;  // floats before those of shares (the join's words), and before those of tiles of rows
  int shares;          // requests with a single row: shares of a key head's keys, 0: a workgroup for each request
  int single_waves;    // and its waves for each, 1, 2 or 4
  int row_parts;       // parts of tiles of rows, of each key head, that the workspace holds
};
// A partial result: outputs of `cols` columns, then a maximum and a sum for each, in whole chunks of 16 bytes.
__host__ __device__ inline size_t paged_part_floats(int cols, int hd) { return ((size_t)cols * (hd + 2) + 3) / 4 * 4; }
// Tiles of rows: columns and keys of one, and the fewest key tiles of a part, which go by the type.
template <typename T>
constexpr int ROW_TILE = sizeof(T) == 2 ? 128 : 64;
template <typename T>
constexpr int ROW_KEYS = sizeof(T) == 2 ? 64 : 32;
template <typename T>
constexpr int SPLIT_TILES = sizeof(T) == 2 ? 8 : 4;
// Workgroups that tiles of rows and their parts are to give: as many as the GPU holds at once.  (1024, and parts of 16 key
// tiles at least, were no faster for four chunks of 256 rows and 28 single rows.)
constexpr int ROW_GRID = 512;

// How a call of these sizes is launched, and its workspace.
struct PagedPlan {
  int shares, single_waves;
  bool row_split;                  // the keys of tiles of rows may be split
  long parts_at, rows_at, floats;  // floats of workspace before shares, before tiles of rows, in all
  int single_grid, row_grid;       // workgroups of single rows, of tiles of rows
  int tile_grid;                   // of these, as many as there can be tiles
  int join_singles, join_rows;  // workgroups of the join, 0: nothing can be split
};
// False: more workgroups than a launch takes.
bool paged_plan(int dtype, int head_dim, int n_kv_heads, int n_heads, int n_seq, bool single, int M, int cap, PagedPlan* p);
// Floats of workspace that are enough for every step of up to M rows; false as above, for M rows.
bool paged_workspace(int dtype, int head_dim, int n_kv_heads, int n_heads, int n_seq, bool single, int M, int cap, long* floats);
hipError_t launch_attention_paged(int dtype, int head_dim, const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s);
hipError_t launch_paged_rows(int dtype, int head_dim, const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s);

}  // namespace af
