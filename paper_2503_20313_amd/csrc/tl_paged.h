// Geometry of the paged-cache operators: what the host resolves from tl_paged_dims and the kernels are given.
#pragma once
#include "tl_fast_div.h"
#include "tl_host.h"

namespace tl {

constexpr int kPagedD = 128;          // head_dim
constexpr int kMaxBatch = 4096;       // the planning kernels keep a few words per request in LDS
constexpr int kBlk = 64;              // keys per block: the unit in which the schedule cuts the key axis
constexpr int kTileRows = 256;        // query rows (token-major, the query heads of a key head side by side) of a tile
constexpr int kFewRows = 32;          // requests with at most so many rows per key head go to the few-row kernel, one tile each

// Schedule: a header of 16 ints -- 0, items, cut tiles of the tile class, 0, what it was made for --, the cut tiles' first items, then the items.
constexpr int kSchedHeader = 16, kSchedDims = 4;
// An item is a tile, or a run of its key blocks: request, first token row, tokens, sequence length, tile, first and end key block,
// first partial slot of the tile, index of the run, runs of the tile, 1 for few rows, 0.
constexpr int kItemInts = 12;

struct PagedGeom {
  int B, T, max_new, max_blocks, page, page_shift, n_pages, Hq, Hk, G, window;
  long page_stride;        // elements
  int rt;                  // row tiles of 16 in the few-row kernel (0: that class is empty)
  int has_tiles;           // requests with more than kFewRows rows may occur
  int cap_few, cap_tile;   // items per key head at most
  int side;                // items per key head that run side by side: the key axes are cut for so many
  int sched_items;         // where the items start in the schedule, in ints
  int rows_few, rows_tile; // rows of a partial result
  FastDiv by_group;        // G: row of a request -> token
};

// Header word i of a schedule for `g`.  Words from kSchedDims on are all that items, and the room for them in schedule, tables, rows and
// workspace, follow from; the other fields are made of these, and page_stride, which no item depends on, may be another for every layer.
__host__ __device__ __forceinline__ int sched_header(const PagedGeom& g, int i, int items, int cuts) {
  const int h[kSchedHeader] = {0, items, cuts, 0, g.B, g.T, g.max_new, g.max_blocks, g.page, g.n_pages, g.Hq, g.Hk, g.window, g.side, 0, 0};
  return h[i];
}
// A schedule serves the dims it was made for and no others: every word is compared (ordinary dims share any hash of them).  One that was
// never made is zero, which no batch is.
__host__ __device__ __forceinline__ bool sched_made_for(const int* schedule, const PagedGeom& g) {
  int other = 0;
#pragma unroll
  for (int i = kSchedDims; i < kSchedHeader; i++) other |= schedule[i] ^ sched_header(g, i, 0, 0);
  return other == 0;
}

struct Item { int b, q0, n, seq, tile, k0, k1, slot, run, runs, few; };

__host__ __device__ __forceinline__ Item load_item(const int* schedule, const PagedGeom& g, int idx) {
  const int* rec = schedule + g.sched_items + (long)idx * kItemInts;
  Item i;
  i.b = rec[0]; i.q0 = rec[1]; i.n = rec[2]; i.seq = rec[3]; i.tile = rec[4]; i.k0 = rec[5]; i.k1 = rec[6]; i.slot = rec[7]; i.run = rec[8]; i.runs = rec[9]; i.few = rec[10];
  return i;
}
// Item `idx` of a launch, if the schedule has it.  Before that is known nothing behind the header is read: the schedule of smaller dims
// ends anywhere behind it.
__host__ __device__ __forceinline__ bool sched_item(const int* schedule, const PagedGeom& g, int idx, Item* it) {
  if (!sched_made_for(schedule, g) || idx >= schedule[1]) return false;
  *it = load_item(schedule, g, idx);
  return true;
}

int resolve_paged(const tl_ctx* ctx, const tl_paged_dims* d, PagedGeom* g);

// Last check before a launch: a real context, and its device is the current one (the stream belongs to that device).
inline int check_paged_launch(const tl_ctx* ctx, const char* what) {
  if (int e = check_op_ctx(ctx)) return e;
  int dev = -1;
  TL_HIP(hipGetDevice(&dev));
  if (dev != ctx->device) return fail(TL_ERR_INVALID_ARG, "%s: the context was created on device %d, the current device is %d", what, ctx->device, dev);
  return TL_OK;
}

// A grid's work items are counted in 32 bits a dimension, and a larger one is cut off at its end without an error: workgroups beyond kGridX
// go into rows of a second dimension, of which the last may reach beyond `workgroups`.
constexpr unsigned kGridX = 1u << 16;
constexpr long kMostWorkgroups = 65535L * kGridX;
inline dim3 grid_of(long workgroups) {
  return workgroups <= (long)kGridX ? dim3((unsigned)workgroups) : dim3(kGridX, (unsigned)((workgroups + kGridX - 1) / kGridX));
}
__device__ __forceinline__ unsigned workgroup_index() { return blockIdx.y * kGridX + blockIdx.x; }

inline bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace tl
