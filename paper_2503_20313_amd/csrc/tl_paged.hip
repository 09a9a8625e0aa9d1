// A paged key/value cache and the attention that reads it: block tables and slot maps from request lengths, the attention's work
// table, and attention of a chunk of new tokens per request over its cached keys.  gfx950 only, head_dim 128.
//
// Cache: page p, key head h, row r at p * page_stride + (h * page_size + r) * 128 elements, so the rows of a page and head are one
// contiguous piece (4 KiB for the smallest page) and 16 keys never straddle pages.
#include <atomic>

#include "tl_gemm_tile.h"
#include "tl_host.h"
#include "tl_paged.h"
#include "tl_softmax.h"

namespace tl {

typedef short short8_t __attribute__((ext_vector_type(8)));

// ======================================================================================
// Block tables and slot maps.  Two scans over the requests (tokens, then new pages), done by every workgroup for itself in LDS;
// then a thread per token finds its request by binary search, and a thread per new page writes its table entry.  Where several
// workgroups share the maps and lengths or the head of the free list are written in place, those are left to a second launch of one
// workgroup, so that no workgroup's inputs change under it.
//
// Bound by latency: lengths, scans, free list, stores, each a few hundred nanoseconds behind the other.  A token to a thread: 64 k tokens of
// 512 requests 14 -> 7 us against four in a row and a second launch; small steps take one wave, without barriers (6.5 -> 4.4 us).
// ======================================================================================
struct SlotsParams {
  const int *ctx_lens, *new_lens, *free_pages, *free_from;
  int n_free;
  int *free_to, *block_table, *query_start, *seq_lens, *slots, *positions, *counts;
  int B, T, max_new, max_blocks, page, page_shift, n_pages;
};

// Inclusive scan over the workgroup's threads; *total = the sum.  All threads call it.
template <int NT>
__device__ __forceinline__ int block_scan(int v, int* s_wave, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  if constexpr (NT == 64) {
    *total = __shfl(v, 63);
    return v;
  }
  __syncthreads();   // (s_wave may still be read by the previous scan)
  if (lane == 63) s_wave[wave] = v;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; w++) {
    const int x = s_wave[w];
    if (w < wave) before += x;
    all += x;
  }
  *total = all;
  return v + before;
}

// Over the 64 lanes of a wave, in every lane: rotations inside rows of 16 lanes, then the four rows.
template <class F>
__device__ __forceinline__ int wave_reduce(int x, F f) {
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, true));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, true));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, true));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, true));
  return f(f(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16)), f(__builtin_amdgcn_readlane(x, 32), __builtin_amdgcn_readlane(x, 48)));
}

// The largest i in [0, n) with a[i] <= x, for a[0] <= x and ascending a: of equal entries the last, so empty requests are passed over.
__device__ __forceinline__ int last_at_most(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

constexpr int kMaps = 1, kLengths = 2;

template <int PARTS, int NT>     // what this launch writes; kLengths: by workgroup 0.  NT = 64: at most 64 requests
__global__ void __launch_bounds__(NT) paged_slots_kernel(const SlotsParams p) {
  constexpr int kReq = NT == 64 ? 1 : kMaxBatch / NT;      // requests per thread at most
  constexpr int kRoom = NT == 64 ? 64 : kMaxBatch;
  __shared__ int s_wave[NT / 64];
  __shared__ int s_start[kRoom + 1], s_page[kRoom + 1], s_ctx[kRoom];
  const int tid = threadIdx.x;
  const int per = (p.B + NT - 1) / NT, b0 = tid * per;     // a thread's requests: b0 .. b0 + per - 1
  const int cap = p.max_blocks * p.page;
  const int from = p.free_from ? max(p.free_from[0], 0) : 0;
  int len[kReq];
  int sum = 0, over = 0;
  // Tokens that do not fit: requests may ask for 2^43 together, so their sum stays at the largest int where it gets there.
  auto add_over = [](int x, int y) { return (int)min((unsigned)x + (unsigned)y, 0x7fffffffu); };
#pragma unroll
  for (int i = 0; i < kReq; i++) {
    len[i] = 0;
    if (i < per && b0 + i < p.B) {
      const int c = min(max(p.ctx_lens[b0 + i], 0), cap), want = max(p.new_lens[b0 + i], 0);
      s_ctx[b0 + i] = c;
      len[i] = min(min(want, p.max_new), cap - c);
      sum += len[i];             // (max_new is at most 2^18: 2^12 * 2^18, the sums fit)
      over = add_over(over, want - len[i]);
    }
  }
  int all_tokens, all_pages;
  int at = block_scan<NT>(sum, s_wave, &all_tokens) - sum;
  // tokens that do not fit the rows are cut off at the end
  int pages = 0;
#pragma unroll
  for (int i = 0; i < kReq; i++)
    if (i < per && b0 + i < p.B) {
      const int lo = min(at, p.T), hi = min(at + len[i], p.T);
      over = add_over(over, len[i] - (hi - lo));
      at += len[i];
      s_start[b0 + i] = lo;
      len[i] = hi - lo;
      const int c = s_ctx[b0 + i];
      pages += ((c + len[i] + p.page - 1) >> p.page_shift) - ((c + p.page - 1) >> p.page_shift);
    }
  int pg = block_scan<NT>(pages, s_wave, &all_pages) - pages;
#pragma unroll
  for (int i = 0; i < kReq; i++)
    if (i < per && b0 + i < p.B) {
      const int c = s_ctx[b0 + i];
      s_page[b0 + i] = pg;
      pg += ((c + len[i] + p.page - 1) >> p.page_shift) - ((c + p.page - 1) >> p.page_shift);
    }
  const int n_tokens = min(all_tokens, p.T);
  const int left = max(p.n_free - from, 0);          // pages that the list still holds
  const bool lengths = (PARTS & kLengths) && blockIdx.x == 0;
  if (lengths) {
    over = wave_reduce(over, add_over);
    if constexpr (NT > 64) {
      __syncthreads();   // (s_wave may still be read by the scan)
      if ((tid & 63) == 0) s_wave[tid >> 6] = over;
      __syncthreads();
      over = 0;
#pragma unroll
      for (int w = 0; w < NT / 64; w++) over = add_over(over, s_wave[w]);
    }
  }
  if (tid == 0) { s_start[p.B] = n_tokens; s_page[p.B] = all_pages; }
  __syncthreads();   // every input that this workgroup may write in place has been read
  if (PARTS & kMaps) {
    const int step = gridDim.x * NT;
    for (int i = blockIdx.x * NT + tid; i < all_pages; i += step) {
      const int page = i < left ? p.free_pages[from + i] : -1;
      const int b = last_at_most(s_page, p.B, i);
      const int j = ((s_ctx[b] + p.page - 1) >> p.page_shift) + i - s_page[b];
      p.block_table[(long)b * p.max_blocks + j] = page;
    }
    for (int t = blockIdx.x * NT + tid; t < p.T; t += step) {
      int slot = -1, pos = 0;
      if (t < n_tokens) {
        const int b = last_at_most(s_start, p.B, t);
        const int c = s_ctx[b], have = (c + p.page - 1) >> p.page_shift;
        pos = c + t - s_start[b];
        const int blk = pos >> p.page_shift;
        int page;
        if (blk < have) page = p.block_table[(long)b * p.max_blocks + blk];   // the partly filled page of the cached tokens
        else {
          const int i = s_page[b] + blk - have;
          page = i < left ? p.free_pages[from + i] : -1;
        }
        if ((unsigned)page < (unsigned)p.n_pages) slot = (page << p.page_shift) + (pos & (p.page - 1));
      }
      p.slots[t] = slot;
      p.positions[t] = pos;
    }
  }
  if (lengths) {
    for (int b = tid; b <= p.B; b += NT) {
      p.query_start[b] = s_start[b];
      if (b < p.B) p.seq_lens[b] = s_ctx[b] + s_start[b + 1] - s_start[b];
    }
    if (tid == 0) {
      const int taken = min(all_pages, left);
      if (p.free_to) p.free_to[0] = from + taken;
      p.counts[0] = n_tokens;
      p.counts[1] = taken;
      p.counts[2] = all_pages - taken;
      p.counts[3] = over;
    }
  }
}

// ======================================================================================
// Schedule: the attention's work table.  A tile is kTileRows query rows of one request (all of a request's rows, if they are at
// most kFewRows); its keys are the blocks its rows can see.  A tile whose key axis is longer than its class's chunk is cut into
// runs of equal length, joined afterwards.  The chunk is an even share of the work, or up to half as much again where that lets all
// items run side by side; the items stand in order of their length, the longest first, for the hardware to hand out.
// Measured with every chunk from a quarter of the share to uncut, the even share is within 3 % of the best in batches that do not fit
// side by side (64 requests of 500..8000 tokens: 188 us, at a quarter 197; in the requests' order instead of by length 222), and a
// longer one that makes them fit is worth it up to half (128 requests of 1000..10000: 78 us against 87), not beyond.
//
// Bound by latency: one workgroup, a chain of passes over the requests.  The lengths are read once, into LDS; small batches take one
// wave, whose reductions need no barriers.
// ======================================================================================
struct SchedParams {
  const int *query_start, *seq_lens;
  int* out;
  PagedGeom g;
};

// A block of 64 keys costs in a tile kCostTile / kCostFew of what it costs with few rows: 2.0 us against 0.75, the chip at work.
constexpr int kCostFew = 3, kCostTile = 8;
constexpr int kChunks = 5;                    // chunk lengths tried: an even share, and 1 .. 4 eighths of it more
constexpr int kMinChunk = 4;                  // blocks of a run at least
constexpr int kBuckets = 64;

// Key blocks that rows [tile*rows, +rows) of a request see.
__device__ __forceinline__ void tile_span(const PagedGeom& g, int n, int seq, int tile, int rows, int* lo, int* hi) {
  const int t0 = tile * rows / g.G, t1 = min((tile * rows + rows - 1) / g.G, n - 1);
  const int end = max(seq - n + t1 + 1, 0);
  const int start = g.window ? max(seq - n + t0 - g.window + 1, 0) : 0;
  *hi = (end + kBlk - 1) / kBlk;
  *lo = min(start / kBlk, *hi);
}

template <int NT>
__global__ void __launch_bounds__(NT) paged_schedule_kernel(const SchedParams p) {
  const PagedGeom& g = p.g;
  constexpr int NW = NT / 64;
  __shared__ int s_wave[NW];
  __shared__ int s_q0[kMaxBatch], s_n[kMaxBatch], s_seq[kMaxBatch];
  __shared__ int s_first[kMaxBatch + 1];     // tiles (of the tile class) of the requests before this one
  __shared__ unsigned long long s_work;
  __shared__ int s_count[kChunks], s_long;
  __shared__ int s_bucket[kBuckets], s_slots[2], s_cut;
  const int tid = threadIdx.x, lane = tid & 63;
  auto add = [](int x, int y) { return x + y; };
  auto top = [](int x, int y) { return max(x, y); };
  bool bad = false;      // row starts that do not ascend inside the rows, lengths outside the dims: no request can be trusted
  for (int b = tid; b < g.B; b += NT) {
    const int lo = p.query_start[b], hi = p.query_start[b + 1], seq = p.seq_lens[b];
    bad |= lo < 0 || hi < lo || hi > g.T || hi - lo > g.max_new || seq < 0 || seq > g.max_blocks * g.page;
    s_q0[b] = lo;
    s_n[b] = hi - lo;
    s_seq[b] = seq;
  }
  if (tid == 0) s_work = 0;
  if (tid < kChunks) s_count[tid] = 0;
  if (tid < kBuckets) s_bucket[tid] = 0;
  if (tid < 2) s_slots[tid] = 0;
  if (tid == 0) { s_cut = 0; s_long = 0; }
  if (__syncthreads_or(bad)) {
    if (tid == 0) {
#pragma unroll
      for (int i = 0; i < kSchedHeader; i++) p.out[i] = sched_header(g, i, 0, 0);
    }
    return;
  }
  auto is_few = [&](int b) { return g.rt > 0 && s_n[b] * g.G <= kFewRows; };   // (at most 2^28)
  int n_tiles = 0;
  if (g.has_tiles) {
    for (int base = 0; base < g.B; base += NT) {
      const int b = base + tid;
      const int mine = b < g.B && !is_few(b) ? (s_n[b] * g.G + kTileRows - 1) / kTileRows : 0;
      int v = mine;      // inclusive scan
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
      }
      int total = __shfl(v, 63);
      if constexpr (NW > 1) {
        __syncthreads();
        if (lane == 63) s_wave[tid >> 6] = v;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int i = 0; i < NW; i++) {
          const int x = s_wave[i];
          if (i < (tid >> 6)) v += x;
          total += x;
        }
      }
      if (b < g.B) s_first[b] = n_tiles + v - mine;
      n_tiles += total;
    }
    if (tid == 0) s_first[g.B] = n_tiles;
    __syncthreads();
  }
  // ---- all tiles of both classes: number i is request i's few rows, if it has few, then tile number i - B of the tile class
  const int n_all = g.B + n_tiles;
  struct Tile { int b, tile, lo, hi; bool few; };
  auto tile_at = [&](int i, Tile* t) -> bool {
    t->few = i < g.B;
    t->b = i; t->tile = 0;
    if (t->few) {
      if (s_n[i] == 0 || !is_few(i)) return false;
      tile_span(g, s_n[i], s_seq[i], 0, kFewRows, &t->lo, &t->hi);
    } else {
      t->b = last_at_most(s_first, g.B, i - g.B);
      t->tile = s_first[t->b + 1] - 1 - (i - g.B);
      tile_span(g, s_n[t->b], s_seq[t->b], t->tile, kTileRows, &t->lo, &t->hi);
    }
    return true;
  };
  // (every pass below goes over them; a thread's first one stays in registers)
  Tile mine = {0, 0, 0, 0, false};
  const bool has = tid < n_all && tile_at(tid, &mine);
  auto tile_of = [&](int i, Tile* t) -> bool {
    if (i >= NT) return tile_at(i, t);
    *t = mine;
    return has;
  };
  unsigned long long work = 0;
  for (int i = tid; i < n_all; i += NT) {
    Tile t;
    if (tile_of(i, &t)) work += (unsigned long long)(unsigned)(t.hi - t.lo) * (unsigned)(t.few ? kCostFew : kCostTile);
  }
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) work += __shfl_xor(work, d);
  if constexpr (NW > 1) {
    if (lane == 0) atomicAdd(&s_work, work);
    __syncthreads();
    work = s_work;
  }
  // ---- the chunk lengths, in blocks
  // (divisions are 32 bits wide wherever the numbers are: together 0.3 us)
  const unsigned long long up = work + (unsigned)(g.side - 1);
  const unsigned long long share = (up >> 32) ? up / (unsigned)g.side : (unsigned)up / (unsigned)g.side;
  int chunk_f[kChunks], chunk_t[kChunks], count[kChunks];
#pragma unroll
  for (int j = 0; j < kChunks; j++) {
    const unsigned long long c = (share * (8 + j) + 7) / 8;
    const unsigned long long most = 1ull << 24;      // (a key axis has at most 2^22 blocks)
    chunk_f[j] = max((int)min((c + kCostFew - 1) / kCostFew, most), kMinChunk);
    chunk_t[j] = max((int)min((c + kCostTile - 1) / kCostTile, most), kMinChunk);
    count[j] = 0;
  }
  auto runs_of = [&](const Tile& t, int cf, int ct) -> int {
    const unsigned c = (unsigned)(t.few ? cf : ct);
    return max((int)(((unsigned)(t.hi - t.lo) + c - 1) / c), 1);
  };
  auto item_cost = [&](const Tile& t, int n) -> int { return ((t.hi - t.lo + n - 1) / n) * (t.few ? kCostFew : kCostTile); };   // of the longest run
  for (int i = tid; i < n_all; i += NT) {
    Tile t;
    if (!tile_of(i, &t)) continue;
#pragma unroll
    for (int j = 0; j < kChunks; j++) count[j] += runs_of(t, chunk_f[j], chunk_t[j]);
  }
#pragma unroll
  for (int j = 0; j < kChunks; j++) {
    count[j] = wave_reduce(count[j], add);
    if constexpr (NW > 1) {
      if (lane == 0) atomicAdd(&s_count[j], count[j]);
    }
  }
  if constexpr (NW > 1) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kChunks; j++) count[j] = s_count[j];
  }
  int chunk_few = chunk_f[0], chunk_tile = chunk_t[0];
#pragma unroll
  for (int j = kChunks - 1; j >= 0; j--)
    if (count[j] <= g.side) { chunk_few = chunk_f[j]; chunk_tile = chunk_t[j]; }

  // ---- the items, by buckets of their cost.  (Places inside a bucket and partial slots go by arrival: they say where and when an item
  // is computed, not what.)
  int longest = 0;
  for (int i = tid; i < n_all; i += NT) {
    Tile t;
    if (tile_of(i, &t)) longest = max(longest, item_cost(t, runs_of(t, chunk_few, chunk_tile)));
  }
  longest = wave_reduce(longest, top);
  if constexpr (NW > 1) {
    if (lane == 0) atomicMax(&s_long, longest);
    __syncthreads();
    longest = s_long;
  }
  const float per_cost = (float)kBuckets / ((float)longest + 1.f);
  auto bucket_of = [&](const Tile& t, int n) -> int { return kBuckets - 1 - min((int)((float)item_cost(t, n) * per_cost), kBuckets - 1); };
  for (int i = tid; i < n_all; i += NT) {
    Tile t;
    if (!tile_of(i, &t)) continue;
    const int n = runs_of(t, chunk_few, chunk_tile);
    atomicAdd(&s_bucket[bucket_of(t, n)], n);
  }
  __syncthreads();
  int n_items = 0;
  if (tid < 64) {
    static_assert(kBuckets == 64, "one lane each");
    const int mine = s_bucket[lane];
    int v = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(v, d);
      if (lane >= d) v += o;
    }
    s_bucket[lane] = v - mine;
    n_items = __shfl(v, 63);
  }
  __syncthreads();
  int* items = p.out + g.sched_items;
  for (int base = 0; base < n_all; base += NT) {
    const int i = base + tid;
    Tile t = {0, 0, 0, 0, false};
    int n = 0, to = 0, slot = 0;
    if (i < n_all && tile_of(i, &t)) {
      n = runs_of(t, chunk_few, chunk_tile);
      to = atomicAdd(&s_bucket[bucket_of(t, n)], n);
      if (n > 1) {
        slot = atomicAdd(&s_slots[t.few ? 0 : 1], n);
        if (!t.few) p.out[kSchedHeader + atomicAdd(&s_cut, 1)] = to;
      }
    }
    // the wave's runs, 64 at a time: run number r of the wave belongs to the last lane whose first run is not after it
    int v = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(v, d);
      if (lane >= d) v += o;
    }
    const int first = v - n, all = __shfl(v, 63);
    for (int r0 = 0; r0 < all; r0 += 64) {
      const int r = r0 + lane;
      int own = 0;
#pragma unroll
      for (int d = 32; d >= 1; d /= 2) {
        const int f = __shfl(first, own + d > 63 ? 63 : own + d);
        if (own + d <= 63 && f <= r) own += d;
      }
      const int ob = __shfl(t.b, own), ot = __shfl(t.tile, own), olo = __shfl(t.lo, own), ohi = __shfl(t.hi, own), oc = __shfl(n, own), oto = __shfl(to, own);
      const int oslot = __shfl(slot, own), of = __shfl(t.few ? 1 : 0, own), s = r - __shfl(first, own);
      if (r < all) {
        int* rec = items + (long)(oto + s) * kItemInts;       // (below the number of items there is room for: see resolve_paged)
        const u32x4 q0 = {(unsigned)ob, (unsigned)s_q0[ob], (unsigned)s_n[ob], (unsigned)s_seq[ob]};
        const unsigned len = (unsigned)(ohi - olo);                 // (at most 2^22 blocks, in fewer than 2^10 runs)
        const u32x4 q1 = {(unsigned)ot, (unsigned)olo + len * (unsigned)s / (unsigned)oc, (unsigned)olo + len * (unsigned)(s + 1) / (unsigned)oc, (unsigned)oslot};
        const u32x4 q2 = {(unsigned)s, (unsigned)oc, (unsigned)of, 0};
        *(u32x4*)rec = q0;
        *(u32x4*)(rec + 4) = q1;
        *(u32x4*)(rec + 8) = q2;
      }
    }
  }
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int i = 0; i < kSchedHeader; i++) p.out[i] = sched_header(g, i, n_items, s_cut);
  }
}

// ======================================================================================
// Attention.
// ======================================================================================
// The exponents' reference of a row follows the row's maximum only where that has left it by more than kLazy (in exponents of two), so that
// sums and O need no rescaling in nearly every block.  Every weight is 2^-kLazy times exp2 of what lies above the reference: in (0, 1], as
// with a reference that is the maximum itself, so whatever a sum of such weights holds is finite here too (weights up to 2^kLazy would let
// values above 2^120 overflow).  At the other end, weights below 2^(kLazy - 126) of the largest are zero.
constexpr float kLazy = 8.f;

struct PagedAttn {
  PagedGeom g;
  const bf16_t* q;
  const bf16_t *k_cache, *v_cache;
  const int *block_table, *schedule;
  bf16_t* o;
  float* lse;               // [T, Hq] or null
  long q_stride, o_stride;
  float scale_log2e;
  float lazy;               // how far, in scores, a row's maximum may leave the exponents' reference: kLazy in exponents
  float *part_few, *part_tile;     // partial results: [slot][key head][row][128], unnormalised, and [slot][key head][row][2]: maximum, sum
  float *ml_few, *ml_tile;
  float *group_few, *group_ml;     // few-row class: what the runs of a group were joined to, at the group's first run's place
  unsigned *arrived;               // few-row class: per (slot, key head) runs of a group that have arrived, groups of a tile that have; zero between calls
};

__device__ __forceinline__ bool not_finite(unsigned bits16) { return (bits16 & 0x7f80u) == 0x7f80u; }

// 16 bytes of a value row whose non-finite elements became zeros; any = there were some.
__device__ __forceinline__ u32x4 finite_only(u32x4 v, bool* any) {
#pragma unroll
  for (int e = 0; e < 4; e++) {
    if (not_finite(v[e])) { v[e] &= 0xffff0000u; *any = true; }
    if (not_finite(v[e] >> 16)) { v[e] &= 0xffffu; *any = true; }
  }
  return v;
}

// Row `row` of a request (token-major, the query heads of the key head side by side): its token and query head.
__device__ __forceinline__ int token_of(const PagedGeom& g, int row, int head, int* hq) {
  const int token = (int)g.by_group.div((unsigned)row);
  *hq = head * g.G + row - token * g.G;
  return token;
}

__device__ __forceinline__ float log_sum(float m, float l, float scale_log2e) {
  return l == 0.f ? -INFINITY : (__builtin_fmaf(m, scale_log2e, kLazy) + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}
// What a row's sum is multiplied by: a row that sees nothing is zero.
__device__ __forceinline__ float row_scale(float l) { return l > 0.f || l != l ? 1.f / l : 0.f; }

// One quad of an output row.
__device__ __forceinline__ void store_out(const PagedAttn& p, const Item& it, int head, int row, int d4, floatx4 o, float m, float l) {
  int hq;
  const int token = token_of(p.g, row, head, &hq);
  const float inv = row_scale(l);
  bf16x4 v;
#pragma unroll
  for (int e = 0; e < 4; e++) v[e] = (bf16_t)(o[e] * inv);
  *(bf16x4*)(p.o + (long)(it.q0 + token) * p.o_stride + (long)hq * kPagedD + d4) = v;
  if (p.lse && d4 == 0) p.lse[(long)(it.q0 + token) * p.g.Hq + hq] = log_sum(m, l, p.scale_log2e);
}

// A row's maximum and sum, in memory as one 8-byte word; written and read past the die's L2, where another die's part of the same
// cache line may be older.
__device__ __forceinline__ void store_ml(float* ml, long at, float m, float l) {
  const unsigned long long w = (unsigned long long)__builtin_bit_cast(unsigned, m) | ((unsigned long long)__builtin_bit_cast(unsigned, l) << 32);
  __hip_atomic_store((unsigned long long*)ml + at, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Sum of up to N partial results of one quad of a row, `step` rows apart, in order: all loads in flight together.  SAME_LAUNCH: the
// parts were written by this launch.
template <int N, bool SAME_LAUNCH>
__device__ __forceinline__ void join_quad(const float* part, const float* ml, long at, long step, int count, int d4, float scale_log2e, floatx4* o, float* m, float* l) {
  floatx4 v[N];
  float mm[N], ll[N];
#pragma unroll
  for (int s = 0; s < N; s++) {
    mm[s] = -INFINITY; ll[s] = 0.f;
    v[s] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (s < count) {
      const unsigned long long* w = (const unsigned long long*)ml + at + s * step;
      const unsigned long long x = SAME_LAUNCH ? __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : *w;
      mm[s] = __builtin_bit_cast(float, (unsigned)x);
      ll[s] = __builtin_bit_cast(float, (unsigned)(x >> 32));
      v[s] = *(const floatx4*)(part + (at + s * step) * kPagedD + d4);
    }
  }
  float top = *m;
#pragma unroll
  for (int s = 0; s < N; s++) top = fmaxf(top, mm[s]);
  const float ref = top == -INFINITY ? 0.f : top;
  const float f0 = __builtin_amdgcn_exp2f((*m - ref) * scale_log2e);
  *l *= f0;
#pragma unroll
  for (int e = 0; e < 4; e++) (*o)[e] *= f0;
#pragma unroll
  for (int s = 0; s < N; s++) {
    const float f = __builtin_amdgcn_exp2f((mm[s] - ref) * scale_log2e);
    *l += ll[s] * f;
#pragma unroll
    for (int e = 0; e < 4; e++) (*o)[e] += v[s][e] * f;
  }
  *m = top;
}

// --------------------------------------------------------------------------------------
// Few rows (single tokens, a handful of speculated ones): bound by reading K and V once.  A workgroup takes an item; its 8 waves
// take units of 32 keys in turn, each into a place of its own in LDS (K and V of a unit, filled by direct-to-LDS loads), so a wave
// never waits for another and a compute unit has up to 128 KiB in flight.  (4 waves with two units each have as much: 256 requests of
// 1000 tokens 182 us against 178, and beside tiles, whose workgroups have 8 waves, a mixed batch 105 against 98.)  Per unit and tile of 16 rows:
//   S^T[keys, q] = K . Q^T   (16x16x32 matrix instructions; a lane owns one query row and holds 4 keys of each half unit)
//   online softmax           (over the lane's 8 keys and the 4 lane groups)
//   O^T[d, q] += V^T . P^T   (P^T straight from the score registers; V^T by transposing LDS reads in the same key order)
// The waves' results are joined in LDS at the end.
// The loads are marked as streaming: every line is read once per call, and kept out of the caches' way 64 requests of 500..8000 tokens
// (1.05 GB) take 167 us against 188, one of 130000 90 against 101 (6.3 and 5.9 TB/s).
// --------------------------------------------------------------------------------------
constexpr int kFewWaves = 8;
constexpr int kUnit = 32;
constexpr int kUnitBytes = 2 * kUnit * kPagedD * 2;      // K rows, V rows: 16 KiB

constexpr int kFewLds = kFewWaves * kUnitBytes;
constexpr int kJoin = 16;                                // runs that one workgroup joins at a time

template <int RT>      // row tiles of 16
__device__ __forceinline__ void few_rows_item(const PagedAttn& p, const Item& it, int head, char* smem) {
  constexpr int NW = kFewWaves;
  const PagedGeom& g = p.g;
  const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, gr = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_rows = it.n * g.G;
  const int first_pos = it.seq - it.n;
  const int key_end = min(it.k1 * kBlk, max(it.seq, 0)), key_begin = it.k0 * kBlk;
  const int units = (max(key_end - key_begin, 0) + kUnit - 1) / kUnit;
  const int n = units > wave ? (units - wave + NW - 1) / NW : 0;       // this wave's units: wave, wave + NW, ..

  const int reach = g.window ? g.window : 0x40000000;     // a query at pos sees keys in (pos - reach, pos]
  // keys in [clean_lo, clean_hi) are seen by every row
  const int clean_lo = max(first_pos + it.n - 1 - reach + 1, 0), clean_hi = first_pos + 1;

  // ---- pages: lane 2i + half holds the page of half unit `half` of this wave's unit i (of the 32 units from `window0` on)
  const int* table = p.block_table + (long)it.b * g.max_blocks;
  auto key_of = [&](int i) __attribute__((always_inline)) { return key_begin + (wave + i * NW) * kUnit; };
  int ent = -1;
  auto load_pages = [&](int i0) __attribute__((always_inline)) {
    const int key = key_of(i0 + (lane >> 1)) + (lane & 1) * 16;
    int e = key < key_end ? table[key >> g.page_shift] : -1;
    ent = (unsigned)e < (unsigned)g.n_pages ? e : -1;
  };
  if (n > 0) load_pages(0);       // in front of the Q loads: the first K rows wait for it alone

  // ---- Q fragments and the positions of the lane's rows
  bf16x8 qf[RT][4];
  int pos[RT];
#pragma unroll
  for (int u = 0; u < RT; u++) {
    const int row = min(u * 16 + l15, n_rows - 1);
    int hq;
    const int token = token_of(g, row, head, &hq);
    const bf16_t* src = p.q + (long)(it.q0 + token) * p.q_stride + (long)hq * kPagedD + gr * 8;
#pragma unroll
    for (int s = 0; s < 4; s++) qf[u][s] = *(const bf16x8*)(src + s * 32);
    pos[u] = first_pos + token;
  }
  const unsigned smem_u = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem);
  char* st = smem + wave * kUnitBytes;
  const unsigned st_u = smem_u + wave * kUnitBytes;
  // LDS slot (row, pc) holds 16-byte chunk pc ^ (row % 16) of a K row, pc ^ ((row % 4) << 2) of a V row: conflict-free fragment reads
  const int lr = lane >> 4;
  unsigned koff[4];
#pragma unroll
  for (int j = 0; j < 4; j++) koff[j] = (unsigned)(lr * 256 + ((l15 ^ (4 * j + lr)) << 4));
  const unsigned voff = (unsigned)(lr * 256 + ((l15 ^ (lr << 2)) << 4));
  auto half_base = [&](const bf16_t* cache, int i, int half) __attribute__((always_inline)) -> const char* {
    const int pg = max(__builtin_amdgcn_readlane(ent, ((i & 31) << 1) + half), 0);    // (a page that is none: page 0, masked)
    const int row = (key_of(i) + half * 16) & (g.page - 1);
    return (const char*)uniform64((unsigned long long)(cache + (long)pg * g.page_stride + ((long)head * g.page + row) * kPagedD));
  };
  auto issue = [&](const bf16_t* cache, int i, bool is_k) __attribute__((always_inline)) {
    const unsigned dst = st_u + (is_k ? 0 : kUnitBytes / 2);
#pragma unroll
    for (int half = 0; half < 2; half++) {
      const char* base = half_base(cache, i, half);
#pragma unroll
      for (int j = 0; j < 4; j++) lds_load16_sbase_nt(base + j * 1024, is_k ? koff[j] : voff, dst + half * 4096 + j * 1024);
    }
  };
  auto halves_valid = [&](int i) __attribute__((always_inline)) -> int {
    return (__builtin_amdgcn_readlane(ent, (i & 31) << 1) >= 0 ? 1 : 0) | (__builtin_amdgcn_readlane(ent, ((i & 31) << 1) + 1) >= 0 ? 2 : 0);
  };

  // ---- LDS read offsets (within a unit)
  const int k_rd = l15 * 256 + ((gr ^ l15) << 4);
  const int v_r = l15 >> 2;
  int v_rd[8];
#pragma unroll
  for (int dt = 0; dt < 8; dt++)
    v_rd[dt] = kUnitBytes / 2 + (gr * 4 + v_r) * 256 + (((dt * 2 + ((lane & 2) >> 1)) ^ (v_r << 2)) << 4) + (lane & 1) * 8;

  floatx4 zero4 = {0.f, 0.f, 0.f, 0.f};
  floatx4 oacc[RT][8];
  float m_run[RT], l_run[RT], mc[RT];
#pragma unroll
  for (int u = 0; u < RT; u++) {
    m_run[u] = -INFINITY;
    l_run[u] = mc[u] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; dt++) oacc[u][dt] = zero4;
  }

  // K and V of the next unit are requested as soon as this unit's fragments have left their place, so that behind K of a unit, when it
  // is needed, its V is on its way, and behind V the next K: 8 loads each
  int ok = 0, ok_next = 0;       // halves of the unit that have a page
  if (n > 0) {
    ok_next = halves_valid(0);
    issue(p.k_cache, 0, true);
    issue(p.v_cache, 0, false);
  }
  for (int i = 0; i < n; i++) {
    const bool more = i + 1 < n;
    const int key0 = key_of(i);
    ok = ok_next;
    wait_vmcnt<8>();
    floatx4 c[RT][2];
#pragma unroll
    for (int hf = 0; hf < 2; hf++)
#pragma unroll
      for (int s = 0; s < 4; s++) {
        const bf16x8 kf = *(const bf16x8*)(st + hf * 4096 + (k_rd ^ (s << 6)));
#pragma unroll
        for (int u = 0; u < RT; u++) c[u][hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[u][s], s == 0 ? zero4 : c[u][hf], 0, 0, 0);
      }
    if (more) {
      if (((i + 1) & 31) == 0) load_pages(i + 1);
      ok_next = halves_valid(i + 1);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the fragments are in registers: their place may be filled again
      issue(p.k_cache, i + 1, true);
    }
    const bool masked = key0 < clean_lo || key0 + kUnit > clean_hi || ok != 3;
    // Weights as two bf16 numbers, their first 8 bits and the next 8: the matrix cores have the time for a second product here (64 requests of
    // 500..8000 tokens 167.2 -> 167.6 us, one of 1000 15.1 -> 15.3, 40 beside 8 prompt chunks 90.6 -> 92.1).  Cut, not rounded, and the
    // second part of a weight that is not zero at least 2^-126 (or the weight itself), so that both are positive: seen infinities stay what they are.
    bf16x8 pf[RT], pl[RT];
    bool grown = false;
    float top[RT];                 // of this lane's 8 scores
#pragma unroll
    for (int u = 0; u < RT; u++) {
      if (masked) {
#pragma unroll
        for (int hf = 0; hf < 2; hf++)
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const int key = key0 + hf * 16 + gr * 4 + e;
            if (key > pos[u] || key <= pos[u] - reach || !((ok >> hf) & 1)) c[u][hf][e] = -INFINITY;
          }
      }
      top[u] = fmaxf(c[u][0][0], c[u][1][0]);
#pragma unroll
      for (int e = 1; e < 4; e++) top[u] = fmaxf(fmaxf(top[u], c[u][0][e]), c[u][1][e]);
      grown |= !(top[u] - m_run[u] <= p.lazy);
    }
    if (__builtin_amdgcn_ballot_w64(grown)) {
      // some row's maximum has left its exponents' reference by more than kLazy: the row's four lanes follow together
#pragma unroll
      for (int u = 0; u < RT; u++) {
        float m = fmaxf(top[u], __shfl_xor(top[u], 16));
        m = fmaxf(m_run[u], fmaxf(m, __shfl_xor(m, 32)));
        const bool row = !(m - m_run[u] <= p.lazy);
        const float ms = m == -INFINITY ? 0.f : m;         // nothing seen so far: every exponent below is -inf
        const float alpha = row ? __builtin_amdgcn_exp2f((m_run[u] - ms) * p.scale_log2e) : 1.f;
        if (row) { m_run[u] = m; mc[u] = __builtin_fmaf(-ms, p.scale_log2e, -kLazy); }
        l_run[u] *= alpha;
#pragma unroll
        for (int dt = 0; dt < 8; dt++)
#pragma unroll
          for (int e = 0; e < 4; e++) oacc[u][dt][e] *= alpha;
      }
    }
#pragma unroll
    for (int u = 0; u < RT; u++)
#pragma unroll
      for (int hf = 0; hf < 2; hf++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float pv = __builtin_amdgcn_exp2f(__builtin_fmaf(c[u][hf][e], p.scale_log2e, mc[u]));
          const float first = __uint_as_float(__float_as_uint(pv) & 0xffff0000u);
          pf[u][hf * 4 + e] = (bf16_t)first;
          pl[u][hf * 4 + e] = (bf16_t)__builtin_amdgcn_fmed3f(pv - first, pv, 0x1p-126f);
          l_run[u] += pv;
        }
    if (more) wait_vmcnt<8>(); else wait_vmcnt<0>();     // V of unit i
    // Where some row does not see some key of the unit: rows of V that nobody sees become zero, whatever they hold, and non-finite
    // values of the others are taken out of the product (a zero weight times infinity is not zero) and added below where they are seen.
    unsigned long long odd = 0;
    if (masked) {
      const int row = lane >> 1, key = key0 + row;
      const bool seen = key < min(it.seq, key_end) && key > first_pos - reach && ((ok >> (row >> 4)) & 1);
      char* at = st + kUnitBytes / 2 + row * 256 + (lane & 1) * 128;
      bool any = false;
#pragma unroll
      for (int c16 = 0; c16 < 8; c16++) {
        u32x4 v = {0, 0, 0, 0};
        if (seen) v = finite_only(*(const u32x4*)(at + c16 * 16), &any);
        *(u32x4*)(at + c16 * 16) = v;
      }
      odd = __builtin_amdgcn_ballot_w64(any);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
#pragma unroll
    for (int dt = 0; dt < 8; dt++) {
      const short4_t lo = lds_read_tr(st + v_rd[dt]), hi = lds_read_tr(st + v_rd[dt] + 4096);
      const bf16x8 vf = __builtin_bit_cast(bf16x8, (short8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int u = 0; u < RT; u++) {
        oacc[u][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[u], oacc[u][dt], 0, 0, 0);
        oacc[u][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[u], oacc[u][dt], 0, 0, 0);
      }
    }
    while (odd) {   // (rare)
      const int r = __builtin_amdgcn_readfirstlane(__builtin_ctzll(odd)) >> 1;
      odd &= ~(3ull << (2 * r));
      const int key = key0 + r;
      const int pg = __builtin_amdgcn_readfirstlane(table[key >> g.page_shift]);
      const bf16_t* vrow = p.v_cache + (long)pg * g.page_stride + ((long)head * g.page + (key & (g.page - 1))) * kPagedD + gr * 4;
#pragma unroll
      for (int u = 0; u < RT; u++) {
        float mine = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++)
          if (e == (r >> 4) * 4 + (r & 3)) mine = (float)pf[u][e] + (float)pl[u][e];
        const float w = __shfl(mine, l15 + (((r >> 2) & 3) << 4));
        const bool sees = key <= pos[u] && key > pos[u] - reach;
#pragma unroll
        for (int dt = 0; dt < 8; dt++) {
          const bf16x4 v = *(const bf16x4*)(vrow + dt * 16);
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const float x = (float)v[e];
            if (sees && !(__builtin_fabsf(x) < INFINITY)) oacc[u][dt][e] += w * x;
          }
        }
      }
    }
    if (more) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      issue(p.v_cache, i + 1, false);
    }
  }

  // ---- join the waves: row maxima, then scaled rows, then their sums
  constexpr int ROWS = RT * 16, PITCH = kPagedD + 4, NP = NW / 2;      // half of the waves' rows at a time
  float* s_o = (float*)smem;                        // [NP][ROWS][PITCH]
  float* s_ml = s_o + NP * ROWS * PITCH;            // [NW][ROWS][2]
  static_assert((NP * ROWS * PITCH + NW * ROWS * 2 + 1) * 4 <= NW * kUnitBytes, "the join fits");
  __syncthreads();                                  // the units' places are no longer read
#pragma unroll
  for (int u = 0; u < RT; u++) {
    l_run[u] += __shfl_xor(l_run[u], 16);
    l_run[u] += __shfl_xor(l_run[u], 32);
    if (gr == 0) {
      s_ml[(wave * ROWS + u * 16 + l15) * 2] = m_run[u];
      s_ml[(wave * ROWS + u * 16 + l15) * 2 + 1] = l_run[u];
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < RT; u++) {
    const int row = u * 16 + l15;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; w++) m = fmaxf(m, s_ml[(w * ROWS + row) * 2]);
    const float f = __builtin_amdgcn_exp2f((m_run[u] - (m == -INFINITY ? 0.f : m)) * p.scale_log2e);
#pragma unroll
    for (int dt = 0; dt < 8; dt++)
#pragma unroll
      for (int e = 0; e < 4; e++) oacc[u][dt][e] *= f;
  }
  auto each_quad = [&](auto f) {                    // this wave's rows in LDS and in registers
#pragma unroll
    for (int u = 0; u < RT; u++)
#pragma unroll
      for (int dt = 0; dt < 8; dt++) f((floatx4*)(s_o + ((wave % NP) * ROWS + u * 16 + l15) * PITCH + dt * 16 + gr * 4), oacc[u][dt]);
  };
  if (wave >= NP) each_quad([](floatx4* at, floatx4& v) { *at = v; });      // the upper waves' rows, then onto the lower ones'
  __syncthreads();
  if (wave < NP)
    each_quad([](floatx4* at, floatx4& v) {
      const floatx4 o = *at;
#pragma unroll
      for (int e = 0; e < 4; e++) v[e] += o[e];
      *at = v;
    });
  __syncthreads();
  for (int i = tid; i < n_rows * 32; i += NW * 64) {
    const int row = i >> 5, d4 = (i & 31) * 4;
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; w++) m = fmaxf(m, s_ml[(w * ROWS + row) * 2]);
    const float ms = m == -INFINITY ? 0.f : m;
    floatx4 o = zero4;
#pragma unroll
    for (int w = 0; w < NW; w++) l += s_ml[(w * ROWS + row) * 2 + 1] * __builtin_amdgcn_exp2f((s_ml[(w * ROWS + row) * 2] - ms) * p.scale_log2e);
#pragma unroll
    for (int w = 0; w < NP; w++) {
      const floatx4 v = *(const floatx4*)(s_o + (w * ROWS + row) * PITCH + d4);
#pragma unroll
      for (int e = 0; e < 4; e++) o[e] += v[e];
    }
    if (it.runs == 1) store_out(p, it, head, row, d4, o, m, l);
    else {
      const long at = ((long)(it.slot + it.run) * g.Hk + head) * g.rows_few + row;
      store16_device_scope(p.part_few + at * kPagedD + d4, __builtin_bit_cast(u32x4, o));
      if (d4 == 0) store_ml(p.ml_few, at, m, l);
    }
  }
  if (it.runs == 1) return;
  // ---- join the runs: the last of every kJoin runs to arrive joins them, the last group to arrive joins the groups (of one group: the
  // runs go into the output at once).  Always in the order of the runs, so the result does not depend on who is last.
  // No acquire at device scope, which drops the whole L2 of the die under everybody's loads (32 requests of 2000 tokens in 8 runs each:
  // 28 us, 15 without).  It is not needed: parts and groups are written through, once a launch, to places of their own in whole cache
  // lines, and read after their arrival only, so no die can hold an older line of them; maxima and sums, which share lines, are read
  // past the L2.
  int* s_last = (int*)(s_ml + NW * ROWS * 2);
  const int groups = (it.runs + kJoin - 1) / kJoin;
#pragma unroll
  for (int level = 0; level < 2; level++) {
    const int first = level == 0 ? it.run & ~(kJoin - 1) : 0, stride = level == 0 ? 1 : kJoin;
    const int count = level == 0 ? min(kJoin, it.runs - first) : groups;
    const float *part = level == 0 ? p.part_few : p.group_few, *ml = level == 0 ? p.ml_few : p.group_ml;
    unsigned* cnt = p.arrived + ((long)(it.slot + first) * g.Hk + head) * 2 + level;
    wait_all_vmem();                                // this wave's part is where every die sees it
    __syncthreads();
    if (tid == 0) {
      const unsigned before = __hip_atomic_fetch_add(cnt, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      *s_last = before + 1 == (unsigned)count;
      if (*s_last) __hip_atomic_store(cnt, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!*s_last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    const bool whole = level == 1 || groups == 1;
    const long step = (long)g.Hk * g.rows_few * stride;
    for (int i = tid; i < n_rows * 32; i += NW * 64) {
      const int row = i >> 5, d4 = (i & 31) * 4;
      const long at = ((long)(it.slot + first) * g.Hk + head) * g.rows_few + row;
      floatx4 o = zero4;
      float m = -INFINITY, l = 0.f;
      for (int s = 0; s < count; s += kJoin) join_quad<kJoin, true>(part, ml, at + s * step, step, min(count - s, kJoin), d4, p.scale_log2e, &o, &m, &l);
      if (whole) store_out(p, it, head, row, d4, o, m, l);
      else {
        store16_device_scope(p.group_few + at * kPagedD + d4, __builtin_bit_cast(u32x4, o));
        if (d4 == 0) store_ml(p.group_ml, at, m, l);
      }
    }
    if (whole) return;
  }
}

// --------------------------------------------------------------------------------------
// Tiles of 256 rows (chunks of prompts): bound by the matrix products.  8 waves of 32 rows; blocks of 64 keys go through three LDS
// stages filled by direct-to-LDS loads; a lane owns one query row.  Scores of block b + 1 are computed while block b goes through
// the softmax, as in the sequence-parallel attention; here a block's rows come from up to four pages, looked up three blocks ahead.
// --------------------------------------------------------------------------------------
// The sums that the tile kernel's blocks left out: a non-finite value v of a key that only some of the tile's rows see.  Its weight is
// positive unless the score is -inf, so it adds itself, or NaN in that case.
__device__ __forceinline__ void add_non_finite(const PagedAttn& p, const Item& it, int head, const bf16x8 (&qf)[8], int q_pos, int reach, int key_lo, int key_end,
                                               int clean_lo, int clean_hi, floatx16 (&oacc)[4]) {
  const PagedGeom& g = p.g;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int* table = p.block_table + (long)it.b * g.max_blocks;
  for (int key = max(it.k0 * kBlk, key_lo); key < min(it.k1 * kBlk, key_end); key++) {
    const int pg = __builtin_amdgcn_readfirstlane(table[key >> g.page_shift]);
    if ((unsigned)pg >= (unsigned)g.n_pages) continue;
    const long at = (long)pg * g.page_stride + ((long)head * g.page + (key & (g.page - 1))) * kPagedD;
    const unsigned two = ((const unsigned*)(p.v_cache + at))[lane];
    if (!__builtin_amdgcn_ballot_w64(not_finite(two) || not_finite(two >> 16))) continue;
    const int blk = key & ~(kBlk - 1);
    bool masked = blk < clean_lo || blk + kBlk > clean_hi;
    for (int i = 0; i < kBlk && !masked; i += 16)      // (all before clean_hi: inside the table)
      masked = (unsigned)__builtin_amdgcn_readfirstlane(table[(blk + i) >> g.page_shift]) >= (unsigned)g.n_pages;
    if (!masked) continue;                             // its block was taken as it is
    float s = 0.f;
#pragma unroll
    for (int st = 0; st < 8; st++) {
      const bf16x8 k = *(const bf16x8*)(p.k_cache + at + st * 16 + h * 8);
#pragma unroll
      for (int e = 0; e < 8; e++) s += (float)k[e] * (float)qf[st][e];
    }
    float lo, hi;
    both_halves(s, lo, hi);
    s = lo + hi;
    const bool visible = key <= q_pos && key > q_pos - reach;
#pragma unroll
    for (int dt = 0; dt < 4; dt++)
#pragma unroll
      for (int q4 = 0; q4 < 4; q4++) {
        const bf16x4 v = *(const bf16x4*)(p.v_cache + at + dt * 32 + q4 * 8 + h * 4);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float x = (float)v[e];
          if (visible && !(__builtin_fabsf(x) < INFINITY)) oacc[dt][q4 * 4 + e] += s == -INFINITY ? __builtin_nanf("") : x;
        }
      }
  }
}

constexpr int kStageBytes = kBlk * kPagedD * 2;      // K or V rows of a block: 16 KiB
constexpr int kTileLds = 3 * 2 * kStageBytes;
constexpr int kTileThreads = 512;

__device__ __forceinline__ void tile_item(const PagedAttn& p, const Item& it, int head, char* smem) {
  __shared__ unsigned long long s_odd[8];      // per wave: met values that were not finite
  const PagedGeom& g = p.g;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first_pos = it.seq - it.n;
  const int reach = g.window ? g.window : 0x40000000;
  const int n_rows = it.n * g.G, row0 = it.tile * kTileRows;
  const int tile_t0 = (int)g.by_group.div((unsigned)row0), tile_t1 = min((int)g.by_group.div((unsigned)(row0 + kTileRows - 1)), it.n - 1);
  const int key_end = max(min(first_pos + tile_t1 + 1, it.seq), 0);        // keys that some row of the tile sees: [key_lo, key_end)
  const int key_lo = max(first_pos + tile_t0 - reach + 1, 0);
  const int clean_lo = max(first_pos + tile_t1 - reach + 1, 0), clean_hi = first_pos + tile_t0 + 1;   // ... that every row sees
  const int wrow0 = row0 + wave * 32;
  const bool active = wrow0 < n_rows;
  const int w_t0 = min((int)g.by_group.div((unsigned)wrow0), it.n - 1), w_t1 = min((int)g.by_group.div((unsigned)(wrow0 + 31)), it.n - 1);
  const int w_last = active ? first_pos + w_t1 : -1;            // last key of the wave's rows
  const int w_clean_lo = max(first_pos + w_t1 - reach + 1, 0), w_clean_hi = first_pos + w_t0 + 1;
  int hq_unused;
  const int q_pos = first_pos + token_of(g, min(wrow0 + l32, n_rows - 1), head, &hq_unused);

  // ---- pages of a block: lane l holds the page of its 16 keys number l % 4, or -1
  const int* table = p.block_table + (long)it.b * g.max_blocks;
  auto load_pages = [&](int blk) __attribute__((always_inline)) -> int {
    const int key = blk * kBlk + (lane & 3) * 16;
    return key < key_end ? table[key >> g.page_shift] : -1;
  };
  auto groups_valid = [&](int pg) __attribute__((always_inline)) -> int {
    return (int)__builtin_amdgcn_ballot_w64((unsigned)pg < (unsigned)g.n_pages) & 15;
  };
  // ---- stage loads: a wave-wide load is 4 rows of 256 bytes; wave w issues rows 4w.. and 32 + 4w.. of K and of V.
  // LDS slot (row, pc) holds 16-byte chunk pc ^ f(row): K: f = row % 16, V: f = (row % 4) << 2
  const int lr = lane >> 4, pc = lane & 15;
  const unsigned koff = (unsigned)(lr * 256 + ((pc ^ ((wave & 3) * 4 + lr)) << 4));
  const unsigned voff = (unsigned)(lr * 256 + ((pc ^ (lr << 2)) << 4));
  const unsigned smem_u = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem);
  auto issue_block = [&](int blk, int stage, int pg) __attribute__((always_inline)) {
    const unsigned sk = smem_u + (unsigned)__builtin_amdgcn_readfirstlane(stage) * (2 * kStageBytes);
#pragma unroll
    for (int i = 0; i < 2; i++) {
      int page = __builtin_amdgcn_readlane(pg, i * 2 + (wave >> 2));
      if ((unsigned)page >= (unsigned)g.n_pages) page = 0;       // no page: any will do, its keys are masked
      const int prow = (blk * kBlk + i * 32 + wave * 4) & (g.page - 1);
      const long at = (long)page * g.page_stride + ((long)head * g.page + prow) * kPagedD;
      const char* kb = (const char*)uniform64((unsigned long long)(p.k_cache + at));
      const char* vb = (const char*)uniform64((unsigned long long)(p.v_cache + at));
      const unsigned to = sk + (unsigned)(i * 8 + wave) * 1024;
      lds_load16_sbase(kb, koff, to);
      lds_load16_sbase(vb, voff, to + kStageBytes);
    }
  };
  // the wave's 32 Q rows, whole rows at a time, behind the first two stages; rows behind the request's last: that one
  const int q_lds = 2 * 2 * kStageBytes + wave * (32 * kPagedD * 2);
  auto issue_q = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 8; j++) {
      int hq;
      const int r = j * 4 + lr, token = token_of(g, min(wrow0 + r, n_rows - 1), head, &hq);
      lds_load16_at((const char*)(p.q + (long)(it.q0 + token) * p.q_stride + (long)hq * kPagedD) + ((pc ^ (r & 15)) << 4), smem_u + (unsigned)q_lds + j * 1024);
    }
  };

  // ---- per-lane LDS read offsets (as in the sequence-parallel attention)
  const int k_lane_off = l32 * 256 + ((h ^ (l32 & 15)) << 4);
  auto kread = [&](int kb, int i) __attribute__((always_inline)) -> bf16x8 {
    return *(const bf16x8*)(smem + (i & 1) * 32 * 256 + (kb ^ ((i >> 1) << 5)));
  };
  const int v_r = (lane & 15) >> 2;
  int v_off[4];
#pragma unroll
  for (int dt = 0; dt < 4; dt++) {
    const int col = dt * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    v_off[dt] = (v_r + 4 * h) * 256 + ((col >> 3) ^ (v_r << 2)) * 16 + (col & 4) * 2;
  }
  auto vread = [&](const char* sv, int j) __attribute__((always_inline)) -> bf16x8 {
    const char* pv = sv + (j >> 2) * 16 * 256 + v_off[j & 3];
    const short4_t lo = lds_read_tr(pv), hi = lds_read_tr(pv + 8 * 256);
    return __builtin_bit_cast(bf16x8, (short8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  bf16x8 qf[8];
  floatx16 zero16;
#pragma unroll
  for (int e = 0; e < 16; e++) zero16[e] = 0.f;
  floatx16 oacc[4];
#pragma unroll
  for (int dt = 0; dt < 4; dt++) oacc[dt] = zero16;
  float m_run = -INFINITY, l_run = 0.f, mc = 0.f, m_blk;

  auto block_max = [&](const floatx16 (&sc)[2]) __attribute__((always_inline)) -> float {
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; e++) m = raw_max(raw_max(m, sc[0][e]), sc[1][e]);
    return m;
  };
  auto sees = [&](int key) __attribute__((always_inline)) -> bool { return key <= q_pos && key > q_pos - reach; };

  int st_cur = 0, st_nxt = 1, st_ld = 2;
  int ok_cur = 15, ok_nxt = 15;      // valid groups of 16 keys of blocks blk, blk + 1
  int pg_ahead = -1;                 // pages of block blk + 2
  const int end = it.k1;
  unsigned long long odd = 0;        // lanes of this wave that took a non-finite value out of a block
  // some row of the tile does not see some key of the block
  auto masked_for_some = [&](int blk, int ok) __attribute__((always_inline)) -> bool {
    return blk * kBlk < clean_lo || blk * kBlk + kBlk > clean_hi || ok != 15;
  };

  auto block = [&](int blk, floatx16 (&c)[2], floatx16 (&n)[2]) __attribute__((always_inline)) {
    wait_vmcnt<0>();
    __syncthreads();
    int ok_ld = 15;
    if (blk + 2 < end) {
      ok_ld = groups_valid(pg_ahead);
      issue_block(blk + 2, st_ld, pg_ahead);
      pg_ahead = load_pages(blk + 3);
    }
    const int kv0 = blk * kBlk;
    char* sv = smem + st_cur * 2 * kStageBytes + kStageBytes;
    if (masked_for_some(blk, ok_cur)) {
      // rows of V that no row of the tile sees become zero, whatever they hold; non-finite values of the others are taken out of
      // the product (a zero weight times infinity is not zero) and added at the end where they are seen
      const int r = tid >> 3, key = kv0 + r;
      const bool seen = key < key_end && key >= key_lo && ((ok_cur >> (r >> 4)) & 1);
      char* at = sv + r * 256 + (tid & 7) * 32;
      bool any = false;
#pragma unroll
      for (int i = 0; i < 2; i++) {
        u32x4 v = {0, 0, 0, 0};
        if (seen) v = finite_only(*(const u32x4*)(at + i * 16), &any);
        *(u32x4*)(at + i * 16) = v;
      }
      odd |= __builtin_amdgcn_ballot_w64(any);
      __syncthreads();
    }
    if (kv0 <= w_last) {
      const int kb = st_nxt * 2 * kStageBytes + k_lane_off;
      constexpr int RD = 2, RN = RD + 1;
      bf16x8 fr[RN];
#pragma unroll
      for (int i = 0; i < RD; i++) fr[i] = kread(kb, i);
      __builtin_amdgcn_sched_barrier(0);
      const bool need_mask = kv0 < w_clean_lo || kv0 + kBlk > w_clean_hi || ok_cur != 15;
      if (need_mask) {
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
          for (int e = 0; e < 16; e++) {
            const int key = kv0 + t * 32 + (e >> 2) * 8 + h * 4 + (e & 3);
            if (!sees(key) || !((ok_cur >> (t * 2 + (e >> 3))) & 1)) c[t][e] = -INFINITY;
          }
        m_blk = block_max(c);
      }
      // The exponents' reference m_run follows the row's maximum only where that has left it by more than kLazy.  (It follows at once from
      // -inf, and the comparison is false for NaN.)
      if (__builtin_amdgcn_ballot_w64(!(m_blk - m_run <= p.lazy))) {
        const float m_new = fmaxf(m_run, halves_max(m_blk));   // (m_blk: of the lane's own half of the keys)
        const bool grown = !(m_new - m_run <= p.lazy);
        const float ms = m_new == -INFINITY ? 0.f : m_new;     // nothing seen so far: every exponent below is -inf
        const float alpha = grown ? __builtin_amdgcn_exp2f((m_run - ms) * p.scale_log2e) : 1.f;
        if (grown) { m_run = m_new; mc = __builtin_fmaf(-ms, p.scale_log2e, -kLazy); }
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < 4; dt++)
#pragma unroll
          for (int e = 0; e < 16; e++) oacc[dt][e] *= alpha;
      }
      // Weights rounded to bf16, once, as they enter the matrix instruction (their sum is of the unrounded ones): results are off by a third
      // more than their own rounding makes.  A second product with what the rounding of weights leaves would mend that, and take a prompt of 8192
      // tokens from 558 to 760 us, a chunk of 509 behind 31003 from 145 to 192.
      bf16x8 pf[4];
      float m_next = -INFINITY;
      static_for<0, 32>([&](auto s_c) {
        constexpr int f = decltype(s_c)::value;
        if constexpr (f + RD < 16) fr[(f + RD) % RN] = kread(kb, f + RD);
        else if constexpr (f + RD < 32) fr[(f + RD) % RN] = vread(sv, f + RD - 16);
        if constexpr (f < 16) {
          floatx16& acc = n[f & 1];
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[f % RN], qf[f >> 1], f < 2 ? zero16 : acc, 0, 0, 0);
        } else {
          constexpr int j = f - 16;
          oacc[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[f % RN], pf[j >> 2], oacc[j & 3], 0, 0, 0);
        }
        if constexpr (f >= 18 && f < 22) {
          constexpr int q = f - 18;
#pragma unroll
          for (int e = q * 4; e < q * 4 + 4; e++) m_next = raw_max3(m_next, n[0][e], n[1][e]);
        }
        static_for<0, 32>([&](auto y_c) {
          constexpr int y = decltype(y_c)::value;
          if constexpr (y * 7 / 8 == f) {
            constexpr int gq = y / 8, i = y % 8;
            const float pv = __builtin_amdgcn_exp2f(__builtin_fmaf(c[gq >> 1][(gq & 1) * 8 + i], p.scale_log2e, mc));
            pf[gq][i] = (bf16_t)pv;
            l_run += pv;
          }
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      m_blk = m_next;
    }
    const int st_free = st_cur;
    st_cur = st_nxt; st_nxt = st_ld; st_ld = st_free;
    ok_cur = ok_nxt; ok_nxt = ok_ld;
  };

  if (it.k0 < end) {
    const int p0 = load_pages(it.k0), p1 = load_pages(it.k0 + 1);
    pg_ahead = load_pages(it.k0 + 2);
    ok_cur = groups_valid(p0);
    issue_block(it.k0, 0, p0);
    if (it.k0 + 1 < end) {
      ok_nxt = groups_valid(p1);
      issue_block(it.k0 + 1, 1, p1);
    }
    issue_q();
    wait_vmcnt<0>();
#pragma unroll
    for (int st = 0; st < 8; st++) qf[st] = *(const bf16x8*)(smem + q_lds + (k_lane_off ^ (st << 5)));
    __syncthreads();
    floatx16 sa[2], sb[2];
#pragma unroll
    for (int i = 0; i < 16; i++)
      sa[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kread(k_lane_off, i), qf[i >> 1], i < 2 ? zero16 : sa[i & 1], 0, 0, 0);
    m_blk = block_max(sa);
    for (int blk = it.k0; blk < end; blk += 2) {
      block(blk, sa, sb);
      if (blk + 1 < end) block(blk + 1, sb, sa);
    }
  }

  // ---- (rare) the non-finite values that were taken out: each makes its column of every row that sees its key what the sum would be
  s_odd[wave] = odd;
  __syncthreads();
  odd = 0;
#pragma unroll
  for (int w = 0; w < 8; w++) odd |= uniform64(s_odd[w]);
  if (odd && active) add_non_finite(p, it, head, qf, q_pos, reach, key_lo, key_end, clean_lo, clean_hi, oacc);

  float l_lo, l_hi;
  both_halves(l_run, l_lo, l_hi);
  const float l = l_lo + l_hi;
  // ---- rows through LDS (the stages are free behind the barrier above), so that a wave stores whole rows: straight from the
  // accumulators, 16 bytes to a row at a time, an item's last 6 us were these stores.  LDS slot (row, c) holds 16-byte chunk c ^ (row % 16).
  if (!active) return;
  const int rows = min(n_rows - wrow0, 32);
  if (it.runs == 1) {
    char* to = smem + wave * (32 * kPagedD * 2);
    const float inv = row_scale(l);
#pragma unroll
    for (int dt = 0; dt < 4; dt++)
#pragma unroll
      for (int q4 = 0; q4 < 4; q4++) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = (bf16_t)(oacc[dt][q4 * 4 + e] * inv);
        *(bf16x4*)(to + l32 * 256 + (((dt * 4 + q4) ^ (l32 & 15)) << 4) + h * 8) = v;
      }
    if (p.lse && h == 0 && l32 < rows) {
      int hq;
      const int token = token_of(g, wrow0 + l32, head, &hq);
      p.lse[(long)(it.q0 + token) * g.Hq + hq] = log_sum(m_run, l, p.scale_log2e);
    }
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const int r = j * 4 + lr;
      if (r < rows) {
        int hq;
        const int token = token_of(g, wrow0 + r, head, &hq);
        *(u32x4*)(p.o + (long)(it.q0 + token) * p.o_stride + (long)hq * kPagedD + pc * 8) = *(const u32x4*)(to + r * 256 + ((pc ^ (r & 15)) << 4));
      }
    }
  } else {
    char* to = smem + wave * (32 * kPagedD * 4);
    const long at = ((long)(it.slot + it.run) * g.Hk + head) * g.rows_tile + wrow0 - row0;
#pragma unroll
    for (int dt = 0; dt < 4; dt++)
#pragma unroll
      for (int q4 = 0; q4 < 4; q4++) {
        const floatx4 v = {oacc[dt][q4 * 4], oacc[dt][q4 * 4 + 1], oacc[dt][q4 * 4 + 2], oacc[dt][q4 * 4 + 3]};
        *(floatx4*)(to + l32 * 512 + (((dt * 8 + q4 * 2 + h) ^ (l32 & 15)) << 4)) = v;
      }
    if (h == 0 && l32 < rows) { p.ml_tile[(at + l32) * 2] = m_run; p.ml_tile[(at + l32) * 2 + 1] = l; }
#pragma unroll
    for (int j = 0; j < 16; j++) {
      const int r = j * 2 + h;
      if (r < rows) *(floatx4*)(p.part_tile + (at + r) * kPagedD + l32 * 4) = *(const floatx4*)(to + r * 512 + ((l32 ^ (r & 15)) << 4));
    }
  }
}

// --------------------------------------------------------------------------------------
// Kernels.  A batch that can only have few rows per request (a decode step) takes the first; else one launch holds the items of both
// classes, so that single tokens run beside the chunks.
// --------------------------------------------------------------------------------------
static_assert(kTileLds <= kFewLds && 2 * 2 * kStageBytes + kTileRows * kPagedD * 2 <= kFewLds && kTileRows * kPagedD * 4 <= kFewLds, "one launch, one size");

template <int RT>
__global__ void __launch_bounds__(kFewWaves * 64) paged_few_rows_kernel(const PagedAttn p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const unsigned wg = workgroup_index();
  const int idx = wg / (unsigned)p.g.Hk, head = wg - idx * p.g.Hk;
  Item it;
  if (!sched_item(p.schedule, p.g, idx, &it)) return;
  few_rows_item<RT>(p, it, head, smem);
}

template <bool FEW>    // FEW: the batch may have few-row items
__global__ void __launch_bounds__(kTileThreads) paged_mixed_kernel(const PagedAttn p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const unsigned wg = workgroup_index();
  const int idx = wg / (unsigned)p.g.Hk, head = wg - idx * p.g.Hk;
  Item it;
  if (!sched_item(p.schedule, p.g, idx, &it)) return;
  if (!FEW || !it.few) tile_item(p, it, head, smem);
  else few_rows_item<2>(p, it, head, smem);
}

// Joins the runs of the cut tiles; all workgroups share them, where a tile's last run alone would read its partial results, 128 KiB a
// run, at one compute unit's pace.  A job is 8 rows of a tile and key head, a thread has one quad, and four runs at a time keep the
// registers few enough for eight workgroups a compute unit: a mixed batch with 23 cut tiles takes 5 us more in the whole call with 16 runs at a
// time and up to 64 rows a job.
constexpr int kTileJoin = 4, kJoinRows = 8;
__global__ void __launch_bounds__(256) paged_join_kernel(const PagedAttn p) {
  const PagedGeom& g = p.g;
  if (!sched_made_for(p.schedule, g)) return;
  const int parts = (g.rows_tile + kJoinRows - 1) / kJoinRows, jobs = p.schedule[2] * g.Hk * parts;
  const long step = (long)g.Hk * g.rows_tile;
  for (int job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int cut = job / (g.Hk * parts), rest = job - cut * g.Hk * parts, head = rest / parts;
    const Item it = load_item(p.schedule, g, p.schedule[kSchedHeader + cut]);
    const int row0 = it.tile * kTileRows, n = min(it.n * g.G - row0, kTileRows);
    const int r = (rest - head * parts) * kJoinRows + (threadIdx.x >> 5), d4 = (threadIdx.x & 31) * 4;
    if (r >= n) continue;
    const long at = ((long)it.slot * g.Hk + head) * g.rows_tile + r;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    for (int s = 0; s < it.runs; s += kTileJoin)
      join_quad<kTileJoin, false>(p.part_tile, p.ml_tile, at + s * step, step, min(it.runs - s, kTileJoin), d4, p.scale_log2e, &o, &m, &l);
    store_out(p, it, head, row0 + r, d4, o, m, l);
  }
}

// ======================================================================================
// Host side
// ======================================================================================
int resolve_paged(const tl_ctx* ctx, const tl_paged_dims* d, PagedGeom* g) {
  if (int e = check_ctx(ctx)) return e;
  if (!d) return fail(TL_ERR_INVALID_ARG, "dims must not be null");
  if (d->batch <= 0 || d->max_tokens <= 0 || d->max_blocks <= 0 || d->n_pages <= 0 || d->heads_q <= 0 || d->heads_kv <= 0)
    return fail(TL_ERR_INVALID_ARG, "tl_paged_dims: batch, max_tokens, max_blocks, n_pages and heads must be positive");
  if (d->max_new < 0 || d->max_new > d->max_tokens) return fail(TL_ERR_INVALID_ARG, "tl_paged_dims: max_new=%d outside [0, max_tokens=%d]", d->max_new, d->max_tokens);
  if (d->window < 0) return fail(TL_ERR_INVALID_ARG, "tl_paged_dims: window must not be negative");
  if (d->batch > kMaxBatch) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_dims: at most %d requests (batch=%d)", kMaxBatch, d->batch);
  if (d->max_tokens > 1 << 18) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_dims: at most %d new tokens (max_tokens=%d)", 1 << 18, d->max_tokens);
  if (d->head_dim != kPagedD) return fail(TL_ERR_UNSUPPORTED_SHAPE, "head_dim %d is not supported (128 only)", d->head_dim);
  if (d->page_size < 16 || d->page_size > 256 || (d->page_size & (d->page_size - 1)))
    return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_dims: page_size %d is not 16, 32, 64, 128 or 256", d->page_size);
  if (d->heads_q % d->heads_kv) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_dims: heads_kv=%d must divide heads_q=%d", d->heads_kv, d->heads_q);
  if (d->heads_q > 1024) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_dims: at most 1024 heads");
  if ((long)d->n_pages * d->page_size > 0x7fffffffL) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_dims: n_pages*page_size does not fit 32 bits");
  if ((long)d->max_blocks * d->page_size > 1L << 28) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_dims: a request may have at most 2^28 tokens");
  const long dense = (long)d->heads_kv * d->page_size * kPagedD;
  if (d->page_stride != 0 && d->page_stride < dense) return fail(TL_ERR_INVALID_ARG, "tl_paged_dims: page_stride is shorter than a page");
  if (d->page_stride % 8) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_dims: page_stride must be a multiple of 8 elements");
  memset(g, 0, sizeof *g);
  g->B = d->batch; g->T = d->max_tokens; g->max_new = d->max_new ? d->max_new : d->max_tokens; g->max_blocks = d->max_blocks;
  g->page = d->page_size; g->n_pages = d->n_pages; g->Hq = d->heads_q; g->Hk = d->heads_kv; g->G = d->heads_q / d->heads_kv;
  while ((1 << g->page_shift) < g->page) g->page_shift++;
  g->by_group = make_fast_div((unsigned)g->G);
  g->window = d->window < 1 << 29 ? d->window : 0;      // longer than any request: all of it
  g->page_stride = d->page_stride ? (long)d->page_stride : dense;
  // Classes.  A tile of the few-row class is a request with at most kFewRows rows; other requests make ceil(rows / kTileRows) tiles.
  const long most_rows = (long)g->max_new * g->G, all_rows = (long)g->T * g->G;
  g->rt = g->G > kFewRows ? 0 : (most_rows <= 16 ? 1 : 2);
  g->has_tiles = most_rows > (g->rt ? kFewRows : 0);
  // Runs.  A class's chunk is at least its blocks / side, so a tile of b > chunk blocks is cut into ceil(b / chunk) < 2 b / chunk runs:
  // all cut tiles together make less than 2 * side of them (there are fewer than `side`), and all tiles at most tiles + side items.
  const int cus = ctx->num_cus < 1024 ? ctx->num_cus : 1024;
  g->side = ceil_div(cus, g->Hk);
  g->sched_items = kSchedHeader + (g->side + 3) / 4 * 4;
  const long tiles = all_rows / kTileRows + (g->rt ? (g->B < all_rows / (kFewRows + 1) + 1 ? g->B : all_rows / (kFewRows + 1) + 1) : g->B);
  g->cap_few = g->rt ? g->B + g->side : 0;
  g->cap_tile = g->has_tiles ? (int)(tiles + g->side) : 0;
  g->rows_few = g->rt ? (int)(most_rows < kFewRows ? most_rows : kFewRows) : 0;
  g->rows_tile = g->has_tiles ? (int)(most_rows < kTileRows ? most_rows : kTileRows) : 0;
  if (((long)g->cap_tile + g->cap_few) * g->Hk > 0x7fffffffL)
    return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_dims: too many tiles for one launch");
  return TL_OK;
}

// Two counters per partial slot and key head: 2 * side * heads_kv of those, side = ceil(compute units / heads_kv).
constexpr size_t kArrivedBytes = 2 * (2 * (1024 + 1024)) * 4;

// Lets kernel number `which` of this file use `bytes` of dynamic LDS on `device`; asked of the runtime once (it takes a microsecond a call).
static int allow_lds(const void* kernel, int which, int device, int bytes) {
  static std::atomic<unsigned long long> done[4];
  const unsigned long long bit = 1ull << (device & 63);
  if (device < 64 && (done[which].load(std::memory_order_acquire) & bit)) return TL_OK;
  TL_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (device < 64) done[which].fetch_or(bit, std::memory_order_release);
  return TL_OK;
}

struct PagedSizes { size_t schedule, ws, part_few, ml_few, group_few, group_ml, part_tile, ml_tile; };

static PagedSizes paged_sizes(const PagedGeom& g) {
  PagedSizes s;
  s.schedule = ((size_t)g.sched_items + ((size_t)g.cap_few + g.cap_tile) * kItemInts) * 4;
  const size_t few = (size_t)2 * g.side * g.Hk * g.rows_few, tile = (size_t)2 * g.side * g.Hk * g.rows_tile;   // partial rows
  s.part_few = kArrivedBytes;             // (in front: the arrival counters, the same for all dims, so that calls of any may share a workspace)
  s.ml_few = s.part_few + few * kPagedD * 4;
  s.group_few = s.ml_few + (few * 8 + 255) / 256 * 256;
  s.group_ml = s.group_few + few * kPagedD * 4;
  s.part_tile = s.group_ml + (few * 8 + 255) / 256 * 256;
  s.ml_tile = s.part_tile + tile * kPagedD * 4;
  s.ws = s.ml_tile + (tile * 8 + 255) / 256 * 256;
  return s;
}

}  // namespace tl

using namespace tl;

extern "C" {

int tl_paged_query(const tl_ctx* ctx, const tl_paged_dims* dims, size_t* schedule_bytes, size_t* ws_bytes, int* info) {
  PagedGeom g;
  if (int e = resolve_paged(ctx, dims, &g)) return e;
  if (!schedule_bytes || !ws_bytes || !info) return fail(TL_ERR_INVALID_ARG, "tl_paged_query: null pointer argument");
  const PagedSizes s = paged_sizes(g);
  *schedule_bytes = s.schedule;
  *ws_bytes = s.ws;
  const int v[8] = {kTileRows, g.rt ? kFewRows : 0, kBlk, g.cap_few, g.cap_tile, g.side, kMinChunk, g.G};
  memcpy(info, v, sizeof v);
  return TL_OK;
}

int tl_paged_slots(tl_ctx* ctx, const tl_paged_dims* dims, const int* ctx_lens, const int* new_lens, const int* free_pages, int n_free, const int* free_from,
                   int* free_to, int* block_table, int* query_start, int* seq_lens, int* slots, int* positions, int* counts, void* stream) {
  PagedGeom g;
  if (int e = resolve_paged(ctx, dims, &g)) return e;
  if (!ctx_lens || !new_lens || !block_table || !query_start || !seq_lens || !slots || !positions || !counts || (n_free > 0 && !free_pages))
    return fail(TL_ERR_INVALID_ARG, "tl_paged_slots: null pointer argument");
  if (n_free < 0) return fail(TL_ERR_INVALID_ARG, "tl_paged_slots: n_free must not be negative");
  const void* ptrs[] = {ctx_lens, new_lens, free_pages, free_from, free_to, block_table, query_start, seq_lens, slots, positions, counts};
  for (const void* q : ptrs)
    if (!aligned4(q)) return fail(TL_ERR_INVALID_ARG, "tl_paged_slots: device pointers must be 4-byte aligned");
  if (int e = check_paged_launch(ctx, "tl_paged_slots")) return e;
  const SlotsParams p = {ctx_lens, new_lens, free_pages, free_from, n_free, free_to, block_table, query_start, seq_lens, slots, positions, counts,
                         g.B, g.T, g.max_new, g.max_blocks, g.page, g.page_shift, g.n_pages};
  hipStream_t s = (hipStream_t)stream;
  const bool in_place = seq_lens == ctx_lens || (free_to && free_to == free_from);
  if (g.B <= 64 && g.T <= 256) hipLaunchKernelGGL((paged_slots_kernel<kMaps | kLengths, 64>), dim3(1), dim3(64), 0, s, p);
  else {
    const int wgs = ceil_div(g.T, 1024);
    if (wgs == 1 || !in_place) hipLaunchKernelGGL((paged_slots_kernel<kMaps | kLengths, 1024>), dim3(wgs), dim3(1024), 0, s, p);
    else {
      hipLaunchKernelGGL((paged_slots_kernel<kMaps, 1024>), dim3(wgs), dim3(1024), 0, s, p);
      hipLaunchKernelGGL((paged_slots_kernel<kLengths, 1024>), dim3(1), dim3(1024), 0, s, p);
    }
  }
  TL_HIP(hipGetLastError());
  return TL_OK;
}

int tl_paged_schedule(tl_ctx* ctx, const tl_paged_dims* dims, const int* query_start, const int* seq_lens, int* schedule, size_t schedule_bytes, void* stream) {
  PagedGeom g;
  if (int e = resolve_paged(ctx, dims, &g)) return e;
  if (!query_start || !seq_lens || !schedule) return fail(TL_ERR_INVALID_ARG, "tl_paged_schedule: null pointer argument");
  if (!aligned4(query_start) || !aligned4(seq_lens) || !aligned16(schedule))
    return fail(TL_ERR_INVALID_ARG, "tl_paged_schedule: schedule must be 16-byte aligned, the lengths 4-byte aligned");
  const PagedSizes z = paged_sizes(g);
  if (schedule_bytes < z.schedule) return fail(TL_ERR_WORKSPACE_TOO_SMALL, "tl_paged_schedule: schedule of %zu bytes, %zu needed", schedule_bytes, z.schedule);
  if (int e = check_paged_launch(ctx, "tl_paged_schedule")) return e;
  const SchedParams p = {query_start, seq_lens, schedule, g};
  // tiles of both classes at most: up to 64 in one wave (B = 64: 6.3 us against 7.3 with four), up to 256 in four (8 prompt chunks and 40 single tokens:
  // 8.6 against 12.2 with one and 9.7 with sixteen), more in sixteen (1000 requests: 10.9 against 16.1 with four)
  const int most = g.B + (g.has_tiles ? g.cap_tile - g.side : 0);
  auto launch = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    hipLaunchKernelGGL(paged_schedule_kernel<NT>, dim3(1), dim3(NT), 0, (hipStream_t)stream, p);
  };
  if (most <= 64) launch(std::integral_constant<int, 64>{});
  else if (most <= 256) launch(std::integral_constant<int, 256>{});
  else launch(std::integral_constant<int, 1024>{});
  TL_HIP(hipGetLastError());
  return TL_OK;
}

int tl_paged_attention(tl_ctx* ctx, const tl_paged_dims* dims, const void* q, long long q_stride, const void* k_cache, const void* v_cache,
                       const int* block_table, const int* schedule, void* o, long long o_stride, float* lse, float scale, void* workspace, size_t ws_bytes,
                       void* stream) {
  PagedGeom g;
  if (int e = resolve_paged(ctx, dims, &g)) return e;
  if (!q || !k_cache || !v_cache || !block_table || !schedule || !o || !workspace) return fail(TL_ERR_INVALID_ARG, "tl_paged_attention: null pointer argument");
  if (!(scale > 0.f) || !(scale * 1.4426950408889634f < __builtin_inff())) return fail(TL_ERR_INVALID_ARG, "tl_paged_attention: scale must be positive and finite");
  if (q_stride < (long long)g.Hq * kPagedD || o_stride < (long long)g.Hq * kPagedD)
    return fail(TL_ERR_INVALID_ARG, "tl_paged_attention: a row stride is shorter than the row's heads");
  if (q_stride % 8 || o_stride % 8) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_paged_attention: row strides must be multiples of 8 elements");
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o) || !aligned16(schedule))
    return fail(TL_ERR_INVALID_ARG, "tl_paged_attention: device pointers must be 16-byte aligned");
  if (!aligned128(workspace)) return fail(TL_ERR_INVALID_ARG, "tl_paged_attention: workspace must be 128-byte aligned");
  if (!aligned4(block_table) || !aligned4(lse)) return fail(TL_ERR_INVALID_ARG, "tl_paged_attention: block_table and lse must be 4-byte aligned");
  const PagedSizes z = paged_sizes(g);
  if (ws_bytes < z.ws) return fail(TL_ERR_WORKSPACE_TOO_SMALL, "tl_paged_attention: workspace of %zu bytes, %zu needed", ws_bytes, z.ws);
  if (int e = check_paged_launch(ctx, "tl_paged_attention")) return e;
  PagedAttn p;
  memset(&p, 0, sizeof p);
  p.g = g;
  p.q = (const bf16_t*)q; p.k_cache = (const bf16_t*)k_cache; p.v_cache = (const bf16_t*)v_cache;
  p.block_table = block_table; p.schedule = schedule;
  p.o = (bf16_t*)o; p.lse = lse;
  p.q_stride = q_stride; p.o_stride = o_stride;
  p.scale_log2e = scale * 1.4426950408889634f;
  p.lazy = kLazy / p.scale_log2e < 3.0e38f ? kLazy / p.scale_log2e : 3.0e38f;
  char* ws = (char*)workspace;
  p.arrived = (unsigned*)ws;
  p.part_few = (float*)(ws + z.part_few); p.ml_few = (float*)(ws + z.ml_few);
  p.group_few = (float*)(ws + z.group_few); p.group_ml = (float*)(ws + z.group_ml);
  p.part_tile = (float*)(ws + z.part_tile); p.ml_tile = (float*)(ws + z.ml_tile);
  hipStream_t s = (hipStream_t)stream;
  auto launch = [&](auto kernel, int which, long grid, int threads, int lds) -> int {
    if (int e = allow_lds((const void*)kernel, which, ctx->device, lds)) return e;
    hipLaunchKernelGGL(kernel, grid_of(grid), dim3(threads), lds, s, p);
    TL_HIP(hipGetLastError());
    return TL_OK;
  };
  if (!g.has_tiles) return launch(g.rt == 1 ? paged_few_rows_kernel<1> : paged_few_rows_kernel<2>, g.rt == 1 ? 0 : 1, (long)g.cap_few * g.Hk, kFewWaves * 64, kFewLds);
  if (int e = launch(g.rt ? paged_mixed_kernel<true> : paged_mixed_kernel<false>, g.rt ? 2 : 3, ((long)g.cap_tile + g.cap_few) * g.Hk, kTileThreads, kFewLds)) return e;
  hipLaunchKernelGGL(paged_join_kernel, dim3(8 * ctx->num_cus), dim3(256), 0, s, p);
  TL_HIP(hipGetLastError());
  return TL_OK;
}

}  // extern "C"
