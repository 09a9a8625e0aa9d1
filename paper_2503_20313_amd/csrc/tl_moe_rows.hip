// A mixture-of-experts layer in training, everything but the products: rows sorted by expert and their places, token rows into that
// order and back with weights applied, the gradients of both, and the gradient of the routing weights.  gfx950 only.
//
// Row (t, j), number t*topk + j, is token t at its j-th expert; row_pos[t, j] is its place in the matrices whose rows are sorted by
// expert.  A place outside [0, max_rows) takes no part, and nothing is read or written for it: whatever row_pos holds, every
// access stays inside the matrices.
#include "tl_moe_choice.h"

namespace tl {

// Sum over the 64 lanes of a wave, in every lane, always in the same order.
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
  return x;
}

// ======================================================================================
// Rows sorted by expert (stable), and the place of every row.  A chunk of consecutive rows is a workgroup's: it counts its rows of
// every expert, adds up what stands before them -- all rows of the experts before, and the rows of the chunks before with the
// same expert -- and places them.  One chunk: one launch.  Several: the counts of all chunks are left in the workspace by a launch
// of their own, and every workgroup adds them up for itself.
// Inside a chunk wave w owns a run of 64*RPT rows and walks it 64 rows at a time; the lanes with the same expert are found with one
// ballot per bit of the expert's number, which gives every row its rank among them.
// ======================================================================================
struct SortParams {
  const int* ids;
  int n, first, E;
  int *offsets, *sorted_row, *row_pos;
  int* hist;           // [chunks][E]
  int chunks;
};

__device__ __forceinline__ unsigned long long lanes_alike(int e, bool valid, int bits) {
  unsigned long long same = __builtin_amdgcn_ballot_w64(valid);
  for (int b = 0; b < bits; b++) {
    const unsigned long long bal = __builtin_amdgcn_ballot_w64(valid && ((e >> b) & 1));
    same &= ((e >> b) & 1) ? bal : ~bal;
  }
  return same;
}

// A row's expert among ours, or -1.
__device__ __forceinline__ int own_expert(const SortParams& p, int r) {
  if (r >= p.n) return -1;
  const unsigned e = (unsigned)p.ids[r] - (unsigned)p.first;
  return e < (unsigned)p.E ? (int)e : -1;
}

template <int RPT>
__global__ void __launch_bounds__(kSortThreads) moe_count_kernel(const SortParams p) {
  __shared__ int s_cnt[kMaxSortExperts];
  const int tid = threadIdx.x;
  if (tid < kMaxSortExperts) s_cnt[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < RPT; u++) {
    const int e = own_expert(p, (blockIdx.x * RPT + u) * kSortThreads + tid);
    if (e >= 0) atomicAdd(&s_cnt[e], 1);
  }
  __syncthreads();
  if (tid < p.E) p.hist[(long)blockIdx.x * p.E + tid] = s_cnt[tid];
}

template <int RPT, bool ONE>       // ONE: this is the only chunk (RPT is 1 then)
__global__ void __launch_bounds__(kSortThreads) moe_place_kernel(const SortParams p) {
  __shared__ int s_cnt[kSortWaves][kMaxSortExperts];
  __shared__ int s_sum[2][kSortThreads];     // rows of an expert in the chunks before this one, and in all: by groups of chunks
  __shared__ int s_base[kMaxSortExperts], s_scan[kMaxSortExperts];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bits = 32 - __builtin_clz(max(p.E - 1, 1));
  const unsigned long long below = (1ull << lane) - 1;
  const int lo = blockIdx.x * (kSortThreads * RPT) + wave * (64 * RPT);
  for (int i = tid; i < kSortWaves * kMaxSortExperts; i += kSortThreads) (&s_cnt[0][0])[i] = 0;
  int e[RPT];
#pragma unroll
  for (int u = 0; u < RPT; u++) e[u] = own_expert(p, lo + u * 64 + lane);
  const int room = 1 << bits;                // experts, up to a power of two
  if constexpr (!ONE) {
    // thread (g, x): chunks g, g + groups, .. of expert x, eight at a time in flight
    const int x = tid & (room - 1), g = tid >> bits, groups = kSortThreads >> bits;
    int before = 0, all = 0;
    if (x < p.E)
      for (int c0 = g; c0 < p.chunks; c0 += 8 * groups) {
        int v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = c0 + i * groups < p.chunks ? p.hist[(long)(c0 + i * groups) * p.E + x] : 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
          all += v[i];
          if (c0 + i * groups < (int)blockIdx.x) before += v[i];
        }
      }
    // the wave's lanes of one expert, then (below) the waves: 131000 rows of 2 experts 30.0 us with one thread an expert adding all up
    for (int d = 32; d >= room; d >>= 1) {
      before += __shfl_xor(before, d);
      all += __shfl_xor(all, d);
    }
    s_sum[0][tid] = before;
    s_sum[1][tid] = all;
  }
  __syncthreads();
  // ---- rank of every row among the wave's rows of its expert
  int rank[RPT];
#pragma unroll
  for (int u = 0; u < RPT; u++) {
    const bool valid = e[u] >= 0;
    const unsigned long long same = lanes_alike(e[u], valid, bits);
    int start = 0;
    if (valid) start = s_cnt[wave][e[u]];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // (the counts pass between the lanes of this wave)
    if (valid && (same & below) == 0) s_cnt[wave][e[u]] = start + __builtin_popcountll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    rank[u] = start + __builtin_popcountll(same & below);
  }
  __syncthreads();
  // ---- where the chunk's rows of every expert start, and each wave's among them
  if (tid < kMaxSortExperts) {
    int run = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; w++) {
      const int c = s_cnt[w][tid];
      s_cnt[w][tid] = run;
      run += c;
    }
    int before = 0, all = run;
    if constexpr (!ONE) {
      all = 0;
      if (tid < room)
        for (int g = tid; g < kSortThreads; g += max(room, 64)) { before += s_sum[0][g]; all += s_sum[1][g]; }
    }
    int scan = all;      // inclusive, over the wave's 64 experts
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(scan, d);
      if (lane >= d) scan += o;
    }
    s_scan[tid] = scan;
    s_base[tid] = scan - all + before;
  }
  __syncthreads();
  if (tid < kMaxSortExperts) {
    int start = 0;       // all rows of the experts of the waves before
    for (int w = 0; w < wave; w++) start += s_scan[w * 64 + 63];
    s_base[tid] += start;
    if (blockIdx.x == 0 && tid < p.E) {
      p.offsets[tid + 1] = start + s_scan[tid];
      if (tid == 0) p.offsets[0] = 0;
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < RPT; u++) {
    const int r = lo + u * 64 + lane;
    if (r >= p.n) continue;
    int pos = -1;
    if (e[u] >= 0) {
      pos = s_base[e[u]] + s_cnt[wave][e[u]] + rank[u];
      p.sorted_row[pos] = r;
    }
    p.row_pos[r] = pos;
  }
}

// ======================================================================================
// Rows of tokens <-> rows sorted by expert.  Bound by memory: every row is read or written once, a wave to 1 KiB of a row (of 2 or 4 KiB: the
// same within 3 %).  Matrices larger than the caches are read and written as streaming: 8192 tokens of 4096, top-5, dispatched in 78.7 us without, 63.5 with
// (6.3 TB/s), combined 91.8 and 73.7, their gradients 148 and 134 us (5.5 TB/s, reads and writes in equal parts).  Smaller ones
// are not: their rows may still be there from the product before, or be there for the one behind (1024 tokens, top-8, gradients of
// combine: 24.4 us, with streaming loads 30.9).
// ======================================================================================
template <bool STREAM>
__device__ __forceinline__ u32x4 load_piece(const u32x4* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p); else return *p;
}
template <bool STREAM>
__device__ __forceinline__ void store_piece(u32x4* p, u32x4 v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, p); else *p = v;
}

struct RowsParams {
  const bf16_t *x, *ys, *add;      // token rows; sorted rows; token rows or null
  const float* w;
  const int* row_pos;
  bf16_t *out, *dys;
  float* dw;
  long T;
  int H8, topk, max_rows;          // H8: 16-byte pieces of a row
  int segs;                        // pieces of a row that waves share
};

// Token t's places, lane j the j-th, and which of them take part.
__device__ __forceinline__ unsigned long long places_of(const RowsParams& p, long t, int lane, int* pos) {
  *pos = lane < p.topk ? p.row_pos[t * p.topk + lane] : -1;
  return __builtin_amdgcn_ballot_w64((unsigned)*pos < (unsigned)p.max_rows);
}

template <bool STREAM>
__global__ void __launch_bounds__(256) moe_dispatch_kernel(const RowsParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long items = p.T * p.segs;
  for (long it = (long)blockIdx.x * 4 + wave; it < items; it += (long)gridDim.x * 4) {
    const long t = it / p.segs;
    const int c = (int)(it - t * p.segs) * 64 + lane;
    int pos;
    unsigned long long part = places_of(p, t, lane, &pos);
    if (!part || c >= p.H8) continue;
    const u32x4 v = ((const u32x4*)p.x)[t * p.H8 + c];
    while (part) {
      const int j = __builtin_ctzll(part);
      part &= part - 1;
      store_piece<STREAM>((u32x4*)p.out + (long)__builtin_amdgcn_readlane(pos, j) * p.H8 + c, v);
    }
  }
}

// out[t] = (add[t] +) sum over j, in their order, of (w[t, j]) ys[row_pos[t, j]]; one rounding.
template <bool WEIGHTED, bool STREAM>
__global__ void __launch_bounds__(256) moe_gather_sum_kernel(const RowsParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long items = p.T * p.segs;
  for (long it = (long)blockIdx.x * 4 + wave; it < items; it += (long)gridDim.x * 4) {
    const long t = it / p.segs;
    const int c = (int)(it - t * p.segs) * 64 + lane;
    int pos;
    unsigned long long part = places_of(p, t, lane, &pos);
    float w = 0.f;
    if (WEIGHTED && lane < p.topk) w = p.w[t * p.topk + lane];
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; e++) acc[e] = 0.f;
    const bool in = c < p.H8;
    if (WEIGHTED && p.add && in) acc_bf16x8(acc, ((const u32x4*)p.add)[t * p.H8 + c]);
    // four rows at a time, their loads in flight together
    while (part) {
      u32x4 v[4];
      float wj[4];
#pragma unroll
      for (int q = 0; q < 4; q++) {
        v[q] = u32x4{0, 0, 0, 0};
        wj[q] = 0.f;
        if (part) {
          const int j = __builtin_ctzll(part);
          part &= part - 1;
          if (WEIGHTED) wj[q] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j));
          if (in) v[q] = load_piece<STREAM>((const u32x4*)p.ys + (long)__builtin_amdgcn_readlane(pos, j) * p.H8 + c);
        }
      }
#pragma unroll
      for (int q = 0; q < 4; q++) {
        if constexpr (WEIGHTED) {
#pragma unroll
          for (int e = 0; e < 4; e++) {
            acc[2 * e] = __builtin_fmaf(wj[q], __uint_as_float(v[q][e] << 16), acc[2 * e]);
            acc[2 * e + 1] = __builtin_fmaf(wj[q], __uint_as_float(v[q][e] & 0xffff0000u), acc[2 * e + 1]);
          }
        } else {
          acc_bf16x8(acc, v[q]);
        }
      }
    }
    if (in) store_piece<STREAM>((u32x4*)p.out + t * p.H8 + c, pack_bf16x8(acc));
  }
}

// dys[row_pos[t, j]] = w[t, j] dout[t], dw[t, j] = <dout[t], ys[row_pos[t, j]]>.  WAVES waves take a token, two rows of it at a time, their loads
// in flight together (8192 tokens of 4096, top-5, 131 us, one row 134, four 132; one token of 7640, top-8, 12.0, 14.3 and 14.6); a row of ys is read before its place
// is written, by the same lane, so dys may be ys.  Lane j of a wave keeps its share of dw[t, j].  (68
// registers, seven waves a SIMD; held to 64, eight are spilled: 135 us.)
template <int WAVES, bool STREAM_LOADS, bool STREAM_STORES>
__global__ void __launch_bounds__(256) moe_combine_grad_kernel(const RowsParams p) {
  constexpr int U = 2, R = 2, STEP = 64 * WAVES;
  __shared__ float s_dot[4][kMaxChoices];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = wave % WAVES;
  for (long t = (long)blockIdx.x * (4 / WAVES) + wave / WAVES; t < p.T; t += (long)gridDim.x * (4 / WAVES)) {
    int pos;
    const unsigned long long part = places_of(p, t, lane, &pos);
    float w = 0.f, mine = 0.f;
    if (lane < p.topk) w = p.w[t * p.topk + lane];
    const u32x4* src = (const u32x4*)p.x + t * p.H8;
    for (int c0 = share * 64 + lane; c0 - lane < p.H8; c0 += STEP * U) {
      u32x4 g[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        g[u] = u32x4{0, 0, 0, 0};
        if (c0 + u * STEP < p.H8) g[u] = src[c0 + u * STEP];
      }
      for (unsigned long long left = part; left;) {
        u32x4 v[R][U];
        long row[R];
        int j[R];
        float wj[R];
#pragma unroll
        for (int q = 0; q < R; q++) {
          j[q] = -1;
          if (!left) continue;
          j[q] = __builtin_ctzll(left);
          left &= left - 1;
          row[q] = (long)__builtin_amdgcn_readlane(pos, j[q]) * p.H8;
          wj[q] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j[q]));
#pragma unroll
          for (int u = 0; u < U; u++) {
            v[q][u] = u32x4{0, 0, 0, 0};
            if (c0 + u * STEP < p.H8) v[q][u] = load_piece<STREAM_LOADS>((const u32x4*)p.ys + row[q] + c0 + u * STEP);
          }
        }
#pragma unroll
        for (int q = 0; q < R; q++) {
          if (j[q] < 0) continue;
          float dot = 0.f;
#pragma unroll
          for (int u = 0; u < U; u++) {
            float o[8];
#pragma unroll
            for (int e = 0; e < 4; e++) {
              const float g0 = __uint_as_float(g[u][e] << 16), g1 = __uint_as_float(g[u][e] & 0xffff0000u);
              dot = __builtin_fmaf(g0, __uint_as_float(v[q][u][e] << 16), dot);
              dot = __builtin_fmaf(g1, __uint_as_float(v[q][u][e] & 0xffff0000u), dot);
              o[2 * e] = wj[q] * g0;
              o[2 * e + 1] = wj[q] * g1;
            }
            if (c0 + u * STEP < p.H8) store_piece<STREAM_STORES>((u32x4*)p.dys + row[q] + c0 + u * STEP, pack_bf16x8(o));
          }
          dot = wave_sum(dot);
          if (lane == j[q]) mine += dot;
        }
      }
    }
    if constexpr (WAVES == 1) {
      if (lane < p.topk) p.dw[t * p.topk + lane] = mine;
    } else {
      static_assert(WAVES == 4, "a workgroup to a token");
      if (lane < kMaxChoices) s_dot[wave][lane] = mine;
      __syncthreads();
      if (threadIdx.x < (unsigned)p.topk) p.dw[t * p.topk + threadIdx.x] = s_dot[0][threadIdx.x] + s_dot[1][threadIdx.x] + s_dot[2][threadIdx.x] + s_dot[3][threadIdx.x];
      __syncthreads();
    }
  }
}

// ======================================================================================
// Gradient of the routing weights with respect to the logits.  With p = softmax(logits) and e_j the chosen experts:
//   w_j = p_{e_j}:                     dl_i = p_i (sum_{j: e_j = i} dw_j - sum_k p_{e_k} dw_k)
//   w_j = p_{e_j} / sum_k p_{e_k}:     dl_i = sum_{j: e_j = i} w_j (dw_j - sum_k w_k dw_k),  w the softmax over the chosen logits
// LANES lanes hold a token's logits, PER each, and one choice each: as few as hold the choices, for the reductions over them are what the
// time goes into (16384 tokens, 64 experts, top-8: 9.7 us with 64 lanes of one logit, 5.8 with 16 of four).  Everything is fp32: the exponentials are of differences to the
// largest logit, the sums of at most 256 terms.  Masks (-inf) are left out of the sums and products,
// for 0 times an infinity is NaN: a masked choice's dw reaches nobody, and what the others are does not reach a masked logit.
// ======================================================================================
struct RouteGradParams {
  const float *logits, *dw;
  const int* ids;
  float* dlogits;
  long T;
  int E, topk, renormalize;
};

template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) x += __shfl_xor(x, d);
  return x;
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float x) {
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}

template <int LANES, int PER>
__global__ void __launch_bounds__(256) moe_route_grad_kernel(const RouteGradParams p) {
  const int i = threadIdx.x % LANES, lane0 = (threadIdx.x & 63) - i;
  const long t = (long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const bool real = t < p.T;
  const long tr = real ? t : p.T - 1;
  float l[PER];
#pragma unroll
  for (int q = 0; q < PER; q++) l[q] = i + q * LANES < p.E ? p.logits[tr * p.E + i + q * LANES] : -INFINITY;
  int id = -1;
  float g = 0.f;
  if (i < p.topk) {
    id = p.ids[tr * p.topk + i];
    if ((unsigned)id < (unsigned)p.E) g = p.dw[tr * p.topk + i]; else id = -1;
  }
  // the logit of this lane's choice
  float chosen = -INFINITY;
#pragma unroll
  for (int q = 0; q < PER; q++) {
    const float v = __shfl(l[q], lane0 + (id < 0 ? 0 : id % LANES));
    if (id >= 0 && id / LANES == q) chosen = v;
  }
  float top;
  if (p.renormalize) top = lanes_max<LANES>(chosen);
  else {
    top = l[0];
#pragma unroll
    for (int q = 1; q < PER; q++) top = fmaxf(top, l[q]);
    top = lanes_max<LANES>(top);
  }
  if (top == -INFINITY) top = 0.f;             // (nothing but masks, and NaN, which a maximum passes over: exponentials of 0 and NaN)
  float e[PER], sum = 0.f;
#pragma unroll
  for (int q = 0; q < PER; q++) {
    e[q] = expf(l[q] - top);
    sum += e[q];
  }
  const float mine = id >= 0 ? expf(chosen - top) : 0.f;
  sum = lanes_sum<LANES>(p.renormalize ? mine : sum);
  const float w = mine / sum;
  const float mean = lanes_sum<LANES>(chosen == -INFINITY ? 0.f : w * g);
  float a = p.renormalize ? w * (g - mean) : g;           // what choice i adds to its expert
  if (chosen == -INFINITY) a = 0.f;
  float d[PER];
#pragma unroll
  for (int q = 0; q < PER; q++) d[q] = 0.f;
  for (int j = 0; j < p.topk; j++) {
    const int ej = __shfl(id, lane0 + j);
    const float aj = __shfl(a, lane0 + j);
#pragma unroll
    for (int q = 0; q < PER; q++)
      if (ej == i + q * LANES) d[q] += aj;
  }
#pragma unroll
  for (int q = 0; q < PER; q++)
    if (real && i + q * LANES < p.E) {
      float v = d[q];
      if (!p.renormalize) v = e[q] == 0.f ? 0.f : e[q] / sum * (v - mean);      // (zero for a mask, whatever the others are)
      p.dlogits[t * p.E + i + q * LANES] = v;
    }
}

// ======================================================================================
// Host side
// ======================================================================================
static bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

static int check_tokens(const char* what, int T, int topk) {
  if (T <= 0 || topk <= 0) return fail(TL_ERR_INVALID_ARG, "%s: T and topk must be positive", what);
  if (topk > kMaxChoices) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: topk=%d is more than %d", what, topk, kMaxChoices);
  if ((long)T * topk >= (1L << 31)) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: T*topk must fit 31 bits", what);
  return TL_OK;
}

static int check_rows(const char* what, const void* sorted, const int* row_pos, int T, int H, int topk, int max_rows) {
  if (int e = check_tokens(what, T, topk)) return e;
  if (H <= 0 || max_rows <= 0) return fail(TL_ERR_INVALID_ARG, "%s: H and max_rows must be positive", what);
  if (H % 8) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: H=%d is not a multiple of 8", what, H);
  if (!sorted || !row_pos) return fail(TL_ERR_INVALID_ARG, "%s: null pointer argument", what);
  if (!aligned16(sorted) || !aligned4(row_pos)) return fail(TL_ERR_INVALID_ARG, "%s: matrices must be 16-byte aligned, row_pos 4-byte", what);
  return TL_OK;
}

static RowsParams rows_params(const int* row_pos, int T, int H, int topk, int max_rows) {
  RowsParams p;
  memset(&p, 0, sizeof p);
  p.row_pos = row_pos;
  p.T = T; p.H8 = H / 8; p.topk = topk; p.max_rows = max_rows;
  return p;
}

constexpr long kMaxGrid = 1 << 20;     // workgroups; each goes on to further tokens
static int rows_grid(long waves) { return (int)((waves + 3) / 4 < kMaxGrid ? (waves + 3) / 4 : kMaxGrid); }

static int check_sort(const char* what, int T, int topk, int E) {
  if (int e = check_tokens(what, T, topk)) return e;
  if (E <= 0) return fail(TL_ERR_INVALID_ARG, "%s: E must be positive", what);
  if (E > kMaxSortExperts) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: at most %d experts (got %d)", what, kMaxSortExperts, E);
  if ((long)T * topk > kMaxSortRows) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: at most 2^20 rows (got %ld)", what, (long)T * topk);
  return TL_OK;
}

}  // namespace tl

using namespace tl;

extern "C" {

int tl_moe_sort_query(const tl_ctx* ctx, int T, int topk, int E, size_t* ws_bytes) {
  if (int e = check_ctx(ctx)) return e;
  if (!ws_bytes) return fail(TL_ERR_INVALID_ARG, "tl_moe_sort_query: ws_bytes must not be null");
  if (int e = check_sort("tl_moe_sort_query", T, topk, E)) return e;
  const size_t b = (size_t)sort_chunks((long)T * topk) * E * sizeof(int);
  *ws_bytes = (b + 255) / 256 * 256;
  return TL_OK;
}

int tl_moe_sort(tl_ctx* ctx, const int* topk_ids, int T, int topk, int first_expert, int E, int* expert_offsets, int* sorted_row, int* row_pos,
                void* workspace, size_t ws_bytes, void* stream) {
  if (int e = check_ctx(ctx)) return e;
  size_t need;
  if (int e = check_sort("tl_moe_sort", T, topk, E)) return e;
  if (first_expert < 0 || (long)first_expert + E > (1L << 31)) return fail(TL_ERR_INVALID_ARG, "tl_moe_sort: first_expert must not be negative, nor the last expert beyond 2^31 - 1");
  if (!topk_ids || !expert_offsets || !sorted_row || !row_pos || !workspace) return fail(TL_ERR_INVALID_ARG, "tl_moe_sort: null pointer argument");
  if (!aligned4(topk_ids) || !aligned4(expert_offsets) || !aligned4(sorted_row) || !aligned4(row_pos) || !aligned4(workspace))
    return fail(TL_ERR_INVALID_ARG, "tl_moe_sort: pointers must be 4-byte aligned");
  if (int e = tl_moe_sort_query(ctx, T, topk, E, &need)) return e;
  if (ws_bytes < need) return fail(TL_ERR_WORKSPACE_TOO_SMALL, "tl_moe_sort: workspace of %zu bytes, %zu needed", ws_bytes, need);
  if (int e = check_op_ctx(ctx)) return e;
  SortParams p;
  memset(&p, 0, sizeof p);
  p.ids = topk_ids; p.n = T * topk; p.first = first_expert; p.E = E;
  p.offsets = expert_offsets; p.sorted_row = sorted_row; p.row_pos = row_pos;
  p.hist = (int*)workspace;
  p.chunks = sort_chunks(p.n);
  hipStream_t s = (hipStream_t)stream;
  if (p.chunks == 1) {     // (of a row a thread: more are taken where that would make more than 128 chunks)
    hipLaunchKernelGGL((moe_place_kernel<1, true>), dim3(1), dim3(kSortThreads), 0, s, p);
    TL_HIP(hipGetLastError());
    return TL_OK;
  }
  auto go = [&](auto rpt_c) {
    constexpr int RPT = decltype(rpt_c)::value;
    hipLaunchKernelGGL(moe_count_kernel<RPT>, dim3(p.chunks), dim3(kSortThreads), 0, s, p);
    hipLaunchKernelGGL((moe_place_kernel<RPT, false>), dim3(p.chunks), dim3(kSortThreads), 0, s, p);
  };
  switch (sort_rows_per_thread(p.n)) {
    case 1: go(std::integral_constant<int, 1>{}); break;
    case 2: go(std::integral_constant<int, 2>{}); break;
    case 4: go(std::integral_constant<int, 4>{}); break;
    default: go(std::integral_constant<int, 8>{}); break;
  }
  TL_HIP(hipGetLastError());
  return TL_OK;
}

int tl_moe_dispatch(tl_ctx* ctx, const void* x, const int* row_pos, int T, int H, int topk, int max_rows, void* xs, void* stream) {
  if (int e = check_ctx(ctx)) return e;
  if (int e = check_rows("tl_moe_dispatch", xs, row_pos, T, H, topk, max_rows)) return e;
  if (!x) return fail(TL_ERR_INVALID_ARG, "tl_moe_dispatch: null pointer argument");
  if (!aligned16(x)) return fail(TL_ERR_INVALID_ARG, "tl_moe_dispatch: matrices must be 16-byte aligned");
  if (int e = check_op_ctx(ctx)) return e;
  RowsParams p = rows_params(row_pos, T, H, topk, max_rows);
  p.x = (const bf16_t*)x; p.out = (bf16_t*)xs;
  p.segs = ceil_div(p.H8, 64);
  const dim3 grid(rows_grid(p.T * p.segs));
  if (dispatch_choice(T, H, topk, max_rows).stream_stores) hipLaunchKernelGGL(moe_dispatch_kernel<true>, grid, dim3(256), 0, (hipStream_t)stream, p);
  else hipLaunchKernelGGL(moe_dispatch_kernel<false>, grid, dim3(256), 0, (hipStream_t)stream, p);
  TL_HIP(hipGetLastError());
  return TL_OK;
}

int tl_moe_dispatch_grad(tl_ctx* ctx, const void* dxs, const int* row_pos, int T, int H, int topk, int max_rows, void* dx, void* stream) {
  if (int e = check_ctx(ctx)) return e;
  if (int e = check_rows("tl_moe_dispatch_grad", dxs, row_pos, T, H, topk, max_rows)) return e;
  if (!dx) return fail(TL_ERR_INVALID_ARG, "tl_moe_dispatch_grad: null pointer argument");
  if (!aligned16(dx)) return fail(TL_ERR_INVALID_ARG, "tl_moe_dispatch_grad: matrices must be 16-byte aligned");
  if (int e = check_op_ctx(ctx)) return e;
  RowsParams p = rows_params(row_pos, T, H, topk, max_rows);
  p.ys = (const bf16_t*)dxs; p.out = (bf16_t*)dx;
  p.segs = ceil_div(p.H8, 64);
  const dim3 grid(rows_grid(p.T * p.segs));
  if (gather_choice(T, H, topk, max_rows).stream_loads) hipLaunchKernelGGL((moe_gather_sum_kernel<false, true>), grid, dim3(256), 0, (hipStream_t)stream, p);
  else hipLaunchKernelGGL((moe_gather_sum_kernel<false, false>), grid, dim3(256), 0, (hipStream_t)stream, p);
  TL_HIP(hipGetLastError());
  return TL_OK;
}

int tl_moe_combine(tl_ctx* ctx, const void* ys, const float* topk_w, const int* row_pos, int T, int H, int topk, int max_rows, const void* add, void* out,
                   void* stream) {
  if (int e = check_ctx(ctx)) return e;
  if (int e = check_rows("tl_moe_combine", ys, row_pos, T, H, topk, max_rows)) return e;
  if (!topk_w || !out) return fail(TL_ERR_INVALID_ARG, "tl_moe_combine: null pointer argument");
  if (!aligned4(topk_w) || !aligned16(out) || !aligned16(add)) return fail(TL_ERR_INVALID_ARG, "tl_moe_combine: matrices must be 16-byte aligned, topk_w 4-byte");
  if (int e = check_op_ctx(ctx)) return e;
  RowsParams p = rows_params(row_pos, T, H, topk, max_rows);
  p.ys = (const bf16_t*)ys; p.w = topk_w; p.add = (const bf16_t*)add; p.out = (bf16_t*)out;
  p.segs = ceil_div(p.H8, 64);
  const dim3 grid(rows_grid(p.T * p.segs));
  if (gather_choice(T, H, topk, max_rows).stream_loads) hipLaunchKernelGGL((moe_gather_sum_kernel<true, true>), grid, dim3(256), 0, (hipStream_t)stream, p);
  else hipLaunchKernelGGL((moe_gather_sum_kernel<true, false>), grid, dim3(256), 0, (hipStream_t)stream, p);
  TL_HIP(hipGetLastError());
  return TL_OK;
}

int tl_moe_combine_grad(tl_ctx* ctx, const void* dout, const void* ys, const float* topk_w, const int* row_pos, int T, int H, int topk, int max_rows, void* dys,
                        float* dtopk_w, void* stream) {
  if (int e = check_ctx(ctx)) return e;
  if (int e = check_rows("tl_moe_combine_grad", ys, row_pos, T, H, topk, max_rows)) return e;
  if (!dout || !topk_w || !dys || !dtopk_w) return fail(TL_ERR_INVALID_ARG, "tl_moe_combine_grad: null pointer argument");
  if (!aligned16(dout) || !aligned16(dys) || !aligned4(topk_w) || !aligned4(dtopk_w))
    return fail(TL_ERR_INVALID_ARG, "tl_moe_combine_grad: matrices must be 16-byte aligned, weights 4-byte");
  if (int e = check_op_ctx(ctx)) return e;
  RowsParams p = rows_params(row_pos, T, H, topk, max_rows);
  p.x = (const bf16_t*)dout; p.ys = (const bf16_t*)ys; p.w = topk_w; p.dys = (bf16_t*)dys; p.dw = dtopk_w;
  const RowsChoice choice = combine_grad_choice(T, H, topk, max_rows);
  auto go = [&](auto waves_c) {
    constexpr int WAVES = decltype(waves_c)::value;
    const dim3 grid(rows_grid(p.T * WAVES));
    if (choice.stream_loads) hipLaunchKernelGGL((moe_combine_grad_kernel<WAVES, true, true>), grid, dim3(256), 0, (hipStream_t)stream, p);
    else if (choice.stream_stores) hipLaunchKernelGGL((moe_combine_grad_kernel<WAVES, false, true>), grid, dim3(256), 0, (hipStream_t)stream, p);
    else hipLaunchKernelGGL((moe_combine_grad_kernel<WAVES, false, false>), grid, dim3(256), 0, (hipStream_t)stream, p);
  };
  if (choice.waves == 1) go(std::integral_constant<int, 1>{}); else go(std::integral_constant<int, 4>{});
  TL_HIP(hipGetLastError());
  return TL_OK;
}

int tl_moe_route_grad(tl_ctx* ctx, const float* gate_logits, const int* topk_ids, const float* dtopk_w, int T, int E, int topk, int renormalize, float* dlogits,
                      void* stream) {
  if (int e = check_ctx(ctx)) return e;
  if (int e = check_tokens("tl_moe_route_grad", T, topk)) return e;
  if (E <= 0) return fail(TL_ERR_INVALID_ARG, "tl_moe_route_grad: E must be positive");
  if (E > kMaxSortExperts || topk > E) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_moe_route_grad: E <= %d and topk <= E required", kMaxSortExperts);
  if (!gate_logits || !topk_ids || !dtopk_w || !dlogits) return fail(TL_ERR_INVALID_ARG, "tl_moe_route_grad: null pointer argument");
  if (!aligned4(gate_logits) || !aligned4(topk_ids) || !aligned4(dtopk_w) || !aligned4(dlogits))
    return fail(TL_ERR_INVALID_ARG, "tl_moe_route_grad: pointers must be 4-byte aligned");
  if (T > (1 << 24)) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_moe_route_grad: at most 2^24 tokens (got %d)", T);
  if (int e = check_op_ctx(ctx)) return e;
  RouteGradParams p;
  memset(&p, 0, sizeof p);
  p.logits = gate_logits; p.ids = topk_ids; p.dw = dtopk_w; p.dlogits = dlogits;
  p.T = T; p.E = E; p.topk = topk; p.renormalize = renormalize;
  auto go = [&](auto lanes_c, auto per_c) {
    constexpr int LANES = decltype(lanes_c)::value, PER = decltype(per_c)::value;
    hipLaunchKernelGGL((moe_route_grad_kernel<LANES, PER>), dim3(ceil_div(T, 256 / LANES)), dim3(256), 0, (hipStream_t)stream, p);
  };
  using std::integral_constant;
  auto per = [&](auto lanes_c) {
    constexpr int LANES = decltype(lanes_c)::value;
    switch (route_per(E, LANES)) {
      case 1: go(lanes_c, integral_constant<int, 1>{}); break;
      case 2: go(lanes_c, integral_constant<int, 2>{}); break;
      case 4: go(lanes_c, integral_constant<int, 4>{}); break;
      case 8: go(lanes_c, integral_constant<int, 8>{}); break;
      default: go(lanes_c, integral_constant<int, 256 / LANES>{});
    }
  };
  if (route_lanes(topk) == 16) per(integral_constant<int, 16>{}); else per(integral_constant<int, 32>{});
  TL_HIP(hipGetLastError());
  return TL_OK;
}

}  // extern "C"
