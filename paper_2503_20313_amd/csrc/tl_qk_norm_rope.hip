// RMS norm of every query and key head and the position rotation in one pass; in the cache form keys and values go straight to
// their places in the pages.  gfx950 only, head_dim 128.
//
//   y = x * rsqrt(mean(x^2) + eps) * w          per head, fp32
//   (y_i, y_j) -> (y_i cos - y_j sin, y_j cos + y_i sin)   for the pairs (i, j) = (i, i + rot/2) or (2i, 2i + 1), rounded once
//
// Bound by memory: every element is read once and written once.  16 lanes own a head (8 elements, one 16-byte access, each), so the
// mean is four lane rotations inside a row of 16 lanes and a pair's partner sits in the same row; a row of lanes takes kHeads heads
// of one token, which share the token's angles.  4096 rows of 32 + 32 heads (136 MB moved): kHeads 1, 2, 3, 4: 27.8, 24.4, 25.4, 25.2 us;
// 8001 rows of 32 + 8 + 8 heads into pages in random order (199 MB): 47.2, 38.8, 38.8, 39.3.
// Results larger than the dies' L2s together are stored as streaming, as they would not stay there: 33.1 -> 25.2 and 44.3 -> 39.3 us (kHeads 4).
// Smaller ones, a decode step's, are left for the attention that reads them next.
#include "tl_paged.h"

namespace tl {

constexpr int kHeads = 2;      // heads of a token that a row of 16 lanes takes

struct RopeParams {
  const bf16_t *q, *k, *v;
  long q_stride, k_stride, v_stride, qo_stride, ko_stride;
  bf16_t *q_out, *k_out, *k_cache, *v_cache;   // k_out: dense form; k_cache, v_cache: cache form
  const bf16_t *wq, *wk;                       // null: no norm
  const float* cos_sin;
  const int *positions, *slots;
  int T, Hq, Hk, heads, groups;                // heads of a token (values among them), groups of kHeads
  int max_position, rot, neighbours;
  int page, page_shift, n_slots;
  long page_stride;
  float eps;
};

// Sum over the 16 lanes of a row, in every lane of it.
__device__ __forceinline__ float row_sum(float x) {
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x128, 0xf, 0xf, true));  // row_ror:8
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x124, 0xf, 0xf, true));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x122, 0xf, 0xf, true));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x121, 0xf, 0xf, true));
  return x;
}

__device__ __forceinline__ void unpack8(u32x4 v, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; e++) {
    x[2 * e] = __uint_as_float(v[e] << 16);
    x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
  }
}

template <bool CACHE, bool STREAM>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(const RopeParams p) {
  const long task = (long)workgroup_index() * 16 + (threadIdx.x >> 4);
  const int t = (int)(task / p.groups), h0 = (int)(task - (long)t * p.groups) * kHeads;
  if (t >= p.T) return;   // (whole rows of lanes)
  const int l = threadIdx.x & 15;
  // (position, slot and heads are on their way together; a row that is left out has been read for nothing)
  const int pos = p.rot ? p.positions[t] : 0;
  const int slot = CACHE ? p.slots[t] : 0;
  u32x4 raw[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; i++) {
    const int h = h0 + i;
    if (h >= p.heads) continue;
    const bf16_t* src = h < p.Hq ? p.q + t * p.q_stride + (long)h * kPagedD
                        : h < p.Hq + p.Hk ? p.k + t * p.k_stride + (long)(h - p.Hq) * kPagedD
                                          : p.v + t * p.v_stride + (long)(h - p.Hq - p.Hk) * kPagedD;
    raw[i] = *(const u32x4*)(src + l * 8);
  }
  if (p.rot && (unsigned)pos >= (unsigned)p.max_position) return;
  if (CACHE && (unsigned)slot >= (unsigned)p.n_slots) return;
  // the lane's angles.  Halves: elements l*8.. of the first half meet those of lane l + rot/16; neighbours: pairs l*4..
  const int half = p.rot >> 1, hl = p.rot >> 4;
  const bool turns = l * 8 < p.rot;
  const bool second = !p.neighbours && l >= hl;      // the lane holds second members of its pairs
  float cs[8], sn[8];
  if (turns) {
    const float* row = p.cos_sin + (long)pos * p.rot;
    if (p.neighbours) {
      *(floatx4*)cs = *(const floatx4*)(row + l * 4);
      *(floatx4*)sn = *(const floatx4*)(row + half + l * 4);
    } else {
      const int at = (second ? l - hl : l) * 8;
      *(floatx4*)cs = *(const floatx4*)(row + at);
      *(floatx4*)(cs + 4) = *(const floatx4*)(row + at + 4);
      *(floatx4*)sn = *(const floatx4*)(row + half + at);
      *(floatx4*)(sn + 4) = *(const floatx4*)(row + half + at + 4);
    }
  }
  const int partner = ((threadIdx.x & 48) + (turns ? (second ? l - hl : l + hl) : l)) << 2;
  long at_page = 0;
  int at_row = 0;
  if (CACHE) {
    at_page = (long)(slot >> p.page_shift) * p.page_stride;
    at_row = slot & (p.page - 1);
  }
#pragma unroll
  for (int i = 0; i < kHeads; i++) {
    const int h = h0 + i;
    if (h >= p.heads) continue;   // the same for all lanes of a row, which is what row_sum and the exchange below need
    const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hk;
    bf16_t* dst;
    if (is_q) dst = p.q_out + t * p.qo_stride + (long)h * kPagedD;
    else if (CACHE) dst = (is_v ? p.v_cache : p.k_cache) + at_page + ((long)(is_v ? h - p.Hq - p.Hk : h - p.Hq) * p.page + at_row) * kPagedD;
    else dst = p.k_out + t * p.ko_stride + (long)(h - p.Hq) * kPagedD;
    u32x4 res = raw[i];
    if (!is_v) {
      float x[8];
      unpack8(raw[i], x);
      const bf16_t* w = is_q ? p.wq : p.wk;
      if (w) {
        float ss = 0.f, wv[8];
#pragma unroll
        for (int e = 0; e < 8; e++) ss = __builtin_fmaf(x[e], x[e], ss);
        const float r = 1.f / sqrtf(row_sum(ss) * (1.f / kPagedD) + p.eps);
        unpack8(*(const u32x4*)(w + l * 8), wv);
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = x[e] * r * wv[e];
      }
      if (p.rot && p.neighbours) {
        if (turns) {
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const float a = x[2 * e], b = x[2 * e + 1];
            x[2 * e] = a * cs[e] - b * sn[e];
            x[2 * e + 1] = b * cs[e] + a * sn[e];
          }
        }
      } else if (p.rot) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const float o = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(partner, __builtin_bit_cast(int, x[e])));
          if (turns) x[e] = second ? x[e] * cs[e] + o * sn[e] : x[e] * cs[e] - o * sn[e];
        }
      }
      res = pack_bf16x8(x);
    }
    if constexpr (STREAM) __builtin_nontemporal_store(res, (u32x4*)(dst + l * 8)); else *(u32x4*)(dst + l * 8) = res;
  }
}

// In place every row lies where it lay: with another stride a row would be written over one that is still to be read.
static int check_in_place(const char* what, const char* name, const void* in, long long in_stride, const void* out, long long out_stride, int T) {
  if (in == out && in_stride != out_stride && T > 1) return fail(TL_ERR_INVALID_ARG, "%s: %s in place has one row stride, not two", what, name);
  return TL_OK;
}

static long rope_workgroups(int T, int heads) { return ((long)T * ceil_div(heads, kHeads) + 15) / 16; }

static int check_rope(const char* what, const void* q, long long q_stride, const void* k, long long k_stride, const void* q_out, long long qo_stride, int T,
                      int Hq, int Hk, int heads, int head_dim, const void* wq, const void* wk, float eps, const int* positions, const float* cos_sin, int max_position,
                      int rot_dim) {
  if (!q || !k || !q_out) return fail(TL_ERR_INVALID_ARG, "%s: null pointer argument", what);
  if (T <= 0 || Hq <= 0 || Hk <= 0) return fail(TL_ERR_INVALID_ARG, "%s: rows and heads must be positive", what);
  if (head_dim != kPagedD) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: head_dim %d is not supported (128 only)", what, head_dim);
  if (Hq > 1024 || Hk > 1024) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: at most 1024 heads", what);
  if (rope_workgroups(T, heads) > kMostWorkgroups) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: too many rows and heads for one launch", what);
  if (!!wq != !!wk) return fail(TL_ERR_INVALID_ARG, "%s: q_weight and k_weight are given together or not at all", what);
  if (wq && !(eps >= 0.f)) return fail(TL_ERR_INVALID_ARG, "%s: eps must not be negative", what);
  if (rot_dim < 0 || rot_dim > kPagedD || rot_dim % 16) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: rot_dim %d is not a multiple of 16 up to 128", what, rot_dim);
  if (rot_dim && (!positions || !cos_sin || max_position <= 0)) return fail(TL_ERR_INVALID_ARG, "%s: a rotation needs positions, cos_sin and max_position", what);
  if (q_stride < (long long)Hq * kPagedD || k_stride < (long long)Hk * kPagedD || qo_stride < (long long)Hq * kPagedD)
    return fail(TL_ERR_INVALID_ARG, "%s: a row stride is shorter than the row's heads", what);
  if (q_stride % 8 || k_stride % 8 || qo_stride % 8) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: row strides must be multiples of 8 elements", what);
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(wq) || !aligned16(wk) || !aligned16(cos_sin))
    return fail(TL_ERR_INVALID_ARG, "%s: device pointers must be 16-byte aligned", what);
  if (!aligned4(positions)) return fail(TL_ERR_INVALID_ARG, "%s: positions must be 4-byte aligned", what);
  return check_in_place(what, "q", q, q_stride, q_out, qo_stride, T);
}

static RopeParams rope_params(const void* q, long long q_stride, const void* k, long long k_stride, void* q_out, long long qo_stride, int T, int Hq, int Hk,
                              int heads, const void* wq, const void* wk, float eps, const int* positions, const float* cos_sin, int max_position, int rot_dim,
                              int interleaved) {
  RopeParams p;
  memset(&p, 0, sizeof p);
  p.q = (const bf16_t*)q; p.k = (const bf16_t*)k; p.q_out = (bf16_t*)q_out;
  p.q_stride = q_stride; p.k_stride = k_stride; p.qo_stride = qo_stride;
  p.wq = (const bf16_t*)wq; p.wk = (const bf16_t*)wk;
  p.cos_sin = cos_sin; p.positions = positions;
  p.T = T; p.Hq = Hq; p.Hk = Hk; p.heads = heads; p.groups = ceil_div(heads, kHeads);
  p.max_position = max_position; p.rot = rot_dim; p.neighbours = interleaved ? 1 : 0;
  p.eps = eps;
  return p;
}

constexpr long kL2Bytes = 32L << 20;      // of the eight dies

template <bool CACHE>
static int launch_rope(const RopeParams& p, void* stream) {
  const bool stream_out = (long)p.T * p.heads * kPagedD * 2 > kL2Bytes;
  hipLaunchKernelGGL((stream_out ? qk_norm_rope_kernel<CACHE, true> : qk_norm_rope_kernel<CACHE, false>), grid_of(rope_workgroups(p.T, p.heads)), dim3(256), 0, (hipStream_t)stream, p);
  TL_HIP(hipGetLastError());
  return TL_OK;
}

}  // namespace tl

using namespace tl;

extern "C" {

int tl_qk_norm_rope(tl_ctx* ctx, const void* q, long long q_stride, const void* k, long long k_stride, void* q_out, long long q_out_stride, void* k_out,
                    long long k_out_stride, int T, int heads_q, int heads_kv, int head_dim, const void* q_weight, const void* k_weight, float eps,
                    const int* positions, const float* cos_sin, int max_position, int rot_dim, int interleaved, void* stream) {
  const char* what = "tl_qk_norm_rope";
  if (int e = check_ctx(ctx)) return e;
  if (int e = check_rope(what, q, q_stride, k, k_stride, q_out, q_out_stride, T, heads_q, heads_kv, heads_q + heads_kv, head_dim, q_weight, k_weight, eps,
                         positions, cos_sin, max_position, rot_dim))
    return e;
  if (!k_out) return fail(TL_ERR_INVALID_ARG, "%s: null pointer argument", what);
  if (k_out_stride < (long long)heads_kv * kPagedD) return fail(TL_ERR_INVALID_ARG, "%s: a row stride is shorter than the row's heads", what);
  if (k_out_stride % 8) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: row strides must be multiples of 8 elements", what);
  if (!aligned16(k_out)) return fail(TL_ERR_INVALID_ARG, "%s: device pointers must be 16-byte aligned", what);
  if (int e = check_in_place(what, "k", k, k_stride, k_out, k_out_stride, T)) return e;
  if (int e = check_paged_launch(ctx, what)) return e;
  RopeParams p = rope_params(q, q_stride, k, k_stride, q_out, q_out_stride, T, heads_q, heads_kv, heads_q + heads_kv, q_weight, k_weight, eps, positions,
                             cos_sin, max_position, rot_dim, interleaved);
  p.k_out = (bf16_t*)k_out; p.ko_stride = k_out_stride;
  return launch_rope<false>(p, stream);
}

int tl_qk_norm_rope_cache(tl_ctx* ctx, const tl_paged_dims* dims, const void* q, long long q_stride, const void* k, long long k_stride, const void* v,
                          long long v_stride, void* q_out, long long q_out_stride, void* k_cache, void* v_cache, const int* slots, const void* q_weight,
                          const void* k_weight, float eps, const int* positions, const float* cos_sin, int max_position, int rot_dim, int interleaved,
                          void* stream) {
  const char* what = "tl_qk_norm_rope_cache";
  PagedGeom g;
  if (int e = resolve_paged(ctx, dims, &g)) return e;
  if (int e = check_rope(what, q, q_stride, k, k_stride, q_out, q_out_stride, g.T, g.Hq, g.Hk, g.Hq + 2 * g.Hk, kPagedD, q_weight, k_weight, eps, positions,
                         cos_sin, max_position, rot_dim))
    return e;
  if (!v || !k_cache || !v_cache || !slots) return fail(TL_ERR_INVALID_ARG, "%s: null pointer argument", what);
  if (v_stride < (long long)g.Hk * kPagedD) return fail(TL_ERR_INVALID_ARG, "%s: a row stride is shorter than the row's heads", what);
  if (v_stride % 8) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: row strides must be multiples of 8 elements", what);
  if (!aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache)) return fail(TL_ERR_INVALID_ARG, "%s: device pointers must be 16-byte aligned", what);
  if (!aligned4(slots)) return fail(TL_ERR_INVALID_ARG, "%s: slots must be 4-byte aligned", what);
  if (int e = check_paged_launch(ctx, what)) return e;
  RopeParams p = rope_params(q, q_stride, k, k_stride, q_out, q_out_stride, g.T, g.Hq, g.Hk, g.Hq + 2 * g.Hk, q_weight, k_weight, eps, positions, cos_sin,
                             max_position, rot_dim, interleaved);
  p.v = (const bf16_t*)v; p.v_stride = v_stride;
  p.k_cache = (bf16_t*)k_cache; p.v_cache = (bf16_t*)v_cache;
  p.slots = slots;
  p.page = g.page; p.page_shift = g.page_shift; p.n_slots = g.n_pages * g.page; p.page_stride = g.page_stride;
  return launch_rope<true>(p, stream);
}

}  // extern "C"
