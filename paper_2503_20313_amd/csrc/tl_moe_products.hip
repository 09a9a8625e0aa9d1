// The experts' products on rows sorted by expert, and their gradients: Y_e = X_e W_e, dX_e = dY_e W_e^T, dW_e = X_e^T dY_e, with X_e the
// rows [expert_offsets[e], expert_offsets[e + 1]).  gfx950 only.
//
// One tile kernel in three layouts (tl_gemm_tile.h): W as it is, W read along its rows, and both operands read along the rows of the
// expert, which is then the axis that is summed over.
#include "tl_gemm_tile.h"
#include "tl_host.h"

namespace tl {

constexpr int kMaxProductExperts = 256;

struct ProductParams {
  const bf16_t *x, *w, *dy;
  const int* offsets;
  bf16_t* out;
  const float* add;
  float* out32;
  int max_rows, K, N, E;
  int nbm, nbn;            // column blocks; for dW also row blocks of an expert's K x N
  int swizzle, group_m;
};

// dW in fp32: (add +) the product.
struct AddRows32 {
  static constexpr bool SCALED = false, GATED = false, F32 = true;
  const float* add;
  float* c;
  long ldc;
  __device__ __forceinline__ bf16_t* row(int, float&) const { return nullptr; }
  __device__ __forceinline__ void group(int) const {}
  __device__ __forceinline__ void store(int, int, u32x4) const {}
  __device__ __forceinline__ void store4(int r, int col, floatx4 v) const {
    const long at = (long)r * ldc + col;
    if (add) {
      const floatx4 a = *(const floatx4*)(add + at);
#pragma unroll
      for (int e = 0; e < 4; e++) v[e] += a[e];
    }
    *(floatx4*)(c + at) = v;
  }
};

// Rows of expert e, whatever expert_offsets holds: inside [0, max_rows), or none.
__device__ __forceinline__ void rows_of(const ProductParams& p, int e, int* lo, int* n) {
  *lo = min(max(p.offsets[e], 0), p.max_rows);
  *n = max(min(max(p.offsets[e + 1], 0), p.max_rows) - *lo, 0);
}

template <class Cfg, bool GRAD_X>
__global__ void __launch_bounds__(Cfg::NTHREADS) moe_product_kernel(const ProductParams p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  __shared__ int s_lo[kMaxProductExperts], s_n[kMaxProductExperts], s_first[kMaxProductExperts + 1];
  const int tid = threadIdx.x, lane = tid & 63;
  // ---- the row tiles of all experts
  for (int e = tid; e < kMaxProductExperts; e += Cfg::NTHREADS) {
    int lo = 0, n = 0;
    if (e < p.E) rows_of(p, e, &lo, &n);
    s_lo[e] = lo;
    s_n[e] = n;
  }
  __syncthreads();
  if (tid < 64) {
    int v = 0, mine[4];
#pragma unroll
    for (int i = 0; i < 4; i++) { mine[i] = (s_n[lane * 4 + i] + Cfg::BM - 1) / Cfg::BM; v += mine[i]; }
    int scan = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(scan, d);
      if (lane >= d) scan += o;
    }
    int at = scan - v;
#pragma unroll
    for (int i = 0; i < 4; i++) { s_first[lane * 4 + i] = at; at += mine[i]; }
    if (lane == 63) s_first[kMaxProductExperts] = at;
  }
  __syncthreads();
  Sched sc;
  sc.nbm = __builtin_amdgcn_readfirstlane(s_first[kMaxProductExperts]);
  sc.nbn = p.nbn;
  sc.n_tiles = sc.nbm * sc.nbn;
  sc.G = gridDim.x;
  sc.first_block = 0;
  sc.swizzle = p.swizzle;
  sc.group_m = p.group_m < sc.nbm ? p.group_m : (sc.nbm > 0 ? sc.nbm : 1);
  const int kdim = GRAD_X ? p.N : p.K, ndim = GRAD_X ? p.K : p.N;
  for (int pos = blockIdx.x; pos < sc.n_tiles; pos += sc.G) {
    const int tile = sched_tile(sc, pos), bm = tile / sc.nbn, bn = tile - bm * sc.nbn;
    int e = 0;    // the last expert whose tiles start at or before bm (one without tiles starts where the next one does)
#pragma unroll
    for (int d = kMaxProductExperts / 2; d >= 1; d /= 2)
      if (s_first[e + d] <= bm) e += d;
    e = __builtin_amdgcn_readfirstlane(e);
    const int r0 = (bm - s_first[e]) * Cfg::BM, rows = __builtin_amdgcn_readfirstlane(min(s_n[e] - r0, Cfg::BM));
    const long at = __builtin_amdgcn_readfirstlane(s_lo[e] + r0);
    const int col = bn * Cfg::BN, cols = min(Cfg::BN, ndim - col);
    const bf16_t* w = p.w + (long)e * p.K * p.N;
    if constexpr (GRAD_X)
      gemm_tile<Cfg>(p.dy + at * p.N, p.N, nullptr, 1, w + (long)col * p.N, p.N, DenseRows{p.out + at * p.K + col, p.K}, rows, cols, kdim, smem);
    else
      gemm_tile<Cfg>(p.x + at * p.K, p.K, nullptr, 1, w + col, p.N, DenseRows{p.out + at * p.N + col, p.N}, rows, cols, kdim, smem);
  }
}

template <class Cfg, class Out>
__global__ void __launch_bounds__(Cfg::NTHREADS) moe_grad_w_kernel(const ProductParams p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int per = p.nbm * p.nbn;
  const int e = blockIdx.x / per, tile = blockIdx.x - e * per;
  const int bm = tile / p.nbn, bn = tile - bm * p.nbn;
  int lo, n;
  rows_of(p, e, &lo, &n);
  lo = __builtin_amdgcn_readfirstlane(lo);
  n = __builtin_amdgcn_readfirstlane(n);
  const int row = bm * Cfg::BM, rows = min(Cfg::BM, p.K - row), col = bn * Cfg::BN, cols = min(Cfg::BN, p.N - col);
  const long at = ((long)e * p.K + row) * p.N + col;
  Out out;
  if constexpr (StoresF32<Out>::value) out = Out{p.add ? p.add + at : nullptr, p.out32 + at, p.N};
  else out = Out{p.out + at, p.N};
  if (n == 0) {     // an expert without rows
    for (int i = threadIdx.x; i < rows * (cols / 8); i += Cfg::NTHREADS) {
      const int r = i / (cols / 8), c = (i - r * (cols / 8)) * 8;
      if constexpr (StoresF32<Out>::value) {
        out.store4(r, c, floatx4{0.f, 0.f, 0.f, 0.f});
        out.store4(r, c + 4, floatx4{0.f, 0.f, 0.f, 0.f});
      } else {
        out.store(r, c, u32x4{0, 0, 0, 0});
      }
    }
    return;
  }
  gemm_tile<Cfg, Out>(p.x + (long)lo * p.K + row, p.K, nullptr, 1, p.dy + (long)lo * p.N + col, p.N, out, rows, cols, n, smem);
}

// ======================================================================================
// Host side
// ======================================================================================
typedef TileCfg<256, 256, 2, 4, 32, 4, false, true> CfgX256;      // dX: W along its rows
typedef TileCfg<128, 128, 2, 2, 64, 4, false, true> CfgX128;
typedef TileCfg<256, 256, 2, 4, 32, 4, true, false> CfgW256;      // dW: both operands in the rows that are summed over
typedef TileCfg<128, 128, 2, 2, 64, 4, true, false> CfgW128;

static int check_product(const char* what, int max_rows, int K, int N, int E) {
  if (max_rows <= 0 || K <= 0 || N <= 0 || E <= 0) return fail(TL_ERR_INVALID_ARG, "%s: max_rows, K, N and E must be positive", what);
  if (E > kMaxProductExperts) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: at most %d experts (got %d)", what, kMaxProductExperts, E);
  if (K % 8 || N % 8) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: K=%d and N=%d must be multiples of 8", what, K, N);
  if (K > (1 << 20) || N > (1 << 20)) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: K and N must not exceed 2^20", what);
  return TL_OK;
}

static int check_product_call(tl_ctx* ctx, const char* what, int way, const void* a, const void* b, const void* out, const int* offsets, int max_rows, int K, int N,
                              int E, const void* workspace, size_t ws_bytes) {
  if (int e = check_ctx(ctx)) return e;
  size_t need;
  if (int e = check_product(what, max_rows, K, N, E)) return e;
  if (!a || !b || !out || !offsets || !workspace) return fail(TL_ERR_INVALID_ARG, "%s: null pointer argument", what);
  if (!aligned16(a) || !aligned16(b) || !aligned16(out) || ((uintptr_t)offsets & 3) || !aligned128(workspace))
    return fail(TL_ERR_INVALID_ARG, "%s: matrices must be 16-byte aligned, the workspace 128-byte, expert_offsets 4-byte", what);
  if (int e = tl_moe_gemm_query(ctx, way, max_rows, K, N, E, &need)) return e;
  if (ws_bytes < need) return fail(TL_ERR_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need);
  return check_op_ctx(ctx);
}

// The small tile where the large ones would leave compute units without work.
static bool small_tiles(const tl_ctx* ctx, long tiles256) { return tiles256 < ctx->num_cus; }

template <bool GRAD_X>
static int launch_product(tl_ctx* ctx, ProductParams& p, hipStream_t s) {
  const int ndim = GRAD_X ? p.K : p.N;
  const long tiles = (long)(ceil_div(p.max_rows, 256) + p.E / 2) * ceil_div(ndim, 256);
  p.swizzle = 1;
  p.group_m = 4;
  if (small_tiles(ctx, tiles)) {
    p.nbn = ceil_div(ndim, 128);
    typedef typename std::conditional<GRAD_X, CfgX128, Cfg128x128>::type Cfg;
    return launch_fused<Cfg>(moe_product_kernel<Cfg, GRAD_X>, p, ctx->num_cus, s);
  }
  p.nbn = ceil_div(ndim, 256);
  typedef typename std::conditional<GRAD_X, CfgX256, Cfg256x256>::type Cfg;
  return launch_fused<Cfg>(moe_product_kernel<Cfg, GRAD_X>, p, ctx->num_cus, s);
}

}  // namespace tl

using namespace tl;

extern "C" {

int tl_moe_gemm_query(const tl_ctx* ctx, int way, int max_rows, int K, int N, int E, size_t* ws_bytes) {
  if (int e = check_ctx(ctx)) return e;
  if (!ws_bytes) return fail(TL_ERR_INVALID_ARG, "tl_moe_gemm_query: ws_bytes must not be null");
  if (way != TL_MOE_FORWARD && way != TL_MOE_GRAD_X && way != TL_MOE_GRAD_W) return fail(TL_ERR_INVALID_ARG, "tl_moe_gemm_query: %d is not one of the three products", way);
  if (int e = check_product("tl_moe_gemm_query", max_rows, K, N, E)) return e;
  *ws_bytes = 256;
  return TL_OK;
}

int tl_moe_gemm(tl_ctx* ctx, const void* x, const void* w, const int* expert_offsets, int max_rows, int K, int N, int E, void* y, void* workspace, size_t ws_bytes,
                void* stream) {
  if (int e = check_product_call(ctx, "tl_moe_gemm", TL_MOE_FORWARD, x, w, y, expert_offsets, max_rows, K, N, E, workspace, ws_bytes)) return e;
  ProductParams p;
  memset(&p, 0, sizeof p);
  p.x = (const bf16_t*)x; p.w = (const bf16_t*)w; p.out = (bf16_t*)y; p.offsets = expert_offsets;
  p.max_rows = max_rows; p.K = K; p.N = N; p.E = E;
  return launch_product<false>(ctx, p, (hipStream_t)stream);
}

int tl_moe_gemm_grad_x(tl_ctx* ctx, const void* dy, const void* w, const int* expert_offsets, int max_rows, int K, int N, int E, void* dx, void* workspace,
                       size_t ws_bytes, void* stream) {
  if (int e = check_product_call(ctx, "tl_moe_gemm_grad_x", TL_MOE_GRAD_X, dy, w, dx, expert_offsets, max_rows, K, N, E, workspace, ws_bytes)) return e;
  ProductParams p;
  memset(&p, 0, sizeof p);
  p.dy = (const bf16_t*)dy; p.w = (const bf16_t*)w; p.out = (bf16_t*)dx; p.offsets = expert_offsets;
  p.max_rows = max_rows; p.K = K; p.N = N; p.E = E;
  return launch_product<true>(ctx, p, (hipStream_t)stream);
}

int tl_moe_gemm_grad_w(tl_ctx* ctx, const void* x, const void* dy, const int* expert_offsets, int max_rows, int K, int N, int E, const float* dw_add, void* dw,
                       int dw_f32, void* workspace, size_t ws_bytes, void* stream) {
  if (int e = check_ctx(ctx)) return e;
  if (dw_add && !dw_f32) return fail(TL_ERR_INVALID_ARG, "tl_moe_gemm_grad_w: dw_add needs dw in fp32");
  if (!aligned16(dw_add)) return fail(TL_ERR_INVALID_ARG, "tl_moe_gemm_grad_w: dw_add must be 16-byte aligned");
  if (int e = check_product_call(ctx, "tl_moe_gemm_grad_w", TL_MOE_GRAD_W, x, dy, dw, expert_offsets, max_rows, K, N, E, workspace, ws_bytes)) return e;
  ProductParams p;
  memset(&p, 0, sizeof p);
  p.x = (const bf16_t*)x; p.dy = (const bf16_t*)dy; p.offsets = expert_offsets;
  p.out = (bf16_t*)dw; p.out32 = (float*)dw; p.add = dw_add;
  p.max_rows = max_rows; p.K = K; p.N = N; p.E = E;
  const bool small = small_tiles(ctx, (long)E * ceil_div(K, 256) * ceil_div(N, 256));
  const int tile = small ? 128 : 256;
  p.nbm = ceil_div(K, tile);
  p.nbn = ceil_div(N, tile);
  const long grid = (long)E * p.nbm * p.nbn;
  if (grid >= (1L << 22)) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_moe_gemm_grad_w: E*K*N is too large for one launch");
  hipStream_t s = (hipStream_t)stream;
  if (dw_f32) return small ? launch_fused<CfgW128>(moe_grad_w_kernel<CfgW128, AddRows32>, p, (int)grid, s) : launch_fused<CfgW256>(moe_grad_w_kernel<CfgW256, AddRows32>, p, (int)grid, s);
  return small ? launch_fused<CfgW128>(moe_grad_w_kernel<CfgW128, DenseRows>, p, (int)grid, s) : launch_fused<CfgW256>(moe_grad_w_kernel<CfgW256, DenseRows>, p, (int)grid, s);
}

}  // extern "C"
