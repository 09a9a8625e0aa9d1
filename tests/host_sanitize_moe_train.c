/* Walks the host side of a mixture-of-experts layer's training operators (sizes, limits, argument checks) through a context made by
 * tl_ctx_create_host -- no GPU, no HIP call -- for a build whose host code carries AddressSanitizer and UndefinedBehaviorSanitizer.
 * Prints "host_sanitize_moe_train ok <calls>". */
#include <stdio.h>
#include <string.h>

#include "tilelink_mi355.h"

static int calls = 0, bad = 0;
#define EXPECT(cond) do { calls++; if (!(cond)) { bad++; fprintf(stderr, "line %d: %s failed (%s)\n", __LINE__, #cond, tl_last_error()); } } while (0)
#define STOPPED_BY_CONTEXT(call) do { EXPECT((call) == TL_ERR_INVALID_ARG); EXPECT(strstr(tl_last_error(), "tl_ctx_create_host") != NULL); } while (0)

int main(void) {
  static const int rows[] = {1, 255, 4097, 1 << 20, 0x7fffffff}, dims[] = {8, 136, 2056, 8192, 1 << 20}, experts[] = {1, 7, 256}, cus[] = {1, 104, 256, 4000};
  static const int tokens[] = {1, 1000, 1 << 15, 1 << 20, 0x7fffffff}, topks[] = {1, 5, 32, 33};
  tl_config cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.world_size = 1; cfg.channels_per_rank = 1;
  char mem[256];                                   /* addresses that nothing may follow */
  void* p = (void*)(((size_t)mem + 127) / 128 * 128);
  int* ip = (int*)p;
  float* fp = (float*)p;
  for (unsigned c = 0; c < sizeof cus / sizeof *cus; c++) {
    tl_ctx* ctx = NULL;
    EXPECT(tl_ctx_create_host(&cfg, cus[c], &ctx) == TL_OK);
    if (!ctx) continue;
    for (unsigned e = 0; e < 3; e++) for (unsigned r = 0; r < 5; r++) for (unsigned k = 0; k < 5; k++) for (unsigned n = 0; n < 5; n++) {
      const int R = rows[r], K = dims[k], N = dims[n], E = experts[e];
      size_t ws = 0;
      EXPECT(tl_moe_gemm_query(ctx, TL_MOE_FORWARD, R, K, N, E, &ws) == TL_OK && ws >= 128);
      STOPPED_BY_CONTEXT(tl_moe_gemm(ctx, p, p, ip, R, K, N, E, p, p, ws, NULL));
      EXPECT(tl_moe_gemm(ctx, p, p, ip, R, K, N, E, p, p, ws - 1, NULL) == TL_ERR_WORKSPACE_TOO_SMALL);
      EXPECT(tl_moe_gemm_query(ctx, TL_MOE_GRAD_X, R, K, N, E, &ws) == TL_OK && ws >= 128);
      STOPPED_BY_CONTEXT(tl_moe_gemm_grad_x(ctx, p, p, ip, R, K, N, E, p, p, ws, NULL));
      const int st = tl_moe_gemm_query(ctx, TL_MOE_GRAD_W, R, K, N, E, &ws);
      if (st != TL_OK) { EXPECT(st == TL_ERR_UNSUPPORTED_SHAPE && (long long)E * ((K + 127) / 128) * ((N + 127) / 128) >= 1 << 22); continue; }
      STOPPED_BY_CONTEXT(tl_moe_gemm_grad_w(ctx, p, p, ip, R, K, N, E, fp, p, 1, p, ws, NULL));
      STOPPED_BY_CONTEXT(tl_moe_gemm_grad_w(ctx, p, p, ip, R, K, N, E, NULL, p, 0, p, ws, NULL));
      EXPECT(tl_moe_gemm_grad_w(ctx, p, p, ip, R, K, N, E, NULL, p, 0, p, ws - 1, NULL) == TL_ERR_WORKSPACE_TOO_SMALL);
    }
    for (unsigned t = 0; t < 5; t++) for (unsigned k = 0; k < 4; k++) for (unsigned e = 0; e < 3; e++) {
      const int T = tokens[t], topk = topks[k], E = experts[e];
      size_t ws = 0;
      const int st = tl_moe_sort_query(ctx, T, topk, E, &ws);
      if (st == TL_OK) {
        STOPPED_BY_CONTEXT(tl_moe_sort(ctx, ip, T, topk, 0, E, ip, ip, ip, p, ws, NULL));
        EXPECT(tl_moe_sort(ctx, ip, T, topk, 0x7fffffff, E, ip, ip, ip, p, ws, NULL) == TL_ERR_INVALID_ARG);
        EXPECT(tl_moe_sort(ctx, ip, T, topk, 0, E, ip, ip, ip, p, ws - 1, NULL) == TL_ERR_WORKSPACE_TOO_SMALL);
      } else {
        EXPECT(st == TL_ERR_UNSUPPORTED_SHAPE && (topk > 32 || (long long)T * topk > 1 << 20));
      }
      for (unsigned r = 0; r < 5; r++) {
        const int a = tl_moe_dispatch(ctx, p, ip, T, dims[4], topk, rows[r], p, NULL), b = tl_moe_dispatch_grad(ctx, p, ip, T, 8, topk, rows[r], p, NULL);
        const int d = tl_moe_combine(ctx, p, fp, ip, T, 2056, topk, rows[r], NULL, p, NULL), f = tl_moe_combine_grad(ctx, p, p, fp, ip, T, 8, topk, rows[r], p, fp, NULL);
        const int want = topk > 32 || (long long)T * topk >= 1LL << 31 ? TL_ERR_UNSUPPORTED_SHAPE : TL_ERR_INVALID_ARG;
        EXPECT(a == want && b == want && d == want && f == want);
      }
      const int g = tl_moe_route_grad(ctx, fp, ip, fp, T, E, topk, 1, fp, NULL);
      EXPECT(g == (topk > 32 || topk > E || T > 1 << 24 ? TL_ERR_UNSUPPORTED_SHAPE : TL_ERR_INVALID_ARG));
    }
    EXPECT(tl_ctx_destroy(ctx) == TL_OK);
  }
  if (bad) { printf("%d of %d failed\n", bad, calls); return 1; }
  printf("host_sanitize_moe_train ok %d\n", calls);
  return 0;
}
