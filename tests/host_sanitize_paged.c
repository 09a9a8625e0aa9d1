/* Walks the host side of the paged-cache operators (dims rules, sizes, argument checks) through a context made by
 * tl_ctx_create_host -- no GPU, no HIP call -- for a build whose host code carries AddressSanitizer and UndefinedBehaviorSanitizer.
 * Every dims that the query accepts must fit the room it states; prints "host_sanitize_paged ok <calls>". */
#include <stdio.h>
#include <string.h>

#include "tilelink_mi355.h"

static int calls = 0, bad = 0;
#define EXPECT(cond) do { calls++; if (!(cond)) { bad++; fprintf(stderr, "line %d: %s failed (%s)\n", __LINE__, #cond, tl_last_error()); } } while (0)

int main(void) {
  static const int batches[] = {1, 63, 4096}, tokens[] = {1, 100, 1 << 18}, news[] = {0, 1, 7}, blocks[] = {1, 1000, 1 << 20}, pages[] = {16, 64, 256};
  static const int heads[][2] = {{1, 1}, {8, 1}, {40, 1}, {1024, 1}, {1024, 1024}, {30, 6}}, windows[] = {0, 1, 0x7fffffff}, cus[] = {1, 104, 256, 4000};
  tl_config cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.world_size = 1; cfg.channels_per_rank = 1;
  char mem[256];                                   /* addresses that nothing may follow */
  void* p = (void*)(((size_t)mem + 127) / 128 * 128);
  int* ip = (int*)p;
  for (unsigned c = 0; c < sizeof cus / sizeof *cus; c++) {
    tl_ctx* ctx = NULL;
    EXPECT(tl_ctx_create_host(&cfg, cus[c], &ctx) == TL_OK);
    if (!ctx) continue;
    for (unsigned b = 0; b < 3; b++) for (unsigned t = 0; t < 3; t++) for (unsigned n = 0; n < 3; n++) for (unsigned k = 0; k < 3; k++)
      for (unsigned g = 0; g < 3; g++) for (unsigned h = 0; h < 6; h++) for (unsigned w = 0; w < 3; w++) {
        tl_paged_dims d;
        memset(&d, 0, sizeof d);
        d.batch = batches[b]; d.max_tokens = tokens[t]; d.max_new = news[n]; d.max_blocks = blocks[k]; d.page_size = pages[g];
        d.n_pages = (int)(0x7fffffffLL / pages[g]); d.heads_q = heads[h][0]; d.heads_kv = heads[h][1]; d.head_dim = 128; d.window = windows[w];
        size_t sched = 0, ws = 0;
        int info[8];
        int e = tl_paged_query(ctx, &d, &sched, &ws, info);
        calls++;
        if (e != TL_OK) { EXPECT(e == TL_ERR_INVALID_ARG || e == TL_ERR_UNSUPPORTED_SHAPE); continue; }
        EXPECT(info[3] >= 0 && info[4] >= 0 && info[3] + info[4] > 0 && sched >= 64 + 48 * ((size_t)info[3] + info[4]) && ws >= 32768);
        const long long row = 128LL * d.heads_q, kv = 128LL * d.heads_kv;
        EXPECT(tl_paged_schedule(ctx, &d, ip, ip, ip, sched, NULL) == TL_ERR_INVALID_ARG);            /* the context, nothing else */
        EXPECT(strstr(tl_last_error(), "tl_ctx_create_host") != NULL);
        EXPECT(tl_paged_attention(ctx, &d, p, row, p, p, ip, ip, p, row, NULL, 0.1f, p, ws, NULL) == TL_ERR_INVALID_ARG);
        EXPECT(strstr(tl_last_error(), "tl_ctx_create_host") != NULL);
        EXPECT(tl_paged_attention(ctx, &d, p, row, p, p, ip, ip, p, row, NULL, 0.1f, p, ws - 1, NULL) == TL_ERR_WORKSPACE_TOO_SMALL);
        EXPECT(tl_qk_norm_rope_cache(ctx, &d, p, row, p, kv, p, kv, p, row, p, p, ip, NULL, NULL, 0.f, ip, (float*)p, 1, 128, 0, NULL) == TL_ERR_INVALID_ARG);
        EXPECT(strstr(tl_last_error(), "tl_ctx_create_host") != NULL);
        EXPECT(tl_paged_slots(ctx, &d, ip, ip, ip, 1, NULL, NULL, ip, ip, ip, ip, ip, ip, NULL) == TL_ERR_INVALID_ARG);
        EXPECT(strstr(tl_last_error(), "tl_ctx_create_host") != NULL);
      }
    EXPECT(tl_paged_query(ctx, NULL, NULL, NULL, NULL) == TL_ERR_INVALID_ARG);
    EXPECT(tl_qk_norm_rope(ctx, p, 128, p, 128, p, 128, p, 128, 0x7fffffff, 1, 1, 128, NULL, NULL, 0.f, ip, (float*)p, 1, 128, 0, NULL) == TL_ERR_INVALID_ARG);
    EXPECT(tl_ctx_destroy(ctx) == TL_OK);
  }
  if (bad) { fprintf(stderr, "%d of %d checks failed\n", bad, calls); return 1; }
  printf("host_sanitize_paged ok %d\n", calls);
  return 0;
}
