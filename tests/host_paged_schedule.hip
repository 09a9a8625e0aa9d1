// The checks that stand in front of every use of a schedule, on the host: geometries as the library resolves them (a context made by
// tl_ctx_create_host, 256 compute units), headers as the schedule kernel writes them, in buffers of exactly a schedule's size.
// Prints "host_paged_schedule ok <checks>".
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "tl_paged.h"

using namespace tl;

static int checks = 0, bad = 0;
#define EXPECT(cond) do { checks++; if (!(cond)) { bad++; fprintf(stderr, "line %d: %s failed\n", __LINE__, #cond); } } while (0)

static tl_ctx* ctx;

static tl_paged_dims dims(int batch, int max_tokens, int max_new, int max_blocks) {
  tl_paged_dims d;
  memset(&d, 0, sizeof d);
  d.batch = batch; d.max_tokens = max_tokens; d.max_new = max_new; d.max_blocks = max_blocks;
  d.page_size = 16; d.n_pages = 8192; d.heads_q = 32; d.heads_kv = 8; d.head_dim = 128;
  return d;
}
// A schedule for d in a buffer of its size, with one item.
static int* schedule_for(const tl_paged_dims& d) {
  size_t bytes = 0, ws = 0;
  int info[8];
  PagedGeom g;
  EXPECT(tl_paged_query(ctx, &d, &bytes, &ws, info) == TL_OK && resolve_paged(ctx, &d, &g) == TL_OK);
  int* s = (int*)malloc(bytes);
  memset(s, 0x11, bytes);
  for (int i = 0; i < kSchedHeader; i++) s[i] = sched_header(g, i, 1, 0);
  return s;
}
static bool serves(const int* schedule, const tl_paged_dims& d) {
  PagedGeom g;
  EXPECT(resolve_paged(ctx, &d, &g) == TL_OK);
  return sched_made_for(schedule, g);
}

int main() {
  tl_config cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.world_size = 1; cfg.channels_per_rank = 1;
  if (tl_ctx_create_host(&cfg, 256, &ctx) != TL_OK) return 1;

  // two dims whose fields a multiplicative 32-bit hash does not tell apart
  const tl_paged_dims one = dims(128, 1024, 13, 64), two = dims(256, 4096, 2988, 2048);
  int *s1 = schedule_for(one), *s2 = schedule_for(two);
  EXPECT(serves(s1, one) && serves(s2, two));
  EXPECT(!serves(s2, one) && !serves(s1, two));

  // every field by itself
  const struct { int tl_paged_dims::*field; int value; } other[] = {
      {&tl_paged_dims::batch, 127}, {&tl_paged_dims::max_tokens, 1025}, {&tl_paged_dims::max_new, 12}, {&tl_paged_dims::max_blocks, 65}, {&tl_paged_dims::page_size, 32},
      {&tl_paged_dims::n_pages, 8191}, {&tl_paged_dims::heads_q, 64}, {&tl_paged_dims::heads_kv, 4}, {&tl_paged_dims::window, 1}};
  for (const auto& o : other) {
    tl_paged_dims d = one;
    d.*o.field = o.value;
    EXPECT(!serves(s1, d));
  }
  // the pages' distance may be another for every layer; "no window" and one longer than any request are the same
  tl_paged_dims d = one;
  d.page_stride = 1 << 20;
  EXPECT(serves(s1, d));
  d.window = 0x7fffffff;
  EXPECT(serves(s1, d));
  // one that was never made
  memset(s1, 0, kSchedHeader * 4);
  EXPECT(!serves(s1, one));
  free(s1);
  free(s2);

  // Items are looked for over the launch of the call's own dims, far beyond the end of a schedule of smaller ones: none is found, and
  // nothing behind the header is read.
  const tl_paged_dims least = dims(1, 1, 1, 1), most = dims(4096, 8192, 512, 64);
  int* sl = schedule_for(least);
  PagedGeom gl, gm;
  Item it;
  EXPECT(resolve_paged(ctx, &least, &gl) == TL_OK && resolve_paged(ctx, &most, &gm) == TL_OK && gm.cap_few + gm.cap_tile > 100 * gl.cap_few);
  for (int idx = 0; idx < gm.cap_few + gm.cap_tile; idx++) EXPECT(!sched_item(sl, gm, idx, &it));
  // under its own dims: the items that it has, every one inside the room
  EXPECT(sched_item(sl, gl, 0, &it) && !sched_item(sl, gl, 1, &it));
  for (int i = 0; i < kSchedHeader; i++) sl[i] = sched_header(gl, i, gl.cap_few, 0);
  for (int idx = 0; idx < gl.cap_few; idx++) EXPECT(sched_item(sl, gl, idx, &it) && it.few == 0x11111111);
  EXPECT(!sched_item(sl, gl, gl.cap_few, &it));
  free(sl);

  // another number of compute units: items side by side, and with them room and layout, are others
  tl_ctx* small = nullptr;
  EXPECT(tl_ctx_create_host(&cfg, 64, &small) == TL_OK);
  int* s = schedule_for(one);
  PagedGeom g;
  EXPECT(resolve_paged(small, &one, &g) == TL_OK && !sched_made_for(s, g));
  free(s);
  tl_ctx_destroy(small);
  tl_ctx_destroy(ctx);
  if (bad) { fprintf(stderr, "%d of %d checks failed\n", bad, checks); return 1; }
  printf("host_paged_schedule ok %d\n", checks);
  return 0;
}
