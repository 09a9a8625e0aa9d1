// Which kernel a call of a mixture-of-experts layer in training takes, by the library's own rules (256 compute units): reads one call a line from
// the standard input, prints its kernel.  Built with the host compiler pass alone; nothing is launched.
//   sort T topk E | route_grad E topk | dispatch, dispatch_grad, combine, combine_grad T H topk max_rows | gemm, gemm_grad_x, gemm_grad_w max_rows K N E
#include <string>

#include "tl_moe_choice.h"

using namespace tl;

static std::string product(const tl_ctx* ctx, bool grad_x, int max_rows, int K, int N, int E) {
  const ProductShape s = product_shape(ctx, grad_x, max_rows, K, N, E);
  if (s.tile) return "tiles " + std::to_string(s.tile) + (s.cut ? " cut" : " whole");
  const FewChoice c = few_choice(ctx, grad_x, max_rows, E, grad_x ? K : N);
  return std::string("few ") + (c.wide ? "wide " : "narrow ") + std::to_string(c.waves) + " " + std::to_string(c.beside);
}
static std::string flags(const RowsChoice& c) { return std::string(c.stream_loads ? " stream" : " cached") + (c.stream_stores ? " stream" : " cached"); }

int main() {
  tl_config cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.world_size = 1; cfg.channels_per_rank = 1;
  tl_ctx* ctx;
  if (tl_ctx_create_host(&cfg, 256, &ctx) != TL_OK) return 1;
  char line[256], word[32];
  int a, b, c, d;
  while (fgets(line, sizeof line, stdin)) {
    a = b = c = d = 0;
    if (sscanf(line, "%31s %d %d %d %d", word, &a, &b, &c, &d) < 3) return 1;
    const std::string op = word;
    std::string kernel;
    if (op == "sort") kernel = (sort_chunks((long)a * b) == 1 ? "one chunk " : "chunks ") + std::to_string(sort_rows_per_thread((long)a * b));
    else if (op == "route_grad") kernel = std::to_string(route_lanes(b)) + " " + std::to_string(route_per(a, route_lanes(b)));
    else if (op == "dispatch") kernel = flags(dispatch_choice(a, b, c, d));
    else if (op == "dispatch_grad" || op == "combine") kernel = flags(gather_choice(a, b, c, d));
    else if (op == "combine_grad") kernel = std::to_string(combine_grad_choice(a, b, c, d).waves) + flags(combine_grad_choice(a, b, c, d));
    else if (op == "gemm" || op == "gemm_grad_x") kernel = product(ctx, op == "gemm_grad_x", a, b, c, d);
    else if (op == "gemm_grad_w") {
      const GradWShape s = grad_w_shape(ctx, a, b, c, d);
      kernel = std::to_string(s.bm) + "x" + std::to_string(s.bn) + (s.places ? " cut" : " whole");
    } else return 1;
    printf("%s %s\n", op.c_str(), kernel.c_str() + (kernel[0] == ' '));
  }
  tl_ctx_destroy(ctx);
  return 0;
}
