// Host-only: the tiles and splits that the feed-forward products take for sizes given on the command line, a line each.
//   forward END ROWS IN_DIM WIDTH GROUP FMT EXACT     END 0 linear, 1 gated, 2 the gated unit's backward pass
//   gradients MATRICES ROWS IN_DIM WIDTH
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "eco_ffn.hpp"

int main(int argc, char **argv) {
  const auto number = [&](int i) { return static_cast<uint64_t>(std::strtoull(argv[i], nullptr, 10)); };
  for (int i = 1; i < argc;) {
    if (!std::strcmp(argv[i], "forward") && i + 7 < argc) {
      eco::FfnWeights w;
      std::memset(&w, 0, sizeof w);
      const uint64_t dim = number(i + 3), width = number(i + 4), group = number(i + 5);
      w.matrices = number(i + 1) ? 2 : 1;
      w.rows = static_cast<uint32_t>(width);
      w.dim = static_cast<uint32_t>(dim);
      w.fmt = static_cast<int>(number(i + 6));
      w.group_blocks = group >= dim ? 0 : static_cast<uint32_t>(group / eco::FFN_BLOCK);
      const eco::FfnPlan p = eco::ffn_plan(static_cast<int>(number(i + 1)), w, number(i + 2), number(i + 7) != 0);
      std::printf("%d %d %u %u %u\n", p.rows_tile, p.width_tile, p.split.whole, p.split.tail, p.split.splits);
      i += 8;
    } else if (!std::strcmp(argv[i], "gradients") && i + 4 < argc) {
      const uint64_t matrices = number(i + 1), rows = number(i + 2), dim = number(i + 3), width = number(i + 4), half = eco::ffn_round_up(width, 64);
      const eco::FfnGradPlan p = eco::ffn_grad_plan({dim, rows, matrices == 2 ? 2 * half : width, 1}, {dim, width, rows, static_cast<uint32_t>(matrices)});
      std::printf("%d %u %u %u %u %u\n", p.shape, p.of_input, p.input.whole, p.input.splits, p.weights.whole, p.weights.splits);
      i += 5;
    } else {
      std::fprintf(stderr, "unknown: %s\n", argv[i]);
      return 1;
    }
  }
  return 0;
}
