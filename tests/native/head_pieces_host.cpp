// Host-only check of how the backward pass of the losses at the output projection cuts the vocabulary: the piece that head_piece takes costs, by the model of
// rounds and steps that it states, at most a hundredth more than the best of its candidates, each summed here over the pieces as the call goes through them.
#include <cstdint>
#include <cstdio>

#include "eco_head.hpp"

namespace eco { uint64_t dim_tile(int shape, uint64_t dim); }

static uint64_t up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

static double cost_of(uint64_t rows, uint64_t dim, uint64_t vocab, uint64_t piece) {
  const uint64_t tile = eco::dim_tile(eco::HEAD_LARGE, dim);
  double cost = 0;
  for (uint64_t first = 0; first < vocab; first += piece) {
    const uint64_t n = up(vocab - first < piece ? vocab - first : piece, 256);
    cost += (double)up(n * up(rows, 256), 256) * ((double)dim / 64 + 8) + (double)up(n * up(dim, tile), 256) * ((double)rows / 64 + 8) * (double)tile / 256;
  }
  return cost;
}

int main() {
  const uint64_t rows_of[] = {129, 700, 2047, 4096, 8192, 20000}, dims[] = {64, 512, 576, 1024, 1152, 2048, 2500},
                 vocabs[] = {32000, 50304, 65536, 100501, 102400, 131072, 200000, 262144, 1 << 20};
  int bad = 0, checked = 0, even = 0;
  for (uint64_t rows : rows_of)
    for (uint64_t dim : dims)
      for (uint64_t vocab : vocabs) {
        const uint64_t all = up(vocab, 256);
        for (uint64_t most : {all * 256, ((uint64_t{512} << 20) / (2 * up(rows, 256) * 256)) / 256 * 256, (uint64_t)8192}) {
          if (most > all * 256) most = all * 256;
          const uint64_t piece = eco::head_piece(eco::HEAD_LARGE, rows, dim, vocab, most);
          if (piece == 0 || piece % 256 || piece > most) { std::printf("FAILED: a piece of %llu, at most %llu\n", (unsigned long long)piece, (unsigned long long)most); return 1; }
          const uint64_t fewest = up(all, most / 256);
          double best = 1e300;
          for (uint64_t pieces = fewest; pieces <= 2 * fewest && pieces <= all && pieces < fewest + 64; ++pieces) {
            const double c = cost_of(rows, dim, vocab, up(all, pieces) * 256);
            if (c < best) best = c;
            even += all % pieces == 0;
          }
          ++checked;
          if (0.99 * cost_of(rows, dim, vocab, piece) > best) {
            if (++bad <= 10)
              std::printf("FAILED: %llu x %llu x %llu, at most %llu: pieces of %llu cost %g, the best %g\n", (unsigned long long)rows, (unsigned long long)dim,
                          (unsigned long long)vocab, (unsigned long long)most, (unsigned long long)piece, cost_of(rows, dim, vocab, piece), best);
          }
        }
      }
  if (bad || !even) return 1;
  std::printf("pieces ok: %d\n", checked);
  return 0;
}
