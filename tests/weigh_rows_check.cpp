// The rows that the kernels of attention weights go over for a tile of tokens (csrc/serve.h): always rows of the sequence,
// and among them every row that sees a token of the tile.
#include <stdint.h>
#include <stdio.h>

#include "serve.h"

int main() {
  int bad = 0;
  auto check = [&](const pkv::SequenceRows& g, int32_t begin, int32_t last, int32_t window, int32_t sinks) {
    const pkv::RowRange r = pkv::rows_that_see(g, begin, last, window, sinks);
    bool ok = r.first >= 0 && r.first <= r.end && r.end <= (g.count > 0 ? g.count : 0);
    if (g.count < 200)
      for (int32_t i = 0; i < g.count; ++i) {
        const int64_t pos = int64_t(g.kv_len) - g.trail + i;
        bool sees = false;
        for (int64_t t = begin; t <= last && t <= pos; ++t) sees = sees || window == 0 || pos - t < window || t < sinks;
        ok = ok && (!sees || (i >= r.first && i < r.end));
      }
    if (!ok && bad++ < 10)
      printf("count %d trail %d kv_len %d tokens %d..%d window %d sinks %d: rows %d..%d\n", g.count, g.trail, g.kv_len,
             begin, last, window, sinks, r.first, r.end);
  };
  for (int32_t kv_len : {1, 5, 40, 300})
    for (int32_t trail : {-3, 0, 1, 4, 39, 64})
      for (int32_t most : {1, 3, 64})
        for (int32_t begin = 0; begin < kv_len; begin += 16)
          for (int32_t window : {0, 1, 7, 50, 1 << 30, INT32_MAX})
            for (int32_t sinks : {0, 3, 20, INT32_MAX}) {
              const pkv::SequenceRows g{0, trail < most ? trail : most, kv_len, trail};
              const int32_t last = begin + 15 < kv_len ? begin + 15 : kv_len - 1;
              check(g, begin, last, window, sinks);
            }
  const int32_t top = 1 << 30;  // far from the rows, either way
  for (int32_t kv_len : {20000, top})
    for (int32_t count : {1, 60, 5000})
      for (int32_t begin : {0, 256, 12800, top - 256})
        for (int32_t window : {0, 1, 100, INT32_MAX}) check(pkv::SequenceRows{0, count, kv_len, count}, begin, begin + 255, window, 4);
  printf("%d bad\n", bad);
  return bad != 0;
}
