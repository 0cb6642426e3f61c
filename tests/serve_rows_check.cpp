// The rows of a sequence that the attention kernels work out from token_start and kv_lens (csrc/serve.h), for every mix of
// values that such arrays can hold: never a row outside the call, never more than the bounds.
#include <stdint.h>
#include <stdio.h>

#include <algorithm>

#include "serve.h"

int main() {
  const int32_t least = INT32_MIN, most = INT32_MAX;
  const int32_t numbers[] = {least, least + 1, least + 5, -(1 << 30) - 1, -(1 << 30), -(1 << 24), -7, -1, 0, 1, 3, 4, 5, 6,
                             100, (1 << 24) - 2, (1 << 24) - 1, 1 << 24, 1 << 30, most - 4, most - 1, most};
  int bad = 0;
  for (int32_t num_tokens : {1, 5, 100, (1 << 24) - 1})
    for (int32_t max_tokens : {1, 4, 100, (1 << 24) - 1})
      for (int32_t max_kv : {1, 64, 1 << 30})
        for (int32_t start : numbers)
          for (int32_t end : numbers)
            for (int32_t kv_len : numbers) {
              pkv::ServeArgs s{};
              s.num_tokens = num_tokens;
              s.max_tokens = std::min(max_tokens, num_tokens);
              s.max_kv = max_kv;
              const pkv::SequenceRows r = pkv::rows_of_sequence(s, start, end, kv_len);
              const int64_t first = std::clamp<int64_t>(start, 0, num_tokens), last = std::clamp<int64_t>(end, 0, num_tokens);
              const int64_t count = std::min<int64_t>(last - first, s.max_tokens);
              bool ok = r.kv_len == std::clamp<int64_t>(kv_len, 0, max_kv) && r.trail == last - first;
              ok = ok && (count > 0 ? r.start == first && r.count == count && r.start + r.count <= num_tokens : r.count <= 0);
              if (!ok && bad++ < 10)
                printf("start %d end %d kv_len %d of %d (%d): start %d count %d kv_len %d trail %d\n", start, end, kv_len,
                       num_tokens, s.max_tokens, r.start, r.count, r.kv_len, r.trail);
            }
  printf("%d bad\n", bad);
  return bad != 0;
}
