// pic_page_blocks on blocks whose source tokens lie anywhere, also where counting on from them leaves 32 bits (run under
// UndefinedBehaviorSanitizer).  What lies past a pool's end the composition skips, so no piece of such a block may name a
// token of one.  Prints "blocks driver: OK".
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "pic.h"

int main() {
  const pic_pages pg = {8, 16, 8};
  const int32_t table[8] = {3, 1, 7, 0, 2, 4, 5, 6};
  const int32_t sources[] = {0, -5, INT32_MIN, INT32_MAX, INT32_MAX - 15, INT32_MAX - 63, INT32_MAX - 64};
  for (int32_t src : sources)
    for (int32_t dst : {0, 9, 63}) {
      const pic_block b = {0, src, dst, 64, 5};
      pic_block out[8];
      int32_t n = 0;
      if (pic_page_blocks(&pg, 1, table, &b, 1, out, 8, &n) != PIC_OK) return 1;
      int32_t t = 0;
      for (int32_t i = 0; i < n; ++i) {
        const int64_t want = (int64_t)src + t;
        if (want <= INT32_MAX ? out[i].src_token != want : out[i].src_token >= 0) {
          std::fprintf(stderr, "block from %d at slot %d: piece %d from %d\n", src, dst, i, out[i].src_token);
          return 1;
        }
        t += out[i].n_tokens;
      }
      if (t != 64) return 1;
    }
  std::printf("blocks driver: OK\n");
}
