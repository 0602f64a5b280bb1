/* Sizes of the attention of pieces at which the number of its workgroups is reckoned from the largest factors, for a UBSan build (no GPU needed).  Built and run by
 * tests/test_chunk_sizes.py; prints "ok <calls>". */
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "../include/nsa_sel.h"

int main(void) {
  const int sequences[] = {1, 255, 256, 16383, 16384, 1 << 24};
  const int heads[] = {1, 255, 256, 1 << 16, 1 << 28, 1 << 30};
  const int windows[] = {0, 1, (1 << 30) - 1, INT32_MAX};
  long calls = 0;
  size_t first = 0;
  for (size_t a = 0; a < sizeof sequences / sizeof *sequences; ++a)
    for (size_t b = 0; b < sizeof heads / sizeof *heads; ++b)
      for (size_t c = 0; c < sizeof windows / sizeof *windows; ++c)
        for (int wide = 0; wide < 2; ++wide) {
          nsa_sel_cache_shape s;
          memset(&s, 0, sizeof s);
          s.n_tokens = 1;
          s.nseq = sequences[a];
          s.hq = s.hkv = heads[b];
          s.d = 128;
          s.page = 16;
          s.n_pages = 1;
          s.max_pages = wide ? 1 << 26 : 1;
          s.window = windows[c];
          size_t n = 0;
          ++calls;
          if (nsa_sel_cache_chunk_workspace_bytes(&s, &n) != NSA_SEL_OK || n == 0 || (first && n != first)) {
            fprintf(stderr, "failed: %d sequences, %d heads\n", s.nseq, s.hkv);
            return 1;
          }
          first = n;
        }
  printf("ok %ld\n", calls);
  return 0;
}
