/* Host-side exercise of the rotation, the read of a cache and the attention of pieces of prompts for an AddressSanitizer / UBSan build (no GPU needed): workspace sizes of shapes
 * at the limits and past them, and the refusals that come before any launch.  Built and run by tests/test_more_operators_build.py; prints "ok <calls>". */
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "../include/nsa_sel.h"

#define CHECK(cond)                                                     \
  do {                                                                  \
    if (!(cond)) {                                                      \
      fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); \
      return 1;                                                         \
    }                                                                   \
  } while (0)

int main(void) {
  long calls = 0, good = 0;
  const int tokens[] = {0, 1, 2, 65, 4096, 1 << 20, (1 << 28) - 1, INT32_MAX, -1, INT32_MIN};
  const int heads[][2] = {{1, 1}, {8, 8}, {5, 1}, {28, 4}, {64, 8}, {16, 1}, {17, 1}, {8, 3}, {0, 0}, {8, 0}, {2147483640, 2147483640}, {2147483647, 1}};
  const int pages[] = {16, 64, 256, 8, 0, 48, 512, INT32_MIN};
  const int widths[] = {0, 1, 1000, 1 << 22, 1 << 26, INT32_MAX, -1};
  const int windows[] = {0, 1, INT32_MAX, -1};
  const int64_t strides[] = {0, 8, 128, 1024, INT64_MAX, INT64_MAX - 7, INT64_MIN, -1024};
  void* p = (void*)(uintptr_t)4096;
  void* q = (void*)(uintptr_t)8192;
  void* odd = (void*)(uintptr_t)4098;
  for (size_t a = 0; a < sizeof tokens / sizeof *tokens; ++a)
    for (size_t b = 0; b < sizeof heads / sizeof *heads; ++b)
      for (size_t c = 0; c < sizeof pages / sizeof *pages; ++c)
        for (size_t d = 0; d < sizeof widths / sizeof *widths; ++d)
          for (size_t f = 0; f < sizeof windows / sizeof *windows; ++f)
            for (int k = 0; k < 8; ++k) {
              nsa_sel_cache_shape s;
              memset(&s, 0, sizeof s);
              s.n_tokens = tokens[a];
              s.nseq = k % 4 == 0 ? tokens[a] : k % 4 == 1 ? 1 : k % 4 == 2 ? 1 << 20 : INT32_MAX;
              s.hq = heads[b][0];
              s.hkv = heads[b][1];
              s.d = 128;
              s.dtype = k & 1;
              s.page = pages[c];
              s.n_pages = k < 4 ? 7 : INT32_MAX;
              s.max_pages = widths[d];
              s.block = 64;
              s.window = windows[f];
              size_t n = 0;
              const int rc = nsa_sel_cache_chunk_workspace_bytes(&s, &n);
              calls += 2;
              CHECK(rc == NSA_SEL_OK || rc == NSA_SEL_EINVAL || rc == NSA_SEL_EUNSUPPORTED);
              CHECK(nsa_sel_cache_chunk_workspace_bytes(&s, NULL) == rc);
              CHECK(nsa_sel_cache_read(&s, p, p, p, p, p, p, p, q, 8, q, INT64_MIN, NULL) != NSA_SEL_OK || s.n_tokens == 0);
              if (rc != NSA_SEL_OK) {
                CHECK(nsa_sel_cache_attention_chunk(&s, p, p, p, p, p, p, p, p, NULL, NULL, q, p, p, (size_t)1 << 62, NULL) == rc);
                continue;
              }
              ++good;
              CHECK(n < (size_t)1 << 30);
              if (s.n_tokens == 0) {
                CHECK(nsa_sel_cache_attention_chunk(&s, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, 0, NULL) == NSA_SEL_OK);
                continue;
              }
              CHECK(nsa_sel_cache_attention_chunk(&s, NULL, p, p, p, p, p, p, p, NULL, NULL, q, p, p, n, NULL) == NSA_SEL_EINVAL);
              CHECK(nsa_sel_cache_attention_chunk(&s, odd, p, p, p, p, p, p, p, NULL, NULL, q, p, p, n, NULL) == NSA_SEL_EINVAL);
              CHECK(nsa_sel_cache_attention_chunk(&s, p, p, p, p, p, p, p, p, NULL, p, q, p, p, n, NULL) == NSA_SEL_EINVAL);
              CHECK(nsa_sel_cache_attention_chunk(&s, p, p, p, p, p, p, p, p, NULL, NULL, p, p, p, n, NULL) == NSA_SEL_EINVAL);
              CHECK(nsa_sel_cache_attention_chunk(&s, p, p, p, p, p, p, p, p, NULL, NULL, q, p, p, n - 1, NULL) == NSA_SEL_EWORKSPACE);
              CHECK(nsa_sel_cache_attention_chunk(&s, p, p, p, p, p, p, p, p, NULL, NULL, q, p, NULL, n, NULL) == NSA_SEL_EINVAL);
              calls += 6;
            }
  for (size_t a = 0; a < sizeof tokens / sizeof *tokens; ++a)
    for (size_t b = 0; b < sizeof heads / sizeof *heads; ++b)
      for (size_t c = 0; c < sizeof strides / sizeof *strides; ++c)
        for (int rot = -16; rot <= 160; rot += 8) {
          nsa_sel_rotary_shape s;
          memset(&s, 0, sizeof s);
          s.n_tokens = tokens[a];
          s.nseq = c & 1 ? 1 : tokens[a];
          s.hq = heads[b][0];
          s.hkv = heads[b][1];
          s.d = 128;
          s.rot = rot;
          s.factor = 1.0;
          // one pointer is odd: no call gets as far as a launch
          const int rc = nsa_sel_rotary(&s, p, strides[c], heads[b][1] > 0 ? p : NULL, strides[c], p, NULL, p, odd, strides[c], heads[b][1] > 0 ? q : NULL, strides[c], NULL);
          ++calls;
          CHECK(rc == NSA_SEL_EINVAL || rc == NSA_SEL_EUNSUPPORTED || (rc == NSA_SEL_OK && s.n_tokens == 0));
        }
  CHECK(nsa_sel_cache_chunk_workspace_bytes(NULL, NULL) == NSA_SEL_EINVAL);
  CHECK(nsa_sel_rotary(NULL, p, 8, p, 8, p, p, p, q, 8, q, 8, NULL) == NSA_SEL_EINVAL);
  CHECK(good > 100);
  printf("ok %ld\n", calls);
  return 0;
}
