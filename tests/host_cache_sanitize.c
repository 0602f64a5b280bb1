/* Host-side exercise of the C ABI over a paged cache for an AddressSanitizer / UBSan build (no GPU needed): workspace sizes of shapes at the limits and
 * past them, and the refusals that come before any launch.  Built and run by tests/test_cache_host_sanitizers.py; prints "ok <calls>". */
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
  const int tokens[] = {0, 1, 2, 48, 65, 512, 4096, 1 << 20, 1 << 26, (1 << 28) - 1, INT32_MAX};
  const int heads[][2] = {{1, 1}, {8, 8}, {5, 1}, {28, 4}, {64, 8}, {9, 1}, {8, 3}, {0, 0}, {2147483640, 2147483640}};
  const int pages[] = {16, 64, 256, 8, 0, 48, 512, -16, INT32_MIN};
  const int widths[] = {0, 1, 5, 1000, 1 << 22, 1 << 26, INT32_MAX, -1};
  const int topks[] = {0, 1, 16, 32, 33, -1};
  const int windows[] = {0, 1, 512, INT32_MAX, -1};
  void* p = (void*)(uintptr_t)4096;
  void* q = (void*)(uintptr_t)8192;
  void* odd = (void*)(uintptr_t)4098;
  for (size_t a = 0; a < sizeof tokens / sizeof *tokens; ++a)
    for (size_t b = 0; b < sizeof heads / sizeof *heads; ++b)
      for (size_t c = 0; c < sizeof pages / sizeof *pages; ++c)
        for (size_t d = 0; d < sizeof widths / sizeof *widths; ++d)
          for (size_t e = 0; e < sizeof topks / sizeof *topks; ++e)
            for (size_t f = 0; f < sizeof windows / sizeof *windows; ++f)
              for (int k = 0; k < 6; ++k) {
                nsa_sel_cache_shape s;
                memset(&s, 0, sizeof s);
                s.n_tokens = tokens[a];
                s.nseq = k % 3 == 0 ? tokens[a] : k % 3 == 1 ? 1 : 1 << 20;
                s.hq = heads[b][0];
                s.hkv = heads[b][1];
                s.d = 128;
                s.dtype = k & 1;
                s.page = pages[c];
                s.n_pages = 7;
                s.max_pages = widths[d];
                s.block = e & 1 ? 64 : 128;
                s.topk = topks[e];
                s.window = windows[f];
                size_t n = 0;
                const int rc = nsa_sel_cache_workspace_bytes(&s, &n);
                ++calls;
                CHECK(rc == NSA_SEL_OK || rc == NSA_SEL_EINVAL || rc == NSA_SEL_EUNSUPPORTED);
                if (rc != NSA_SEL_OK) {
                  CHECK(nsa_sel_cache_attention(&s, p, p, p, p, p, p, p, p, p, NULL, NULL, q, p, p, (size_t)1 << 62, NULL) == rc);
                  continue;
                }
                ++good;
                CHECK(n < (size_t)1 << 60);
                const int32_t* idx = s.topk ? p : NULL;
                if (s.n_tokens == 0) {
                  CHECK(nsa_sel_cache_attention(&s, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL, 0, NULL) == NSA_SEL_OK);
                  CHECK(nsa_sel_cache_append(&s, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, NULL, NULL, 128, 0, NULL, NULL, NULL, NULL, NULL, NULL, NULL) == NSA_SEL_OK);
                  continue;
                }
                CHECK(nsa_sel_cache_attention(&s, NULL, idx, p, p, p, p, p, p, p, NULL, NULL, q, p, p, n, NULL) == NSA_SEL_EINVAL);
                CHECK(nsa_sel_cache_attention(&s, odd, idx, p, p, p, p, p, p, p, NULL, NULL, q, p, p, n, NULL) == NSA_SEL_EINVAL);
                CHECK(nsa_sel_cache_attention(&s, p, s.topk ? NULL : p, p, p, p, p, p, p, p, NULL, NULL, q, p, p, n, NULL) == NSA_SEL_EINVAL);
                if (n > 0) CHECK(nsa_sel_cache_attention(&s, p, idx, p, p, p, p, p, p, p, NULL, NULL, q, p, p, n - 1, NULL) == NSA_SEL_EWORKSPACE);
                CHECK(nsa_sel_cache_append(&s, p, INT64_MAX, p, INT64_MAX, p, INT64_MAX, p, p, p, p, 128, 0, p, p, p, p, q, NULL, NULL) == NSA_SEL_EINVAL);
                CHECK(nsa_sel_cache_append(&s, p, 8, p, 8, p, INT64_MIN, p, p, p, p, 16, 0, p, p, p, p, q, NULL, NULL) == NSA_SEL_EINVAL);
                CHECK(nsa_sel_cache_append(&s, NULL, 0, p, (int64_t)s.hkv * 128, p, (int64_t)s.hkv * 128, p, p, p, NULL, 16, 0, p, p, p, p, NULL, NULL, NULL) == NSA_SEL_EINVAL);
                CHECK(nsa_sel_select_blocks_cached(&s, p, 8, p, NULL, 1, 2, p, NULL) != NSA_SEL_OK);
                CHECK(nsa_sel_select_blocks_cached(&s, p, 0, p, p, 1, 2, p, NULL) != NSA_SEL_OK);
                calls += 8;
              }
  CHECK(nsa_sel_cache_workspace_bytes(NULL, NULL) == NSA_SEL_EINVAL);
  CHECK(good > 100);
  printf("ok %ld\n", calls);
  return 0;
}
