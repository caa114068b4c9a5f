// Host-side checks of the 8-bit cache's C ABI for a build with AddressSanitizer and UndefinedBehaviorSanitizer on the host
// code: each case fails validation before any HIP call, or is host arithmetic alone.  Exit status 0 when every call
// returns the expected status.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "arckv.h"

static int failures = 0;
#define EXPECT(call, want)                                                                              \
  do {                                                                                                  \
    const int got_ = (int)(call);                                                                       \
    if (got_ != (int)(want)) {                                                                          \
      printf("FAIL line %d: %s returned %d, expected %d\n", __LINE__, #call, got_, (int)(want));        \
      ++failures;                                                                                       \
    }                                                                                                   \
  } while (0)

int main() {
  void *fake = (void *)0x1000, *odd = (void *)0x1001, *ws = (void *)0x10000;
  float *f = (float *)fake;
  int32_t *i = (int32_t *)fake;
  const arckv_qcache good = {2, 100, 128, ARCKV_E4M3, fake, fake, f, f, fake};
  arckv_qcache bad[6] = {good, good, good, good, good, good};
  bad[0].P = 0;
  bad[1].rows = -5;
  bad[2].K = odd;
  bad[3].K_scale = nullptr;
  bad[4].rows = INT32_MIN;
  bad[5].P = INT32_MIN;
  for (const arckv_qcache &c : bad) {
    EXPECT(arckv_qcache_write(&c, 1, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
    EXPECT(arckv_qcache_read(&c, 0, 1, ARCKV_BF16, nullptr, fake, fake, nullptr), ARCKV_ERR_INVALID_ARG);
    EXPECT(arckv_select_blocks(&c, 4, 0.0f, fake, nullptr, nullptr, 1, f, i, nullptr), ARCKV_ERR_INVALID_ARG);
    EXPECT(arckv_attend_qcache(&c, 4, 0, 0, 0.0f, fake, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, f, ws,
                               (size_t)1 << 40, nullptr), ARCKV_ERR_INVALID_ARG);
  }
  arckv_qcache c = good;
  c.d = 64;
  EXPECT(arckv_qcache_write(&c, 1, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_UNSUPPORTED);
  c = good;
  c.format = 7;
  EXPECT(arckv_qcache_read(&c, 0, 1, ARCKV_BF16, nullptr, fake, fake, nullptr), ARCKV_ERR_UNSUPPORTED);
  c = good;
  c.rows = INT32_MAX;
  EXPECT(arckv_attend_qcache(&c, 4, 0, 0, 0.0f, fake, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, f, ws,
                             (size_t)1 << 40, nullptr), ARCKV_ERR_UNSUPPORTED);
  EXPECT(arckv_qcache_write(nullptr, 1, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_qcache_write(&good, INT32_MAX, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_UNSUPPORTED);
  EXPECT(arckv_qcache_write(&good, 101, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_qcache_write(&good, INT32_MIN, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_qcache_read(&good, INT32_MAX, INT32_MAX, ARCKV_F32, nullptr, fake, fake, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_qcache_read(&good, INT32_MIN, 1, ARCKV_F32, nullptr, fake, fake, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_select_blocks(&good, 4, INFINITY, fake, nullptr, nullptr, 1, f, i, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_select_blocks(&good, 4, 0.0f, fake, nullptr, nullptr, INT32_MAX, f, i, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_select_blocks(&good, INT32_MAX, 0.0f, fake, nullptr, nullptr, 1, f, i, nullptr), ARCKV_ERR_UNSUPPORTED);

  // workspace sizes over the whole range of arguments, and a short workspace
  size_t bytes = 0, most = 0;
  const int32_t sizes[] = {1, 2, 63, 64, 65, 768, 769, 4096, 1 << 20, 1 << 26};
  for (int32_t P : sizes)
    for (int32_t rows : sizes)
      for (int32_t F : sizes) {
        EXPECT(arckv_attend_qcache_workspace_size(P, rows, 16, 0, F, &bytes), P <= 1 << 20 ? ARCKV_OK : ARCKV_ERR_UNSUPPORTED);
        if (bytes > most) most = bytes;
      }
  if (most == 0 || most > (size_t)64 << 20) { printf("FAIL workspace up to %zu\n", most); ++failures; }
  EXPECT(arckv_attend_qcache_workspace_size(1, 1, 1, INT32_MAX, 0, &bytes), ARCKV_ERR_UNSUPPORTED);
  EXPECT(arckv_attend_qcache_workspace_size(1, 1, 1, 0, INT32_MAX, &bytes), ARCKV_ERR_UNSUPPORTED);
  EXPECT(arckv_attend_qcache_workspace_size(1, 1, 1, 0, 0, nullptr), ARCKV_ERR_INVALID_ARG);
  c = good;
  c.rows = 100000;
  EXPECT(arckv_attend_qcache_workspace_size(c.P, c.rows, 4, 0, 0, &bytes), ARCKV_OK);
  EXPECT(arckv_attend_qcache(&c, 4, 0, 0, 0.0f, fake, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, f, ws, bytes - 1,
                             nullptr), ARCKV_ERR_WORKSPACE);

  printf("%s: %d failures\n", failures ? "FAILED" : "ok", failures);
  return failures ? 1 : 0;
}
