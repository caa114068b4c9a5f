// Host-side checks of the 4-bit cache's and the rotary entry points' C ABI for a build with AddressSanitizer and
// UndefinedBehaviorSanitizer on the host code: each case fails validation before any HIP call, or is host arithmetic alone.
// Exit status 0 when every call returns the expected status.
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
  const size_t plenty = (size_t)1 << 40;
  const arckv_ncache good = {2, 100, 128, fake, fake, fake, fake};
  arckv_ncache bad[6] = {good, good, good, good, good, good};
  bad[0].P = 0;
  bad[1].rows = -5;
  bad[2].K = odd;
  bad[3].K_scale = nullptr;
  bad[4].rows = INT32_MIN;
  bad[5].P = INT32_MIN;
  for (const arckv_ncache &c : bad) {
    EXPECT(arckv_ncache_write(&c, 1, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
    EXPECT(arckv_ncache_read(&c, 0, 1, ARCKV_BF16, nullptr, fake, fake, nullptr), ARCKV_ERR_INVALID_ARG);
    EXPECT(arckv_attend_ncache(&c, 4, 0, 0.0f, fake, nullptr, nullptr, nullptr, nullptr, nullptr, f, ws, plenty, nullptr),
           ARCKV_ERR_INVALID_ARG);
  }
  arckv_ncache c = good;
  c.rows = INT32_MAX;
  EXPECT(arckv_ncache_write(&c, 1, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_UNSUPPORTED);
  EXPECT(arckv_ncache_write(&good, INT32_MAX, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_ncache_write(&good, INT32_MIN, ARCKV_BF16, fake, fake, nullptr, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_ncache_read(&good, INT32_MAX, INT32_MAX, ARCKV_F32, nullptr, fake, fake, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_ncache_read(&good, INT32_MIN, 1, ARCKV_F32, nullptr, fake, fake, nullptr), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_attend_ncache(&good, INT32_MAX, 0, 0.0f, fake, nullptr, nullptr, nullptr, nullptr, nullptr, f, ws, plenty, nullptr),
         ARCKV_ERR_UNSUPPORTED);
  EXPECT(arckv_attend_ncache(&good, 4, INT32_MIN, 0.0f, fake, nullptr, nullptr, nullptr, nullptr, nullptr, f, ws, plenty, nullptr),
         ARCKV_ERR_INVALID_ARG);

  // workspace sizes over the whole range of arguments, and a short workspace
  size_t bytes = 0, most = 0;
  const int32_t sizes[] = {1, 2, 63, 64, 65, 256, 257, 768, 769, 4096, 1 << 20, 1 << 26};
  for (int32_t P : sizes)
    for (int32_t rows : sizes)
      for (int32_t F : sizes) {
        EXPECT(arckv_attend_ncache_workspace_size(P, rows, 16, F, &bytes), P <= 1 << 20 ? ARCKV_OK : ARCKV_ERR_UNSUPPORTED);
        if (bytes > most) most = bytes;
      }
  if (most == 0 || most > (size_t)64 << 20) { printf("FAIL workspace up to %zu\n", most); ++failures; }
  EXPECT(arckv_attend_ncache_workspace_size(1, 1, 1, INT32_MAX, &bytes), ARCKV_ERR_UNSUPPORTED);
  EXPECT(arckv_attend_ncache_workspace_size(1, 1, 1, 0, nullptr), ARCKV_ERR_INVALID_ARG);
  c = good;
  c.rows = 100000;
  EXPECT(arckv_attend_ncache_workspace_size(c.P, c.rows, 4, 0, &bytes), ARCKV_OK);
  EXPECT(arckv_attend_ncache(&c, 4, 0, 0.0f, fake, nullptr, nullptr, nullptr, nullptr, nullptr, f, ws, bytes - 1, nullptr),
         ARCKV_ERR_WORKSPACE);

  // rotary: strides at the ends of their range
  const double *freq = (const double *)fake;
  const arckv_rotary_params p = {5, 128, 128, ARCKV_ROTARY_HALVES, ARCKV_BF16, 0, 1.0f};
  const arckv_rotary_rows rows = {3, fake, 384, 128, ws, 384, 128};
  for (const int64_t s : {INT64_MIN, INT64_MAX, (int64_t)-8, (int64_t)1, INT64_MAX - 7}) {
    for (int i = 0; i < 4; ++i) {
      arckv_rotary_rows r = rows;
      (i == 0 ? r.x_token : i == 1 ? r.x_head : i == 2 ? r.y_token : r.y_head) = s;
      EXPECT(arckv_rotary(&p, nullptr, freq, &r, nullptr, nullptr), s > 0 && s % 8 == 0 ? ARCKV_ERR_UNSUPPORTED : ARCKV_ERR_INVALID_ARG);
    }
  }
  for (const int32_t n : {INT32_MIN, -1, 0}) {
    arckv_rotary_params q = p;
    q.N = n;
    EXPECT(arckv_rotary(&q, nullptr, freq, &rows, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
    arckv_rotary_rows r = rows;
    r.heads = n;
    EXPECT(arckv_rotary(&p, nullptr, freq, &r, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
    q = p;
    q.d_rot = n;
    EXPECT(arckv_rotary(&q, nullptr, freq, &rows, nullptr, nullptr), ARCKV_ERR_INVALID_ARG);
  }
  arckv_rotary_rows wide = rows;
  wide.heads = 1 << 20;
  wide.x_token = wide.y_token = (int64_t)1 << 34;
  arckv_rotary_params q = p;
  q.N = 1 << 26;
  EXPECT(arckv_rotary(&q, nullptr, freq, &wide, &wide, nullptr), ARCKV_ERR_UNSUPPORTED);

  // frequencies: every mode fills d_rot / 2 numbers and no more
  for (int32_t d = 2; d <= 128; d += 2)
    for (int32_t mode = 0; mode < 5; ++mode) {
      double *out = new double[d / 2];
      EXPECT(arckv_rotary_frequencies(d, 1e4, mode, 2.0, 4096.0, 1.0, 32.0, out), mode == 2 && d == 2 ? ARCKV_ERR_INVALID_ARG : ARCKV_OK);
      if (!(mode == 2 && d == 2))
        for (int i = 0; i < d / 2; ++i)
          if (!(out[i] > 0.0 && out[i] <= 1.0)) { printf("FAIL d_rot %d mode %d: %g\n", d, mode, out[i]); ++failures; }
      delete[] out;
    }
  double one[64];
  EXPECT(arckv_rotary_frequencies(INT32_MIN, 1e4, 0, 1.0, 0.0, 0.0, 0.0, one), ARCKV_ERR_INVALID_ARG);
  EXPECT(arckv_rotary_frequencies(64, 1.0000001, ARCKV_STRETCH_INDEX, 2.0, 1e300, 1e-300, 1e300, one), ARCKV_OK);

  // a valid call that needs no workspace and gets none forms no address from the null pointer in its place; it goes as far
  // as HIP, only where there is no device
  int devices = 0;
  if (hipGetDeviceCount(&devices) != hipSuccess || devices == 0) {
    EXPECT(arckv_attend_ncache_workspace_size(good.P, good.rows, 4, 0, &bytes), ARCKV_OK);
    EXPECT(bytes, 0);
    EXPECT(arckv_attend_ncache(&good, 4, 0, 0.0f, fake, nullptr, nullptr, nullptr, nullptr, nullptr, f, nullptr, 0, nullptr),
           ARCKV_ERR_HIP);
  }
  printf("%s: %d failures\n", failures ? "FAILED" : "ok", failures);
  return failures ? 1 : 0;
}
