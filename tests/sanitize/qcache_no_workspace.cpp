// A valid call that needs no workspace and gets none, for a build with AddressSanitizer and UndefinedBehaviorSanitizer on
// the host code.  Its device pointers are invented: it goes as far as HIP only where there is no device.
#include <hip/hip_runtime.h>
#include <stdio.h>

#include "arckv.h"

int main() {
  int devices = 0;
  if (hipGetDeviceCount(&devices) == hipSuccess && devices > 0) {
    printf("a device is visible: not run\n");
    return 0;
  }
  void *fake = (void *)0x1000;
  float *f = (float *)fake;
  const arckv_qcache c = {2, 100, 128, ARCKV_E4M3, fake, fake, f, f, fake};
  size_t bytes = 1;
  const arckv_status size = arckv_attend_qcache_workspace_size(c.P, c.rows, 4, 0, 0, &bytes);
  const arckv_status call = arckv_attend_qcache(&c, 4, 0, 0, 0.0f, fake, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, f,
                                                nullptr, 0, nullptr);
  const bool good = size == ARCKV_OK && bytes == 0 && call == ARCKV_ERR_HIP;
  printf("%s: size %d, %zu bytes, call %d\n", good ? "ok" : "FAILED", (int)size, bytes, (int)call);
  return good ? 0 : 1;
}
