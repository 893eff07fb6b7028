// The device query that launches share, from several threads at once, under ThreadSanitizer (built by
// tests/test_seq_sanitize.py). The HIP calls are stand-ins: no runtime and no device.
#include <stdio.h>

#include <thread>
#include <vector>

#include "common.h"

static int g_device = 0;
hipError_t hipGetDevice(int* dev) {
  *dev = g_device;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* n, hipDeviceAttribute_t, int) {
  *n = 304;
  return hipSuccess;
}

int main() {
  std::vector<std::thread> threads;
  int got[8] = {};
  for (int i = 0; i < 8; ++i) threads.emplace_back([&got, i] { got[i] = hsa::compute_units(); });
  for (std::thread& t : threads) t.join();
  for (int n : got)
    if (n != 304) return 1;
  printf("device_query ok\n");
  return 0;
}
