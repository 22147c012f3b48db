// What the library remembers about devices (csrc/sq_internal.h), against calls of the runtime that
// only count, for tests/test_device_state.py.
#include <cstdio>

#include "sq_internal.h"

namespace {
int current = 0, limits = 0, queries = 0;
hipError_t answer = hipSuccess;
void kernel_a() {}
void kernel_b() {}
}  // namespace

extern "C" {
hipError_t hipGetDevice(int* device) {
  *device = current;
  return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) {
  ++limits;
  return answer;
}
hipError_t hipDeviceGetAttribute(int* value, hipDeviceAttribute_t, int device) {
  ++queries;
  *value = 100 + device;
  return answer;
}
}

int main() {
  // (device, kernel, answer of the runtime) one after another: calls of the runtime, and the status
  const struct {
    int device, kernel;
    hipError_t answer;
  } steps[] = {{0, 0, hipErrorInvalidValue}, {0, 0, hipSuccess}, {0, 0, hipSuccess}, {1, 0, hipSuccess}, {1, 0, hipSuccess},
               {0, 0, hipSuccess},           {0, 1, hipSuccess}, {1, 1, hipSuccess}, {99, 0, hipSuccess}, {99, 0, hipSuccess}};
  for (const auto& s : steps) {
    current = s.device;
    answer = s.answer;
    const hipError_t e = s.kernel ? sq::set_max_lds<kernel_b>(100) : sq::set_max_lds<kernel_a>(100);
    std::printf("%d %d\n", limits, static_cast<int>(e));
  }
  for (const int device : {0, 1, 1, 0, 2}) {
    current = device;
    int cus = 0;
    const hipError_t e = sq::device_cus(&cus);
    std::printf("%d %d %d\n", queries, cus, static_cast<int>(e));
  }
  return 0;
}
