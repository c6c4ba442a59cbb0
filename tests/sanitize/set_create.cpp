// What a failed creation of an optimizer's set leaves behind, on the CPU: the HIP calls that it makes are this program's own (they
// stand before the runtime's), each failing in turn as the runtime's would, with its error pending until it is asked for.  Test
// infrastructure only.  Exit status: the number of failed checks.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include <hip/hip_runtime_api.h>

#include "frameft.h"

enum Call { kNone, kGetDevice, kMalloc, kMemcpy };
static Call g_failing = kNone;
static hipError_t g_pending = hipSuccess;
static int g_allocated = 0;

static hipError_t result(Call c, hipError_t e) {
  if (c != g_failing) return hipSuccess;
  return g_pending = e;
}

extern "C" {
hipError_t hipGetDevice(int* d) {
  *d = 0;
  return result(kGetDevice, hipErrorNoDevice);
}
hipError_t hipMalloc(void** p, size_t n) {
  *p = nullptr;
  const hipError_t e = result(kMalloc, hipErrorOutOfMemory);
  if (e == hipSuccess) *p = std::malloc(n), ++g_allocated;
  return e;
}
hipError_t hipFree(void* p) {
  std::free(p), --g_allocated;
  return hipSuccess;
}
hipError_t hipMemcpy(void* to, const void* from, size_t n, hipMemcpyKind) {
  const hipError_t e = result(kMemcpy, hipErrorUnknown);
  if (e == hipSuccess) std::memcpy(to, from, n);
  return e;
}
hipError_t hipGetLastError(void) {
  const hipError_t e = g_pending;
  g_pending = hipSuccess;
  return e;
}
}

int main() {
  int failed = 0;
  auto check = [&](bool ok, const char* what, int call) {
    if (!ok) std::printf("failed: %s, call %d (%s)\n", what, call, ff_last_error()), ++failed;
  };
  static float c[300], m[300], v[300];
  float* pc = c;
  void *pm = m, *pv = v;
  const int64_t n = 300;
  for (int call = kNone; call <= kMemcpy; ++call) {
    g_failing = (Call)call;
    ff_adamw_set* set = nullptr;
    const ff_status st = ff_adamw_set_create(1, &n, FF_STATES_F32, FF_F32, &pc, nullptr, &pm, &pv, nullptr, nullptr, nullptr, &set);
    const ff_status want[] = {FF_OK, FF_EDEVICE, FF_ENOMEM, FF_EDEVICE};
    check(st == want[call], "status", call);
    check((set != nullptr) == (call == kNone), "handle", call);
    // the next launch asks for the last error as its own
    check(hipGetLastError() == hipSuccess, "an error is left for the next call", call);
    if (set) {
      g_failing = kGetDevice;
      const void* g = c;
      ff_adamw_hyper h{};
      h.lr = 0.1, h.eps = 1e-8, h.step = 1, h.grad_scale = 1.0;
      check(ff_adamw_set_step(set, &g, &h, nullptr) == FF_EINVAL, "step without a device", call);
      check(hipGetLastError() == hipSuccess, "an error is left by a step without a device", call);
      g_failing = kNone;
    }
    ff_adamw_set_destroy(set);
    check(g_allocated == 0, "memory of the device is left", call);
  }
  std::printf("set creation: %d failed checks\n", failed);
  return failed;
}
