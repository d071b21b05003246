// The norms' and rotations' plans and launches as the library makes them, without a GPU: stands in for the few HIP calls on the way
// (tests/test_rope_launch_host.py links it with the library's objects and calls it).
#include <hip/hip_runtime.h>

#include <cstdlib>
#include <cstring>

#include "rf2.h"

static char copied[4096];                       // what the last copy to the device took there
static uint32_t grids[16];
static int launches = 0;
static dim3 pushed[2];

extern "C" {
hipError_t hipGetDeviceCount(int* n) { *n = 1; return hipSuccess; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { *p = std::malloc(n); return *p ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipFree(void* p) { std::free(p); return hipSuccess; }
hipError_t hipMemcpy(void* to, const void* from, size_t n, hipMemcpyKind) {
  std::memcpy(to, from, n);
  std::memcpy(copied, from, n < sizeof copied ? n : sizeof copied);
  return hipSuccess;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  pushed[0] = grid, pushed[1] = block;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
  *grid = pushed[0], *block = pushed[1], *lds = 0, *stream = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3, void**, size_t, hipStream_t) {
  if (launches < 16) grids[launches] = grid.x;
  ++launches;
  return hipSuccess;
}

// A plan's tables: turns and rest of 64 pairs, int32, and their axes, uint8; then those of the other way.
int rope_tables(const rf2_rope_config* cfg, const double* freq, char* out, int size) {
  rf2_rope_plan* plan = nullptr;
  if (rf2_rope_plan_create(cfg, freq, &plan) != RF2_OK) return -1;
  std::memcpy(out, copied, (size_t)size);
  rf2_rope_plan_destroy(plan);
  return 0;
}

// Workgroups of the launches of a call (`rows` of rf2_rope_tensors, or of rf2_rope_gradients).
int rope_grids(const rf2_rope_config* cfg, int backward, int batch, int tokens, const rf2_rows* rows, uint32_t* out) {
  rf2_rope_plan* plan = nullptr;
  if (rf2_rope_plan_create(cfg, nullptr, &plan) != RF2_OK) return -1;
  launches = 0;
  void* const at = (void*)4096;
  const bool norm = cfg->norm == RF2_NORM_RMS;
  const void* const w = norm ? at : nullptr;
  float* const dw = norm ? (float*)at : nullptr;
  const int rc = backward ? rf2_rope_backward(plan, batch, tokens, (const rf2_rope_gradients*)rows, (const int32_t*)at, 0, w, w, dw, dw, at, nullptr)
                          : rf2_rope_apply(plan, batch, tokens, (const rf2_rope_tensors*)rows, (const int32_t*)at, 0, w, w, nullptr);
  rf2_rope_plan_destroy(plan);
  if (rc != RF2_OK) return rc;
  std::memcpy(out, grids, sizeof grids);
  return launches;
}
}
