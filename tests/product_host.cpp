// The host side of csrc/product.hip (compiled without its kernels) on a stand-in for the HIP runtime with several devices:
// says which calls it makes of the runtime, and which kernels it launches.  Commands from stdin, a line each:
//   device N                                         the current device from here on
//   fail N                                           the next N attributes cannot be set
//   create name slots in out x_dtype y_dtype gate max_rows
//   run name rows slots                              slots 0: without offsets
//   destroy name
// Lines out: "create rc", "run rc", "destroy rc" behind what the call did, "attribute device kernel bytes",
// "launch device kernel workgroups threads lds", "malloc device bytes", "free device".
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <iostream>
#include <map>
#include <sstream>
#include <string>

#include "eep.h"
#include "eep_internal.hpp"

static int device = 0, failing = 0;
static std::map<const void*, std::string>& kernels() {  // (registered before main, in any order)
  static std::map<const void*, std::string> all;
  return all;
}
static dim3 grid, block;
static size_t lds;
static hipStream_t on;

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
  kernels()[host] = name;
}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t bytes, hipStream_t st) {
  grid = g, block = b, lds = bytes, on = st;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* bytes, hipStream_t* st) {
  *g = grid, *b = block, *bytes = lds, *st = on;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 g, dim3 b, void**, size_t bytes, hipStream_t) {
  std::printf("launch %d %s %u %u %zu\n", device, kernels().at(f).c_str(), g.x, b.x, bytes);
  return hipSuccess;
}
hipError_t hipGetDevice(int* d) { *d = device; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* value, hipDeviceAttribute_t, int) { *value = 256; return hipSuccess; }
hipError_t hipMalloc(void** p, size_t bytes) {
  std::printf("malloc %d %zu\n", device, bytes);
  *p = std::malloc(bytes);
  return *p ? hipSuccess : hipErrorOutOfMemory;
}
hipError_t hipFree(void* p) {
  if (p) std::printf("free %d\n", device);
  std::free(p);
  return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipFuncSetAttribute(const void* f, hipFuncAttribute, int bytes) {
  if (failing > 0) { --failing; return hipErrorInvalidDevice; }
  std::printf("attribute %d %s %d\n", device, kernels().at(f).c_str(), bytes);
  return hipSuccess;
}
}

namespace eep {
hipError_t launch_fill(int32_t*, int32_t, int64_t, hipStream_t) { return hipSuccess; }
}  // namespace eep

int main() {
  std::map<std::string, eep_product*> products;
  alignas(16) static char memory[64];  // addresses that nothing reads
  std::map<std::string, eep_product_config> shapes;
  for (std::string line; std::getline(std::cin, line);) {
    std::istringstream in(line);
    std::string what, name;
    in >> what;
    if (what == "device") {
      in >> device;
    } else if (what == "fail") {
      in >> failing;
    } else if (what == "create") {
      eep_product_config c = {};
      in >> name >> c.num_slots >> c.in_features >> c.out_features >> c.x_dtype >> c.y_dtype >> c.gate >> c.max_rows;
      shapes[name] = c;
      std::printf("create %d\n", eep_product_create(&c, &products[name]));
    } else if (what == "run") {
      int rows = 0, slots = 0;
      in >> name >> rows >> slots;
      const eep_product_config& c = shapes[name];
      const bool codes = c.x_dtype == EEP_FP8_E4M3;
      std::printf("run %d\n", eep_expert_product(products[name], memory, codes ? (const float*)memory : nullptr, memory,
                                                 codes ? (const float*)memory : nullptr, slots ? (const int32_t*)memory : nullptr,
                                                 memory, c.y_dtype == EEP_FP8_E4M3 ? (float*)memory : nullptr, rows, nullptr));
    } else if (what == "destroy") {
      in >> name;
      std::printf("destroy %d\n", eep_product_destroy(products[name]));
      products.erase(name);
    } else {
      return 2;
    }
  }
  return 0;
}
