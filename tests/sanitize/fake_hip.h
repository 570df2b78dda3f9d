// HIP's calls for checks that run without a GPU: memory is the host's, a launch is
// run_kernel()'s, which the including file defines, and the launch that `fail_in` names fails.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstring>
#include <map>
#include <string>

static std::map<const void*, std::string> kernels;
static int fail_in = -1;  // launches before the one that fails; < 0: none does
static hipError_t last_error = hipSuccess;
static int launches = 0;

static void run_kernel(const std::string& name, dim3 grid, dim3 block, void** args);

template <typename T>
static T arg(void** a, int i) { return *static_cast<T*>(a[i]); }

extern "C" {

void** __hipRegisterFatBinary(const void*) { static void* none = nullptr; return &none; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
  kernels[host] = name;
}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
static struct { dim3 grid, block; size_t lds; hipStream_t st; } config;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t st) {
  config = {grid, block, lds, st};
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* st) {
  *grid = config.grid;
  *block = config.block;
  *lds = config.lds;
  *st = config.st;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  ++launches;
  if (fail_in == 0) {
    fail_in = -1;
    return last_error = hipErrorLaunchFailure;
  }
  if (fail_in > 0) --fail_in;
  run_kernel(kernels.at(f), grid, block, args);
  return hipSuccess;
}
hipError_t hipGetLastError() {
  const hipError_t e = last_error;
  last_error = hipSuccess;
  return e;
}
const char* hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipMemcpyAsync(void* to, const void* from, size_t n, hipMemcpyKind, hipStream_t) {
  std::memmove(to, from, n);
  return hipSuccess;
}
hipError_t hipMemsetAsync(void* to, int v, size_t n, hipStream_t) {
  std::memset(to, v, n);
  return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipGetDevice(int* d) {
  *d = 0;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) {
  *v = 256;
  return hipSuccess;
}
hipError_t hipPointerGetAttributes(hipPointerAttribute_t*, const void*) { return hipErrorInvalidValue; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetSymbolAddress(void**, const void*) { return hipErrorInvalidSymbol; }

}  // extern "C"
