// Stand-ins for the HIP runtime that note which kernels a library launches,
// with what grids, and launch nothing: loaded before the library, in a process
// without a device, so that its choice of kernels can be looked at for any
// sizes.
#include <cxxabi.h>
#include <stdint.h>
#include <stdlib.h>

#include <map>
#include <string>

struct Dim3 {
  uint32_t x, y, z;
};

// (never destroyed: the library unregisters at exit)
static std::map<const void*, std::string>& names() {
  static auto* m = new std::map<const void*, std::string>;
  return *m;
}
static std::string& log() {
  static auto* s = new std::string;
  return *s;
}
static struct {
  Dim3 grid, block;
  size_t lds;
  void* stream;
} pending;

extern "C" {

void** __hipRegisterFatBinary(const void*) {
  static void* handle;
  return &handle;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
  int status = 0;
  char* plain = abi::__cxa_demangle(name, nullptr, nullptr, &status);
  names()[host] = status == 0 ? plain : name;
  free(plain);
}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void* stream) {
  pending = {grid, block, lds, stream};
  return 0;
}
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream) {
  *grid = pending.grid;
  *block = pending.block;
  *lds = pending.lds;
  *stream = pending.stream;
  return 0;
}
int hipLaunchKernel(const void* host, Dim3 grid, Dim3 block, void**, size_t, void*) {
  log() += names()[host] + "|" + std::to_string(grid.x) + "|" + std::to_string(block.x) + "\n";
  return 0;
}
int hipGetLastError() { return 0; }
int hipGetDevice(int* d) {
  *d = 0;
  return 0;
}
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipDeviceGetAttribute(int* v, int, int) {
  *v = 256;
  return 0;
}
int hipOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void*, int, size_t) {
  *n = 2;
  return 0;
}
const char* hipGetErrorString(int) { return "error"; }

// What was launched since the last call.
const char* launch_log_take() {
  static std::string out;
  out.swap(log());
  log().clear();
  return out.c_str();
}
}
