// Stands in for the parts of the HIP runtime that libincvit.so calls to register
// and launch kernels: a launch is written down (kernel, grid, block, LDS bytes)
// and not run.  Loaded before the library in a process without a GPU.
#include <cstddef>
#include <cstdint>
#include <map>
#include <string>
#include <vector>

namespace {
struct Dim { uint32_t x, y, z; };
std::map<const void*, std::string>& names() {
  static std::map<const void*, std::string> n;
  return n;
}
std::string& log() {
  static std::string s;
  return s;
}
std::string& all() {
  static std::string s;
  return s;
}
int add(const void* f, Dim g, Dim b, size_t lds) {
  auto it = names().find(f);
  log() += (it == names().end() ? std::string("?") : it->second);
  for (uint64_t v : {(uint64_t)g.x, (uint64_t)g.y, (uint64_t)g.z, (uint64_t)b.x, (uint64_t)lds}) log() += " " + std::to_string(v);
  log() += "\n";
  return 0;
}
}  // namespace

extern "C" {
const char* launch_log_take() {  // the launches since the last call
  static std::string out;
  out.swap(log());
  log().clear();
  return out.c_str();
}
const char* launch_log_kernels() {  // every kernel of the library
  for (const auto& n : names()) all() += n.second + "\n";
  return all().c_str();
}
void** __hipRegisterFatBinary(const void*) {
  static void* one;
  return &one;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* device, unsigned, void*, void*, void*, void*, int*) {
  names()[host] = device;
}
int hipLaunchKernel(const void* f, Dim g, Dim b, void**, size_t lds, void*) { return add(f, g, b, lds); }
int hipExtLaunchKernel(const void* f, Dim g, Dim b, void**, size_t lds, void*, void*, void*, int) { return add(f, g, b, lds); }
int hipGetDevice(int* d) {
  *d = 0;
  return 0;
}
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipGetLastError() { return 0; }
int hipMemcpyAsync(void*, const void*, size_t, int, void*) { return 0; }
}
