// A CUDA runtime for tests of the library's host side on machines without a GPU: "device" memory is host memory, copies are
// memcpy, kernels are only noted by name.  Any function can be told to fail once, and a stream capture can be pretended.
#include <stddef.h>
#include <string.h>

#include <map>
#include <string>

namespace {
std::map<const void*, std::string> names;      // host stub -> kernel
std::string log_;                              // kernels launched, one line each
std::map<std::string, int> countdown;          // function -> calls until it fails
int last_error = 0, capturing = 0;
const int kError = 1;                          // cudaErrorInvalidValue

int result(const char* fn) {
  auto it = countdown.find(fn);
  if (it != countdown.end() && --it->second == 0) {
    countdown.erase(it);
    return kError;
  }
  return 0;
}
int launch(const char* fn, const void* stub) {
  const int e = result(fn);
  if (e) last_error = e;
  else log_ += (names.count(stub) ? names[stub] : std::string("?")) + "\n";
  return e;
}
struct dim3_ { unsigned x, y, z; };
}  // namespace

extern "C" {
void fake_fail(const char* fn, int nth) { countdown[fn] = nth; }      // the nth call from now on
void fake_capture(int on) { capturing = on; }
const char* fake_log(void) { return log_.c_str(); }
void fake_reset(void) { log_.clear(); countdown.clear(); capturing = 0; last_error = 0; }

void** __cudaRegisterFatBinary(void*) { static void* handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char* stub, char*, const char* name, int, void*, void*, void*, void*, int*) { names[stub] = name; }
void __cudaRegisterVar(void**, char*, char*, const char*, int, size_t, int, int) {}
unsigned __cudaPushCallConfiguration(dim3_, dim3_, size_t, void*) { return 0; }
int __cudaPopCallConfiguration(dim3_* grid, dim3_* block, size_t* smem, void* stream) {
  *grid = *block = dim3_{1, 1, 1};
  *smem = 0;
  memset(stream, 0, sizeof(void*));
  return 0;
}
int cudaLaunchKernel(const void* stub, dim3_, dim3_, void**, size_t, void*) { return launch("cudaLaunchKernel", stub); }
int cudaLaunchKernelExC(const void*, const void* stub, void**) { return launch("cudaLaunchKernelExC", stub); }
int cudaGetLastError(void) { const int e = last_error; last_error = 0; return e; }
const char* cudaGetErrorString(int) { return "a fake failure"; }
int cudaGetDevice(int* dev) { *dev = 0; return result("cudaGetDevice"); }
int cudaDeviceGetAttribute(int* v, int, int) { *v = 148; return result("cudaDeviceGetAttribute"); }
int cudaEventRecord(void*, void*) { return result("cudaEventRecord"); }
int cudaFuncSetAttribute(const void*, int, int) { return result("cudaFuncSetAttribute"); }
int cudaGetDriverEntryPoint(const char*, void** fn, unsigned long long, void*) { *fn = nullptr; return kError; }
int cudaGetSymbolAddress(void** p, const void*) { *p = nullptr; return result("cudaGetSymbolAddress"); }
int cudaMemcpyAsync(void* to, const void* from, size_t n, int, void*) {
  const int e = result("cudaMemcpyAsync");
  if (!e) memcpy(to, from, n);
  return e;
}
int cudaMemsetAsync(void* to, int v, size_t n, void*) {
  const int e = result("cudaMemsetAsync");
  if (!e) memset(to, v, n);
  return e;
}
int cudaStreamIsCapturing(void*, int* status) { *status = capturing; return result("cudaStreamIsCapturing"); }
int cudaStreamSynchronize(void*) { return result("cudaStreamSynchronize"); }
}
