// The fake CUDA runtime, which here also keeps the first words of the first argument of the training kernels' launches.
#define cudaLaunchKernel noted_launch
#define cudaLaunchKernelExC noted_launch_ex
#include "fake_cudart.cpp"
#undef cudaLaunchKernel
#undef cudaLaunchKernelExC

#include <vector>

namespace {
constexpr size_t kWords = 40;                  // 320 bytes (their parameters are longer)
std::vector<void*> words;
void keep(const void* stub, void** args) {
  const std::string& name = names[stub];
  if (name.find("train_") == std::string::npos && name.find("bias_reduce") == std::string::npos) return;
  const size_t at = words.size();
  words.resize(at + kWords);
  memcpy(&words[at], args[0], kWords * sizeof(void*));
}
}  // namespace

extern "C" {
void fake_forget_args(void) { words.clear(); }
int fake_launches(void) { return static_cast<int>(words.size() / kWords); }
void fake_args(int launch, void** out) { memcpy(out, &words[launch * kWords], kWords * sizeof(void*)); }

int cudaLaunchKernel(const void* stub, dim3_ grid, dim3_ block, void** args, size_t smem, void* stream) {
  keep(stub, args);
  return noted_launch(stub, grid, block, args, smem, stream);
}
int cudaLaunchKernelExC(const void* config, const void* stub, void** args) {
  keep(stub, args);
  return noted_launch_ex(config, stub, args);
}
}
