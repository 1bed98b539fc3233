// Stands in for the CUDA runtime when the built objects of the paged cache are linked for the CPU: no kernel runs, every launch is
// logged ("kernel grid.x grid.y grid.z block dynamic-bytes").  A launch whose shared memory, with up to 1 KB of static arrays
// besides, passes the default 48 KB without the limit having been raised is refused as the runtime refuses it; so is the n-th launch
// of a kernel named by fake_fail.
#include <map>
#include <regex>
#include <string>

#include "asl_internal.cuh"
#define cudaGetLastError fake_no_error
#include "fake_cuda_runtime.cpp"
#undef cudaGetLastError
#include "attend.cuh"

namespace {
struct Kernel { std::string name; int limit; };
std::map<const void*, Kernel> g_kernels;
cudaError_t g_last = cudaSuccess;

std::string plain_name(const char* mangled) {            // <length>some_kernel, possibly among other names
  const std::string s(mangled);
  std::smatch m;
  return std::regex_search(s, m, std::regex("[0-9]((pages|attend|rows)_[a-z_]*kernel)")) ? m[1].str() : s;
}
cudaError_t fail(cudaError_t e) { return g_last = e; }
}  // namespace

extern "C" {
void** __cudaRegisterFatBinary(void*) { static void* handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char* host, char*, const char* name, int, uint3*, uint3*, dim3*, dim3*, int*) {
  g_kernels[host] = Kernel{plain_name(name), 0};
}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void*) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return fail(cudaErrorNotSupported); }
cudaError_t cudaFuncSetAttribute(const void* f, cudaFuncAttribute what, int value) {
  if (what == cudaFuncAttributeMaxDynamicSharedMemorySize) g_kernels[f].limit = value;
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* cfg, const void* f, void**) {
  const Kernel& k = g_kernels[f];
  const size_t bytes = cfg->dynamicSmemBytes;
  if (fails(k.name.c_str())) return fail(cudaErrorLaunchOutOfResources);
  if (k.limit ? bytes > (size_t)k.limit : bytes + 1024 > 48 * 1024) return fail(cudaErrorInvalidValue);
  g_log += k.name;
  for (size_t x : {(size_t)cfg->gridDim.x, (size_t)cfg->gridDim.y, (size_t)cfg->gridDim.z, (size_t)cfg->blockDim.x, bytes}) g_log += " " + std::to_string(x);
  g_log += "\n";
  return cudaSuccess;
}
cudaError_t cudaGetLastError() { const cudaError_t e = g_last; g_last = cudaSuccess; return e; }
}  // extern "C"

asl_status asl_launch_attend_narrow(asl_ctx*, const asl_pages*, const AttendArgs&, int, bool, cudaStream_t st) { return launch("narrow", st); }
asl_status asl_launch_attend_wide(asl_ctx*, const asl_pages*, const AttendArgs&, int, cudaStream_t st) { return launch("wide", st); }
asl_status asl_attend_narrow_ready() { return ASL_OK; }
asl_status asl_attend_wide_ready() { return ASL_OK; }
