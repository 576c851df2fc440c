// A stand-in HIP runtime that writes down what is launched: kernels by their names, with their grids.  Built with the
// library's host code into a library of its own (tests/launches.py); nothing runs, device pointers are never touched.
#include <cxxabi.h>

#include <cstdio>
#include <cstdlib>
#include <map>
#include <string>

#include <hip/hip_runtime.h>

#include "lora_internal.h"

namespace lora {
hipError_t launch_shrink(const KernelArgs&, const uint32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_expand(const KernelArgs&, const uint32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_reduce(const KernelArgs&, const uint32_t*, hipStream_t) { return hipSuccess; }
hipError_t launch_step(const KernelArgs&, const uint32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_fill(uint32_t*, uint32_t, uint64_t, hipStream_t) { return hipSuccess; }
hipError_t launch_base(const BaseArgs&, int, hipStream_t) { return hipSuccess; }
}  // namespace lora

namespace {
std::map<const void*, std::string>& kernels() {
    static std::map<const void*, std::string> k;
    return k;
}
std::string g_log, g_names;
dim3 g_grid, g_block;

// "name<arguments>" of a kernel's mangled name
std::string readable(const char* mangled) {
    int status = 0;
    char* d = abi::__cxa_demangle(mangled, nullptr, nullptr, &status);
    std::string s = status == 0 ? d : mangled;
    std::free(d);
    for (const char* cut : {"void ", "lora::", "(anonymous namespace)::"})
        for (size_t at; (at = s.find(cut)) != std::string::npos;) s.erase(at, std::string(cut).size());
    return s.substr(0, s.rfind('('));
}
}  // namespace

extern "C" {
void** __hipRegisterFatBinary(const void*) {
    static void* handle;
    return &handle;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*, dim3*, dim3*, int*) {
    kernels()[f] = readable(name);
}
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int d) { return d == 0 ? hipSuccess : hipErrorInvalidDevice; }
hipError_t hipStreamGetDevice(hipStream_t, hipDevice_t* d) { *d = 0; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
    g_grid = grid;
    g_block = block;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* s) {
    *grid = g_grid;
    *block = g_block;
    *lds = 0;
    *s = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
    char line[96];
    std::snprintf(line, sizeof line, "\t%u\t%u\t%u\t%u\n", grid.x, grid.y, grid.z, block.x);
    g_log += kernels()[f] + line;
    return hipSuccess;
}

// What was launched since the last question, a line each: name, grid, threads of a workgroup.
const char* launches_log() {
    static std::string out;
    out.swap(g_log);
    g_log.clear();
    return out.c_str();
}
// The kernels that there are, a line each.
const char* launches_kernels() {
    g_names.clear();
    for (const auto& k : kernels()) g_names += k.second + "\n";
    return g_names.c_str();
}
}
