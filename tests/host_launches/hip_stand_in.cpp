// Stands in for the HIP runtime where libzr.so is loaded without a GPU: nothing runs, and every launch is recorded with its
// kernel's name and grid.  Loaded ahead of the library, so that its calls end here.
#include <cstddef>
#include <cstdint>
#include <cstring>
#include <map>
#include <string>

namespace {
struct Dim3 { uint32_t x, y, z; };
struct Config { Dim3 grid, block; size_t lds; void* stream; };
std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
std::string& log() { static std::string s; return s; }
thread_local Config config;
}  // namespace

extern "C" {

void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, Dim3*, Dim3*, int*) { names()[host] = name; }
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void* stream) { config = {grid, block, lds, stream}; return 0; }
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream)
{
    *grid = config.grid; *block = config.block; *lds = config.lds; *stream = config.stream;
    return 0;
}
int hipLaunchKernel(const void* host, Dim3 grid, Dim3, void**, size_t, void*)
{
    const auto it = names().find(host);
    log() += (it == names().end() ? "?" : it->second) + " " + std::to_string((uint64_t)grid.x * grid.y * grid.z) + "\n";
    return 0;
}
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipGetLastError() { return 0; }
int hipEventRecord(void*, void*) { return 0; }
int hipGetSymbolAddress(void**, const void*) { return 1; }
int hipMemcpyAsync(void*, const void*, size_t, int, void*) { return 1; }
int hipStreamSynchronize(void*) { return 1; }

// what was launched since the last call: a line each, the kernel's mangled name and its workgroups; the length that it needs
size_t launches_taken(char* out, size_t size)
{
    const size_t n = log().size() + 1;
    if (n <= size) { memcpy(out, log().c_str(), n); log().clear(); }
    return n;
}

}  // extern "C"
