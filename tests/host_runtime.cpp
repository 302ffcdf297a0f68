// A runtime without a GPU for libaxonn_linear.so, loaded before it: launches and raised LDS limits are written down, nothing runs.
#include <cstddef>
#include <cstdint>
#include <map>
#include <string>
#include <vector>

namespace {
struct Dim { uint32_t x, y, z; };
struct Config {
    Dim grid, block;
    size_t lds;
    void* stream;
};
std::map<const void*, std::string> g_names;
std::vector<Config> g_configs;
std::string g_log;   // a line for each launch and each raised limit
unsigned char g_array[16];

void write(const char* what, const void* fn, uint64_t workgroups, uint64_t threads, uint64_t lds) {
    const auto at = g_names.find(fn);
    g_log += std::string(what) + ' ' + (at == g_names.end() ? "?" : at->second) + ' ' + std::to_string(workgroups) + ' ' + std::to_string(threads) + ' ' + std::to_string(lds) + '\n';
}
}  // namespace

extern "C" {
const char* host_runtime_log() { return g_log.c_str(); }
void host_runtime_clear() { g_log.clear(); }
const char* host_runtime_kernels() {
    g_log.clear();
    for (const auto& [fn, name] : g_names) g_log += name + '\n';
    return g_log.c_str();
}

void** __hipRegisterFatBinary(const void*) {
    static void* module;
    return &module;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* fn, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { g_names[fn] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
int __hipPushCallConfiguration(Dim grid, Dim block, size_t lds, void* stream) {
    g_configs.push_back({grid, block, lds, stream});
    return 0;
}
int __hipPopCallConfiguration(Dim* grid, Dim* block, size_t* lds, void** stream) {
    const Config c = g_configs.back();
    g_configs.pop_back();
    *grid = c.grid;
    *block = c.block;
    *lds = c.lds;
    *stream = c.stream;
    return 0;
}
int hipLaunchKernel(const void* fn, Dim grid, Dim block, void**, size_t lds, void*) {
    write("launch", fn, (uint64_t)grid.x * grid.y * grid.z, (uint64_t)block.x * block.y * block.z, lds);
    return 0;
}
int hipFuncSetAttribute(const void* fn, int, int value) {
    write("limit", fn, 0, 0, (uint64_t)value);
    return 0;
}
int hipGetDevice(int* device) {
    *device = 0;
    return 0;
}
int hipGetLastError() { return 0; }
int hipGetSymbolAddress(void** p, const void*) {
    *p = g_array;
    return 0;
}
int hipMemset(void*, int, size_t) { return 0; }
int hipMemcpy(void*, const void*, size_t, int) { return 1; }
int hipDeviceSynchronize() { return 0; }
int hipEventCreate(void**) { return 1; }
int hipEventDestroy(void*) { return 1; }
int hipEventRecord(void*, void*) { return 1; }
int hipEventSynchronize(void*) { return 1; }
int hipEventElapsedTime(float*, void*, void*) { return 1; }
}
