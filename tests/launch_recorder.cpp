// Stands in for the HIP runtime in a process without a GPU: kernels are noted, none runs.  Loaded with global visibility before libgp.so,
// whose calls of the functions below then end here (tests/launches.py).
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <map>
#include <new>
#include <string>
#include <vector>

namespace {

struct Dim3 {
    uint32_t x, y, z;
};
struct Launch {
    const void* function;
    Dim3 grid, block;
    uint64_t lds, lds_asked;
};
struct Pending {
    Dim3 grid, block;
    size_t lds;
    void* stream;
};

struct Recorder {
    std::map<const void*, std::string> names;
    std::map<const void*, uint64_t> asked;  // dynamic LDS that hipFuncSetAttribute allowed
    std::vector<Launch> launches;
    std::vector<Pending> pending;
};
Recorder& recorder()
{
    static Recorder* r = new Recorder;
    return *r;
}
bool g_no_memory = false;

}  // namespace

extern "C" {

int hipGetDevice(int* device) { return *device = 0, 0; }
int hipGetLastError() { return 0; }
const char* hipGetErrorString(int) { return "(recorded)"; }
int hipEventCreate(void** event) { return *event = malloc(1), 0; }
int hipEventDestroy(void* event) { return free(event), 0; }
int hipEventRecord(void*, void*) { return 0; }
int hipFuncSetAttribute(const void* function, int, int value) { return recorder().asked[function] = (uint64_t)value, 0; }

void __hipRegisterFunction(void**, const void* function, char*, const char* name, unsigned, void*, void*, void*, void*, int*)
{
    recorder().names[function] = name;
}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void* stream)
{
    return recorder().pending.push_back({grid, block, lds, stream}), 0;
}
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream)
{
    const Pending p = recorder().pending.back();
    recorder().pending.pop_back();
    return *grid = p.grid, *block = p.block, *lds = p.lds, *stream = p.stream, 0;
}
int hipLaunchKernel(const void* function, Dim3 grid, Dim3 block, void**, size_t lds, void*)
{
    Recorder& r = recorder();
    const auto asked = r.asked.find(function);
    return r.launches.push_back({function, grid, block, lds, asked == r.asked.end() ? 0 : asked->second}), 0;
}

// what was noted since the last recorder_clear
int64_t recorder_count() { return (int64_t)recorder().launches.size(); }
const char* recorder_name(int64_t i) { return recorder().names[recorder().launches[i].function].c_str(); }
void recorder_sizes(int64_t i, uint64_t out[8])
{
    const Launch& l = recorder().launches[i];
    const uint64_t v[8] = {l.grid.x, l.grid.y, l.grid.z, l.block.x, l.block.y, l.block.z, l.lds, l.lds_asked};
    memcpy(out, v, sizeof v);
}
void recorder_clear() { recorder().launches.clear(); }
// libgp.so's own allocations fail from here on, or no longer
void recorder_no_memory(int on) { g_no_memory = on != 0; }

}  // extern "C"

void* operator new(size_t bytes)
{
    void* const p = g_no_memory ? nullptr : malloc(bytes ? bytes : 1);
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }
