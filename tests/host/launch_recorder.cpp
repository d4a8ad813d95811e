// Stands in for the HIP runtime under libleap_hip.so on a machine without a GPU: every launch is written down, nothing runs.
// Loaded before the library, with its symbols global; the library's calls then end here (test infrastructure, built with g++).
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <map>
#include <string>

namespace {
struct grid3 {
    uint32_t x, y, z;
};
struct configuration {
    grid3 grid, block;
    size_t shared;
    void *stream;
};
configuration g_pending;
std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> n;
    return n;
}
std::string &record()
{
    static std::string r;
    return r;
}
}  // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *)
{
    static void *modules;
    return &modules;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names()[host] = name; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
int __hipPushCallConfiguration(grid3 grid, grid3 block, size_t shared, void *stream)
{
    g_pending = {grid, block, shared, stream};
    return 0;
}
int __hipPopCallConfiguration(grid3 *grid, grid3 *block, size_t *shared, void **stream)
{
    *grid = g_pending.grid, *block = g_pending.block, *shared = g_pending.shared, *stream = g_pending.stream;
    return 0;
}
int hipLaunchKernel(const void *host, grid3 grid, grid3 block, void **, size_t, void *)
{
    char line[128];
    std::snprintf(line, sizeof line, " %u %u %u %u %u %u\n", grid.x, grid.y, grid.z, block.x, block.y, block.z);
    record() += names()[host] + line;
    return 0;
}
int hipGetLastError() { return 0; }

// The mangled names of all the kernels there are, a line each.
long registered_kernels(char *to, long room)
{
    std::string all;
    for (const auto &n : names()) all += n.second + "\n";
    if ((long)all.size() < room) std::memcpy(to, all.c_str(), all.size() + 1);
    return (long)all.size();
}

// What was launched since the last call: a kernel's mangled name, its blocks and its threads a line.
long recorded_launches(char *to, long room)
{
    const long n = (long)record().size();
    if (n < room) {
        std::memcpy(to, record().c_str(), n + 1);
        record().clear();
    }
    return n;
}
}
