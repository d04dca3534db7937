// Stands in for the HIP runtime's launch functions in a process without a GPU:
// records which kernel a call would launch, with which grid, on which of several
// pretended devices, and which kernels had their LDS limit raised there.  Loaded
// with its symbols global before the library, so that the library's calls come here.
#include <cxxabi.h>
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <string>
#include <vector>

namespace {
struct Dim3 {
    uint32_t x, y, z;
};
struct Call {
    Dim3 grid, block;
    size_t shared;
    void *stream;
};
std::map<const void *, std::string> &kernels() {
    static std::map<const void *, std::string> k;
    return k;
}
std::vector<std::string> &events() {
    static std::vector<std::string> e;
    return e;
}
std::vector<Call> pushed;
int device = 0, refusals = 0;

std::string name_of(const void *f) {
    const auto it = kernels().find(f);
    return it == kernels().end() ? "?" : it->second;
}
}  // namespace

extern "C" {

void __hipRegisterFunction(void **, const void *host, char *, const char *mangled, unsigned, void *, void *, void *,
                           void *, int *) {
    int status = 0;
    char *plain = abi::__cxa_demangle(mangled, nullptr, nullptr, &status);
    kernels()[host] = plain ? plain : mangled;
    free(plain);
}

int hipGetDevice(int *d) {
    *d = device;
    return 0;
}
int hipGetLastError() { return 0; }

int hipFuncSetAttribute(const void *f, int, int value) {
    if (refusals > 0) {
        --refusals;
        return 1;
    }
    events().push_back("attribute\t" + std::to_string(device) + "\t" + name_of(f) + "\t" + std::to_string(value));
    return 0;
}

int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t shared, void *stream) {
    pushed.push_back({grid, block, shared, stream});
    return 0;
}
int __hipPopCallConfiguration(Dim3 *grid, Dim3 *block, size_t *shared, void **stream) {
    const Call c = pushed.back();
    pushed.pop_back();
    *grid = c.grid, *block = c.block, *shared = c.shared, *stream = c.stream;
    return 0;
}
int hipLaunchKernel(const void *f, Dim3 grid, Dim3 block, void **, size_t shared, void *) {
    char sizes[160];
    snprintf(sizes, sizeof sizes, "\t%u %u %u\t%u\t%zu", grid.x, grid.y, grid.z, block.x * block.y * block.z, shared);
    events().push_back("launch\t" + std::to_string(device) + "\t" + name_of(f) + sizes);
    return 0;
}

void recorder_device(int d) { device = d; }
void recorder_refuse(int n) { refusals = n; }
void recorder_clear() { events().clear(); }
int recorder_events() { return (int)events().size(); }
const char *recorder_event(int i) { return events()[(size_t)i].c_str(); }
int recorder_kernels() { return (int)kernels().size(); }
const char *recorder_kernel(int i) {
    auto it = kernels().begin();
    std::advance(it, i);
    return it->second.c_str();
}
}
