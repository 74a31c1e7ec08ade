// The HIP runtime that runs nothing (fake_hip.cpp), writing down as well where device memory lies and which of it is given back, and what
// X and x_scales a product of microscaled weights is launched with.
#define hipMalloc plain_malloc
#define hipFree plain_free
#define hipLaunchKernel plain_launch
#include "fake_hip.cpp"
#undef hipMalloc
#undef hipFree
#undef hipLaunchKernel

#include <cinttypes>
#include <cstdio>

namespace {
void note(const char* what, const void* p) {
    char line[64];
    std::snprintf(line, sizeof(line), "%s %" PRIxPTR, what, reinterpret_cast<uintptr_t>(p));
    calls.push_back(line);
}
}  // namespace

extern "C" {

int hipMalloc(void** p, size_t n) {
    const int e = plain_malloc(p, n);
    if (!e) note("have", *p);
    return e;
}
int hipFree(void* p) {
    note("free", p);
    return plain_free(p);
}
int hipLaunchKernel(const void* stub, Dim3 g, Dim3 b, void** args, size_t shared, void* stream) {
    const int e = plain_launch(stub, g, b, args, shared, stream);
    const std::string& name = kernels[stub];
    for (const char* of : {"mx4_rows", "mx4_ring", "mx4_tiles"})
        if (!e && name.find(of) != std::string::npos) {
            const void* const* at = static_cast<const void* const*>(args[0]);      // X and x_scales come first
            note("x", at[0]);
            note("x_scales", at[1]);
        }
    return e;
}

}  // extern "C"
