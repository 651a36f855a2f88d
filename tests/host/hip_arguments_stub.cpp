// hip_runtime_stub.cpp with two things more: what a kernel is given (as int32, by its place), and a current device that can be changed.
#define hipLaunchKernel stub_plain_launch
#define hipGetDevice stub_plain_device
#include "hip_runtime_stub.cpp"
#undef hipLaunchKernel
#undef hipGetDevice

static std::vector<std::vector<int>> g_ints;
static int g_device = 0, g_count = 0;

extern "C" {
// from here on the first `count` arguments of every launch are kept, each read as an int32 (every kernel has to have as many)
void stub_keep_arguments(int count) { g_count = count; g_ints.clear(); }
size_t stub_kept() { return g_ints.size(); }
int stub_argument(size_t launch, int at) { return g_ints[launch][at]; }
void stub_set_device(int d) { g_device = d; }
int hipGetDevice(int *d) { *d = g_device; return 0; }
int hipLaunchKernel(const void *kernel, Dim3 grid, Dim3 block, void **args, size_t lds, void *stream)
{
    std::vector<int> v(g_count);
    for (int i = 0; i < g_count; i++) std::memcpy(&v[i], args[i], sizeof(int));
    if (g_count) g_ints.push_back(v);
    return stub_plain_launch(kernel, grid, block, args, lds, stream);
}
}
