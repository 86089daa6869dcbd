// Stand-in for the HIP runtime under libhadfl.so, for host-only tests of the head's operators: a launch is written down instead of run, and
// refused as the runtime refuses it where a dimension has 2^32 threads or more.  One line a launch: the mangled kernel, the workgroups and threads of a dimension,
// and for products of operands that lie in planes the row stride, rows and columns of both, for those through registers the columns of each that
// is a tensor of the caller's or of the workspace.
// Loaded ahead of libhadfl.so with RTLD_GLOBAL, so that its symbols are found first.
#include <hip/hip_runtime.h>

#include <cstring>
#include <map>
#include <string>

namespace {

struct Plane {                     // what direct_product.h passes as Plane3
    const void* p;
    long long rep, plane;
    int ld, lines, cols;
    const unsigned* top;
};
struct Tensor {                    // tile_product.h: Source
    const void* p;
    long long rep, row;
    int rows, cols;
};
std::map<const void*, std::string> g_names;
std::string g_trace;
dim3 g_grid, g_block;
size_t g_shmem;
hipStream_t g_stream;
hipError_t g_last = hipSuccess;

}  // namespace

extern "C" {

void check_reset(void) { g_trace.clear(); g_last = hipSuccess; }
const char* check_trace(void) { return g_trace.c_str(); }
const char* check_names(void)                                  // every kernel of the library, mangled, one a line
{
    static std::string all;
    all.clear();
    for (const auto& k : g_names) all += k.second + "\n";
    return all.c_str();
}

void** __hipRegisterFatBinary(const void*) { static void* h; return &h; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { g_names[host] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shmem, hipStream_t s)
{
    g_grid = grid; g_block = block; g_shmem = shmem; g_stream = s;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shmem, hipStream_t* s)
{
    *grid = g_grid; *block = g_block; *shmem = g_shmem; *s = g_stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t)
{
    const unsigned g[3] = {grid.x, grid.y, grid.z}, b[3] = {block.x, block.y, block.z};
    for (int i = 0; i < 3; ++i)
        if (!g[i] || (unsigned long long)g[i] * b[i] >> 32) return g_last = hipErrorInvalidConfiguration;
    const std::string& name = g_names[f];
    g_trace += name;
    for (int i = 0; i < 3; ++i) g_trace += " " + std::to_string(g[i]) + " " + std::to_string(b[i]);
    if (name.find("13direct_kernel") != std::string::npos || name.find("19layer_planes_kernel") != std::string::npos)
        for (int i = 0; i < 2; ++i) {
            Plane p;
            std::memcpy(&p, args[i], sizeof(p));
            g_trace += " " + std::to_string(p.ld) + " " + std::to_string(p.lines) + " " + std::to_string(p.cols);
        }
    if (name.find("14product_kernel") != std::string::npos || name.find("20layer_product_kernel") != std::string::npos)
        for (int i = name.find("14product_kernelINS0_6Source") == std::string::npos && name.find("20layer_product_kernel") == std::string::npos; i < 2; ++i) {
            Tensor t;
            std::memcpy(&t, args[i], sizeof(t));
            g_trace += " " + std::to_string(t.cols);
        }
    g_trace += "\n";
    return hipSuccess;
}
hipError_t hipMemcpyAsync(void*, const void*, size_t, hipMemcpyKind, hipStream_t) { return hipErrorNotSupported; }
hipError_t hipHostMalloc(void**, size_t, unsigned) { return hipErrorNotSupported; }
hipError_t hipHostFree(void*) { return hipErrorNotSupported; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600*, int) { return hipErrorNotSupported; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetSymbolAddress(void**, const void*) { return hipErrorNotSupported; }
hipError_t hipGetLastError(void) { const hipError_t e = g_last; g_last = hipSuccess; return e; }
const char* hipGetErrorString(hipError_t) { return "error"; }
hipError_t hipStreamCreateWithFlags(hipStream_t*, unsigned) { return hipErrorNotSupported; }
hipError_t hipStreamDestroy(hipStream_t) { return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipEventCreate(hipEvent_t*) { return hipErrorNotSupported; }
hipError_t hipEventCreateWithFlags(hipEvent_t*, unsigned) { return hipErrorNotSupported; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventElapsedTime(float*, hipEvent_t, hipEvent_t) { return hipErrorNotSupported; }

}
