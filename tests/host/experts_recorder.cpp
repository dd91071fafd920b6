// Stands in for the HIP runtime's launch call: nothing runs, the grid and block of the last launch, its kernel's name and the last of its arguments, if that is
// how a product's operands come in (fp8_tile_kernel), are kept.
#include <hip/hip_runtime.h>

#include <map>
#include <string.h>

static std::map<const void *, const char *> &names()
{
    static std::map<const void *, const char *> of;
    return of;
}

extern "C" {
int recorded[4];   // launches so far; workgroups, threads, way of the last one
char recorded_name[512];

// what a library's kernels are called (they are registered when it is loaded, after this)
void __hipRegisterFunction(void **, const void *host, char *, const char *device, unsigned, void *, void *, void *, void *, int *) { names()[host] = device; }

hipError_t hipLaunchKernel(const void *kernel, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    ++recorded[0];
    recorded[1] = (int)(grid.x * grid.y * grid.z);
    recorded[2] = (int)(block.x * block.y * block.z);
    strncpy(recorded_name, names()[kernel], sizeof recorded_name - 1);
    recorded[3] = strstr(recorded_name, "fp8_tile_kernel") ? *static_cast<const int *>(args[3]) : -1;
    return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void *, hipFuncAttribute, int) { return hipSuccess; }
}
