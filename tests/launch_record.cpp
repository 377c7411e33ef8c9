// A stand-in for the HIP runtime, linked with the host half of zs_fp8_gemm.hip on a machine without a GPU: which kernels
// a product launches.  Each line of the input is a product, "f32|bf16 M N K w_rows workspace_bytes"; the line printed for it is
// the status and then "kernel grid" for each launch.  No kernel runs and no operand is read.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "zipserv.h"

namespace {
std::map<const void *, std::string> &names() // of the kernels, by their host address (registered before main)
{
    static std::map<const void *, std::string> all;
    return all;
}
struct Launch {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} pushed;
std::string launched;
} // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *p; return &p; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *)
{
    names()[host] = name;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream)
{
    pushed = {grid, block, lds, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = pushed.grid, *block = pushed.block, *lds = pushed.lds, *stream = pushed.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3, void **, size_t, hipStream_t)
{
    launched += " " + names()[f] + " " + std::to_string(grid.x);
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipGetDevice(int *device)
{
    *device = 0;
    return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void *, hipFuncAttribute, int) { return hipSuccess; }
int zs_compute_units(void) { return 256; }
}

int main(int argc, char **)
{
    if (argc > 1) { // the kernels that there are
        for (const auto &k : names()) std::printf("%s\n", k.second.c_str());
        return 0;
    }
    char out[8];
    long long m, n, k, room;
    int w_rows;
    while (std::scanf("%7s %lld %lld %lld %d %lld", out, &m, &n, &k, &w_rows, &room) == 6) {
        const auto at = reinterpret_cast<uint8_t *>(1 << 20); // (nothing reads it)
        const auto scales = reinterpret_cast<const float *>(at);
        void *const scratch = room ? at : nullptr;
        const int64_t ld = (k + 15) / 16 * 16, ldc = (n + 3) / 4 * 4, ldsw = (n + w_rows - 1) / w_rows;
        launched.clear();
        const int rc = std::strcmp(out, "f32") == 0
                           ? zs_fp8_gemm(at, ld, scales, m, at, ld, scales, ldsw, w_rows, reinterpret_cast<float *>(at), ldc, m, n, k, scratch, room, nullptr)
                           : zs_fp8_gemm_bf16(at, ld, scales, m, at, ld, scales, ldsw, w_rows, reinterpret_cast<uint16_t *>(at), ldc, m, n, k, scratch, room, nullptr);
        std::printf("%d%s\n", rc, launched.c_str());
    }
    return 0;
}
