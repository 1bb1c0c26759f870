// Which kernels a call of the products launches, without a GPU: librtoss.so linked against stand-ins for the few runtime calls it makes, on a
// device of 256 compute units.  Reads calls, one a line,
//     what dt M K N pitch rows weights
// (what: 0 8-bit product, 1 gated block, 2 gated block in 8 bits, 3 its gradients, of the rows and of the weights where asked for, 4 row codes; dt: of the
// result, or of all; pitch: elements that operands' rows lie further apart than they are long, their first element pitch / 2 elements behind an
// aligned address) and prints the status and, for every launch, the kernel's handle (its offset in the library), the number of workgroups and lanes,
// the dynamic LDS and the limit that was set for it.
#include <dlfcn.h>
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <map>
#include <vector>

#include "rtoss.h"

struct Launch {
    const void* kernel;
    dim3 grid, block;
    size_t lds;
};
static std::vector<Launch> g_launches;
static std::map<const void*, int> g_limit;
static Launch g_call;

extern "C" {
hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }
hipError_t hipFuncSetAttribute(const void* kernel, hipFuncAttribute, int bytes) { return g_limit[kernel] = bytes, hipSuccess; }
hipError_t hipOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void*, int, size_t) { return *n = 2, hipSuccess; }
hipError_t hipLaunchKernel(const void* kernel, dim3 grid, dim3 block, void**, size_t lds, hipStream_t)
{
    return g_launches.push_back(Launch{kernel, grid, block, lds}), hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t) { return g_call = Launch{nullptr, grid, block, lds}, hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t*)
{
    return *grid = g_call.grid, *block = g_call.block, *lds = g_call.lds, hipSuccess;
}
}

int main()
{
    int what, dt, K, N, pitch, rows, weights;
    long long M;
    while (scanf("%d %d %lld %d %d %d %d %d", &what, &dt, &M, &K, &N, &pitch, &rows, &weights) == 8) {
        // addresses that nothing reads, further from one another than any matrix is long
        const auto at = [](int i, size_t offset = 0) { return (char*)((size_t)(i + 1) << 42) + offset; };
        const size_t eb = what == 0 || what == 2 ? 1 : dt == RTOSS_F32 ? 4 : 2, first = pitch / 2 * eb;
        const int64_t ld = pitch ? K + pitch : 0;
        const rtoss_gated_desc g{M, K, N, (rtoss_dtype)dt, RTOSS_ACT_SILU, ld, ld, what == 3 && pitch ? N + pitch : 0};
        g_launches.clear();
        rtoss_status st = RTOSS_EINVAL;
        if (what == 0) {
            const rtoss_matmul_desc d{M, N, K, ld, ld, (rtoss_dtype)dt};
            st = rtoss_matmul_i8(&d, (int8_t*)at(0, first), nullptr, (int8_t*)at(1, first), nullptr, at(2), nullptr);
        } else if (what == 1) {
            st = rtoss_gated_ff(&g, at(0, first), at(1, first), at(2, first), at(3), nullptr, nullptr, nullptr);
        } else if (what == 2) {
            st = rtoss_gated_ff_i8(&g, (int8_t*)at(0, first), nullptr, (int8_t*)at(1, first), nullptr, (int8_t*)at(2, first), nullptr, at(3), nullptr);
        } else if (what == 3) {
            size_t bytes = 0;
            st = rtoss_gated_ff_backward_size(&g, &bytes);
            if (st == RTOSS_OK)
                st = rtoss_gated_ff_backward(&g, at(0, first), at(1, first), at(2, first), at(3, first), at(4), at(5), rows ? at(6) : nullptr,
                                             weights ? at(7) : nullptr, weights ? at(8) : nullptr, at(9), bytes, nullptr);
        } else {
            st = rtoss_quantize_rows(at(0, first), (rtoss_dtype)dt, M, K, ld, (int8_t*)at(1), 0, (float*)at(2), nullptr);
        }
        printf("%d", (int)st);
        for (const Launch& l : g_launches) {
            Dl_info info{};
            size_t offset = 0;
            if (dladdr(l.kernel, &info)) offset = (size_t)((const char*)l.kernel - (const char*)info.dli_fbase);
            const auto limit = g_limit.find(l.kernel);
            printf(" %zx %llu %u %zu %d", offset, (unsigned long long)l.grid.x * l.grid.y, l.block.x, l.lds, limit == g_limit.end() ? 64 * 1024 : limit->second);
        }
        printf("\n");
    }
    return 0;
}
