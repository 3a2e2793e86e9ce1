// Launches without a GPU: this program takes the place of the HIP runtime's launch functions and looks at what the library
// would launch.  The limit of a kernel's dynamic LDS belongs to the kernel on its device and not to a call: another thread's call
// may set it between a call's own setting and its launch, so all calls have to set the same, and it has to hold for every launch.
// Built against the library and run by tests/test_launches_cpu.py.
#define __HIP_PLATFORM_AMD__
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <map>

#include "spo.h"

static constexpr size_t kDefaultLds = 64 * 1024, kMostLds = 160 * 1024;
struct Limits {
    int least = INT32_MAX, most = 0;
    size_t asked = 0;  // the largest launch's
};
static std::map<const void *, Limits> kernels;
static size_t pushed_lds;
static long long launches;

extern "C" {
hipError_t hipFuncSetAttribute(const void *f, hipFuncAttribute, int value) {
    Limits &l = kernels[f];
    l.least = value < l.least ? value : l.least;
    l.most = value > l.most ? value : l.most;
    return hipSuccess;
}
hipError_t __hipPushCallConfiguration(dim3, dim3, size_t lds, hipStream_t) {
    pushed_lds = lds;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *s) {
    *grid = *block = dim3(1, 1, 1);
    *lds = pushed_lds;
    *s = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3, dim3, void **, size_t lds, hipStream_t) {
    ++launches;
    Limits &l = kernels[f];
    l.asked = lds > l.asked ? lds : l.asked;
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
}

// non-NULL, aligned dummies: never dereferenced on the host
static float *f = reinterpret_cast<float *>(uintptr_t(1) << 20);
static int32_t *ids = reinterpret_cast<int32_t *>(uintptr_t(1) << 21);
static void *ws = reinterpret_cast<void *>(uintptr_t(1) << 22);
static const size_t big = size_t(1) << 50;
static int failures = 0;
#define EXPECT(what)                                                            \
    do {                                                                        \
        if (!(what)) {                                                          \
            std::fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #what);     \
            ++failures;                                                         \
        }                                                                       \
    } while (0)

int main() {
    for (int64_t T : {1, 2, 3, 5, 16, 17, 300})
        for (int64_t H : {64, 256, 768, 1024, 4096, 8192, 16384, 65536})
            for (int64_t V : {17, 3000, 40000, 151936}) {
                spo_logprob_desc d{};
                d.struct_size = sizeof d;
                d.dtype = SPO_BF16;
                d.T = T, d.H = H, d.V = V;
                d.hidden = d.W = f;
                d.target = ids;
                EXPECT(spo_logprob_fwd(&d, f, f, f, nullptr, nullptr, ws, big, nullptr) == SPO_OK);
                EXPECT(spo_logprob_bwd(&d, f, f, f, f, nullptr, nullptr, f, SPO_BF16, f, SPO_BF16, 0, nullptr, 0, ws, big, nullptr) == SPO_OK);
            }
    for (int products : {SPO_PRODUCTS_FP16, SPO_PRODUCTS_SPLIT})
        for (int64_t batch : {1, 4})
            for (int64_t rows : {10, 300, 1024, 2048, 4096})
                for (int64_t cols : {20, 1000, 4096}) {
                    spo_orth_desc d{};
                    d.struct_size = sizeof d;
                    d.batch = batch, d.rows = rows, d.cols = cols, d.steps = 5, d.products = products;
                    EXPECT(spo_orthogonalize(&d, f, SPO_BF16, 0, 0, f, SPO_FP32, ws, big, nullptr) == SPO_OK);
                }
    EXPECT(launches > 1000);
    int limited = 0;
    for (const auto &k : kernels) {
        const Limits &l = k.second;
        limited += l.most > 0;
        if (l.most > 0 && l.least != l.most) {
            std::fprintf(stderr, "a kernel's limit is set to %d by one call and %d by another\n", l.least, l.most);
            ++failures;
        }
        EXPECT(l.asked <= (l.most > 0 ? static_cast<size_t>(l.most) : kDefaultLds));
        EXPECT(l.asked <= kMostLds);
    }
    EXPECT(limited > 10);
    if (failures) return 1;
    std::puts("limits are the kernels' own");
    return 0;
}
