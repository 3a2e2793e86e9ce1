// Launches without a GPU: this program takes the place of the HIP runtime's launch functions and looks at what normalisations and
// AdamW steps would launch: within a launch's limits whatever the sizes, and as few launches as the header says.  Built against
// the library and run by tests/test_train_cpu.py.
#define __HIP_PLATFORM_AMD__
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include <map>
#include <vector>

#include "spo.h"

static long long launches;
static int failures = 0;
#define EXPECT(what)                                                        \
    do {                                                                    \
        if (!(what)) {                                                      \
            std::fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #what); \
            ++failures;                                                     \
        }                                                                   \
    } while (0)

static std::map<const void *, int> limits;
static struct {
    dim3 grid, block;
    size_t lds;
} pushed;

extern "C" {
hipError_t hipFuncSetAttribute(const void *f, hipFuncAttribute, int value) {
    EXPECT(!limits.count(f) || limits[f] == value);   // a kernel's own, whatever the call
    limits[f] = value;
    return hipSuccess;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t) {
    pushed = {grid, block, lds};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *s) {
    *grid = pushed.grid, *block = pushed.block, *lds = pushed.lds, *s = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **, size_t lds, hipStream_t) {
    ++launches;
    const uint64_t threads = uint64_t(block.x) * block.y * block.z;
    EXPECT(grid.x > 0 && grid.y > 0 && grid.z == 1 && threads > 0 && threads <= 1024);
    EXPECT(uint64_t(grid.x) * block.x < uint64_t(1) << 32 && grid.y < 65536);
    EXPECT(lds <= size_t(limits.count(f) ? limits[f] : 64 * 1024) && lds <= 160 * 1024);
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
}

// non-NULL, aligned dummies: never dereferenced on the host
static float *f = reinterpret_cast<float *>(uintptr_t(1) << 20);
static uint8_t *codes = reinterpret_cast<uint8_t *>(uintptr_t(1) << 21);
static void *ws = reinterpret_cast<void *>(uintptr_t(1) << 22);
static const size_t big = size_t(1) << 60;

static long long counted(int rc) {
    EXPECT(rc == SPO_OK);
    const long long n = launches;
    launches = 0;
    return n;
}

int main() {
    for (int64_t rows : {1LL, 2LL, 3LL, 700LL, 8192LL, 300000LL, 5000000LL, (1LL << 31) - 1})
        for (int64_t cols = 1; cols <= 65536; cols += cols < 70 ? 1 : cols / 9)
            for (int types = 0; types < 8; ++types) {
                spo_norm_desc d{};
                d.struct_size = sizeof d;
                d.kind = types & 1;
                d.x_dtype = types >> 1 & 1;
                d.y_dtype = types >> 2 & 1;
                d.rows = rows, d.cols = cols;
                d.x = d.weight = d.bias = f;
                EXPECT(counted(spo_norm_fwd(&d, f, 0, f, f, nullptr)) == 1);
                const long long most = cols <= 16384 ? 2 : 3;
                EXPECT(counted(spo_norm_bwd(&d, f, f, f, d.y_dtype, 0, f, d.x_dtype, f, f, SPO_FP32, 0, ws, big, nullptr)) == most);
                EXPECT(counted(spo_norm_bwd(&d, f, f, f, d.y_dtype, 0, f, d.x_dtype, nullptr, nullptr, 0, 0, ws, big, nullptr)) == most - 1);
            }
    for (int bits : {32, 8})
        for (int count : {1, 2, 48, 49, 60, 61, 500})
            for (int64_t n : {1LL, 64LL, 100000LL, 1LL << 33, 1LL << 35}) {
                spo_adamw_tensor t{};
                t.param = t.m = t.v = f;
                t.grad = f;
                t.m_scale = t.v_scale = codes;
                t.n = n;
                std::vector<spo_adamw_tensor> of(count, t);
                const spo_adamw_desc d{sizeof(spo_adamw_desc), bits, count, of.data()};
                const int held = bits == 32 ? 60 : 48;
                const long long want = (count + held - 1) / held;
                EXPECT(counted(spo_adamw_update(&d, 1e-3, nullptr, 0.9, 0.999, 1e-8, 5, nullptr, f, 1.0, 0, nullptr, 0, nullptr)) == want);
                EXPECT(counted(spo_adamw_update(&d, 1e-3, f, 0.9, 0.999, 1e-8, 5, nullptr, f, 1.0, 0, ws, big, nullptr)) == want + 1);
                EXPECT(counted(spo_grad_norm(&d, f, ws, big, nullptr)) == (count + 159) / 160 + 1);
                EXPECT(counted(spo_adamw_state_values(codes, codes, codes, codes, n, f, f, SPO_BF16, nullptr)) == 1);
            }
    if (failures) return 1;
    std::puts("launches within their limits");
    return 0;
}
