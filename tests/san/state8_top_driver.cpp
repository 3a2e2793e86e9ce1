// A block's scale from its 64 values as the step's kernel forms it: reads "mantissa" and blocks of 64 floats (their bits in hexadecimal), writes each block's
// scale and whether all that its codes stand for is NaN.  Built with the sanitizers and run by tests/test_train_edges_cpu.py.
#include <cinttypes>
#include <cstdio>

#include "state8.hpp"

template <typename C>
static void block(const float *x) {
    uint32_t top = 0;
    for (int i = 0; i < spo::kStateBlock; ++i) {
        const uint32_t u = C::magnitude(x[i]);
        top = u > top ? u : top;
    }
    const uint32_t scale = C::scale(top);
    bool none = true;
    for (int i = 0; i < spo::kStateBlock; ++i) {
        const float held = C::decode(C::encode(x[i], scale, C::threshold(spo::turn_at(5, static_cast<uint32_t>(i)))) >> 24, scale);
        none = none && held != held;
    }
    std::printf("%u %d\n", scale, none ? 1 : 0);
}

int main() {
    int mantissa;
    while (std::scanf("%d", &mantissa) == 1) {
        float x[spo::kStateBlock];
        for (float &v : x) {
            uint32_t u;
            if (std::scanf("%" SCNx32, &u) != 1) return 1;
            v = spo::bits_float(u);
        }
        if (mantissa == 3) block<spo::FirstCode>(x);
        else block<spo::RootCode>(x);
    }
    return 0;
}
