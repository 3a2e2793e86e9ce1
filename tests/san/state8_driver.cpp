// Codes of an optimiser's moments in 8 bits on the host: reads "mantissa step" and blocks of 64 floats (their bits in hexadecimal), writes each block's
// scale, its codes and the bits of what they stand for.  Built with the sanitizers and run by tests/test_train_cpu.py.
#include <cstdio>
#include <cinttypes>

#include "state8.hpp"

template <typename C>
static void block(const float *x, uint32_t step, uint32_t start) {
    uint32_t top = 0;
    for (int i = 0; i < spo::kStateBlock; ++i) {
        const uint32_t u = spo::float_bits(x[i]) & 0x7fffffffu;
        top = u > top ? u : top;
    }
    const uint32_t scale = C::scale(top);
    std::printf("%u", scale);
    for (int i = 0; i < spo::kStateBlock; ++i) {
        const uint32_t threshold = C::threshold(spo::turn_at(spo::turn_of(step, start), static_cast<uint32_t>(i)));
        const uint32_t code = C::encode(x[i], scale, threshold) >> 24;
        std::printf(" %u %" PRIx32, code, spo::float_bits(C::decode(code, scale)));
    }
    std::printf("\n");
}

int main() {
    int mantissa;
    uint64_t step;
    while (std::scanf("%d %" SCNu64, &mantissa, &step) == 2) {
        float x[spo::kStateBlock];
        for (float &v : x) {
            uint32_t u;
            if (std::scanf("%" SCNx32, &u) != 1) return 1;
            v = spo::bits_float(u);
        }
        if (mantissa == 3) block<spo::FirstCode>(x, static_cast<uint32_t>(step), spo::kTurnFirst);
        else block<spo::RootCode>(x, static_cast<uint32_t>(step), spo::kTurnRoot);
    }
    return 0;
}
