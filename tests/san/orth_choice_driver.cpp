// Products of orthogonalised updates (csrc/orth_choice.hpp): room for the sums of squares that any kind of tiles leaves.
#define __host__
#define __device__
#define __forceinline__ inline

#include "orth_choice.hpp"

#include <cstdio>

using namespace spo;

int main() {
    int bad = 0;
    for (int64_t k = 64; k <= 65536; k += k < 2048 ? 64 : 4032)
        for (int64_t L = k; L <= 65536; L += L < 2048 ? 64 : 4032)
            for (Kind kind : {Kind::few, Kind::small, Kind::middle, Kind::large})
                if (square_sums(k, L, kind) > square_room(k, L) && bad++ < 10)
                    std::fprintf(stderr, "%lld x %lld on tiles of %lld: %lld sums, room for %lld\n", (long long)k, (long long)L,
                                 (long long)edge_of(kind), (long long)square_sums(k, L, kind), (long long)square_room(k, L));
    if (bad) return 1;
    std::printf("sums of squares have room\n");
    return 0;
}
