// Products of orthogonalised updates (csrc/orth_choice.hpp): room for the sums of squares that any kind of tiles leaves, or, with
// batch, rows, cols and products as arguments, the kinds that are chosen.
#define __host__
#define __device__
#define __forceinline__ inline

#include "orth_choice.hpp"

#include <cstdio>
#include <cstdlib>

using namespace spo;

int main(int argc, char **argv) {
    if (argc == 5) {
        const int64_t batch = std::atoll(argv[1]), rows = std::atoll(argv[2]), cols = std::atoll(argv[3]);
        const OrthKinds q = orth_kinds(padded(std::min(rows, cols)), padded(std::max(rows, cols)), batch,
                                       as_pairs(std::min(rows, cols), std::atoi(argv[4]) != 0));
        const char *name[] = {"few", "small", "middle", "large"};
        std::printf("%s %s %s\n", name[static_cast<int>(q.gram)], name[static_cast<int>(q.poly)], name[static_cast<int>(q.update)]);
        return 0;
    }
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
