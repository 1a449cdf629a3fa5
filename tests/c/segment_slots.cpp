// The slots of long bands' segments: for any ascending offsets no two segments share one, and none lies past the last.
#include <stdio.h>
#include <stdlib.h>

#include <set>
#include <vector>

#include "../../paper_2609_29119_amd/csrc/layers/tile.hpp"

int main(int argc, char** argv) {
    srand(argc > 1 ? atoi(argv[1]) : 0);
    for (int turn = 0; turn < 4000; ++turn) {
        const int shift = 6 + rand() % 7, fine = shift - rand() % (shift - 5);
        std::vector<int64_t> off = {rand() % 50};
        const int bands = 1 + rand() % 40;
        for (int i = 0; i < bands; ++i) {
            const int kind = rand() % 4, t = 1 << shift;
            off.push_back(off.back() + (kind == 0 ? 0 : kind == 1 ? t + rand() % 3 - 1 : kind == 2 ? rand() % (5 * t) : rand() % 40));
        }
        const int64_t rows = off.back() + rand() % 20, count = nsl::slot_count(rows, fine);
        std::set<int64_t> taken;
        for (int i = 0; i < bands; ++i) {
            const int64_t len = off[i + 1] - off[i];
            if (len <= int64_t(1) << shift) continue;   // bands of one segment have none
            for (int64_t s = 0; s << fine < len; ++s) {
                const int64_t slot = nsl::slot_of(off[i], s, fine);
                if (slot < 0 || slot >= count || !taken.insert(slot).second) {
                    printf("turn %d: band %d, segment %lld: slot %lld of %lld\n", turn, i, (long long)s, (long long)slot, (long long)count);
                    return 1;
                }
            }
        }
    }
    return 0;
}
