// The layers' search for the band of a work item, on the host: the device's
// rounds of 64 lanes are walked one lane at a time, over the same arithmetic.
// Every item of random layouts is compared with a plain scan over the bands;
// with offsets in any order, no tile may leave the row.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../../paper_2609_29119_amd/csrc/layers/tile.hpp"

using namespace nsl;

static Tile<int64_t> search(const std::vector<int64_t>& off, int rows, int64_t mult, int shift, int64_t p) {
    const int n_bands = static_cast<int>(off.size()) - 1;
    BandSearch s(n_bands);
    int bound[64] = {};
    while (s.more()) {
        s.open();
        int count = 0;
        for (int lane = 0; lane < 64; ++lane) {
            const int i = s.lo + lane * s.step;
            bound[lane] = band_bound(off.data(), n_bands, rows, i);
            count += i < s.hi && item_from<int64_t>(mult, bound[lane], shift, i, p);
        }
        s.close(count);
    }
    const int b = s.next_held() ? bound[s.at + 1] : band_bound(off.data(), n_bands, rows, s.lo + 1);
    return tile_of<int64_t>(s.lo, bound[s.at], b, mult, shift, p);
}

static int fail(const char* what, int n_bands, long long p) {
    std::printf("%s: %d bands, item %lld\n", what, n_bands, p);
    return 1;
}

int main(int argc, char** argv) {
    std::mt19937 rng(argc > 1 ? std::atoi(argv[1]) : 0);
    std::vector<int> counts = {0, 1, 2, 61, 62, 63, 64, 65, 126, 127, 128, 221, 4000, 5000, 5121, 8190, 8191, 12000, 20000};
    for (int n = 4030; n <= 4200; ++n) counts.push_back(n);
    long long wrong = 0;
    for (int n_bands : counts) {
        const int shift = 5 + static_cast<int>(rng() % 5), longest = 1 + static_cast<int>(rng() % 200);
        const int64_t mult = 1 + rng() % 3;
        std::vector<int64_t> off(n_bands + 1);
        off[0] = rng() % 50;
        for (int g = 0; g < n_bands; ++g) off[g + 1] = off[g] + (rng() % 8 ? rng() % longest : 0);
        const int rows = static_cast<int>(off[n_bands] + rng() % 50);
        const int64_t items = tile_count(shift, n_bands, mult, rows);
        // a plain scan: band g - 1's items begin at floor(mult start / 2^shift) + g
        std::vector<char> seen(static_cast<size_t>(mult) * rows / 1 + 1, 0);
        int g = 0;
        for (int64_t p = 0; p < items; ++p) {
            while (g + 1 < n_bands + 2 && item_from<int64_t>(mult, band_bound(off.data(), n_bands, rows, g + 1), shift, g + 1, p))
                ++g;
            const Tile<int64_t> t = search(off, rows, mult, shift, p);
            const int a = band_bound(off.data(), n_bands, rows, g), b = band_bound(off.data(), n_bands, rows, g + 1);
            if (t.band != g - 1 || t.start != a || t.len != b - a) ++wrong;
            if (wrong == 1 && (t.band != g - 1 || t.start != a || t.len != b - a)) fail("wrong band", n_bands, p);
            if (t.live && !wrong)   // every row of every band belongs to one item
                for (int64_t r = t.first; r < t.first + (int64_t(1) << shift) && r < mult * t.len; ++r)
                    if (seen[mult * t.start + r]++) return fail("a row of two items", n_bands, p);
        }
        if (!wrong)
            for (int64_t r = 0; r < mult * rows; ++r)
                if (!seen[r]) return fail("a row of no item", n_bands, r);
        // offsets in any order, and past the row: in range all the same
        for (auto& o : off) o = rng() % 3 ? static_cast<int64_t>(rng() % (rows + 1)) : static_cast<int64_t>(rng()) - (1LL << 31);
        for (int64_t p = 0; p < items; p += 1 + rng() % 5) {
            const Tile<int64_t> t = search(off, rows, mult, shift, p);
            if (t.band < -1 || t.band > n_bands) return fail("band out of range", n_bands, p);
            if (t.start < 0 || t.len < 0 || t.start + t.len > rows) return fail("tile out of range", n_bands, p);
        }
        // the join of a band's chunks, from its own two bounds: items in range
        for (int band = 0; band < n_bands; ++band) {
            const int64_t b0 = band_bound(off.data(), n_bands, rows, band + 1), b1 = band_bound(off.data(), n_bands, rows, band + 2);
            const int64_t n_rows = b1 > b0 ? (b1 - b0) * mult : 0, chunks = (n_rows + (int64_t(1) << shift) - 1) >> shift;
            if (chunks && ((b0 * mult) >> shift) + band + 1 + chunks > items) return fail("chunk out of range", n_bands, band);
        }
    }
    if (wrong) std::printf("%lld wrong items\n", wrong);
    return wrong ? 1 : 0;
}
