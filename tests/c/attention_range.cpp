// Index arithmetic of the attention's kernels at the longest rows, on the host.
#include <cstdio>

#include "../../paper_2609_29119_amd/csrc/layers/attention.hpp"

int main() {
    const int longest = (1 << 30) - 1;
    int bad = 0;
    for (int k0 : {0, 128, longest / 128 * 128, (longest / 128 - 1) * 128})
        for (int left : {0, 1, longest - 128, longest})
            for (int len : {1, 200, longest}) {
                const long long want = static_cast<long long>(k0) + 128 + left;
                bad += nsl::queries_end(k0, left, len) != (want < len ? want : len);
            }
    if (bad) std::printf("%d wrong ends\n", bad);
    return bad != 0;
}
