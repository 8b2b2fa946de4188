// The pieces of the attention over the paged K/V cache (kv_split.h) where the lengths' sum is near and beyond 2^32: requests
// may be 2^30 tokens long and share blocks.  Pieces cover a request, and there are no more of them than B + S.
#include <cstdio>
#include <random>
#include <vector>

#include "../../paper_2501_01792_amd/csrc/kv_split.h"

using namespace hk::kvattn;

static int check(const std::vector<int> &len, int64_t S)
{
    int64_t total = 0, n = 0;
    for (int L : len) total += L;
    const int64_t C = piece_tokens(total, S);
    const unsigned __int128 least = ((unsigned __int128)total + S - 1) / S;
    const int64_t want = least < (unsigned)kStep ? kStep : (int64_t)((least + kStep - 1) / kStep * kStep);
    if (C != want) {
        std::printf("total %ld, S %ld: pieces of %ld tokens, not %ld\n", (long)total, (long)S, (long)C, (long)want);
        return 1;
    }
    for (int L : len) {
        const int64_t k = pieces_of(L, C);
        if (k < 1 || k * C < L || (k > 1 && (k - 1) * C >= L)) {
            std::printf("len %d: %ld pieces of %ld\n", L, (long)k, (long)C);
            return 1;
        }
        n += k;
    }
    if (n > (int64_t)len.size() + S) {
        std::printf("total %ld, S %ld: %ld pieces of %ld requests\n", (long)total, (long)S, (long)n, (long)len.size());
        return 1;
    }
    return 0;
}

int main()
{
    const int most = 1 << 30;
    // sums of 2^32 - 127 .. 2^32 + 127, the last one's length making up the difference
    for (int d = -127; d <= 127; ++d)
        for (int64_t S : {1, 2, 64, 127, 128, 129, 1000, 1 << 20})
            if (check({most, most, most, most / 2, most / 2 + (d < 0 ? d : 0), d > 0 ? d : 0}, S)) return 1;
    std::mt19937 rng(5);
    for (int trial = 0; trial < 20000; ++trial) {
        std::vector<int> len(1 + rng() % 9);
        for (int &L : len) L = rng() % 3 ? (int)(rng() % (uint32_t)most) + 1 : most;
        if (check(len, 1 + rng() % (1 << (1 + rng() % 21)))) return 1;
    }
    return 0;
}
