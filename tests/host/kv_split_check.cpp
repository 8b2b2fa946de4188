// Replays the cut of the attention over the paged K/V cache (kv_split.h) on the host: for batches of every kind of length the
// pieces cover each request once, and there are no more of them than the launch and the scratch hold, also where the host's
// total is only a bound.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "../../paper_2501_01792_amd/csrc/kv_split.h"

using namespace hk::kvattn;

int main()
{
    std::mt19937 rng(7);
    long checked = 0;
    for (int trial = 0; trial < 4000; ++trial) {
        const int B = 1 + rng() % 70, T = 1 + rng() % 64, g = 1 << rng() % 4, Hkv = 1 + rng() % 72;
        const int top = 1 << (1 + rng() % 17);
        std::vector<int> len(B);
        int64_t total = 0;
        for (int &n : len) {
            n = rng() % 5 == 0 ? (int)(rng() % 3) : (int)(rng() % top);
            total += n;
        }
        const int64_t bound = total + (rng() % 2 ? 0 : rng() % 100000);
        const int splits = rng() % 3 ? 0 : (int)(rng() % 65);
        const Plan p = plan(B, T, (int64_t)Hkv * g, Hkv, 128, bound, splits);
        const int64_t held = (int64_t)p.tiles * 16 * (p.shared ? kWaves : 1);      // rows of a workgroup
        if (p.rows != T * g || p.tiles < 1 || p.tiles > kMaxTiles || held * p.row_groups < p.rows || held * (p.row_groups - 1) >= p.rows ||
            p.pieces != B + p.extra || p.extra < 0 || p.groups < p.pieces * Hkv * p.row_groups) {
            std::printf("plan: rows %ld tiles %d groups %d\n", (long)p.rows, p.tiles, p.row_groups);
            return 1;
        }
        const int64_t C = piece_tokens(total, p.extra);
        int64_t n = 0;
        for (int L : len) {
            const int k = pieces_of(L, C);
            if (k < 1 || (p.extra <= 0 && k != 1) || (k > 1 && ((k - 1) * C >= L || C % kStep)) || k * C < L) {
                std::printf("len %d: %d pieces of %ld\n", L, k, (long)C);
                return 1;
            }
            n += k;
            ++checked;
        }
        if (n > p.pieces) {
            std::printf("%ld pieces, the launch holds %ld (B %d, extra %ld, total %ld)\n", (long)n, (long)p.pieces, B, (long)p.extra, (long)total);
            return 1;
        }
    }
    std::printf("%ld requests\n", checked);
    return 0;
}
