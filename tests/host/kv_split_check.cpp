// Replays the cut of the attention over the paged K/V cache (kv_split.h) on the host, for batches of every kind of length and
// tree, also where the host's total is only a bound: pieces cover each request once, and there are no more of them than the
// launch and the scratch hold; ranges cover the line once, and no two parts of unfinished units share a slot.
#include <algorithm>
#include <cstdio>
#include <random>
#include <set>
#include <vector>

#include "../../paper_2501_01792_amd/csrc/kv_split.h"

using namespace hk::kvattn;
namespace ranges = hk::ranges;

int main()
{
    std::mt19937 rng(7);
    long requests = 0, parts = 0;
    for (int trial = 0; trial < 4000; ++trial) {
        const int B = 1 + rng() % 70, T = 1 + rng() % 64, g = 1 << rng() % 4, Hkv = 1 + rng() % 72;
        const int top = 1 << (1 + rng() % 17), dh = rng() % 2 ? 64 : 128;
        const bool tree = T > 1 || rng() % 2;
        std::vector<int> len(B), nodes(B);
        int64_t total = 0;
        for (int i = 0; i < B; ++i) {
            len[i] = rng() % 5 == 0 ? (int)(rng() % 3) : (int)(rng() % top);
            nodes[i] = tree ? (int)(rng() % (T + 1)) : 1;
            total += len[i];
        }
        const int64_t bound = total + (rng() % 2 ? 0 : rng() % 100000);
        const int splits = rng() % 3 ? 0 : (int)(rng() % 65);
        const int64_t room = *std::max_element(len.begin(), len.end()) + (rng() % 2 ? 0 : rng() % 100000);
        const Plan p = plan(B, T, (int64_t)Hkv * g, Hkv, dh, rng() % 2, bound, room, splits);
        const int held = p.tiles * 16 * (p.shared ? kWaves : 1);
        if (p.rows != T * g || p.tiles < 1 || p.tiles > kMaxTiles || (!p.shared && held < p.rows) || p.groups < 1) {
            std::printf("plan: rows %ld tiles %d groups %ld\n", (long)p.rows, p.tiles, (long)p.groups);
            return 1;
        }
        if (p.shared) {
            std::vector<int64_t> begin(B + 1, 0);
            for (int i = 0; i < B; ++i)
                begin[i + 1] = begin[i] + (int64_t)unit_tiles(len[i], nodes[i], tree) * unit_groups(nodes[i], g, held) * Hkv;
            const int64_t line = begin[B];
            const int used = ranges_used(line, (int)p.groups);
            if (used > p.groups || ranges::range_begin(0, line, used) != 0 || ranges::range_begin(used, line, used) != line) return 2;
            std::set<int64_t> slots;
            int64_t pos = 0;
            for (int w = 0; w < used && line > 0; ++w) {
                const int64_t end = ranges::range_begin(w + 1, line, used);
                if (pos != ranges::range_begin(w, line, used) || end <= pos) return 3;
                while (pos < end) {
                    const int r = (int)(std::upper_bound(begin.begin(), begin.end(), pos) - begin.begin()) - 1;
                    const int tiles = unit_tiles(len[r], nodes[r], tree);
                    const int64_t unit = (pos - begin[r]) / tiles, first = pos - begin[r] - unit * tiles;
                    const int64_t n = std::min<int64_t>(tiles - first, end - pos);
                    if (n != tiles) {
                        const int64_t slot = 2 * w + (first == 0);
                        if ((slot + 1) * held > p.slots || !slots.insert(slot).second) {
                            std::printf("slot %ld of %ld rows\n", (long)slot, (long)p.slots);
                            return 4;
                        }
                        // what the merge looks for: the parts of the unit are those of consecutive ranges, the first begins it
                        const int64_t u0 = begin[r] + unit * tiles;
                        const int w0 = ranges::owner(u0, line, used), w1 = ranges::owner(u0 + tiles - 1, line, used);
                        if (w < w0 || w > w1 || (w == w0) != (first == 0)) return 5;
                    }
                    pos += n;
                    ++parts;
                }
            }
            if (pos != line && line > 0) return 6;
            continue;
        }
        const int64_t C = piece_tokens(total, p.extra);
        int64_t n = 0;
        for (int L : len) {
            const int k = pieces_of(L, C);
            if (k < 1 || (p.extra <= 0 && k != 1) || (k > 1 && ((k - 1) * C >= L || C % kStep)) || k * C < L) {
                std::printf("len %d: %d pieces of %ld\n", L, k, (long)C);
                return 7;
            }
            n += k;
            ++requests;
        }
        if (n * Hkv > p.groups || (p.extra > 0 && n * Hkv * p.rows > p.slots)) {
            std::printf("%ld pieces, the launch holds %ld (B %d, extra %ld, total %ld)\n", (long)n, (long)(p.groups / Hkv), B, (long)p.extra, (long)total);
            return 8;
        }
    }
    std::printf("%ld requests in pieces, %ld parts of ranges\n", requests, parts);
    return 0;
}
