// The cut of the attention over the paged K/V cache (kv_split.h) where requests differ much in length: whatever the host knows of
// them (their sum or only the table's room), no workgroup walks much more of one request than its share.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "../../paper_2501_01792_amd/csrc/kv_split.h"

using namespace hk::kvattn;

static int check(const std::vector<int> &len, int T, int H, int Hkv, int dh, bool codes, bool exact, int64_t room)
{
    const int64_t B = len.size();
    int64_t sum = 0, longest = 0;
    for (int L : len) {
        sum += L;
        longest = std::max<int64_t>(longest, L);
    }
    const Plan p = plan(B, T, H, Hkv, dh, codes, exact ? sum : B * room, room, 0);
    if (p.shared) return 0;
    const int64_t walked = std::min(longest, piece_tokens(sum, p.extra));
    const int64_t resident = kUnits * resident_pieces(dh, p.tiles, codes, T > 1);
    // 1 MB of K and V; four times a request's share, or a workgroup's; rounded up to whole rounds
    const int64_t least = (1 << 20) / (dh * (codes ? 2 : 4));
    const int64_t share = std::max(sum / B, sum * Hkv / resident);
    const int64_t most = std::max(least, 4 * share + kStep);
    if (walked > most) {
        std::printf("B %ld, %d K/V heads of %d, %s, T %d, longest %ld of %ld tokens, room %ld, sum %s: %ld tokens in a piece, at most %ld\n", (long)B, Hkv, dh,
                    codes ? "8 bits" : "16 bits", T, (long)longest, (long)sum, (long)room, exact ? "known" : "not known", (long)walked, (long)most);
        return 1;
    }
    int64_t n = 0;
    for (int L : len) n += pieces_of(L, piece_tokens(sum, p.extra));
    return n * Hkv > p.groups;
}

int main()
{
    struct One { int B, others, longest, H, Hkv; bool codes; };
    for (const One &o : {One{33, 128, 12288, 32, 32, false}, {128, 1000, 32768, 8, 8, true}, {32, 700, 16384, 32, 32, false}, {64, 40, 30000, 64, 8, true},
                         {256, 100, 100000, 8, 8, true}, {512, 500, 32768, 8, 8, true}, {8, 100, 8192, 40, 40, false}})
        for (bool exact : {true, false})
            for (int wide : {1, 4}) {
                std::vector<int> len(o.B, o.others);
                len[o.B / 3] = o.longest;
                if (check(len, 1, o.H, o.Hkv, 128, o.codes, exact, (int64_t)wide * o.longest)) return 1;
            }
    std::mt19937 rng(11);
    for (int trial = 0; trial < 20000; ++trial) {
        const int B = 1 + rng() % 512, Hkv = 1 + rng() % 72, T = 1 + rng() % 4, low = 1 + rng() % 2000, high = 1 << rng() % 18;
        std::vector<int> len(B);
        for (int &L : len) L = 1 + rng() % (rng() % 20 ? low : high);
        const int64_t room = *std::max_element(len.begin(), len.end()) * (rng() % 2 ? 1 : 1 + rng() % 8);
        if (check(len, T, Hkv, Hkv, rng() % 2 ? 64 : 128, rng() % 2, rng() % 2, room)) return 1;
    }
    return 0;
}
