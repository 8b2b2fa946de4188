// How the attention over the paged K/V cache is cut into workgroups: plain integer arithmetic, callable from host and device
// code, so that it can be checked on a CPU.
//
// Query rows: the T nodes of a request x the g = H / Hkv query heads of a K/V head, row = node * g + head, in tiles of 16 (the
// matrix instruction's columns).
//
// Up to two tiles, every wavefront of a workgroup holds all rows and the tokens are shared out among them.  A request's tokens
// are cut into pieces of C, the same C for all, found on the device from the lengths: with S extra pieces to give away, C =
// sum(len) / S rounded up to a step of the workgroup makes at most B + S of them.  S = 0: one piece per request, whatever its
// length, and no merge.
//
// More tiles, and the wavefronts of a workgroup share the tokens and hold one or two tiles each (`shared`).  Such work is
// bound by arithmetic, so the compute units have to get equal shares of it, whatever the lengths and trees are: a unit is a row
// group (the rows of a workgroup) of a K/V head of a request, it takes its tokens' and its nodes' tiles of 32 one after the other,
// and the tiles of all units form a line that the workgroups, as many as are resident at once, cut into equal ranges.  A
// workgroup leaves at most two units unfinished, the first and the last of its range.
#pragma once
#include <stdint.h>

#include "attn_ranges.h"

namespace hk {
namespace kvattn {

constexpr int kTileTokens = 32;                      // tokens a wavefront takes at once
constexpr int kWaves = 4;
constexpr int kStep = kTileTokens * kWaves;          // tokens of a round of a workgroup whose wavefronts share them out
// Tiles of 16 query rows in a wavefront.  Three would need more registers than two workgroups a compute unit leave; at two the
// streaming form is as fast as the shared one or faster (8 requests of up to 1024 tokens x 32 heads, 24 rows, int8: 27 and 35 us;
// 16 requests of 2000, 32 rows on 8 K/V heads, 16 bits: 39 and 40).
constexpr int kMaxTiles = 2;
constexpr int kUnits = 256;                          // compute units
// Tiles of a range at least: fewer cost more in beginnings and partial results than they gain in workgroups, but for one or two
// short requests.  us with 4 / 2: 8 requests of 200 tokens, 80 rows on 8 K/V heads 19.9 / 27.1; 4 of 500, 128 rows 30.6 / 32.8; 2 of
// 1000, 128 rows 29.3 / 31.9; 40 heads of 33 rows, 300 tokens 15.4 / 17.2; one of 1000, 64 rows 21.9 / 20.8 (24.5 with 8); one of 300,
// 128 rows 25.9 / 21.7.  4 of 2000, 256 rows: 45.3 with 2, 4 or 8.
constexpr int kLeastRange = 4;
constexpr int64_t kMostGroups = (int64_t(1) << 23);  // a launch holds fewer than 2^32 threads

// Workgroups of a compute unit that the registers leave room for: the shared form, and the other one (`codes`: 8 bits, `tree`: nodes).
// (Three of the shared form's smaller one at dh = 128 spill: 33 rows of 40 heads 41 us for 38.)
HK_HOST_DEVICE constexpr int resident(int head_dim, int tiles) { return head_dim == 64 && tiles == 1 ? 3 : 2; }
HK_HOST_DEVICE constexpr int resident_pieces(int head_dim, int tiles, bool codes, bool tree)
{
    return tiles == 2 ? 2 : head_dim == 64 ? 4 : tree ? 2 : codes ? 4 : 3;
}

constexpr int64_t kWholeBytes = 1 << 20, kMostSearched = 512;

// Are requests left whole (one piece each, no merge, which is a launch of its own) where attn_splits leaves the choice?
// Not where one of them may be long among short ones: a workgroup per K/V head would walk it alone (us, whole / cut: one request of
// 12288 tokens among 32 of 128, 32 K/V heads, 16 bits 184 / 58; 32768 among 127 of 1000, 8 K/V heads, int8 278 / 74; 30000 among 63
// of 40 217 / 27; lengths from 64 to 8192, as many in each octave, 128 requests 146 / 114).  The host knows the table's width and the
// sum of the lengths, or a bound of it, so it is ruled out where
//   * the longest that there can be has 1 MB of K and V at most, or
//   * it has at most four times a request's share of the tokens, or, with more requests than that, a resident workgroup's share.
//     A sum that is no less than all the table has room for says nothing.
// What that costs where lengths are alike all the same (the table wide, the sum unknown or small): 128 requests of 250 to 500
// tokens on 8 K/V heads, int8 23 / 27; 25 x 12 heads, 12 nodes, 16 bits 11 / 17.  Beyond 512 requests every workgroup's search for
// its piece costs more than that: 1024 of 250 to 500 140 / 200, one of 32768 among them 368 / 241; so these are left alone.
// Where it is ruled out:
//   * Short requests are left whole, 512 tokens on average.  8 requests of 300 tokens and 8 K/V heads, int8: 6.9 us whole, 11.0
//     cut; 16 bits, 560 tokens 13.3 and 13.5, 1125 tokens 18.8 and 17.7; one request of 3000, int8: 24.9 and 11.0.
//   * Where they fill the chip, `want` workgroups.
//   * Where they give every compute unit one: what the cut gains in balance, its merge and its shorter pieces lose.  8 requests x
//     32 K/V heads, 560 / 1125 / 2250 / 6000 tokens on average (from half of the longest on), e4m3, one token: 12 / 20 / 33 / 82 us
//     whole, 17 / 25 / 36 / 87 cut; 24 nodes over int8: 21 / 32 / 50 / 103 and 25 / 45 / 65 / 129.  dh = 64 (25 requests x 12 heads, 12
//     nodes, 16 bits): 15 / 27 and 21 / 30, beyond that the cut is as fast or faster.
inline bool left_whole(int64_t B, int64_t Hkv, int head_dim, bool codes, int64_t total_tokens, int64_t room, int64_t want)
{
    const int64_t longest = room < total_tokens ? room : total_tokens, shares = B * Hkv < want ? B : (want + Hkv - 1) / Hkv;
    const bool small = longest * head_dim * (codes ? 2 : 4) <= kWholeBytes;
    const bool alike = total_tokens < room * B && room * shares <= 4 * total_tokens;
    if (!small && !alike && B <= kMostSearched) return false;
    if (total_tokens <= 512 * B || B * Hkv >= want) return true;
    return B * Hkv >= kUnits && total_tokens <= (head_dim == 64 ? 1536 : 8192) * B;
}

struct Plan {
    int64_t rows;            // T * g
    bool shared;             // the wavefronts of a workgroup share the tokens, not the rows
    int tiles;               // tiles of a wavefront
    int64_t extra;           // S
    int64_t groups;          // workgroups of the launch
    int64_t slots;           // rows of unfinished results
    int64_t partial_floats;  // slots of head_dim sums, then of (m, l), then what the merge has to know of a request or range
};

// room: the longest request that the table has room for.
inline Plan plan(int64_t B, int64_t T, int64_t H, int64_t Hkv, int head_dim, bool codes, int64_t total_tokens, int64_t room, int splits)
{
    Plan p;
    p.rows = T * (H / Hkv);
    const int64_t all = (p.rows + 15) / 16;
    p.shared = all > kMaxTiles;
    p.extra = 0;
    if (p.shared) {
        // two tiles a wavefront where one leaves rows for another workgroup: 16 requests of up to 8192 tokens, 512 rows 354 us
        // for 488, 16 of 2000, 256 rows 75 for 84 (small batches lose: 4 of 2000 45 for 43, one of 4000 47 for 44)
        p.tiles = all > kWaves ? 2 : 1;
        const int64_t held = 16 * kWaves * p.tiles;
        // tiles of the line at most: those of the tokens, a last one of each request that is not full, two of nodes
        const int64_t line = (total_tokens / kTileTokens + 3 * B) * Hkv * ((p.rows + held - 1) / held);
        const int64_t want = splits > 0 ? B * Hkv * splits : kUnits * resident(head_dim, p.tiles);
        const int64_t fit = (line + kLeastRange - 1) / kLeastRange;
        p.groups = want < fit ? want : fit > 0 ? fit : 1;
        p.slots = p.groups > 1 ? 2 * p.groups * held : 0;
    } else {
        p.tiles = (int)all;
        int64_t S = 0;
        const int64_t want = kUnits * resident_pieces(head_dim, p.tiles, codes, T > 1);
        if (splits > 0) {
            S = splits > 1 ? B * splits : 0;
        } else if (!left_whole(B, Hkv, head_dim, codes, total_tokens, room, want)) {
            S = (want + Hkv - 1) / Hkv - B;
            const int64_t few = (want / 2 + Hkv - 1) / Hkv;  // a piece has two resident workgroups' shares of the tokens at most
            S = S > few ? S : few;
            const int64_t most = total_tokens / kStep;       // a piece has a round at least
            S = S < most ? S : most;
        }
        p.extra = S;
        p.groups = (B + S) * Hkv;
        p.slots = S > 0 ? p.groups * p.rows : 0;
    }
    p.partial_floats = p.slots > 0 ? p.slots * (head_dim + 2) + (p.shared ? 4 * p.groups : 2 * B) : 0;
    return p;
}

// Tokens of a piece, the lengths' sum being `total`.
HK_HOST_DEVICE inline int64_t piece_tokens(int64_t total, int64_t S)
{
    if (S <= 0) return int64_t(1) << 40;
    const int64_t C = ranges::quot(total + S - 1, S);
    return C < kStep ? kStep : (C + kStep - 1) / kStep * kStep;
}

// The shared form's line.  Tiles of a unit of a request (a request without tokens and nodes' rows of its own has an empty one:
// its rows are written all the same), its row groups, and the ranges that take part when the line has `total` tiles.
HK_HOST_DEVICE inline int unit_tiles(int len, int nodes, bool tree)
{
    const int n = (len + kTileTokens - 1) / kTileTokens + (tree ? (nodes + kTileTokens - 1) / kTileTokens : 0);
    return n > 0 ? n : 1;
}
HK_HOST_DEVICE inline int unit_groups(int nodes, int g, int held) { return (nodes * g + held - 1) / held; }
HK_HOST_DEVICE inline int ranges_used(int64_t total, int groups)
{
    const int64_t fit = (total + kLeastRange - 1) / kLeastRange;
    return fit < groups ? (int)(fit > 0 ? fit : 1) : groups;
}

// Pieces of a request; one without tokens has one, which writes its output.
HK_HOST_DEVICE inline int pieces_of(int len, int64_t C)
{
    if (C > 0x7fffffff || len <= 0) return 1;
    return (int)(((uint32_t)len + (uint32_t)(C - 1)) / (uint32_t)C);
}

}  // namespace kvattn
}  // namespace hk
