// How the attention over the paged K/V cache is cut into workgroups: plain integer arithmetic, callable from host and device
// code, so that it can be checked on a CPU.
//
// Query rows: the T nodes of a request x the g = H / Hkv query heads of a K/V head, row = node * g + head, in tiles of 16 (the
// matrix instruction's columns).  Up to two tiles, every wavefront of a workgroup holds all rows and the tokens are shared out
// among them; more, and the wavefronts share the tokens and hold one or two tiles each (`shared`), in as many workgroups
// (`row_groups`) as that takes.
// Tokens: a request's tokens are cut into pieces of C, the same C for all, found on the device from the lengths: with S extra
// pieces to give away, C = sum(len) / S rounded up to a step of the workgroup makes at most B + S of them.  S = 0: one piece per
// request, whatever its length, and no merge.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define HK_HOST_DEVICE __host__ __device__
#else
#define HK_HOST_DEVICE
#endif

namespace hk {
namespace kvattn {

constexpr int kTileTokens = 32;                      // tokens a wavefront takes at once
constexpr int kWaves = 4;
constexpr int kStep = kTileTokens * kWaves;          // tokens of a workgroup's round
constexpr int kMaxTiles = 2;                         // tiles of 16 query rows in a wavefront
constexpr int kWantGroups = 1024;                    // workgroups that fill the chip: 256 compute units x 4
constexpr int64_t kMostGroups = (int64_t(1) << 23);  // a launch holds fewer than 2^32 threads

struct Plan {
    int64_t rows;            // T * g
    bool shared;             // the wavefronts of a workgroup share the tokens, not the rows
    int tiles, row_groups;   // tiles of a wavefront, workgroups that share a piece
    int64_t extra;           // S
    int64_t pieces;          // B + S: pieces of the launch (device: at most)
    int64_t groups;          // workgroups of the launch
    int64_t partial_floats;
};

inline Plan plan(int64_t B, int64_t T, int64_t H, int64_t Hkv, int head_dim, int64_t total_tokens, int splits)
{
    Plan p;
    p.rows = T * (H / Hkv);
    const int64_t all = (p.rows + 15) / 16;
    p.shared = all > kMaxTiles;
    const int64_t wide = p.shared ? kWaves : 1;          // wavefronts that hold different rows
    p.row_groups = (int)((all + wide * kMaxTiles - 1) / (wide * kMaxTiles));
    p.tiles = (int)((all + wide * p.row_groups - 1) / (wide * p.row_groups));
    const int64_t across = Hkv * p.row_groups;
    int64_t S = 0;
    if (splits > 0) {
        S = splits > 1 ? B * splits : 0;
    } else if (B * across < kWantGroups) {
        S = (kWantGroups + across - 1) / across - B;
        const int64_t most = total_tokens / kStep;           // a piece has a round at least
        S = S < most ? S : most;
    }
    p.extra = S;
    p.pieces = B + S;
    p.groups = (p.pieces * Hkv + 7) / 8 * 8 * p.row_groups;
    p.partial_floats = S > 0 ? p.pieces * Hkv * p.rows * (head_dim + 2) : 0;
    return p;
}

// Tokens of a piece, the lengths' sum being `total`.
HK_HOST_DEVICE inline int64_t piece_tokens(int64_t total, int64_t S)
{
    if (S <= 0) return int64_t(1) << 40;
    const int64_t C = (((uint64_t)total | (uint64_t)S) >> 32) == 0 ? (int64_t)(((uint32_t)total + (uint32_t)(S - 1)) / (uint32_t)S) : (total + S - 1) / S;
    return C < kStep ? kStep : (C + kStep - 1) / kStep * kStep;
}

// Pieces of a request; one without tokens has one, which writes its output.
HK_HOST_DEVICE inline int pieces_of(int len, int64_t C)
{
    if (C > 0x7fffffff || len <= 0) return 1;
    return (int)(((uint32_t)len + (uint32_t)(C - 1)) / (uint32_t)C);
}

}  // namespace kvattn
}  // namespace hk
