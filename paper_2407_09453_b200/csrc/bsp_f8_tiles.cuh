// How many tiles the products of 8-bit matrices are cut into.  Sizes go up to 2^31 - 1, so that a sum of one with a tile's side is one of 64 bits.
// Plain arithmetic: the host compiler takes it, too.
#pragma once
#include <cstdint>

namespace bsp {

constexpr int64_t kF8MostTiles = 0x7FFFFFFF;             // CTAs of a launch

// Tiles of `side` that cover n entries.
inline int64_t f8_cover(int64_t n, int64_t side) { return (n + side - 1) / side; }

// Tiles of 256 x 256 for pairs of CTAs, `pairs` of which are there at a time: tiles in a row, tiles that stay whole (the ones of the last wave
// are halved where two for each of them find pairs of their own), and all.  False: more than an int counts, a step of the pairs included.
struct F8PairTiles { int across, whole, all; };
inline bool f8_pair_tiles(int64_t M, int64_t N, int pairs, F8PairTiles &t)
{
    const int64_t across = f8_cover(N, 256), tiles = f8_cover(M, 256) * across;
    if (tiles > kF8MostTiles - 2 * (int64_t)pairs) return false;
    const int last = (int)(tiles % pairs);
    t.across = (int)across;
    t.whole = (int)tiles - (2 * last <= pairs ? last : 0);
    t.all = (int)(2 * tiles - t.whole);
    return true;
}

// Tiles of 128 x BN, each shared by `split` CTAs: tiles in a row, and CTAs.  False: more than a launch takes.
inline bool f8_tile_grid(int64_t M, int64_t N, int BN, int split, int &across, int64_t &ctas)
{
    across = (int)f8_cover(N, BN);
    ctas = f8_cover(M, 128) * across * split;
    return ctas <= kF8MostTiles;
}

}  // namespace bsp
