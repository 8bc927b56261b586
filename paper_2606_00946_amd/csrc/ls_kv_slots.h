// From the work slots of a KV-cache launch to rows: plain arithmetic, for the
// kernels and for the host.
//
// A launch deals its slots to the sequences in order, sequence b's starting at a
// number that its offset in the call's rows gives.  Where the first sequence's
// offset is not 0, the slots before its first are nobody's.
#pragma once

#include <cstdint>

namespace ls {

constexpr int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

// First slot of a sequence whose rows start at `off`, a slot being 2^shift positions
// that they touch: as many as that and more.
constexpr int64_t block_slot(int32_t off, int32_t b, int shift) { return (off >> shift) + 2 * (int64_t)b; }

// A block of 2^shift positions and the new rows [row0, row1) in it (none where row0 >= row1).
struct BlockRows {
    int64_t j;               // the block's place in the sequence
    int32_t row0, row1;
};

// The i-th of the blocks that n rows after `past` touch.
constexpr BlockRows block_rows(int64_t i, int32_t n, int64_t past, int shift) {
    const int64_t j = (past >> shift) + i, pos = j << shift, size = (int64_t)1 << shift;
    if (i < 0 || pos >= past + n) return {0, 0, 0};
    return {j, (int32_t)(pos < past ? past - pos : 0), (int32_t)least(past + n - pos, size)};
}

// First slot of a sequence whose rows start at `off`, a slot being `tile` of its rows
// times G heads.
constexpr int64_t tile_slot(int32_t off, int32_t b, int32_t G, int32_t tile) { return (int64_t)off * G / tile + b; }

// Rows [r0, r0 + rows) of a sequence's i-th tile, of n * G.
struct TileRows {
    int64_t r0;
    int32_t rows;
};
constexpr TileRows tile_rows(int64_t i, int32_t n, int32_t G, int32_t tile) {
    const int64_t r0 = i * tile, left = (int64_t)n * G - r0;
    if (i < 0 || left <= 0) return {0, 0};
    return {r0, (int32_t)least(left, tile)};
}

// A tree's parts, `pairs` of (head, piece) for each of `tiles` row tiles: eight pairs beside
// each other, then their next tile, so that the tiles that read the same codes run on one
// XCD (workgroups go round eight) at about one time.
struct TreePlace {
    uint32_t pair, tile;
};
constexpr TreePlace tree_place(uint32_t at, uint32_t pairs, uint32_t tiles) {
    const uint32_t even = pairs & ~7u;
    if (at < even * tiles) return {at / (8 * tiles) * 8 + (at & 7), at % (8 * tiles) >> 3};
    const uint32_t r = at - even * tiles, w = pairs - even;
    return {even + r % w, r / w};
}

// The first n of 16 bits.
constexpr uint32_t first_bits(int32_t n) { return n >= 16 ? 0xFFFFu : n <= 0 ? 0u : (1u << n) - 1; }

// Which of the 16 tokens of a block a drafted row sees.  The block starts `rel` tokens after the
// cached ones (before them: below 0); cached tokens i count unless i < gone and i >= sink, new ones by
// the mask, whose words rel >> 6 and the next are lo and hi, up to the n-th.
constexpr uint32_t tree_bits(int32_t rel, int32_t n, int32_t gone, int32_t sink, uint64_t lo, uint64_t hi) {
    const uint32_t cached = first_bits(rel > 0 ? 0 : -(rel < -16 ? -16 : rel)), s = (uint32_t)rel & 63;
    const uint64_t bits = lo >> s | (s ? hi << (64 - s) : 0);
    return (cached & (~first_bits(gone) | first_bits(sink))) | ((uint32_t)bits & first_bits(n - rel) & ~cached);
}

}  // namespace ls
