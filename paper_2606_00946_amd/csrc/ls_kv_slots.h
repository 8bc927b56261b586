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

}  // namespace ls
