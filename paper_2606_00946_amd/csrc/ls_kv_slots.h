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

// Attention of trees.  A sequence's heads lie one behind the other on a line, each with
// kTreeStart units for the start and the end and then its own; the line is cut into equal
// stretches, at the same places for all of the sequence's row tiles, and a workgroup has one
// stretch of one tile.  A head that several of them share falls into pieces; one of fewer than
// kTreeLeast units goes to the neighbour instead.  Measured, us (8 kv heads of 128 where nothing else is said):
// kTreeStart 3, 6, 9, 12: 32 sequences of 40 drafts x 4 over 2,000 tokens 91, 81, 82, 82; 24 of 96 x 2 of 64 dimensions
// 56, 51, 52, 53; 8 of 16 x 4 over 3,000 31, 32, 25, 29.  kTreeLeast 2, 4, 8: the second of these 56, 51, 56; 4 of 16 x 2
// of 256 dimensions over 8,000 43, 39, 43; one of 8 x 16, one kv head, over 60,000 31, 33, 38.  Others alike.
constexpr int32_t kTreeStart = 6, kTreeLeast = 4;

// The length of a line's stretches, `want` of them or fewer (now and then one more, where heads are
// shorter than a stretch may be): whole heads, or equal parts of each, where cuts anywhere would gain
// less than the start and the end that a cut head costs once more, and its join, 3/2 of a start in all; not so
// short that pieces vanish.  With 0, 3/2 and 3 starts: the 32 sequences above 92, 81 and 80 us, 32 of 16 to 64
// drafts over 64 to 8,192 tokens 96, 95 and 88, 2 of 64 over 60,000 153, 153 and 155.
constexpr int32_t tree_stretch(int32_t units, int32_t heads, int32_t want) {
    const int32_t head = units + kTreeStart, each = want < heads ? (heads + want - 1) / want : 1, of_head = want < heads ? 1 : want / heads;
    const int32_t even = each * ((head + of_head - 1) / of_head), any = (head * heads + want - 1) / want;
    const int32_t least = kTreeStart + 2 * kTreeLeast, best = even <= any + kTreeStart * 3 / 2 ? even : any;
    return best >= least || best == each * head ? best : head < least ? head : least;
}

// A head's unit at which a cut lies, x behind the head's place on the line.
constexpr int32_t tree_cut(int32_t x, int32_t units) {
    const int32_t u = x - kTreeStart;
    return u < kTreeLeast ? 0 : u > units - kTreeLeast ? units : u;
}

// The stretches (`per` long) with pieces of the head at `at`: first and last.
struct TreePieces {
    int32_t first, last;
};
constexpr TreePieces tree_pieces(int32_t at, int32_t units, int32_t per) {
    TreePieces p = {at / per, (at + kTreeStart + units - 1) / per};
    if (p.first < p.last && tree_cut((p.first + 1) * per - at, units) == 0) ++p.first;
    if (p.first < p.last && tree_cut(p.last * per - at, units) == units) --p.last;
    return p;
}

// Where the sums of a head's j-th piece lie: a stretch has at most one piece that starts
// inside a head, and at most one that is cut off at its end.
constexpr int32_t tree_slot(int32_t first, int32_t j) { return j == 0 ? 2 * first + 1 : 2 * (first + j); }

// Stretch and tile of a sequence's `at`-th workgroup: eight stretches beside each other, then
// their next tile, so that the tiles that read the same codes run on one XCD (workgroups go
// round eight) at about one time.
struct TreePlace {
    int32_t stretch, tile;
};
constexpr TreePlace tree_place(int32_t at, int32_t stretches, int32_t tiles) {
    const int32_t even = stretches & ~7;
    if (at < even * tiles) return {at / (8 * tiles) * 8 + (at & 7), at % (8 * tiles) >> 3};
    const int32_t r = at - even * tiles, w = stretches - even;
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
