// Launches of the KV cache's calls for drafts and pages: positions given row by
// row, attention for trees, keeping drafts, forking and compaction.
#pragma once

#include "ls_internal.h"

namespace ls {

// Rows' positions on several axes; pair i of the rotary dimensions turns by axis
// (axis[i / 16] >> 2 (i % 16)) & 3.
struct KvPositions {
    const int32_t* pos;             // [n_axes x T]
    int32_t n_axes;                 // 0: none, a row's position is its place in the sequence
    bool mixed;                     // eight pairs from a multiple of eight on lie on several axes
    uint32_t axis[8];
};
hipError_t launch_kv_append_at(const KvView& c, const KvRope& r, const KvPositions& at, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, const void* q, int64_t q_stride, int32_t Hq, void* q_out,
                               int64_t q_out_stride, int n_cu, hipStream_t s);

// Which new tokens a row sees, and where it stands.
struct KvTree {
    const uint64_t* mask;           // [T x words]
    int32_t words;
    const int32_t* pos;             // [T]
};
hipError_t launch_kv_tree(const KvView& c, const KvTree& t, const void* q, int64_t q_stride, int32_t Hq, float scale,
                          int32_t window, int32_t sinks, void* out, int64_t out_stride, void* workspace,
                          int64_t workspace_bytes, int n_cu, hipStream_t s);

// The KV workspace starts with the counts of attention's parts, which are zero between launches.
constexpr int64_t kKvCountBytes = 65536;

// Up to kMaxLayers layers' caches of one shape in a launch.
constexpr int kMaxLayers = 64;
struct KvLayers {
    uint8_t* codes[2][kMaxLayers];  // keys, values
    float* scales[2][kMaxLayers];
    int32_t n;
};
hipError_t launch_kv_keep(const KvView& c, const KvLayers& l, const int32_t* kept, const int32_t* n_kept, hipStream_t s);

// Rows of a page table that take over other rows' first tokens.
struct KvForks {
    const int32_t* pages;
    int32_t* pages_out;
    int32_t rows, W, n;
    const int32_t *src, *dst, *tokens;
};
hipError_t launch_kv_fork(const KvView& c, const KvLayers& l, const KvForks& f, bool tables, hipStream_t s);

// Compaction: `plan` finds the moves of a table's pages, `move` carries them out
// in some layers and, with `tables`, writes the new table.
struct KvCompact {
    const int32_t* pages;
    int32_t* pages_out;
    int64_t entries;
    int32_t *where, *n_used;
    int32_t n_pages;
    int32_t *counts, *from, *to;    // of each chunk of pages, and of the whole; moves
};
int64_t kv_compact_bytes(int64_t n_pages);
void kv_compact_carve(KvCompact& k, void* workspace);
hipError_t launch_kv_compact_plan(const KvCompact& k, int n_cu, hipStream_t s);
hipError_t launch_kv_compact_move(const KvView& c, const KvLayers& l, const KvCompact& k, bool tables, int n_cu,
                                  hipStream_t s);

}  // namespace ls
