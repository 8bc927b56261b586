// What moves tokens and pages of the paged 8-bit KV cache (k_kv.h) between steps,
// in all layers at once: keeping drafts, forking sequences, compaction.  All three
// copy codes, so HBM bounds the large calls and the chain of dependent reads
// (lengths, table, codes) the small ones.
#include <algorithm>

#include "k_kv.h"
#include "ls_kv_calls.h"
#include "ls_scratch.h"

namespace ls {
namespace {

// ---- keeping drafts ---------------------------------------------------------------

// A sequence's kept tokens: the list ends before the first entry that is not above
// the one before it, or not one of the new tokens.  Kept token i comes from new
// token kept[i] >= i, so a page's tokens come from it or from later pages, and
// pages may be rewritten in their order.  `moves`: the first that is not in its place,
// and none after it is.
__device__ __forceinline__ int kept_count(const int32_t* kept, int want, int n, int& moves) {
    const int lane = threadIdx.x & 63;
    want = min(max(want, 0), n);
    moves = want;
    for (int i0 = 0; i0 < want; i0 += 64) {
        const int i = i0 + lane;
        const int32_t k = i < want ? kept[i] : n, before = i > 0 && i < want ? kept[i - 1] : -1;
        const uint64_t bad = __ballot(k <= before || k >= n), away = __ballot(k != i);
        if (away) moves = min(moves, i0 + __ffsll((long long)away) - 1);
        if (bad) return min(i0 + __ffsll((long long)bad) - 1, want);
    }
    return want;
}

// Where a token lies: its page, or -1, and its row there.
struct Spot {
    int32_t page, row;
};
__device__ __forceinline__ Spot spot_of(const KvView& c, int b, int64_t pos) {
    const int64_t j = pos >> c.page_shift;
    return {j < c.W ? (int32_t)page_id(c, b, (int)j) : -1, (int32_t)pos & (c.page - 1)};
}

// Largest magnitude of four codes.
template <bool FP8>
__device__ __forceinline__ float top_of(uint32_t w) {
    const float4v f = code_values<FP8>(w);
    return fmaxf(fmaxf(fabsf(f.x), fabsf(f.y)), fmaxf(fabsf(f.z), fabsf(f.w)));
}

// Codes brought to another scale, which covers them.  FP8: at most 448 (1 + 2^-22), which rounds to 448, so that
// nothing has to be clamped (54 us with, 48 without where int8 takes 41).
template <bool FP8>
__device__ __forceinline__ uint32_t regraded(uint32_t w, float again) {
    const float4v f = code_values<FP8>(w);
    if constexpr (!FP8) return codes_of<false>(f.x * again, f.y * again, f.z * again, f.w * again);
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f.x * again, f.y * again, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f.z * again, f.w * again, lo, true);
}

// The scale that a largest magnitude asks for; for int8 by one product with 1 / 127 as 32 bits
// hold it, within 2^-23 of the quotient (64 sequences, 32 layers: 41.4 us, with the quotient 41.9).
template <bool FP8>
__device__ __forceinline__ float kept_scale(float a) {
    return FP8 ? scale_of<true>(a) : fminf(fmaxf(a * (1.0f / 127.0f), kScaleMin), kScaleMax);
}

// A wave: one layer's keys or values of a sequence and head, kept tokens i0 to n.  Page by page, 16 tokens
// at a time: a lane holds, of every 64 dimensions, 16 of one key, or four of each of four
// values.  Once for the largest magnitude that moves in, once for the codes; a page of
// 16 tokens stays in registers between the two.
template <int D, bool FP8, bool VALUE>
__device__ __forceinline__ void keep_rows(const KvView& c, uint8_t* codes, float* scales, int b, int h, int64_t past,
                                          const int32_t* kept, int i0, int n) {
    constexpr int ND = D / 64, NT = VALUE ? 4 : 1;       // tokens of a lane
    const int lane = threadIdx.x & 63;
    const int first = VALUE ? (lane >> 4) * 4 : lane >> 2;      // the lane's first token of a block
    const int64_t head = (int64_t)c.page * D;
    for (int64_t j = (past + i0) >> c.page_shift; j << c.page_shift < past + n; ++j) {
        const int64_t pos0 = j << c.page_shift;
        const int r0 = (int)max(past + i0 - pos0, (int64_t)0), r1 = (int)min(past + n - pos0, (int64_t)c.page);
        const int64_t page = j < c.W ? page_id(c, b, (int)j) : -1;
        if (page < 0) continue;
        uint8_t* mine = codes + (page * c.H + h) * head;
        const float held = scales[page * c.H + h];
        uint4v x[NT][ND];
        float from[NT];                  // the tokens' scales
        uint32_t moves;                  // the lane's tokens that move, a byte each
        auto load = [&](int blk) {
            moves = 0;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int row = blk * 16 + first + t;
                Spot s = {(int32_t)page, row};
                if (row >= r0 && row < r1) {
                    const int i = (int)(pos0 + row - past);
                    const int32_t k = kept[i];
                    if (k != i) s = spot_of(c, b, past + k);
                }
                moves |= s.page >= 0 && (s.page != page || s.row != row) ? 255u << 8 * t : 0u;
                if (s.page < 0) s = {(int32_t)page, row};
                const int64_t at = (int64_t)s.page * c.H + h;
                from[t] = fminf(scales[at], kScaleMax);        // what a page's scale can cover
                const uint8_t* p = codes + at * head + (s.row >> 4) * 16 * D;
                const int byte = VALUE ? ((s.row & 15) >> 2) * 256 + (lane & 15) * 16 : (s.row & 15) * 64 + (lane & 3) * 16;
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    x[t][d] = *reinterpret_cast<const uint4v*>(p + d * 1024 + byte);
                    if constexpr (VALUE)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[t][d][e] = x[t][d][e] >> 8 * (s.row & 3) & 255u;
                }
            }
        };
        float top = 0.0f;
        uint64_t any = 0;
        const int b0 = r0 >> 4, b1 = (r1 + 15) >> 4;
        for (int blk = b0; blk < b1; ++blk) {
            load(blk);
            any |= __ballot(moves != 0);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float m = 0.0f;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) m = fmaxf(m, top_of<FP8>(x[t][d][e]));
                top = fmaxf(top, moves >> 8 * t & 1 ? m * from[t] : 0.0f);
            }
        }
        if (!any) continue;
        const float scale = fmaxf(kept_scale<FP8>(wave_max(top)), held), inv = 1.0f / scale;
        // what a code of token t is to be multiplied by; finite, since a token of zeros asks for no scale: from the largest
        // onto the smallest it would be infinite
        auto again = [&](int t) { return fminf(from[t] * inv, 0x1p+64f); };
        int loaded = b1 - 1;
        for (int blk = scale > held ? 0 : b0; blk < b1; ++blk) {
            if (blk != loaded) load(blk);
            loaded = blk;
            uint8_t* p = mine + blk * 16 * D;
            // the block's tokens may come from later rows of it: all have been read before any lane writes
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if constexpr (!VALUE) {
                if (blk * 16 + first < r1 && (moves != 0 || scale > held)) {
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        uint4v o;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = regraded<FP8>(x[0][d][e], again(0));
                        *reinterpret_cast<uint4v*>(p + d * 1024 + first * 64 + (lane & 3) * 16) = o;
                    }
                }
            } else {
                // of the lane's four tokens those that move are written, or all up to r1 where the scale grew: the others are
                // nobody's, or stay what they are, int8 -128 and NaN too
                const int live = r1 - (blk * 16 + first);
                const uint32_t m = !(scale > held) ? moves : live >= 4 ? ~0u : live > 0 ? (1u << 8 * live) - 1 : 0u;
                if (m) {
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        uint4v* at = reinterpret_cast<uint4v*>(p + d * 1024) + lane;
                        const uint4v old = m != ~0u ? *at : uint4v{0, 0, 0, 0};
                        uint4v o;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t w = 0;
#pragma unroll
                            for (int t = 0; t < 4; ++t)
                                w |= (regraded<FP8>(x[t][d][e], again(t)) & 255u) << 8 * t;
                            o[e] = (w & m) | (old[e] & ~m);
                        }
                        *at = o;
                    }
                }
            }
        }
        if (lane == 0 && scale > held) scales[page * c.H + h] = scale;
    }
}

// Waves: (layer, sequence, head, key or value).  Measured: 64 sequences of 16 to 64 drafts, up to 9
// of them kept, 32 layers of 8 heads of 128 (int8): 48 us, where its bytes would take 4.  Vector
// instructions take 64 % of the cycles (550 a wave, most of them for the 16 tokens of a block whichever
// of them move), the chain list, table, codes the rest.  Waves that keep 2, 4 or 8 heads
// in turn read lists and tables less often and decode only what moves, but wait for one head's codes
// after the other: 56, 59 and 61 us beside 52.  One sequence of 8 drafts: 7.5 us.  int8 has room for six
// waves a SIMD (the same lists over and over: 41 us, with five 44); FP8 would spill.
template <int D, bool FP8>
__global__ __launch_bounds__(256, FP8 || D == 256 ? 1 : 6) void kv_keep_kernel(KvView c, KvLayers l,
                                                                               const int32_t* __restrict__ kept,
                                                                               const int32_t* __restrict__ n_kept,
                                                                               uint32_t n_items) {
    const uint32_t w = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (w >= n_items) return;
    const int value = w & 1, h = (int)((w >> 1) % (uint32_t)c.H);
    const uint32_t rest = (w >> 1) / (uint32_t)c.H;
    const int b = (int)(rest % (uint32_t)c.B), layer = (int)(rest / (uint32_t)c.B);
    int t0, n;
    seq_rows(c, b, t0, n);
    const int64_t past = min(max(c.past[b], 0), 1 << 30);
    int i0;
    n = kept_count(kept + t0, n_kept[b], n, i0);
    if (i0 >= n) return;
    if (value)
        keep_rows<D, FP8, true>(c, l.codes[1][layer], l.scales[1][layer], b, h, past, kept + t0, i0, n);
    else
        keep_rows<D, FP8, false>(c, l.codes[0][layer], l.scales[0][layer], b, h, past, kept + t0, i0, n);
}

// ---- forking ----------------------------------------------------------------------

// The first workgroups write the tables, 256 entries of a fork each; a wave of the
// others copies, for a fork and layer, one head's keys or values of the last page.
// Measured: 96 beams, 16 layers of 4 heads of 128, pages of 64: 25.5 us, 5.3 TB/s; 8 samples in
// 32 layers, 14.7 MB: 8.9 us, 5 of them the kernel's (lengths, table, codes one after the other).
__global__ __launch_bounds__(256) void kv_fork_kernel(KvView c, KvLayers l, KvForks f, uint32_t table_groups,
                                                      uint32_t n_items) {
    auto known = [&](int i, int& s, int& d, int& n) {
        s = f.src[i];
        d = f.dst[i];
        n = (int)min((int64_t)max(f.tokens[i], 0), (int64_t)f.W << c.page_shift);
        return s >= 0 && s < f.rows && d >= 0 && d < f.rows;
    };
    int s, d, n;
    if (blockIdx.x < table_groups) {
        const int chunks = (f.W + 255) / 256;
        const int i = (int)(blockIdx.x / (uint32_t)chunks), j = (int)(blockIdx.x % (uint32_t)chunks) * 256 + threadIdx.x;
        if (known(i, s, d, n) && j < n >> c.page_shift) f.pages_out[(int64_t)d * f.W + j] = f.pages[(int64_t)s * f.W + j];
        return;
    }
    const uint32_t w = __builtin_amdgcn_readfirstlane((blockIdx.x - table_groups) * 4 + (threadIdx.x >> 6));
    if (w >= n_items) return;
    const int lane = threadIdx.x & 63, value = w & 1, h = (int)((w >> 1) % (uint32_t)c.H);
    const uint32_t rest = (w >> 1) / (uint32_t)c.H;
    const int layer = (int)(rest % (uint32_t)l.n), i = (int)(rest / (uint32_t)l.n);
    if (!known(i, s, d, n)) return;
    const int part = n & (c.page - 1), j = n >> c.page_shift;
    if (part == 0) return;
    const int32_t from = f.pages[(int64_t)s * f.W + j], to = f.pages_out[(int64_t)d * f.W + j];
    if (from < 0 || from >= c.n_pages || to < 0 || to >= c.n_pages || from == to) return;
    const int64_t head = (int64_t)c.page * c.D, a = (int64_t)from * c.H + h, z = (int64_t)to * c.H + h;
    const uint4v* src = reinterpret_cast<const uint4v*>(l.codes[value][layer] + a * head);
    uint4v* dst = reinterpret_cast<uint4v*>(l.codes[value][layer] + z * head);
    const int pieces = ((part + 15) >> 4) * c.D;             // of 16 bytes
    constexpr int kAtOnce = 8;
    for (int p0 = lane; p0 < pieces; p0 += 64 * kAtOnce) {
        uint4v x[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (p0 + k * 64 < pieces) x[k] = src[p0 + k * 64];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (p0 + k * 64 < pieces) dst[p0 + k * 64] = x[k];
    }
    if (lane == 0) l.scales[value][layer][z] = l.scales[value][layer][a];
}

// ---- compaction ---------------------------------------------------------------------
// U pages are in use.  The k-th of those from U on goes to the k-th id below U that is
// not: as few moves as there can be, no page is read that another is written over, and
// the same answer every time.  where[] says first which pages are in use, then which
// move it is (-2 - k), then the page's new id.

constexpr int kChunk = 4096;         // pages of a workgroup

__global__ __launch_bounds__(256) void compact_clear_kernel(int32_t* where, int32_t n) {
    const int64_t i = (int64_t)blockIdx.x * 1024 + threadIdx.x;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k * 256 < n) where[i + k * 256] = -1;
}

__global__ __launch_bounds__(256) void compact_mark_kernel(KvCompact m) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m.entries; i += (int64_t)gridDim.x * 256) {
        const int32_t p = m.pages[i];
        if (p >= 0 && p < m.n_pages) m.where[p] = 0;
    }
}

// Sum over a workgroup of 256 threads, for all of them.
__device__ __forceinline__ int32_t group_sum(int32_t x, int32_t (&lds)[4]) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

// Pages in use of [chunk * kChunk + from, + to).
__device__ __forceinline__ int32_t in_use(const KvCompact& m, int64_t lo, int64_t hi) {
    int32_t x = 0;
    for (int64_t i = lo + threadIdx.x; i < hi; i += 256) x += m.where[i] != -1;
    return x;
}

__global__ __launch_bounds__(256) void compact_count_kernel(KvCompact m) {
    __shared__ int32_t lds[4];
    const int64_t lo = (int64_t)blockIdx.x * kChunk, hi = min(lo + kChunk, (int64_t)m.n_pages);
    const int32_t x = group_sum(in_use(m, lo, hi), lds);
    if (threadIdx.x == 0) m.counts[blockIdx.x] = x;
}

// A chunk's pages: their places among those in use, from the chunks' counts.
__global__ __launch_bounds__(256) void compact_emit_kernel(KvCompact m, int32_t chunks) {
    __shared__ int32_t lds[4], wave_base[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, chunk = blockIdx.x;
    int32_t before = 0, all = 0;
    for (int i = threadIdx.x; i < chunks; i += 256) {
        const int32_t x = m.counts[i];
        all += x;
        before += i < chunk ? x : 0;
    }
    before = group_sum(before, lds);
    const int32_t used = group_sum(all, lds);
    // places below `used` that are in use: whole chunks, and the part of the one it lies in.  That one is read while its own
    // workgroup rewrites it: in use is whatever is not -1, before and after
    const int32_t last = used / kChunk;
    int32_t below = 0;
    for (int i = threadIdx.x; i < last; i += 256) below += m.counts[i];
    below = group_sum(below + in_use(m, (int64_t)last * kChunk, used), lds);
    if (chunk == 0 && threadIdx.x == 0) {
        *m.n_used = used;
        m.counts[chunks] = used - below;             // moves
    }
    // a wave's quarter of the chunk, 64 pages at a time
    const int64_t lo = (int64_t)chunk * kChunk + wave * (kChunk / 4);
    int32_t mine = 0;
#pragma unroll 4
    for (int k = 0; k < kChunk / 256; ++k) {
        const int64_t i = lo + k * 64 + lane;
        mine += __popcll(__ballot(i < m.n_pages && m.where[i] != -1));
    }
    if (lane == 0) wave_base[wave] = mine;
    __syncthreads();
    int32_t rank = before;
    for (int w = 0; w < wave; ++w) rank += wave_base[w];
    for (int k = 0; k < kChunk / 256; ++k) {
        const int64_t i = lo + k * 64 + lane;
        const bool is = i < m.n_pages && m.where[i] != -1;
        const uint64_t mask = __ballot(is);
        const int32_t r = rank + __popcll(mask & ((1ull << lane) - 1));
        rank += __popcll(mask);
        if (i >= m.n_pages) continue;
        if (i < used) {
            if (is) m.where[i] = (int32_t)i; else m.to[i - r] = (int32_t)i;
        } else if (is) {
            m.where[i] = -2 - (r - below);
            m.from[r - below] = (int32_t)i;
        }
    }
}

// The whole plan of a small pool in one workgroup: the pages in use as bits in LDS, and how many
// there are before each 32.  A call whose pages all stay, with as many entries or twice as many as
// pages (one workgroup / the four launches): 10.3 / 18.6 us at 256 pages, 10.6 / 22.7 at 4,096,
// 11.3 / 23.6 at 16,384, 15.7 / 23.0 at 32,768, 20.3 to 25.3 / 24.2 to 24.7 at 65,536, so up to there.
constexpr int kOnePages = 1 << 16, kOneEntries = 1 << 17, kOneThreads = 1024;
__global__ __launch_bounds__(kOneThreads) void compact_plan_kernel(KvCompact m, int32_t* n_moves) {
    __shared__ uint32_t bits[kOnePages / 32];
    __shared__ int32_t before[kOnePages / 32], sums[kOneThreads / 64], below_sums[kOneThreads / 64];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, words = (m.n_pages + 31) / 32;
    for (int i = t; i < words; i += kOneThreads) bits[i] = 0;
    __syncthreads();
    constexpr int kAtOnce = 8;
    for (int i0 = t; i0 < m.entries; i0 += kOneThreads * kAtOnce) {
        int32_t p[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) p[k] = i0 + k * kOneThreads < m.entries ? m.pages[i0 + k * kOneThreads] : -1;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (p[k] >= 0 && p[k] < m.n_pages) atomicOr(&bits[p[k] >> 5], 1u << (p[k] & 31));
    }
    __syncthreads();
    // a thread's run of words, then the threads before it
    const int run = (words + kOneThreads - 1) / kOneThreads, w0 = min(t * run, words), w1 = min(w0 + run, words);
    int32_t mine = 0;
    for (int i = w0; i < w1; ++i) mine += __popc(bits[i]);
    const int32_t upto = (int32_t)wave_scan((uint32_t)mine);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int32_t rank = upto - mine, used = 0;
    for (int w = 0; w < kOneThreads / 64; ++w) {
        rank += w < wave ? sums[w] : 0;
        used += sums[w];
    }
    int32_t low = 0;                         // pages in use below `used`
    for (int i = w0; i < w1; ++i) {
        before[i] = rank;
        rank += __popc(bits[i]);
        const int left = used - i * 32;
        low += __popc(left >= 32 ? bits[i] : left > 0 ? bits[i] & ((1u << left) - 1) : 0u);
    }
    const int32_t low_upto = (int32_t)wave_scan((uint32_t)low);
    if (lane == 63) below_sums[wave] = low_upto;
    __syncthreads();
    int32_t below = 0;
    for (int w = 0; w < kOneThreads / 64; ++w) below += below_sums[w];
    if (t == 0) {
        *m.n_used = used;
        *n_moves = used - below;
    }
    for (int32_t i = t; i < m.n_pages; i += kOneThreads) {
        const uint32_t word = bits[i >> 5], bit = 1u << (i & 31);
        const bool is = word & bit;
        const int32_t r = before[i >> 5] + __popc(word & (bit - 1));
        m.where[i] = !is ? -1 : i < used ? i : -2 - (r - below);
        if (i < used && !is) m.to[i - r] = i;
        if (i >= used && is) m.from[r - below] = i;
    }
}

// The first workgroups write the table and the moved pages' new ids, the others take
// moves in turn, a workgroup 16 KB of a page's keys or values in one layer at a time.
// Measured: 3,900 moves of pages of 16 in 4 layers of 8 heads of 128, 1.03 GB: 217 us, 4.75 TB/s.
__global__ __launch_bounds__(256) void compact_move_kernel(KvView c, KvLayers l, KvCompact m, uint32_t table_groups,
                                                           const int32_t* n_moves) {
    if (blockIdx.x < table_groups) {
        const int64_t step = (int64_t)table_groups * 256;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m.entries; i += step) {
            int32_t p = m.pages[i];
            if (p >= 0 && p < m.n_pages) {
                // a moved page's entry may be the move or, already, where it goes
                const int32_t w = __hip_atomic_load(&m.where[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                p = w <= -2 ? m.to[-2 - w] : w;
            }
            m.pages_out[i] = p;
        }
        const int32_t moves = *n_moves;
        for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < moves; k += step)
            __hip_atomic_store(&m.where[m.from[k]], m.to[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return;
    }
    const int64_t page = (int64_t)c.H * c.page * c.D / 16;       // pieces of 16 bytes
    constexpr int kAtOnce = 4, kPiece = 256 * kAtOnce;
    const int64_t per_page = (page + kPiece - 1) / kPiece;
    const int64_t items = (int64_t)*n_moves * l.n * 2 * per_page;
    for (int64_t w = blockIdx.x - table_groups; w < items; w += gridDim.x - table_groups) {
        const int64_t piece = w % per_page, rest = w / per_page;
        const int value = (int)(rest & 1), layer = (int)((rest >> 1) % l.n);
        const int64_t k = (rest >> 1) / l.n;
        const int64_t a = m.from[k], z = m.to[k];
        const uint4v* src = reinterpret_cast<const uint4v*>(l.codes[value][layer]) + a * page;
        uint4v* dst = reinterpret_cast<uint4v*>(l.codes[value][layer]) + z * page;
        uint4v x[kAtOnce];
        const int64_t p0 = piece * kPiece + threadIdx.x;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (p0 + i * 256 < page) x[i] = src[p0 + i * 256];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (p0 + i * 256 < page) dst[p0 + i * 256] = x[i];
        if (piece == 0)
            for (int h = threadIdx.x; h < c.H; h += 256)
                l.scales[value][layer][z * c.H + h] = l.scales[value][layer][a * c.H + h];
    }
}

int32_t chunks_of(int64_t n_pages) { return (int32_t)((n_pages + kChunk - 1) / kChunk); }

}  // namespace

hipError_t launch_kv_keep(const KvView& c, const KvLayers& l, const int32_t* kept, const int32_t* n_kept, hipStream_t s) {
    const int64_t items = (int64_t)l.n * c.B * c.H * 2, groups = (items + 3) / 4;
    if (groups >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    auto run = [&](auto d, auto fp8) {
        kv_keep_kernel<decltype(d)::value, decltype(fp8)::value>
            <<<(uint32_t)groups, 256, 0, s>>>(c, l, kept, n_kept, (uint32_t)items);
        return hipGetLastError();
    };
    auto by_dim = [&](auto fp8) {
        if (c.D == 64) return run(std::integral_constant<int, 64>{}, fp8);
        if (c.D == 128) return run(std::integral_constant<int, 128>{}, fp8);
        return run(std::integral_constant<int, 256>{}, fp8);
    };
    return c.fp8 ? by_dim(std::true_type{}) : by_dim(std::false_type{});
}

hipError_t launch_kv_fork(const KvView& c, const KvLayers& l, const KvForks& f, bool tables, hipStream_t s) {
    const int64_t table_groups = tables ? (int64_t)f.n * ((f.W + 255) / 256) : 0;
    const int64_t items = (int64_t)f.n * l.n * c.H * 2, groups = table_groups + (items + 3) / 4;
    if (groups >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    kv_fork_kernel<<<(uint32_t)groups, 256, 0, s>>>(c, l, f, (uint32_t)table_groups, (uint32_t)items);
    return hipGetLastError();
}

int64_t kv_compact_bytes(int64_t n_pages) { return 4 * ((int64_t)chunks_of(n_pages) + 1 + (n_pages / 2 + 1) * 2) + 3 * 256; }

// No more pages move than there are in use, nor than there are ids below.
void kv_compact_carve(KvCompact& k, void* workspace) {
    WsCarve ws{(char*)workspace, (size_t)kv_compact_bytes(k.n_pages)};
    k.counts = ws.take<int32_t>(chunks_of(k.n_pages) + 1);
    k.from = ws.take<int32_t>(k.n_pages / 2 + 1);
    k.to = ws.take<int32_t>(k.n_pages / 2 + 1);
}

hipError_t launch_kv_compact_plan(const KvCompact& k, int n_cu, hipStream_t s) {
    const int32_t chunks = chunks_of(k.n_pages);
    if (k.n_pages <= kOnePages && k.entries <= kOneEntries) {
        compact_plan_kernel<<<1, kOneThreads, 0, s>>>(k, k.counts + chunks);
        return hipGetLastError();
    }
    const int64_t marks = std::min<int64_t>((k.entries + 255) / 256, (int64_t)n_cu * 8);
    compact_clear_kernel<<<(uint32_t)(((int64_t)k.n_pages + 1023) / 1024), 256, 0, s>>>(k.where, k.n_pages);
    if (marks > 0) compact_mark_kernel<<<(uint32_t)marks, 256, 0, s>>>(k);
    compact_count_kernel<<<(uint32_t)chunks, 256, 0, s>>>(k);
    compact_emit_kernel<<<(uint32_t)chunks, 256, 0, s>>>(k, chunks);
    return hipGetLastError();
}

hipError_t launch_kv_compact_move(const KvView& c, const KvLayers& l, const KvCompact& k, bool tables, int n_cu,
                                  hipStream_t s) {
    const int64_t work = std::max<int64_t>(k.entries, k.n_pages / 2);
    const uint32_t table_groups = tables ? (uint32_t)std::min<int64_t>((work + 255) / 256, n_cu) : 0;
    compact_move_kernel<<<table_groups + (uint32_t)n_cu * 8, 256, 0, s>>>(c, l, k, table_groups, k.counts + chunks_of(k.n_pages));
    return hipGetLastError();
}

}  // namespace ls
