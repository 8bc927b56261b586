// Attention of drafted tokens over the paged 8-bit KV cache (k_kv.h): a tree behind
// each sequence's cached tokens.
//
// out_i = sum_j softmax_j(scale q_i . k_j) v_j over the cached tokens that row i's
// position sees and the new tokens whose bit its mask has, with the weights and
// their reference as in k_kv_attend.hip.
//
// A tree's rows (new tokens x query heads of one kv head) are more than a decode step's
// and fewer than a prompt's, over as many cached tokens: at 4 D operations and 2 D
// bytes a token, reading (5.1 TB/s) and computing (1,170 TFLOP/s) take the same time at
// about 115 rows.
// So the tokens are what is dealt out: a wave takes 32 of a unit's 128 tokens with all
// of a tile's 32 or 64 rows, codes go from memory to registers in 16-byte loads and
// each operand made of them serves all rows; only the queries are in LDS.
//
// Measured, 8 kv heads: 32 sequences of 16 to 64 drafts x 4 heads of 128 over 64 to 8,192 tokens
// (fp8) 101 us, 382 TFLOP/s; 2 of 64 x 8 over 64k to 128k tokens (int8) 455 us, 798 TFLOP/s; 24 of
// 33 to 160 x 2 heads of 64 under a window of 2,048 (int8) 80 us; one of 8 drafts over 300
// tokens 11.8 us.  In the long one the matrix pipes are busy for 40 % of the cycles and the vector
// instructions (the exponential, its argument and sum, conversions of codes and weights) take 56 %: a wave
// alternates between the two, and two waves a SIMD, which is what the registers allow, seldom
// have one in each.  Raising a wave's priority for its products did not change that.  256 dimensions:
// 16 of 32 x 4 heads over 2,000 tokens 52 us, 2 of 64 x 8 over 30,000 268, the matrix pipes busy for 35 and 49 %.
// Registers that do not fit (64 rows of 128 dimensions, and 256 dimensions) are read back between
// pieces and in steps that a mask cuts, not in the others.
#include <algorithm>

#include "k_kv_attend.h"
#include "ls_kv_calls.h"
#include "ls_scratch.h"

namespace ls {
namespace {

using float16v = float __attribute__((ext_vector_type(16)));

// What lies before a chunk of 64 sequences: workgroups, and those of cut lines.
struct TreeChunk {
    int64_t groups, cut;
};

struct TreeArgs : AttnCall {
    int32_t fit;                     // workgroups that fit the device
    int32_t words;
    // stretches of lines that are cut: two slots each for pieces' sums, and four counts (TreeWork::join)
    float* part_o;                   // [2 fit][ROWS][D]
    float2v* part_ml;                // [2 fit][ROWS] a row's reference and sum
    uint32_t* arrived;               // [fit][4], zero between launches
    // of many sequences, by kv_tree_plan_kernel: what a workgroup has of a line, and what lies before each chunk
    float* each;
    TreeChunk* chunk;                // [chunks + 1]
    const uint64_t* mask;
    const int32_t* pos;
    int64_t groups;                  // no more have work
};

static_assert(kMaxParts * 2 * 4 == kKvCountBytes, "the counts' part of the workspace");

// log2 of a row's largest weight when the reference moves up: all 16 tokens of a lane's step
// may have it within kMostWeight, and later ones four times that.
constexpr float kTreeTop = 10.0f;

// A sequence of the call; units of one kv head and row tile, and row tiles.
struct TreeSeq {
    int32_t t0, n, past, units, tiles;
};
template <int ROWS>
__device__ __forceinline__ TreeSeq tree_seq(const KvView& c, const TreeArgs& a, int b) {
    TreeSeq s;
    seq_rows(c, b, s.t0, s.n);
    s.past = past_of(c, b);
    s.tiles = (s.n * a.G + ROWS - 1) / ROWS;             // rows of a call are below 2^30
    s.units = s.n == 0 ? 0 : max((span_of(c, a, s.past, s.n).n + kUnit - 1) / kUnit, 1);
    return s;
}

// Which tokens of the 16 from `tok` on a row at position `pos` sees: cached ones by the
// window, new ones by the mask's bits.
__device__ __forceinline__ uint32_t tree_sight(const TreeArgs& a, const uint64_t* mask, int32_t past, int32_t n, int32_t pos,
                                               int32_t tok) {
    const int32_t rel = tok - past, w = rel >> 6;
    const bool drafts = rel > -16;
    const uint64_t lo = drafts && w >= 0 && w < a.words ? mask[w] : 0, hi = drafts && w + 1 < a.words ? mask[w + 1] : 0;
    const int32_t gone = a.window > 0 ? max(pos - a.window, -1) + 1 - tok : 0;
    return tree_bits(rel, n, gone, a.sinks - tok, lo, hi);
}

// A value as of this place: what is made of it is not computed ahead, to be kept in registers
// (or in memory, which costs microseconds) through all that comes before.
__device__ __forceinline__ int here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// Four bits as bytes.
__device__ __forceinline__ uint32_t bytes_of(uint32_t four) { return ((four & 15u) * 0x00204081u & 0x01010101u) * 0xFFu; }

// The dimension of a row's accumulator o[c][i] in a lane of half `hi`, less c (D = 64: less
// c): of dimension block i / 8 (64 wide, plus 128 for every four c), or of the whole 64.
template <int D>
__device__ __forceinline__ constexpr int dim_of(int i, int hi) {
    const int m = 8 * (i >> 2) + 4 * hi + (i & 3);       // the product's row
    return D == 64 ? 4 * (m & 15) + 2 * (m >> 4) : 4 * (m & 15);
}

template <int D, int NR>
struct TreeLds {
    static constexpr int ROWS = 32 * NR;
    union {
        uint4v q[D / 16][NR][64];            // queries: [16 dimensions][32 rows][lane]
        float comb[4][ROWS][64 + 4];         // 64 dimensions of the waves' sums
    };
    float2v ml[4][ROWS];
    float undo[ROWS];                        // what undoes a row's scaling
};

// A lane's value for the whole wave.
__device__ __forceinline__ int64_t of_lane64(int64_t x, int l) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, l));
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// A workgroup's stretch of a sequence's line (tree_cut) for one row tile: a wave's copy in LDS, since there are no
// registers to spare between its pieces.
struct TreeStretch {
    int32_t b, t0, n, past, units, r0;
    int32_t stretch, first_group;        // the stretch, and the first workgroup of this tile among those of cut lines
    int32_t h;                           // the head that is next
    int32_t per, hi;                     // stretches' length; the stretch's end
};

// Tries, from a share of 0.3 of a stretch more for each tile to a whole one.  Straight to the whole one: 32 sequences
// of 16 to 64 drafts over 64 to 8,192 tokens 101 us instead of 95, 2 of 64 over 60,000 162 instead of 153.
constexpr int kTries = 6;

// What a workgroup has of a line in a try, when lines are `all` long in all, each times its tiles; whether it is the
// last one, which cuts nothing and needs no look at what it gives.
__device__ __forceinline__ bool tree_try(int pass, float all, float tiles, float fit, float& each) {
    if (pass < kTries) {
        each = all / fmaxf(fit - tiles * (0.3f + 0.7f / (kTries - 1) * (float)pass), 0.0f);
    } else if (pass == kTries) {
        each = 2.0f * all / fit;
    } else {
        each = INFINITY;
        return true;
    }
    return false;
}

// The length of a line's stretches where a workgroup has `each` of it.
__device__ __forceinline__ int32_t tree_per(int32_t units, int32_t heads, float length, float each, float fit) {
    return tree_stretch(units, heads, max((int32_t)fminf(ceilf(length / each), fit), 1));
}

// The piece at hand.  PLANNED: kv_tree_plan_kernel has been over the sequences.
template <int ROWS, bool PLANNED>
struct TreeWork {
    const KvView& c;
    const TreeArgs& a;
    TreeStretch& kept;
    int b, h, t0, n, r0, rows, u0, u1;
    int32_t past;

    // The index-th workgroup's; whether it has one.  Stretches are as long as lets all workgroups that fit the device have
    // one and no more (a line's last stretch costs up to a whole one more: how much of one on average is tried); where
    // there are more tiles than that, long lines are still cut, into stretches twice what each workgroup would have.
    __device__ __forceinline__ bool find(int64_t index) {
        const int lane = here(threadIdx.x & 63);
        auto seq_at = [&](int b) { return b < c.B ? tree_seq<ROWS>(c, a, b) : TreeSeq{0, 0, 0, 0, 0}; };
        const float fit = (float)a.fit;
        float all = 0.0f, each = 0.0f, tiles = 0.0f;
        bool found = false;
        int first = 0;                               // sequences that are passed over, and what lies before them
        TreeChunk before{0, 0};
        TreeSeq early;                               // of the first 64 sequences, a lane each
        if constexpr (PLANNED) {
            const int chunks = (c.B + 63) >> 6;
            if (a.chunk[chunks].groups <= index) return false;
            int lo = 0, n = chunks;                  // the last chunk that starts at or before `index`, 64 ways at a time
            while (n > 1) {
                const int step = (n + 63) >> 6, i = lane * step;
                const uint64_t m = __ballot(i < n && a.chunk[lo + i].groups <= index);
                const int k = 63 - __clzll((long long)m);
                lo += k * step;
                n = min(step, n - k * step);
            }
            first = of(lo) * 64;
            before = a.chunk[of(lo)];
            each = *a.each;
            found = true;
        } else {
            early = seq_at(lane);
        }
        // first the sums, then some tries, then the workgroup's place; one body for all: the code's own length is what it
        // costs
#pragma clang loop unroll(disable)
        for (int pass = PLANNED ? kTries + 1 : 0;; ++pass) {
            int64_t groups = before.groups, cut = before.cut;        // workgroups, and those of cut lines
#pragma clang loop unroll(disable)
            for (int b0 = first; b0 < c.B; b0 += 64) {
                const TreeSeq s = !PLANNED && b0 == 0 ? early : seq_at(b0 + lane);
                const int32_t length = (s.units + kTreeStart) * c.H;
                if (pass == 0) all += wave_sum((float)length * (float)s.tiles);
                const int32_t per = pass == 0 ? length : tree_per(s.units, c.H, (float)length, each, fit);
                const int32_t w = (int32_t)((uint32_t)(length + per - 1) / (uint32_t)per), mine = w * s.tiles;
                const int32_t upto = (int32_t)wave_scan((uint32_t)mine), cuts = (int32_t)wave_scan(w > 1 ? (uint32_t)mine : 0u);
                const uint64_t here_it_is = found ? __ballot(groups + upto > index) : 0;
                if (here_it_is) {
                    const int k = __ffsll((long long)here_it_is) - 1;
                    TreeStretch x;
                    x.b = b0 + k;
                    x.t0 = __builtin_amdgcn_readlane(s.t0, k);
                    x.n = __builtin_amdgcn_readlane(s.n, k);
                    x.past = __builtin_amdgcn_readlane(s.past, k);
                    x.units = __builtin_amdgcn_readlane(s.units, k);
                    const int32_t all_w = __builtin_amdgcn_readlane(w, k), its = __builtin_amdgcn_readlane(s.tiles, k);
                    const TreePlace p =
                        tree_place((int32_t)(index - groups) - (__builtin_amdgcn_readlane(upto, k) - all_w * its), all_w, its);
                    x.r0 = p.tile * ROWS;
                    x.stretch = p.stretch;
                    x.first_group = (int32_t)cut + __builtin_amdgcn_readlane(cuts, k) - all_w * its + p.tile * all_w;
                    x.per = __builtin_amdgcn_readlane(per, k);
                    x.hi = (int32_t)min((int64_t)(p.stretch + 1) * x.per, (int64_t)__builtin_amdgcn_readlane(length, k));
                    x.h = (int32_t)((uint32_t)p.stretch * (uint32_t)x.per / (uint32_t)(x.units + kTreeStart));
                    kept = x;
                    return true;
                }
                groups += __builtin_amdgcn_readlane(upto, 63);
                cut += __builtin_amdgcn_readlane(cuts, 63);
            }
            if (found) return false;
            if (pass == 0) {
                tiles = (float)groups;
                // offsets that overlap make more tiles than the launch has workgroups for: a cut head might be left half done
                if (groups > a.groups - a.fit) pass = kTries + 1;
            } else if ((pass <= kTries ? groups : cut) <= a.fit) {
                found = true;
                continue;
            }
            if (tree_try(pass, all, tiles, fit, each)) found = true;
        }
    }
    // The next piece; whether there is one.
    __device__ __forceinline__ bool next() {
        const int32_t units = of(kept.units), lo = of(kept.stretch) * of(kept.per), hi = of(kept.hi);
        for (h = of(kept.h);; ++h) {
            const int32_t place = h * (units + kTreeStart);
            if (place >= hi) return false;
            u0 = tree_cut(lo - place, units);
            u1 = place + units + kTreeStart <= hi ? units : tree_cut(hi - place, units);
            if (u0 < u1) break;
        }
        kept.h = h + 1;
        b = of(kept.b);
        t0 = of(kept.t0);
        n = of(kept.n);
        past = of(kept.past);
        r0 = of(kept.r0);
        rows = min(n * a.G - r0, ROWS);
        return true;
    }
    static __device__ __forceinline__ int32_t of(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
    // Joins the head's pieces, where there are several: put(slot) writes the workgroup's sums, add(slot, first, step, n) makes
    // them the sums of the pieces from `first` on, `step` apart, in their order.  Pieces are added in groups of
    // kJoin: whoever finishes a group's last piece adds the group's pieces, whoever finishes the last group adds the
    // groups' sums.  Whether the sums are the head's then.  A stretch has four counts: of the group that its piece inside
    // a head leads, of the one that its piece at a head's start does, of that head's groups.
    template <class Put, class Add>
    __device__ __forceinline__ bool join(Put put, Add add) const {
        const int32_t units = of(kept.units), stretch = of(kept.stretch);
        if (u0 == 0 && u1 == units) return true;
        const TreePieces range = tree_pieces(h * (units + kTreeStart), units, of(kept.per));
        const int piece = (int)(stretch - range.first), pieces = (int)(range.last - range.first) + 1;
        const int group = piece / kJoin, lead = group * kJoin, members = min(kJoin, pieces - lead), groups = (pieces - 1) / kJoin + 1;
        const int32_t first = of(kept.first_group) + range.first;
        auto slot = [&](int j) { return tree_slot(first, j); };
        put(slot(piece));
        if (!arrive(a.arrived + 4 * (first + lead) + (group == 0), members)) return false;
        add(slot, lead, 1, members);
        if (groups == 1) return true;
        // the group's sum in the place of its first piece, which all of the workgroup has read
        __syncthreads();
        put(slot(lead));
        if (!arrive(a.arrived + 4 * first + 2, groups)) return false;
        add(slot, 0, kJoin, groups);
        return true;
    }
};

// Sequences that every workgroup goes through by itself; more go through kv_tree_plan_kernel, a launch that takes 6 us
// for these.  Without and with it, 8 drafts each over 500 tokens, us: 8 kv heads of 128: 128 sequences 36 and 42, 160 45
// and 51, 192 68 and 67, 256 77 and 72, 512 183 and 145; one of 64: 128 13 and 19, 192 18 and 19, 256 23 and 19.
constexpr int kFewSeqs = 192;

// The search of TreeWork::find for many sequences, where going through all of them in every workgroup takes as
// long as their number squared (4,096 of 8 drafts x 8 heads, one kv head 7.1 ms instead of 0.21; 65,536 of one draft
// 707 ms instead of 1.1): one workgroup finds what each of the others has and where the chunks start.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
template <int ROWS>
__global__ __launch_bounds__(kPlanThreads) void kv_tree_plan_kernel(KvView c, TreeArgs a) {
    __shared__ float lengths[kPlanWaves];
    __shared__ TreeChunk chunks[kPlanWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float fit = (float)a.fit;
    // a sequence's workgroups, those of a cut line, and its line times its tiles
    auto seq = [&](int b, float each, float& length) {
        const TreeSeq s = b < c.B ? tree_seq<ROWS>(c, a, b) : TreeSeq{0, 0, 0, 0, 0};
        const int32_t line = (s.units + kTreeStart) * c.H, per = tree_per(s.units, c.H, (float)line, each, fit);
        const int32_t w = (int32_t)((uint32_t)(line + per - 1) / (uint32_t)per);
        length = (float)line * (float)s.tiles;
        return TreeChunk{(int64_t)w * s.tiles, w > 1 ? (int64_t)w * s.tiles : 0};
    };
    auto wave_total = [](TreeChunk x) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            x.groups += __shfl_xor(x.groups, o);
            x.cut += __shfl_xor(x.cut, o);
        }
        return x;
    };
    float all;
    auto totals = [&](float each) {
        TreeChunk sum{0, 0};
        float mine = 0.0f;
        for (int b = threadIdx.x; b < c.B; b += kPlanThreads) {
            float length;
            const TreeChunk x = seq(b, each, length);
            sum.groups += x.groups;
            sum.cut += x.cut;
            mine += length;
        }
        sum = wave_total(sum);
        mine = wave_sum(mine);
        __syncthreads();
        if (lane == 0) {
            chunks[wave] = sum;
            lengths[wave] = mine;
        }
        __syncthreads();
        sum = {0, 0};
        all = 0.0f;
        for (int w = 0; w < kPlanWaves; ++w) {
            sum.groups += chunks[w].groups;
            sum.cut += chunks[w].cut;
            all += lengths[w];
        }
        return sum;
    };
    // as in find, but without tries that cannot succeed, since each tile takes a workgroup at least
    float each = INFINITY;
    const int64_t tiles = totals(each).groups;
    if (tiles <= a.groups - a.fit)
        for (int pass = tiles > a.fit ? kTries : 0;; ++pass) {
            if (tree_try(pass, all, (float)tiles, fit, each)) break;
            const TreeChunk x = totals(each);
            if ((pass < kTries ? x.groups : x.cut) <= a.fit) break;
        }
    TreeChunk before{0, 0};
    for (int b0 = 0; b0 < c.B; b0 += kPlanThreads) {
        float length;
        const TreeChunk x = wave_total(seq(b0 + threadIdx.x, each, length));
        __syncthreads();
        if (lane == 0) chunks[wave] = x;
        __syncthreads();
        for (int w = 0; w < kPlanWaves; ++w) {
            const int i = (b0 >> 6) + w;
            if (w == wave && lane == 0 && i * 64 < c.B) a.chunk[i] = before;
            before.groups += chunks[w].groups;
            before.cut += chunks[w].cut;
        }
    }
    if (threadIdx.x == 0) {
        a.chunk[(c.B + 63) >> 6] = before;
        *a.each = each;
    }
}

template <int D, bool FP8, int NR, bool PLANNED>
__global__ __launch_bounds__(256, 2) void kv_tree_kernel(KvView c, TreeArgs a) {
    constexpr int ROWS = 32 * NR, ND = D / 64, NC = D / 32;
    constexpr bool HELD = D * NR <= 128;
    constexpr int DEPTH = D * NR <= 128 ? 2 : 1;         // steps whose codes are on their way
    __shared__ TreeLds<D, NR> lds;
    __shared__ TreeStretch stretch[4];
    TreeWork<ROWS, PLANNED> work{c, a, stretch[__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)]};
    for (int64_t i = blockIdx.x; i < a.groups && work.find(i); i += gridDim.x) while (work.next()) {
        const int thread = here(threadIdx.x), lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
        const int col = lane & 31, hi = lane >> 5;
        const int b = work.b, h = work.h, t0 = work.t0, n = work.n, r0 = work.r0, rows = work.rows, u0 = work.u0, u1 = work.u1;
        const int32_t past = work.past;
        const Span span = span_of(c, a, past, n);
        // A wave's blocks, two a step, are looked up 32 steps at a time, lane 2 i + e holding block e of step i.
        const Blocks blocks(c, b, h);
        const int steps = u1 - u0;
        auto tile_of = [&](int i, int e) { return (u0 + i) * kUnit + wave * 2 + e; };
        auto load_pages = [&](int i0) {
            return blocks.pages[min(span.tile(tile_of(i0 + (lane >> 1), lane & 1)), blocks.n_blocks - 1) >> blocks.shift];
        };
        auto checked = [&](int32_t page, int i0) {
            const int i = i0 + (lane >> 1);
            const bool there = (i < steps) & (tile_of(i, lane & 1) < span.n) & ((uint32_t)page < (uint32_t)blocks.n_pages);
            return there ? page : -1;
        };
        auto load_scale = [&](const float* p, int32_t page) {
            return page >= 0 ? fmaxf(p[(int64_t)page * blocks.H], kScaleMin) : 1.0f;
        };
        auto of_lane = [](float x, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)); };
        const int32_t first_pages = load_pages(0);
        int32_t later = load_pages(32);

        // The tile's queries in half precision, in the order in which the products read them; a thread's share of a row is
        // D * NR / 8 dimensions.
        {
            constexpr int PER = 8 / NR;                      // threads of a row
            constexpr int N = D / PER / 8;                   // 16-byte pieces of a thread
            const int row = thread / PER, j = thread % PER;
            const int r = r0 + row;
            const uint32_t flip = a.scale2 < 0.0f ? 0x80008000u : 0u;
            uint4v raw[N];
            const uint16_t* p = a.q + (int64_t)(t0 + r / a.G) * a.q_stride + ((int64_t)h * a.G + r % a.G) * D + j * N * 8;
#pragma unroll
            for (int i = 0; i < N; ++i)
                raw[i] = (row < rows ? *reinterpret_cast<const uint4v*>(p + i * 8) : uint4v{0, 0, 0, 0}) ^ flip;
            float undo = 1.0f;
            if (!c.f16) {
                uint32_t top = 0;            // largest magnitude, as bits: the exponent decides
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        top = max(top, max((raw[i][e] << 16) & 0x7FFFFFFFu, raw[i][e] & 0x7FFF0000u));
#pragma unroll
                for (int o = 1; o < PER; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
                const float f = half_range_factor(top);
                undo = half_range_undo(top);
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2v x = unpack2<false>(raw[i][e]);
                        raw[i][e] = pack2<true>(x.x * f, x.y * f);
                    }
            }
            if (j == 0) lds.undo[row] = undo;
            // dimensions 8 p .. of a row: product 4 (p / 8) + 2 (p / 4 % 2) + p % 2, half p / 2 % 2
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int p8 = j * N + i;
                lds.q[(p8 >> 3) * 4 + (p8 >> 2 & 1) * 2 + (p8 & 1)][row >> 5][(p8 >> 1 & 1) * 32 + (row & 31)] = raw[i];
            }
        }
        // the lane's rows: their tokens and positions
        auto token_of = [&](int i) { return t0 + (r0 + min(i, rows - 1)) / a.G; };       // of a row of the tile
        auto pos_of = [&](int t) { return a.window > 0 ? min(max(a.pos[t], past), kMaxPast) : past; };
        float s2[NR];
        int32_t pos_max = past;
#pragma unroll
        for (int g = 0; g < NR; ++g) pos_max = max(pos_max, pos_of(token_of(g * 32 + col)));
        if (a.window > 0)
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) pos_max = max(pos_max, __shfl_xor(pos_max, o));
        __syncthreads();
#pragma unroll
        for (int g = 0; g < NR; ++g) s2[g] = fabsf(a.scale2) * lds.undo[g * 32 + col];

        // 32 rows of up to 128 dimensions have room in registers
        uint4v held[HELD ? D / 16 : 1][NR];
        if constexpr (HELD)
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
                for (int g = 0; g < NR; ++g) held[k][g] = lds.q[k][g][lane];

        // blocks (of the span) that all rows see whole, but for the sinks
        const int32_t base_i = span.n_sink - span.win;
        const int32_t full_lo = a.window > 0 ? max(span.n_sink, ((pos_max - a.window + 16) >> 4) + base_i) : 0;
        const int32_t full_hi = (past >> 4) + base_i;        // not itself

        // Codes of a step: keys [64 dimensions][32 of them], values [token block][64 or 128 dimensions][token groups hi and hi + 2]
        struct Raw {
            uint4v k[ND][2];
            uint4v v[2][ND == 4 ? 2 : 1][2];
        };
        auto fetch_k = [&](int64_t at0, int64_t at1, Raw& r) {
            const uint8_t* p = blocks.k + (lane & 16 ? at1 : at0) + (lane & 15) * 64 + hi * 16;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int j = 0; j < 2; ++j) r.k[d][j] = *reinterpret_cast<const uint4v*>(p + d * 1024 + j * 32);
        };
        auto fetch_v = [&](int64_t at0, int64_t at1, Raw& r) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint8_t* p = blocks.v + (e == 0 ? at0 : at1);
                if constexpr (D == 64) {
                    // two of the four dimensions that 16 bytes hold, the lanes 16 apart the other two
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const uint2v x = *reinterpret_cast<const uint2v*>(p + (hi + 2 * g) * 256 + (lane & 15) * 16 + (lane >> 4 & 1) * 8);
                        r.v[e][0][g] = uint4v{x[0], x[1], 0, 0};
                    }
                } else {
#pragma unroll
                    for (int d = 0; d < D / 128; ++d)
#pragma unroll
                        for (int g = 0; g < 2; ++g)
                            r.v[e][d][g] = *reinterpret_cast<const uint4v*>(p + (2 * d + (lane >> 4 & 1)) * 1024 + (hi + 2 * g) * 256 +
                                                                            (lane & 15) * 16);
                }
            }
        };

        float m_run[NR], l_run[NR];
        float16v o[NR][NC] = {};
#pragma unroll
        for (int g = 0; g < NR; ++g) {
            m_run[g] = kNoMax;
            l_run[g] = 0.0f;
        }
        // where the codes lie of the steps that are fetched; the scales, and which blocks are absent (bits), of those that
        // are computed and of the next
        int64_t offset;
        float ks, vs, log_vs = 0.0f, inv_vs = 0.0f, ks_next, vs_next;
        uint64_t absent, absent_next;
        auto look_up = [&](int32_t page, int i0) {
            page = checked(page, i0);
            offset = blocks.at(page, span.tile(tile_of(i0 + (lane >> 1), lane & 1)));
            ks_next = load_scale(blocks.ks, page);
            vs_next = load_scale(blocks.vs, page);
            absent_next = __ballot(page < 0);
        };
        look_up(first_pages, 0);
        // one step; the codes of step i + DEPTH go into the registers that it has read
        auto step = [&](int i, Raw& raw) {
            const int l = (i & 31) * 2, l1 = (i + DEPTH & 31) * 2;
            if (l == 0) {
                ks = ks_next;
                vs = vs_next;
                absent = absent_next;
                log_vs = __builtin_amdgcn_logf(vs);
                inv_vs = __builtin_amdgcn_rcpf(vs);
            }
            const float f[2] = {of_lane(ks, l), of_lane(ks, l + 1)};
            const float log_scale[2] = {of_lane(log_vs, l), of_lane(log_vs, l + 1)};
            const float inv_scale[2] = {of_lane(inv_vs, l), of_lane(inv_vs, l + 1)};
            const uint32_t gone = (uint32_t)(absent >> l) & 3;
            if (l1 == 0) {
                look_up(later, i + DEPTH);
                later = load_pages(i + DEPTH + 32);
            }
            const int64_t at0 = of_lane64(offset, l1), at1 = of_lane64(offset, l1 + 1);
            float16v s[NR] = {};
            auto product = [&](int k, const uint4v (&query)[NR]) {
                const uint4v codes = raw.k[k >> 2][k >> 1 & 1];
                const half8 key = code_halves8<FP8>(codes[2 * (k & 1)], codes[2 * (k & 1) + 1]);
#pragma unroll
                for (int g = 0; g < NR; ++g)
                    s[g] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key, __builtin_bit_cast(half8, query[g]), s[g], 0, 0, 0);
            };
            if constexpr (HELD) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) product(k, held[k]);
            } else {
                // the queries' operands are read kAhead products ahead; the barriers keep the reads from gathering in front,
                // where their registers would not fit
                constexpr int kAhead = 2;
                uint4v queries[kAhead + 1][NR];
                auto read_queries = [&](int k) {
#pragma unroll
                    for (int g = 0; g < NR; ++g) queries[k % (kAhead + 1)][g] = lds.q[k][g][lane];
                };
#pragma unroll
                for (int k = 0; k < kAhead; ++k) read_queries(k);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    if (k + kAhead < D / 16) read_queries(k + kAhead);
                    __builtin_amdgcn_sched_barrier(0);
                    product(k, queries[k % (kAhead + 1)]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            fetch_k(at0, at1, raw);
            const int i0 = tile_of(i, 0);
            const bool masked = (gone != 0) | (i0 < full_lo) | (i0 + 1 >= full_hi);
            if (masked) {
                const int own = here(col);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int32_t tok = span.tile(i0 + e) * 16;
                    uint32_t any = 0;
#pragma unroll
                    for (int g = 0; g < NR; ++g) {
                        const int t = token_of(g * 32 + own);
                        uint32_t seen = (gone >> e & 1) == 0 ? tree_sight(a, a.mask + (int64_t)t * a.words, past, n, pos_of(t), tok) : 0u;
                        any |= seen;
                        seen >>= 4 * hi;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float x = s[g][e * 8 + k];
                            s[g][e * 8 + k] = seen >> (8 * (k >> 2) + (k & 3)) & 1 ? x : -INFINITY;
                        }
                    }
                    // value codes of tokens that no row of the tile sees stay out of the product: they may be NaN
#pragma unroll
                    for (int w = 1; w < 32; w <<= 1) any |= (uint32_t)__shfl_xor((int)any, w);
                    const uint32_t keep0 = bytes_of(any >> 4 * hi), keep1 = bytes_of(any >> (4 * hi + 8));
#pragma unroll
                    for (int d = 0; d < (ND == 4 ? 2 : 1); ++d) {
                        raw.v[e][d][0] &= keep0;
                        raw.v[e][d][1] &= keep1;
                    }
                }
            }
            half8 p[NR][2];
            // from the logits as they are rounded for the reference, or in one operation less: the same while a logit's last
            // bit is below 1, from 2^24 on too large or small by up to that bit
            float fs[NR][2], sum[NR][2];
            auto weigh = [&](auto rounded, int g) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float off = log_scale[e] - m_run[g];
                    sum[g][e] = 0.0f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float x = s[g][e * 8 + k];
                        const float w = __builtin_amdgcn_exp2f(rounded ? fmaf(x, fs[g][e], log_scale[e]) - m_run[g] : fmaf(x, fs[g][e], off));
                        sum[g][e] += w;
                        p[g][e][k] = (_Float16)w;
                    }
                }
            };
#pragma unroll
            for (int g = 0; g < NR; ++g) {
#pragma unroll
                for (int e = 0; e < 2; ++e) fs[g][e] = fmaxf(f[e] * s2[g], 1e-37f);        // not 0: -inf of a hidden token stays
                weigh(std::false_type{}, g);
                const float level = sum[g][0] + sum[g][1];
                if (__any(off_range(level, false))) {
                    float mx = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = s[g][e * 8];
#pragma unroll
                        for (int k = 1; k < 8; ++k) top = fmaxf(top, s[g][e * 8 + k]);
                        mx = fmaxf(mx, fmaf(top, fs[g][e], log_scale[e]));
                    }
                    mx = fmaxf(mx, __shfl_xor(mx, 32));
                    float to = raised(m_run[g], mx, kTreeTop);
                    const bool low = is_low(m_run[g], mx, false);
                    if (__any(low)) {
                        float largest = l_run[g];
#pragma unroll
                        for (int i = 0; i < NC; ++i)
#pragma unroll
                            for (int k = 0; k < 16; ++k) largest = fmaxf(largest, fabsf(o[g][i][k]));
                        largest = fmaxf(largest, __shfl_xor(largest, 32));
                        to = low ? lowered(m_run[g], mx, largest) : to;
                    }
                    if (__any((to != m_run[g]) | (level > kMostWeight))) {
                        const float by = __builtin_amdgcn_exp2f(m_run[g] - to);
                        m_run[g] = to;
                        l_run[g] *= by;
#pragma unroll
                        for (int i = 0; i < NC; ++i) o[g][i] *= by;
                        weigh(std::true_type{}, g);
                    }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) l_run[g] = fmaf(sum[g][e], inv_scale[e], l_run[g]);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const half8 value = code_halves8<FP8>(raw.v[e][i >> 2][0][i & 3], raw.v[e][i >> 2][1][i & 3]);
#pragma unroll
                    for (int g = 0; g < NR; ++g)
                        o[g][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value, p[g][e], o[g][i], 0, 0, 0);
                    if (NR > 1) __builtin_amdgcn_sched_barrier(0);
                }
            fetch_v(at0, at1, raw);
        };
        Raw raw[DEPTH];
#pragma unroll
        for (int k = 0; k < DEPTH; ++k) {
            const int64_t at0 = of_lane64(offset, 2 * k), at1 = of_lane64(offset, 2 * k + 1);
            fetch_k(at0, at1, raw[k]);
            fetch_v(at0, at1, raw[k]);
        }
        for (int i = 0; i < steps; i += DEPTH)
#pragma unroll
            for (int k = 0; k < DEPTH; ++k)
                if (k == 0 || i + k < steps) step(i + k, raw[k]);

        // the four waves' sums, 64 dimensions at a time; then a thread has 2 or 4 NR of them, side by side in a row
        const int late = here(threadIdx.x), late_col = late & 31, late_hi = late >> 5 & 1;
        float f_wave[NR];
#pragma unroll
        for (int g = 0; g < NR; ++g) {
            l_run[g] += __shfl_xor(l_run[g], 32);
            if (late_hi == 0) lds.ml[wave][g * 32 + late_col] = float2v{m_run[g], l_run[g]};
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < NR; ++g) {
            float m_all = kNoMax;
#pragma unroll
            for (int w = 0; w < 4; ++w) m_all = fmaxf(m_all, lds.ml[w][g * 32 + late_col].x);
            f_wave[g] = __builtin_amdgcn_exp2f(m_run[g] - m_all);
        }
        constexpr int PER = 8 / NR, W = 64 / PER;            // threads of a row, and their dimensions of 64
        const int row = late / PER, d0 = late % PER * W;
        float m_row = kNoMax, l_row = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) m_row = fmaxf(m_row, lds.ml[w][row].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) l_row = fmaf(lds.ml[w][row].y, __builtin_amdgcn_exp2f(lds.ml[w][row].x - m_row), l_row);
        float4v sums[ND][W / 4];
#pragma unroll
        for (int d = 0; d < ND; ++d) {
#pragma unroll
            for (int g = 0; g < NR; ++g) {
                float* to = lds.comb[wave][g * 32 + late_col];
                if constexpr (D == 64) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        *reinterpret_cast<float2v*>(to + dim_of<D>(i, late_hi)) = float2v{o[g][0][i], o[g][1][i]} * f_wave[g];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int k = (d & 1) * 8 + i;
                        *reinterpret_cast<float4v*>(to + dim_of<D>(k, late_hi)) =
                            float4v{o[g][d / 2 * 4][k], o[g][d / 2 * 4 + 1][k], o[g][d / 2 * 4 + 2][k], o[g][d / 2 * 4 + 3][k]} * f_wave[g];
                    }
                }
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < W / 4; ++j) {
                sums[d][j] = *reinterpret_cast<const float4v*>(&lds.comb[0][row][d0 + j * 4]);
#pragma unroll
                for (int w = 1; w < 4; ++w) sums[d][j] += *reinterpret_cast<const float4v*>(&lds.comb[w][row][d0 + j * 4]);
            }
            __syncthreads();
        }

        auto put = [&](int32_t slot) {
            if (row >= rows) return;
            const int64_t at = (int64_t)slot * ROWS + row;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int j = 0; j < W / 4; ++j) {
                    float* to = a.part_o + at * D + d * 64 + d0 + j * 4;
                    put_shared(to, float2v{sums[d][j].x, sums[d][j].y});
                    put_shared(to + 2, float2v{sums[d][j].z, sums[d][j].w});
                }
            if (d0 == 0) put_shared((float*)&a.part_ml[at], float2v{m_row, l_row});
        };
        auto add = [&](auto slot, int from, int step, int n) {
            if (row >= rows) return;
            m_row = kNoMax;
            l_row = 0.0f;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int j = 0; j < W / 4; ++j) sums[d][j] = float4v{0, 0, 0, 0};
            for (int i = 0; i < n; ++i) {
                const int64_t at = (int64_t)slot(from + i * step) * ROWS + row;
                const float2v ml = get_shared((const float*)&a.part_ml[at]);
                float2v x[ND][W / 4][2];
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int j = 0; j < W / 4; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) x[d][j][e] = get_shared(a.part_o + at * D + d * 64 + d0 + j * 4 + 2 * e);
                const float top = fmaxf(m_row, ml.x), by = __builtin_amdgcn_exp2f(m_row - top), f = __builtin_amdgcn_exp2f(ml.x - top);
                m_row = top;
                l_row = l_row * by + ml.y * f;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int j = 0; j < W / 4; ++j)
                        sums[d][j] = sums[d][j] * by + float4v{x[d][j][0].x, x[d][j][0].y, x[d][j][1].x, x[d][j][1].y} * f;
            }
        };
        const bool last = work.join(put, add);
        if (last && row < rows) {
            const float norm = l_row > 0.0f ? 1.0f / l_row : 0.0f;
            const int r = r0 + row;
            uint16_t* out = a.out + (int64_t)(t0 + r / a.G) * a.out_stride + ((int64_t)h * a.G + r % a.G) * D + d0;
            auto pair = [&](float x, float y) { return c.f16 ? pack2<true>(x * norm, y * norm) : pack2<false>(x * norm, y * norm); };
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int j = 0; j < W / 4; ++j)
                    *reinterpret_cast<uint2v*>(out + d * 64 + j * 4) =
                        uint2v{pair(sums[d][j].x, sums[d][j].y), pair(sums[d][j].z, sums[d][j].w)};
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_kv_tree(const KvView& c, const KvTree& t, const void* q, int64_t q_stride, int32_t Hq, float scale,
                          int32_t window, int32_t sinks, void* out, int64_t out_stride, void* workspace,
                          int64_t workspace_bytes, int n_cu, hipStream_t s) {
    TreeArgs a{};
    a.q = (const uint16_t*)q;
    a.out = (uint16_t*)out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.G = Hq / c.H;
    a.scale2 = scale * 1.4426950408889634f;
    a.window = window;
    a.sinks = sinks;
    a.mask = t.mask;
    a.words = t.words;
    a.pos = t.pos;
    // Tiles of 64 rows halve the conversions and the codes' way from the caches, and leave half as many workgroups something
    // to do: worth it once tiles of 32 are more than fit the device at one time.  Measured with 32 and 64, 8 kv heads of 128
    // where nothing else is said, us: 16 sequences of 2,000 tokens with 128 rows (512 tiles of 32) 33 and 57, 20 of them
    // (640) 66 and 43; 32 with 48 rows (512) 33 and 62, 50 with 64 rows (800) 70 and 52; 128 of 1,000 with 36 rows 91 and 64;
    // 80 with 128 rows, 2 heads (640) 72 and 49; 8 of 4,000 with 128 rows, 16 heads (512) 48 and 78, 32 heads (1,024) 103
    // and 90; 20 with 128 rows of 64 dimensions (640) 42 and 33.  Half-filled tiles can lose: 10 of 4,000 with 66 rows, 32
    // heads 110 and 128.  Lengths are on the device: of uneven ones a last tile is taken to be half full.  Over very long
    // caches the conversions count alone: 4 of 16,000 with 512 rows 152 and 161; 2 of 88,000 with 512 rows 530 and 455.  How
    // long is taken from the table's width, which can be far more than is cached: 8 of 2,000 with 256 rows in tables of
    // 2,064, 16,384 and 131,072 tokens 34, 33 and 66 (31 with 32), 8 of 16,000 in the last 173 (156).
    const int64_t all_rows = (int64_t)c.T * a.G, most_rows = (int64_t)c.max_new * a.G;
    const int64_t tiles32 = std::min(all_rows / 32 + c.B / 2, (most_rows + 31) / 32 * c.B);
    const bool wide = c.D != 256 && ((most_rows > 32 && tiles32 * c.H > (int64_t)n_cu * 2) ||
                                     (most_rows >= 256 && all_rows * c.limit >= 1 << 26));
    const int rows = wide ? 64 : 32;
    const int64_t tiles = (int64_t)c.T * a.G / rows + c.B;
    const int64_t line = ((int64_t)c.limit / (16 * kUnit) + 2 + kTreeStart) * c.H;
    if (tiles * c.H >= (int64_t)1 << 24 || line >= (int64_t)1 << 31) return hipErrorInvalidConfiguration;
    // workgroups that fit the device, as far as the workspace has two slots for each
    WsCarve ws{(char*)workspace, (size_t)workspace_bytes};
    a.arrived = ws.take<uint32_t>(kMaxParts * 2);
    const bool planned = c.B > kFewSeqs;
    if (planned) {
        a.each = ws.take<float>(1);
        a.chunk = ws.take<TreeChunk>((int64_t)(c.B + 63) / 64 + 1);
    }
    const int64_t room = (workspace_bytes - (int64_t)ws.off - 512) / ((int64_t)rows * (c.D + 2) * 4 * 2);
    a.fit = (int32_t)std::min<int64_t>({(int64_t)n_cu * 2, room, kMaxParts / 2});
    a.part_ml = ws.take<float2v>((int64_t)a.fit * 2 * rows);
    a.part_o = ws.take<float>((int64_t)a.fit * 2 * rows * c.D);
    if (!ws.ok()) return hipErrorInvalidConfiguration;
    a.groups = tiles + a.fit;
    const int64_t wgs = std::min<int64_t>(a.groups, 1 << 20);
    auto launch = [&](auto d, auto fp8, auto tiles_of) {
        constexpr int D = decltype(d)::value, NR = decltype(tiles_of)::value;
        constexpr bool FP8 = decltype(fp8)::value;
        if (!planned) {
            kv_tree_kernel<D, FP8, NR, false><<<(uint32_t)wgs, 256, 0, s>>>(c, a);
            return hipGetLastError();
        }
        kv_tree_plan_kernel<32 * NR><<<1, kPlanThreads, 0, s>>>(c, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        kv_tree_kernel<D, FP8, NR, true><<<(uint32_t)wgs, 256, 0, s>>>(c, a);
        return hipGetLastError();
    };
    auto run = [&](auto d, auto fp8) {
        if constexpr (decltype(d)::value != 256)
            if (rows == 64) return launch(d, fp8, std::integral_constant<int, 2>{});
        return launch(d, fp8, std::integral_constant<int, 1>{});
    };
    auto by_dim = [&](auto fp8) {
        if (c.D == 64) return run(std::integral_constant<int, 64>{}, fp8);
        if (c.D == 128) return run(std::integral_constant<int, 128>{}, fp8);
        return run(std::integral_constant<int, 256>{}, fp8);
    };
    return c.fp8 ? by_dim(std::true_type{}) : by_dim(std::false_type{});
}

}  // namespace ls
