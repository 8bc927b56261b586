// Attention of drafted tokens over the paged 8-bit KV cache (k_kv.h): a tree behind
// each sequence's cached tokens.
//
// out_i = sum_j softmax_j(scale q_i . k_j) v_j over the cached tokens that row i's
// position sees and the new tokens whose bit its mask has, with the weights and
// their reference as in k_kv_attend.hip.
//
// A tree's rows (new tokens x query heads of one kv head) are more than a decode step's
// and fewer than a prompt's, over as many cached tokens: at 4 D operations and 2 D
// bytes a token, reading and computing take the same time at about 130 rows.  So the
// tokens are what is dealt out: a wave takes 32 of a unit's 128 tokens with all of a
// tile's 32 or 64 rows, codes go from memory to registers in 16-byte loads and each
// operand made of them serves all rows.  Only the queries are in LDS.
#include <algorithm>

#include "k_kv_attend.h"
#include "ls_kv_calls.h"
#include "ls_scratch.h"

namespace ls {
namespace {

using float16v = float __attribute__((ext_vector_type(16)));

struct TreeArgs : AttnArgs {
    const uint64_t* mask;
    int32_t words;
    const int32_t* pos;
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
__device__ __forceinline__ TreeSeq tree_seq(const KvView& c, const AttnArgs& a, int b) {
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

template <int D, bool FP8, int NR>
__global__ __launch_bounds__(256, 2) void kv_tree_kernel(KvView c, TreeArgs a, bool cut) {
    constexpr int ROWS = 32 * NR, ND = D / 64, NC = D / 32;
    __shared__ TreeLds<D, NR> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, hi = lane >> 5;

    // Segments (sequence, head, row tile) are cut into equal parts of at most `most` units, so that about as many parts
    // as workgroups hold all units (not cut: a part is a segment).
    uint32_t most = 1u << 30;
    TreeSeq mine = {0, 0, 0, 0, 0};          // of the first 64 sequences, a lane each
    if (lane < c.B) mine = tree_seq<ROWS>(c, a, lane);
    if (cut) {
        uint64_t all = 0, segs = 0;
        for (int b0 = 0; b0 < c.B; b0 += 64) {
            TreeSeq s = mine;
            if (b0 > 0) {
                s.units = s.tiles = 0;
                if (b0 + lane < c.B) s = tree_seq<ROWS>(c, a, b0 + lane);
            }
            const uint64_t x = (uint64_t)s.units * s.tiles;
            // below 2^23 units, and 2^30 rows of a call: sums of 64 in two halves
            all += __builtin_amdgcn_readlane(wave_scan((uint32_t)(x & 0xFFFFFu)), 63) +
                   ((uint64_t)__builtin_amdgcn_readlane(wave_scan((uint32_t)(x >> 20 & 0xFFFFFu)), 63) << 20) +
                   ((uint64_t)__builtin_amdgcn_readlane(wave_scan((uint32_t)(x >> 40)), 63) << 40);
            segs += __builtin_amdgcn_readlane(wave_scan((uint32_t)s.tiles), 63);
        }
        const uint64_t room = max((int64_t)gridDim.x - (int64_t)(segs * (uint32_t)c.H), (int64_t)1);
        const uint64_t each = (all * (uint32_t)c.H + room - 1) / room;
        most = (uint32_t)min(max(each, (uint64_t)kMinUnits), (uint64_t)1 << 30);
    }
    for (uint64_t part = blockIdx.x;; part += gridDim.x) {
        // sequences' first parts are the sums of the parts before them
        uint64_t base = 0;
        uint32_t own = 0, count = 0, before = 0;
        uint64_t found = 0;
        TreeSeq its = mine;
        int b0 = 0;
        for (; b0 < c.B; b0 += 64) {
            if (b0 > 0) {
                its = TreeSeq{0, 0, 0, 0, 0};
                if (b0 + lane < c.B) its = tree_seq<ROWS>(c, a, b0 + lane);
            }
            own = ((uint32_t)its.units + most - 1) / most;
            count = own * (uint32_t)its.tiles * (uint32_t)c.H;
            before = wave_scan(count);
            found = __ballot(base + before > part);
            if (found) break;
            base += __builtin_amdgcn_readlane(before, 63);
        }
        if (!found) return;
        const int k = __ffsll((long long)found) - 1;
        const int b = b0 + k;
        const int t0 = __builtin_amdgcn_readlane(its.t0, k), n = __builtin_amdgcn_readlane(its.n, k);
        const int32_t past = __builtin_amdgcn_readlane(its.past, k);
        const int32_t units = __builtin_amdgcn_readlane(its.units, k);
        const uint32_t tiles = __builtin_amdgcn_readlane(its.tiles, k);
        const uint32_t pieces = __builtin_amdgcn_readlane(own, k);
        const uint64_t start = base + __builtin_amdgcn_readlane(before - count, k);
        const TreePlace place = tree_place((uint32_t)(part - start), pieces * (uint32_t)c.H, tiles);
        const uint32_t pair = place.pair, tile = place.tile;
        const int h = (int)(pair / pieces), piece = (int)(pair % pieces);
        const uint64_t seg = start + ((uint64_t)h * tiles + tile) * pieces;     // the segment's first part as its sums lie

        const Span span = span_of(c, a, past, n);
        // the first `units % pieces` parts are a unit longer
        const int32_t len = (int32_t)((uint32_t)units / pieces), more = units - len * (int32_t)pieces;
        const int32_t u0 = piece * len + min(piece, more), u1 = u0 + len + (piece < more ? 1 : 0);
        const int r0 = (int)tile * ROWS, rows = min(n * a.G - r0, ROWS);

        // A wave's blocks, two a step: their pages and scales 32 steps at a time, lane 2 i + e holding block e of step i.
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
            const int row = threadIdx.x / PER, j = threadIdx.x % PER;
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
        // the lane's rows: what they see of the cache, and of the new tokens
        int32_t pos[NR];
        const uint64_t* mask[NR];
        float s2[NR];
        int32_t pos_max = past;
#pragma unroll
        for (int g = 0; g < NR; ++g) {
            const int t = t0 + (r0 + min(g * 32 + col, rows - 1)) / a.G;
            pos[g] = a.window > 0 ? min(max(a.pos[t], past), kMaxPast) : past;
            mask[g] = a.mask + (int64_t)t * a.words;
            pos_max = max(pos_max, pos[g]);
        }
        if (a.window > 0)
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) pos_max = max(pos_max, __shfl_xor(pos_max, o));
        __syncthreads();
#pragma unroll
        for (int g = 0; g < NR; ++g) s2[g] = fabsf(a.scale2) * lds.undo[g * 32 + col];

        // blocks (of the span) that all rows see whole, but for the sinks
        const int32_t base_i = span.n_sink - span.win;
        const int32_t full_lo = a.window > 0 ? max(span.n_sink, ((pos_max - a.window + 16) >> 4) + base_i) : 0;
        const int32_t full_hi = (past >> 4) + base_i;        // not itself

        // Codes of a step: keys [64 dimensions][32 of them], values [token block][64 or 128 dimensions][token groups hi and hi + 2]
        struct Raw {
            uint4v k[ND][2];
            uint4v v[2][ND == 4 ? 2 : 1][2];
        };
        auto fetch_k = [&](int i, int32_t pages, Raw& r) {
            const int32_t p0 = __builtin_amdgcn_readlane(pages, (i & 31) * 2), p1 = __builtin_amdgcn_readlane(pages, (i & 31) * 2 + 1);
            const int64_t at0 = blocks.at(p0, span.tile(tile_of(i, 0))), at1 = blocks.at(p1, span.tile(tile_of(i, 1)));
            const uint8_t* p = blocks.k + (lane & 16 ? at1 : at0) + (lane & 15) * 64 + hi * 16;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int j = 0; j < 2; ++j) r.k[d][j] = *reinterpret_cast<const uint4v*>(p + d * 1024 + j * 32);
        };
        auto fetch_v = [&](int i, int32_t pages, Raw& r) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int32_t page = __builtin_amdgcn_readlane(pages, (i & 31) * 2 + e);
                const uint8_t* p = blocks.v + blocks.at(page, span.tile(tile_of(i, e)));
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
        // pages of the steps whose codes are fetched; of those that are computed, with their scales
        int32_t ahead = checked(first_pages, 0), pages = ahead, pages_next = -1;
        float ks = load_scale(blocks.ks, pages), vs = load_scale(blocks.vs, pages), ks_next = 1.0f, vs_next = 1.0f;
        Raw raw;
        fetch_k(0, ahead, raw);
        fetch_v(0, ahead, raw);
        for (int i = 0; i < steps; ++i) {
            if (((i + 1) & 31) == 0) {
                ahead = checked(later, i + 1);
                later = load_pages(i + 33);
                pages_next = ahead;
                ks_next = load_scale(blocks.ks, ahead);
                vs_next = load_scale(blocks.vs, ahead);
            }
            if (i > 0 && (i & 31) == 0) {
                pages = pages_next;
                ks = ks_next;
                vs = vs_next;
            }
            float16v s[NR] = {};
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const half8 key = code_halves8<FP8>(raw.k[d][j][2 * p], raw.k[d][j][2 * p + 1]);
#pragma unroll
                        for (int g = 0; g < NR; ++g)
                            s[g] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                                key, __builtin_bit_cast(half8, lds.q[(d * 2 + j) * 2 + p][g][lane]), s[g], 0, 0, 0);
                    }
            fetch_k(i + 1, ahead, raw);
            const int i0 = tile_of(i, 0);
            float f[2], log_scale[2], inv_scale[2];
            int32_t there[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int l = (i & 31) * 2 + e;
                there[e] = __builtin_amdgcn_readlane(pages, l);
                const float b = of_lane(vs, l);
                f[e] = of_lane(ks, l);
                log_scale[e] = __builtin_amdgcn_logf(b);
                inv_scale[e] = __builtin_amdgcn_rcpf(b);
            }
            const bool masked = ((there[0] | there[1]) < 0) | (i0 < full_lo) | (i0 + 1 >= full_hi);
            if (masked) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int32_t tok = span.tile(i0 + e) * 16;
                    uint32_t any = 0;
#pragma unroll
                    for (int g = 0; g < NR; ++g) {
                        uint32_t seen = there[e] >= 0 ? tree_sight(a, mask[g], past, n, pos[g], tok) : 0u;
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
                }
            fetch_v(i + 1, ahead, raw);
        }

        // the four waves' sums, 64 dimensions at a time; then a thread has 2 or 4 NR of them, side by side in a row
        float f_wave[NR];
#pragma unroll
        for (int g = 0; g < NR; ++g) {
            l_run[g] += __shfl_xor(l_run[g], 32);
            if (hi == 0) lds.ml[wave][g * 32 + col] = float2v{m_run[g], l_run[g]};
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < NR; ++g) {
            float m_all = kNoMax;
#pragma unroll
            for (int w = 0; w < 4; ++w) m_all = fmaxf(m_all, lds.ml[w][g * 32 + col].x);
            f_wave[g] = __builtin_amdgcn_exp2f(m_run[g] - m_all);
        }
        constexpr int PER = 8 / NR, W = 64 / PER;            // threads of a row, and their dimensions of 64
        const int row = threadIdx.x / PER, d0 = (threadIdx.x % PER) * W;
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
                float* to = lds.comb[wave][g * 32 + col];
                if constexpr (D == 64) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        *reinterpret_cast<float2v*>(to + dim_of<D>(i, hi)) = float2v{o[g][0][i], o[g][1][i]} * f_wave[g];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int k = (d & 1) * 8 + i;
                        *reinterpret_cast<float4v*>(to + dim_of<D>(k, hi)) =
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

        bool last = true;
        if (pieces > 1) {
            auto put = [&](uint64_t slot) {
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
            // adds n parts, `step` apart from `first`, in their order
            auto add = [&](uint64_t first, int step, int n) {
                if (row >= rows) return;
                m_row = kNoMax;
                l_row = 0.0f;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int j = 0; j < W / 4; ++j) sums[d][j] = float4v{0, 0, 0, 0};
                for (int i = 0; i < n; ++i) {
                    const int64_t at = (int64_t)(first + (uint64_t)i * step) * ROWS + row;
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
            // Parts are added in groups of kJoin: whoever finishes a group's last part adds the group's parts, whoever
            // finishes the last group adds the groups' sums; always in the order of the parts.
            const int gr = piece / kJoin, members = min(kJoin, (int)pieces - gr * kJoin), groups = ((int)pieces - 1) / kJoin + 1;
            const uint64_t lead = seg + (uint32_t)gr * kJoin;        // the group's first part
            put(seg + (uint32_t)piece);
            last = arrive(a.arrived + lead * 2, members);
            if (last) {
                add(lead, 1, members);
                if (groups > 1) {
                    // the group's sum in the place of its first part, which all of the workgroup has read
                    __syncthreads();
                    put(lead);
                    last = arrive(a.arrived + seg * 2 + 1, groups);
                    if (last) add(seg, kJoin, groups);
                }
            }
        }
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
    // tiles of 32 rows where no tree has more, or where the sums of 64 would not fit the registers
    const int rows = c.D == 256 || (int64_t)c.max_new * a.G <= 32 ? 32 : 64;
    WsCarve ws{(char*)workspace, (size_t)workspace_bytes};
    a.arrived = ws.take<uint32_t>(kMaxParts * 2);
    // as many parts as workgroups fit the device, and 2.5 for each segment where that is more; segments stay whole
    // where the workspace does not hold that many parts
    const int64_t segments = ((int64_t)c.T * a.G / rows + c.B) * c.H, fit = (int64_t)n_cu * 2;
    if (segments >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    const int64_t room = std::min<int64_t>((workspace_bytes - (int64_t)ws.off - 1024) / (rows * (c.D + 2) * 4), kMaxParts);
    const bool cut = segments * 3 <= room * 2;
    const int64_t wgs = cut ? std::min(std::max(fit, segments * 5 / 2), room) : std::min<int64_t>(segments, 1 << 20);
    if (cut) {
        a.part_ml = ws.take<float2v>(wgs * rows);
        a.part_o = ws.take<float>(wgs * rows * c.D);
    }
    if (!ws.ok()) return hipErrorInvalidConfiguration;
    auto run = [&](auto d, auto fp8, auto nr) {
        kv_tree_kernel<decltype(d)::value, decltype(fp8)::value, decltype(nr)::value><<<(uint32_t)wgs, 256, 0, s>>>(c, a, cut);
        return hipGetLastError();
    };
    auto by_rows = [&](auto d, auto fp8) {
        if constexpr (decltype(d)::value != 256)
            if (rows == 64) return run(d, fp8, std::integral_constant<int, 2>{});
        return run(d, fp8, std::integral_constant<int, 1>{});
    };
    auto by_dim = [&](auto fp8) {
        if (c.D == 64) return by_rows(std::integral_constant<int, 64>{}, fp8);
        if (c.D == 128) return by_rows(std::integral_constant<int, 128>{}, fp8);
        return by_rows(std::integral_constant<int, 256>{}, fp8);
    };
    return c.fp8 ? by_dim(std::true_type{}) : by_dim(std::false_type{});
}

}  // namespace ls
