// Attention over the paged 8-bit KV cache (k_kv.h).
//
// out_i = sum_j softmax_j(scale q_i . k_j) v_j over the tokens j that row i sees.
//
// With key scale a_j and value scale b_j of token j's page and head, and codes
// K_j, V_j, the row's weights are carried as w_j = b_j 2^(x_j - m), x_j the
// base-2 logit, so that the value scales enter through x_j + log2 b_j and V_j stays
// as stored:
//   out = sum_j w_j V_j / sum_j (w_j / b_j).
// m is any reference, not only the maximum.  w_j enters the product in half
// precision, 11 bits from 2^-14 on; codes and 16-bit queries are exact there, a
// bf16 query after scaling its row by a power of two.  m therefore follows the
// weights of the tokens at hand: it moves up before one of them does not fit, and
// down where all of them are small (a first token that takes nearly all weight and
// has values near zero must not cost the others their bits).  m, the sums and the
// products are fp32.
#include <algorithm>

#include "k_kv_attend.h"
#include "ls_scratch.h"

namespace ls {
namespace {

struct AttnArgs : AttnCall {
    int32_t few;                     // sequences with up to this many rows (new tokens x G) split along the keys
    // segments (sequence, kv head) that are cut: sums of each part, and counts of those that are there
    float* part_o;                   // [parts][16][D]
    float2v* part_ml;                // [parts][16] running maximum and sum
    uint32_t* arrived;               // [parts][2], zero between launches
    // tiles of many rows whose tokens several workgroups share: [tile][share][kTileRows]
    float* tile_o;
    float2v* tile_ml;
};

constexpr int kFewRows = 16;         // rows of a kv head that split_part takes
// Workgroups of kv_split_kernel on a compute unit, by its registers.
template <int D>
constexpr int kSplitPerCu = D == 64 ? 4 : D == 128 ? 2 : 1;
// A sequence of the call as split_part sees it; units of one kv head, 0: too many rows for it.
struct Seq {
    int32_t t0, n, past, units;
};
__device__ __forceinline__ Seq seq_of(const KvView& c, const AttnArgs& a, int b) {
    Seq s;
    seq_rows(c, b, s.t0, s.n);
    s.past = past_of(c, b);
    s.units = 0;
    if (s.n != 0 && (int64_t)s.n * a.G <= a.few)
        s.units = max((span_of(c, a, s.past, s.n).n + kUnit - 1) / kUnit, 1);
    return s;
}

// Rows of a kv head (new token, then query head) as 16 columns: a column's query
// in half precision, scaled by a power of two for bf16, in the lanes' shares of
// the 16x16x32 product's second operand.  Returns what undoes the scaling.
template <int D, bool F16>
__device__ __forceinline__ float load_queries(const AttnArgs& a, int D_heads_h, int t0, int col, int rows,
                                              half8 (&q)[D / 64][2]) {
    const int g = (threadIdx.x & 63) >> 4;
    uint4v raw[D / 64][2];
    const uint16_t* p = a.q + (int64_t)(t0 + col / a.G) * a.q_stride + ((int64_t)D_heads_h * a.G + col % a.G) * D + g * 16;
#pragma unroll
    for (int dt = 0; dt < D / 64; ++dt)
#pragma unroll
        for (int s = 0; s < 2; ++s)
            raw[dt][s] = col < rows ? *reinterpret_cast<const uint4v*>(p + dt * 64 + s * 8) : uint4v{0, 0, 0, 0};
    if constexpr (F16) {
#pragma unroll
        for (int dt = 0; dt < D / 64; ++dt)
#pragma unroll
            for (int s = 0; s < 2; ++s) q[dt][s] = __builtin_bit_cast(half8, raw[dt][s]);
        return 1.0f;
    } else {
        uint32_t top = 0;            // largest magnitude, as bits: the exponent decides
#pragma unroll
        for (int dt = 0; dt < D / 64; ++dt)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    top = max(top, max((raw[dt][s][i] << 16) & 0x7FFFFFFFu, raw[dt][s][i] & 0x7FFF0000u));
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const float f = half_range_factor(top);
#pragma unroll
        for (int dt = 0; dt < D / 64; ++dt)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2v x = unpack2<false>(raw[dt][s][i]);
                    q[dt][s][2 * i] = (_Float16)(x.x * f);
                    q[dt][s][2 * i + 1] = (_Float16)(x.y * f);
                }
        return half_range_undo(top);
    }
}

// Partial sums of a segment's 16 rows: a thread holds dimensions d0 .. d0 + 3 of
// every 64 of a row.
template <int D>
__device__ __forceinline__ void put_part(const AttnArgs& a, int64_t part, int row, int d0, int rows,
                                         const float4v (&v)[D / 64], float m, float l) {
    if (row >= rows) return;
    const int64_t at = part * kFewRows + row;
#pragma unroll
    for (int dt = 0; dt < D / 64; ++dt) {
        put_shared(a.part_o + at * D + dt * 64 + d0, float2v{v[dt].x, v[dt].y});
        put_shared(a.part_o + at * D + dt * 64 + d0 + 2, float2v{v[dt].z, v[dt].w});
    }
    if (d0 == 0) put_shared((float*)&a.part_ml[at], float2v{m, l});
}

// Adds n parts, `step` apart from `first`, in their order; eight are read at a time.
template <int D>
__device__ __forceinline__ void add_parts(const AttnArgs& a, uint32_t first, int step, int n, int row, int d0, int rows,
                                          float4v (&v)[D / 64], float& m, float& l) {
    constexpr int kAtOnce = D == 256 ? 4 : 8;
    if (row >= rows) return;
    m = kNoMax;
    l = 0.0f;
#pragma unroll
    for (int dt = 0; dt < D / 64; ++dt) v[dt] = float4v{0, 0, 0, 0};
    for (int i0 = 0; i0 < n; i0 += kAtOnce) {
        float2v ml[kAtOnce], x[kAtOnce][D / 64][2];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int64_t at = ((int64_t)first + (int64_t)min(i0 + i, n - 1) * step) * kFewRows + row;
            ml[i] = get_shared((const float*)&a.part_ml[at]);
#pragma unroll
            for (int dt = 0; dt < D / 64; ++dt) {
                x[i][dt][0] = get_shared(a.part_o + at * D + dt * 64 + d0);
                x[i][dt][1] = get_shared(a.part_o + at * D + dt * 64 + d0 + 2);
            }
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, ml[i].x);
        const float f = __builtin_amdgcn_exp2f(m - top);
        m = top;
        l *= f;
#pragma unroll
        for (int dt = 0; dt < D / 64; ++dt) v[dt] *= f;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const float e = i0 + i < n ? __builtin_amdgcn_exp2f(ml[i].x - m) : 0.0f;
            l = fmaf(ml[i].y, e, l);
#pragma unroll
            for (int dt = 0; dt < D / 64; ++dt)
                v[dt] += float4v{x[i][dt][0].x, x[i][dt][0].y, x[i][dt][1].x, x[i][dt][1].y} * e;
        }
    }
}

// Few rows (up to 16 of a kv head) against a long cache: bound by HBM.  The
// sequences' heads are cut into parts of about equal length, a workgroup each; a
// segment (sequence, head) of one part is finished there, the others leave partial
// sums, which the last workgroup to finish adds.  A wave takes 32 of a unit's 128
// tokens at a time: scores transposed (tokens x rows), so that their registers are
// the second operand of the product with the values as they stand; codes go from
// memory to registers in 16-byte loads, two steps ahead of their use.  Measured: 64
// sequences of 105k tokens in all, 8 kv heads of 128: 50.9 us, 4.25 TB/s; 4 sequences of
// 281k tokens 115 us, 5.0 TB/s (a large copy: 4.8); 1 sequence of 300 tokens 8.0 us.
template <int D>
struct SplitLds {
    float comb[4][16][D + 4];
    float2v ml[4][16];
};
template <int D, bool FP8, bool F16>
__device__ __forceinline__ void split_part(const KvView& c, const AttnArgs& a, bool cut, uint32_t block, uint32_t blocks_,
                                           SplitLds<D>& lds) {
    constexpr int ND = D / 64;
    auto& comb = lds.comb;
    auto& ml = lds.ml;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;

    // Segments are cut into equal parts of at most `most` units, so that about as many parts as workgroups hold all units and a
    // long sequence weighs no more on one workgroup than its share (not cut: a part is a segment, found at once).
    uint32_t most = ~0u;
    Seq mine;                            // of the first 64 sequences, a lane each
    if (cut) {
        mine.units = 0;
        if (lane < c.B) mine = seq_of(c, a, lane);
        uint64_t all = __builtin_amdgcn_readlane(wave_scan((uint32_t)mine.units), 63);      // below 2^23 each
        for (int b0 = 64; b0 < c.B; b0 += 64)
            all += __builtin_amdgcn_readlane(wave_scan(b0 + lane < c.B ? (uint32_t)seq_of(c, a, b0 + lane).units : 0u), 63);
        all *= (uint32_t)c.H;
        const uint32_t room = blocks_ - (uint32_t)(c.B * c.H);
        // 2^24 units and more, the largest segment, cut nothing
        const uint64_t each = all >> 31 ? (all + room - 1) / room : ((uint32_t)all + room - 1) / room;
        most = (uint32_t)min(max(each, (uint64_t)kMinUnits), (uint64_t)1 << 24);
    }
    for (uint32_t part = block;; part += blocks_) {
        Seq seq;
        int b = 0, h, piece = 0, pieces = 1;
        uint32_t seg = part;             // first part of the segment
        if (cut) {
            // sequences' first parts are the sums of the parts before them
            uint32_t base = 0, own = 0, end = 0;
            uint64_t m = 0;
            Seq its = mine;
            int b0 = 0;
            for (; b0 < c.B; b0 += 64) {
                if (b0 > 0) {
                    its.units = 0;
                    if (b0 + lane < c.B) its = seq_of(c, a, b0 + lane);
                }
                own = ((uint32_t)its.units + most - 1) / most;
                end = base + wave_scan(own * (uint32_t)c.H);
                m = __ballot(end > part);
                if (m) break;
                base = __builtin_amdgcn_readlane(end, 63);
            }
            if (!m) return;
            const int k = __ffsll((long long)m) - 1;
            b = b0 + k;
            seq.t0 = __builtin_amdgcn_readlane(its.t0, k);
            seq.n = __builtin_amdgcn_readlane(its.n, k);
            seq.past = __builtin_amdgcn_readlane(its.past, k);
            seq.units = __builtin_amdgcn_readlane(its.units, k);
            pieces = __builtin_amdgcn_readlane(own, k);
            const uint32_t start = __builtin_amdgcn_readlane(end, k) - (uint32_t)pieces * c.H;
            h = (int)((part - start) / (uint32_t)pieces);
            seg = start + (uint32_t)h * pieces;
            piece = (int)(part - seg);
        } else {
            if (part >= (uint32_t)(c.B * c.H)) return;
            b = (int)(part / (uint32_t)c.H);
            h = (int)(part % (uint32_t)c.H);
            seq = seq_of(c, a, b);
            if (seq.units == 0) continue;
        }
        const int t0 = seq.t0, n = seq.n;
        const int32_t past = seq.past;
        const Span span = span_of(c, a, past, n);
        const int32_t end_tok = min(past + n, c.limit);
        // the first `seq.units % pieces` parts are a unit longer
        const int32_t len = (int32_t)((uint32_t)seq.units / (uint32_t)pieces), more = seq.units - len * pieces;
        const int32_t u0 = piece * len + min(piece, more), u1 = u0 + len + (piece < more ? 1 : 0);
        const int rows = n * a.G;
        const int32_t pos = past + col / a.G;                // the column's position
        const int32_t pos_last = past + n - 1;

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

        half8 q[ND][2];
        const float s2 = a.scale2 * load_queries<D, F16>(a, h, t0, col, rows, q);

        // blocks (of the span) that all rows see whole, but for the sinks
        const int32_t base_i = span.n_sink - span.win;
        const int32_t full_lo = a.window > 0 ? max(span.n_sink, ((pos_last - a.window + 16) >> 4) + base_i) : 0;
        const int32_t full_hi = ((past - 15) >> 4) + base_i;

        struct Raw { uint4v k[2][ND], v[2][ND]; };
        // codes of step i (of page 0 for an absent block: hidden from the sums)
        auto fetch = [&](int i, int32_t pages, const uint8_t* codes, uint32_t lane_at, uint4v (&r)[2][ND]) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int32_t page = __builtin_amdgcn_readlane(pages, (i & 31) * 2 + e);
                const uint8_t* p = codes + blocks.at(page, span.tile(tile_of(i, e)));
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) r[e][dt] = *reinterpret_cast<const uint4v*>(p + lane_at + dt * 1024);
            }
        };
        auto fetch_k = [&](int i, int32_t pages, Raw& r) { fetch(i, pages, blocks.k, col * 64 + g * 16, r.k); };
        auto fetch_v = [&](int i, int32_t pages, Raw& r) { fetch(i, pages, blocks.v, lane * 16, r.v); };
        float m_run = kNoMax, l_run = 0.0f;
        float4v o[ND][4] = {};
        // pages of the steps whose codes are fetched; of those that are computed, with their scales
        int32_t ahead = checked(first_pages, 0), pages = ahead, pages_next = -1;
        float ks = load_scale(blocks.ks, pages), vs = load_scale(blocks.vs, pages), ks_next = 1.0f, vs_next = 1.0f;
        // One step; the codes of step i + 2 go into the registers that it has read.
        auto step = [&](int i, Raw& r) {
            float4v s[2] = {};
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        s[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                            code_halves8<FP8>(r.k[e][dt][2 * k], r.k[e][dt][2 * k + 1]), q[dt][k], s[e], 0, 0, 0);
            fetch_k(i + 2, ahead, r);
            float f[2], lv[2], iv[2];
            const int i0 = tile_of(i, 0);
            int32_t there[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int l = (i & 31) * 2 + e;
                there[e] = __builtin_amdgcn_readlane(pages, l);
                const float b = of_lane(vs, l);
                f[e] = of_lane(ks, l) * s2;
                lv[e] = __builtin_amdgcn_logf(b);
                iv[e] = __builtin_amdgcn_rcpf(b);
            }
            float x[2][4];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k) x[e][k] = fmaf(s[e][k], f[e], lv[e]);
            const bool masked = ((there[0] | there[1]) < 0) | (i0 < full_lo) | (i0 + 1 > full_hi);
            if (masked) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int32_t tok = span.tile(i0 + e) * 16;
                    const Sight see = sight(a, there[e], pos, tok);
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[e][k] = see.sees(4 * g + k) ? x[e][k] : -INFINITY;
                    const uint32_t keep = there[e] >= 0 ? kept_bytes(a, tok + 4 * g, max(past + 1 - a.window, 0), end_tok) : 0u;
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) r.v[e][dt] &= keep;
                }
            }
            half8 p;
            float sum[2];
            auto weigh = [&] {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        w[k] = __builtin_amdgcn_exp2f(x[e][k] - m_run);
                        p[4 * e + k] = (_Float16)w[k];
                    }
                    sum[e] = (w[0] + w[1]) + (w[2] + w[3]);
                }
            };
            weigh();
            if (__any(off_range(sum[0] + sum[1], masked))) {
                float mx = -INFINITY;
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int k = 0; k < 4; ++k) mx = fmaxf(mx, x[e][k]);
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                float to = raised(m_run, mx, kSplitTop);
                const bool low = is_low(m_run, mx, masked);
                if (__any(low)) {
                    float most = l_run;
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(o[dt][k][i]));
                    most = fmaxf(most, __shfl_xor(most, 16));
                    most = fmaxf(most, __shfl_xor(most, 32));
                    to = low ? lowered(m_run, mx, most) : to;
                }
                const float by = __builtin_amdgcn_exp2f(m_run - to);
                m_run = to;
                l_run *= by;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[dt][k] *= by;
                weigh();
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) l_run = fmaf(sum[e], iv[e], l_run);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    o[dt][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(code_halves8<FP8>(r.v[0][dt][k], r.v[1][dt][k]), p,
                                                                      o[dt][k], 0, 0, 0);
            fetch_v(i + 2, ahead, r);
        };
        Raw r0, r1;
        fetch_k(0, ahead, r0);
        fetch_v(0, ahead, r0);
        fetch_k(1, ahead, r1);
        fetch_v(1, ahead, r1);
        for (int i = 0; i < steps; i += 2) {
            if (((i + 2) & 31) == 0) {
                ahead = checked(later, i + 2);
                later = load_pages(i + 34);
                pages_next = ahead;
                ks_next = load_scale(blocks.ks, ahead);
                vs_next = load_scale(blocks.vs, ahead);
            }
            if (i > 0 && (i & 31) == 0) {
                pages = pages_next;
                ks = ks_next;
                vs = vs_next;
            }
            step(i, r0);
            step(i + 1, r1);
        }

        // the four waves' sums
        l_run += __shfl_xor(l_run, 16);
        l_run += __shfl_xor(l_run, 32);
        if (g == 0) ml[wave][col] = float2v{m_run, l_run};
        __syncthreads();
        float m_all = kNoMax;
#pragma unroll
        for (int w = 0; w < 4; ++w) m_all = fmaxf(m_all, ml[w][col].x);
        const float f = __builtin_amdgcn_exp2f(m_run - m_all);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<float4v*>(&comb[wave][col][dt * 64 + g * 16 + 4 * r]) =
                    float4v{o[dt][0][r], o[dt][1][r], o[dt][2][r], o[dt][3][r]} * f;
        __syncthreads();
        const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * 4;
        float m_row = kNoMax, l_row = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) m_row = fmaxf(m_row, ml[w][row].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) l_row = fmaf(ml[w][row].y, __builtin_amdgcn_exp2f(ml[w][row].x - m_row), l_row);
        float4v v[ND];
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            v[dt] = *reinterpret_cast<const float4v*>(&comb[0][row][dt * 64 + d0]);
#pragma unroll
            for (int w = 1; w < 4; ++w) v[dt] += *reinterpret_cast<const float4v*>(&comb[w][row][dt * 64 + d0]);
        }
        bool last = true;
        if (pieces > 1) {
            // Parts are added in groups of kJoin: whoever finishes a group's last part adds the group's parts,
            // whoever finishes the last group adds the groups' sums; always in the order of the parts.
            const int gr = piece / kJoin, members = min(kJoin, pieces - gr * kJoin), groups = (pieces - 1) / kJoin + 1;
            const uint32_t lead = seg + (uint32_t)gr * kJoin;        // the group's first part
            put_part<D>(a, part, row, d0, rows, v, m_row, l_row);
            last = arrive(a.arrived + (int64_t)lead * 2, members);
            if (last) {
                add_parts<D>(a, lead, 1, members, row, d0, rows, v, m_row, l_row);
                if (groups > 1) {
                    // the group's sum in the place of its first part, which all of the workgroup has read
                    __syncthreads();
                    put_part<D>(a, lead, row, d0, rows, v, m_row, l_row);
                    last = arrive(a.arrived + (int64_t)seg * 2 + 1, groups);
                    if (last) add_parts<D>(a, seg, kJoin, groups, row, d0, rows, v, m_row, l_row);
                }
            }
        }
        if (last && row < rows) {
            const float norm = l_row > 0.0f ? 1.0f / l_row : 0.0f;
            uint16_t* out = a.out + (int64_t)(t0 + row / a.G) * a.out_stride + ((int64_t)h * a.G + row % a.G) * D;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
                *reinterpret_cast<uint2v*>(out + dt * 64 + d0) =
                    uint2v{pack2<F16>(v[dt].x * norm, v[dt].y * norm), pack2<F16>(v[dt].z * norm, v[dt].w * norm)};
        }
        __syncthreads();

    }
}

// Many rows (prompts): bound by the matrix cores and the exponentials.  A
// workgroup takes kTileRows rows (new tokens x query heads of one kv head, so
// that the group's heads share what is staged) and walks the cache 64 tokens at a
// time: codes become halves on their way into LDS, in the order in which the
// 32x32x16 products read them (a wave's operand is 1 KB in a row, no bank is hit
// twice), double-buffered, with the next codes in flight.  Scores are transposed
// (tokens x rows): their registers are the second operand of the product with the
// values.  Few tiles: `splits` workgroups share a tile's tokens and
// kv_tile_join_kernel adds their sums.  Measured: prompts of 6.9k and 6.4k tokens, 32
// query heads of 128: 1.34 to 1.45 ms, 880 to 950 TFLOP/s (a large half-precision
// product: 1,290), the matrix pipe busy for 43 % of the time; 3 prompts of 64 dimensions
// under a window of 1,024: 125 to 133 us, 440 to 470 TFLOP/s.
constexpr int kTileRows = 128;

using float16v = float __attribute__((ext_vector_type(16)));

// What a tile's rows [r0, r0 + rows) of sequence b see, 64 tokens a step; the share of split `sp` of `splits`.
struct TileWork {
    Span span;
    int32_t u0, u1, shares;
};
__device__ __forceinline__ TileWork tile_work(const KvView& c, const AttnArgs& a, int32_t past, int r0, int rows,
                                              int sp, int splits) {
    const int tok0 = r0 / a.G, tok1 = (r0 + rows - 1) / a.G;
    TileWork w;
    w.span = span_of(c, a, past + tok0, tok1 - tok0 + 1);
    const int steps = (w.span.n + 3) >> 2;
    w.shares = min(splits, max(steps >> 2, 1));      // no share below four steps
    w.u0 = sp < w.shares ? (int)((int64_t)steps * sp / w.shares) : 0;
    w.u1 = sp < w.shares ? (int)((int64_t)steps * (sp + 1) / w.shares) : 0;
    return w;
}

// The tile of slot `slot`: sequence, its rows' start and count (0: none, or few enough for split_part).
__device__ __forceinline__ int tile_of_slot(const KvView& c, const AttnArgs& a, int64_t slot, int& b, int& t0, int& r0) {
    const int G = a.G;
    auto first = [G](int off, int b) { return tile_slot(off, b, G, kTileRows); };
    b = seq_of_slot(c, slot, first);
    int n;
    seq_rows(c, b, t0, n);
    const TileRows its = tile_rows(slot - first(t0, b), n, G, kTileRows);
    r0 = (int)its.r0;
    return (int64_t)n * G <= a.few ? 0 : its.rows;
}

template <int D>
struct TileLds {
    uint4v k[2][2][D / 16][64];              // keys: [buffer][32 tokens][16 dimensions][lane]
    uint4v v[2][4][D / 32][64];              // values: [buffer][16 tokens][32 dimensions][lane]
};
template <int D, bool FP8, bool F16>
__device__ __forceinline__ void tile_part(const KvView& c, const AttnArgs& a, int64_t n_slots, int32_t splits, uint32_t block,
                                          TileLds<D>& lds) {
    constexpr int ND = D / 64, NK = D / 16, NV = D / 32;
    auto& lk = lds.k;
    auto& lv = lds.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, hi = lane >> 5;
    const int h = block % c.H;
    const int sp = (int)((block / c.H) % splits);
    const int64_t slot = n_slots - 1 - block / c.H / splits;     // a sequence's last rows see most: first
    int b, t0, r0;
    const int rows = tile_of_slot(c, a, slot, b, t0, r0);
    if (rows == 0) return;
    const int32_t past = past_of(c, b);
    const TileWork work = tile_work(c, a, past, r0, rows, sp, splits);
    const Span span = work.span;
    if (sp >= work.shares) return;
    int n_all, t_;
    seq_rows(c, b, t_, n_all);
    const int32_t end_tok = min(past + n_all, c.limit), lo_tok = a.window > 0 ? max(past + r0 / a.G + 1 - a.window, 0) : 0;

    // this wave's rows and the positions they span
    const int w0 = wave * 32, wrows = min(max(rows - w0, 0), 32);
    const int row = r0 + w0 + col;
    const int32_t pos = past + row / a.G;
    const int32_t pos_min = past + (r0 + w0) / a.G, pos_max = past + (r0 + w0 + max(wrows, 1) - 1) / a.G;

    half8 q[NK];
    float s2 = fabsf(a.scale2);
    {
        uint4v raw[NK];
        const uint16_t* p = a.q + (int64_t)(t0 + row / a.G) * a.q_stride + ((int64_t)h * a.G + row % a.G) * D + hi * 8;
        const uint32_t flip = a.scale2 < 0.0f ? 0x80008000u : 0u;
#pragma unroll
        for (int s = 0; s < NK; ++s)
            raw[s] = (col < wrows ? *reinterpret_cast<const uint4v*>(p + s * 16) : uint4v{0, 0, 0, 0}) ^ flip;
        if constexpr (F16) {
#pragma unroll
            for (int s = 0; s < NK; ++s) q[s] = __builtin_bit_cast(half8, raw[s]);
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int s = 0; s < NK; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    top = max(top, max((raw[s][i] << 16) & 0x7FFFFFFFu, raw[s][i] & 0x7FFF0000u));
            top = max(top, (uint32_t)__shfl_xor((int)top, 32));
            const float f = half_range_factor(top);
#pragma unroll
            for (int s = 0; s < NK; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2v x = unpack2<false>(raw[s][i]);
                    q[s][2 * i] = (_Float16)(x.x * f);
                    q[s][2 * i + 1] = (_Float16)(x.y * f);
                }
            s2 *= half_range_undo(top);
        }
    }

    // Blocks (of the span) that all of the wave's rows see whole, but for the sinks, and that any row sees.
    const int32_t base_i = span.n_sink - span.win;
    const int32_t full_lo = a.window > 0 ? max(span.n_sink, ((pos_max - a.window + 16) >> 4) + base_i) : 0;
    const int32_t full_hi = ((pos_min - 15) >> 4) + base_i;
    const int32_t any_lo = a.window > 0 ? max(span.n_sink, ((pos_min - a.window + 1) >> 4) + base_i) : 0;
    const int32_t any_hi = (pos_max >> 4) + base_i;
    const int32_t sink_hi = a.window > 0 ? (min(a.sinks, c.limit) + 15) >> 4 : 0;

    // A step's four pages and eight scales are one register each: lane e holds block e's page, and its key scale, lane
    // 4 + e its value scale.
    const Blocks blocks(c, b, h);
    const int e4 = lane & 3;
    auto load_page = [&](int t) {
        return blocks.pages[min(span.tile(t * 4 + e4), blocks.n_blocks - 1) >> blocks.shift];
    };
    auto checked = [&](int32_t page, int t) {
        const bool there = (t < work.u1) & (t * 4 + e4 < span.n) & ((uint32_t)page < (uint32_t)blocks.n_pages);
        return there ? page : -1;
    };
    const float* scales = lane & 4 ? blocks.vs : blocks.ks;
    auto load_scale = [&](int32_t page) { return scales[(int64_t)max(page, 0) * blocks.H]; };
    auto of_lane = [](float x, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)); };

    // the wave's share of a step: block `wave` of the four
    uint4v rk[ND], rv[ND];
    int32_t kept = 0;                // block whose value codes are masked by token, -1: none are, -2: all are
    auto fetch = [&](int t, int32_t pages) {
        const int32_t page = __builtin_amdgcn_readlane(pages, wave);
        const int32_t blk = span.tile(t * 4 + wave);
        const int64_t base = blocks.at(page, blk);
        const uint8_t* kp = blocks.k + base;
        const uint8_t* vp = blocks.v + base;
        const uint32_t k_at = (lane & 15) * 64 + (lane >> 4) * 16, v_at = lane * 16;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            rk[dt] = *reinterpret_cast<const uint4v*>(kp + k_at + dt * 1024);
            rv[dt] = *reinterpret_cast<const uint4v*>(vp + v_at + dt * 1024);
        }
        const bool whole = (blk * 16 >= lo_tok) & (blk * 16 + 16 <= end_tok);
        kept = page < 0 ? -2 : whole ? -1 : blk;
    };
    auto stage = [&](int buf) {
        // keys: lane (token lane % 16, dimensions 16 (lane / 16) ..) holds both halves of a product step's operand
        const int kl = (wave & 1) * 16 + (lane & 15);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            uint4v* d = lk[buf][wave >> 1][dt * 4 + (lane >> 4)];
            d[kl] = __builtin_bit_cast(uint4v, code_halves8<FP8>(rk[dt][0], rk[dt][1]));
            d[32 + kl] = __builtin_bit_cast(uint4v, code_halves8<FP8>(rk[dt][2], rk[dt][3]));
        }
        // values: lanes 32 apart hold token groups g and g + 2 of four dimensions; after the exchange each holds both
        // groups of two dimensions, one operand register set each
        if (kept != -1) {
            const uint32_t keep = kept >= 0 ? kept_bytes(a, kept * 16 + (lane >> 4) * 4, lo_tok, end_tok) : 0u;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) rv[dt] &= keep;
        }
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            const auto x = __builtin_amdgcn_permlane32_swap(rv[dt][0], rv[dt][2], false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(rv[dt][1], rv[dt][3], false, false);
            uint4v* d = &lv[buf][wave][dt * 2 + hi][((lane >> 4) & 1) * 32 + (lane & 15)];
            d[0] = __builtin_bit_cast(uint4v, code_halves8<FP8>(x[0], x[1]));
            d[16] = __builtin_bit_cast(uint4v, code_halves8<FP8>(y[0], y[1]));
        }
    };

    float m_run = kNoMax, l_run = 0.0f;
    float16v o[NV] = {};
    // One step: scores, weights, product.  LDS reads are issued well before their products (the scheduling barriers keep
    // them there).
    auto compute = [&](int t, int buf, int32_t pages, float scale) {
        const uint32_t have = (uint32_t)__ballot(pages >= 0) & 15u;
        const int i0 = t * 4, i3 = i0 + 3;
        if ((wrows == 0) | (have == 0) | (i0 > any_hi) | ((i3 < any_lo) & (i0 >= sink_hi))) return;
        scale = pages >= 0 ? fmaxf(scale, kScaleMin) : 1.0f;
        const float log_scale = __builtin_amdgcn_logf(scale), inv_scale = __builtin_amdgcn_rcpf(scale);
        float16v s[2] = {};
        constexpr int KC = D == 256 ? 4 : NK, VC = D == 256 ? 1 : 2;     // products, and blocks, whose operands are read at once
#pragma unroll
        for (int k0 = 0; k0 < NK; k0 += KC) {
            uint4v kf[KC][2];
#pragma unroll
            for (int k = 0; k < KC; ++k)
#pragma unroll
                for (int g = 0; g < 2; ++g) kf[k][g] = lk[buf][g][k0 + k][lane];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < KC; ++k)
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    s[g] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, kf[k][g]), q[k0 + k], s[g], 0, 0, 0);
        }
        uint4v vf[2][VC][NV];                // values of VC blocks, twice
        auto read_values = [&](int e0) {
#pragma unroll
            for (int e = 0; e < VC; ++e)
#pragma unroll
                for (int i = 0; i < NV; ++i) vf[(e0 / VC) & 1][e][i] = lv[buf][e0 + e][i][lane];
        };
        read_values(0);
        __builtin_amdgcn_sched_barrier(0);
        const bool masked = (have != 15u) | (i0 < full_lo) | (i3 > full_hi);
        if (masked) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const Sight v = sight(a, have >> e & 1 ? 0 : -1, pos, span.tile(i0 + e) * 16);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float x = s[e >> 1][(e & 1) * 8 + i];
                    s[e >> 1][(e & 1) * 8 + i] = v.sees(8 * (i >> 2) + 4 * hi + (i & 3)) ? x : -INFINITY;
                }
            }
        }
        float f[4], sum[4];
        half8 p[4];
        // from the logits as they are rounded for the reference, or in one operation less: the same while a logit's last
        // bit is below 1, from 2^24 on too large or small by up to that bit
        auto weigh = [&](auto rounded) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float log = of_lane(log_scale, 4 + e), off = log - m_run;
                sum[e] = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float x = s[e >> 1][(e & 1) * 8 + i];
                    const float w = __builtin_amdgcn_exp2f(rounded ? fmaf(x, f[e], log) - m_run : fmaf(x, f[e], off));
                    sum[e] += w;
                    p[e][i] = (_Float16)w;
                }
            }
        };
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = fmaxf(of_lane(scale, e) * s2, 1e-37f);      // not 0: -inf of a hidden token stays
        weigh(std::false_type{});
        const float level = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        if (__any(off_range(level, masked))) {
            float mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float top = s[e >> 1][(e & 1) * 8];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, s[e >> 1][(e & 1) * 8 + i]);
                mx = fmaxf(mx, fmaf(top, f[e], of_lane(log_scale, 4 + e)));
            }
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            float to = raised(m_run, mx, kTileTop);
            const bool low = is_low(m_run, mx, masked);
            if (__any(low)) {
                float most = l_run;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) most = fmaxf(most, fabsf(o[i][k]));
                most = fmaxf(most, __shfl_xor(most, 32));
                to = low ? lowered(m_run, mx, most) : to;
            }
            if (__any((to != m_run) | (level > kMostWeight))) {
                const float by = __builtin_amdgcn_exp2f(m_run - to);
                m_run = to;
                l_run *= by;
#pragma unroll
                for (int i = 0; i < NV; ++i) o[i] *= by;
                weigh(std::true_type{});
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) l_run = fmaf(sum[e], of_lane(inv_scale, 4 + e), l_run);
#pragma unroll
        for (int e0 = 0; e0 < 4; e0 += VC) {
            if (e0 + VC < 4) read_values(e0 + VC);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < VC; ++e)
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, vf[(e0 / VC) & 1][e][i]),
                                                                  p[e0 + e], o[i], 0, 0, 0);
        }
    };

    // pages are looked up three steps ahead, codes and scales fetched two and codes staged one
    int32_t page0 = checked(load_page(work.u0), work.u0), page1 = checked(load_page(work.u0 + 1), work.u0 + 1);
    int32_t next = load_page(work.u0 + 2);
    float scale0 = load_scale(page0), scale1 = load_scale(page1);
    fetch(work.u0, page0);
    stage(work.u0 & 1);
    fetch(work.u0 + 1, page1);
    __syncthreads();
    for (int t = work.u0; t < work.u1; ++t) {
        // the other buffer's readers passed the barrier that ended the step before
        stage((t + 1) & 1);
        const int32_t page2 = checked(next, t + 2);
        next = load_page(t + 3);
        const float scale2 = load_scale(page2);
        fetch(t + 2, page2);
        compute(t, t & 1, page0, scale0);
        __syncthreads();
        page0 = page1;
        page1 = page2;
        scale0 = scale1;
        scale1 = scale2;
    }

    l_run += __shfl_xor(l_run, 32);
    if (col >= wrows) return;
    if (work.shares == 1) {
        const float norm = l_run > 0.0f ? 1.0f / l_run : 0.0f;
        uint16_t* out = a.out + (int64_t)(t0 + row / a.G) * a.out_stride + ((int64_t)h * a.G + row % a.G) * D;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        w[2 * i + e] = pack2<F16>(o[dt * 2 + e][4 * k + i] * norm, o[dt * 2 + e][8 + 4 * k + i] * norm);
                uint4v* d = reinterpret_cast<uint4v*>(out + dt * 64 + k * 32 + hi * 16);
                d[0] = uint4v{w[0], w[1], w[2], w[3]};
                d[1] = uint4v{w[4], w[5], w[6], w[7]};
            }
    } else {
        const int64_t at = (((slot * c.H + h) * splits + sp) * kTileRows + w0 + col);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float4v*>(a.tile_o + at * D + dt * 64 + k * 32 + hi * 16 + i * 4) =
                        float4v{o[dt * 2][4 * k + i], o[dt * 2][8 + 4 * k + i], o[dt * 2 + 1][4 * k + i],
                                o[dt * 2 + 1][8 + 4 * k + i]};
        if (hi == 0) a.tile_ml[at] = float2v{m_run, l_run};
    }
}

// A launch whose sequences all have few rows, and one of both kinds: the tiles'
// workgroups first, since they take longest, then the others', which fill the gaps.
template <int D, bool FP8, bool F16>
__global__ __launch_bounds__(256, kSplitPerCu<D>) void kv_split_kernel(KvView c, AttnArgs a, bool cut) {
    __shared__ SplitLds<D> lds;
    split_part<D, FP8, F16>(c, a, cut, blockIdx.x, gridDim.x, lds);
}

template <int D, bool FP8, bool F16>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void kv_mixed_kernel(KvView c, AttnArgs a, int64_t n_slots, int32_t splits,
                                                                         bool cut) {
    __shared__ union Lds {
        TileLds<D> tile;
        SplitLds<D> split;
        __device__ Lds() {}
    } lds;
    const uint32_t tiles = (uint32_t)(n_slots * c.H * splits);
    if (blockIdx.x < tiles)
        tile_part<D, FP8, F16>(c, a, n_slots, splits, blockIdx.x, lds.tile);
    else
        split_part<D, FP8, F16>(c, a, cut, blockIdx.x - tiles, gridDim.x - tiles, lds.split);
}

// Adds the partial sums of a tile's shares in their order: a workgroup for each
// eight rows of a tile and kv head.  Bound by latency: 8 us after a step of 4 chunks.
template <int D, bool F16>
__global__ __launch_bounds__(256) void kv_tile_join_kernel(KvView c, AttnArgs a, int32_t splits) {
    constexpr int kPieces = kTileRows / 8;
    const int piece = blockIdx.x % kPieces, h = (blockIdx.x / kPieces) % c.H;
    const int64_t slot = blockIdx.x / kPieces / c.H;
    int b, t0, r0;
    const int rows = tile_of_slot(c, a, slot, b, t0, r0);
    const int i = piece * 8 + (threadIdx.x >> 5), d0 = (threadIdx.x & 31) * (D / 32);
    if (i >= rows) return;
    const int shares = tile_work(c, a, past_of(c, b), r0, rows, 0, splits).shares;
    if (shares == 1) return;
    float m = kNoMax, l = 0.0f, v[D / 32] = {};
    for (int sp = 0; sp < shares; ++sp) {
        const int64_t at = ((slot * c.H + h) * splits + sp) * kTileRows + i;
        const float2v p = a.tile_ml[at];
        const float m2 = fmaxf(m, p.x);
        const float f = __builtin_amdgcn_exp2f(m - m2), e = __builtin_amdgcn_exp2f(p.x - m2);
        m = m2;
        l = l * f + p.y * e;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) v[k] = v[k] * f + a.tile_o[at * D + d0 + k] * e;
    }
    const float norm = l > 0.0f ? 1.0f / l : 0.0f;
    const int row = r0 + i;
    uint16_t* out = a.out + (int64_t)(t0 + row / a.G) * a.out_stride + ((int64_t)h * a.G + row % a.G) * D + d0;
#pragma unroll
    for (int k = 0; k < D / 32; k += 2) *reinterpret_cast<uint32_t*>(out + k) = pack2<F16>(v[k] * norm, v[k + 1] * norm);
}

// Shares of a tile: enough workgroups for two on every compute unit, where the
// workspace holds their sums (by slot, so that empty slots count: with 8 kv heads of
// 128 dimensions more than about 58 slots leave one share).  Which sequences have many rows
// is known on the device only; of k of them, at most max_new tokens each and the
// others one, k is put at its least (1.5 and 2 times that: the same within 2 % for 2 to 6
// chunks of equal and of unequal lengths).
int tile_splits(const KvView& c, const AttnArgs& a, int64_t slots, int n_cu, int64_t room) {
    const int64_t one = slots * c.H * kTileRows * (c.D + 2) * 4;
    const int64_t k = std::min<int64_t>(c.B, std::max(c.T - c.B, 0) / std::max(c.max_new - 1, 1) + 1);
    const int64_t tiles = std::max(k, (int64_t)c.T * a.G / kTileRows + k / 2) * c.H;
    return (int)std::max<int64_t>(1, std::min<int64_t>({(2 * (int64_t)n_cu + tiles - 1) / tiles, room / one, 64}));
}

}  // namespace

// The counts of a new workspace (the last of a segment's parts leaves them at zero).
__global__ void kv_clear_kernel(uint32_t* p, int n) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) p[i] = 0;
}

hipError_t launch_kv_workspace_init(void* workspace, hipStream_t s) {
    kv_clear_kernel<<<1, 256, 0, s>>>((uint32_t*)workspace, kMaxParts * 2);
    return hipGetLastError();
}

hipError_t launch_kv_attention(const KvView& c, const void* q, int64_t q_stride, int32_t Hq, float scale,
                               int32_t window, int32_t sinks, void* out, int64_t out_stride, void* workspace,
                               int64_t workspace_bytes, int n_cu, hipStream_t s) {
    AttnArgs a;
    a.q = (const uint16_t*)q;
    a.out = (uint16_t*)out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.G = Hq / c.H;
    a.scale2 = scale * 1.4426950408889634f;
    a.window = window;
    a.sinks = sinks;
    a.few = kFewRows;
    WsCarve ws{(char*)workspace, (size_t)workspace_bytes};
    a.arrived = ws.take<uint32_t>(kMaxParts * 2);
    // as many parts as workgroups fit the device, and 2.5 for each segment where that is more; segments stay whole
    // where half the workspace does not hold that many parts
    const int64_t segments = (int64_t)c.B * c.H;
    const int64_t fit = (int64_t)n_cu * (c.D == 64 ? kSplitPerCu<64> : c.D == 128 ? kSplitPerCu<128> : kSplitPerCu<256>);
    const int64_t room = std::min<int64_t>(workspace_bytes / 2 / (kFewRows * (c.D + 2) * 4), kMaxParts);
    const bool cut = segments * 3 <= room * 2;
    const int64_t wgs = cut ? std::min(std::max(fit, segments * 5 / 2), room) : segments;
    if (cut) {
        a.part_ml = ws.take<float2v>(wgs * kFewRows);
        a.part_o = ws.take<float>(wgs * kFewRows * c.D);
    }
    const int64_t slots = (int64_t)c.T * a.G / kTileRows + c.B;
    const bool tiles = (int64_t)c.max_new * a.G > a.few;
    const int splits = tiles ? tile_splits(c, a, slots, n_cu, workspace_bytes - (int64_t)ws.off - 4096) : 1;
    const int64_t tile_wgs = tiles ? slots * c.H * splits : 0, joiners = splits > 1 ? slots * c.H * (kTileRows / 8) : 0;
    if (splits > 1) {
        a.tile_ml = ws.take<float2v>(tile_wgs * kTileRows);
        a.tile_o = ws.take<float>(tile_wgs * kTileRows * c.D);
    }
    if (!ws.ok() || wgs + tile_wgs >= (int64_t)1 << 24 || joiners >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    return by_types(c, [&](auto fp8, auto f16) {
        auto run = [&](auto d) {
            constexpr int D = decltype(d)::value;
            if (tiles)
                kv_mixed_kernel<D, fp8.value, f16.value>
                    <<<(uint32_t)(tile_wgs + wgs), 256, 0, s>>>(c, a, slots, splits, cut);
            else
                kv_split_kernel<D, fp8.value, f16.value><<<(uint32_t)wgs, 256, 0, s>>>(c, a, cut);
            if (joiners)
                kv_tile_join_kernel<D, f16.value><<<(uint32_t)joiners, 256, 0, s>>>(c, a, splits);
            return hipGetLastError();
        };
        if (c.D == 64) return run(std::integral_constant<int, 64>{});
        if (c.D == 128) return run(std::integral_constant<int, 128>{});
        return run(std::integral_constant<int, 256>{});
    });
}

}  // namespace ls
