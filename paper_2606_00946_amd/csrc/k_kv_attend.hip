// Attention over the paged 8-bit KV cache (k_kv.h).
//
// out_i = sum_j softmax_j(scale q_i . k_j) v_j over the tokens j that row i sees.
//
// With key scale a_j and value scale b_j of token j's page and head, and codes
// K_j, V_j, the row's weights are carried as w_j = b_j 2^(x_j - m), x_j the
// base-2 logit, so that the value scales enter through the running maximum of
// x_j + log2 b_j and V_j stays as stored:
//   out = sum_j w_j V_j / sum_j (w_j / b_j).
// w_j is at most 2^15 and enters the product in half precision (11 bits, the
// rounding of the probabilities); codes and 16-bit queries are exact there, a
// bf16 query after scaling its row by a power of two.  The maximum, the sums and
// the products are fp32.
#include "k_kv.h"

namespace ls {
namespace {

using mask_t = uint64_t;

struct AttnArgs {
    const uint16_t* q;
    uint16_t* out;
    int64_t q_stride, out_stride;
    int32_t G;                       // query heads of a kv head
    float scale2;                    // softmax scale * log2 e
    int32_t window, sinks;
    int32_t few;                     // sequences with up to this many rows (new tokens x G) split along the keys
    // joining of split rows: partial sums of each workgroup's first and last segment
    float* part_o;                   // [workgroups][2][16][D]
    float2v* part_ml;                // [workgroups][2][16] running maximum and sum
    int64_t* first;                  // [B + 1] unit of each sequence's start, then the units of a workgroup
};

// What a sequence's rows see, in 16-token blocks: the first n_sink and those from
// win on, n in all; block i of them is tile(i).
struct Span {
    int32_t n_sink, win, n;
    __device__ __forceinline__ int32_t tile(int32_t i) const { return i < n_sink ? i : win + (i - n_sink); }
};

__device__ __forceinline__ Span span_of(const KvView& c, const AttnArgs& a, int64_t past, int32_t rows) {
    const int64_t end = min(past + rows, (int64_t)c.W << c.page_shift);
    int64_t lo = 0;
    if (a.window > 0) lo = min(max(past + 1 - a.window, (int64_t)0), end);
    Span s;
    s.win = (int32_t)(lo >> 4);
    s.n_sink = (int32_t)((min((int64_t)a.sinks, lo) + 15) >> 4);
    if (s.n_sink >= s.win) s.n_sink = s.win = 0;
    s.n = s.n_sink + (int32_t)((end + 15) >> 4) - s.win;
    return s;
}

constexpr int kUnit = 8;             // 16-token blocks of a work unit: two for each wave of a workgroup
constexpr float kNoMax = -1e30f;     // running maximum of nothing
constexpr float kTop = 7.0f;         // weights start below 2^7 ...
constexpr float kGrow = 8.0f;        // ... and the maximum moves when one would pass 2^15

// Units of one kv head of sequence b; 0: not this kernel's.
__device__ __forceinline__ int32_t units_of(const KvView& c, const AttnArgs& a, int b) {
    int t0, n;
    seq_rows(c, b, t0, n);
    if (n == 0 || (int64_t)n * a.G > a.few) return 0;
    const Span s = span_of(c, a, max(c.past[b], 0), n);
    return max((s.n + kUnit - 1) / kUnit, 1);
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
        const int e = max((int)(top >> 23), 27);                // biased: the row's largest is below 2^(e - 126)
        const float f = __uint_as_float((uint32_t)(min(267 - e, 254)) << 23);     // 2^(140 - e): below 2^14 and up
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
        return __uint_as_float((uint32_t)(254 - min(267 - e, 254)) << 23);
    }
}

// Few rows (up to 16 of a kv head) against a long cache: bound by HBM.  All the
// sequences' heads are laid end to end in units of 128 tokens and cut into equal
// shares, one workgroup each, whatever the lengths; a segment (sequence, head)
// that lies in one share is finished there, the others leave partial sums that
// kv_join_kernel adds.  A wave takes 32 of a unit's tokens at a time: scores
// transposed (tokens x rows), so that their registers are the second operand of
// the product with the values as they stand; codes go from memory to registers in
// 16-byte loads, one step ahead of their use.
template <int D, bool FP8, bool F16>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void kv_split_kernel(KvView c, AttnArgs a, int32_t min_units) {
    constexpr int ND = D / 64;
    __shared__ float comb[4][16][D + 4];
    __shared__ float2v ml[4][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;

    // the launch's units, this workgroup's share and where it starts
    int64_t total = 0;
    for (int b = lane; b < c.B; b += 64) total += units_of(c, a, b);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o);
    total = uniform(total) * c.H;
    const int64_t share = max((total + gridDim.x - 1) / gridDim.x, (int64_t)min_units);
    int64_t at = (int64_t)blockIdx.x * share;
    const int64_t stop = min(at + share, total);
    const bool scribe = blockIdx.x == 0 && wave == 0;        // writes the sequences' starts for the join
    if (at >= stop && !scribe) return;
    int b = 0;
    int64_t start = 0;               // first unit of sequence b
    {
        int64_t base = 0;
        bool found = false;
        for (int b0 = 0; b0 < c.B; b0 += 64) {
            const int64_t u = b0 + lane < c.B ? (int64_t)units_of(c, a, b0 + lane) * c.H : 0;
            int64_t end = u;         // inclusive sums
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int64_t v = __shfl_up(end, o);
                if (lane >= o) end += v;
            }
            end += base;
            if (scribe && b0 + lane < c.B) a.first[b0 + lane] = end - u;
            const mask_t m = __ballot(end > at);
            if (!found && m) {
                const int k = __ffsll((long long)m) - 1;
                b = b0 + k;
                start = __shfl(end - u, k);
                found = true;
                if (!scribe) break;
            }
            base = __shfl(end, 63);
        }
        if (scribe && lane == 0) {
            a.first[c.B] = total;
            a.first[c.B + 1] = share;
        }
    }
    b = __builtin_amdgcn_readfirstlane(b);
    start = uniform(start);

    while (at < stop) {
        const int32_t per_head = units_of(c, a, b);
        if (per_head == 0) { ++b; continue; }
        int t0, n;
        seq_rows(c, b, t0, n);
        const int64_t past = max(c.past[b], 0);
        const Span span = span_of(c, a, past, n);
        const int64_t end_tok = min(past + n, (int64_t)c.W << c.page_shift);
        const int32_t h = (int32_t)((at - start) / per_head);
        const int32_t u0 = (int32_t)((at - start) - (int64_t)h * per_head);
        const int32_t u1 = (int32_t)min((int64_t)per_head, u0 + (stop - at));
        const int rows = n * a.G;
        const int64_t pos = past + col / a.G;                // the column's position
        const int64_t pos_last = past + n - 1;

        half8 q[ND][2];
        const float undo = load_queries<D, F16>(a, h, t0, col, rows, q);
        const float s2 = a.scale2 * undo;

        // pages of step i's two blocks, and what is known of them
        struct Meta { int32_t page[2]; float ks[2], vs[2]; };
        auto tile_of = [&](int i, int e) { return (u0 + i) * kUnit + wave * 2 + e; };
        auto find_page = [&](int i, Meta& m) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int t = tile_of(i, e);
                int32_t p = -1;
                if (i < u1 - u0 && t < span.n) {
                    const int32_t j = span.tile(t) >> (c.page_shift - 4);
                    p = uniform_load(c.pages + (int64_t)b * c.W + j);
                    if (p >= c.n_pages) p = -1;
                }
                m.page[e] = p;
            }
        };
        auto find_scales = [&](Meta& m) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                m.ks[e] = m.vs[e] = 1.0f;
                if (m.page[e] >= 0) {
                    m.ks[e] = uniform_load(c.ks + (int64_t)m.page[e] * c.H + h);
                    m.vs[e] = uniform_load(c.vs + (int64_t)m.page[e] * c.H + h);
                }
            }
        };
        struct Raw { uint4v k[2][ND], v[2][ND]; };
        auto fetch = [&](int i, const Meta& m, Raw& r) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int t = tile_of(i, e);
                const int64_t base = m.page[e] < 0 ? 0 : block_at(c, m.page[e], h, span.tile(t) & ((c.page >> 4) - 1));
                const uint8_t* kp = c.k + base + col * 64 + g * 16;
                const uint8_t* vp = c.v + base + lane * 16;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    r.k[e][dt] = *reinterpret_cast<const uint4v*>(kp + dt * 1024);
                    r.v[e][dt] = *reinterpret_cast<const uint4v*>(vp + dt * 1024);
                }
            }
        };
        float m_run = kNoMax, l_run = 0.0f;
        float4v o[ND][4] = {};
        auto compute = [&](int i, const Meta& m, Raw& r) {
            if (m.page[0] < 0 && m.page[1] < 0) return;
            float x[2][4], mx = -INFINITY;
            float iv[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float4v s = {0, 0, 0, 0};
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                            code_halves8<FP8>(r.k[e][dt][2 * k], r.k[e][dt][2 * k + 1]), q[dt][k], s, 0, 0, 0);
                const float f = m.ks[e] * s2, lv = __builtin_amdgcn_logf(m.vs[e]);
                iv[e] = __builtin_amdgcn_rcpf(m.vs[e]);
                const int64_t tok = (int64_t)span.tile(tile_of(i, e)) * 16;
                const bool all = m.page[e] >= 0 && tok + 15 <= past &&
                                 (a.window == 0 || tok > pos_last - a.window || tok + 15 < a.sinks);
                if (all) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[e][k] = fmaf(s[k], f, lv);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int64_t j = tok + 4 * g + k;
                        const bool see = m.page[e] >= 0 && j <= pos && (a.window == 0 || j > pos - a.window || j < a.sinks);
                        x[e][k] = see ? fmaf(s[k], f, lv) : -INFINITY;
                    }
                    // codes of nobody's tokens may be NaN: out of the product
                    const int64_t left = m.page[e] >= 0 ? end_tok - (tok + 4 * g) : 0;
                    const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * (int)left)) - 1;
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) r.v[e][dt] &= keep;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) mx = fmaxf(mx, x[e][k]);
            }
            if (__any(mx > m_run + kGrow)) {
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m2 = fmaxf(m_run, mx);
                const float f = __builtin_amdgcn_exp2f(m_run - m2);
                m_run = m2;
                l_run *= f;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[dt][k] *= f;
            }
            half8 p;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = __builtin_amdgcn_exp2f(x[e][k] - (m_run - kTop));
                l_run = fmaf((w[0] + w[1]) + (w[2] + w[3]), iv[e], l_run);
#pragma unroll
                for (int k = 0; k < 4; ++k) p[4 * e + k] = (_Float16)w[k];
            }
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    o[dt][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                        code_halves8<FP8>(r.v[0][dt][k], r.v[1][dt][k]), p, o[dt][k], 0, 0, 0);
        };

        const int steps = u1 - u0;
        Meta m0, m1, m2;
        Raw r0, r1;
        find_page(0, m0);
        find_page(1, m1);
        find_scales(m0);
        fetch(0, m0, r0);
        for (int i = 0; i < steps; ++i) {
            find_page(i + 2, m2);
            find_scales(m1);
            fetch(i + 1, m1, r1);
            compute(i, m0, r0);
            m0 = m1;
            m1 = m2;
            r0 = r1;
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
        const bool whole = u0 == 0 && u1 == per_head;
        const float norm = l_row > 0.0f ? 1.0f / l_row : 0.0f;
        const int64_t slot = ((int64_t)blockIdx.x * 2 + (u0 == 0 ? 1 : 0)) * 16 + row;
        if (row < rows) {
            uint16_t* out = a.out + (int64_t)(t0 + row / a.G) * a.out_stride + ((int64_t)h * a.G + row % a.G) * D;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
                float4v v = {0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < 4; ++w) v += *reinterpret_cast<const float4v*>(&comb[w][row][dt * 64 + d0]);
                if (whole) {
                    v *= norm;
                    *reinterpret_cast<uint2v*>(out + dt * 64 + d0) =
                        uint2v{pack2<F16>(v.x, v.y), pack2<F16>(v.z, v.w)};
                } else {
                    *reinterpret_cast<float4v*>(a.part_o + slot * D + dt * 64 + d0) = v;
                }
            }
            if (!whole && d0 == 0) a.part_ml[slot] = float2v{m_row, l_row};
        }
        __syncthreads();

        at += u1 - u0;
        if (at - start == (int64_t)per_head * c.H) {
            start = at;
            ++b;
        }
    }
}

// Adds the partial sums of segments that several workgroups shared, in their
// order.  One workgroup for each sequence and kv head.
template <int D, bool F16>
__global__ __launch_bounds__(256) void kv_join_kernel(KvView c, AttnArgs a) {
    const int b = blockIdx.x / c.H, h = blockIdx.x % c.H;
    const int64_t share = a.first[c.B + 1];
    const int64_t s0 = a.first[b], per_head = (a.first[b + 1] - s0) / c.H;
    if (per_head == 0) return;
    const int64_t lo = s0 + h * per_head, hi = lo + per_head;
    const int64_t w0 = lo / share, w1 = (hi - 1) / share;
    if (w0 == w1) return;
    int t0, n;
    seq_rows(c, b, t0, n);
    const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * 4;
    if (row >= n * a.G) return;
    float m = kNoMax, l = 0.0f;
    float4v v[D / 64] = {};
    for (int64_t w = w0; w <= w1; ++w) {
        const int64_t slot = (w * 2 + (w == w0 ? 1 : 0)) * 16 + row;
        const float2v p = a.part_ml[slot];
        const float m2 = fmaxf(m, p.x);
        const float f = __builtin_amdgcn_exp2f(m - m2), e = __builtin_amdgcn_exp2f(p.x - m2);
        m = m2;
        l = l * f + p.y * e;
#pragma unroll
        for (int dt = 0; dt < D / 64; ++dt)
            v[dt] = v[dt] * f + *reinterpret_cast<const float4v*>(a.part_o + slot * D + dt * 64 + d0) * e;
    }
    const float norm = l > 0.0f ? 1.0f / l : 0.0f;
    uint16_t* out = a.out + (int64_t)(t0 + row / a.G) * a.out_stride + ((int64_t)h * a.G + row % a.G) * D;
#pragma unroll
    for (int dt = 0; dt < D / 64; ++dt)
        *reinterpret_cast<uint2v*>(out + dt * 64 + d0) =
            uint2v{pack2<F16>(v[dt].x * norm, v[dt].y * norm), pack2<F16>(v[dt].z * norm, v[dt].w * norm)};
}

// One wave per row and query head; 64 keys at a time, a lane each.
template <bool FP8, bool F16>
__global__ __launch_bounds__(256) void kv_attend_kernel(KvView c, const uint16_t* __restrict__ q, int64_t q_stride,
                                                        int32_t Hq, float scale, int32_t window, int32_t sinks,
                                                        uint16_t* __restrict__ out, int64_t out_stride, int32_t few) {
    __shared__ float qs[4][256];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + wave;
    if (w >= (int64_t)c.T * Hq) return;
    const int hq = (int)(w % Hq), t = (int)(w / Hq);
    const int h = hq / (Hq / c.H);
    int lo = 0, n = c.B;
    while (n > 1) {
        const int m = n >> 1;
        if (min(max(c.off[lo + m], 0), c.T) <= t) { lo += m; n -= m; } else { n = m; }
    }
    const int b = lo;
    if ((int64_t)(min(max(c.off[b + 1], 0), c.T) - min(max(c.off[b], 0), c.T)) * (Hq / c.H) <= few) return;
    const int64_t pos = (int64_t)max(c.past[b], 0) + t - min(max(c.off[b], 0), c.T);
    for (int d = lane; d < c.D; d += 64) {
        const uint16_t u = q[t * q_stride + (int64_t)hq * c.D + d];
        qs[wave][d] = unpack2<F16>(u).x;
    }
    __builtin_amdgcn_wave_barrier();
    const int nd = c.D >> 6;
    float m = -INFINITY, l = 0.0f, o[4] = {0, 0, 0, 0};
    const int64_t end = min(pos + 1, (int64_t)c.W << c.page_shift);
    for (int64_t j0 = 0; j0 < end; j0 += 64) {
        const int64_t j = j0 + lane;
        const bool seen = j < end && (window <= 0 || j > pos - window || j < sinks);
        const int64_t page = seen ? page_id(c, b, (int)(j >> c.page_shift)) : -1;
        if (__ballot(page >= 0) == 0) continue;
        const int r = (int)j & (c.page - 1);
        float x = -INFINITY, vs = 0.0f;
        if (page >= 0) {
            const uint8_t* tk = c.k + block_at(c, page, h, r >> 4) + (r & 15) * 64;
            float acc = 0.0f;
            for (int dt = 0; dt < nd; ++dt)
                for (int d = 0; d < 64; d += 4) {
                    const float4v f = code_values<FP8>(*reinterpret_cast<const uint32_t*>(tk + dt * 1024 + d));
                    for (int i = 0; i < 4; ++i) acc = fmaf(f[i], qs[wave][dt * 64 + d + i], acc);
                }
            x = acc * c.ks[page * c.H + h] * scale;
            vs = c.vs[page * c.H + h];
        }
        const float m2 = fmaxf(m, wave_max(x));
        const float f = m == -INFINITY ? 0.0f : expf(m - m2);
        const float p = page >= 0 ? expf(x - m2) : 0.0f;
        m = m2;
        float s = p;
        for (int k = 32; k >= 1; k >>= 1) s += __shfl_xor(s, k);
        l = l * f + s;
        for (int i = 0; i < nd; ++i) o[i] *= f;
        for (int k = 0; k < 64; ++k) {
            const int pk = __shfl((int)page, k);
            if (pk < 0) continue;
            const float pv = __shfl(p * vs, k);
            const int rk = (int)(j0 + k) & (c.page - 1);
            const uint8_t* tv = c.v + block_at(c, pk, h, rk >> 4) + ((rk & 15) >> 2) * 256 + lane * 4 + (rk & 3);
            for (int i = 0; i < nd; ++i) o[i] = fmaf(pv, code_values<FP8>(tv[i * 1024]).x, o[i]);
        }
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    for (int i = 0; i < nd; ++i)
        out[t * out_stride + (int64_t)hq * c.D + i * 64 + lane] = (uint16_t)pack2<F16>(o[i] * inv, 0.0f);
}

}  // namespace

int64_t kv_attention_workspace_bytes(const KvView& c, int n_cu) {
    const int64_t slots = (int64_t)n_cu * 2 * 2 * 16;
    return slots * (c.D + 2) * 4 + ((int64_t)c.B + 2) * 8;
}

hipError_t launch_kv_attention(const KvView& c, const void* q, int64_t q_stride, int32_t Hq, float scale,
                               int32_t window, int32_t sinks, void* out, int64_t out_stride, void* workspace, int n_cu,
                               hipStream_t s) {
    const int64_t groups = ((int64_t)c.T * Hq + 3) / 4;
    if (groups >= (int64_t)1 << 24 || (int64_t)c.B * c.H >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    AttnArgs a;
    a.q = (const uint16_t*)q;
    a.out = (uint16_t*)out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.G = Hq / c.H;
    a.scale2 = scale * 1.4426950408889634f;
    a.window = window;
    a.sinks = sinks;
    a.few = 16;
    const uint32_t wgs = (uint32_t)n_cu * 2;
    const int64_t slots = (int64_t)wgs * 2 * 16;
    a.first = (int64_t*)workspace;
    a.part_ml = (float2v*)(a.first + c.B + 2);
    a.part_o = (float*)(a.part_ml + slots) + (c.B & 1 ? 2 : 0);       // 16-byte aligned
    hipError_t e = by_types(c, [&](auto fp8, auto f16) {
        auto run = [&](auto d) {
            constexpr int D = decltype(d)::value;
            kv_split_kernel<D, fp8.value, f16.value><<<wgs, 256, 0, s>>>(c, a, 2);
            kv_join_kernel<D, f16.value><<<(uint32_t)(c.B * c.H), 256, 0, s>>>(c, a);
            return hipGetLastError();
        };
        if (c.D == 64) return run(std::integral_constant<int, 64>{});
        if (c.D == 128) return run(std::integral_constant<int, 128>{});
        return run(std::integral_constant<int, 256>{});
    });
    if (e != hipSuccess || (int64_t)c.max_new * a.G <= a.few) return e;
    return by_types(c, [&](auto fp8, auto f16) {
        kv_attend_kernel<fp8.value, f16.value><<<(uint32_t)groups, 256, 0, s>>>(
            c, (const uint16_t*)q, q_stride, Hq, scale, window, sinks, (uint16_t*)out, out_stride, a.few);
        return hipGetLastError();
    });
}

}  // namespace ls
