// Appending to, and reading from, the paged 8-bit KV cache (k_kv.h).
//
// A token's key is rotated by its position, a pair (a, b) of dimensions going to
// (a cos - b sin, b cos + a sin), and stored with its value as 8-bit codes under
// one scale for each page and head.  Both directions are bound by HBM: the
// rows once in 16 bits, the codes once in 8.
#include <algorithm>

#include "k_kv.h"
#include "ls_kv_calls.h"

namespace ls {
namespace {

// Eight floats of a 16-byte row piece.
template <bool F16>
__device__ __forceinline__ void widen8(uint4v w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2v u = unpack2<F16>(w[i]);
        x[2 * i] = u.x;
        x[2 * i + 1] = u.y;
    }
}

__device__ __forceinline__ uint4v load8(const uint16_t* p) { return *reinterpret_cast<const uint4v*>(p); }

// The u-th of a row's D / 16 units: two runs of eight dimensions, at a and b, that
// hold eight rotary pairs (x[i] with x[8 + i], or neighbours when interleaved), or
// sixteen dimensions past the rotary ones.
struct Unit {
    int a, b;
    bool turns;
};
__device__ __forceinline__ Unit unit_of(const KvRope& r, int u) {
    if (u * 16 >= r.rotary || r.interleaved) return {u * 16, u * 16 + 8, u * 16 < r.rotary};
    return {u * 8, (r.rotary >> 1) + u * 8, true};
}

// cos and sin of a unit's eight pairs at a position.
struct Turn {
    float4v c[2], s[2];
};
__device__ __forceinline__ Turn turn_of(const KvRope& r, const Unit& t, int u, int64_t pos) {
    Turn f = {{{1, 1, 1, 1}, {1, 1, 1, 1}}, {{0, 0, 0, 0}, {0, 0, 0, 0}}};
    if (t.turns) {
        const int64_t at = min(pos, (int64_t)r.n_pos - 1) * (r.rotary >> 1) + u * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f.c[i] = reinterpret_cast<const float4v*>(r.cos + at)[i];
            f.s[i] = reinterpret_cast<const float4v*>(r.sin + at)[i];
        }
    }
    return f;
}

// Where the positions of a call's rows come from: their places in their sequences,
// an axis for each unit of pairs, or an axis for each pair.
enum Where { PLACE, UNIT, PAIR };

__device__ __forceinline__ int axis_of(const KvPositions& at, int pair) { return at.axis[pair >> 4] >> 2 * (pair & 15) & 3; }

// The same of the call's row t on the axes of the unit's pairs; a position below 0 counts as 0.  A
// unit on one axis costs one more load; one on several axes reads its pairs' angles one by one.
template <Where AT>
__device__ __forceinline__ Turn turn_at(const KvRope& r, const KvPositions& at, const Unit& t, int u, int64_t pos, int64_t row,
                                        int32_t T) {
    if constexpr (AT == PLACE) return turn_of(r, t, u, pos);
    if constexpr (AT == UNIT)
        return turn_of(r, t, u, t.turns ? max(at.pos[(int64_t)axis_of(at, u * 8) * T + row], 0) : 0);
    Turn f = {{{1, 1, 1, 1}, {1, 1, 1, 1}}, {{0, 0, 0, 0}, {0, 0, 0, 0}}};
    if (t.turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int32_t p = at.pos[(int64_t)axis_of(at, u * 8 + i) * T + row];
            const int64_t e = (int64_t)min(max(p, 0), r.n_pos - 1) * (r.rotary >> 1) + u * 8 + i;
            f.c[i >> 2][i & 3] = r.cos[e];
            f.s[i >> 2][i & 3] = r.sin[e];
        }
    }
    return f;
}

// Rotates a unit's values; each product and sum is rounded by itself.
__device__ __forceinline__ void rotate(const KvRope& r, const Unit& t, const Turn& f, float (&x)[16]) {
    if (!t.turns) return;
    auto pair = [&](float& a, float& b, int i) {
        const float c = f.c[i >> 2][i & 3], s = f.s[i >> 2][i & 3];
        const float u = a * c - b * s, v = b * c + a * s;
        a = u;
        b = v;
    };
    if (r.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) pair(x[2 * i], x[2 * i + 1], i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) pair(x[i], x[8 + i], i);
    }
}

// NaN to 0; the magnitude that counts towards a scale.
__device__ __forceinline__ float clean(float& x) {
    x = x == x ? x : 0.0f;
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.0f;
}
__device__ __forceinline__ float clean16(float (&x)[16]) {
    float a = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) a = fmaxf(a, clean(x[i]));
    return a;
}

template <bool FP8>
__device__ __forceinline__ uint4v codes16(const float (&x)[16], float inv) {
    uint4v w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = codes_of<FP8>(x[4 * i] * inv, x[4 * i + 1] * inv, x[4 * i + 2] * inv, x[4 * i + 3] * inv);
    return w;
}

// Codes brought from one scale to another (again = old / new).
template <bool FP8>
__device__ __forceinline__ uint32_t regraded(uint32_t w, float again) {
    const float4v f = code_values<FP8>(w);
    return codes_of<FP8>(f.x * again, f.y * again, f.z * again, f.w * again);
}

// A page's rows [row0, row1) are new; `src` is row row0's, `pos0` the page's first
// position, `row` the call's row of row0.
struct PageWork {
    int64_t page, pos0, row;
    // The call's row of the page's row i, or of the new one next to it.
    __device__ __forceinline__ int64_t row_of(int i) const { return row + min(max(i, row0), row1 - 1) - row0; }
    const uint16_t* src;
    int64_t stride;
    int row0, row1;
};

// Brings the rows before row0 of a page and head to a new scale: a wave.
template <int D, bool FP8, bool VALUE>
__device__ __forceinline__ void regrade_rows(uint8_t* base, int row0, float again) {
    const int lane = threadIdx.x & 63;
    for (int blk = 0; blk * 16 < row0; ++blk)
#pragma unroll
        for (int dt = 0; dt < D / 64; ++dt) {
            uint4v* tile = reinterpret_cast<uint4v*>(base + (blk * D / 64 + dt) * 1024) + lane;
            uint4v o = *tile;
            if constexpr (!VALUE) {
                if (blk * 16 + (lane >> 2) >= row0) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = regraded<FP8>(o[i], again);
            } else {
                const int below = row0 - (blk * 16 + (lane >> 4) * 4);      // of the lane's four tokens
                if (below <= 0) continue;
                const uint32_t m = below < 4 ? (1u << 8 * below) - 1 : ~0u;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = (regraded<FP8>(o[i], again) & m) | (o[i] & ~m);
            }
            *tile = o;
        }
    // before any lane reads or writes beside these bytes
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");
}

// One new row in the page (a decode step): a row's units side by side for as many
// heads as a wave holds, so that one pass of loads serves them all.
template <int D, bool FP8, bool F16, bool VALUE, Where AT>
__device__ __forceinline__ void append_row(const KvView& c, const KvRope& r, const KvPositions& at, const PageWork& w, int h0,
                                           int heads) {
    constexpr int U = D / 16;
    const int lane = threadIdx.x & 63, u = lane % U, h = h0 + lane / U;
    const bool on = lane / U < heads;
    const Unit t = VALUE ? Unit{u * 16, u * 16 + 8, false} : unit_of(r, u);
    float* sp = (VALUE ? c.vs : c.ks) + w.page * c.H + (on ? h : h0);
    const float held = w.row0 > 0 ? *sp : 0.0f;
    uint4v raw[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if (on) {
        raw[0] = load8(w.src + h * D + t.a);
        raw[1] = load8(w.src + h * D + t.b);
    }
    const Turn f = turn_at<AT>(r, at, t, u, w.pos0 + w.row0, w.row, c.T);
    float x[16];
    widen8<F16>(raw[0], x);
    widen8<F16>(raw[1], x + 8);
    rotate(r, t, f, x);
    float a = clean16(x);
#pragma unroll
    for (int o = 1; o < U; o <<= 1) a = fmaxf(a, __shfl_xor(a, o));
    const float scale = fmaxf(scale_of<FP8>(a), held), inv = 1.0f / scale;
    const float again = held * inv;
    uint8_t* pages = VALUE ? c.v : c.k;
    // heads whose scale grew: what they hold, one after the other
    uint64_t grown = __ballot(on && w.row0 > 0 && scale > held && u == 0);
    while (grown) {
        const int l = __ffsll((long long)grown) - 1;
        grown &= grown - 1;
        regrade_rows<D, FP8, VALUE>(pages + block_at(c, w.page, h0 + l / U, 0), w.row0, __shfl(again, l));
    }
    if (!on) return;
    const uint4v q = codes16<FP8>(x, inv);
    uint8_t* base = pages + block_at(c, w.page, h, w.row0 >> 4);
    const int row = w.row0 & 15;
    if constexpr (!VALUE) {
        *reinterpret_cast<uint2v*>(base + (t.a >> 6) * 1024 + row * 64 + (t.a & 63)) = uint2v{q[0], q[1]};
        *reinterpret_cast<uint2v*>(base + (t.b >> 6) * 1024 + row * 64 + (t.b & 63)) = uint2v{q[2], q[3]};
    } else {
        uint8_t* d = base + (t.a >> 6) * 1024 + (row >> 2) * 256 + (t.a & 63) * 4 + (row & 3);
#pragma unroll
        for (int i = 0; i < 16; ++i) d[4 * i] = (uint8_t)(q[i >> 2] >> 8 * (i & 3));
    }
    if (u == 0 && scale != held) *sp = scale;
}

// A page and head's keys or values in general.  A lane holds D / 64 units of a
// 16-token block: keys a rotary unit of one token, values four dimensions of four
// tokens.  New rows of one block (ONE; `turns`: its positions' table rows) stay in
// registers between finding the scale and writing the codes; those of several are
// read again, from the caches (pages of 32 and 64, an axis for each pair, 4 tokens of each of 9
// sequences 12.3 and 8.7 us, 8 of each of 32 10.6 and 8.3).
template <int D, bool FP8, bool F16, bool VALUE, bool ONE, Where AT>
__device__ __forceinline__ void append_page(const KvView& c, const KvRope& r, const KvPositions& at, const PageWork& w, int h,
                                            const Turn (&turns)[D / 64]) {
    constexpr int U = D / 16, N = D / 64;
    const int lane = threadIdx.x & 63;
    float* sp = (VALUE ? c.vs : c.ks) + w.page * c.H + h;
    uint8_t* base = (VALUE ? c.v : c.k) + block_at(c, w.page, h, 0);
    const float held = w.row0 > 0 ? *sp : 0.0f;
    const int b0 = w.row0 >> 4, b1 = ONE ? b0 + 1 : (w.row1 + 15) >> 4;
    const uint16_t* src = w.src + h * D;
    float x[N][16];
    auto load = [&](int blk) {
        uint4v raw[N][2];
        if constexpr (!VALUE) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int e = n * 64 + lane, row = blk * 16 + e / U;
                const Unit t = unit_of(r, e % U);
                const bool on = row >= w.row0 && row < w.row1;
                const uint16_t* p = src + (row - w.row0) * w.stride;
                raw[n][0] = on ? load8(p + t.a) : uint4v{0, 0, 0, 0};
                raw[n][1] = on ? load8(p + t.b) : uint4v{0, 0, 0, 0};
            }
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int row = blk * 16 + (lane >> 4) * 4 + t;
                    const bool on = row >= w.row0 && row < w.row1;
                    const uint2v v = on ? *reinterpret_cast<const uint2v*>(src + (row - w.row0) * w.stride + n * 64 +
                                                                           (lane & 15) * 4)
                                        : uint2v{0, 0};
                    raw[n][t >> 1][2 * (t & 1)] = v[0];
                    raw[n][t >> 1][2 * (t & 1) + 1] = v[1];
                }
        }
        float a = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if constexpr (!VALUE) {
                widen8<F16>(raw[n][0], x[n]);
                widen8<F16>(raw[n][1], x[n] + 8);
                const int e = n * 64 + lane;
                const Unit t = unit_of(r, e % U);
                const int row = blk * 16 + e / U;
                rotate(r, t, ONE ? turns[n] : turn_at<AT>(r, at, t, e % U, w.pos0 + row, w.row_of(row), c.T), x[n]);
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const float2v lo = unpack2<F16>(raw[n][t >> 1][2 * (t & 1)]);
                    const float2v hi = unpack2<F16>(raw[n][t >> 1][2 * (t & 1) + 1]);
                    x[n][t] = lo.x;
                    x[n][4 + t] = lo.y;
                    x[n][8 + t] = hi.x;
                    x[n][12 + t] = hi.y;
                }
            }
            a = fmaxf(a, clean16(x[n]));
        }
        return a;
    };
    float a = 0.0f;
    for (int blk = b0; blk < b1; ++blk) a = fmaxf(a, load(blk));
    a = wave_max(a);
    const float scale = fmaxf(scale_of<FP8>(a), held), inv = 1.0f / scale;
    const float again = held * inv;
    if (w.row0 > 0 && scale > held) regrade_rows<D, FP8, VALUE>(base, w.row0, again);
    for (int blk = b0; blk < b1; ++blk) {
        if (!ONE) (void)load(blk);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint4v q = codes16<FP8>(x[n], inv);
            if constexpr (!VALUE) {
                const int e = n * 64 + lane, row = e / U;
                const Unit t = unit_of(r, e % U);
                if (blk * 16 + row < w.row0 || blk * 16 + row >= w.row1) continue;
                uint8_t* d = base + blk * 16 * D + row * 64;
                *reinterpret_cast<uint2v*>(d + (t.a >> 6) * 1024 + (t.a & 63)) = uint2v{q[0], q[1]};
                *reinterpret_cast<uint2v*>(d + (t.b >> 6) * 1024 + (t.b & 63)) = uint2v{q[2], q[3]};
            } else {
                const int t0 = blk * 16 + (lane >> 4) * 4;      // the lane's four tokens
                if (t0 >= w.row1 || t0 + 4 <= w.row0) continue;
                uint4v* tile = reinterpret_cast<uint4v*>(base + blk * 16 * D + n * 1024) + lane;
                if (t0 < w.row0 || t0 + 4 > w.row1) {
                    // bytes of the rows before row0 are held (and just regraded by this lane), those from row1 on nobody's
                    const uint32_t below = t0 < w.row0 ? (1u << 8 * (w.row0 - t0)) - 1 : 0u;
                    const uint32_t above = t0 + 4 > w.row1 ? ~((1u << 8 * (w.row1 - t0)) - 1) : 0u;
                    const uint4v o = *tile;
                    q = (o & (below | above)) | (q & ~(below | above));
                }
                *tile = q;
            }
        }
    }
    if (lane == 0 && scale != held) *sp = scale;
}

// Waves [0, n_items): (slot, `heads` kv heads, key or value), a slot being a page
// that a sequence's new tokens touch.  Sequence b owns the slots from
// off[b] / page + 2 b on: at least as many as pages it touches.  The waves after
// them rotate a row of the queries each, as many heads at a time as a wave holds.
// Measured: 69k tokens of 8 kv and 32 query heads of 128: 305 us, 5.1 TB/s; 256 single
// tokens 6.2 us; one token 3.1 us.  By given positions: 55k tokens on three axes in runs of
// pairs 246 us, the same rate; 32 trees of 16 to 64 drafts 10.2 us, the chain of offsets, positions and
// table rows.
template <int D, bool FP8, bool F16, Where AT>
__global__ __launch_bounds__(256) void kv_append_kernel(KvView c, KvRope r, KvPositions at, const uint16_t* __restrict__ k,
                                                        int64_t k_stride, const uint16_t* __restrict__ v,
                                                        int64_t v_stride, const uint16_t* q, int64_t q_stride,
                                                        int32_t Hq, uint16_t* q_out, int64_t q_out_stride,
                                                        uint32_t n_items, int32_t heads) {
    constexpr int U = D / 16;
    const int lane = threadIdx.x & 63;
    const uint32_t w = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (w < n_items) {
        const bool value = w & 1;
        const uint32_t groups = (uint32_t)(c.H + heads - 1) / (uint32_t)heads;
        const int h0 = (int)((w >> 1) % groups) * heads;
        const int64_t slot = (w >> 1) / groups;
        const int sh = c.page_shift;
        auto first = [sh](int off, int b) { return block_slot(off, b, sh); };
        const int b = seq_of_slot(c, slot, first);
        int t0, n;
        seq_rows(c, b, t0, n);
        const int64_t past = max(c.past[b], 0);
        const BlockRows its = block_rows(slot - first(t0, b), n, past, sh);
        PageWork p;
        p.row0 = its.row0;
        p.row1 = its.row1;
        if (p.row0 >= p.row1 || its.j >= c.W) return;
        p.pos0 = its.j << sh;
        p.page = page_id(c, b, (int)its.j);
        if (p.page < 0) return;
        p.stride = value ? v_stride : k_stride;
        p.row = t0 + (p.pos0 + p.row0 - past);
        p.src = (value ? v : k) + p.row * p.stride;
        const int hn = min(heads, c.H - h0);
        auto append = [&](auto is_value) {
            constexpr bool V = decltype(is_value)::value;
            if (p.row1 - p.row0 == 1) {
                append_row<D, FP8, F16, V, V ? PLACE : AT>(c, r, at, p, h0, hn);
                return;
            }
            Turn turns[D / 64] = {};
            const int row = p.row0 & ~15;
            if (p.row1 <= row + 16) {
                if constexpr (!V)
#pragma unroll
                    for (int i = 0; i < D / 64; ++i) {
                        const int e = i * 64 + lane;
                        turns[i] = turn_at<AT>(r, at, unit_of(r, e % U), e % U, p.pos0 + row + e / U, p.row_of(row + e / U), c.T);
                    }
                for (int i = 0; i < hn; ++i) append_page<D, FP8, F16, V, true, AT>(c, r, at, p, h0 + i, turns);
            } else {
                for (int i = 0; i < hn; ++i) append_page<D, FP8, F16, V, false, AT>(c, r, at, p, h0 + i, turns);
            }
        };
        if (value) append(std::true_type{}); else append(std::false_type{});
        return;
    }
    const int64_t t = (int64_t)w - n_items;
    if (!q || t >= c.T) return;
    int64_t pos = 0;
    if constexpr (AT == PLACE) {
        const int b = seq_of_slot(c, t, [](int off, int) { return (int64_t)off; });
        pos = max((int64_t)max(c.past[b], 0) + t - min(max(c.off[b], 0), c.T), (int64_t)0);
    }
    const int u = lane % U;
    const Unit m = unit_of(r, u);
    const Turn f = turn_at<AT>(r, at, m, u, pos, t, c.T);
    const uint16_t* src = q + t * q_stride;
    uint16_t* dst = q_out + t * q_out_stride;
    // a lane reads all that it writes first: q_out may be q
    constexpr int kAtOnce = 4, kStep = 64 / U;
    for (int h = lane / U; h < Hq; h += kStep * kAtOnce) {
        uint4v raw[kAtOnce][2];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (h + i * kStep < Hq) {
                raw[i][0] = load8(src + (h + i * kStep) * D + m.a);
                raw[i][1] = load8(src + (h + i * kStep) * D + m.b);
            }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (h + i * kStep < Hq) {
                float x[16];
                widen8<F16>(raw[i][0], x);
                widen8<F16>(raw[i][1], x + 8);
                rotate(r, m, f, x);
                uint4v o[2];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e >> 2][e & 3] = pack2<F16>(x[2 * e], x[2 * e + 1]);
                uint16_t* d = dst + (h + i * kStep) * D;
                *reinterpret_cast<uint4v*>(d + m.a) = o[0];
                *reinterpret_cast<uint4v*>(d + m.b) = o[1];
            }
    }
}

// Waves: (16-token block of a sequence's rows, head, key or value).  Bound by HBM: 265 MB
// in 52 us, 5.1 TB/s; 16 short tails 4.4 us.
template <bool FP8, bool F16>
__global__ __launch_bounds__(256) void kv_read_kernel(KvView c, uint16_t* __restrict__ k_out,
                                                      uint16_t* __restrict__ v_out, uint32_t n_items) {
    const uint32_t w = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (w >= n_items) return;
    const int lane = threadIdx.x & 63;
    const bool value = w & 1;
    const int h = (int)((w >> 1) % (uint32_t)c.H);
    const int64_t slot = (w >> 1) / (uint32_t)c.H;
    auto first = [](int off, int b) { return block_slot(off, b, 4); };
    const int b = seq_of_slot(c, slot, first);
    int t0, n;
    seq_rows(c, b, t0, n);
    const int64_t past = max(c.past[b], 0);
    const BlockRows its = block_rows(slot - first(t0, b), n, past, 4);
    const int row0 = its.row0, row1 = its.row1;
    if (row0 >= row1) return;
    const int64_t pos0 = its.j << 4;
    const int64_t j = pos0 >> c.page_shift;
    const int64_t page = j < c.W ? page_id(c, b, (int)j) : -1;
    const int64_t ld = (int64_t)c.H * c.D;
    uint16_t* out = (value ? v_out : k_out) + (t0 + pos0 - past) * ld + (int64_t)h * c.D;   // row of token pos0
    const float s = page >= 0 ? (value ? c.vs : c.ks)[page * c.H + h] : 0.0f;
    const uint8_t* tiles =
        (value ? c.v : c.k) + block_at(c, max(page, (int64_t)0), h, (int)(pos0 & (c.page - 1)) >> 4);
    for (int dt = 0; dt < (c.D >> 6); ++dt) {
        uint4v g = {0, 0, 0, 0};
        if (page >= 0) g = *(reinterpret_cast<const uint4v*>(tiles + dt * 1024) + lane);
        float4v f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = page >= 0 ? code_values<FP8>(g[i]) * s : float4v{0, 0, 0, 0};
        if (!value) {
            const int row = lane >> 2;
            if (row < row0 || row >= row1) continue;
            uint4v o[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i >> 1][2 * (i & 1)] = pack2<F16>(f[i].x, f[i].y);
                o[i >> 1][2 * (i & 1) + 1] = pack2<F16>(f[i].z, f[i].w);
            }
            uint4v* dst = reinterpret_cast<uint4v*>(out + row * ld + dt * 64 + (lane & 3) * 16);
            dst[0] = o[0];
            dst[1] = o[1];
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int row = (lane >> 4) * 4 + t;
                if (row < row0 || row >= row1) continue;
                const uint2v o = {pack2<F16>(f[0][t], f[1][t]), pack2<F16>(f[2][t], f[3][t])};
                *reinterpret_cast<uint2v*>(out + row * ld + dt * 64 + (lane & 15) * 4) = o;
            }
        }
    }
}

}  // namespace

hipError_t launch_kv_append_at(const KvView& c, const KvRope& r, const KvPositions& at, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, const void* q, int64_t q_stride, int32_t Hq, void* q_out,
                               int64_t q_out_stride, int n_cu, hipStream_t s) {
    const int64_t slots = (int64_t)(c.T >> c.page_shift) + 2 * (int64_t)c.B;
    // heads a wave takes in turn: all that one pass of a single row's loads serves, fewer while that leaves waves idle
    int heads = std::min(c.H, 1024 / c.D);
    while (c.max_new > 1 && heads > 1 && slots * 2 * ((c.H + heads - 1) / heads) < (int64_t)n_cu * 16) heads >>= 1;
    const int64_t n_items = slots * 2 * ((c.H + heads - 1) / heads);
    const int64_t groups = (n_items + (q ? c.T : 0) + 3) / 4;
    if (groups >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    return by_types(c, [&](auto fp8, auto f16) {
        auto run = [&](auto d) {
            auto launch = [&](auto where) {
                kv_append_kernel<decltype(d)::value, fp8.value, f16.value, decltype(where)::value>
                    <<<(uint32_t)groups, 256, 0, s>>>(c, r, at, (const uint16_t*)k, k_stride, (const uint16_t*)v, v_stride,
                                                      (const uint16_t*)q, q_stride, Hq, (uint16_t*)q_out, q_out_stride,
                                                      (uint32_t)n_items, heads);
                return hipGetLastError();
            };
            if (at.n_axes == 0) return launch(std::integral_constant<Where, PLACE>{});
            if (at.mixed) return launch(std::integral_constant<Where, PAIR>{});
            return launch(std::integral_constant<Where, UNIT>{});
        };
        if (c.D == 64) return run(std::integral_constant<int, 64>{});
        if (c.D == 128) return run(std::integral_constant<int, 128>{});
        return run(std::integral_constant<int, 256>{});
    });
}

hipError_t launch_kv_read(const KvView& c, void* k_out, void* v_out, hipStream_t s) {
    const int64_t n_items = ((int64_t)(c.T >> 4) + 2 * (int64_t)c.B) * c.H * 2;
    const int64_t groups = (n_items + 3) / 4;
    if (groups >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    return by_types(c, [&](auto fp8, auto f16) {
        kv_read_kernel<fp8.value, f16.value>
            <<<(uint32_t)groups, 256, 0, s>>>(c, (uint16_t*)k_out, (uint16_t*)v_out, (uint32_t)n_items);
        return hipGetLastError();
    });
}

}  // namespace ls
