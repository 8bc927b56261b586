// Appending to, and reading from, the paged 8-bit KV cache (k_kv.h).
//
// A token's key is rotated by its position, a pair (a, b) of dimensions going to
// (a cos - b sin, b cos + a sin), and stored with its value as 8-bit codes under
// one scale for each page and head.  Both directions are bound by HBM: the
// rows once in 16 bits, the codes once in 8.
#include "k_kv.h"

namespace ls {
namespace {

// 16 floats of a 32-byte row piece.
template <bool F16>
__device__ __forceinline__ void load16(const uint16_t* p, float (&x)[16]) {
    const uint4v* q = reinterpret_cast<const uint4v*>(p);
    const uint4v a = q[0], b = q[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2v u = unpack2<F16>(a[i]), w = unpack2<F16>(b[i]);
        x[2 * i] = u.x;
        x[2 * i + 1] = u.y;
        x[8 + 2 * i] = w.x;
        x[8 + 2 * i + 1] = w.y;
    }
}

// Dimensions d .. d + 15 (d a multiple of 16) of a row, rotated for `pos`.
template <bool F16>
__device__ __forceinline__ void load_rotated(const KvRope& r, const uint16_t* row, int d, int64_t pos, float (&x)[16]) {
    load16<F16>(row + d, x);
    if (d >= r.rotary) return;
    const int half = r.rotary >> 1;
    const int64_t at = min(pos, (int64_t)r.n_pos - 1) * half;
    if (r.interleaved) {
        const float* c = r.cos + at + (d >> 1);
        const float* s = r.sin + at + (d >> 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = a * c[i] - b * s[i];
            x[2 * i + 1] = b * c[i] + a * s[i];
        }
    } else {
        const bool hi = d >= half;
        float y[16];
        load16<F16>(row + (hi ? d - half : d + half), y);
        const float* c = r.cos + at + (hi ? d - half : d);
        const float* s = r.sin + at + (hi ? d - half : d);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float xc = x[i] * c[i], ys = y[i] * s[i];
            x[i] = hi ? xc + ys : xc - ys;
        }
    }
}

// NaN to 0; the magnitude that counts towards a scale.
__device__ __forceinline__ float clean(float& x) {
    x = x == x ? x : 0.0f;
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.0f;
}

// One wave's share: a page and head's keys or values.  Two passes over the new
// rows, the second from the caches: the largest magnitude, then the codes.
// Keys: a lane holds 16 dimensions of one token (lane / 4).  Values: four
// dimensions of the four tokens 4 (lane / 16) ...
template <bool FP8, bool F16>
__device__ void append_page(const KvView& c, const KvRope& r, bool value, int h, int64_t page, int64_t pos0, int row0,
                            int row1, bool open, const uint16_t* src, int64_t stride) {
    // rows row0 .. row1 of the page are new and come from src (row row0 first); pos0: the page's first position;
    // open: the rows before row0 are held already
    const int lane = threadIdx.x & 63;
    const int nd = c.D >> 6;
    float* sp = (value ? c.vs : c.ks) + page * c.H + h;
    uint8_t* base = (value ? c.v : c.k) + block_at(c, page, h, 0);
    const float held = open ? *sp : 0.0f;
    const int b0 = row0 >> 4, b1 = (row1 + 15) >> 4;
    float x[16];
    auto load = [&](int blk, int dt) {
        float a = 0.0f;
        if (!value) {
            const int row = blk * 16 + (lane >> 2);
            if (row >= row0 && row < row1) {
                load_rotated<F16>(r, src + (row - row0) * stride + (int64_t)h * c.D, dt * 64 + (lane & 3) * 16,
                                  pos0 + row, x);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = 0.0f;
            }
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int row = blk * 16 + (lane >> 4) * 4 + t;
                uint2v w = {0, 0};
                if (row >= row0 && row < row1)
                    w = *reinterpret_cast<const uint2v*>(src + (row - row0) * stride + (int64_t)h * c.D + dt * 64 +
                                                         (lane & 15) * 4);
                const float2v u = unpack2<F16>(w[0]), v = unpack2<F16>(w[1]);
                x[t] = u.x;
                x[4 + t] = u.y;
                x[8 + t] = v.x;
                x[12 + t] = v.y;
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) a = fmaxf(a, clean(x[i]));
        return a;
    };
    float amax = 0.0f;
    for (int blk = b0; blk < b1; ++blk)
        for (int dt = 0; dt < nd; ++dt) amax = fmaxf(amax, load(blk, dt));
    amax = wave_max(amax);
    const float scale = fmaxf(scale_of<FP8>(amax), held);
    const float inv = 1.0f / scale;
    const float again = held * inv;       // of codes that the page held
    const bool regrade = open && again != 1.0f;
    for (int blk = regrade ? 0 : b0; blk < b1; ++blk) {
        for (int dt = 0; dt < nd; ++dt) {
            uint4v* tile = reinterpret_cast<uint4v*>(base + (int64_t)blk * 16 * c.D + dt * 1024) + lane;
            (void)load(blk, dt);
            uint4v w;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = codes_of<FP8>(x[4 * i] * inv, x[4 * i + 1] * inv, x[4 * i + 2] * inv, x[4 * i + 3] * inv);
            if (!value) {
                const int row = blk * 16 + (lane >> 2);
                if (row < row0) {
                    if (!regrade) continue;
                    const uint4v o = *tile;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4v f = code_values<FP8>(o[i]);
                        w[i] = codes_of<FP8>(f.x * again, f.y * again, f.z * again, f.w * again);
                    }
                }
                if (row < row1) *tile = w;
            } else {
                const int t0 = blk * 16 + (lane >> 4) * 4;    // the lane's four tokens
                if (t0 >= row1 || (t0 + 4 <= row0 && !regrade)) continue;
                if (t0 < row0 || t0 + 4 > row1) {
                    // bytes below `lo` are held, those from `hi` on are nobody's yet
                    const int lo = min(max(row0 - t0, 0), 4), hi = min(row1 - t0, 4);
                    const uint32_t below = lo < 4 ? (1u << 8 * lo) - 1 : ~0u;
                    const uint32_t above = hi < 4 ? ~((1u << 8 * hi) - 1) : 0u;
                    const uint4v o = *tile;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t g = o[i];
                        if (regrade) {
                            const float4v f = code_values<FP8>(g);
                            g = codes_of<FP8>(f.x * again, f.y * again, f.z * again, f.w * again);
                        }
                        w[i] = (g & below) | (o[i] & above) | (w[i] & ~below & ~above);
                    }
                }
                *tile = w;
            }
        }
    }
    if (lane == 0 && scale != held) *sp = scale;
}

// Waves [0, n_items): (slot, head, key or value), a slot being a page that a
// sequence's new tokens touch.  Sequence b owns the slots from
// off[b] / page + 2 b on: at least as many as pages it touches.  The waves
// after them rotate the queries, 16 dimensions a lane.
template <bool FP8, bool F16>
__global__ __launch_bounds__(256) void kv_append_kernel(KvView c, KvRope r, const uint16_t* __restrict__ k,
                                                        int64_t k_stride, const uint16_t* __restrict__ v,
                                                        int64_t v_stride, const uint16_t* q, int64_t q_stride,
                                                        int32_t Hq, uint16_t* q_out, int64_t q_out_stride,
                                                        int64_t n_items) {
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w < n_items) {
        const bool value = w & 1;
        const int h = (int)((w >> 1) % c.H);
        const int64_t slot = (w >> 1) / c.H;
        const int sh = c.page_shift;
        auto first = [sh](int off, int b) { return (int64_t)(off >> sh) + 2 * (int64_t)b; };
        const int b = seq_of_slot(c, slot, first);
        int t0, n;
        seq_rows(c, b, t0, n);
        const int64_t past = max(c.past[b], 0);
        const int64_t j = (past >> sh) + (slot - first(t0, b));      // the page's place in the sequence
        const int64_t pos0 = j << sh;
        if (pos0 >= past + n || j >= c.W) return;
        const int64_t page = page_id(c, b, (int)j);
        if (page < 0) return;
        const int row0 = (int)(max(past, pos0) - pos0);
        const int row1 = (int)(min(past + n, pos0 + c.page) - pos0);
        if (row0 >= row1) return;
        const int64_t t = t0 + (pos0 + row0 - past);
        append_page<FP8, F16>(c, r, value, h, page, pos0, row0, row1, row0 > 0,
                              value ? v + t * v_stride : k + t * k_stride, value ? v_stride : k_stride);
        return;
    }
    if (!q) return;
    const int pieces = c.D >> 4;
    const int64_t e = (w - n_items) * 64 + (threadIdx.x & 63);
    if (e >= (int64_t)c.T * Hq * pieces) return;
    const int d = (int)(e % pieces) * 16;
    const int64_t th = e / pieces;
    const int h = (int)(th % Hq);
    const int t = (int)(th / Hq);
    // the row's sequence: the last one that starts at or before it and has rows
    int lo = 0, n = c.B;
    while (n > 1) {
        const int m = n >> 1;
        if (min(max(c.off[lo + m], 0), c.T) <= t) { lo += m; n -= m; } else { n = m; }
    }
    const int64_t pos = max((int64_t)max(c.past[lo], 0) + t - min(max(c.off[lo], 0), c.T), (int64_t)0);
    float x[16];
    load_rotated<F16>(r, q + t * q_stride + (int64_t)h * c.D, d, pos, x);
    uint4v o[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i >> 2][i & 3] = pack2<F16>(x[2 * i], x[2 * i + 1]);
    // all of the wave's loads come before its stores: q_out may be q, and a lane
    // reads the other half of a pair that another lane of the wave writes
    __builtin_amdgcn_wave_barrier();
    uint4v* dst = reinterpret_cast<uint4v*>(q_out + t * q_out_stride + (int64_t)h * c.D + d);
    dst[0] = o[0];
    dst[1] = o[1];
}

// Waves: (16-token block of a sequence's rows, head, key or value).
template <bool FP8, bool F16>
__global__ __launch_bounds__(256) void kv_read_kernel(KvView c, uint16_t* __restrict__ k_out,
                                                      uint16_t* __restrict__ v_out, int64_t n_items) {
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= n_items) return;
    const int lane = threadIdx.x & 63;
    const bool value = w & 1;
    const int h = (int)((w >> 1) % c.H);
    const int64_t slot = (w >> 1) / c.H;
    auto first = [](int off, int b) { return (int64_t)(off >> 4) + 2 * (int64_t)b; };
    const int b = seq_of_slot(c, slot, first);
    int t0, n;
    seq_rows(c, b, t0, n);
    const int64_t past = max(c.past[b], 0);
    const int64_t blk = (past >> 4) + (slot - first(t0, b));
    const int64_t pos0 = blk << 4;
    if (pos0 >= past + n) return;
    const int64_t j = pos0 >> c.page_shift;
    const int64_t page = j < c.W ? page_id(c, b, (int)j) : -1;
    const int row0 = (int)(max(past, pos0) - pos0), row1 = (int)(min(past + n, pos0 + 16) - pos0);
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

hipError_t launch_kv_append(const KvView& c, const KvRope& r, const void* k, int64_t k_stride, const void* v,
                            int64_t v_stride, const void* q, int64_t q_stride, int32_t Hq, void* q_out,
                            int64_t q_out_stride, hipStream_t s) {
    const int64_t n_items = ((int64_t)(c.T >> c.page_shift) + 2 * (int64_t)c.B) * c.H * 2;
    const int64_t q_waves = q ? ((int64_t)c.T * Hq * (c.D >> 4) + 63) / 64 : 0;
    const int64_t groups = (n_items + q_waves + 3) / 4;
    if (groups >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    return by_types(c, [&](auto fp8, auto f16) {
        kv_append_kernel<fp8.value, f16.value><<<(uint32_t)groups, 256, 0, s>>>(
            c, r, (const uint16_t*)k, k_stride, (const uint16_t*)v, v_stride, (const uint16_t*)q, q_stride, Hq,
            (uint16_t*)q_out, q_out_stride, n_items);
        return hipGetLastError();
    });
}

hipError_t launch_kv_read(const KvView& c, void* k_out, void* v_out, hipStream_t s) {
    const int64_t n_items = ((int64_t)(c.T >> 4) + 2 * (int64_t)c.B) * c.H * 2;
    const int64_t groups = (n_items + 3) / 4;
    if (groups >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    return by_types(c, [&](auto fp8, auto f16) {
        kv_read_kernel<fp8.value, f16.value>
            <<<(uint32_t)groups, 256, 0, s>>>(c, (uint16_t*)k_out, (uint16_t*)v_out, n_items);
        return hipGetLastError();
    });
}

}  // namespace ls
