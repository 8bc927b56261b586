// Attention over the paged 8-bit KV cache (k_kv.h).
//
// out_i = sum_j softmax_j(scale q_i . k_j) v_j over the tokens j that row i sees.
#include "k_kv.h"

namespace ls {
namespace {

// One wave per row and query head; 64 keys at a time, a lane each.
template <bool FP8, bool F16>
__global__ __launch_bounds__(256) void kv_attend_kernel(KvView c, const uint16_t* __restrict__ q, int64_t q_stride,
                                                        int32_t Hq, float scale, int32_t window, int32_t sinks,
                                                        uint16_t* __restrict__ out, int64_t out_stride) {
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

hipError_t launch_kv_attention(const KvView& c, const void* q, int64_t q_stride, int32_t Hq, float scale,
                               int32_t window, int32_t sinks, void* out, int64_t out_stride, hipStream_t s) {
    const int64_t groups = ((int64_t)c.T * Hq + 3) / 4;
    if (groups >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    return by_types(c, [&](auto fp8, auto f16) {
        kv_attend_kernel<fp8.value, f16.value><<<(uint32_t)groups, 256, 0, s>>>(
            c, (const uint16_t*)q, q_stride, Hq, scale, window, sinks, (uint16_t*)out, out_stride);
        return hipGetLastError();
    });
}

}  // namespace ls
