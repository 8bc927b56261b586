// Device helpers of the paged 8-bit KV cache: 8-bit codes, tile layout, the
// lookup from a launch's work slots to sequences, wave reductions.
//
// Layout.  A page holds, per head, tiles of 16 tokens x 64 dimensions, 1 KB
// each: keys [16 tokens][64], values [4][64][4 tokens].  One 16-byte load per
// lane reads a tile with a wave, and what a lane gets is an operand of the
// 16x16x32 matrix instruction as it stands: 16 dimensions of one token for
// q.k, and for p.v four tokens of four dimensions, the token order in which the
// scores' result registers hold them.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <type_traits>

#include "ls_internal.h"
#include "ls_kv_slots.h"

namespace ls {

using half8 = _Float16 __attribute__((ext_vector_type(8)));
using half4 = _Float16 __attribute__((ext_vector_type(4)));
using half2v = _Float16 __attribute__((ext_vector_type(2)));
using float4v = float __attribute__((ext_vector_type(4)));
using float2v = float __attribute__((ext_vector_type(2)));
using uint4v = uint32_t __attribute__((ext_vector_type(4)));
using uint2v = uint32_t __attribute__((ext_vector_type(2)));

constexpr float kScaleMin = 0x1p-64f, kScaleMax = 0x1p+64f;

// ---- 16-bit tensors ----------------------------------------------------------
// Two elements of a dword as floats, and back (round to nearest, ties to even).
template <bool F16>
__device__ __forceinline__ float2v unpack2(uint32_t w) {
    if constexpr (F16) {
        const half2v h = __builtin_bit_cast(half2v, w);
        return float2v{(float)h.x, (float)h.y};
    } else {
        return float2v{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)};
    }
}

template <bool F16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (F16) {
        const half2v h = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, h);
    } else {
        using bf2 = __bf16 __attribute__((ext_vector_type(2)));
        const bf2 h = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, h);
    }
}

// ---- 8-bit codes ---------------------------------------------------------------
// Four codes of a dword as floats.
template <bool FP8>
__device__ __forceinline__ float4v code_values(uint32_t w) {
    if constexpr (FP8) {
        const float2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        const float2v b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        return float4v{a.x, a.y, b.x, b.y};
    } else {
        return float4v{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)};
    }
}

// Four scaled values as codes: saturated, rounded to nearest with ties to even.
template <bool FP8>
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
    constexpr float M = FP8 ? 448.0f : 127.0f;
    a = fminf(fmaxf(a, -M), M);
    b = fminf(fmaxf(b, -M), M);
    c = fminf(fmaxf(c, -M), M);
    d = fminf(fmaxf(d, -M), M);
    if constexpr (FP8) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        return ((uint32_t)(int)rintf(a) & 255u) | ((uint32_t)(int)rintf(b) & 255u) << 8 |
               ((uint32_t)(int)rintf(c) & 255u) << 16 | (uint32_t)(int)rintf(d) << 24;
    }
}

// The scale of a largest magnitude a >= 0 (finite).  FP8: the smallest power of
// two s with a <= 448 s; 448 = 0.875 * 2^9.
template <bool FP8>
__device__ __forceinline__ float scale_of(float a) {
    float s;
    if constexpr (FP8) {
        const uint32_t u = __float_as_uint(a);
        const int e = (int)(u >> 23) - 126 - ((u & 0x7FFFFFu) <= 0x600000u ? 9 : 8);
        s = __uint_as_float((uint32_t)(min(max(e, -64), 64) + 127) << 23);
    } else {
        s = a / 127.0f;
    }
    return fminf(fmaxf(s, kScaleMin), kScaleMax);
}

// Four codes of a dword in half precision: exact, every code is a half value.
template <bool FP8>
__device__ __forceinline__ half4 code_halves(uint32_t w) {
    if constexpr (FP8) {
        const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false);
        const half2v b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true);
        return half4{a.x, a.y, b.x, b.y};
    } else {
        // 0x6400 | u is 1024 + u: the biased code as a half's mantissa, then the bias and the 1024 off
        const uint32_t u = w ^ 0x80808080u;
        const half2v off = {(_Float16)1152.0f, (_Float16)1152.0f};
        const half2v a = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off;
        const half2v b = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off;
        return half4{a.x, a.y, b.x, b.y};
    }
}

template <bool FP8>
__device__ __forceinline__ half8 code_halves8(uint32_t lo, uint32_t hi) {
    const half4 a = code_halves<FP8>(lo), b = code_halves<FP8>(hi);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// ---- addresses -------------------------------------------------------------------
// Byte offset of 16-token block `blk` of a page and head.
__device__ __forceinline__ int64_t block_at(const KvView& c, int64_t page, int h, int blk) {
    return ((page * c.H + h) * c.page + blk * 16) * c.D;
}

// Page id of the sequence's page j, or -1 (absent, outside the pool, outside the table).
__device__ __forceinline__ int64_t page_id(const KvView& c, int b, int j) {
    if (j < 0 || j >= c.W) return -1;
    const int32_t p = c.pages[(int64_t)b * c.W + j];
    return p >= 0 && p < c.n_pages ? p : -1;
}

// A sequence's rows [t0, t0 + n) of the call's tensors, whatever the offsets hold.
__device__ __forceinline__ void seq_rows(const KvView& c, int b, int& t0, int& n) {
    t0 = min(max(c.off[b], 0), c.T);
    n = min(max(c.off[b + 1], t0), c.T) - t0;
}

// The sequence that owns work slot `slot` when sequence b's slots start at
// first(off[b], b), non-decreasing in b: a 64-way search by the whole wave.  Slots
// before sequence 0's first give 0.
template <class F>
__device__ __forceinline__ int seq_of_slot(const KvView& c, int64_t slot, F first) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = c.B;
    while (n > 1) {
        const int step = (n + 63) >> 6;
        const int i = lane * step;
        const bool le = i < n && first(min(max(c.off[lo + i], 0), c.T), lo + i) <= slot;
        const uint64_t m = __ballot(le);
        const int k = m ? 63 - __clzll((long long)m) : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Sums of a lane and those below it.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);    // the row's lane 1, 2, 4, 8 below
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);    // row ends to the rows above
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);
    return x;
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}

// Calls f with the code type and the tensors' type as compile-time constants.
template <class F>
hipError_t by_types(const KvView& c, F f) {
    if (c.fp8) return c.f16 ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
    return c.f16 ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

}  // namespace ls
