// What the kernels of attention over the paged 8-bit KV cache share: the tokens
// that rows see, where their pages lie, the reference of a row's weights, partial
// sums of split rows.
#pragma once

#include "k_kv.h"

namespace ls {
namespace {

struct AttnCall {
    const uint16_t* q;
    uint16_t* out;
    int64_t q_stride, out_stride;
    int32_t G;                       // query heads of a kv head
    float scale2;                    // softmax scale * log2 e
    int32_t window, sinks;
};

// What a sequence's rows see, in 16-token blocks: the first n_sink and those from
// win on, n in all; block i of them is tile(i).
struct Span {
    int32_t n_sink, win, n;
    __device__ __forceinline__ int32_t tile(int32_t i) const { return i < n_sink ? i : win + (i - n_sink); }
};

__device__ __forceinline__ Span span_of(const KvView& c, const AttnCall& a, int32_t past, int32_t rows) {
    const int32_t end = min(past + rows, c.limit);
    const int32_t lo = a.window > 0 ? min(max(past + 1 - a.window, 0), end) : 0;
    Span s;
    s.win = lo >> 4;
    s.n_sink = (min(a.sinks, lo) + 15) >> 4;
    if (s.n_sink >= s.win) s.n_sink = s.win = 0;
    s.n = s.n_sink + ((end + 15) >> 4) - s.win;
    return s;
}

// Positions fit 32 bits: tables end at 2^30 tokens, and a past beyond that counts as that.
constexpr int32_t kMaxPast = 1 << 30;
__device__ __forceinline__ int32_t past_of(const KvView& c, int b) { return min(max(c.past[b], 0), kMaxPast); }

// Which of a block's 16 tokens a row sees: up to `last`, and those after `gone` or
// before `sink`.  Bounds are relative to the block, so 32 bits do; the tests are
// joined without branches.
struct Sight {
    int32_t last, gone, sink;
    __device__ __forceinline__ bool sees(int i) const { return (i <= last) & ((i > gone) | (i < sink)); }
};
__device__ __forceinline__ Sight sight(const AttnCall& a, int32_t page, int32_t pos, int32_t tok) {
    Sight s;
    s.last = page < 0 ? -1 : pos - tok;
    s.gone = a.window > 0 ? max(pos - a.window, -1) - tok : -1;
    s.sink = a.sinks - tok;
    return s;
}

// Bytes of four tokens' value codes, from token `tok` on, that enter the product: those
// before `end` that some row sees, `lo` being where the window of the first row
// starts.  The others belong to nobody or are hidden, and may be NaN.
__device__ __forceinline__ uint32_t first_bytes(int32_t n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1; }
__device__ __forceinline__ uint32_t kept_bytes(const AttnCall& a, int32_t tok, int32_t lo, int32_t end) {
    uint32_t m = first_bytes(end - tok);
    if (a.window > 0) m &= ~first_bytes(lo - tok) | first_bytes(a.sinks - tok);
    return m;
}

// The pages of one sequence and kv head: where a 16-token block of it lies.
struct Blocks {
    const int32_t* pages;            // the sequence's row of the table
    int32_t n_blocks;                // blocks that the row covers
    int32_t n_pages, shift, mask;    // 16-token blocks of a page: 2^shift
    int64_t page_bytes;
    int32_t block_bytes, H;
    const uint8_t *k, *v;
    const float *ks, *vs;
    __device__ __forceinline__ Blocks(const KvView& c, int b, int h)
        : pages(c.pages + (int64_t)b * c.W), n_blocks(c.limit >> 4), n_pages((int32_t)c.n_pages), shift(c.page_shift - 4),
          mask((c.page >> 4) - 1), page_bytes((int64_t)c.H * c.page * c.D), block_bytes(16 * c.D), H(c.H),
          k(c.k + (int64_t)h * c.page * c.D), v(c.v + (int64_t)h * c.page * c.D), ks(c.ks + h), vs(c.vs + h) {}
    // Offset of its codes; of some codes for an absent one.
    __device__ __forceinline__ int64_t at(int32_t page, int32_t blk) const {
        return (int64_t)max(page, 0) * page_bytes + (blk & mask) * block_bytes;
    }
};

constexpr int kMaxParts = 8192;        // of a launch that cuts segments
constexpr int kUnit = 8;             // 16-token blocks of a work unit: two for each wave of a workgroup
constexpr int kJoin = 16;            // parts that one workgroup adds
// Segments of up to this many units stay whole.  4 and 16: 12 windows of 4,096 tokens 19.0 and 19.1 us, 64 decoding
// sequences 51.0 and 53.5; 8: 16.9 and 50.9.
constexpr int kMinUnits = 8;
constexpr float kNoMax = -3e38f;     // reference of nothing: below every logit
// A logit's weight is 2^(logit - reference).  log2 of a row's largest weight when the
// reference moves up: all of a lane's tokens of a step (8 and 32) may have it within
// kMostWeight, and later ones twice and eight times that.
constexpr float kSplitTop = 12.0f, kTileTop = 8.0f;
// The reference under which a largest logit mx has that weight; from 2^26 on, where the
// difference could be rounded to 16, the weight 1.
__device__ __forceinline__ float raised(float m, float mx, float top) { return fmaxf(m, fabsf(mx) < 0x1p+26f ? mx - top : mx); }
// Bounds of the sum of a lane's weights in a step (8 or 32 tokens), beyond which the reference
// may move.  No weight is too large for a half; and an error of 2^-25, where a weight has less
// than 11 bits, is 2^-16 of the sum.  Steps that the mask cuts have lanes with one token or
// two, often small ones: there it is 2^-11.  Measured against no lower bound: 3 prompts of 64
// dimensions under a window of 1,024 124 -> 125 to 131 us, a mixed step 61.6 -> 62.7, the
// others 0 to 2 %.
constexpr float kMostWeight = 0x1.ffp+15f;
constexpr float kLeast = -9.0f, kLeastCut = -14.0f;       // log2
__device__ __forceinline__ bool off_range(float sum, bool cut) {
    return (sum > kMostWeight) | ((sum < (cut ? 0x1p-14f : 0x1p-9f)) & (sum > 0.0f));
}
// Whether all weights of a row in the step are below that, mx being its largest logit and m the reference.
__device__ __forceinline__ bool is_low(float m, float mx, bool cut) {
    return (mx - m < (cut ? kLeastCut : kLeast)) & (mx > -INFINITY);
}
// The reference that makes the largest 1, as far as the sums have room, `most` being their largest magnitude.
__device__ __forceinline__ float lowered(float m, float mx, float most) {
    const float room = fmaxf(100.0f - __builtin_amdgcn_logf(fmaxf(most, 1.0f)), 0.0f);
    return fmaxf(mx, m - room);
}

// Power of two that brings a row of bf16 queries whose largest magnitude has the
// bits `top` below 2^14, and its reciprocal.  Above 2^-100 only: smaller rows
// round to zero scores in fp32 anyway.
__device__ __forceinline__ float half_range_factor(uint32_t top) {
    return __uint_as_float((uint32_t)(267 - max((int)(top >> 23), 27)) << 23);
}
__device__ __forceinline__ float half_range_undo(uint32_t top) {
    return __uint_as_float((uint32_t)(max((int)(top >> 23), 27) - 13) << 23);
}

// Two floats to, and from, memory that other workgroups of the launch read and
// write: past the caches that each XCD has for itself.  A fence would write back and
// drop that whole cache instead, in every workgroup: twice the kernel's time.
__device__ __forceinline__ void put_shared(float* p, float2v x) {
    __hip_atomic_store((uint64_t*)p, __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2v get_shared(const float* p) {
    return __builtin_bit_cast(float2v, __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Counts the workgroup's part as written; whether it was the last of `members`,
// whose parts are then all to be read here.  Nobody waits.  The last one leaves the
// count at zero for the next launch.
__device__ __forceinline__ bool arrive(uint32_t* count, int members) {
    __shared__ int is_last;
    // every thread's stores are past the caches before any of them passes the barrier
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        is_last = before == (uint32_t)members - 1;
        if (is_last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return is_last;
}

}  // namespace
}  // namespace ls
