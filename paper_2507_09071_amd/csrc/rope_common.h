// What the kernels that rotate heads have in common: rotary positions alone, into a cache, behind a norm (internal to the library).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "blindsight.h"

namespace bs {

// Heads that are rotated or copied.
struct RopeJob {
    const void *src;
    void *dst;
    int64_t src_head, src_token, dst_head, dst_token;
    int32_t n_heads;
    int32_t rotate, paged;   // paged: dst is a pool of pages, dst_token the stride of a slot
};

struct RopeArgs {
    RopeJob jobs[3];
    int32_t n_jobs, n_heads;       // heads of all jobs
    int32_t n_tokens, groups;      // groups of channels per token that a thread takes
    int32_t pairs, rotary_dim, head_dim;
    int32_t head_splits, heads_each;
    const int32_t *positions;
    int64_t axis_stride;
    float magnitude;
    float direction;               // of the sines: 1 or -1
    // pages
    const int32_t *token_seq, *token_slot, *token_order, *page_table;
    int32_t n_seqs, max_pages, page_size, n_pages, n_kv_heads;
    int64_t page_stride;
    float *weights;
    int32_t *order;
    int64_t row_stride;
    double quarter_turns[BS_ROPE_MAX_PAIRS];   // per position: freq * 2 / pi
    uint8_t axis[BS_ROPE_MAX_PAIRS];
};

template <typename T, int V>
struct __align__(sizeof(T) * V) Vec { T x[V]; };

// cos and sin of position * quarter_turns * (pi / 2): the multiple of a quarter turn is taken off in 64 bits, and the rest, at most
// half a quarter turn, goes through the series of sine and cosine in fp32: the first term left out is below 1.8e-9 (sine) and 1.2e-10 (cosine), what fp32
// rounds on the way is up to 6.6e-8, about 2^-24.  The 64-bit angle is off by at most 3 |angle| 2^-53: 1e-9 at three million radians, 7e-7 at 2^31.
__device__ inline void rotation(double quarter_turns, int32_t position, float &c, float &s)
{
    const double t = quarter_turns * (double)position, n = rint(t);
    const float x = (float)((t - n) * 1.5707963267948966);
    const float x2 = x * x;
    const float sn = x + x * x2 * fmaf(x2, fmaf(x2, fmaf(x2, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f);
    const float cs = 1.f + x2 * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f);
    const int q = (int)(n - 4.0 * floor(n * 0.25));   // which quarter
    c = (q & 1) ? sn : cs;
    s = (q & 1) ? cs : sn;
    if (q == 1 || q == 2) c = -c;
    if (q >= 2) s = -s;
}

// Checks of a rotation's arguments, and what bs_cache_append and its kind are called with: fills in the jobs (q, if there is one, then K, then V) and the pages.
int check_rope(const bs_rope *r, int32_t n_tokens, int32_t head_dim, const int32_t *positions, int64_t axis_stride);
RopeJob job_of(const bs_heads &x, const bs_heads &y, bool rotate);
int append_args(RopeArgs *a, const bs_cache *cache, const bs_heads *k, const bs_heads *v, int32_t n_tokens, const int32_t *token_seq, const int32_t *token_slot,
                const bs_rope *rope, const int32_t *positions, int64_t axis_stride, const bs_heads *q, const bs_heads *q_out, const bs_slots *slots,
                const int32_t *token_order);
// The rotation, the heads of all jobs, and the channels that a thread takes at a time (returned).
int fill_rope(RopeArgs &a, const bs_rope *rope, int32_t dtype, int32_t head_dim, bool inverse);

}  // namespace bs
