// Root-mean-square norm of every head of q and k with the rotary positions behind it, its gradient, and the same on the way into a paged cache.
//
// A row x of d channels becomes R (x r (w + offset)), r = (mean x^2 + eps)^-1/2, R the rotation of the row's token.  Back, with g = R^T dy, v = x r, u = g (w + offset):
// dx = r (u - v mean(u v)), and the weight's gradient is the sum of g v over all rows.  Nothing is kept from the way there: x is read for dx anyway, and r is one
// sum of it.  The bound is HBM: rows are read once and written once (back: two read, one written).
#include <algorithm>
#include <cmath>

#include "device_map.h"
#include "paged_cache.h"
#include "rope_common.h"

namespace bs {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxParts = 2048;   // partial sums of the weights' gradients: one per workgroup, eight workgroups on each of 256 CUs

struct NormArgs {
    RopeArgs rope;
    const void *weight[3];         // of each job; null: ones
    int32_t norm[3];               // a job's rows are normed
    int32_t wide;                  // weights in fp32
    int32_t lane_bits;             // lanes of a row
    float eps, offset, inv_d;
    // the gradient: jobs are x and dx
    const void *dy[2];
    int64_t dy_head[2], dy_token[2];
    float *parts;                  // [workgroup][job][d]; null: weights are frozen
    int32_t n_parts;
    float *dweight;                // [job][d]
};

// Channels of a thread: V from lo on and V from hi on, with their angles, N times.  Whole rows lie in 2^lane_bits neighbouring lanes, the smallest power
// of two that has them, so that sums over a row stay within a wave; lanes behind the row's last channels idle.
template <int V, bool HALF, int N>
struct Channels {
    int lo[N], hi[N];
    bool there[N], turns[N];
    float c[N][V], s[N][V];

    __device__ void place(const RopeArgs &a, int g0)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int g = g0 + 64 * n;
            const bool alone = !HALF && V == 1;   // a pair does not fit a piece
            there[n] = g < a.groups;
            turns[n] = g * V < a.pairs;
            lo[n] = turns[n] ? (alone ? 2 * g : V * g) : a.rotary_dim + V * (g - a.pairs / V);
            hi[n] = turns[n] ? lo[n] + (alone ? 1 : a.pairs) : lo[n] + (a.head_dim - a.rotary_dim) / 2;
        }
    }
    __device__ void angles(const RopeArgs &a, int g0, int t)
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                c[n][e] = 1.f;
                s[n][e] = 0.f;
                if (turns[n]) {
                    const int i = HALF || V == 1 ? (g0 + 64 * n) * V + e : (2 * e < V ? lo[n] : hi[n] - V) / 2 + e;
                    rotation(a.quarter_turns[i], a.positions[a.axis[i] * a.axis_stride + t], c[n][e], s[n][e]);
                    c[n][e] *= a.magnitude;
                    s[n][e] *= a.magnitude * a.direction;
                }
            }
    }
    // z: the V channels from lo on, then those from hi on
    __device__ void turn(int n, float (&z)[2 * V]) const
    {
        if (!turns[n]) return;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float &a = HALF ? z[e] : z[2 * e], &b = HALF ? z[V + e] : z[2 * e + 1];
            const float x = a, y = b;
            a = fmaf(x, c[n][e], -y * s[n][e]);
            b = fmaf(y, c[n][e], x * s[n][e]);
        }
    }
};

template <typename T, int V>
__device__ inline void load_row(const T *row, int lo, int hi, bool there, float (&z)[2 * V])
{
    Vec<T, V> u{}, w{};
    if (there) {
        u = *reinterpret_cast<const Vec<T, V> *>(row + lo);
        w = *reinterpret_cast<const Vec<T, V> *>(row + hi);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        z[e] = (float)u.x[e];
        z[V + e] = (float)w.x[e];
    }
}

template <typename T, int V>
__device__ inline void store_row(T *row, int lo, int hi, const float (&z)[2 * V])
{
    Vec<T, V> u, w;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        u.x[e] = (T)z[e];
        w.x[e] = (T)z[V + e];
    }
    *reinterpret_cast<Vec<T, V> *>(row + lo) = u;
    *reinterpret_cast<Vec<T, V> *>(row + hi) = w;
}

template <typename W, int V>
__device__ inline void load_weight_as(const void *weight, int lo, int hi, float (&z)[2 * V])
{
    const W *w = static_cast<const W *>(weight);
    if ((uintptr_t)w % (sizeof(W) * V) == 0) {
        load_row<W, V>(w, lo, hi, true, z);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            z[e] = (float)w[lo + e];
            z[V + e] = (float)w[hi + e];
        }
    }
}

template <int V>
__device__ inline void load_weight(const NormArgs &a, int job, int lo, int hi, bool there, float (&z)[2 * V])
{
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) z[e] = 1.f;
    if (!there || !a.weight[job]) return;
    if (a.wide) load_weight_as<float, V>(a.weight[job], lo, hi, z);
    else load_weight_as<__bf16, V>(a.weight[job], lo, hi, z);
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) z[e] += a.offset;
}

// Over the 2^bits lanes of a row.
__device__ inline float row_sum(float x, int bits)
{
    for (int off = 1 << bits >> 1; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

// One thread: its channels of one token, of heads_each heads.
template <typename T, int V, bool HALF, int N>
__global__ __launch_bounds__(kThreads) void norm_rows(const NormArgs p)
{
    const RopeArgs &a = p.rope;
    const uint32_t idx = blockIdx.x * kThreads + threadIdx.x, per_split = (uint32_t)a.n_tokens << p.lane_bits;
    const int split = (int)(idx / per_split);
    if (split >= a.head_splits) return;
    const int item = (int)(idx - split * per_split);
    const int t = item >> p.lane_bits, g = item & ((1 << p.lane_bits) - 1);
    Channels<V, HALF, N> ch;
    ch.place(a, g);
    ch.angles(a, g, t);
    // where the token's rows go in the cache
    int64_t page_at = -1;
    int at = 0, seq = 0, slot = 0;
    if (a.token_slot) {
        seq = a.token_seq ? a.token_seq[t] : t;
        slot = a.token_slot[t];
        if (seq >= 0 && seq < a.n_seqs && slot >= 0 && slot < a.max_pages * a.page_size) {
            const int page = a.page_table[(int64_t)seq * a.max_pages + slot / a.page_size];
            at = slot % a.page_size;
            if (page >= 0 && page < a.n_pages) page_at = page * a.page_stride;
        }
    }
    const int head = split * a.heads_each, end = min(a.n_heads, head + a.heads_each);
    int first = 0;
    for (int j = 0; j < a.n_jobs; ++j) {
        const RopeJob &job = a.jobs[j];
        const int last = first + job.n_heads;
        if (max(head, first) < min(end, last) && (!job.paged || page_at >= 0)) {
            const T *src = static_cast<const T *>(job.src) + t * job.src_token;
            T *dst = static_cast<T *>(job.dst) + (job.paged ? page_at + at * job.dst_token : t * job.dst_token);
            float w[N][2 * V];
            if (p.norm[j]) {
#pragma unroll
                for (int n = 0; n < N; ++n) load_weight<V>(p, j, ch.lo[n], ch.hi[n], ch.there[n], w[n]);
            }
            for (int h = max(head, first); h < min(end, last); ++h) {
                const T *x = src + (h - first) * job.src_head;
                T *y = dst + (h - first) * job.dst_head;
                if (p.norm[j]) {
                    float z[N][2 * V], sum = 0.f;
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        load_row<T, V>(x, ch.lo[n], ch.hi[n], ch.there[n], z[n]);
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e) sum = fmaf(z[n][e], z[n][e], sum);
                    }
                    const float r = 1.f / sqrtf(fmaf(row_sum(sum, p.lane_bits), p.inv_d, p.eps));
#pragma unroll
                    for (int n = 0; n < N; ++n) {
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e) z[n][e] *= r * w[n][e];
                        if (job.rotate) ch.turn(n, z[n]);
                        if (ch.there[n]) store_row<T, V>(y, ch.lo[n], ch.hi[n], z[n]);
                    }
                } else {
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        if (ch.there[n]) {
                            const Vec<T, V> u = *reinterpret_cast<const Vec<T, V> *>(x + ch.lo[n]), o = *reinterpret_cast<const Vec<T, V> *>(x + ch.hi[n]);
                            *reinterpret_cast<Vec<T, V> *>(y + ch.lo[n]) = u;
                            *reinterpret_cast<Vec<T, V> *>(y + ch.hi[n]) = o;
                        }
                }
                if (job.paged && j == a.n_jobs - 1 && g == 0) {   // (V's rows: once per KV head)
                    const int64_t row = ((int64_t)seq * a.n_kv_heads + (h - first)) * a.row_stride + slot;
                    if (a.weights) a.weights[row] = 0.f;
                    if (a.order) a.order[row] = a.token_order ? a.token_order[t] : slot;
                }
            }
        }
        first = last;
    }
}

// One thread: its channels of one token at a time, of heads_each heads; it adds up its part of the weights' gradients over all of them.
template <typename T, int V, bool HALF, int N>
__global__ __launch_bounds__(kThreads) void norm_grad_rows(const NormArgs p)
{
    const RopeArgs &a = p.rope;
    __shared__ float sums[kWaves][2][2 * BS_ROPE_MAX_PAIRS];
    const uint32_t per_split = (uint32_t)a.n_tokens << p.lane_bits;
    const int g = threadIdx.x & ((1 << p.lane_bits) - 1);
    Channels<V, HALF, N> ch;
    ch.place(a, g);
    float w[2][N][2 * V], dw[2][N][2 * V];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (j < a.n_jobs) load_weight<V>(p, j, ch.lo[n], ch.hi[n], ch.there[n], w[j][n]);
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) dw[j][n][e] = 0.f;
        }
    for (uint64_t idx = (uint64_t)blockIdx.x * kThreads + threadIdx.x; idx < (uint64_t)per_split * a.head_splits; idx += (uint64_t)gridDim.x * kThreads) {
        const int split = (int)(idx / per_split), t = (int)(idx - (uint64_t)split * per_split) >> p.lane_bits;
        ch.angles(a, g, t);
        const int head = split * a.heads_each, end = min(a.n_heads, head + a.heads_each);
        int first = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (j >= a.n_jobs) break;
            const RopeJob &job = a.jobs[j];
            const int last = first + job.n_heads;
            const T *src = static_cast<const T *>(job.src) + t * job.src_token, *dys = static_cast<const T *>(p.dy[j]) + t * p.dy_token[j];
            T *dst = static_cast<T *>(job.dst) + t * job.dst_token;
            for (int h = max(head, first); h < min(end, last); ++h) {
                float x[N][2 * V], u[N][2 * V], square = 0.f, dot = 0.f;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    load_row<T, V>(src + (h - first) * job.src_head, ch.lo[n], ch.hi[n], ch.there[n], x[n]);
                    load_row<T, V>(dys + (h - first) * p.dy_head[j], ch.lo[n], ch.hi[n], ch.there[n], u[n]);
                }
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    ch.turn(n, u[n]);
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) {
                        square = fmaf(x[n][e], x[n][e], square);
                        dot = fmaf(u[n][e] * w[j][n][e], x[n][e], dot);
                    }
                }
                const float r = 1.f / sqrtf(fmaf(row_sum(square, p.lane_bits), p.inv_d, p.eps));
                const float k = row_sum(dot, p.lane_bits) * p.inv_d * r * r;   // mean(u v) r
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    float z[2 * V];
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) {
                        z[e] = r * fmaf(-x[n][e], k, u[n][e] * w[j][n][e]);
                        dw[j][n][e] = fmaf(u[n][e], x[n][e] * r, dw[j][n][e]);
                    }
                    if (ch.there[n]) store_row<T, V>(dst + (h - first) * job.dst_head, ch.lo[n], ch.hi[n], z);
                }
            }
            first = last;
        }
    }
    if (!p.parts) return;
    // over the rows of a wave, then the waves: always in the same order
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) {
                float x = dw[j][n][e];
                for (int off = 1 << p.lane_bits; off < 64; off <<= 1) x += __shfl_xor(x, off, 64);
                if (lane == g && ch.there[n]) sums[threadIdx.x >> 6][j][(e < V ? ch.lo[n] + e : ch.hi[n] + e - V)] = x;
            }
    __syncthreads();
    for (int i = threadIdx.x; i < a.n_jobs * a.head_dim; i += kThreads) {
        const int j = i / a.head_dim, c = i - j * a.head_dim;
        float x = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) x += sums[v][j][c];
        (p.n_parts == 1 ? p.dweight : p.parts + (int64_t)blockIdx.x * a.n_jobs * a.head_dim)[i] = x;
    }
}

// Sums of the workgroups, in 64 bits and always in the same order: a workgroup takes 16 of the n_jobs d channels, 64 threads each.
__global__ __launch_bounds__(1024) void norm_grad_join(const float *__restrict__ parts, int n_parts, int n, float *__restrict__ dweight)
{
    __shared__ double sums[64][16];
    const int c = threadIdx.x & 15, v = threadIdx.x >> 4, i = blockIdx.x * 16 + c;
    double x = 0.0;
    for (int k0 = v; k0 < n_parts; k0 += 8 * 64) {   // loads of eight parts go out together
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = i < n && k0 + 64 * k < n_parts ? parts[(int64_t)(k0 + 64 * k) * n + i] : 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) x += y[k];
    }
    sums[v][c] = x;
    __syncthreads();
    if (v > 0 || i >= n) return;
    for (int k = 1; k < 64; ++k) x += sums[k][c];
    dweight[i] = (float)x;
}

template <typename T, int V, bool HALF, int N>
hipError_t launch_rows(const NormArgs &p, bool gradient, dim3 grid, hipStream_t st)
{
    return gradient ? launch_kernel(norm_grad_rows<T, V, HALF, N>, grid, dim3(kThreads), 0, st, p) : launch_kernel(norm_rows<T, V, HALF, N>, grid, dim3(kThreads), 0, st, p);
}

template <typename T, bool HALF>
hipError_t launch_layout(const NormArgs &p, int vec, bool gradient, dim3 grid, hipStream_t st)
{
    switch (vec) {
    case 8: if constexpr (sizeof(T) == 2) return launch_rows<T, 8, HALF, 1>(p, gradient, grid, st); else return hipErrorInvalidValue;
    case 4: return launch_rows<T, 4, HALF, 1>(p, gradient, grid, st);
    case 2: return launch_rows<T, 2, HALF, 1>(p, gradient, grid, st);
    default: return p.rope.groups <= 64 ? launch_rows<T, 1, HALF, 1>(p, gradient, grid, st) : launch_rows<T, 1, HALF, 2>(p, gradient, grid, st);
    }
}

int check_norm(const bs_norm *norm)
{
    if (!norm || !(norm->eps >= 1.17549435e-38f) || !std::isfinite(norm->eps) || !std::isfinite(norm->offset)) return BS_EINVAL;
    if (norm->weight_dtype != BS_BF16 && norm->weight_dtype != BS_F32) return BS_EUNSUPPORTED;
    return ((uintptr_t)norm->weight[0] | (uintptr_t)norm->weight[1]) % element_bytes(norm->weight_dtype) != 0 ? BS_EINVAL : BS_OK;
}

// Jobs, their norms and the rotation are set; `gradient`: dy and parts as well.
int run_norm(NormArgs &p, const bs_norm &norm, const bs_rope *rope, int32_t dtype, int32_t head_dim, bool gradient, hipStream_t st)
{
    RopeArgs &a = p.rope;
    int vec = fill_rope(a, rope, dtype, head_dim, gradient);
    const int e = element_bytes(dtype);
    for (int j = 0; gradient && j < a.n_jobs; ++j)
        while (vec > 1 && ((uintptr_t)p.dy[j] % (e * vec) != 0 || p.dy_head[j] % vec != 0 || p.dy_token[j] % vec != 0)) vec /= 2;
    a.groups = head_dim / (2 * vec);
    while (1 << p.lane_bits < std::min(a.groups, 64)) ++p.lane_bits;
    p.wide = norm.weight_dtype == BS_F32;
    p.eps = norm.eps;
    p.offset = norm.offset;
    p.inv_d = 1.f / head_dim;
    // Heads share a thread's angles and weights; where there are too few tokens to fill the chip they are split over threads.
    const int64_t items = (int64_t)a.n_tokens << p.lane_bits;
    if (items > INT32_MAX) return BS_EUNSUPPORTED;   // (with several splits there are few, so threads are counted in 32 bits)
    hipError_t err = hipSuccess;
    if (items > 0) {
        a.head_splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(a.n_heads, (256 * 2048 + items - 1) / items));
        a.heads_each = (a.n_heads + a.head_splits - 1) / a.head_splits;
        a.head_splits = (a.n_heads + a.heads_each - 1) / a.heads_each;
        int64_t wgs = (items * a.head_splits + kThreads - 1) / kThreads;
        if (gradient) wgs = std::min<int64_t>(wgs, kMaxParts);
        p.n_parts = (int32_t)std::min<int64_t>(wgs, kMaxParts);
        const bool half = !rope || rope->layout == BS_ROPE_HALF;
        const dim3 grid((unsigned)wgs);
        if (dtype == BS_BF16) err = half ? launch_layout<__bf16, true>(p, vec, gradient, grid, st) : launch_layout<__bf16, false>(p, vec, gradient, grid, st);
        else err = half ? launch_layout<float, true>(p, vec, gradient, grid, st) : launch_layout<float, false>(p, vec, gradient, grid, st);
        if (err != hipSuccess) return fail_hip(err, "norm_rows launch");
    }
    if (gradient && p.dweight && p.n_parts != 1) {   // (no tokens: sums of nothing)
        const int n = a.n_jobs * head_dim;
        err = launch_kernel(norm_grad_join, dim3((unsigned)((n + 15) / 16)), dim3(1024), 0, st, p.parts, p.n_parts, n, p.dweight);
    }
    return err == hipSuccess ? BS_OK : fail_hip(err, "norm_grad_join launch");
}

// Heads of x and y, element for element; the sizes that both directions check.
int check_call(const bs_heads *x, const bs_heads *y, int32_t n_tensors, int32_t dtype, int32_t n_tokens, int32_t head_dim)
{
    for (int i = 0; i < n_tensors; ++i) {
        if (check_heads(&x[i], n_tokens == 0) || check_heads(&y[i], n_tokens == 0) || x[i].n_heads != y[i].n_heads || x[i].n_heads > (1 << 20)) return BS_EINVAL;
        if (((uintptr_t)x[i].data | (uintptr_t)y[i].data) % element_bytes(dtype) != 0 || check_rows_apart(y[i], n_tokens, head_dim)) return BS_EINVAL;
    }
    return BS_OK;
}

int check_sizes(int32_t n_tensors, int32_t dtype, int32_t n_tokens, int32_t head_dim)
{
    if (n_tensors < 1 || n_tensors > 2 || n_tokens < 0 || head_dim < 2 || head_dim % 2 != 0 || head_dim > 2 * BS_ROPE_MAX_PAIRS) return BS_EINVAL;
    return dtype != BS_BF16 && dtype != BS_F32 ? BS_EUNSUPPORTED : BS_OK;
}

}  // namespace
}  // namespace bs

extern "C" int bs_norm_rope(const bs_norm *norm, const bs_rope *rope, const bs_heads *x, const bs_heads *y, int32_t n_tensors, int32_t dtype, int32_t n_tokens,
                            int32_t head_dim, const int32_t *positions, int64_t axis_stride, void *stream)
{
    using namespace bs;
    if (!x || !y) return BS_EINVAL;
    if (int rc = check_sizes(n_tensors, dtype, n_tokens, head_dim)) return rc;
    if (int rc = check_norm(norm)) return rc;
    if (rope)
        if (int rc = check_rope(rope, n_tokens, head_dim, positions, axis_stride)) return rc;
    if (int rc = check_call(x, y, n_tensors, dtype, n_tokens, head_dim)) return rc;
    NormArgs p{};
    RopeArgs &a = p.rope;
    a.n_jobs = n_tensors;
    for (int i = 0; i < n_tensors; ++i) {
        a.jobs[i] = job_of(x[i], y[i], rope != nullptr);
        p.weight[i] = norm->weight[i];
        p.norm[i] = 1;
    }
    a.n_tokens = n_tokens;
    a.positions = positions;
    a.axis_stride = axis_stride;
    return run_norm(p, *norm, rope, dtype, head_dim, false, (hipStream_t)stream);
}

extern "C" int64_t bs_norm_rope_grad_workspace(int32_t n_tensors, int32_t dtype, int32_t n_tokens, int32_t head_dim)
{
    using namespace bs;
    if (int rc = check_sizes(n_tensors, dtype, n_tokens, head_dim)) return rc;
    return (int64_t)kMaxParts * n_tensors * head_dim * 4;
}

extern "C" int bs_norm_rope_grad(const bs_norm *norm, const bs_rope *rope, const bs_heads *x, const bs_heads *dy, const bs_heads *dx, float *dweight, int32_t n_tensors,
                                 int32_t dtype, int32_t n_tokens, int32_t head_dim, const int32_t *positions, int64_t axis_stride, void *workspace,
                                 int64_t workspace_bytes, void *stream)
{
    using namespace bs;
    if (!x || !dy || !dx) return BS_EINVAL;
    if (int rc = check_sizes(n_tensors, dtype, n_tokens, head_dim)) return rc;
    if (int rc = check_norm(norm)) return rc;
    if (rope)
        if (int rc = check_rope(rope, n_tokens, head_dim, positions, axis_stride)) return rc;
    if (int rc = check_call(x, dx, n_tensors, dtype, n_tokens, head_dim)) return rc;
    if ((uintptr_t)dweight % 4 != 0) return BS_EINVAL;
    if (dweight && (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < (int64_t)kMaxParts * n_tensors * head_dim * 4)) return BS_EINVAL;
    NormArgs p{};
    RopeArgs &a = p.rope;
    a.n_jobs = n_tensors;
    for (int i = 0; i < n_tensors; ++i) {
        if (check_heads(&dy[i], n_tokens == 0) || dy[i].n_heads != x[i].n_heads || (uintptr_t)dy[i].data % element_bytes(dtype) != 0) return BS_EINVAL;
        a.jobs[i] = job_of(x[i], dx[i], rope != nullptr);
        p.weight[i] = norm->weight[i];
        p.dy[i] = dy[i].data;
        p.dy_head[i] = dy[i].head_stride;
        p.dy_token[i] = dy[i].token_stride;
    }
    a.n_tokens = n_tokens;
    a.positions = positions;
    a.axis_stride = axis_stride;
    p.dweight = dweight;
    p.parts = dweight ? static_cast<float *>(workspace) : nullptr;
    return run_norm(p, *norm, rope, dtype, head_dim, true, (hipStream_t)stream);
}

extern "C" int bs_cache_append_norm(const bs_cache *cache, const bs_heads *k, const bs_heads *v, int32_t n_tokens, const int32_t *token_seq, const int32_t *token_slot,
                                    const bs_norm *norm, const bs_rope *rope, const int32_t *positions, int64_t axis_stride, const bs_heads *q, const bs_heads *q_out,
                                    const bs_slots *slots, const int32_t *token_order, void *stream)
{
    using namespace bs;
    NormArgs p{};
    RopeArgs &a = p.rope;
    if (int rc = check_norm(norm)) return rc;
    if (int rc = append_args(&a, cache, k, v, n_tokens, token_seq, token_slot, rope, positions, axis_stride, q, q_out, slots, token_order)) return rc;
    if (cache->n_kv_heads > (1 << 20)) return BS_EUNSUPPORTED;
    const int k_job = a.n_jobs - 2;
    for (int j = 0; j <= k_job; ++j) {
        a.jobs[j].rotate = rope != nullptr;
        p.norm[j] = 1;
        p.weight[j] = norm->weight[j == k_job];
    }
    return run_norm(p, *norm, rope, cache->dtype, cache->head_dim, false, (hipStream_t)stream);
}
