// Root-mean-square norm of every head of q and k with the rotary positions behind it, its gradient, and the same on the way into a paged cache.
//
// A row x of d channels becomes R (x r (w + offset)), r = (mean x^2 + eps)^-1/2, R the rotation of the row's token.  Back, with g = R^T dy, v = x r, u = g (w + offset):
// dx = r (u - v mean(u v)), and the weight's gradient is the sum of g v over all rows.  Nothing is kept from the way there: x is read for dx anyway, and r is one
// sum of it.  The bound is HBM: rows are read once and written once (back: two read, one written).  39.5K tokens of 28 + 4 heads, d 128, bf16: 648 MB in 122 us and
// back 971 MB in 191 + 6 for the weights' sums, 5.3 and 5.1 TB/s, where a copy reaches 5.3; in fp32 5K tokens of them, 369 MB back in 77 + 4.5 us.  A decoding step is
// the latency of a row behind its length, its page and its angles, which all but the page are loaded at once: 5.4 us on its own, 6.3 into the cache; the prompt of 39.5K tokens
// into the cache, q, k and v token by token, 729 MB: 145 us, 5.0 TB/s, in both orders of a page's axes.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device_map.h"
#include "paged_cache.h"
#include "rope_common.h"

namespace bs {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxParts = 2048;   // partial sums of the weights' gradients: one per workgroup, eight workgroups on each of 256 CUs

struct NormArgs {
    int32_t split_end[2];          // where the splits of the first, of the second job end
    int32_t lane_bits, n_axes;     // lanes of a row: 2^lane_bits
    RopeArgs rope;
    const void *weight[3];         // of each job; null: ones
    int32_t norm[3];               // a job's rows are normed
    int32_t wide;                  // weights in fp32
    float eps, offset, inv_d;
    // the gradient: jobs are x and dx
    const void *dy[2];
    int64_t dy_head[2], dy_token[2];
    float *parts;                  // [workgroup][d]; null: weights are frozen
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
    // All loads of it go out together: the positions on all axes, and which of them turns a pair, do not wait for each other.
    __device__ void angles(const NormArgs &p, int g0, int t)
    {
        const RopeArgs &a = p.rope;
        int32_t at[BS_ROPE_MAX_AXES];
#pragma unroll
        for (int x = 0; x < BS_ROPE_MAX_AXES; ++x) at[x] = a.positions[min(x, p.n_axes - 1) * a.axis_stride + t];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            constexpr bool kWhole = HALF || V == 1;
            constexpr int H = kWhole ? V : V / 2;   // pairs that lie together: all, or those of lo and those of hi
            const int i0 = turns[n] ? (kWhole ? (g0 + 64 * n) * V : lo[n] / 2) : 0, i1 = kWhole || !turns[n] ? 0 : hi[n] / 2;
            double f[V];
            int x[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int i = e < H ? i0 + e : i1 + e - H;
                f[e] = a.quarter_turns[i];
                x[e] = a.axis[i];
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                rotation(f[e], x[e] == 0 ? at[0] : x[e] == 1 ? at[1] : x[e] == 2 ? at[2] : at[3], c[n][e], s[n][e]);
                c[n][e] = turns[n] ? c[n][e] * a.magnitude : 1.f;
                s[n][e] = turns[n] ? s[n][e] * a.magnitude * a.direction : 0.f;
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

// A thread's channels of a row as they are in memory.
template <typename T, int V, int N>
struct Pieces {
    Vec<T, V> lo[N], hi[N];
    template <typename C>
    __device__ void load(const T *row, const C &ch)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            lo[n] = hi[n] = Vec<T, V>{};
            if (ch.there[n]) {
                lo[n] = *reinterpret_cast<const Vec<T, V> *>(row + ch.lo[n]);
                hi[n] = *reinterpret_cast<const Vec<T, V> *>(row + ch.hi[n]);
            }
        }
    }
    template <typename C>
    __device__ void store(T *row, const C &ch) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (ch.there[n]) {
                *reinterpret_cast<Vec<T, V> *>(row + ch.lo[n]) = lo[n];
                *reinterpret_cast<Vec<T, V> *>(row + ch.hi[n]) = hi[n];
            }
    }
    __device__ void get(int n, float (&z)[2 * V]) const
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            z[e] = (float)lo[n].x[e];
            z[V + e] = (float)hi[n].x[e];
        }
    }
    __device__ void set(int n, const float (&z)[2 * V])
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            lo[n].x[e] = (T)z[e];
            hi[n].x[e] = (T)z[V + e];
        }
    }
};

template <typename W, int V>
__device__ inline void load_weight_as(const void *weight, int lo, int hi, float (&z)[2 * V])
{
    const W *w = static_cast<const W *>(weight);
    if ((uintptr_t)w % (sizeof(W) * V) == 0) {
        const Vec<W, V> u = *reinterpret_cast<const Vec<W, V> *>(w + lo), o = *reinterpret_cast<const Vec<W, V> *>(w + hi);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            z[e] = (float)u.x[e];
            z[V + e] = (float)o.x[e];
        }
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

// Sum over the 2^bits lanes of a row, in each of them: neighbours, quads, eights and sixteens by data-parallel moves, beyond that by swaps of half rows.
__device__ inline float row_sum(float x, int bits)
{
    const auto moved = [](float y, auto control) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), decltype(control)::value, 0xf, 0xf, true));
    };
    if (bits > 0) x += moved(x, std::integral_constant<int, 0xb1>{});    // lanes 1 0 3 2
    if (bits > 1) x += moved(x, std::integral_constant<int, 0x4e>{});    // lanes 2 3 0 1
    if (bits > 2) x += moved(x, std::integral_constant<int, 0x141>{});   // eight lanes reversed
    if (bits > 3) x += moved(x, std::integral_constant<int, 0x140>{});   // sixteen lanes reversed
    if (bits > 4) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (bits > 5) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return x;
}

// 1 / rms, off by at most one unit in the last place (the argument is a normal number: eps is).
__device__ inline float inverse_rms(float sum, const NormArgs &p) { return __builtin_amdgcn_rsqf(fmaf(row_sum(sum, p.lane_bits), p.inv_d, p.eps)); }

// The job and heads of a split (blockIdx.y).
struct Share { int job, first, last; };
__device__ inline Share share_of(const NormArgs &p, int split)
{
    Share w;
    w.job = split < p.split_end[0] ? 0 : split < p.split_end[1] ? 1 : 2;
    w.first = (split - (w.job > 0 ? p.split_end[w.job - 1] : 0)) * p.rope.heads_each;
    w.last = min(w.first + p.rope.heads_each, p.rope.jobs[w.job].n_heads);
    return w;
}

// One thread: its channels of one token, of heads_each heads of one job (blockIdx.y).  A row is requested while the one before it is turned, the first one before
// anything else.
template <typename T, int V, bool HALF, int N>
__global__ __launch_bounds__(kThreads) void norm_rows(const NormArgs p)
{
    const RopeArgs &a = p.rope;
    const uint32_t item = blockIdx.x * kThreads + threadIdx.x;
    const int t = (int)(item >> p.lane_bits), g = (int)item & ((1 << p.lane_bits) - 1);
    if (t >= a.n_tokens) return;
    const Share w = share_of(p, blockIdx.y);
    const RopeJob &job = a.jobs[w.job];
    Channels<V, HALF, N> ch;
    ch.place(a, g);
    const T *src = static_cast<const T *>(job.src) + t * job.src_token + w.first * job.src_head;
    Pieces<T, V, N> row;
    row.load(src, ch);
    // where the token's rows go
    T *dst = static_cast<T *>(job.dst) + w.first * job.dst_head;
    int seq = 0, slot = 0;
    if (job.paged) {
        seq = a.token_seq ? a.token_seq[t] : t;
        slot = a.token_slot[t];
        if (seq < 0 || seq >= a.n_seqs || slot < 0 || slot >= a.max_pages * a.page_size) return;
        const int page = a.page_table[(int64_t)seq * a.max_pages + slot / a.page_size];
        if (page < 0 || page >= a.n_pages) return;
        dst += page * a.page_stride + slot % a.page_size * job.dst_token;
    } else {
        dst += t * job.dst_token;
    }
    if (!p.norm[w.job]) {   // V as it is
        for (int h = w.first; h < w.last; ++h) {
            const Pieces<T, V, N> now = row;
            if (h + 1 < w.last) row.load(src += job.src_head, ch);
            now.store(dst, ch);
            dst += job.dst_head;
            if (g == 0) {   // (once per KV head)
                const int64_t at = ((int64_t)seq * a.n_kv_heads + h) * a.row_stride + slot;
                if (a.weights) a.weights[at] = 0.f;
                if (a.order) a.order[at] = a.token_order ? a.token_order[t] : slot;
            }
        }
        return;
    }
    float weight[N][2 * V];
#pragma unroll
    for (int n = 0; n < N; ++n) load_weight<V>(p, w.job, ch.lo[n], ch.hi[n], ch.there[n], weight[n]);
    if (job.rotate) ch.angles(p, g, t);
    for (int h = w.first; h < w.last; ++h) {
        Pieces<T, V, N> now = row;
        if (h + 1 < w.last) row.load(src += job.src_head, ch);
        float z[N][2 * V], sum = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            now.get(n, z[n]);
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) sum = fmaf(z[n][e], z[n][e], sum);
        }
        const float r = inverse_rms(sum, p);
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) z[n][e] *= r * weight[n][e];
            if (job.rotate) ch.turn(n, z[n]);
            now.set(n, z[n]);
        }
        now.store(dst, ch);
        dst += job.dst_head;
    }
}

// One thread: its channels of one token at a time, of heads_each heads of one job (blockIdx.y); it adds up its part of the weight's gradient over all of them.
template <typename T, int V, bool HALF, int N>
__global__ __launch_bounds__(kThreads) void norm_grad_rows(const NormArgs p)
{
    const RopeArgs &a = p.rope;
    __shared__ float sums[kWaves][2 * BS_ROPE_MAX_PAIRS];
    const int g = threadIdx.x & ((1 << p.lane_bits) - 1);
    const Share w = share_of(p, blockIdx.y);
    const RopeJob &job = a.jobs[w.job];
    Channels<V, HALF, N> ch;
    ch.place(a, g);
    float weight[N][2 * V], dw[N][2 * V];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        load_weight<V>(p, w.job, ch.lo[n], ch.hi[n], ch.there[n], weight[n]);
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) dw[n][e] = 0.f;
    }
    for (uint64_t item = (uint64_t)blockIdx.x * kThreads + threadIdx.x; item >> p.lane_bits < (uint64_t)a.n_tokens; item += (uint64_t)gridDim.x * kThreads) {
        const int t = (int)(item >> p.lane_bits);
        const T *src = static_cast<const T *>(job.src) + t * job.src_token + w.first * job.src_head;
        const T *dys = static_cast<const T *>(p.dy[w.job]) + t * p.dy_token[w.job] + w.first * p.dy_head[w.job];
        T *dst = static_cast<T *>(job.dst) + t * job.dst_token + w.first * job.dst_head;
        Pieces<T, V, N> row, dy;
        row.load(src, ch);
        dy.load(dys, ch);
        if (job.rotate) ch.angles(p, g, t);
        for (int h = w.first; h < w.last; ++h) {
            Pieces<T, V, N> now = row;
            const Pieces<T, V, N> grad = dy;
            if (h + 1 < w.last) {
                row.load(src += job.src_head, ch);
                dy.load(dys += p.dy_head[w.job], ch);
            }
            float x[N][2 * V], u[N][2 * V], square = 0.f, dot = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                now.get(n, x[n]);
                grad.get(n, u[n]);
                if (job.rotate) ch.turn(n, u[n]);
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) {
                    square = fmaf(x[n][e], x[n][e], square);
                    dot = fmaf(u[n][e] * weight[n][e], x[n][e], dot);
                }
            }
            const float r = inverse_rms(square, p);
            const float k = row_sum(dot, p.lane_bits) * p.inv_d * r * r;   // mean(u v) r
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float z[2 * V];
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) {
                    z[e] = r * fmaf(-x[n][e], k, u[n][e] * weight[n][e]);
                    dw[n][e] = fmaf(u[n][e], x[n][e] * r, dw[n][e]);
                }
                now.set(n, z);
            }
            now.store(dst, ch);
            dst += job.dst_head;
        }
    }
    if (!p.parts) return;
    // over the rows of a wave, then the waves: always in the same order
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
            float x = dw[n][e];
            for (int off = 1 << p.lane_bits; off < 64; off <<= 1) x += __shfl_xor(x, off, 64);
            if (lane == g && ch.there[n]) sums[threadIdx.x >> 6][e < V ? ch.lo[n] + e : ch.hi[n] + e - V] = x;
        }
    __syncthreads();
    for (int c = threadIdx.x; c < a.head_dim; c += kThreads) {
        float x = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) x += sums[v][c];
        p.parts[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.head_dim + c] = x;
    }
}

// Sums of the workgroups, in 64 bits and always in the same order: a workgroup takes 16 channels of a job (blockIdx.y), in pieces of two, 128 threads for each.
__global__ __launch_bounds__(1024) void norm_grad_join(const float *__restrict__ parts, int per_split, int splits0, int splits, int d, float *__restrict__ dweight)
{
    __shared__ double sums[16][16];
    const int job = blockIdx.y, c = blockIdx.x * 16 + (threadIdx.x & 7) * 2, v = threadIdx.x >> 3, wave = threadIdx.x >> 6;
    const int begin = (job == 0 ? 0 : splits0) * per_split, end = (job == 0 ? splits0 : splits) * per_split;
    double x = 0.0, y = 0.0;
    for (int k0 = begin + v; k0 < end; k0 += 16 * 128) {   // loads of sixteen parts go out together
        float2 z[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) z[k] = c < d && k0 + 128 * k < end ? *reinterpret_cast<const float2 *>(parts + (int64_t)(k0 + 128 * k) * d + c) : make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            x += z[k].x;
            y += z[k].y;
        }
    }
#pragma unroll
    for (int off = 8; off < 64; off <<= 1) {
        x += __shfl_xor(x, off, 64);
        y += __shfl_xor(y, off, 64);
    }
    if ((threadIdx.x & 63) < 8) {
        sums[wave][(threadIdx.x & 7) * 2] = x;
        sums[wave][(threadIdx.x & 7) * 2 + 1] = y;
    }
    __syncthreads();
    const int out = blockIdx.x * 16 + threadIdx.x;
    if (threadIdx.x >= 16 || out >= d) return;
    x = 0.0;
    for (int k = 0; k < 16; ++k) x += sums[k][threadIdx.x];
    dweight[job * d + out] = (float)x;
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
    p.n_axes = rope ? rope->n_axes : 1;
    // Heads of a job share a thread's angles and weights; where there are too few tokens to fill the chip they are split over threads.  Forward: half a million threads
    // (39.5K tokens of 28 + 4 heads 122 us, with a quarter of a million 128), but where that many are there anyway, two heads each, the second of which is requested
    // ahead (847 tokens of 40 + 8 + 8 heads into the cache: 11.2 -> 9.0 us).  Back, where a thread has three times the registers: an eighth of a million (5K tokens, 32 + 16
    // heads in fp32: 79 -> 77 us, and fewer parts to join).
    const int64_t items = (int64_t)a.n_tokens << p.lane_bits;
    if (!gradient && items > INT32_MAX) return BS_EUNSUPPORTED;   // (norm_rows counts them in 32 bits, norm_grad_rows in 64)
    hipError_t err = hipSuccess;
    int splits[3] = {0, 0, 0};   // up to and with each job
    dim3 grid(0);
    if (items > 0) {
        const auto for_threads = [&](int64_t n) { return (n + items - 1) / items; };
        int64_t want = for_threads(gradient ? 131072 : 524288);
        if (!gradient) want = std::min(want, std::max<int64_t>(for_threads(131072), (a.n_heads + 1) / 2));
        a.head_splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min(a.n_heads, 1024), want));
        a.heads_each = (a.n_heads + a.head_splits - 1) / a.head_splits;
        for (int j = 0; j < 3; ++j) splits[j] = (j > 0 ? splits[j - 1] : 0) + (j < a.n_jobs ? (a.jobs[j].n_heads + a.heads_each - 1) / a.heads_each : 0);
        a.head_splits = splits[2];   // (at most 1026)
        p.split_end[0] = splits[0];
        p.split_end[1] = splits[1];
        int64_t wgs = (items + kThreads - 1) / kThreads;
        if (gradient) wgs = std::max<int64_t>(1, std::min<int64_t>(wgs, kMaxParts / a.head_splits));
        grid = dim3((unsigned)wgs, (unsigned)a.head_splits);
        const bool half = !rope || rope->layout == BS_ROPE_HALF;
        if (dtype == BS_BF16) err = half ? launch_layout<__bf16, true>(p, vec, gradient, grid, st) : launch_layout<__bf16, false>(p, vec, gradient, grid, st);
        else err = half ? launch_layout<float, true>(p, vec, gradient, grid, st) : launch_layout<float, false>(p, vec, gradient, grid, st);
        if (err != hipSuccess) return fail_hip(err, "norm_rows launch");
    }
    if (gradient && p.dweight)   // (no tokens: sums of nothing)
        err = launch_kernel(norm_grad_join, dim3((unsigned)((head_dim + 15) / 16), (unsigned)a.n_jobs), dim3(1024), 0, st, p.parts, (int)grid.x, splits[0], splits[2], head_dim, p.dweight);
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
