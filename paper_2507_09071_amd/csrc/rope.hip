// Rotary positions, and new tokens into a paged cache (which rotates on the way).
//
// A pair (a, b) of channels is turned by the angle position * f: (a cos - b sin, b cos + a sin).  The work is reading every row once
// and writing it once, so the bound is HBM, and what an angle costs has to be paid once per token and pair, not once per head: a thread keeps its
// angles over the heads.  39.5K tokens of 28 + 4 heads, 648 MB: 124 us, 5.2 TB/s, a large copy's rate (5.0 to 5.5); the same into pages, token-major
// rows, 730 MB: 154 us, 4.75 TB/s.  Where the pairs do not divide into pieces of 16 bytes, smaller ones cost: 36 of 128 channels, pieces of 4 bytes, 136 us
// (647 MB; at a copy's rate 122), 20 of 64 79 (61).  (Stores past the caches: 121 and 151 us, but 50 -> 67 for rows of which an instruction writes half a line.)
#include <algorithm>
#include <array>
#include <cmath>
#include <cstring>
#include <utility>

#include "device_map.h"
#include "paged_cache.h"
#include "rope_common.h"

namespace bs {

int check_cache(const bs_cache *c)
{
    if (!c || !c->k || !c->v || !c->page_table) return BS_EINVAL;
    if (c->n_kv_heads <= 0 || c->head_dim <= 0 || c->page_size <= 0 || c->n_pages <= 0 || c->n_seqs <= 0 || c->max_pages <= 0) return BS_EINVAL;
    if (c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < 0 || c->page_stride > kMaxStride || c->head_stride > kMaxStride || c->slot_stride > kMaxStride)
        return BS_EINVAL;
    if (c->dtype != BS_BF16 && c->dtype != BS_F32) return BS_EUNSUPPORTED;
    if (c->head_dim % 8 != 0 || c->head_dim > 256 || c->page_size % 16 != 0 || cache_slots(*c) > kMaxSlots) return BS_EUNSUPPORTED;
    if ((int64_t)c->n_seqs * c->n_kv_heads > INT32_MAX) return BS_EUNSUPPORTED;
    const int64_t per16 = 16 / element_bytes(c->dtype);
    if (((uintptr_t)c->k | (uintptr_t)c->v) % 16 != 0 || c->page_stride % per16 != 0 || c->head_stride % per16 != 0 || c->slot_stride % per16 != 0)
        return BS_EUNSUPPORTED;
    // 16 slots of a page are addressed from the first one in 32 bits
    if (c->slot_stride * 16 * element_bytes(c->dtype) > INT32_MAX) return BS_EUNSUPPORTED;
    return BS_OK;
}

int check_heads(const bs_heads *h, bool none)
{
    if (!h || (!h->data && !none) || h->n_heads <= 0 || h->head_stride < 0 || h->token_stride < 0 || h->head_stride > kMaxStride || h->token_stride > kMaxStride) return BS_EINVAL;
    return BS_OK;
}

// Axes from the smallest stride up: each steps over all that the ones before it span.  (Products in 128 bits: strides go up to 2^40.)
template <size_t N>
static int rows_apart(std::array<std::pair<int64_t, int32_t>, N> axes, int32_t row)   // stride, count
{
    std::sort(axes.begin(), axes.end());
    __int128 span = row;
    for (const auto &[stride, count] : axes) {
        if (count <= 1) continue;
        if (stride < span) return BS_EINVAL;
        span += (__int128)stride * (count - 1);
    }
    return span > (int64_t)1 << 60 ? BS_EINVAL : BS_OK;   // (no memory has so much, and offsets are formed in 64 bits)
}

int check_rows_apart(const bs_heads &h, int32_t n_tokens, int32_t head_dim)
{
    return n_tokens == 0 ? BS_OK : rows_apart<2>({{{h.head_stride, h.n_heads}, {h.token_stride, n_tokens}}}, head_dim);
}

int check_rows_apart(const bs_cache &c)
{
    return rows_apart<3>({{{c.page_stride, c.n_pages}, {c.head_stride, c.n_kv_heads}, {c.slot_stride, c.page_size}}}, c.head_dim);
}

int check_slots(const bs_cache &c, const bs_slots *s)
{
    return s->row_stride < cache_slots(c) || s->row_stride > kMaxStride || ((uintptr_t)s->weights | (uintptr_t)s->order) % 4 != 0 ? BS_EINVAL : BS_OK;
}

bool rows_aligned(const bs_heads &h, int32_t dtype)
{
    const int64_t per16 = 16 / element_bytes(dtype);
    return (uintptr_t)h.data % 16 == 0 && h.head_stride % per16 == 0 && h.token_stride % per16 == 0;
}

namespace {

constexpr int kThreads = 256;

// One thread: 2 V channels of one token, of heads_each heads.  Groups 0 .. pairs / V - 1 of a token are V pairs each, the ones behind
// them 2 V channels that are copied.  (Rows of four heads requested together, before the angles are formed: fewer waves fit, 124 -> 130 us for the
// prompt of 39.5K tokens.)
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kThreads) void rope_rows(const RopeArgs a)
{
    const uint32_t idx = blockIdx.x * kThreads + threadIdx.x, per_split = a.n_tokens * a.groups;
    const int split = (int)(idx / per_split);
    if (split >= a.head_splits) return;
    const int item = (int)(idx - split * per_split);
    const int t = item / a.groups, g = item - t * a.groups;
    const bool turns = g * V < a.pairs;
    // V channels from lo on and V from hi on: half of what is rotated, or copied, apart, so that neighbours load neighbouring pieces (interleaved fp32
    // pairs in half of a head of 128, 246 MB: 54 -> 50 us)
    const bool alone = !HALF && V == 1;   // a pair does not fit a piece
    const int lo = turns ? (alone ? 2 * g : V * g) : a.rotary_dim + V * (g - a.pairs / V);
    const int hi = turns ? lo + (alone ? 1 : a.pairs) : lo + (a.head_dim - a.rotary_dim) / 2;

    float c[V], s[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { c[e] = 1.f; s[e] = 0.f; }
    if (turns) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int i = HALF || alone ? g * V + e : (2 * e < V ? lo : hi - V) / 2 + e;
            rotation(a.quarter_turns[i], a.positions[a.axis[i] * a.axis_stride + t], c[e], s[e]);
            c[e] *= a.magnitude;
            s[e] *= a.magnitude * a.direction;
        }
    }
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
    int head = split * a.heads_each;
    const int end = min(a.n_heads, head + a.heads_each);
    int first = 0;
    for (int j = 0; j < a.n_jobs; ++j) {
        const RopeJob &job = a.jobs[j];
        const int last = first + job.n_heads;
        if (!job.paged || page_at >= 0) {
            const T *src = static_cast<const T *>(job.src) + t * job.src_token;
            T *dst = static_cast<T *>(job.dst) + (job.paged ? page_at + at * job.dst_token : t * job.dst_token);
            for (int h = max(head, first); h < min(end, last); ++h) {
                const T *x = src + (h - first) * job.src_head;
                T *y = dst + (h - first) * job.dst_head;
                const Vec<T, V> u = *reinterpret_cast<const Vec<T, V> *>(x + lo), w = *reinterpret_cast<const Vec<T, V> *>(x + hi);
                Vec<T, V> p = u, q = w;
                if (job.rotate && turns) {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float m, n;
                        if constexpr (HALF) { m = (float)u.x[e]; n = (float)w.x[e]; }
                        else { m = (float)(2 * e < V ? u.x[(2 * e) % V] : w.x[(2 * e) % V]); n = (float)(2 * e + 1 < V ? u.x[(2 * e + 1) % V] : w.x[(2 * e + 1) % V]); }
                        const T r = (T)fmaf(m, c[e], -n * s[e]), i = (T)fmaf(n, c[e], m * s[e]);
                        if constexpr (HALF) { p.x[e] = r; q.x[e] = i; }
                        else {
                            (2 * e < V ? p.x[(2 * e) % V] : q.x[(2 * e) % V]) = r;
                            (2 * e + 1 < V ? p.x[(2 * e + 1) % V] : q.x[(2 * e + 1) % V]) = i;
                        }
                    }
                }
                *reinterpret_cast<Vec<T, V> *>(y + lo) = p;
                *reinterpret_cast<Vec<T, V> *>(y + hi) = q;
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

template <typename T, bool HALF>
hipError_t launch_layout(const RopeArgs &a, int vec, hipStream_t st)
{
    const int64_t threads = (int64_t)a.n_tokens * a.groups * a.head_splits;
    const dim3 grid((unsigned)((threads + kThreads - 1) / kThreads));
    switch (vec) {
    case 8: if constexpr (sizeof(T) == 2) return launch_kernel(rope_rows<T, 8, HALF>, grid, dim3(kThreads), 0, st, a); else return hipErrorInvalidValue;
    case 4: return launch_kernel(rope_rows<T, 4, HALF>, grid, dim3(kThreads), 0, st, a);
    case 2: return launch_kernel(rope_rows<T, 2, HALF>, grid, dim3(kThreads), 0, st, a);
    default: return launch_kernel(rope_rows<T, 1, HALF>, grid, dim3(kThreads), 0, st, a);
    }
}

// `rope` null: nothing is rotated.
int run_rope(RopeArgs &a, const bs_rope *rope, int32_t dtype, int32_t head_dim, bool inverse, hipStream_t st)
{
    if (a.n_tokens == 0) return BS_OK;
    const int vec = fill_rope(a, rope, dtype, head_dim, inverse);
    // Heads share a thread's angles; where there are too few tokens to fill the chip they are split over threads.
    const int64_t items = (int64_t)a.n_tokens * a.groups;
    if (items > INT32_MAX) return BS_EUNSUPPORTED;   // (with several splits there are few, so threads are counted in 32 bits)
    a.head_splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(a.n_heads, (256 * 2048 + items - 1) / items));
    a.heads_each = (a.n_heads + a.head_splits - 1) / a.head_splits;
    a.head_splits = (a.n_heads + a.heads_each - 1) / a.heads_each;
    const bool half = !rope || rope->layout == BS_ROPE_HALF;
    hipError_t err;
    if (dtype == BS_BF16) err = half ? launch_layout<__bf16, true>(a, vec, st) : launch_layout<__bf16, false>(a, vec, st);
    else err = half ? launch_layout<float, true>(a, vec, st) : launch_layout<float, false>(a, vec, st);
    return err == hipSuccess ? BS_OK : fail_hip(err, "rope_rows launch");
}

}  // namespace

int check_rope(const bs_rope *r, int32_t n_tokens, int32_t head_dim, const int32_t *positions, int64_t axis_stride)
{
    if (!r || (!positions && n_tokens > 0) || axis_stride < 0 || axis_stride > kMaxStride) return BS_EINVAL;
    if (r->rotary_dim < 2 || r->rotary_dim % 2 != 0 || r->rotary_dim > 2 * BS_ROPE_MAX_PAIRS || r->rotary_dim > head_dim) return BS_EINVAL;
    if ((r->layout != BS_ROPE_HALF && r->layout != BS_ROPE_INTERLEAVED) || r->n_axes < 1 || r->n_axes > BS_ROPE_MAX_AXES) return BS_EINVAL;
    if (!std::isfinite(r->magnitude)) return BS_EINVAL;
    for (int i = 0; i < r->rotary_dim / 2; ++i)
        if (r->axis[i] >= r->n_axes || !std::isfinite(r->freq[i]) || std::fabs(r->freq[i]) > 1e3) return BS_EINVAL;
    return BS_OK;
}

RopeJob job_of(const bs_heads &x, const bs_heads &y, bool rotate)
{
    return {x.data, y.data, x.head_stride, x.token_stride, y.head_stride, y.token_stride, x.n_heads, rotate, 0};
}

int fill_rope(RopeArgs &a, const bs_rope *rope, int32_t dtype, int32_t head_dim, bool inverse)
{
    a.rotary_dim = rope ? rope->rotary_dim : 0;
    a.pairs = a.rotary_dim / 2;
    a.head_dim = head_dim;
    if (rope) {
        a.magnitude = rope->magnitude;
        a.direction = inverse ? -1.f : 1.f;
        for (int i = 0; i < a.pairs; ++i) a.quarter_turns[i] = rope->freq[i] * 0.63661977236758134;
        std::memcpy(a.axis, rope->axis, a.pairs);
    }
    // channels that a thread takes at a time: as many as 16 bytes hold, or less where a size, a stride or a pointer asks for it
    const int e = element_bytes(dtype);
    int vec = 16 / e;
    const auto fits = [&](int v) {
        bool ok = a.pairs % v == 0 && (head_dim - a.rotary_dim) % (2 * v) == 0;
        for (int j = 0; j < a.n_jobs; ++j) {
            const RopeJob &job = a.jobs[j];
            ok = ok && ((uintptr_t)job.src | (uintptr_t)job.dst) % (e * v) == 0 && job.src_head % v == 0 && job.src_token % v == 0 && job.dst_head % v == 0 && job.dst_token % v == 0;
        }
        return ok;
    };
    while (vec > 1 && !fits(vec)) vec /= 2;
    a.groups = head_dim / (2 * vec);
    a.n_heads = 0;
    for (int j = 0; j < a.n_jobs; ++j) a.n_heads += a.jobs[j].n_heads;
    return vec;
}

int append_args(RopeArgs *a, const bs_cache *cache, const bs_heads *k, const bs_heads *v, int32_t n_tokens, const int32_t *token_seq, const int32_t *token_slot,
                const bs_rope *rope, const int32_t *positions, int64_t axis_stride, const bs_heads *q, const bs_heads *q_out, const bs_slots *slots,
                const int32_t *token_order)
{
    if (int rc = check_cache(cache)) return rc;
    if (n_tokens < 0 || check_heads(k, n_tokens == 0) || check_heads(v, n_tokens == 0) || (!token_slot && n_tokens > 0)) return BS_EINVAL;
    if (k->n_heads != cache->n_kv_heads || v->n_heads != cache->n_kv_heads || !q != !q_out) return BS_EINVAL;
    if (q && (check_heads(q, n_tokens == 0) || check_heads(q_out, n_tokens == 0) || q->n_heads != q_out->n_heads || q->n_heads > (1 << 20) || check_rows_apart(*q_out, n_tokens, cache->head_dim))) return BS_EINVAL;
    if (int rc = check_rows_apart(*cache)) return rc;
    if (rope)
        if (int rc = check_rope(rope, n_tokens, cache->head_dim, positions, axis_stride)) return rc;
    if (slots)
        if (int rc = check_slots(*cache, slots)) return rc;
    const int e = element_bytes(cache->dtype);
    if (((uintptr_t)k->data | (uintptr_t)v->data) % e != 0 || (q && ((uintptr_t)q->data | (uintptr_t)q_out->data) % e != 0)) return BS_EINVAL;
    if (q) a->jobs[a->n_jobs++] = job_of(*q, *q_out, true);
    const bs_heads pool_k{cache->k, cache->head_stride, cache->slot_stride, cache->n_kv_heads}, pool_v{cache->v, cache->head_stride, cache->slot_stride, cache->n_kv_heads};
    a->jobs[a->n_jobs] = job_of(*k, pool_k, rope != nullptr);
    a->jobs[a->n_jobs++].paged = 1;
    a->jobs[a->n_jobs] = job_of(*v, pool_v, false);
    a->jobs[a->n_jobs++].paged = 1;
    a->n_tokens = n_tokens;
    a->positions = positions;
    a->axis_stride = axis_stride;
    a->token_seq = token_seq;
    a->token_slot = token_slot;
    a->token_order = token_order;
    a->page_table = cache->page_table;
    a->n_seqs = cache->n_seqs;
    a->max_pages = cache->max_pages;
    a->page_size = cache->page_size;
    a->n_pages = cache->n_pages;
    a->n_kv_heads = cache->n_kv_heads;
    a->page_stride = cache->page_stride;
    if (slots) {
        a->weights = slots->weights;
        a->order = slots->order;
        a->row_stride = slots->row_stride;
    }
    return BS_OK;
}

}  // namespace bs

extern "C" int bs_rope_init(bs_rope *rope, int32_t rotary_dim, int32_t layout, double base, int32_t scaling, double factor,
                            int32_t original_len, double fast, double slow, double magnitude, const int32_t *sections, int32_t n_axes)
{
    if (!rope || rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > 2 * BS_ROPE_MAX_PAIRS) return BS_EINVAL;
    if (layout != BS_ROPE_HALF && layout != BS_ROPE_INTERLEAVED) return BS_EINVAL;
    if (scaling < BS_ROPE_PLAIN || scaling > BS_ROPE_PARTS) return BS_EINVAL;
    if (!(base >= 1.0) || !std::isfinite(base) || !(magnitude > 0.0) || !std::isfinite((float)magnitude)) return BS_EINVAL;
    if (scaling != BS_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return BS_EINVAL;
    if (scaling == BS_ROPE_BASE && rotary_dim == 2) return BS_EINVAL;
    if (scaling == BS_ROPE_PARTS && (original_len <= 0 || !(slow >= 0.0) || !(fast > slow) || !std::isfinite(fast))) return BS_EINVAL;
    const int32_t pairs = rotary_dim / 2;
    if (n_axes < 1 || n_axes > BS_ROPE_MAX_AXES || (!sections && n_axes != 1)) return BS_EINVAL;
    int64_t sum = 0;
    for (int32_t i = 0; sections && i < n_axes; ++i) {
        if (sections[i] < 0) return BS_EINVAL;
        sum += sections[i];
    }
    if (sections && sum != pairs) return BS_EINVAL;
    bs_rope r{};
    r.rotary_dim = rotary_dim;
    r.layout = layout;
    r.n_axes = n_axes;
    r.magnitude = (float)magnitude;
    if (scaling == BS_ROPE_BASE) base *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
    int32_t axis = 0, left = sections ? sections[0] : pairs;
    for (int32_t i = 0; i < pairs; ++i) {
        double f = std::pow(base, -2.0 * i / rotary_dim);
        if (scaling == BS_ROPE_LINEAR) f /= factor;
        if (scaling == BS_ROPE_PARTS) {
            const double turns = original_len * f / 6.2831853071795865, g = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
            f *= g + (1.0 - g) / factor;
        }
        r.freq[i] = f;
        while (left == 0) left = sections[++axis];
        --left;
        r.axis[i] = (uint8_t)axis;
    }
    *rope = r;
    return BS_OK;
}

extern "C" int bs_rope_apply(const bs_rope *rope, const bs_heads *x, const bs_heads *y, int32_t n_tensors, int32_t dtype,
                             int32_t n_tokens, int32_t head_dim, const int32_t *positions, int64_t axis_stride, uint32_t flags, void *stream)
{
    using namespace bs;
    if (!x || !y || n_tensors < 1 || n_tensors > 2 || n_tokens < 0 || (flags & ~BS_ROPE_INVERSE)) return BS_EINVAL;
    if (head_dim < 2 || head_dim % 2 != 0 || head_dim > 2 * BS_ROPE_MAX_PAIRS) return BS_EINVAL;
    if (int rc = check_rope(rope, n_tokens, head_dim, positions, axis_stride)) return rc;
    if (dtype != BS_BF16 && dtype != BS_F32) return BS_EUNSUPPORTED;
    RopeArgs a{};
    a.n_jobs = n_tensors;
    for (int i = 0; i < n_tensors; ++i) {
        if (check_heads(&x[i], n_tokens == 0) || check_heads(&y[i], n_tokens == 0) || x[i].n_heads != y[i].n_heads || x[i].n_heads > (1 << 20)) return BS_EINVAL;
        if (((uintptr_t)x[i].data | (uintptr_t)y[i].data) % element_bytes(dtype) != 0 || check_rows_apart(y[i], n_tokens, head_dim)) return BS_EINVAL;
        a.jobs[i] = job_of(x[i], y[i], true);
    }
    a.n_tokens = n_tokens;
    a.positions = positions;
    a.axis_stride = axis_stride;
    return run_rope(a, rope, dtype, head_dim, flags & BS_ROPE_INVERSE, (hipStream_t)stream);
}

extern "C" int bs_cache_append(const bs_cache *cache, const bs_heads *k, const bs_heads *v, int32_t n_tokens, const int32_t *token_seq,
                               const int32_t *token_slot, const bs_rope *rope, const int32_t *positions, int64_t axis_stride, const bs_heads *q,
                               const bs_heads *q_out, const bs_slots *slots, const int32_t *token_order, void *stream)
{
    using namespace bs;
    RopeArgs a{};
    if (int rc = append_args(&a, cache, k, v, n_tokens, token_seq, token_slot, rope, positions, axis_stride, q, q_out, slots, token_order)) return rc;
    if (q && !rope) return BS_EINVAL;
    return run_rope(a, rope, cache->dtype, cache->head_dim, false, (hipStream_t)stream);
}
