// Attention of one new token per sequence over a paged cache.
#include <algorithm>
#include <cmath>

#include "device_map.h"
#include "paged_cache.h"

namespace bs {
namespace {

constexpr int kThreads = 256;

struct DecodeArgs {
    bs_cache cache;
    const void *q;
    void *out;
    int64_t q_head, q_seq, out_head, out_seq;
    const int32_t *lens;
    int32_t G, window;
    float scale;
    const float *weights;
    float *weights_out;
    int64_t in_stride, out_stride;
};

__device__ inline int64_t row_offset(const bs_cache &c, int seq, int head, int slot)   // -1: no page
{
    const int page = c.page_table[(int64_t)seq * c.max_pages + slot / c.page_size];
    if (page < 0 || page >= c.n_pages) return -1;
    return page * c.page_stride + head * c.head_stride + (slot % c.page_size) * c.slot_stride;
}

// One workgroup per sequence and KV head: scores of 256 slots at a time, a running maximum and sum, channels over the threads.
template <typename T>
__global__ __launch_bounds__(kThreads) void decode_rows(const DecodeArgs a)
{
    __shared__ float q[256], p[kThreads], wave_max[4], acc[kThreads];
    const int seq = blockIdx.x, head = blockIdx.y, tid = threadIdx.x, d = a.cache.head_dim;
    const int n = max(0, min(a.lens[seq], a.cache.max_pages * a.cache.page_size)), begin = a.window > 0 ? max(0, n - a.window) : 0;
    const T *k = static_cast<const T *>(a.cache.k), *v = static_cast<const T *>(a.cache.v);
    const int64_t row = (int64_t)seq * a.cache.n_kv_heads + head;
    const auto score = [&](int j) {
        const int64_t at = j < n ? row_offset(a.cache, seq, head, j) : -1;
        if (at < 0) return -INFINITY;
        float s = 0.f;
        for (int c = 0; c < d; ++c) s = fmaf(q[c], (float)k[at + c], s);
        return s * a.scale;
    };
    const auto block_max = [&](float x) {
        for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
        __syncthreads();
        if ((tid & 63) == 0) wave_max[tid >> 6] = x;
        __syncthreads();
        return fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
    };
    for (int g = 0; g < a.G; ++g) {
        const int h = head * a.G + g;
        __syncthreads();
        if (tid < d) q[tid] = (float)static_cast<const T *>(a.q)[seq * a.q_seq + h * a.q_head + tid];
        __syncthreads();
        float m = -INFINITY, l = 0.f, o = 0.f;   // o: channel tid % d, every (256 / d)-th slot
        for (int j0 = begin; j0 < n; j0 += kThreads) {
            const float s = score(j0 + tid), m_new = fmaxf(m, block_max(s));
            const float alpha = m_new == -INFINITY ? 1.f : __expf(m - m_new);
            p[tid] = m_new == -INFINITY ? 0.f : __expf(s - m_new);
            m = m_new;
            __syncthreads();
            o *= alpha;
            l *= alpha;
            for (int i = tid / d; i < kThreads; i += kThreads / d) {
                const int64_t at = j0 + i < n ? row_offset(a.cache, seq, head, j0 + i) : -1;
                if (at < 0) continue;
                o = fmaf(p[i], (float)v[at + tid % d], o);
                l += p[i];
            }
        }
        __syncthreads();
        acc[tid] = o;
        p[tid] = l;
        __syncthreads();
        float sum = 0.f;
        l = 0.f;
        for (int i = 0; i < kThreads / d; ++i) { sum += acc[i * d + tid % d]; l += p[i * d]; }
        if (tid < d) static_cast<T *>(a.out)[seq * a.out_seq + h * a.out_head + tid] = (T)(n > begin && m > -INFINITY ? sum / l : (l == 0.f ? 0.f : l));
        if (a.weights)
            for (int j = tid; j < n; j += kThreads) {
                const float s = score(j);
                const float before = g == 0 ? a.weights[row * a.in_stride + j] : a.weights_out[row * a.out_stride + j];
                a.weights_out[row * a.out_stride + j] = before + (s == -INFINITY ? 0.f : __expf(s - m) / l);
            }
    }
}

int check_decode(const bs_cache *cache, int32_t n_q_heads)
{
    if (int rc = check_cache(cache)) return rc;
    if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0) return BS_EINVAL;
    if ((cache->head_dim != 64 && cache->head_dim != 128) || cache->n_kv_heads > 65535) return BS_EUNSUPPORTED;
    return BS_OK;
}

}  // namespace
}  // namespace bs

extern "C" int64_t bs_attn_decode_workspace(const bs_cache *cache, int32_t n_q_heads, int32_t)
{
    if (int rc = bs::check_decode(cache, n_q_heads)) return rc;
    return 0;
}

extern "C" int bs_attn_decode(const bs_cache *cache, const bs_heads *q, const bs_heads *out, const int32_t *lens, int32_t window, float scale,
                              const bs_slots *slots, const bs_slots *slots_out, void *workspace, int64_t workspace_bytes, void *stream)
{
    using namespace bs;
    if (check_heads(q) || check_heads(out) || q->n_heads != out->n_heads || !lens || window < 0 || !(scale > 0.f) || !std::isfinite(scale)) return BS_EINVAL;
    if (int rc = check_decode(cache, q->n_heads)) return rc;
    if (!slots != !slots_out || !workspace || (uintptr_t)workspace % 16 != 0) return BS_EINVAL;
    if (slots) {
        if (!slots->weights || !slots_out->weights || check_slots(*cache, slots) || check_slots(*cache, slots_out)) return BS_EINVAL;
        if (slots->weights == slots_out->weights && slots->row_stride != slots_out->row_stride) return BS_EINVAL;
        if (window > 0) return BS_EUNSUPPORTED;
    }
    if (!rows_aligned(*q, cache->dtype) || !rows_aligned(*out, cache->dtype)) return BS_EUNSUPPORTED;
    if (workspace_bytes < bs_attn_decode_workspace(cache, q->n_heads, slots != nullptr)) return BS_EINVAL;
    DecodeArgs a{};
    a.cache = *cache;
    a.q = q->data; a.q_head = q->head_stride; a.q_seq = q->token_stride;
    a.out = out->data; a.out_head = out->head_stride; a.out_seq = out->token_stride;
    a.lens = lens;
    a.G = q->n_heads / cache->n_kv_heads;
    a.window = window;
    a.scale = scale;
    if (slots) {
        a.weights = slots->weights; a.in_stride = slots->row_stride;
        a.weights_out = slots_out->weights; a.out_stride = slots_out->row_stride;
    }
    const dim3 grid((unsigned)cache->n_seqs, (unsigned)cache->n_kv_heads);
    const hipError_t e = cache->dtype == BS_BF16 ? launch_kernel(decode_rows<__bf16>, grid, dim3(kThreads), 0, (hipStream_t)stream, a)
                                                 : launch_kernel(decode_rows<float>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
    return e == hipSuccess ? BS_OK : fail_hip(e, "decode_rows launch");
}
