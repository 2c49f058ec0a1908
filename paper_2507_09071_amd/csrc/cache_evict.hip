// Eviction from a paged cache by accumulated attention weight.
//
// Per sequence and KV head ("row") the `keep` slots with the largest weights stay.  Weights are ranked as unsigned integers of the same
// order, protected slots above all; the rank of the last one kept is found digit by digit from counts (radix selection), ties go
// to the lowest slots.  Kept slots behind `keep` move into the holes before it: the two sets do not overlap, so moves need
// no order among each other, and nothing moves that can stay.  Weights and orders are read once per pass over them (8 bytes a slot),
// moves cost 4 rows each.
#include <algorithm>

#include "device_map.h"
#include "paged_cache.h"

namespace bs {
namespace {

constexpr int kSelectThreads = 1024, kMoveThreads = 256;

struct EvictArgs {
    bs_cache cache;
    const int32_t *lens;
    int32_t *lens_out;
    int32_t keep, keep_first, keep_last;
    const float *weights;
    const int32_t *order;
    float *weights_out;
    int32_t *order_out;
    int64_t in_stride, out_stride;
    int32_t *counts;            // moves of each row
    int32_t *to, *from;         // [row][max_moves]
    int32_t max_moves;
};

__device__ inline int used_slots(const EvictArgs &a, int seq)
{
    return max(0, min(a.lens[seq], a.cache.max_pages * a.cache.page_size));
}

// Larger weight, larger rank; NaN smallest; -0 as 0.  Protected slots: above every weight.
__device__ inline uint32_t rank_of(float w, bool safe)
{
    if (safe) return ~0u;
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Sums x over the threads before this one; *total over all of them.  Two barriers.
__device__ inline int before_in_block(bool x, int *wave_sums, int *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t b = __ballot(x);
    if (lane == 0) wave_sums[wave] = __popcll(b);
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSelectThreads / 64; ++w) {
        const int n = wave_sums[w];
        before += w < wave ? n : 0;
        all += n;
    }
    __syncthreads();
    *total = all;
    return before + __popcll(b & ((1ull << lane) - 1));
}

__global__ __launch_bounds__(kSelectThreads) void evict_select(const EvictArgs a)
{
    __shared__ int hist[256];
    __shared__ int sums[kSelectThreads / 64];
    __shared__ int shared_digit, shared_need, shared_newest;
    const int row = blockIdx.x, tid = threadIdx.x;
    const int n = used_slots(a, row / a.cache.n_kv_heads);
    const float *w = a.weights + row * a.in_stride;
    const int32_t *ord = a.order + row * a.in_stride;
    float *w_out = a.weights_out + row * a.out_stride;
    int32_t *ord_out = a.order_out + row * a.out_stride;
    if (n <= a.keep) {
        for (int j = tid; j < n; j += kSelectThreads) {
            if (w_out != w) w_out[j] = w[j];
            if (ord_out != ord) ord_out[j] = ord[j];
        }
        if (tid == 0) a.counts[row] = 0;
        return;
    }
    if (tid == 0) shared_newest = INT32_MIN;
    __syncthreads();
    int newest = INT32_MIN;
    for (int j = tid; j < n; j += kSelectThreads) newest = max(newest, ord[j]);
    atomicMax(&shared_newest, newest);
    __syncthreads();
    newest = shared_newest;
    const auto rank = [&](int j) {
        const int32_t o = ord[j];
        return rank_of(w[j], o < a.keep_first || (int64_t)o > (int64_t)newest - a.keep_last);
    };
    // the rank of the last slot kept: digits of 8 bits from the top
    uint32_t prefix = 0;
    int need = a.keep;   // slots still to be found among those whose higher digits are `prefix`
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kSelectThreads) {
            const uint32_t r = rank(j);
            if (shift == 24 || (r >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(r >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int d = 255, left = need;
            while (hist[d] < left) left -= hist[d--];
            shared_digit = d;
            shared_need = left;
        }
        __syncthreads();
        prefix |= (uint32_t)shared_digit << shift;
        need = shared_need;
        __syncthreads();
    }
    // `need` slots of rank `prefix` stay, the lowest ones
    int32_t *to = a.to + (int64_t)row * a.max_moves, *from = a.from + (int64_t)row * a.max_moves;
    int ties = 0, holes = 0, late = 0;
    for (int j0 = 0; j0 < n; j0 += kSelectThreads) {
        const int j = j0 + tid;
        const uint32_t r = j < n ? rank(j) : 0;
        const bool tie = j < n && r == prefix;
        int total;
        const int tie_rank = ties + before_in_block(tie, sums, &total);
        ties += total;
        const bool kept = j < n && (r > prefix || (tie && tie_rank < need));
        const bool hole = j < a.keep && !kept, moved = j >= a.keep && kept;
        const int hole_rank = holes + before_in_block(hole, sums, &total);
        holes += total;
        const int late_rank = late + before_in_block(moved, sums, &total);
        late += total;
        if (hole) to[hole_rank] = j;
        if (moved) from[late_rank] = j;
        if (kept && j < a.keep) {
            if (w_out != w) w_out[j] = w[j];
            if (ord_out != ord) ord_out[j] = ord[j];
        }
    }
    if (tid == 0) a.counts[row] = holes;
}

__device__ inline int64_t slot_offset(const bs_cache &c, int seq, int head, int slot)   // -1: no page
{
    const int page = c.page_table[(int64_t)seq * c.max_pages + slot / c.page_size];
    if (page < 0 || page >= c.n_pages) return -1;
    return page * c.page_stride + head * c.head_stride + (slot % c.page_size) * c.slot_stride;
}

// A move is done by as many threads as a row has pieces of 16 bytes.
template <typename T>
__global__ __launch_bounds__(kMoveThreads) void evict_move(const EvictArgs a)
{
    const int row = blockIdx.x, seq = row / a.cache.n_kv_heads, head = row - seq * a.cache.n_kv_heads;
    constexpr int PER = 16 / sizeof(T);
    const int pieces = a.cache.head_dim / PER, n = a.counts[row];
    const T *k = static_cast<const T *>(a.cache.k), *v = static_cast<const T *>(a.cache.v);
    for (int64_t idx = (int64_t)blockIdx.y * kMoveThreads + threadIdx.x; idx < (int64_t)n * pieces; idx += (int64_t)gridDim.y * kMoveThreads) {
        const int i = (int)(idx / pieces), p = (int)(idx - (int64_t)i * pieces);
        const int to = a.to[(int64_t)row * a.max_moves + i], from = a.from[(int64_t)row * a.max_moves + i];
        const int64_t dst = slot_offset(a.cache, seq, head, to), src = slot_offset(a.cache, seq, head, from);
        if (dst >= 0 && src >= 0) {
            const uint4 x = *reinterpret_cast<const uint4 *>(k + src + p * PER), y = *reinterpret_cast<const uint4 *>(v + src + p * PER);
            *reinterpret_cast<uint4 *>(const_cast<T *>(k) + dst + p * PER) = x;
            *reinterpret_cast<uint4 *>(const_cast<T *>(v) + dst + p * PER) = y;
        }
        if (p == 0) {
            a.weights_out[row * a.out_stride + to] = a.weights[row * a.in_stride + from];
            a.order_out[row * a.out_stride + to] = a.order[row * a.in_stride + from];
        }
    }
    // (the lengths were read by the kernel before)
    if (blockIdx.y == 0 && head == 0 && threadIdx.x == 0) a.lens_out[seq] = min(used_slots(a, seq), a.keep);
}

int check_evict(const bs_cache *cache, int32_t keep)
{
    if (int rc = check_cache(cache)) return rc;
    if (keep < 1) return BS_EINVAL;
    return BS_OK;
}

int64_t max_moves(const bs_cache &c, int32_t keep) { return std::max<int64_t>(0, std::min<int64_t>(keep, cache_slots(c) - keep)); }
int64_t counts_bytes(const bs_cache &c) { return ((int64_t)c.n_seqs * c.n_kv_heads * 4 + 15) / 16 * 16; }

}  // namespace
}  // namespace bs

extern "C" int64_t bs_cache_evict_workspace(const bs_cache *cache, int32_t keep)
{
    using namespace bs;
    if (int rc = check_evict(cache, keep)) return rc;
    return counts_bytes(*cache) + (int64_t)cache->n_seqs * cache->n_kv_heads * max_moves(*cache, keep) * 8;
}

extern "C" int bs_cache_evict(const bs_cache *cache, const int32_t *lens, int32_t *lens_out, int32_t keep, int32_t keep_first, int32_t keep_last,
                              const bs_slots *slots, const bs_slots *slots_out, void *workspace, int64_t workspace_bytes, void *stream)
{
    using namespace bs;
    if (int rc = check_evict(cache, keep)) return rc;
    if (!lens || !lens_out || !slots || !slots_out || !workspace || keep_first < 0 || keep_last < 0 || (int64_t)keep_first + keep_last > keep) return BS_EINVAL;
    if (!slots->weights || !slots->order || !slots_out->weights || !slots_out->order) return BS_EINVAL;
    if (check_slots(*cache, slots) || check_slots(*cache, slots_out)) return BS_EINVAL;
    if ((uintptr_t)workspace % 16 != 0 || workspace_bytes < bs_cache_evict_workspace(cache, keep)) return BS_EINVAL;
    // the same arrays, or others: in place, rows lie where they lay
    if ((slots->weights == slots_out->weights || slots->order == slots_out->order) && slots->row_stride != slots_out->row_stride) return BS_EINVAL;
    EvictArgs a{};
    a.cache = *cache;
    a.lens = lens;
    a.lens_out = lens_out;
    a.keep = keep; a.keep_first = keep_first; a.keep_last = keep_last;
    a.weights = slots->weights; a.order = slots->order; a.in_stride = slots->row_stride;
    a.weights_out = slots_out->weights; a.order_out = slots_out->order; a.out_stride = slots_out->row_stride;
    const int64_t rows = (int64_t)cache->n_seqs * cache->n_kv_heads, moves = max_moves(*cache, keep);
    a.max_moves = (int32_t)moves;
    a.counts = static_cast<int32_t *>(workspace);
    a.to = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + counts_bytes(*cache));
    a.from = a.to + rows * moves;
    hipStream_t st = (hipStream_t)stream;
    hipError_t e = launch_kernel(evict_select, dim3((unsigned)rows), dim3(kSelectThreads), 0, st, a);
    if (e != hipSuccess) return fail_hip(e, "evict_select launch");
    const int64_t pieces = (int64_t)cache->head_dim * element_bytes(cache->dtype) / 16;
    const int64_t blocks = std::max<int64_t>(1, std::min({(moves * pieces + kMoveThreads - 1) / kMoveThreads, (int64_t)1024, (4096 + rows - 1) / rows}));
    const dim3 grid((unsigned)rows, (unsigned)blocks);
    e = cache->dtype == BS_BF16 ? launch_kernel(evict_move<__bf16>, grid, dim3(kMoveThreads), 0, st, a) : launch_kernel(evict_move<float>, grid, dim3(kMoveThreads), 0, st, a);
    return e == hipSuccess ? BS_OK : fail_hip(e, "evict_move launch");
}
