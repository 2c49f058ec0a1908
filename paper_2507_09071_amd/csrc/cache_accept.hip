// Accepted drafted tokens move together behind their sequence.
//
// Slot lens + i takes what slot lens + path[i] held.  Everything that a workgroup moves is in LDS before it writes, so any path will do.  A few rows per
// sequence and head: what takes the time is the chain of loads length, path, page, row: 3.2 us for three sequences in fp32, 3.9 us for 64 with 8 KV heads.
#include <algorithm>

#include "device_map.h"
#include "paged_cache.h"

namespace bs {
namespace {

constexpr int kThreads = 256;

struct AcceptArgs {
    bs_cache cache;
    const int32_t *lens, *path, *n_path;
    int32_t *lens_out;            // null: written by accept_lens
    int32_t max_path, item;
    int32_t row_bytes, slice, slices;   // bytes of a row that a workgroup moves, workgroups that move a row
    float *weights;
    int32_t *order;
    int64_t row_stride;
};

// Two arrays of int32 that share memory.
bool overlap(const int32_t *x, int64_t n, const int32_t *y, int64_t m) { return x < y + m && y < x + n; }

__device__ inline int held(int x, int lo, int hi) { return max(lo, min(x, hi)); }

// blockIdx: x sequence, y KV head, z slices of K's rows, then of V's
__global__ __launch_bounds__(kThreads) void accept_rows(const AcceptArgs a)
{
    extern __shared__ uint4 rows[];                        // [max_path][pieces of a slice]
    __shared__ int64_t src[BS_TREE_MAX_TOKENS], dst[BS_TREE_MAX_TOKENS];   // offsets of rows in bytes; -1: stays
    const int tid = threadIdx.x, s = blockIdx.x, h = blockIdx.y, z = blockIdx.z;
    const int P = a.cache.page_size, cap = a.cache.max_pages * P;
    const int len = held(a.lens[s], 0, cap), n = held(a.n_path[s], 0, a.max_path);
    if (z == 0 && h == 0 && tid == 0 && a.lens_out) a.lens_out[s] = min(len + n, cap);

    int from = 0, to = 0;
    bool moves = false;
    if (tid < n) {
        const int p = a.path[(int64_t)s * a.max_path + tid];
        moves = p >= 0 && p < BS_TREE_MAX_TOKENS && p != tid && len + p < cap && len + tid < cap;
        from = len + (moves ? p : 0);
        to = len + tid;
        src[tid] = dst[tid] = -1;
        if (moves) {
            const int32_t *table = a.cache.page_table + (int64_t)s * a.cache.max_pages;
            const int x = table[from / P], y = table[to / P];
            moves = x >= 0 && x < a.cache.n_pages && y >= 0 && y < a.cache.n_pages;
            if (moves) {
                src[tid] = (x * a.cache.page_stride + h * a.cache.head_stride + from % P * a.cache.slot_stride) * a.item;
                dst[tid] = (y * a.cache.page_stride + h * a.cache.head_stride + to % P * a.cache.slot_stride) * a.item;
            }
        }
    }
    const int64_t row = ((int64_t)s * a.cache.n_kv_heads + h) * a.row_stride;
    float w = 0.f;
    int o = 0;
    if (z == 0 && moves) {
        if (a.weights) w = a.weights[row + from];
        if (a.order) o = a.order[row + from];
    }
    __syncthreads();
    const int slice = z % a.slices * a.slice, pieces = min(a.slice, a.row_bytes - slice) / 16;
    char *pool = static_cast<char *>(z < a.slices ? a.cache.k : a.cache.v) + slice;
    for (int i = tid; i < n * pieces; i += kThreads) {
        const int64_t at = src[i / pieces];
        if (at >= 0) rows[i] = *reinterpret_cast<const uint4 *>(pool + at + i % pieces * 16);
    }
    __syncthreads();
    for (int i = tid; i < n * pieces; i += kThreads) {
        const int64_t at = dst[i / pieces];
        if (at >= 0) *reinterpret_cast<uint4 *>(pool + at + i % pieces * 16) = rows[i];
    }
    if (z == 0 && moves) {
        if (a.weights) a.weights[row + to] = w;
        if (a.order) a.order[row + to] = o;
    }
}

// Where the lengths are replaced: once all workgroups have read them.
__global__ __launch_bounds__(kThreads) void accept_lens(const AcceptArgs a, int32_t *lens)
{
    const int s = blockIdx.x * kThreads + threadIdx.x, cap = a.cache.max_pages * a.cache.page_size;
    if (s < a.cache.n_seqs) lens[s] = min(held(lens[s], 0, cap) + held(a.n_path[s], 0, a.max_path), cap);
}

}  // namespace
}  // namespace bs

extern "C" int bs_cache_accept(const bs_cache *cache, const int32_t *lens, int32_t *lens_out, const int32_t *path, const int32_t *n_path, int32_t max_path,
                               const bs_slots *slots, void *stream)
{
    using namespace bs;
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_rows_apart(*cache)) return rc;
    if (!lens || !lens_out || !n_path || max_path < 0 || max_path > BS_TREE_MAX_TOKENS || (!path && max_path > 0)) return BS_EINVAL;
    // the lengths that are written: in place of those that are read, or apart from all that is read
    const int64_t n = cache->n_seqs;
    if (lens_out != lens && overlap(lens_out, n, lens, n)) return BS_EINVAL;
    if (overlap(lens_out, n, n_path, n) || overlap(lens_out, n, path, n * max_path)) return BS_EINVAL;
    if (slots)
        if (int rc = check_slots(*cache, slots)) return rc;
    if (cache->n_kv_heads > 65535) return BS_EUNSUPPORTED;   // of a grid
    AcceptArgs a{};
    a.cache = *cache;
    a.lens = lens;
    a.path = path;
    a.n_path = n_path;
    a.lens_out = lens == lens_out ? nullptr : lens_out;
    a.max_path = max_path;
    a.item = element_bytes(cache->dtype);
    a.row_bytes = cache->head_dim * a.item;
    a.slice = std::min(a.row_bytes, max_path <= 128 ? 256 : 128);   // (32 KB of LDS at most)
    a.slices = (a.row_bytes + a.slice - 1) / a.slice;
    if (slots) {
        a.weights = slots->weights;
        a.order = slots->order;
        a.row_stride = slots->row_stride;
    }
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)cache->n_seqs, (unsigned)cache->n_kv_heads, (unsigned)(2 * a.slices));
    hipError_t err = launch_kernel(accept_rows, grid, dim3(kThreads), (size_t)max_path * a.slice, st, a);
    if (err != hipSuccess) return fail_hip(err, "accept_rows launch");
    if (lens == lens_out) err = launch_kernel(accept_lens, dim3((unsigned)((cache->n_seqs + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, a, lens_out);
    return err == hipSuccess ? BS_OK : fail_hip(err, "accept_lens launch");
}
