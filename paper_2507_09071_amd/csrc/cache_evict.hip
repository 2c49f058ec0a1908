// Eviction from a paged cache by accumulated attention weight.
//
// Per sequence and KV head ("row") the `keep` slots with the largest weights stay.  Weights are ranked as unsigned integers of the same
// order, protected slots above all; the rank of the last one kept is found from counts of its digits, 11, 11 and 10 bits from the top, and
// ties go to the lowest slots.  The first digit is sign, exponent and two bits of the fraction, over which weights spread well, so that few
// lanes of a wave count in the same place; mostly the second one leaves no more slots than are needed, and the third is not looked at.
// Kept slots behind `keep` move into the holes before it: the two sets do not overlap, so moves need no order among each other, and nothing
// moves that can stay.  A workgroup that has a row reads weights and orders (8 bytes a slot) once if they fit its registers, else the
// orders up to three times and the weights twice; in chunks every launch that ranks slots reads both again, up to five and four times.  Moves cost 4 rows each.
//
// Two ways to select.  One workgroup per row with the row's ranks in registers or LDS: one launch, all the chip where there are many rows.  Or a row
// cut into chunks for many workgroups, with a launch per pass: few long rows.  Bound: latency and vector instructions of counts and scans (512 rows of
// 4160 slots, 67 MB: 26 to 28 us, at a copy's rate 13), not memory; 4 rows of 39.5K, seven launches: 33 to 35 us (5.4).  Lengths are on the device, so
// the table's slots decide: those 512 rows take 28 us in a table of 4160 or 8192 slots, 36 in one of 32768 and 64 in one of 131072.
#include <algorithm>
#include <mutex>

#include "device_map.h"
#include "paged_cache.h"

namespace bs {
namespace {

constexpr int kMoveThreads = 256, kChunkThreads = 256;
constexpr int kBins = 2048, kDigits = 3;   // of digits of at most 11 bits

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
    int32_t *moves;             // [row][2 max_moves]: the slots moved into from the front, those they come from up to the end
    int32_t max_moves;
    int32_t at_once;            // the workgroup that selects moves as well
    // rows in chunks
    int32_t chunks;
    int32_t *need;              // of each row, how many ties stay
    int32_t *newest;            // [row][chunk] largest order
    int32_t *hist;              // [row][digit][bin]
    uint64_t *above, *ties;     // [row][words] slots that stay, and of those with the rank of the last one, a bit each
    int4 *marked;               // [row][chunk] how many of them: above in front of `keep` and behind, ties in front and behind
    int32_t words;
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

struct Row {
    const float *w;
    const int32_t *order;
    float *w_out;
    int32_t *order_out;
    int n;
    __device__ Row(const EvictArgs &a, int row)
        : w(a.weights + row * a.in_stride), order(a.order + row * a.in_stride), w_out(a.weights_out + row * a.out_stride),
          order_out(a.order_out + row * a.out_stride), n(used_slots(a, row / a.cache.n_kv_heads)) {}
    __device__ bool moves_out() const { return w_out != w || order_out != order; }
    __device__ void leave(int j, float x, int32_t o) const   // a slot that stays where it is
    {
        if (w_out != w) w_out[j] = x;
        if (order_out != order) order_out[j] = o;
    }
};

// f(slots of N of them) for the thread's slots from `begin` on, THREADS apart: loads of N slots go out together, those behind the end to the
// last slot.
template <int THREADS, int N, typename F>
__device__ inline void for_some(int begin, int end, F f)
{
    for (int j0 = begin; j0 < end; j0 += N * THREADS) {   // (uniform: `begin` is)
        int j[N];
#pragma unroll
        for (int e = 0; e < N; ++e) j[e] = j0 + e * THREADS + (int)threadIdx.x;
        f(j);
    }
}

// x of the lane that a data-parallel move names, 0 where there is none or its row is not in ROWS.
template <int MOVE, int ROWS>
__device__ inline int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, MOVE, ROWS, 0xf, false); }

// Sum over the lanes up to this one: within rows of 16 lanes, then the last lane of a row to the next one, then of the first half to the second.  (Six
// vector instructions; through LDS, as shuffles go, they wait for each other: 512 rows of 4160 slots 30.7 -> 28.7 us.)
__device__ inline int wave_upto(int x)
{
    x += moved<0x111, 0xf>(x);
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);
    x += moved<0x143, 0xc>(x);
    return x;
}

__device__ inline int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_upto(x), 63); }

__device__ inline int wave_max(int x)
{
    // (a lane without a partner: the smallest number)
    x = max(x, __builtin_amdgcn_update_dpp(INT32_MIN, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(INT32_MIN, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(INT32_MIN, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(INT32_MIN, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(INT32_MIN, x, 0x142, 0xa, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(INT32_MIN, x, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(x, 63);
}

template <int THREADS>
struct Sums { int wave[THREADS / 64]; };

// Exclusive sum over the threads; *total.  Two barriers.
template <int THREADS>
__device__ inline int sum_before(Sums<THREADS> &l, int x, int *total)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int upto = wave_upto(x);
    if (lane == 63) l.wave[wave] = upto;
    __syncthreads();
    const int waves_upto = wave_upto(lane < THREADS / 64 ? l.wave[lane] : 0);
    const int before = wave == 0 ? 0 : __builtin_amdgcn_readlane(waves_upto, wave - 1);
    __syncthreads();
    *total = __builtin_amdgcn_readlane(waves_upto, 63);
    return before + upto - x;
}

// How far the rank of the last slot kept is known: its bits from `shift` up; `need` of the in_bin slots that have these bits stay, and all
// that have larger ones.
struct Known {
    uint32_t prefix;
    int shift, need, in_bin;
    __device__ Known(int keep, int n) : prefix(0), shift(32), need(keep), in_bin(n) {}
    __device__ bool done() const { return shift == 0 || in_bin == need; }
    __device__ int bits() const { return shift == 10 ? 10 : 11; }   // of the next digit
    __device__ bool candidate(uint32_t r) const { return shift == 32 || (r >> shift) == prefix; }
    __device__ bool larger(uint32_t r) const { return shift != 32 && (r >> shift) > prefix; }
    __device__ int bin(uint32_t r) const { return (r >> (shift - bits())) & ((1 << bits()) - 1); }
};

// Of each digit, so that the next one need not wait until this one's have been read.
template <int THREADS>
struct DigitLds {
    int wave[kDigits][THREADS / 64];
    int digit[kDigits], need[kDigits], in_bin[kDigits];
};

// Counts a slot in `hist` (LDS).  A wave whose slots all count in one place adds them at once.
__device__ inline void count_in(int *hist, bool counts, int bin)
{
    const uint64_t who = __ballot(counts);
    if (who == 0) return;
    const int first = __builtin_amdgcn_readlane(bin, __builtin_ctzll(who));
    if (__ballot(counts && bin != first) == 0) {
        if ((threadIdx.x & 63) == 0) atomicAdd(&hist[first], __popcll(who));
    } else if (counts) {
        atomicAdd(&hist[bin], 1);
    }
}

// The next digit, from the counts of all its values.  Two barriers.
template <int THREADS>
__device__ inline void next_digit(DigitLds<THREADS> &l, const int *hist, Known &k)
{
    constexpr int EACH = kBins / THREADS;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i_digit = (32 - k.shift) / 11;
    int x[EACH], mine = 0;   // from the largest digit down
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        x[i] = hist[kBins - 1 - (int)threadIdx.x * EACH - i];
        mine += x[i];
    }
    const int upto = wave_upto(mine);
    if (lane == 63) l.wave[i_digit][wave] = upto;
    __syncthreads();
    const int waves_upto = wave_upto(lane < THREADS / 64 ? l.wave[i_digit][lane] : 0);
    int left = k.need - upto + mine - (wave == 0 ? 0 : __builtin_amdgcn_readlane(waves_upto, wave - 1));
    if (left > 0 && left <= mine) {
        bool found = false;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (!found && left <= x[i]) {
                found = true;
                l.digit[i_digit] = kBins - 1 - (int)threadIdx.x * EACH - i;
                l.need[i_digit] = left;
                l.in_bin[i_digit] = x[i];
            }
            if (!found) left -= x[i];
        }
    }
    __syncthreads();
    const int bits = k.bits();
    k.prefix = (k.shift == 32 ? 0 : k.prefix << bits) | (uint32_t)l.digit[i_digit];
    k.shift -= bits;
    k.need = l.need[i_digit];
    k.in_bin = l.in_bin[i_digit];
}

__device__ inline bool is_safe(const EvictArgs &a, int32_t order, int32_t newest)
{
    return order < a.keep_first || (int64_t)order > (int64_t)newest - a.keep_last;
}

__device__ inline int64_t slot_offset(const bs_cache &c, int seq, int head, int slot)   // in elements; -1: no page
{
    const int page = c.page_table[(int64_t)seq * c.max_pages + slot / c.page_size];
    if (page < 0 || page >= c.n_pages) return -1;
    return page * c.page_stride + head * c.head_stride + (slot % c.page_size) * c.slot_stride;
}

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

constexpr int kMovesAtOnce = 256;

// The `n` moves of a row, at most kMovesAtOnce, by one workgroup: where they go from and to, a thread each, then the rows, 16 bytes a thread and
// four of them under way.
template <int THREADS>
__device__ inline void do_moves(const EvictArgs &a, int row, unsigned n)
{
    __shared__ int64_t to[kMovesAtOnce], from[kMovesAtOnce];   // in bytes; to = -1: nothing to copy
    const int seq = row / a.cache.n_kv_heads, head = row - seq * a.cache.n_kv_heads, tid = threadIdx.x;
    const int bytes = a.cache.dtype == BS_BF16 ? 2 : 4;
    const unsigned pieces = a.cache.head_dim * bytes / 16, all = n * pieces;
    const int32_t *moves = a.moves + (int64_t)row * 2 * a.max_moves;
    char *k = static_cast<char *>(a.cache.k), *v = static_cast<char *>(a.cache.v);
    if (tid < (int)n) {
        const int dst = moves[tid], src = moves[2 * a.max_moves - (int)n + tid];
        const float w = a.weights[row * a.in_stride + src];
        const int32_t o = a.order[row * a.in_stride + src];
        const int64_t d = slot_offset(a.cache, seq, head, dst), s = slot_offset(a.cache, seq, head, src);
        to[tid] = d < 0 || s < 0 ? -1 : d * bytes;   // (the caller sees to it that both have a page)
        from[tid] = s * bytes;
        a.weights_out[row * a.out_stride + dst] = w;
        a.order_out[row * a.out_stride + dst] = o;
    }
    __syncthreads();
    for (unsigned idx0 = tid; idx0 < all; idx0 += 4 * THREADS) {
        uintx4 x[4], y[4];
        int64_t at[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const unsigned idx = min(idx0 + u * THREADS, all - 1), i = idx / pieces, p = idx - i * pieces;   // (behind the last one: that again)
            const int64_t dst = to[i];
            at[u] = dst < 0 ? -1 : dst + 16 * p;
            x[u] = *reinterpret_cast<const uintx4 *>(k + (dst < 0 ? 0 : from[i] + 16 * p));
            y[u] = *reinterpret_cast<const uintx4 *>(v + (dst < 0 ? 0 : from[i] + 16 * p));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (at[u] >= 0) {
                *reinterpret_cast<uintx4 *>(k + at[u]) = x[u];
                *reinterpret_cast<uintx4 *>(v + at[u]) = y[u];
            }
        }
    }
}

// ------------------------------------------------------------------------------------ one workgroup per row

constexpr int kRanksMax = 32768;   // 128 KB of LDS
// Beside them: three histograms, what is known of the digits, sums, a count of each 64 slots, the newest order, the moves.
static_assert(kRanksMax * 4 + kDigits * kBins * 4 + sizeof(DigitLds<1024>) + sizeof(Sums<1024>) + kRanksMax / 64 * 4 + 4 + kMovesAtOnce * 16 <= 160 * 1024 - 64, "LDS of a CU");
static_assert(kRanksMax <= 32768, "kept slots and ties are counted in 16 bits each");

// SLOTS > 0: a thread has at most so many slots and keeps them in registers.  Else ranks lie in LDS, and orders and weights are read again.
template <int THREADS, int SLOTS>
__global__ __launch_bounds__(THREADS, 4) void evict_select(const EvictArgs a)
{
    constexpr bool SHORT = SLOTS > 0;
    constexpr int N = SHORT ? SLOTS : 8, kFlags = (SHORT ? SLOTS * THREADS : kRanksMax) / 64;
    __shared__ int hist[kDigits * kBins];
    __shared__ DigitLds<THREADS> digits;
    __shared__ Sums<THREADS> sums;
    __shared__ int flags[kFlags];   // of each 64 slots, how many; then how many before
    __shared__ int newest_lds;
    extern __shared__ uint32_t ranks[];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const Row r(a, row);
    const int n = r.n;
    if (n <= a.keep) {
        for (int j = tid; j < n; j += THREADS) r.leave(j, r.w[j], r.order[j]);
        if (tid == 0) a.counts[row] = 0;
        return;
    }
    uint32_t rank[N];
    int32_t o[N];
    float x[N];
    const auto load = [&](const int (&j)[N]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            o[e] = r.order[min(j[e], n - 1)];
            x[e] = r.w[min(j[e], n - 1)];
        }
    };
    // f(slot, its rank), for all slots; slots behind the last one have no bit set in what f forms of them
    const auto for_slots = [&](auto f) __attribute__((always_inline)) {
        if constexpr (SHORT) {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (e * THREADS < n) f(e * THREADS + tid, rank[e]);
        } else {
            for (int j0 = 0; j0 < n; j0 += THREADS) f(j0 + tid, ranks[j0 + tid]);   // (there is room for whole rounds)
        }
    };
    if (tid == 0) newest_lds = INT32_MIN;
    int newest = INT32_MIN;
    for_some<THREADS, N>(0, n, [&](const int (&j)[N]) {
        load(j);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            newest = max(newest, o[e]);
            if constexpr (!SHORT) { if (j[e] < n) ranks[j[e]] = rank_of(x[e], false); }
        }
    });
    for (int i = tid; i < kDigits * kBins; i += THREADS) hist[i] = 0;
    __syncthreads();
    newest = wave_max(newest);
    if (lane == 0) atomicMax(&newest_lds, newest);
    __syncthreads();
    newest = newest_lds;
    if constexpr (SHORT) {
#pragma unroll
        for (int e = 0; e < N; ++e) rank[e] = rank_of(x[e], is_safe(a, o[e], newest));
    } else {
        for_some<THREADS, N>(0, n, [&](const int (&j)[N]) {   // (a thread's own slots)
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = r.order[min(j[e], n - 1)];
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (j[e] < n && is_safe(a, o[e], newest)) ranks[j[e]] = ~0u;
        });
    }
    Known known(a.keep, n);
    for (int digit = 0; digit < kDigits && !known.done(); ++digit) {
        for_slots([&](int j, uint32_t &u) { count_in(hist + digit * kBins, j < n && known.candidate(u), known.bin(u)); });
        __syncthreads();
        next_digit(digits, hist + digit * kBins, known);
    }

    // How many ties (low half) and how many larger ones lie before each 64 slots: counts, then their sum in the order of slots.
    for_slots([&](int j, uint32_t &u) {
        const uint64_t tie = __ballot(j < n && known.candidate(u)), larger = __ballot(j < n && known.larger(u));
        if (lane == 0 && j < n) flags[j / 64] = __popcll(larger) << 16 | __popcll(tie);
    });
    __syncthreads();
    {
        constexpr int EACH = (kFlags + THREADS - 1) / THREADS;
        const int entries = (n + 63) / 64;
        int mine = 0, c[EACH], total;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            c[i] = tid * EACH + i < entries ? flags[tid * EACH + i] : 0;
            mine += c[i];
        }
        int before = sum_before(sums, mine, &total);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (tid * EACH + i < entries) flags[tid * EACH + i] = before;
            before += c[i];
        }
    }
    __syncthreads();
    // Of equal ranks the lowest slots stay.  A hole in front is on the list behind as many as were evicted before it, a slot that moves in front of as
    // many as are kept behind it.
    int32_t *moves = a.moves + (int64_t)row * 2 * a.max_moves;
    for_slots([&](int j, uint32_t &u) {
        const bool tie = j < n && known.candidate(u), more = j < n && known.larger(u);
        const uint64_t below = (1ull << lane) - 1, all_ties = __ballot(tie), all_more = __ballot(more);
        const uint32_t before = flags[min(j, n - 1) / 64];
        const int ties = (int)(before & 0xffffu) + __popcll(all_ties & below), kept = (int)(before >> 16) + __popcll(all_more & below) + min(ties, known.need);
        const bool stays = more || (tie && ties < known.need);
        if (j < a.keep && !stays) moves[j - kept] = j;
        if (j < n && j >= a.keep && stays) moves[2 * a.max_moves - a.keep + kept] = j;
        if (j == a.keep - 1) digits.need[0] = a.keep - kept - stays;   // how many
        if (j < n) u = stays;   // all that matters from here on
    });
    __syncthreads();
    const int n_moves = digits.need[0];
    if (r.moves_out())
        for_some<THREADS, N>(0, a.keep, [&](const int (&j)[N]) {
            if constexpr (!SHORT) load(j);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t stays = SHORT ? rank[e] : ranks[min(j[e], n - 1)];
                if (j[e] < a.keep && stays) r.leave(j[e], x[e], o[e]);
            }
        });
    if (a.at_once) do_moves<THREADS>(a, row, n_moves);   // (behind a barrier: the list is there)
    else if (tid == 0) a.counts[row] = n_moves;
}

// The lengths, for a call whose first kernel also moves: its workgroups read them.
__global__ __launch_bounds__(kMoveThreads) void evict_lengths(const EvictArgs a)
{
    const int seq = blockIdx.x * kMoveThreads + threadIdx.x;
    if (seq < a.cache.n_seqs) a.lens_out[seq] = min(used_slots(a, seq), a.keep);
}

// ------------------------------------------------------------------------------------ rows in chunks

// Slots [begin, end) of chunk blockIdx.y, whole 64s.
struct Chunk {
    int begin, end;
    __device__ Chunk(const EvictArgs &a, int n)
    {
        const int words = (n + 63) / 64, each = (words + a.chunks - 1) / a.chunks;
        begin = min(n, (int)blockIdx.y * each * 64);
        end = min(n, begin + each * 64);
    }
};

__global__ __launch_bounds__(kChunkThreads) void evict_newest(const EvictArgs a)
{
    __shared__ int waves[kChunkThreads / 64];
    const int row = blockIdx.x, tid = threadIdx.x;
    const Row r(a, row);
    const Chunk c(a, r.n);
    for (int i = (int)blockIdx.y * kChunkThreads + tid; i < kDigits * kBins; i += (int)gridDim.y * kChunkThreads) a.hist[(int64_t)row * kDigits * kBins + i] = 0;
    if (r.n <= a.keep) {   // (the kernels behind have nothing to do then)
        if (r.moves_out())
            for (int j = c.begin + tid; j < c.end; j += kChunkThreads) r.leave(j, r.w[j], r.order[j]);
        if (blockIdx.y == 0 && tid == 0) a.counts[row] = 0;
        return;
    }
    int newest = INT32_MIN;
    for_some<kChunkThreads, 8>(c.begin, c.end, [&](const int (&j)[8]) {
        int32_t o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = r.order[min(j[e], c.end - 1)];
#pragma unroll
        for (int e = 0; e < 8; ++e) newest = max(newest, o[e]);
    });
    newest = wave_max(newest);
    if ((tid & 63) == 0) waves[tid >> 6] = newest;
    __syncthreads();
    if (tid == 0) a.newest[(int64_t)row * a.chunks + blockIdx.y] = max(max(waves[0], waves[1]), max(waves[2], waves[3]));
}

// The largest order of the row, from those of its chunks (fewer than there are threads in a wave: chunks <= 64).
__device__ inline int32_t newest_of(const EvictArgs &a, int row)
{
    const int lane = threadIdx.x & 63;
    return wave_max(lane < a.chunks ? a.newest[(int64_t)row * a.chunks + lane] : INT32_MIN);
}

// What is known of the last rank after `n_digits` digits have been counted.
__device__ inline Known known_after(DigitLds<kChunkThreads> &l, const EvictArgs &a, int row, int n, int n_digits)
{
    Known k(a.keep, n);
    for (int i = 0; i < n_digits && !k.done(); ++i) next_digit(l, a.hist + ((int64_t)row * kDigits + i) * kBins, k);
    return k;
}

// Orders and weights of eight slots of a thread, those behind the chunk's end of its last one.
struct Eight {
    int32_t o[8];
    float x[8];
    __device__ void load(const Row &r, const Chunk &c, const int (&j)[8])
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            o[e] = r.order[min(j[e], c.end - 1)];
            x[e] = r.w[min(j[e], c.end - 1)];
        }
    }
    __device__ void load_first(const Row &r, const Chunk &c)
    {
        int j[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) j[e] = c.begin + e * kChunkThreads + (int)threadIdx.x;
        load(r, c, j);
    }
};

// f(slots, ranks, what was loaded) of eight slots of the chunk at a time; a rank behind the end is not one.  The first eight are there: they are
// requested before anything else.
template <typename F>
__device__ inline void for_ranks(const EvictArgs &a, const Row &r, const Chunk &c, Eight &v, int32_t newest, F f)
{
    for_some<kChunkThreads, 8>(c.begin, c.end, [&](const int (&j)[8]) {
        if (j[0] != c.begin + (int)threadIdx.x) v.load(r, c, j);
        uint32_t rank[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) rank[e] = rank_of(v.x[e], is_safe(a, v.o[e], newest));
        f(j, rank, v);
    });
}

// Counts of the digit behind those that are known; rows whose last rank is known well enough are left.
__global__ __launch_bounds__(kChunkThreads) void evict_count(const EvictArgs a, int digit)
{
    __shared__ int hist[kBins];
    __shared__ DigitLds<kChunkThreads> digits;
    const int row = blockIdx.x, tid = threadIdx.x;
    const Row r(a, row);
    const Chunk c(a, r.n);
    if (r.n <= a.keep || c.begin >= c.end) return;
    Eight v;
    v.load_first(r, c);
    const int32_t newest = newest_of(a, row);
    for (int i = tid; i < kBins; i += kChunkThreads) hist[i] = 0;
    const Known k = known_after(digits, a, row, r.n, digit);
    if (k.done()) return;
    __syncthreads();
    for_ranks(a, r, c, v, newest, [&](const int (&j)[8], const uint32_t (&rank)[8], const Eight &) {
#pragma unroll
        for (int e = 0; e < 8; ++e) count_in(hist, j[e] < c.end && k.candidate(rank[e]), k.bin(rank[e]));
    });
    __syncthreads();
    int *all = a.hist + ((int64_t)row * kDigits + digit) * kBins;
    for (int i = tid; i < kBins; i += kChunkThreads)
        if (hist[i] > 0) atomicAdd(&all[i], hist[i]);
}

// Which slots stay: a bit each, ties apart where only some of them do.
__global__ __launch_bounds__(kChunkThreads) void evict_mark(const EvictArgs a)
{
    __shared__ DigitLds<kChunkThreads> digits;
    const int row = blockIdx.x;
    const Row r(a, row);
    const Chunk c(a, r.n);
    if (r.n <= a.keep || c.begin >= c.end) return;
    Eight v;
    v.load_first(r, c);
    const int32_t newest = newest_of(a, row);
    const Known k = known_after(digits, a, row, r.n, kDigits);
    const bool some = k.in_bin > k.need, out = r.moves_out();
    int4 counts = make_int4(0, 0, 0, 0);
    for_ranks(a, r, c, v, newest, [&](const int (&j)[8], const uint32_t (&rank)[8], const Eight &u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool has = j[e] < c.end, tie = has && k.candidate(rank[e]), stays = has && (k.larger(rank[e]) || (tie && !some));
            const uint64_t above = __ballot(stays), ties = some ? __ballot(tie) : 0;
            if ((threadIdx.x & 63) == 0 && has) {
                a.above[(int64_t)row * a.words + j[e] / 64] = above;
                a.ties[(int64_t)row * a.words + j[e] / 64] = ties;
            }
            const bool front = j[e] < a.keep;
            counts.x += stays && front; counts.y += stays && !front;
            counts.z += some && tie && front; counts.w += some && tie && !front;
            if (out && stays && front) r.leave(j[e], u.x[e], u.o[e]);
        }
    });
    __shared__ int4 waves[kChunkThreads / 64];
    counts = make_int4(wave_sum(counts.x), wave_sum(counts.y), wave_sum(counts.z), wave_sum(counts.w));
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = counts;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kChunkThreads / 64; ++w) {
            counts.x += waves[w].x; counts.y += waves[w].y; counts.z += waves[w].z; counts.w += waves[w].w;
        }
        a.marked[(int64_t)row * a.chunks + blockIdx.y] = counts;
        if (blockIdx.y == 0) a.need[row] = k.need;
    }
}

// The chunk's part of the list of a row's moves: a thread counts 64 slots, a wave writes them.  Of the ties the lowest stay.
__global__ __launch_bounds__(kChunkThreads) void evict_list(const EvictArgs a)
{
    __shared__ Sums<kChunkThreads> sums;
    __shared__ uint64_t lists[kChunkThreads];
    __shared__ int places[kChunkThreads];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const Row r(a, row);
    const Chunk c(a, r.n);
    if (r.n <= a.keep || c.begin >= c.end) return;
    // what the chunks in front of this one have, and all (a wave has them all: chunks <= 64)
    const int words = (r.n + 63) / 64, each = (words + a.chunks - 1) / a.chunks * 64;
    const int begin = min(r.n, lane * each), end = min(r.n, begin + each);
    const int4 m = lane < a.chunks && begin < end ? a.marked[(int64_t)row * a.chunks + lane] : make_int4(0, 0, 0, 0);
    const int need = a.need[row], ties = m.z + m.w, kept = max(0, min(ties, need - (wave_upto(ties) - ties))), kept_front = min(kept, m.z);
    const int holes = min(max(a.keep - begin, 0), end - begin) - m.x - kept_front, late = m.y + kept - kept_front;
    const int upto = wave_upto(holes + late);
    const int ties_before = __shfl(wave_upto(ties) - ties, (int)blockIdx.y, 64), list_before = __shfl(upto - holes - late, (int)blockIdx.y, 64);
    const int all_listed = __shfl(upto, 63, 64);
    if (blockIdx.y == 0 && tid == 0) a.counts[row] = all_listed / 2;

    const uint64_t *above_words = a.above + (int64_t)row * a.words, *ties_words = a.ties + (int64_t)row * a.words;
    int32_t *moves = a.moves + (int64_t)row * 2 * a.max_moves;
    int ties_so_far = ties_before, so_far = list_before, total;
    for (int w0 = c.begin / 64; w0 * 64 < c.end; w0 += kChunkThreads) {
        const int word = w0 + tid;
        const bool has = word * 64 < c.end;
        uint64_t stays = has ? above_words[word] : 0, tie = has ? ties_words[word] : 0;
        const int left = need - ties_so_far - sum_before(sums, __popcll(tie), &total);
        ties_so_far += total;
        for (int drop = __popcll(tie) - max(left, 0); drop > 0; --drop) tie &= ~(1ull << (63 - __builtin_clzll(tie)));
        stays |= tie;
        const int front = has ? min(max(a.keep - word * 64, 0), 64) : 0, in_word = has ? min(r.n - word * 64, 64) : 0;   // slots in front of `keep`, slots
        const uint64_t in_front = front == 64 ? ~0ull : (1ull << front) - 1, all = in_word == 64 ? ~0ull : (1ull << in_word) - 1;
        const uint64_t list = ((~stays & in_front) | (stays & ~in_front)) & all;   // evicted in front, kept behind
        if (r.moves_out())
            for (tie &= in_front; tie != 0; tie &= tie - 1) {
                const int j = word * 64 + __builtin_ctzll(tie);
                r.leave(j, r.w[j], r.order[j]);
            }
        lists[tid] = list;
        places[tid] = so_far + sum_before(sums, __popcll(list), &total);   // (its barriers are behind both)
        so_far += total;
        __syncthreads();
        for (int i = tid >> 6; i < kChunkThreads && (w0 + i) * 64 < c.end; i += kChunkThreads / 64) {
            const uint64_t x = lists[i];
            const int at = places[i] + __popcll(x & ((1ull << lane) - 1));   // holes first
            if ((x >> lane) & 1) moves[at < all_listed / 2 ? at : 2 * a.max_moves - all_listed + at] = (w0 + i) * 64 + lane;
        }
        __syncthreads();
    }
}

// A move by as many threads as a row has pieces of 16 bytes.
__global__ __launch_bounds__(kMoveThreads) void evict_move(const EvictArgs a)
{
    const int row = blockIdx.x, n = a.counts[row], seq = row / a.cache.n_kv_heads, head = row - seq * a.cache.n_kv_heads;
    const int bytes = a.cache.dtype == BS_BF16 ? 2 : 4, pieces = a.cache.head_dim * bytes / 16;
    const int32_t *moves = a.moves + (int64_t)row * 2 * a.max_moves;
    char *k = static_cast<char *>(a.cache.k), *v = static_cast<char *>(a.cache.v);
    for (int64_t idx = (int64_t)blockIdx.y * kMoveThreads + threadIdx.x; idx < (int64_t)n * pieces; idx += (int64_t)gridDim.y * kMoveThreads) {
        const int i = (int)(idx / pieces), p = (int)(idx - (int64_t)i * pieces);
        const int to = moves[i], from = moves[2 * a.max_moves - n + i];
        const int64_t dst = slot_offset(a.cache, seq, head, to), src = slot_offset(a.cache, seq, head, from);
        if (dst >= 0 && src >= 0) {
            const uintx4 x = *reinterpret_cast<const uintx4 *>(k + src * bytes + 16 * p), y = *reinterpret_cast<const uintx4 *>(v + src * bytes + 16 * p);
            *reinterpret_cast<uintx4 *>(k + dst * bytes + 16 * p) = x;
            *reinterpret_cast<uintx4 *>(v + dst * bytes + 16 * p) = y;
        }
        if (p == 0) {
            a.weights_out[row * a.out_stride + to] = a.weights[row * a.in_stride + from];
            a.order_out[row * a.out_stride + to] = a.order[row * a.in_stride + from];
        }
    }
    // (the kernels before have read the lengths)
    if (blockIdx.y == 0 && head == 0 && threadIdx.x == 0) a.lens_out[seq] = min(used_slots(a, seq), a.keep);
}

int check_evict(const bs_cache *cache, int32_t keep)
{
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_rows_apart(*cache)) return rc;
    if (keep < 1) return BS_EINVAL;
    // A grid has fewer than 2^32 threads (see launch_select), with which sizes of the workspace stay within 64 bits.
    const int64_t capacity = cache_slots(*cache), threads = capacity > kRanksMax || capacity <= 8 * 256 ? 256 : capacity <= 16 * 512 ? 512 : 1024;
    if ((int64_t)cache->n_seqs * cache->n_kv_heads * threads > UINT32_MAX) return BS_EUNSUPPORTED;
    return BS_OK;
}

// How a call is laid out and its workspace.
struct Plan {
    int64_t rows, moves;
    int32_t chunks, words;      // chunks 0: one workgroup per row
    bool at_once;
    int64_t at_moves, at_need, at_newest, at_hist, at_above, at_ties, at_marked, bytes;
};

Plan make_plan(const bs_cache &c, int32_t keep)
{
    Plan p{};
    const int64_t capacity = cache_slots(c);
    p.rows = (int64_t)c.n_seqs * c.n_kv_heads;
    p.moves = std::max<int64_t>(0, std::min<int64_t>(keep, capacity - keep));
    // Rows beyond what LDS holds, and few long ones, whose CUs would be too few.  Cut back to half, a workgroup each / in chunks: 4 rows of 8K slots
    // 15.8 / 29.6 us, of 16K 29.0 / 31.4, of 30K 49.4 / 34.8; 32 rows 29.8 / 45.6, 58.4 / 62.9, 101 / 92.
    if (capacity > kRanksMax || (p.rows <= 32 && capacity > 20480)) {
        p.chunks = (int32_t)std::max<int64_t>(1, std::min<int64_t>({64, (capacity + 1023) / 1024, (1024 + p.rows - 1) / p.rows}));
        p.words = (int32_t)((capacity + 63) / 64);
    }
    p.at_once = p.chunks == 0 && p.moves <= kMovesAtOnce;   // (512 rows of 4160 slots, 64 moves: 31.4 us with a kernel for the moves, 28.0 so)
    const auto whole = [](int64_t bytes) { return (bytes + 255) / 256 * 256; };
    p.at_moves = whole(p.rows * 4);
    p.at_need = p.at_moves + whole(p.rows * p.moves * 8);
    p.at_newest = p.at_need + (p.chunks ? whole(p.rows * 4) : 0);
    p.at_hist = p.at_newest + whole(p.rows * p.chunks * 4);
    p.at_above = p.at_hist + (p.chunks ? p.rows * kDigits * kBins * 4 : 0);
    p.at_ties = p.at_above + whole(p.rows * p.words * 8);
    p.at_marked = p.at_ties + whole(p.rows * p.words * 8);
    p.bytes = p.at_marked + p.rows * p.chunks * 16;
    return p;
}

std::mutex g_mutex;
bool g_limits[64];   // dynamic LDS of a device's kernels raised

hipError_t device_setup()
{
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(g_mutex);
    if (g_limits[dev]) return hipSuccess;
    const void *const k = reinterpret_cast<const void *>(evict_select<1024, 0>);
    if ((e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, kRanksMax * 4)) != hipSuccess) return e;
    g_limits[dev] = true;
    return hipSuccess;
}

hipError_t launch_select(const EvictArgs &a, const Plan &p, hipStream_t st)
{
    const int64_t capacity = cache_slots(a.cache);
    if (p.chunks == 0) {
        const dim3 grid((unsigned)p.rows);
        // Eight slots a thread; more only where there are more rows than CUs, which then share one: what a wave does besides its slots (scans,
        // barriers) counts.  Rows of 4160 slots, with 1024 threads / 512 of 16 slots: 512 rows 34.1 / 28.0 us, 128 of 8000 20.1 / 24.6.
        if (capacity <= 8 * 256) return launch_kernel(evict_select<256, 8>, grid, dim3(256), 0, st, a);
        if (capacity <= 8 * 512) return launch_kernel(evict_select<512, 8>, grid, dim3(512), 0, st, a);
        if (capacity <= 8 * 1024 && p.rows <= 256) return launch_kernel(evict_select<1024, 8>, grid, dim3(1024), 0, st, a);
        if (capacity <= 16 * 512) return launch_kernel(evict_select<512, 16>, grid, dim3(512), 0, st, a);
        if (const hipError_t e = device_setup(); e != hipSuccess) return e;
        return launch_kernel(evict_select<1024, 0>, grid, dim3(1024), (capacity + 1023) / 1024 * 4096, st, a);
    }
    const dim3 grid((unsigned)p.rows, (unsigned)p.chunks), block(kChunkThreads);
    hipError_t e = launch_kernel(evict_newest, grid, block, 0, st, a);
    for (int digit = 0; digit < kDigits && e == hipSuccess; ++digit) e = launch_kernel(evict_count, grid, block, 0, st, a, digit);
    if (e == hipSuccess) e = launch_kernel(evict_mark, grid, block, 0, st, a);
    if (e == hipSuccess) e = launch_kernel(evict_list, grid, block, 0, st, a);
    return e;
}

}  // namespace
}  // namespace bs

extern "C" int64_t bs_cache_evict_workspace(const bs_cache *cache, int32_t keep)
{
    using namespace bs;
    if (int rc = check_evict(cache, keep)) return rc;
    return make_plan(*cache, keep).bytes;
}

extern "C" int bs_cache_evict(const bs_cache *cache, const int32_t *lens, int32_t *lens_out, int32_t keep, int32_t keep_first, int32_t keep_last,
                              const bs_slots *slots, const bs_slots *slots_out, void *workspace, int64_t workspace_bytes, void *stream)
{
    using namespace bs;
    if (int rc = check_evict(cache, keep)) return rc;
    if (!lens || !lens_out || !slots || !slots_out || !workspace || keep_first < 0 || keep_last < 0 || (int64_t)keep_first + keep_last > keep) return BS_EINVAL;
    if (!slots->weights || !slots->order || !slots_out->weights || !slots_out->order) return BS_EINVAL;
    if (check_slots(*cache, slots) || check_slots(*cache, slots_out)) return BS_EINVAL;
    const Plan p = make_plan(*cache, keep);
    if ((uintptr_t)workspace % 16 != 0 || workspace_bytes < p.bytes) return BS_EINVAL;
    // the same arrays, or others: in place, rows lie where they lay
    if ((slots->weights == slots_out->weights || slots->order == slots_out->order) && slots->row_stride != slots_out->row_stride) return BS_EINVAL;
    EvictArgs a{};
    a.cache = *cache;
    a.lens = lens;
    a.lens_out = lens_out;
    a.keep = keep; a.keep_first = keep_first; a.keep_last = keep_last;
    a.weights = slots->weights; a.order = slots->order; a.in_stride = slots->row_stride;
    a.weights_out = slots_out->weights; a.order_out = slots_out->order; a.out_stride = slots_out->row_stride;
    char *ws = static_cast<char *>(workspace);
    a.counts = reinterpret_cast<int32_t *>(ws);
    a.moves = reinterpret_cast<int32_t *>(ws + p.at_moves);
    a.max_moves = (int32_t)p.moves;
    a.at_once = p.at_once;
    a.chunks = p.chunks;
    a.need = reinterpret_cast<int32_t *>(ws + p.at_need);
    a.newest = reinterpret_cast<int32_t *>(ws + p.at_newest);
    a.hist = reinterpret_cast<int32_t *>(ws + p.at_hist);
    a.above = reinterpret_cast<uint64_t *>(ws + p.at_above);
    a.ties = reinterpret_cast<uint64_t *>(ws + p.at_ties);
    a.marked = reinterpret_cast<int4 *>(ws + p.at_marked);
    a.words = p.words;
    hipStream_t st = (hipStream_t)stream;
    hipError_t e = launch_select(a, p, st);
    if (e != hipSuccess) return fail_hip(e, "eviction: select launch");
    const dim3 block(kMoveThreads);
    if (p.at_once) {
        e = launch_kernel(evict_lengths, dim3((unsigned)((cache->n_seqs + kMoveThreads - 1) / kMoveThreads)), block, 0, st, a);
        return e == hipSuccess ? BS_OK : fail_hip(e, "evict_lengths launch");
    }
    const int64_t pieces = (int64_t)cache->head_dim * element_bytes(cache->dtype) / 16;
    const int64_t blocks = std::max<int64_t>(1, std::min({(p.moves * pieces + kMoveThreads - 1) / kMoveThreads, (int64_t)1024, (4096 + p.rows - 1) / p.rows}));
    e = launch_kernel(evict_move, dim3((unsigned)p.rows, (unsigned)blocks), block, 0, st, a);
    return e == hipSuccess ? BS_OK : fail_hip(e, "evict_move launch");
}
