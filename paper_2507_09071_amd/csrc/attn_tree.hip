// Attention of a few drafted tokens per sequence (a tree or a chain) over a paged cache.
//
// K and V of a KV head are read once for the T tokens times G query heads that share them, so the work per byte grows with the tree: of a slot's 4 d bytes (bf16)
// 4 d T G FLOP are made, 8 d T G with the probabilities in three numbers.  Up to some thirty rows (T G) HBM bounds it, beyond that what matrix and vector instructions
// take; fp32 is bounded by the matrix pipe from sixteen rows on.  How:
//  * the T G rows of a sequence and KV head are cut into groups of at most M rows; an item is such a group.  More rows than M walk the cache again.  Up to 32 rows
//    four waves take every fourth block of slots each, on their own (tree_shares); more share their blocks and step together: in bf16 four waves of 32 rows
//    (tree_wide), in fp32 two such groups of four.  Which when: rows_of, at the end;
//  * the blocks of all items lie in one row that is cut into equal shares, one per workgroup, found on the device from the lengths; parts of items that were cut
//    are joined by a second kernel in a fixed order;
//  * masks cost nothing but at the end: slots below the length are seen by all, and only blocks that reach behind it (or hold the begin of a window, or a slot
//    without a page) are masked, by 32 bits per row and block.  A window is laid on the words of a token's mask.
// With d 128 in bf16, where a plain read reaches 6.2 TB/s, joins included: two sequences of 150K slots, 16 KV heads, 128 rows of each, 2.47 GB of K and V: 645 to 665 us; its
// loads alone take 450, and what holds the rest back is power, of which the products of the probabilities' three numbers take their share (two numbers: 578).  One of
// 39.5K slots, 4 KV heads, 182 rows, 81 MB that are walked twice: 49 to 51 us.  48 sequences of up to 16K slots, 8 KV heads, up to 80 rows, 504 MB, capped scores: 126 to 131 us.
#include "attn_common.h"
#include "cache_attn.h"

#include <algorithm>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "device_map.h"
#include "paged_cache.h"

namespace bs {
namespace {

// An item in more than one share: the first and the last workgroup that have a part of it, and its rows: n_rows from row0 on of a KV head, of the sequence whose first
// token is `token`.  Filed under the item where there are fewer items than shares, else under the first share; no rows: nothing to join.
struct __align__(16) Cut { int32_t first, last, kvh, row0, n_rows, token, unused[2]; };

struct TreeArgs {
    bs_cache cache;
    const void *q;
    void *out;
    int64_t q_head, q_token, out_head, out_token;
    const int32_t *first, *lens;
    const uint64_t *mask;
    int32_t n_tokens, max_tokens, mask_words;
    int32_t G, window, most_items;   // heads per KV head; items of a sequence at most
    float inv_g;                  // 1 / G
    float scale_log2e;            // of scores as they are, or
    float to_cap, cap_log2e;      // cap > 0: scale / cap, cap log2(e)
    float *part_o;                // [2 shares][M][d]: of share w, 2 w the item that began before it, 2 w + 1 the one that goes on behind it
    float2 *part_ml;              // reference point and sum
    Cut *cuts;
    int32_t by_item;
};

// NRB blocks of 16 rows per wave, WR waves that share a block of slots, WK such groups of waves that take turns.
template <typename T, int D, int NRB, int WR, int WK>
struct Layout {
    static constexpr int kWaves = WR * WK, kThreads = 64 * kWaves, kRows = 16 * NRB * WR, kTurns = WK;
    static constexpr int kEven = 0;
    static constexpr int kItem = 10;                          // beginning an item costs about as much as so many blocks: shares are equal with that counted
                                                              // (200 sequences of 200 to 2K slots, 16 rows, with 4, 6, 8, 10, 12, 16: 152, 144, 139, 136, 138,
                                                              // 140 us; 48 of up to 16K, 30 rows: 169, 140, 123, 115, 114, 117)
    static constexpr int kKeys = sizeof(T) == 2 ? 32 : 16;    // slots of a block
    static constexpr int kRowBytes = D * (int)sizeof(T);
    static constexpr int kBlock = kKeys * kRowBytes;          // one block of K or V
    static constexpr int kLoads = kBlock / 1024;              // LDS-direct instructions per block
    static constexpr int kLoads16 = 16 * kRowBytes / 1024;    // ... per 16 slots, which lie in one page
    static constexpr int kOwn = (kLoads + WR - 1) / WR;       // ... of a wave
    static constexpr int kGroup = 2 * 2 * kBlock;             // ring of a group of waves: two blocks of K and V
    static constexpr int kQuery = WK * kGroup;                // the query rows behind the rings
    static constexpr int kMerge = WR > 1 ? kRows * D * 4 : kGroup;   // a group's results lie over the ring; where its waves have it alone, over its own part
    static constexpr int kEnd = kQuery + kRows * kRowBytes > WK * kMerge ? kQuery + kRows * kRowBytes : WK * kMerge;
    static constexpr int kMl = kEnd;                          // [groups][rows]
    static constexpr int kLds = kMl + WK * kRows * 8;
    static constexpr int kPerCu = D == 64 && WR == 1 ? 2 : 1; // workgroups per CU
    static_assert((kLds + 1024) * kPerCu <= 160 * 1024, "LDS of a CU");   // (with what own_range has)
    static_assert(kRows * D * 4 <= kMerge, "a group's results");
    // exchange of the 16-byte chunks of row r: rows that share their banks get different chunks
    __device__ static int swizzle(int r) { return kRowBytes == 128 ? (r >> 1) & 7 : r & 15; }
};


typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// x as three bf16 numbers each, which hold all 24 bits of its fraction: what each leaves over is exact.  Where values cancel, nothing is left of a row but what its
// probabilities have lost: with two numbers 2.7e-6 of sum p |v|, five times what products of fp32 may be off.  Both sides, two and three: up to 32 rows the same time (16
// sequences of 4K to 16K slots 117 / 115 us, 32 rows 124 / 120), 64 rows 132 / 135, 128 rows 159 / 176, two sequences of 150K slots 578 / 664.
// The numbers are taken apart again as the pairs that they are packed in (else each is rounded twice, once on its own).
__device__ inline void three_numbers(const floatx8 &x, bf16x8 &first, bf16x8 &rest, bf16x8 &last)
{
    uint32_t a[4], b[4], c[4];
    const auto less = [](floatx2 y, uint32_t pair) __attribute__((always_inline)) {
        return (floatx2){y[0] - __builtin_bit_cast(float, pair << 16), y[1] - __builtin_bit_cast(float, pair & 0xffff0000u)};
    };
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const floatx2 y = {x[2 * w], x[2 * w + 1]};
        a[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
        const floatx2 left = less(y, a[w]);
        b[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector(left, bf16x2));
        c[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector(less(left, b[w]), bf16x2));
    }
    first = __builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3]));
    rest = __builtin_bit_cast(bf16x8, make_uint4(b[0], b[1], b[2], b[3]));
    last = __builtin_bit_cast(bf16x8, make_uint4(c[0], c[1], c[2], c[3]));
}

// A sequence: slots in use, its drafted tokens; what is visible of it, from block `first` on; units: of an item, with its beginning; items of it, rows of an item.
struct Seq { int base, token, T, n, begin, first, blocks, units, groups, items, rows; };

template <typename L, typename LOAD>
__device__ inline Seq seq_of(const TreeArgs &a, int s, LOAD load)
{
    Seq v;
    const int cap = a.cache.max_pages * a.cache.page_size;
    v.base = max(0, min(load(a.lens + s), cap));
    v.token = max(0, min(load(a.first + s), a.n_tokens));
    v.T = min(max(v.token, min(load(a.first + s + 1), a.n_tokens)) - v.token, a.max_tokens);
    v.n = min(v.base + v.T, cap);
    v.begin = a.window > 0 ? max(0, v.base - a.window) : 0;
    v.first = v.begin / L::kKeys;
    v.blocks = (v.n + L::kKeys - 1) / L::kKeys - v.first;
    v.groups = (v.T * a.G + L::kRows - 1) / L::kRows;
    v.items = v.groups * a.cache.n_kv_heads;
    // groups of like size, in whole waves: a share is as long for few rows as for many (39.5K slots, 182 rows: 49.6 -> 48.6 us; 8 sequences of 4K to
    // 16K slots, 140 rows: 79 -> 78)
    v.rows = L::kRows;
    if (L::kEven > 0 && v.groups > 1) v.rows = ((v.T * a.G + v.groups - 1) / v.groups + L::kEven - 1) / L::kEven * L::kEven;
    v.units = v.T > 0 ? v.blocks + L::kItem : 0;
    return v;
}
// Row R of a sequence and KV head is token R / G.  (R + 1/2) / G is at least 1 / (2 G) away from whole numbers, and off by less than that for R below 2^21.
__device__ inline int token_of(const TreeArgs &a, int R) { return (int)(((float)R + 0.5f) * a.inv_g); }

struct ScalarLoad { __device__ int operator()(const int32_t *p) const { return scalar_load<int>(p); } };
struct VectorLoad { __device__ int operator()(const int32_t *p) const { return *p; } };

// The share of this workgroup in the row of all units: items of a sequence one behind the other, sequences one behind the other.
struct Place { int seq, item, unit; };   // sequence, item of it, unit of that
struct Range { int begin, end; Place at; int each; };   // `each`: units of a share

// All threads of the workgroup; units of a share: a multiple of the groups of waves.
template <typename L>
__device__ inline Range own_range(const TreeArgs &a, int share, int n_shares)
{
    constexpr int THREADS = L::kThreads, kWaves = THREADS / 64, WK = L::kTurns;
    __shared__ int wave_sums[kWaves], found[3];
    const int tid = threadIdx.x, S = a.cache.n_seqs;
    Range r;
    int total;
    if (S == 1) {
        const Seq v = seq_of<L>(a, 0, ScalarLoad{});
        total = v.units * v.items;
        r.each = max(WK, ((total + n_shares - 1) / n_shares + WK - 1) / WK * WK);
        r.begin = (int)min((int64_t)total, (int64_t)share * r.each);
        r.end = min(total, r.begin + r.each);
        r.at.seq = 0;
        r.at.item = v.units > 0 ? r.begin / v.units : 0;
        r.at.unit = r.begin - r.at.item * v.units;
        return r;
    }
    // a thread adds up a few sequences one behind the other
    const int each = (S + THREADS - 1) / THREADS, s0 = min(S, tid * each), s1 = min(S, s0 + each);
    int mine = 0;
    for (int s = s0; s < s1; ++s) {
        const Seq v = seq_of<L>(a, s, VectorLoad{});
        mine += v.units * v.items;
    }
    int upto = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int x = __shfl_up(upto, off, 64);
        if ((tid & 63) >= off) upto += x;
    }
    if ((tid & 63) == 63) wave_sums[tid >> 6] = upto;
    __syncthreads();
    total = 0;
    int before = upto - mine;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before += w < (tid >> 6) ? wave_sums[w] : 0;
        total += wave_sums[w];
    }
    r.each = max(WK, ((total + n_shares - 1) / n_shares + WK - 1) / WK * WK);
    r.begin = (int)min((int64_t)total, (int64_t)share * r.each);
    r.end = min(total, r.begin + r.each);
    if (r.begin >= before && r.begin < before + mine) {
        int left = r.begin - before, s = s0;
        Seq v = seq_of<L>(a, s, VectorLoad{});
        while (left >= v.units * v.items) {
            left -= v.units * v.items;
            v = seq_of<L>(a, ++s, VectorLoad{});
        }
        found[0] = s;
        found[1] = left / v.units;
        found[2] = left - left / v.units * v.units;
    }
    __syncthreads();
    r.begin = __builtin_amdgcn_readfirstlane(r.begin);
    r.end = __builtin_amdgcn_readfirstlane(r.end);
    r.each = __builtin_amdgcn_readfirstlane(r.each);
    if (r.begin < r.end) {
        r.at.seq = __builtin_amdgcn_readfirstlane(found[0]);
        r.at.item = __builtin_amdgcn_readfirstlane(found[1]);
        r.at.unit = __builtin_amdgcn_readfirstlane(found[2]);
    }
    return r;
}

// tanh, in place, of scores times to_cap.  Below 1/2 an odd polynomial with the least largest relative error there (1.5e-8); capped scores are that small as a rule, so it
// is tried alone.  From 1/2 on 1 - 2 / (e + 1), e = exp(2 |x|), whose last difference makes the error of what is taken off 1.2 times as large at most; no e is too
// large for it, and a NaN stays one.  No branch around a single score: with them the scores of a lane wait for each other (48 sequences of up to 80 rows: 143 -> 128 us).
template <typename V, int N>
__device__ inline void tanh_scores(V (&s)[N], float to_cap)
{
    constexpr int E = sizeof(V) / 4;
    float most = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            s[n][e] *= to_cap;
            most = fmaxf(most, fabsf(s[n][e]));
        }
    const auto near = [](float x) __attribute__((always_inline)) {
        const float x2 = x * x;
        return fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 0.01724148f, -0.05304549f), 0.13325879f), -0.33333144f), x);
    };
    if (__all(most < 0.5f)) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < E; ++e) s[n][e] = near(s[n][e]);
        return;
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = s[n][e];
            float small = near(x), large = fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(fabsf(x) * 2.8853900817779268f) + 1.f), 1.f);
            asm volatile("" : "+v"(small), "+v"(large));   // (both, by all lanes)
            s[n][e] = fabsf(x) < 0.5f ? small : copysignf(large, x);
            if (e % 2 == 1) __builtin_amdgcn_sched_barrier(0);   // (a few at a time: else they take too many registers; scores beyond half the cap 153 -> 149 us)
        }
}

// What drafted token t of a sequence sees of the drafted ones, with the window laid on; returns the first slot that it sees.
__device__ inline int token_sees(const TreeArgs &a, const Seq &seq, int t, uint64_t (&words)[BS_TREE_MAX_TOKENS / 64])
{
    int seen = 0;
#pragma unroll
    for (int w = 0; w < BS_TREE_MAX_TOKENS / 64; ++w) {
        uint64_t x = a.mask ? 0 : bits_between(0, t + 1 - 64 * w);
        if (a.mask && w < a.mask_words) x = a.mask[(int64_t)(seq.token + t) * a.mask_words + w];
        words[w] = x;
    }
#pragma unroll
    for (int w = 0; w < BS_TREE_MAX_TOKENS / 64; ++w) {
        words[w] &= bits_between(0, seq.T - 64 * w);
        seen += __popcll(words[w]);
    }
    if (a.window <= 0) return 0;
    int drop = seen - a.window;   // the first ones
#pragma unroll
    for (int w = 0; w < BS_TREE_MAX_TOKENS / 64; ++w) {
        const int n = __popcll(words[w]);
        if (drop >= n) words[w] = 0;
        else for (int i = 0; i < drop; ++i) words[w] &= words[w] - 1;
        drop -= n;
    }
    return max(0, seq.base - max(0, a.window - seen));
}

// The same of the rows of an item, [8 words][ROWS] and [ROWS], into LDS.  Threads tid of THREADS.
template <int ROWS, int THREADS>
__device__ inline void rows_see(const TreeArgs &a, const Seq &seq, int row0, int n_rows, uint32_t *masks, int *begins, int tid)
{
    for (int r = tid; r < ROWS; r += THREADS) {
        uint64_t words[BS_TREE_MAX_TOKENS / 64];
        begins[r] = token_sees(a, seq, token_of(a, row0 + min(r, n_rows - 1)), words);
#pragma unroll
        for (int w = 0; w < 8; ++w) masks[w * ROWS + r] = (uint32_t)(words[w / 2] >> (32 * (w % 2)));
    }
}

// 32 slots from n0 on that a row sees; word(w): 32 drafted tokens; begin: first slot seen.
template <typename W>
__device__ inline uint32_t row_sees(int n0, int base, int begin, W word)
{
    const int rel = n0 - base;   // drafted token of the first slot
    uint32_t x;
    if (rel >= 0) {
        const int w = min(rel >> 5, 8);
        x = __builtin_amdgcn_alignbit(w < 7 ? word(w + 1) : 0u, w < 8 ? word(w) : 0u, rel & 31);
    } else {
        x = rel > -32 ? (word(0) << (-rel & 31)) | ~(~0u << (-rel & 31)) : ~0u;
    }
    const int before = begin - n0;   // slots that lie before the row's window
    if (before > 0) x &= before < 32 ? ~0u << before : 0u;
    return x;
}

template <typename T, int D, int NRB, int WR, int WK>
__global__ __launch_bounds__(64 * WR * WK, (Layout<T, D, NRB, WR, WK>::kPerCu * WR * WK + 3) / 4) void tree_shares(const TreeArgs a)
{
    using TR = Layout<T, D, NRB, WR, WK>;
    constexpr bool BF16 = sizeof(T) == 2, SHARED = WR > 1;
    static_assert(!(BF16 && SHARED), "bf16 waves that share their blocks are those of tree_wide");
    constexpr int KEYS = TR::kKeys, ROWB = TR::kRowBytes, BLK = TR::kBlock, NI = TR::kLoads, NI16 = TR::kLoads16, SUB = KEYS / 16, OWN = TR::kOwn;
    constexpr int ROWS = TR::kRows, NB = D / 16, CH4 = D / 4, WAVES = TR::kWaves, THREADS = TR::kThreads, KSTEPS = D * (int)sizeof(T) / 64;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wk = wave / WR, wr = wave % WR;
    const int P = a.cache.page_size, cap = a.cache.max_pages * P;

    // items that a sequence could have and has not: nothing to join
    if (a.by_item)
        for (int s = blockIdx.x; s < a.cache.n_seqs; s += gridDim.x)
            for (int i = seq_of<TR>(a, s, ScalarLoad{}).items + tid; i < a.most_items; i += THREADS) a.cuts[s * a.most_items + i] = Cut{};

    const Range range = own_range<TR>(a, blockIdx.x, gridDim.x);
    if (tid == 0 && !a.by_item) a.cuts[blockIdx.x] = Cut{};
    if (range.begin >= range.end) return;

    typedef __attribute__((address_space(3))) void *lds_ptr;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr)lds, ring = lds0 + wk * TR::kGroup;
    // LDS-direct loads: instruction j of 16 slots moves 1 KB, i.e. 1024 / ROWB whole rows; a lane picks the chunk of its row that belongs at
    // its place.  The waves that share a block take every WR-th of its instructions.
    uint32_t voff[OWN];
#pragma unroll
    for (int x = 0; x < OWN; ++x) {
        const int j = (x * WR + wr) % NI16, r = j * (1024 / ROWB) + lane / (ROWB / 16), p = lane % (ROWB / 16);
        voff[x] = r * (uint32_t)(a.cache.slot_stride * sizeof(T)) + ((p ^ TR::swizzle(r)) << 4);
    }
    const auto load_lds = [](uint32_t off, const char *src, uint32_t dst) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(src), "s"(dst) : "memory", "m0");
    };
    const auto wait_loads = [](auto newer) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(newer)::value) : "memory");
    };
    const auto reads_done = []() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
    const auto meet = []() __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    const uint32_t k_read = wk * TR::kGroup + col * ROWB + ((grp ^ TR::swizzle(col)) << 4);
    uint32_t v_read[BF16 ? 2 : 4];   // bf16: of the two halves of a block; fp32: of the four slots of a lane
    if constexpr (BF16) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 16 * h + 4 * grp + (col >> 2);
            v_read[h] = wk * TR::kGroup + BLK + r * ROWB + ((((col >> 1) & 1) ^ TR::swizzle(r)) << 4) + (col & 1) * 8;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * grp + i;
            v_read[i] = wk * TR::kGroup + BLK + r * ROWB + ((col ^ TR::swizzle(r)) << 4);
        }
    }

    Place at = range.at;
    int pos = range.begin;
    Seq seq = seq_of<TR>(a, at.seq, ScalarLoad{});
    while (pos < range.end) {
        while (at.item == seq.items) {   // the next sequence that has some
            at.item = 0;
            seq = seq_of<TR>(a, ++at.seq, ScalarLoad{});
        }
        const int block = max(0, at.unit - TR::kItem);   // the first one
        const int blocks = min(seq.blocks - block, range.end - pos - max(0, TR::kItem - at.unit));
        if (blocks <= 0) break;   // the share ends where the item begins
        const int kvh = at.item / seq.groups, row0 = (at.item - kvh * seq.groups) * ROWS;   // rows: token by token, the group's heads of each
        const int n_rows = min(ROWS, seq.T * a.G - row0);
        // Waves that share their blocks step together, and one group may have none in the last step.
        const int n_steps = SHARED ? (blocks + WK - 1) / WK : (blocks > wk ? (blocks - wk + WK - 1) / WK : 0);
        const int b0 = seq.first + block + wk;   // step i: block b0 + WK i of the sequence

        // Page numbers of 16 slots each; which slots of a block have a page.
        const int32_t *table = a.cache.page_table + (int64_t)at.seq * a.cache.max_pages;
        struct Pages { int32_t page[SUB]; uint32_t in_page[SUB]; };
        const auto pages_of = [&](int i) __attribute__((always_inline)) {
            Pages p;
#pragma unroll
            for (int h = 0; h < SUB; ++h) {
                // (behind the last slots: those again)
                const uint32_t slot = min((b0 + WK * min(i, n_steps - 1)) * KEYS + 16 * h, cap - 16);
                const uint32_t page = slot / (uint32_t)P;
                p.page[h] = scalar_load<int>(table + page);
                p.in_page[h] = slot - page * P;
            }
            return p;
        };
        struct Sources { const char *k[SUB], *v[SUB]; uint32_t there; };
        const auto sources_of = [&](const Pages &p) __attribute__((always_inline)) {
            Sources s;
            s.there = 0;
#pragma unroll
            for (int h = 0; h < SUB; ++h) {
                const bool ok = (uint32_t)p.page[h] < (uint32_t)a.cache.n_pages;
                const int64_t off = ((ok ? p.page[h] : 0) * a.cache.page_stride + kvh * a.cache.head_stride + p.in_page[h] * a.cache.slot_stride) * (int64_t)sizeof(T);
                s.k[h] = static_cast<const char *>(a.cache.k) + off;
                s.v[h] = static_cast<const char *>(a.cache.v) + off;
                s.there |= ok ? 0xffffu << (16 * h) : 0u;
            }
            return s;
        };
        const auto issue = [&](const char *const(&src)[SUB], uint32_t dst) __attribute__((always_inline)) {
#pragma unroll
            for (int x = 0; x < OWN; ++x) {
                const int j = x * WR + wr;
                if (NI % WR == 0 || j < NI) load_lds(voff[x], src[SUB == 1 || j < NI16 ? 0 : SUB - 1], dst + j * 1024);
            }
        };

        // The query rows (all waves together) in the layout of a K block, then the first blocks of keys and values.  A place without a row holds a copy of the last
        // one, whose results are not stored.
        {
            const char *qh = reinterpret_cast<const char *>(static_cast<const T *>(a.q) + seq.token * a.q_token + (int64_t)kvh * a.G * a.q_head);
            constexpr int kAll = ROWS * ROWB / 1024;
#pragma unroll
            for (int i0 = 0; i0 < kAll; i0 += WAVES) {
                const int i = i0 + wave;
                if (kAll % WAVES == 0 || i < kAll) {
                    const int r = i * (1024 / ROWB) + lane / (ROWB / 16), p = lane % (ROWB / 16);
                    const int R = row0 + min(r, n_rows - 1), t = token_of(a, R);
                    load_lds((uint32_t)((t * a.q_token + (R - t * a.G) * a.q_head) * (int64_t)sizeof(T)) + ((p ^ TR::swizzle(r)) << 4), qh, lds0 + TR::kQuery + i * 1024);
                }
            }
        }
        Sources s0{}, s1{};
        Pages next{};
        if (n_steps > 0) {
            const Pages p0 = pages_of(0), p1 = pages_of(1);
            next = pages_of(2);
            s0 = sources_of(p0);
            issue(s0.k, ring);
            issue(s0.v, ring + BLK);
            s1 = sources_of(p1);
            if (!SHARED && n_steps > 1) {
                issue(s1.k, ring + 2 * BLK);
                issue(s1.v, ring + 3 * BLK);
            }
        }
        if (!SHARED && n_steps > 1) wait_loads(std::integral_constant<int, 4 * NI>{});
        else if (!SHARED && n_steps == 1) wait_loads(std::integral_constant<int, 2 * NI>{});
        else wait_loads(std::integral_constant<int, 0>{});
        reads_done();
        meet();
        uint4 q[NRB][KSTEPS];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
            for (int t = 0; t < KSTEPS; ++t)
                q[rb][t] = *reinterpret_cast<const uint4 *>(lds + TR::kQuery + (wr * NRB + rb) * 16 * ROWB + ((col * ROWB + ((grp ^ TR::swizzle(col)) << 4)) ^ (t << 6)));

        floatx4 o[NRB][NB];
        float m_run[NRB], l_run[NRB];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            m_run[rb] = -INFINITY;
            l_run[rb] = 0.f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[rb][nb][i] = 0.f;
        }
        const float c = a.cap_log2e > 0.f ? a.cap_log2e : a.scale_log2e;
        // Slots below this one, if their pages are there, are seen by all rows, but for those before the window's last begin.
        const int window_end = a.window > 0 ? min(seq.base, seq.base - a.window + seq.T) : 0;

        uint32_t there0 = s0.there, there1 = s1.there;   // of this block, of the next one
        int stage = 0;                                   // offset of this block's stage
        for (int i = 0; i < n_steps; ++i) {
            const bool more = i + 1 < n_steps, more2 = i + 2 < n_steps;
            const int n0 = (b0 + WK * i) * KEYS;
            Sources s2{};
            if (SHARED) {
                wait_loads(std::integral_constant<int, 0>{});
                meet();   // all of the block is there, and the stage of the block before is free
                if (more) {
                    issue(s1.k, ring + (stage ^ 2 * BLK));
                    issue(s1.v, ring + (stage ^ 2 * BLK) + BLK);
                }
                if (more2) s1 = s2 = sources_of(next);
            } else if (more2) {
                s2 = sources_of(next);
            }
            next = pages_of(i + 3);

            // ---- S^T = K Q^T: lane: slots 16 h + 4 grp + e of query row `col` of each row block
            if constexpr (!SHARED) {
                if (!more) wait_loads(std::integral_constant<int, NI>{});
                else wait_loads(std::integral_constant<int, 3 * NI>{});
            }
            floatx4 s[NRB][SUB];
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                for (int h = 0; h < SUB; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[rb][h][e] = 0.f;
#pragma unroll
            for (int t = 0; t < KSTEPS; ++t)
#pragma unroll
                for (int h = 0; h < SUB; ++h) {
                    const uint4 f = *reinterpret_cast<const uint4 *>(lds + ((k_read + stage) ^ (t << 6)) + h * 16 * ROWB);
#pragma unroll
                    for (int rb = 0; rb < NRB; ++rb) {
                        if constexpr (BF16) {
                            s[rb][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, q[rb][t]), s[rb][h], 0, 0, 0);
                        } else {
                            const floatx4 x = __builtin_bit_cast(floatx4, f), y = __builtin_bit_cast(floatx4, q[rb][t]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[rb][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], s[rb][h], 0, 0, 0);
                        }
                    }
                }
            if constexpr (!SHARED) {
                reads_done();
                if (more2) issue(s2.k, ring + stage);
            }
            if (a.cap_log2e > 0.f) {
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb) tanh_scores(s[rb], a.to_cap);
            }

            // ---- which of the lane's slots its rows see (4 bits per 16 slots)
            uint32_t exists = there0;   // slots that may be looked at
            if (n0 < seq.begin) exists &= ~0u << min(31, seq.begin - n0);   // (a block has a visible slot: seq.begin - n0 < KEYS)
            if (n0 + KEYS > seq.n) exists &= n0 < seq.n ? ~(~0u << (seq.n - n0)) : 0u;
            if (SHARED && block + wk + WK * i >= block + blocks) exists = 0;   // the group has no block in this step
            const bool masked = n0 + KEYS > seq.base || n0 < window_end || exists != (KEYS == 32 ? ~0u : 0xffffu);
            uint32_t seen[NRB];
            if (masked) {
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb) {
                    // (one or two blocks of an item: loaded when it comes to them, not when the item begins and its first keys are under way)
                    uint32_t x = ~0u;
                    if (n0 + KEYS > seq.base || n0 < window_end) {
                        uint64_t words[BS_TREE_MAX_TOKENS / 64];
                        const int begin = token_sees(a, seq, token_of(a, row0 + min((wr * NRB + rb) * 16 + col, n_rows - 1)), words);
                        x = row_sees(n0, seq.base, begin, [&](int w) __attribute__((always_inline)) {
                            const uint64_t y = w < 2 ? words[0] : w < 4 ? words[1] : w < 6 ? words[2] : words[3];
                            return (uint32_t)(w & 1 ? y >> 32 : y);
                        });
                    }
                    seen[rb] = (x & exists) >> (4 * grp);
#pragma unroll
                    for (int h = 0; h < SUB; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[rb][h][e] = (seen[rb] & (1u << (16 * h + e))) ? s[rb][h][e] : -INFINITY;
                }
            }

            // ---- the running maximum and sum
            float p[NRB][SUB][4];
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                float mx = -INFINITY;
#pragma unroll
                for (int h = 0; h < SUB; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[rb][h][e]);
                mx = max_across_groups(mx);
                // the reference point moves only when the block's maximum exceeds it by 2^8 (any reference gives the same quotient),
                // so the accumulators are rescaled a few times per row and not once per block
                const bool grow = fmaf(mx, c, -(m_run[rb] * c)) > 8.f;
                const float m_new = grow ? mx : m_run[rb];
                const float off = m_new == -INFINITY ? 0.f : -(m_new * c);   // no slot so far: p = 0
                const float alpha = grow ? __builtin_amdgcn_exp2f(fmaf(m_run[rb], c, off)) : 1.f;
                float sum = 0.f;
#pragma unroll
                for (int h = 0; h < SUB; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[rb][h][e] = __builtin_amdgcn_exp2f(fmaf(s[rb][h][e], c, off));
                        sum += p[rb][h][e];
                    }
                l_run[rb] = fmaf(l_run[rb], alpha, sum);
                m_run[rb] = m_new;
                if (__any(alpha != 1.f)) {
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[rb][nb][e] *= alpha;
                }
            }

            // ---- O^T += V^T P^T
            if constexpr (!SHARED) {
                if (more2) wait_loads(std::integral_constant<int, 3 * NI>{});
                else if (more) wait_loads(std::integral_constant<int, 2 * NI>{});
                else wait_loads(std::integral_constant<int, 0>{});
            }
            typedef __attribute__((address_space(3))) bf16x4 *lds_bf16x4;
            const auto read_v = [&](int nb) __attribute__((always_inline)) {   // bf16: channel 16 nb + col, slots 4 grp .. + 3 of both halves
                uint4 f;
                const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + ((v_read[0] + stage) ^ (nb << 5)))));
                const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + ((v_read[BF16 ? 1 : 0] + stage) ^ (nb << 5)))));
                f.x = x.x; f.y = x.y; f.z = y.x; f.w = y.y;
                return f;
            };
            // Values that no row of the call may look at, and any infinity or NaN in a masked block, are replaced by zero: times a probability of zero they would be
            // a NaN.  Rows that do see such a value get one through their sum.
            const uint32_t mine = exists >> (4 * grp);
            uint32_t bad = 0;   // of the lane's slots: a value that is not finite
            if (masked) {
                uint32_t most[4] = {0, 0, 0, 0};   // bf16: two slots in each; fp32: one
                if constexpr (BF16) {
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        const uint4 f = read_v(nb);
                        const uint32_t x[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            if ((x[w] & 0x7f80u) == 0x7f80u) most[w] |= 1u;
                            if ((x[w] & 0x7f800000u) == 0x7f800000u) most[w] |= 2u;
                        }
                    }
#pragma unroll
                    for (int w = 0; w < 4; ++w) bad |= most[w] << (16 * (w / 2) + 2 * (w % 2));
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int n = 0; n < D / 64; ++n) {
                            const uint4 f = *reinterpret_cast<const uint4 *>(lds + v_read[BF16 ? 0 : e] + stage + n * 256);
                            const uint32_t x[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                            for (int w = 0; w < 4; ++w)
                                if ((x[w] & 0x7f800000u) == 0x7f800000u) bad |= 1u << e;
                        }
                }
#pragma unroll
                for (int off = 1; off < 16; off <<= 1) bad |= __shfl_xor(bad, off, 64);   // all channels: the lanes of the same slots
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb)
                    if (seen[rb] & bad) l_run[rb] = __builtin_nanf("");
            }
            const uint32_t fine = mine & ~bad;   // (a slot with a value that is not finite: all of its values)
            if constexpr (BF16) {
                // Probabilities in three bf16 numbers each: where values cancel, nothing is left but what a probability has lost.
                bf16x8 pb[NRB], rest[NRB], last[NRB];
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb) {
                    floatx8 x;
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = p[rb][e >> 2][e & 3];
                    three_numbers(x, pb[rb], rest[rb], last[rb]);
                }
                uint32_t keep[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int at = 16 * (w / 2) + 2 * (w % 2);
                    keep[w] = ((fine >> at) & 1 ? 0xffffu : 0u) | ((fine >> (at + 1)) & 1 ? 0xffff0000u : 0u);
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    uint4 f = read_v(nb);
                    f.x &= keep[0]; f.y &= keep[1]; f.z &= keep[2]; f.w &= keep[3];
#pragma unroll
                    for (int rb = 0; rb < NRB; ++rb) {
                        o[rb][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), pb[rb], o[rb][nb], 0, 0, 0);
                        o[rb][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), rest[rb], o[rb][nb], 0, 0, 0);
                        o[rb][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), last[rb], o[rb][nb], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)   // slot 4 grp + e
#pragma unroll
                    for (int n = 0; n < D / 64; ++n) {
                        floatx4 x = *reinterpret_cast<const floatx4 *>(lds + v_read[BF16 ? 0 : e] + stage + n * 256);
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            x[w] = (fine & (1u << e)) ? x[w] : 0.f;
#pragma unroll
                            for (int rb = 0; rb < NRB; ++rb) o[rb][4 * n + w] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[w], p[rb][0][e], o[rb][4 * n + w], 0, 0, 0);
                        }
                    }
            }
            reads_done();
            if constexpr (!SHARED) {
                if (more2) issue(s2.v, ring + stage + BLK);
            }
            there0 = there1;
            there1 = s2.there;
            stage ^= 2 * BLK;
        }

        // ---- the groups' results over the rings; [row][chunks of 4 channels, exchanged]
        if constexpr (SHARED) meet();   // all waves have read their last block
        float2 *ml = reinterpret_cast<float2 *>(lds + TR::kMl);   // [group][row]
        float4 *merge = reinterpret_cast<float4 *>(lds);
        constexpr int kMergeGroup = TR::kMerge / 16;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            const int row = (wr * NRB + rb) * 16 + col;
            const float l = sum_across_groups(l_run[rb]);
            if (grp == 0) ml[wk * ROWS + row] = make_float2(m_run[rb], l);
            if (row < n_rows) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if constexpr (BF16) {   // channels 16 nb + 4 grp + i
                        merge[wk * kMergeGroup + row * CH4 + ((nb * 4 + grp) ^ (row & (CH4 - 1)))] = make_float4(o[rb][nb][0], o[rb][nb][1], o[rb][nb][2], o[rb][nb][3]);
                    } else {                // channel 64 n + 16 grp + 4 i + w of o[4 n + w][i]: here nb = 4 n + i
                        const int n = nb / 4, i = nb % 4;
                        merge[wk * kMergeGroup + row * CH4 + ((16 * n + 4 * grp + i) ^ (row & (CH4 - 1)))] =
                            make_float4(o[rb][4 * n][i], o[rb][4 * n + 1][i], o[rb][4 * n + 2][i], o[rb][4 * n + 3][i]);
                    }
                }
            }
        }
        __syncthreads();
        const bool begins = block == 0, ends = block + blocks == seq.blocks;
        const int64_t part = (int64_t)(2 * blockIdx.x + (begins ? 1 : 0)) * ROWS;
        for (int idx = tid; idx < n_rows * CH4; idx += THREADS) {
            const int row = idx / CH4, ch = idx % CH4;
            float2 x[WK];
            float4 y[WK];
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                x[w] = ml[w * ROWS + row];
                y[w] = merge[w * kMergeGroup + row * CH4 + (ch ^ (row & (CH4 - 1)))];
                m = fmaxf(m, x[w].x);
            }
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float f = x[w].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x[w].x - m) * c);
                l = fmaf(x[w].y, f, l);
                sum.x = fmaf(y[w].x, f, sum.x); sum.y = fmaf(y[w].y, f, sum.y); sum.z = fmaf(y[w].z, f, sum.z); sum.w = fmaf(y[w].w, f, sum.w);
            }
            if (begins && ends) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const int R = row0 + row, t = token_of(a, R);
                store_row4(static_cast<T *>(a.out) + (seq.token + t) * a.out_token + (int64_t)(kvh * a.G + R - t * a.G) * a.out_head + 4 * ch,
                           make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
            } else {
                *reinterpret_cast<float4 *>(a.part_o + (part + row) * D + 4 * ch) = sum;
                if (ch == 0) a.part_ml[part + row] = make_float2(m, l);
            }
        }
        if (begins && tid == 0 && (a.by_item || !ends))
            a.cuts[a.by_item ? at.seq * a.most_items + at.item : (int)blockIdx.x] = Cut{(int)blockIdx.x, (pos - at.unit + seq.units - 1) / range.each, kvh, row0, ends ? 0 : n_rows, seq.token, {}};
        pos += seq.units - at.unit;   // (behind the share's end if the item is cut)
        at.unit = 0;
        ++at.item;
        if (pos < range.end) __syncthreads();   // the LDS is free again
    }
}

// Many rows (bf16): four waves of 32 rows each walk the same blocks of 32 slots in step; two such workgroups share a CU, so that one has scores and probabilities
// to make while the other waits for its waves.  Two waves load K and two load V, each three or more blocks ahead.  CAP: scores are capped (a kernel of its own: the
// registers that a cap takes cost calls without one 3 %).
template <int D>
struct Wide {
    static constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 32 * kWaves, kKeys = 32, kTurns = 1, kPerCu = 2;
    static constexpr int kEven = 32;                          // rows of a wave
    static constexpr int kItem = 4;                           // (see Layout; 48 sequences of up to 80 rows with 2, 3, 4, 5, 6, 8: 151, 133, 127, 128, 128, 129 us; 16 of 40 rows at
                                                              // d 64: 93, 93, 93, 92, 92, 92)
    static constexpr int kRowBytes = 2 * D, kBlock = kKeys * kRowBytes;                        // a block of K or V
    static constexpr int kLoads16 = 16 * kRowBytes / 1024;    // LDS-direct instructions per 16 slots, which lie in one page
    static constexpr int kSlots = D == 64 ? 8 : 4;            // blocks of K, of V, that the LDS holds
    static constexpr int kValues = kSlots * kBlock;           // V's ring behind K's; at first the query rows, until they are in registers
    static constexpr int kMerge = kRows * D * 4;              // results lie over the rings
    static constexpr int kEnd = 2 * kValues > kMerge ? 2 * kValues : kMerge;
    static constexpr int kMask = kEnd, kBegin = kMask + 8 * kRows * 4, kMl = kBegin + kRows * 4;
    static constexpr int kThere = kMl + kRows * 8;            // [ring][2]: 16 slots have a page
    static constexpr int kBad = kThere + kSlots * 8;          // [ring]: slots with a value that is not finite
    static constexpr int kLds = kBad + kSlots * 4;
    static_assert((kLds + 1024) * kPerCu <= 160 * 1024, "LDS of a CU");
    static_assert(kRows * kRowBytes <= kValues, "query rows");
    // exchange of the 16-byte chunks of row r: rows that share their banks get different chunks.  K is read 16 rows of a chunk at a time, V four rows of four chunks.
    __device__ static int swizzle(int r) { return kRowBytes == 128 ? (r >> 1) & 7 : r & 15; }
    __device__ static int swizzle_v(int r) { return kRowBytes == 128 ? (r & 2) << 1 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3); }
};

template <int D, bool CAP>
__global__ __launch_bounds__(256, 2) void tree_wide(const TreeArgs a)
{
    using TR = Wide<D>;
    constexpr int KEYS = TR::kKeys, ROWB = TR::kRowBytes, BLK = TR::kBlock, NI16 = TR::kLoads16, ROWS = TR::kRows, THREADS = TR::kThreads, RING = TR::kSlots;
    constexpr int KSTEPS = D / 16, CB = D / 32, CH4 = D / 4;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, n31 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int P16 = a.cache.page_size / 16;
    const int64_t page_bytes = a.cache.page_stride * 2, slots16_bytes = a.cache.slot_stride * 32;

    if (a.by_item)   // items that a sequence could have and has not: nothing to join
        for (int s = blockIdx.x; s < a.cache.n_seqs; s += gridDim.x)
            for (int i = seq_of<TR>(a, s, ScalarLoad{}).items + tid; i < a.most_items; i += THREADS) a.cuts[s * a.most_items + i] = Cut{};
    const Range range = own_range<TR>(a, blockIdx.x, gridDim.x);
    if (tid == 0 && !a.by_item) a.cuts[blockIdx.x] = Cut{};
    if (range.begin >= range.end) return;

    typedef __attribute__((address_space(3))) void *lds_ptr;
    typedef __attribute__((address_space(3))) bf16x4 *lds_bf16x4;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr)lds;
    // What the wave loads of a block: 16 of its slots, K or V
    const int sub = wave & 1;
    const bool values = wave & 2;
    const char *pool = static_cast<const char *>(values ? a.cache.v : a.cache.k);
    const uint32_t to0 = lds0 + (values ? TR::kValues : 0) + sub * 16 * ROWB;
    uint32_t voff[NI16];   // as in tree_shares
#pragma unroll
    for (int x = 0; x < NI16; ++x) {
        const int r = x * (1024 / ROWB) + lane / (ROWB / 16), p = lane % (ROWB / 16);
        voff[x] = r * (uint32_t)(a.cache.slot_stride * 2) + ((p ^ (values ? TR::swizzle_v(r) : TR::swizzle(r))) << 4);
    }
    const auto load_lds = [](uint32_t off, const char *src, uint32_t dst) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(src), "s"(dst) : "memory", "m0");
    };
    const auto wait_loads = [](auto newer) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(newer)::value) : "memory");
    };
    const auto meet = []() __attribute__((always_inline)) {   // what the wave reads and writes in LDS is done
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // K^T Q: a lane reads key n31, channels 8 half .. + 7 of 16; V^T P: four keys of a channel, lanes of a sixteen the channels, keys 4 half .. + 3 and 8 behind them
    const uint32_t k_read = n31 * ROWB + ((half ^ TR::swizzle(n31)) << 4);
    uint32_t v_read[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int r = 8 * x + 4 * half + ((lane & 15) >> 2);
        v_read[x] = TR::kValues + r * ROWB + (((2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ TR::swizzle_v(r)) << 4) + (lane & 1) * 8;
    }
    const uint32_t *row_mask = reinterpret_cast<const uint32_t *>(lds + TR::kMask);
    const int *row_begin = reinterpret_cast<const int *>(lds + TR::kBegin);
    uint32_t *flags = reinterpret_cast<uint32_t *>(lds + TR::kThere), *bad = reinterpret_cast<uint32_t *>(lds + TR::kBad);
    const float c = CAP ? a.cap_log2e : a.scale_log2e;

    Place at = range.at;
    int pos = range.begin;
    Seq seq = seq_of<TR>(a, at.seq, ScalarLoad{});
    while (pos < range.end) {
        while (at.item == seq.items) {   // the next sequence that has some
            at.item = 0;
            seq = seq_of<TR>(a, ++at.seq, ScalarLoad{});
        }
        const int block = max(0, at.unit - TR::kItem);   // the first one
        const int n_steps = min(seq.blocks - block, range.end - pos - max(0, TR::kItem - at.unit));
        if (n_steps <= 0) break;   // the share ends where the item begins
        const int kvh = at.item / seq.groups, row0 = (at.item - kvh * seq.groups) * seq.rows;   // rows: token by token, the group's heads of each
        const int n_rows = min(seq.rows, seq.T * a.G - row0);
        const int b0 = seq.first + block;

        // The wave's 16 slots of the next blocks that it requests (a page holds P16 such), and the place in the ring that they go to
        const int32_t *table = a.cache.page_table + (int64_t)at.seq * a.cache.max_pages;
        const char *head = pool + (int64_t)kvh * a.cache.head_stride * 2;
        int page = (b0 * 2 + sub) / P16, in16 = b0 * 2 + sub - page * P16, to = 0;
        const auto page_number = [&]() __attribute__((always_inline)) { return page < a.cache.max_pages ? scalar_load<int>(table + page) : -1; };
        const auto go_on = [&]() __attribute__((always_inline)) {
            in16 += 2;
            const int on = in16 < P16 ? 0 : P16 == 1 ? 2 : 1;   // pages
            in16 -= on * P16;
            page += on;
        };
        const auto issue = [&](int number, int in16) __attribute__((always_inline)) {
            const bool ok = (uint32_t)number < (uint32_t)a.cache.n_pages;
            const char *src = head + (ok ? number : 0) * page_bytes + in16 * slots16_bytes;
#pragma unroll
            for (int x = 0; x < NI16; ++x) load_lds(voff[x], src, to0 + to * BLK + x * 1024);
            if (lane == 0) (values ? bad : flags)[values ? to : to * 2 + sub] = ok && !values ? 0xffffu : 0u;
            to = to + 1 == RING ? 0 : to + 1;
        };
        int next_page = 0;   // of the block to be requested next
        const auto issue_first = [&](int n) __attribute__((always_inline)) {   // up to RING - 1 or RING blocks: their page numbers come together
            int number[RING], at16[RING];
#pragma unroll
            for (int r = 0; r < RING; ++r) {
                number[r] = r < n ? page_number() : 0;
                at16[r] = in16;
                if (r < n) go_on();
            }
            next_page = page_number();
#pragma unroll
            for (int r = 0; r < RING; ++r)
                if (r < n) issue(number[r], at16[r]);
        };

        // Two waves request the first keys, the others the query rows, in the layout of a K block and where values go later, and find what they see.  A place without
        // a row holds a copy of the last one.
        if (!values) {
            issue_first(min(RING, n_steps));
            if (n_steps < RING) wait_loads(std::integral_constant<int, 0>{});
            else wait_loads(std::integral_constant<int, (RING - 1) * NI16>{});
        } else {
            const char *qh = reinterpret_cast<const char *>(static_cast<const __bf16 *>(a.q) + seq.token * a.q_token + (int64_t)kvh * a.G * a.q_head);
            constexpr int kAll = ROWS * ROWB / 1024;
            int l = lane;
            asm volatile("" : "+v"(l));   // (else what depends on the lane alone is kept in registers over all items)
#pragma unroll
            for (int i0 = 0; i0 < kAll; i0 += 2) {
                const int i = i0 + sub, r = i * (1024 / ROWB) + l / (ROWB / 16), p = l % (ROWB / 16);
                const int R = row0 + min(r, n_rows - 1), t = token_of(a, R);
                load_lds((uint32_t)((t * a.q_token + (R - t * a.G) * a.q_head) * 2) + ((p ^ TR::swizzle(r)) << 4), qh, lds0 + TR::kValues + i * 1024);
            }
            rows_see<ROWS, 128>(a, seq, row0, n_rows, reinterpret_cast<uint32_t *>(lds + TR::kMask), reinterpret_cast<int *>(lds + TR::kBegin), tid - 128);
            wait_loads(std::integral_constant<int, 0>{});
        }
        meet();   // the first block's keys, the query rows and what they see are there
        bf16x8 q[KSTEPS];
#pragma unroll
        for (int t = 0; t < KSTEPS; ++t) q[t] = *reinterpret_cast<const bf16x8 *>(lds + TR::kValues + wave * 32 * ROWB + (k_read ^ (t << 5)));
        meet();   // all query rows are in registers
        if (values) issue_first(min(RING - 1, n_steps));

        floatx16 o[CB], s;
        float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[cb][i] = 0.f;
        // Slots below this one, if their pages are there, are seen by all rows, but for those before the window's last begin.
        const int window_end = a.window > 0 ? min(seq.base, seq.base - a.window + seq.T) : 0;
        const bool works = wave * 32 < n_rows;

        // ---- S^T = K Q^T of the block at `from`: lane: row n31, slots 8 b + 4 half + e in [4 b + e]
        const auto scores = [&](int from) __attribute__((always_inline)) {
            floatx16 x;
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
            for (int t = 0; t < KSTEPS; ++t) {
                const bf16x8 f = *reinterpret_cast<const bf16x8 *>(lds + ((k_read + from * BLK) ^ (t << 5)));
                x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, q[t], x, 0, 0, 0);
            }
            return x;
        };
        // ---- which slots of a block may be looked at, and whether that, or what a row may see, is less than all.  Blocks whole_from .. whole_to - 1 are whole if
        // their pages are there.
        const int whole_from = (max(window_end, seq.begin) + KEYS - 1) / KEYS - b0, whole_to = seq.base / KEYS - b0;
        uint32_t exists = ~0u;
        bool masked = false;
        const auto look = [&](int i, uint2 pages) __attribute__((always_inline)) {
            exists = __builtin_amdgcn_readfirstlane(pages.x | pages.y << 16);
            masked = i < whole_from || i >= whole_to || exists != ~0u;
            if (masked) {
                const int n0 = (b0 + i) * KEYS;
                if (n0 < seq.begin) exists &= ~0u << min(31, seq.begin - n0);   // (a block has a visible slot: seq.begin - n0 < KEYS)
                if (n0 + KEYS > seq.n) exists &= n0 < seq.n ? ~(~0u << (seq.n - n0)) : 0u;
            }
        };
        // ---- the largest score of a lane's slots
        const auto largest = [](const floatx16 &x) __attribute__((always_inline)) {
            float m[5];
#pragma unroll
            for (int e = 0; e < 5; ++e) m[e] = fmaxf(fmaxf(x[3 * e], x[3 * e + 1]), x[3 * e + 2]);
            return fmaxf(fmaxf(fmaxf(fmaxf(m[0], m[1]), m[2]), fmaxf(fmaxf(m[3], m[4]), x[15])), -INFINITY);
        };
        // ---- what the lane's row sees of it, and the row's reference point (see tree_shares); l and O follow it.  mx: of the scores as they come
        uint32_t seen = 0;
        const auto refer = [&](int i, float mx) __attribute__((always_inline)) {
            if constexpr (CAP) {
                floatx16 x[1] = {s};
                tanh_scores(x, a.to_cap);
                s = x[0];
            }
            if (masked) {
                seen = (row_sees((b0 + i) * KEYS, seq.base, row_begin[wave * 32 + n31], [&](int w) { return row_mask[w * ROWS + wave * 32 + n31]; }) & exists) >> (4 * half);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = (seen & (1u << (8 * (e / 4) + e % 4))) ? s[e] : -INFINITY;
            }
            if (CAP || masked) mx = largest(s);
            mx = max_across_halves(mx);
            const bool grow = fmaf(mx, c, -(m_run * c)) > 8.f;
            if (__any(grow)) {
                const float m_new = grow ? mx : m_run;
                const float alpha = grow ? __builtin_amdgcn_exp2f((m_run - m_new) * c) : 1.f;   // (m_new is a number where it grew)
                l_run *= alpha;
                m_run = m_new;
#pragma unroll
                for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[cb][e] *= alpha;
            }
        };

        int from = 0;   // place of this block in the rings
        const uint2 *pages = reinterpret_cast<const uint2 *>(flags);
        look(0, pages[0]);   // (the first keys and their flags are there: all waves have waited for them)
        if (works) {
            s = scores(0);
            refer(0, largest(s));
        }
        for (int i = 0; i < n_steps; ++i) {
            if (i + RING - 1 < n_steps) wait_loads(std::integral_constant<int, (RING - 2) * NI16>{});
            else wait_loads(std::integral_constant<int, 0>{});
            meet();   // the next keys, this block's values are there; this block's keys and the values before are free
            if (i + RING - (values ? 1 : 0) < n_steps) {
                issue(next_page, in16);
                go_on();
                next_page = page_number();
            }
            const int next = from + 1 == RING ? 0 : from + 1;
            const uint2 next_pages = pages[next];
            float next_mx = 0.f;
            // Values in a masked block: those that nobody may look at, and any infinity or NaN, are replaced by zero; times a probability of zero they would be a NaN.
            // Rows that do see such a slot get one through their sum.
            if (masked) {
                for (int x = tid; x < BLK / 16; x += THREADS) {
                    const int r = x / (ROWB / 16);
                    uint4 *v = reinterpret_cast<uint4 *>(lds + TR::kValues + from * BLK) + x;
                    const uint4 y = *v;
                    const uint32_t z[4] = {y.x, y.y, y.z, y.w};
                    bool finite = true;
#pragma unroll
                    for (int w = 0; w < 4; ++w) finite = finite && (z[w] & 0x7f80u) != 0x7f80u && (z[w] & 0x7f800000u) != 0x7f800000u;
                    if (!finite || !(exists >> r & 1)) *v = make_uint4(0, 0, 0, 0);
                    if (!finite && (exists >> r & 1)) atomicOr(bad + from, 1u << r);
                }
                meet();
                if (works && (seen & bad[from] >> (4 * half))) l_run = __builtin_nanf("");
            }
            if (works) {
                const auto read_v = [&](int j, int cb) __attribute__((always_inline)) {   // channel 32 cb + n31, slots 16 j + 4 half .. + 3 and 8 behind them
                    const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + ((v_read[0] + from * BLK) ^ (cb << 6)) + j * 16 * ROWB)));
                    const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + ((v_read[1] + from * BLK) ^ (cb << 6)) + j * 16 * ROWB)));
                    return __builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, y.x, y.y));
                };
                // The next block's scores (behind the last one: of whatever is there) beside this one's probabilities.  The first half of the values is read ahead of
                // them, and the wave goes before those that are at their masks and references: both together 682 -> 647 us (two sequences of 150K slots).
                bf16x8 vf[CB];
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) vf[cb] = read_v(0, cb);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(1);
                const floatx16 s_next = scores(next);
                const float off = m_run == -INFINITY ? 0.f : -(m_run * c);   // no slot so far: p = 0
                float sum[2] = {0.f, 0.f};
                bf16x8 pb[2], rest[2], last[2];   // of 16 slots each, as three numbers (see tree_shares)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    floatx8 x;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[e] = __builtin_amdgcn_exp2f(fmaf(s[8 * j + e], c, off));
                        sum[e & 1] += x[e];
                    }
                    three_numbers(x, pb[j], rest[j], last[j]);
                }
                l_run += sum[0] + sum[1];
                // ---- O^T += V^T P^T
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        const bf16x8 f = j == 0 ? vf[cb] : read_v(j, cb);
                        o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, pb[j], o[cb], 0, 0, 0);
                        o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, rest[j], o[cb], 0, 0, 0);
                        o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, last[j], o[cb], 0, 0, 0);
                    }
                __builtin_amdgcn_s_setprio(0);
                s = s_next;
                next_mx = largest(s);
            }
            if (i + 1 < n_steps) {
                look(i + 1, next_pages);
                if (works) refer(i + 1, next_mx);
            }
            from = next;
        }

        // ---- results over the rings; [row][chunks of 4 channels, exchanged]
        meet();   // all waves have read their last block
        float2 *ml = reinterpret_cast<float2 *>(lds + TR::kMl);
        float4 *merge = reinterpret_cast<float4 *>(lds);
        if (works) {
            const int row = wave * 32 + n31;
            const float l = sum_across_halves(l_run);
            if (half == 0) ml[row] = make_float2(m_run, l);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int b = 0; b < 4; ++b)   // channels 32 cb + 8 b + 4 half + i
                    merge[row * CH4 + ((8 * cb + 2 * b + half) ^ (row & (CH4 - 1)))] = make_float4(o[cb][4 * b], o[cb][4 * b + 1], o[cb][4 * b + 2], o[cb][4 * b + 3]);
        }
        __syncthreads();
        const bool begins = block == 0, ends = block + n_steps == seq.blocks;
        const int64_t into = (int64_t)(2 * blockIdx.x + (begins ? 1 : 0)) * ROWS;
        for (int idx = tid; idx < n_rows * CH4; idx += THREADS) {
            const int row = idx / CH4, ch = idx % CH4;
            const float2 x = ml[row];
            const float4 y = merge[row * CH4 + (ch ^ (row & (CH4 - 1)))];
            if (begins && ends) {
                const float inv = x.y == 0.f ? 0.f : 1.f / x.y;
                const int R = row0 + row, t = token_of(a, R);
                store_row4(static_cast<__bf16 *>(a.out) + (seq.token + t) * a.out_token + (int64_t)(kvh * a.G + R - t * a.G) * a.out_head + 4 * ch,
                           make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv));
            } else {
                *reinterpret_cast<float4 *>(a.part_o + (into + row) * D + 4 * ch) = y;
                if (ch == 0) a.part_ml[into + row] = x;
            }
        }
        if (begins && tid == 0 && (a.by_item || !ends))
            a.cuts[a.by_item ? at.seq * a.most_items + at.item : (int)blockIdx.x] = Cut{(int)blockIdx.x, (pos - at.unit + seq.units - 1) / range.each, kvh, row0, ends ? 0 : n_rows, seq.token, {}};
        pos += seq.units - at.unit;   // (behind the share's end if the item is cut)
        at.unit = 0;
        ++at.item;
        if (pos < range.end) __syncthreads();   // the LDS is free again
    }
}

// Joins the parts of the rows of an item that was cut (blockIdx.x), in a fixed order.  Threads are D / 4 channel quads times the parts of a row side by side, or where
// there are few parts times rows side by side, whichever takes fewer rounds of loads (a batch of 48, two to ten parts: 21 -> 8 us).
template <typename T, int D, typename L>
__global__ __launch_bounds__(256) void tree_join(const TreeArgs a)
{
    constexpr int CH4 = D / 4, LANES = 256 / CH4, M = L::kRows;
    __shared__ float4 acc[LANES][CH4];
    __shared__ float2 ml[LANES];
    const int tid = threadIdx.x, ch = tid % CH4, p0 = tid / CH4;
    const Cut cut = a.cuts[blockIdx.x];
    const float c = a.cap_log2e > 0.f ? a.cap_log2e : a.scale_log2e;
    struct Sum { float m, l; float4 o; };
    // every step-th part of a row: loads of eight go out together, those behind the last one to that one
    const auto parts_of = [&](int row, int from, int step) {
        Sum s{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
        for (int w0 = cut.first + from; w0 <= cut.last; w0 += 8 * step) {
            float2 x[8];
            float4 y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int w = min(w0 + i * step, cut.last);
                const int64_t at = (int64_t)(2 * w + (w == cut.first ? 1 : 0)) * M + row;
                x[i] = a.part_ml[at];
                y[i] = *reinterpret_cast<const float4 *>(a.part_o + at * D + 4 * ch);
            }
            const float m_old = s.m;
#pragma unroll
            for (int i = 0; i < 8; ++i) s.m = fmaxf(s.m, x[i].x);
            const float old = m_old == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_old - s.m) * c);
            s.l *= old;
            s.o.x *= old; s.o.y *= old; s.o.z *= old; s.o.w *= old;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (w0 + i * step > cut.last) continue;
                const float f = x[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x[i].x - s.m) * c);
                s.l = fmaf(x[i].y, f, s.l);
                s.o.x = fmaf(y[i].x, f, s.o.x); s.o.y = fmaf(y[i].y, f, s.o.y); s.o.z = fmaf(y[i].z, f, s.o.z); s.o.w = fmaf(y[i].w, f, s.o.w);
            }
        }
        return s;
    };
    const auto finish = [&](int row, const Sum &s) {
        const float inv = s.l == 0.f ? 0.f : 1.f / s.l;
        const int R = cut.row0 + row, t = token_of(a, R);
        store_row4(static_cast<T *>(a.out) + (cut.token + t) * a.out_token + (int64_t)(cut.kvh * a.G + R - t * a.G) * a.out_head + 4 * ch,
                   make_float4(s.o.x * inv, s.o.y * inv, s.o.z * inv, s.o.w * inv));
    };
    const int n_parts = cut.last - cut.first + 1, y = gridDim.y, side = y * LANES;   // rounds of loads: rows side by side, or parts
    if ((n_parts + 7) / 8 * ((cut.n_rows + side - 1) / side) <= (n_parts + 8 * LANES - 1) / (8 * LANES) * ((cut.n_rows + y - 1) / y)) {
        for (int row = blockIdx.y * LANES + p0; row < cut.n_rows; row += gridDim.y * LANES) finish(row, parts_of(row, 0, 1));
        return;
    }
    for (int row = blockIdx.y; row < cut.n_rows; row += gridDim.y) {
        const Sum s = parts_of(row, p0, LANES);
        acc[p0][ch] = s.o;
        if (ch == 0) ml[p0] = make_float2(s.m, s.l);
        __syncthreads();
        if (tid < CH4) {
            Sum all{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
            for (int i = 0; i < LANES; ++i) all.m = fmaxf(all.m, ml[i].x);
#pragma unroll
            for (int i = 0; i < LANES; ++i) {
                const float g = ml[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[i].x - all.m) * c);
                const float4 y = acc[i][ch];
                all.l = fmaf(ml[i].y, g, all.l);
                all.o.x = fmaf(y.x, g, all.o.x); all.o.y = fmaf(y.y, g, all.o.y); all.o.z = fmaf(y.z, g, all.o.z); all.o.w = fmaf(y.w, g, all.o.w);
            }
            finish(row, all);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------ host

constexpr int kMaxDevices = 64;
std::mutex g_mutex;
int g_n_cus[kMaxDevices];   // compute units of a device, once its kernels' limits are raised

template <typename T, int D, int NRB, int WR, int WK>
struct Narrow {
    typedef Layout<T, D, NRB, WR, WK> layout;
    static constexpr auto kernel = tree_shares<T, D, NRB, WR, WK>;
};
template <int D, bool CAP>
struct Broad {
    typedef Wide<D> layout;
    static constexpr auto kernel = tree_wide<D, CAP>;
};

// The kernel for up to M rows of a sequence and KV head: f(its type).  `cap`: scores are capped.
template <typename T, int D, typename F>
auto with_rows(int32_t M, bool cap, F f)
{
    if constexpr (sizeof(T) == 2) {
        switch (M) {
        case 16: return f(Narrow<T, D, 1, 1, 4>{});
        case 32: return f(Narrow<T, D, 2, 1, 4>{});
        default: return cap ? f(Broad<D, true>{}) : f(Broad<D, false>{});
        }
    } else {   // (more than 128 rows do not fit the LDS)
        switch (M) {
        case 16: return f(Narrow<T, D, 1, 1, 4>{});
        case 32: return f(Narrow<T, D, 2, 1, 4>{});
        default: return f(Narrow<T, D, 2, 4, 2>{});
        }
    }
}

// The M that a sequence's rows per KV head are cut by.  Measured with all of them, in us, 32 query heads on 8; bf16: 16 sequences of 4K to 16K slots, fp32: 4
// of 8K to 16K, over the logarithm:
//              rows    bf16: 16     32     40     64    128  |  fp32: 16     32     64    128
//     d 128, M = 16       113.6  187.9  268.9  353.3  683.9  |      80.7  132.5  244.5  482.0
//            M = 32       119.2  120.0  189.6  193.7  370.1  |      96.2   99.6  175.7  332.4
//            M = 128      122.8  126.0  128.3  134.0  171.2  |     244.6  248.1  250.3  256.1
//     d 64,  M = 16        63.4   99.5  140.8  183.4  355.9  |      47.3   72.1  131.0  252.1
//            M = 32        66.7   68.9  103.4  105.9  192.3  |      51.0   51.8   84.7  147.7
//            M = 128       79.9   81.9   94.9   96.3  113.1  |     140.6  141.3  143.9  148.1
// (64 rows of d 128 in fp32 by four waves that share their blocks: no less than twice 32.)
int32_t rows_of(int32_t dtype, int64_t rows)
{
    return rows <= 16 ? 16 : rows <= (dtype == BS_BF16 ? 32 : 64) ? 32 : 128;
}

// What the host has to know of the kernel's layout.
struct Traits { int32_t rows, keys, per_cu, turns, item; };
Traits traits_of(const bs_cache &c, int32_t M)
{
    const auto get = [](auto k) {
        typedef typename decltype(k)::layout L;
        return Traits{L::kRows, L::kKeys, L::kPerCu, L::kTurns, L::kItem};
    };
    if (c.dtype == BS_BF16) return c.head_dim == 64 ? with_rows<__bf16, 64>(M, false, get) : with_rows<__bf16, 128>(M, false, get);
    return c.head_dim == 64 ? with_rows<float, 64>(M, false, get) : with_rows<float, 128>(M, false, get);
}

template <typename T, int D>
hipError_t raise_limits()
{
    for (int i = 0; i < 4; ++i) {
        const hipError_t e = with_rows<T, D>(i == 0 ? 16 : i == 1 ? 32 : 128, i == 3, [](auto k) {
            typedef decltype(k) K;
            return hipFuncSetAttribute(reinterpret_cast<const void *>(K::kernel), hipFuncAttributeMaxDynamicSharedMemorySize, K::layout::kLds);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int device_setup(int *n_cus)
{
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail_hip(e, "hipGetDevice");
    if (dev < 0 || dev >= kMaxDevices) return fail_msg(BS_EUNSUPPORTED, "device ordinal above 63");
    std::lock_guard<std::mutex> lock(g_mutex);
    if (g_n_cus[dev] == 0) {
        e = raise_limits<__bf16, 64>();
        if (e == hipSuccess) e = raise_limits<__bf16, 128>();
        if (e == hipSuccess) e = raise_limits<float, 64>();
        if (e == hipSuccess) e = raise_limits<float, 128>();
        if (e != hipSuccess) return fail_hip(e, "hipFuncSetAttribute");
        int cus = 0;
        e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
        if (e != hipSuccess || cus <= 0) return fail_hip(e, "hipDeviceGetAttribute(compute units)");
        g_n_cus[dev] = cus;
    }
    *n_cus = g_n_cus[dev];
    return BS_OK;
}

int check_tree(const bs_cache *cache, int32_t n_q_heads, int32_t n_tokens, int32_t max_tokens)
{
    if (int rc = check_cache(cache)) return rc;
    if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0 || n_tokens < 0 || max_tokens < 1 || max_tokens > BS_TREE_MAX_TOKENS) return BS_EINVAL;
    if (cache->head_dim != 64 && cache->head_dim != 128) return BS_EUNSUPPORTED;
    return BS_OK;
}

// How a call is laid out over the chip and its workspace: nothing but sizes, so that a graph of a call stays right when lengths change.
struct Plan {
    int32_t M, n_shares, n_cuts, most_items;      // rows of an item; shares; entries of cuts; items of a sequence
    int64_t part_o, part_ml, cuts, bytes;         // offsets
};

int make_plan(const bs_cache &c, int32_t n_q_heads, int32_t n_tokens, int32_t max_tokens, int n_cus, Plan *p)
{
    const int32_t G = n_q_heads / c.n_kv_heads;
    const int64_t rows = (int64_t)G * std::min(std::max(1, n_tokens), max_tokens);   // of a sequence and KV head
    if (rows > 1 << 20) return BS_EUNSUPPORTED;   // (see token_of)
    const Traits t = traits_of(c, rows_of(c.dtype, rows));
    p->M = t.rows;
    const int64_t groups = (rows + p->M - 1) / p->M, per_item = (cache_slots(c) + t.keys - 1) / t.keys + 1, items = (int64_t)c.n_seqs * c.n_kv_heads;
    if (items > INT32_MAX / groups || items * groups > INT32_MAX / 2 / (per_item + t.item)) return BS_EUNSUPPORTED;   // units are counted in 32 bits
    p->most_items = (int32_t)(groups * c.n_kv_heads);
    p->n_shares = (int32_t)std::min<int64_t>((int64_t)n_cus * t.per_cu, (items * groups * per_item + t.turns - 1) / t.turns);
    const auto whole = [](int64_t bytes) { return (bytes + 255) / 256 * 256; };
    p->part_o = 0;
    p->part_ml = whole((int64_t)2 * p->n_shares * p->M * c.head_dim * 4);
    p->cuts = p->part_ml + whole((int64_t)2 * p->n_shares * p->M * 8);
    p->n_cuts = (int32_t)std::min<int64_t>(p->n_shares, items * groups);
    p->bytes = p->cuts + whole((int64_t)p->n_cuts * sizeof(Cut));
    return BS_OK;
}

template <typename T, int D>
int launch(const TreeArgs &a, const Plan &p, hipStream_t st)
{
    return with_rows<T, D>(p.M, a.cap_log2e > 0.f, [&](auto k) {
        typedef decltype(k) K;
        typedef typename K::layout L;
        hipError_t e = launch_kernel(K::kernel, dim3((unsigned)p.n_shares), dim3(L::kThreads), L::kLds, st, a);
        if (e != hipSuccess) return fail_hip(e, "tree_shares launch");
        if (p.n_shares > 1) e = launch_kernel(tree_join<T, D, L>, dim3((unsigned)p.n_cuts, (unsigned)std::max(8, std::min(L::kRows, 4096 / p.n_cuts))), dim3(256), 0, st, a);
        return e == hipSuccess ? BS_OK : fail_hip(e, "tree_join launch");
    });
}

}  // namespace
}  // namespace bs

extern "C" int64_t bs_attn_tree_workspace(const bs_cache *cache, int32_t n_q_heads, int32_t n_tokens, int32_t max_tokens)
{
    using namespace bs;
    if (int rc = check_tree(cache, n_q_heads, n_tokens, max_tokens)) return rc;
    int n_cus = 0;
    Plan p;
    if (int rc = device_setup(&n_cus)) return rc;
    if (int rc = make_plan(*cache, n_q_heads, n_tokens, max_tokens, n_cus, &p)) return rc;
    return p.bytes;
}

extern "C" int bs_attn_tree(const bs_cache *cache, const bs_heads *q, const bs_heads *out, int32_t n_tokens, const int32_t *first, const int32_t *lens, int32_t max_tokens,
                            const uint64_t *mask, int32_t mask_words, int32_t window, float scale, float cap, void *workspace, int64_t workspace_bytes, void *stream)
{
    using namespace bs;
    const bool none = n_tokens == 0;
    if (check_heads(q, none) || check_heads(out, none) || q->n_heads != out->n_heads || !first || !lens || window < 0) return BS_EINVAL;
    if (!(scale > 0.f) || !std::isfinite(scale) || !(cap >= 0.f) || !std::isfinite(cap)) return BS_EINVAL;
    if (cap == 0.f && !std::isfinite(scale * 1.4426950408889634f)) return BS_EUNSUPPORTED;
    if (int rc = check_tree(cache, q->n_heads, n_tokens, max_tokens)) return rc;
    if (mask_words < 0 || (mask ? mask_words < (max_tokens + 63) / 64 : mask_words != 0 && !none) || (uintptr_t)mask % 8 != 0) return BS_EINVAL;   // (an empty mask's address is null)
    if (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < 0) return BS_EINVAL;
    if (!rows_aligned(*q, cache->dtype) || !rows_aligned(*out, cache->dtype)) return BS_EUNSUPPORTED;
    if (int rc = check_rows_apart(*out, n_tokens, cache->head_dim)) return rc;
    const float to_cap = cap > 0.f ? scale / cap : 0.f;
    if (cap > 0.f && (!(to_cap > 0.f) || !std::isfinite(to_cap) || !std::isfinite(cap * 1.4426950408889634f) || !(cap * 1.4426950408889634f > 0.f))) return BS_EUNSUPPORTED;
    int n_cus = 0;
    Plan p;
    if (int rc = device_setup(&n_cus)) return rc;
    if (int rc = make_plan(*cache, q->n_heads, n_tokens, max_tokens, n_cus, &p)) return rc;
    const int32_t G = q->n_heads / cache->n_kv_heads;
    // rows of a sequence and KV head are addressed from its first token's in 32 bits
    if (((__int128)q->token_stride * (std::min(n_tokens, max_tokens) + 1) + (__int128)q->head_stride * G) * element_bytes(cache->dtype) > INT32_MAX) return BS_EUNSUPPORTED;
    if (workspace_bytes < p.bytes) return BS_EINVAL;
    if (none) return BS_OK;
    TreeArgs a{};
    a.cache = *cache;
    a.q = q->data; a.q_head = q->head_stride; a.q_token = q->token_stride;
    a.out = out->data; a.out_head = out->head_stride; a.out_token = out->token_stride;
    a.first = first;
    a.lens = lens;
    a.mask = mask;
    a.mask_words = mask_words;
    a.n_tokens = n_tokens;
    a.max_tokens = std::min(n_tokens, max_tokens);
    a.G = G;
    a.inv_g = 1.f / G;
    a.window = window;
    a.most_items = p.most_items;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.to_cap = to_cap;
    a.cap_log2e = cap * 1.4426950408889634f;
    char *ws = static_cast<char *>(workspace);
    a.part_o = reinterpret_cast<float *>(ws + p.part_o);
    a.part_ml = reinterpret_cast<float2 *>(ws + p.part_ml);
    a.cuts = reinterpret_cast<Cut *>(ws + p.cuts);
    a.by_item = p.n_cuts < p.n_shares;
    hipStream_t st = (hipStream_t)stream;
    if (cache->dtype == BS_BF16) return cache->head_dim == 64 ? launch<__bf16, 64>(a, p, st) : launch<__bf16, 128>(a, p, st);
    return cache->head_dim == 64 ? launch<float, 64>(a, p, st) : launch<float, 128>(a, p, st);
}
