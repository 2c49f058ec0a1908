// Attention of one new token per sequence over a paged cache.
//
// What has to be done is reading K and V of every visible slot once, so the bound is HBM: 4 d FLOP for every query head of a group
// and slot are at most a few dozen per byte, which the matrix pipe does on the side (busy 7 % of the time).  Measured: two sequences of 150K
// slots, 32 / 16 heads of 128, 2.46 GB: 412 us, 6.0 TB/s, what a kernel that only reads reaches; one of 39.5K, 28 / 4 heads, 81 MB: 21 to 24 us, of
// which the two kernels are 17.8 and 4.0 (13 at that rate); 48 sequences of 17 to 16K slots, 40 / 8 heads, 498 MB: 102 us; fp32, 32 / 8 heads, four
// sequences of 8K to 16K: 76 us, 5.0 TB/s.  Farthest from that rate are many short sequences, whose items are two or three blocks for four waves, with an
// empty pipeline and a merge around each: 256 of 5 to 300 slots, 32 / 16 heads, 161 MB: 73 us (26 at that rate), 40 / 8 heads, 84 MB: 44 (13).
// Tried: half as many waves in twice as many workgroups (412 -> 448), a wave per short item (the 73 us 70 -> 56 before probabilities were whole, but
// 3 % and more slower where sequences have 200 to 2K slots), query rows and page numbers of the next item ahead of time (nothing).  How:
//  * the query heads of a KV head are the free dimension of a 16x16 MFMA (one block of 16 rows, or two; groups of 32 beyond that), so K and
//    V are read once for all of them;
//  * the work of all sequences and KV heads ("items") is one row of blocks of 32 slots (16 in fp32: the same bytes), cut into equal
//    shares, one per workgroup, wherever that falls.  Lengths are known on the device only, so every workgroup finds its share by itself, from a
//    sum over the lengths.  A batch of very different lengths is balanced to within four blocks, and one long sequence fills the chip;
//  * the four waves of a workgroup take every fourth block and run on their own: no barrier in the loop.  K and V blocks go from
//    the pages to LDS with 16-byte LDS-direct loads, two blocks deep: 32 KB in flight per wave.  Page numbers come through the scalar cache,
//    a step before they are needed.  Chunks of 16 bytes are exchanged within a row (XOR with its number) so that reads of K's columns are free of conflicts; of V two
//    rows meet in the same banks (two cycles more a read, 16 of 24 reads of a block), which does not show while memory is the bound;
//  * an item that lies within a share is finished there, another's parts are joined by a second, small kernel in a fixed order;
//  * with weights, the scores are left in the workspace (4 bytes per head and slot, where K has 256) and a third kernel turns them
//    into probabilities once the sums are known: reading K again would cost half as much as the attention.
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

constexpr int kWaves = 4, kThreads = 64 * kWaves;

// An item in more than one share: the first and the last workgroup that have a part of it.  Filed under the item where there are fewer items than shares
// (first = last: a whole one), else under the first share (item -1: none goes on behind it).
struct Cut { int32_t item, first, last; };

struct DecodeArgs {
    bs_cache cache;
    const void *q;
    void *out;
    int64_t q_head, q_seq, out_head, out_seq;
    const int32_t *lens;
    int32_t G, groups, window;    // heads per KV head; groups of rows that they make
    int32_t rows;                 // rows of a partial result: at most 16 or 32
    int32_t n_shares;
    float scale_log2e;
    float *part_o;                // [2 n_shares][rows][d]: of share w, 2 w the item that began before it, 2 w + 1 the one that goes on behind it
    float2 *part_ml;              // reference point and sum
    Cut *cuts;
    int32_t by_item;
    // with weights
    int32_t item_blocks;          // room for the blocks of an item
    float *scores;                // [seq][item][block][rows][slots of a block], times scale log2(e)
    float *log_sums;              // [seq][query head], to base 2
    const float *weights;
    float *weights_out;
    int64_t in_stride, out_stride;
};

template <typename T, int D>
struct Traits {
    static constexpr int kKeys = sizeof(T) == 2 ? 32 : 16;    // slots of a block
    static constexpr int kRowBytes = D * (int)sizeof(T);
    static constexpr int kBlock = kKeys * kRowBytes;          // one block of K or V
    static constexpr int kLoads = kBlock / 1024;              // LDS-direct instructions per block
    static constexpr int kLoads16 = 16 * kRowBytes / 1024;    // ... per 16 slots, which lie in one page
    static constexpr int kWave = 4 * kBlock;                  // two stages of K and V
    static constexpr int kRing = kWaves * kWave;
    static constexpr int kPerCu = D == 64 ? 2 : 1;            // workgroups per CU
    static constexpr int kRowsMax = 32;
    static constexpr int kQuery = kRing + kWaves * kRowsMax * 8;   // the query rows
    static constexpr int kLds = kQuery + kRowsMax * kRowBytes;
    // exchange of the 16-byte chunks of row r: rows that share their banks get different chunks
    __device__ static int swizzle(int r) { return kRowBytes == 128 ? (r >> 1) & 7 : r & 15; }
};

// Beginning an item (its query rows, an empty pipeline, the merge of the waves) costs about as much as so many blocks: shares are equal with
// that counted.  Else a share of many short sequences takes longest: 48 sequences of 17 to 16K slots 102 us, 130 without.
constexpr int kItemBlocks = 4;

// Blocks of a sequence that are visible, from block `first` on; `units`: those of an item and what its beginning costs.
struct Visible { int n, begin, first, blocks, units; };
template <int KEYS>
__device__ inline Visible visible(const DecodeArgs &a, int seq)
{
    Visible v;
    v.n = max(0, min(scalar_load<int>(a.lens + seq), a.cache.max_pages * a.cache.page_size));
    v.begin = a.window > 0 ? max(0, v.n - a.window) : 0;
    v.first = v.begin / KEYS;
    v.blocks = (v.n + KEYS - 1) / KEYS - v.first;
    v.units = v.blocks > 0 ? v.blocks + kItemBlocks : 0;
    return v;
}

// The share of this workgroup in the row of all units: items of a sequence one behind the other, sequences one behind the other.
struct Place { int seq, item, unit; };   // sequence, item of it, unit of that
struct Range { int begin, end; Place at; int each; };   // `each`: units of a share

// `items` per sequence.  All threads of the workgroup; units of a share: a multiple of four, for the four waves.
template <int KEYS>
__device__ inline Range own_range(const DecodeArgs &a, int items, int share, int n_shares)
{
    __shared__ int wave_sums[kWaves], found[3];
    const int tid = threadIdx.x, S = a.cache.n_seqs;
    Range r;
    int total;
    if (S == 1) {
        const Visible v = visible<KEYS>(a, 0);
        total = v.units * items;
        r.each = max(kWaves, ((total + n_shares - 1) / n_shares + kWaves - 1) / kWaves * kWaves);
        r.begin = (int)min((int64_t)total, (int64_t)share * r.each);
        r.end = min(total, r.begin + r.each);
        r.at.seq = 0;
        r.at.item = v.units > 0 ? r.begin / v.units : 0;
        r.at.unit = r.begin - r.at.item * v.units;
        return r;
    }
    // a thread adds up a few sequences one behind the other
    const int each = (S + kThreads - 1) / kThreads, s0 = min(S, tid * each), s1 = min(S, s0 + each);
    const auto units_of = [&](int s) {
        const int n = max(0, min(a.lens[s], a.cache.max_pages * a.cache.page_size)), begin = a.window > 0 ? max(0, n - a.window) : 0;
        return n > 0 ? ((n + KEYS - 1) / KEYS - begin / KEYS + kItemBlocks) * items : 0;
    };
    int mine = 0;
    for (int s = s0; s < s1; ++s) mine += units_of(s);
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
    r.each = max(kWaves, ((total + n_shares - 1) / n_shares + kWaves - 1) / kWaves * kWaves);
    r.begin = (int)min((int64_t)total, (int64_t)share * r.each);
    r.end = min(total, r.begin + r.each);
    if (r.begin >= before && r.begin < before + mine) {
        int left = r.begin - before, s = s0, n = units_of(s0);
        while (left >= n) { left -= n; n = units_of(++s); }
        const int units = n / items;
        found[0] = s;
        found[1] = left / units;
        found[2] = left - left / units * units;
    }
    __syncthreads();
    r.at.seq = __builtin_amdgcn_readfirstlane(found[0]);
    r.at.item = __builtin_amdgcn_readfirstlane(found[1]);
    r.at.unit = __builtin_amdgcn_readfirstlane(found[2]);
    r.begin = __builtin_amdgcn_readfirstlane(r.begin);
    r.end = __builtin_amdgcn_readfirstlane(r.end);
    r.each = __builtin_amdgcn_readfirstlane(r.each);
    return r;
}

template <typename T, int D, int NRB, bool WEIGHTS>
__global__ __launch_bounds__(kThreads, D == 64 ? 2 : 1) void decode_shares(const DecodeArgs a)
{
    using TR = Traits<T, D>;
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int KEYS = TR::kKeys, ROWB = TR::kRowBytes, BLK = TR::kBlock, NI = TR::kLoads, NI16 = TR::kLoads16, SUB = KEYS / 16;
    constexpr int ROWS = NRB * 16, NB = D / 16, CH4 = D / 4;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int items = a.cache.n_kv_heads * a.groups, P = a.cache.page_size;

    // rows of sequences without a slot are zero
    for (int s = blockIdx.x; s < a.cache.n_seqs; s += gridDim.x)
        if (visible<KEYS>(a, s).n == 0) {
            for (int i = tid; a.by_item && i < items; i += kThreads) a.cuts[s * items + i] = Cut{s * items + i, 0, 0};
            for (int i = tid; i < a.G * a.cache.n_kv_heads * CH4; i += kThreads)
                store_row4(static_cast<T *>(a.out) + s * a.out_seq + (i / CH4) * a.out_head + i % CH4 * 4, make_float4(0.f, 0.f, 0.f, 0.f));
        }

    const Range range = own_range<KEYS>(a, items, blockIdx.x, gridDim.x);
    if (tid == 0 && !a.by_item) a.cuts[blockIdx.x].item = -1;
    if (range.begin >= range.end) return;

    typedef __attribute__((address_space(3))) void *lds_ptr;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr)lds, ring = lds0 + wave * TR::kWave;
    // LDS-direct loads: instruction j of 16 slots moves 1 KB, i.e. 1024 / ROWB whole rows; a lane picks the chunk of its row that belongs at
    // its place
    uint32_t voff[NI16];
#pragma unroll
    for (int j = 0; j < NI16; ++j) {
        const int r = j * (1024 / ROWB) + lane / (ROWB / 16), p = lane % (ROWB / 16);
        voff[j] = r * (uint32_t)(a.cache.slot_stride * sizeof(T)) + ((p ^ TR::swizzle(r)) << 4);
    }
    const auto load_lds = [](uint32_t off, const char *src, uint32_t dst) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(src), "s"(dst) : "memory", "m0");
    };
    const auto wait_loads = [](auto newer) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(newer)::value) : "memory");
    };
    const auto reads_done = []() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
    // Stores of scores count among the loads in flight.  Those of the second row block are not counted: there may be none.  (What they cost, 412 -> 475 to 500
    // us for two sequences of 150K slots with two heads a group, is the same with half as many, with four blocks' together, past the caches, and to a
    // few lines over and over: memory turns around for them.)
    constexpr int NS = WEIGHTS ? SUB : 0;

    const uint32_t k_read = wave * TR::kWave + col * ROWB + ((grp ^ TR::swizzle(col)) << 4);
    uint32_t v_read[BF16 ? 2 : 4];   // bf16: of the two halves of a block; fp32: of the four slots of a lane
    if constexpr (BF16) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 16 * h + 4 * grp + (col >> 2);
            v_read[h] = wave * TR::kWave + BLK + r * ROWB + ((((col >> 1) & 1) ^ TR::swizzle(r)) << 4) + (col & 1) * 8;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * grp + i;
            v_read[i] = wave * TR::kWave + BLK + r * ROWB + ((col ^ TR::swizzle(r)) << 4);
        }
    }

    Place at = range.at;
    int pos = range.begin;
    Visible vis = visible<KEYS>(a, at.seq);
    while (pos < range.end) {
        while (at.item == items || vis.units == 0) {   // the next sequence that has some
            at.item = 0;
            vis = visible<KEYS>(a, ++at.seq);
        }
        const int block = max(0, at.unit - kItemBlocks);   // the first one
        const int blocks = min(vis.blocks - block, range.end - pos - max(0, kItemBlocks - at.unit));
        if (blocks <= 0) break;   // the share ends where the item begins
        const int kvh = at.item / a.groups, row0 = kvh * a.G + (at.item - kvh * a.groups) * 32;
        const int n_rows = min(ROWS, (kvh + 1) * a.G - row0);
        const int n_steps = blocks > wave ? (blocks - wave + kWaves - 1) / kWaves : 0;
        const int b0 = vis.first + block + wave;   // step i: block b0 + 4 i of the sequence

        // Page numbers of 16 slots each; which slots of a block have a page.
        const int32_t *table = a.cache.page_table + (int64_t)at.seq * a.cache.max_pages;
        struct Pages { int32_t page[SUB]; uint32_t in_page[SUB]; };
        const auto pages_of = [&](int i) __attribute__((always_inline)) {
            Pages p;
#pragma unroll
            for (int h = 0; h < SUB; ++h) {
                // (behind the last slots: those again)
                const uint32_t slot = min((b0 + kWaves * min(i, n_steps - 1)) * KEYS + 16 * h, a.cache.max_pages * P - 16);
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
            for (int h = 0; h < SUB; ++h)
#pragma unroll
                for (int j = 0; j < NI16; ++j) load_lds(voff[j], src[h], dst + (h * NI16 + j) * 1024);
        };

        // The query rows (the waves share them) in the layout of a K block, then the first two blocks of keys and values.  A slot without
        // a row holds a copy of the last one, whose results are not stored.
        {
            const char *qh = reinterpret_cast<const char *>(static_cast<const T *>(a.q) + at.seq * a.q_seq + row0 * a.q_head);
            constexpr int kAll = ROWS * ROWB / 1024;
#pragma unroll
            for (int i0 = 0; i0 < kAll; i0 += kWaves) {
                const int i = i0 + wave;
                if (kAll % kWaves == 0 || i < kAll) {
                    const int r = i * (1024 / ROWB) + lane / (ROWB / 16), p = lane % (ROWB / 16);
                    load_lds(min(r, n_rows - 1) * (uint32_t)(a.q_head * sizeof(T)) + ((p ^ TR::swizzle(r)) << 4), qh, lds0 + TR::kQuery + i * 1024);
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
            if (n_steps > 1) {
                issue(s1.k, ring + 2 * BLK);
                issue(s1.v, ring + 3 * BLK);
                wait_loads(std::integral_constant<int, 4 * NI>{});
            } else {
                wait_loads(std::integral_constant<int, 2 * NI>{});
            }
        } else {
            wait_loads(std::integral_constant<int, 0>{});
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        uint4 q[NRB][D * sizeof(T) / 64];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
            for (int t = 0; t < (int)(D * sizeof(T) / 64); ++t)
                q[rb][t] = *reinterpret_cast<const uint4 *>(lds + TR::kQuery + rb * 16 * ROWB + ((col * ROWB + ((grp ^ TR::swizzle(col)) << 4)) ^ (t << 6)));

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

        float *scores = WEIGHTS ? a.scores + (((int64_t)at.seq * items + at.item) * a.item_blocks + b0) * a.rows * KEYS : nullptr;   // (no window: vis.first = 0)
        uint32_t there0 = s0.there, there1 = s1.there;   // of this block, of the next one
        for (int i = 0; i < n_steps; ++i) {
            const int stage = (i & 1) * 2 * BLK;
            const bool more = i + 1 < n_steps, more2 = i + 2 < n_steps;
            const int n0 = (b0 + kWaves * i) * KEYS;
            Sources s2{};
            if (more2) s2 = sources_of(next);
            next = pages_of(i + 3);

            // ---- S^T = K Q^T: lane: slots 16 h + 4 grp + e of query row `col` of each row block
            if (!more) wait_loads(std::integral_constant<int, NI>{});
            else if (!WEIGHTS || i == 0) wait_loads(std::integral_constant<int, 3 * NI>{});
            else wait_loads(std::integral_constant<int, 3 * NI + NS>{});
            floatx4 s[NRB][SUB];
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                for (int h = 0; h < SUB; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[rb][h][e] = 0.f;
#pragma unroll
            for (int t = 0; t < (int)(D * sizeof(T) / 64); ++t)
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
            reads_done();
            if (more2) issue(s2.k, ring + stage);

            // ---- which of the lane's slots are seen (4 bits per 16 slots), and the running maximum and sum
            uint32_t seen = there0;
            if (n0 < vis.begin) seen &= ~0u << min(31, vis.begin - n0);   // (a block has a visible slot: vis.begin - n0 < KEYS)
            if (n0 + KEYS > vis.n) seen &= ~(~0u << (vis.n - n0));
            seen >>= 4 * grp;
            float p[NRB][SUB][4];
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                const float c = a.scale_log2e;
                float mx = -INFINITY;
#pragma unroll
                for (int h = 0; h < SUB; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[rb][h][e] = (seen & (1u << (16 * h + e))) ? s[rb][h][e] : -INFINITY;
                        mx = fmaxf(mx, s[rb][h][e]);
                    }
                if constexpr (WEIGHTS) {
                    if (rb * 16 + col < n_rows) {
                        float *to = scores + ((int64_t)(kWaves * i) * a.rows + rb * 16 + col) * KEYS + 4 * grp;
#pragma unroll
                        for (int h = 0; h < SUB; ++h)
                            *reinterpret_cast<float4 *>(to + 16 * h) = make_float4(s[rb][h][0] * c, s[rb][h][1] * c, s[rb][h][2] * c, s[rb][h][3] * c);
                    }
                }
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

            // ---- O^T += V^T P^T.  Values of slots that are not seen are replaced by zero: times a probability of zero, an infinity or a NaN would
            // be a NaN.
            if (more2) wait_loads(std::integral_constant<int, 3 * NI + NS>{});
            else if (more) wait_loads(std::integral_constant<int, 2 * NI>{});
            else wait_loads(std::integral_constant<int, 0>{});
            if constexpr (BF16) {
                typedef __attribute__((address_space(3))) bf16x4 *lds_bf16x4;
                // Probabilities in three bf16 numbers each, which hold all 24 bits of their fraction: the matrix pipe waits for memory anyway, and values that
                // cancel leave nothing but what a probability has lost (one number: relative error 0.0023 for two sequences of 150K slots, where the result's own
                // rounding is 0.0017; two: 0.0017, but up to 2^-18 of sum p |v|, whatever is left of that sum).  Time of three for two: 0 to 2 % (412 / 412 us; 64 / 2 heads,
                // 32 sequences of 8K to 16K, 83.7 / 85.1).
                bf16x8 pb[NRB], rest[NRB], last[NRB];
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = p[rb][e >> 2][e & 3];
                        pb[rb][e] = (__bf16)x;
                        const float y = x - (float)pb[rb][e];
                        rest[rb][e] = (__bf16)y;
                        last[rb][e] = (__bf16)(y - (float)rest[rb][e]);
                    }
                uint32_t keep[2][2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int w = 0; w < 2; ++w)
                        keep[h][w] = ((seen >> (16 * h + 2 * w)) & 1 ? 0xffffu : 0u) | ((seen >> (16 * h + 2 * w + 1)) & 1 ? 0xffff0000u : 0u);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    uint4 f;
                    const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + ((v_read[0] + stage) ^ (nb << 5)))));
                    const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + ((v_read[1] + stage) ^ (nb << 5)))));
                    f.x = x.x & keep[0][0]; f.y = x.y & keep[0][1];
                    f.z = y.x & keep[1][0]; f.w = y.y & keep[1][1];
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
                        floatx4 x = *reinterpret_cast<const floatx4 *>(lds + v_read[e] + stage + n * 256);
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            x[w] = (seen & (1u << e)) ? x[w] : 0.f;
#pragma unroll
                            for (int rb = 0; rb < NRB; ++rb) o[rb][4 * n + w] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[w], p[rb][0][e], o[rb][4 * n + w], 0, 0, 0);
                        }
                    }
            }
            reads_done();
            if (more2) issue(s2.v, ring + stage + BLK);
            there0 = there1;
            there1 = s2.there;
        }

        // ---- the four waves' results, each in its part of the ring; [row][chunks of 4 channels, exchanged]
        float2 *ml = reinterpret_cast<float2 *>(lds + TR::kRing);   // [wave][row]
        float4 *stage = reinterpret_cast<float4 *>(lds);
        constexpr int kStageWave = TR::kWave / 16;
        static_assert(ROWS * CH4 <= kStageWave, "a wave's rows in its part of the ring");
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            const int row = rb * 16 + col;
            const float l = sum_across_groups(l_run[rb]);
            if (grp == 0) ml[wave * ROWS + row] = make_float2(m_run[rb], l);
            if (row < n_rows) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if constexpr (BF16) {   // channels 16 nb + 4 grp + i
                        stage[wave * kStageWave + row * CH4 + ((nb * 4 + grp) ^ (row & (CH4 - 1)))] = make_float4(o[rb][nb][0], o[rb][nb][1], o[rb][nb][2], o[rb][nb][3]);
                    } else {                // channel 64 n + 16 grp + 4 i + w of o[4 n + w][i]: here nb = 4 n + i
                        const int n = nb / 4, i = nb % 4;
                        stage[wave * kStageWave + row * CH4 + ((16 * n + 4 * grp + i) ^ (row & (CH4 - 1)))] =
                            make_float4(o[rb][4 * n][i], o[rb][4 * n + 1][i], o[rb][4 * n + 2][i], o[rb][4 * n + 3][i]);
                    }
                }
            }
        }
        __syncthreads();
        const bool begins = block == 0, ends = block + blocks == vis.blocks;
        const int64_t slot = (int64_t)(2 * blockIdx.x + (begins ? 1 : 0)) * a.rows;
        for (int idx = tid; idx < n_rows * CH4; idx += kThreads) {
            const int row = idx / CH4, ch = idx % CH4;
            float2 x[kWaves];
            float4 y[kWaves];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                x[w] = ml[w * ROWS + row];
                y[w] = stage[w * kStageWave + row * CH4 + (ch ^ (row & (CH4 - 1)))];
            }
            const float m = fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x));
            float l = 0.f;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = x[w].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x[w].x - m) * a.scale_log2e);
                l = fmaf(x[w].y, f, l);
                sum.x = fmaf(y[w].x, f, sum.x); sum.y = fmaf(y[w].y, f, sum.y); sum.z = fmaf(y[w].z, f, sum.z); sum.w = fmaf(y[w].w, f, sum.w);
            }
            if (begins && ends) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                store_row4(static_cast<T *>(a.out) + at.seq * a.out_seq + (row0 + row) * a.out_head + 4 * ch, make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
                if (WEIGHTS && ch == 0) a.log_sums[(int64_t)at.seq * a.cache.n_kv_heads * a.G + row0 + row] = l == 0.f ? 0.f : fmaf(m, a.scale_log2e, __builtin_amdgcn_logf(l));
            } else {
                *reinterpret_cast<float4 *>(a.part_o + (slot + row) * D + 4 * ch) = sum;
                if (ch == 0) a.part_ml[slot + row] = make_float2(m, l);
            }
        }
        if (begins && tid == 0 && (a.by_item || !ends)) {
            const int item = at.seq * items + at.item;
            a.cuts[a.by_item ? item : (int)blockIdx.x] = Cut{item, (int)blockIdx.x, (pos - at.unit + vis.units - 1) / range.each};
        }
        pos += vis.units - at.unit;   // (behind the share's end if the item is cut)
        at.unit = 0;
        ++at.item;
        if (pos < range.end) __syncthreads();   // the ring is free again
    }
}

// Joins the parts of a row (blockIdx.y) of an item that was cut (blockIdx.x): threads are D / 4 channel quads times the parts side by side, in a
// fixed order.
template <typename T, int D, bool WEIGHTS>
__global__ __launch_bounds__(256) void decode_join(const DecodeArgs a)
{
    constexpr int CH4 = D / 4, LANES = 256 / CH4;
    __shared__ float4 acc[4][CH4];
    __shared__ float2 ml[4];
    const int tid = threadIdx.x, ch = tid % CH4, p0 = tid / CH4, row = blockIdx.y;
    const int items = a.cache.n_kv_heads * a.groups;
    const Cut cut = a.cuts[blockIdx.x];
    if (a.by_item ? cut.first == cut.last : cut.item < 0) return;
    const int seq = cut.item / items, item = cut.item - seq * items;
    const int kvh = item / a.groups, row0 = kvh * a.G + (item - kvh * a.groups) * 32;
    if (row >= min(a.rows, (kvh + 1) * a.G - row0)) return;
    float m = -INFINITY, l = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    // loads of eight parts go out together ; those behind the last one to that one
    for (int w0 = cut.first + p0; w0 <= cut.last; w0 += 8 * LANES) {
        float2 x[8];
        float4 y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int w = min(w0 + i * LANES, cut.last);
            const int64_t at = (int64_t)(2 * w + (w == cut.first ? 1 : 0)) * a.rows + row;
            x[i] = a.part_ml[at];
            y[i] = *reinterpret_cast<const float4 *>(a.part_o + at * D + 4 * ch);
        }
        const float m_old = m;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, x[i].x);
        const float old = m_old == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_old - m) * a.scale_log2e);
        l *= old;
        sum.x *= old; sum.y *= old; sum.z *= old; sum.w *= old;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (w0 + i * LANES > cut.last) continue;
            const float f = x[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x[i].x - m) * a.scale_log2e);
            l = fmaf(x[i].y, f, l);
            sum.x = fmaf(y[i].x, f, sum.x); sum.y = fmaf(y[i].y, f, sum.y); sum.z = fmaf(y[i].z, f, sum.z); sum.w = fmaf(y[i].w, f, sum.w);
        }
    }
    // the parts that a wave has, across its lanes, then the waves
    const auto across = [](auto f, float x) {
        if constexpr (D == 64) {
            const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
            x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
        }
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    };
    const auto larger = [](float x, float y) { return fmaxf(x, y); };
    const auto plus = [](float x, float y) { return x + y; };
    const float m_wave = across(larger, m), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_wave) * a.scale_log2e);
    l = across(plus, l * f);
    sum = make_float4(across(plus, sum.x * f), across(plus, sum.y * f), across(plus, sum.z * f), across(plus, sum.w * f));
    if ((tid & 63) < CH4) acc[tid >> 6][ch] = sum;
    if ((tid & 63) == 0) ml[tid >> 6] = make_float2(m_wave, l);
    __syncthreads();
    if (tid >= CH4) return;
    const float m_all = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
    l = 0.f;
    sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float g = ml[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[i].x - m_all) * a.scale_log2e);
        const float4 y = acc[i][ch];
        l = fmaf(ml[i].y, g, l);
        sum.x = fmaf(y.x, g, sum.x); sum.y = fmaf(y.y, g, sum.y); sum.z = fmaf(y.z, g, sum.z); sum.w = fmaf(y.w, g, sum.w);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    store_row4(static_cast<T *>(a.out) + seq * a.out_seq + (row0 + row) * a.out_head + 4 * ch, make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
    if (WEIGHTS && ch == 0) a.log_sums[(int64_t)seq * a.cache.n_kv_heads * a.G + row0 + row] = l == 0.f ? 0.f : fmaf(m_all, a.scale_log2e, __builtin_amdgcn_logf(l));
}

// What every slot received: a thread has a slot and adds up its KV head's rows, in order.
template <int KEYS>
__global__ __launch_bounds__(kThreads) void decode_weights(const DecodeArgs a)
{
    constexpr int kSide = kThreads / KEYS;   // blocks side by side
    const int n_kv = a.cache.n_kv_heads, side = threadIdx.x / KEYS, key = threadIdx.x % KEYS;
    const Range range = own_range<KEYS>(a, n_kv, blockIdx.x, gridDim.x);
    Place at = range.at;
    int pos = range.begin;
    if (pos >= range.end) return;
    Visible vis = visible<KEYS>(a, at.seq);
    while (pos < range.end) {
        while (at.item == n_kv || vis.units == 0) {
            at.item = 0;
            vis = visible<KEYS>(a, ++at.seq);
        }
        const int block = max(0, at.unit - kItemBlocks);
        const int blocks = min(vis.blocks - block, range.end - pos - max(0, kItemBlocks - at.unit));
        if (blocks <= 0) break;
        const int64_t row = (int64_t)at.seq * n_kv + at.item;
        const float *logs = a.log_sums + row * a.G;
        // loads of four slots of a thread go out together, those behind the last one to that one
        for (int b = block + side; b < block + blocks; b += 4 * kSide) {
            int j[4];
            float sum[4], w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                j[i] = min((b + i * kSide) * KEYS + key, vis.n - 1);
                sum[i] = 0.f;
                w[i] = a.weights[row * a.in_stride + j[i]];
            }
            for (int g = 0; g < a.groups; ++g) {
                const float *x = a.scores + (row * a.groups + g) * a.item_blocks * a.rows * KEYS;
                const int n_rows = min(a.rows, a.G - 32 * g);
                for (int r = 0; r < n_rows; ++r) {
                    const float log_sum = logs[32 * g + r];
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] += __builtin_amdgcn_exp2f(x[((int64_t)(j[i] / KEYS) * a.rows + r) * KEYS + j[i] % KEYS] - log_sum);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (b + i * kSide < block + blocks && (b + i * kSide) * KEYS + key < vis.n) a.weights_out[row * a.out_stride + j[i]] = w[i] + sum[i];
        }
        pos += vis.units - at.unit;
        at.unit = 0;
        ++at.item;
    }
}

// ------------------------------------------------------------------------------------ host

constexpr int kMaxDevices = 64;
std::mutex g_mutex;
int g_n_cus[kMaxDevices];   // compute units of a device, once its kernels' limits are raised

template <typename T, int D>
hipError_t raise_limits()
{
    const void *const kernels[] = {reinterpret_cast<const void *>(decode_shares<T, D, 1, false>), reinterpret_cast<const void *>(decode_shares<T, D, 2, false>),
                                   reinterpret_cast<const void *>(decode_shares<T, D, 1, true>), reinterpret_cast<const void *>(decode_shares<T, D, 2, true>)};
    for (const void *k : kernels)
        if (const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, Traits<T, D>::kLds); e != hipSuccess) return e;
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

int check_decode(const bs_cache *cache, int32_t n_q_heads)
{
    if (int rc = check_cache(cache)) return rc;
    if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0) return BS_EINVAL;
    if (cache->head_dim != 64 && cache->head_dim != 128) return BS_EUNSUPPORTED;
    return BS_OK;
}

// How a call is laid out over the chip and its workspace.
struct Plan {
    int32_t groups, row_blocks, rows, n_shares;
    int64_t per_item, blocks;                               // at most
    int64_t part_o, part_ml, cuts, scores, log_sums, bytes;   // offsets
    int32_t n_cuts;                                         // entries of them
};

// Nothing but sizes, so that a graph of a call stays right when lengths change.
int make_plan(const bs_cache &c, int32_t n_q_heads, bool weights, int n_cus, Plan *p)
{
    const int32_t G = n_q_heads / c.n_kv_heads, keys = c.dtype == BS_BF16 ? 32 : 16;
    p->groups = (G + 31) / 32;
    p->row_blocks = G > 16 ? 2 : 1;
    p->rows = std::min(G, 32);
    p->per_item = (cache_slots(c) + keys - 1) / keys + 1;   // (a window may begin and end inside a block)
    const int64_t units = p->per_item + kItemBlocks;
    if ((int64_t)c.n_seqs * c.n_kv_heads > INT32_MAX / p->groups || (int64_t)c.n_seqs * c.n_kv_heads * p->groups > INT32_MAX / 2 / units) return BS_EUNSUPPORTED;
    p->blocks = (int64_t)c.n_seqs * c.n_kv_heads * p->groups * p->per_item;
    p->n_shares = (int32_t)std::min<int64_t>((int64_t)n_cus * (c.head_dim == 64 ? 2 : 1), (p->blocks + kWaves - 1) / kWaves);
    const auto whole = [](int64_t bytes) { return (bytes + 255) / 256 * 256; };
    p->part_o = 0;
    p->part_ml = whole((int64_t)2 * p->n_shares * p->rows * c.head_dim * 4);
    p->n_cuts = (int32_t)std::min<int64_t>(p->n_shares, (int64_t)c.n_seqs * c.n_kv_heads * p->groups);
    p->cuts = p->part_ml + whole((int64_t)2 * p->n_shares * p->rows * 8);
    p->scores = p->cuts + whole((int64_t)p->n_cuts * sizeof(Cut));
    p->log_sums = p->scores + (weights ? whole(p->blocks * p->rows * keys * 4) : 0);
    p->bytes = p->log_sums + (weights ? whole((int64_t)c.n_seqs * n_q_heads * 4) : 0);
    return BS_OK;
}

template <typename T, int D, bool WEIGHTS>
int launch(const DecodeArgs &a, const Plan &p, int n_cus, hipStream_t st)
{
    const dim3 grid((unsigned)p.n_shares), block(kThreads);
    hipError_t e = p.row_blocks == 1 ? launch_kernel(decode_shares<T, D, 1, WEIGHTS>, grid, block, Traits<T, D>::kLds, st, a)
                                     : launch_kernel(decode_shares<T, D, 2, WEIGHTS>, grid, block, Traits<T, D>::kLds, st, a);
    if (e != hipSuccess) return fail_hip(e, "decode_shares launch");
    if (p.n_shares > 1) e = launch_kernel(decode_join<T, D, WEIGHTS>, dim3((unsigned)p.n_cuts, (unsigned)p.rows), dim3(256), 0, st, a);
    if (e != hipSuccess) return fail_hip(e, "decode_join launch");
    if constexpr (WEIGHTS) {
        const int64_t wgs = std::min<int64_t>((int64_t)n_cus * 8, (p.blocks / p.groups + 3) / 4);
        e = launch_kernel(decode_weights<Traits<T, D>::kKeys>, dim3((unsigned)wgs), block, 0, st, a);
        if (e != hipSuccess) return fail_hip(e, "decode_weights launch");
    }
    return BS_OK;
}

template <typename T, int D>
int launch(const DecodeArgs &a, const Plan &p, int n_cus, hipStream_t st)
{
    return a.weights ? launch<T, D, true>(a, p, n_cus, st) : launch<T, D, false>(a, p, n_cus, st);
}

}  // namespace
}  // namespace bs

extern "C" int64_t bs_attn_decode_workspace(const bs_cache *cache, int32_t n_q_heads, int32_t with_weights)
{
    using namespace bs;
    if (int rc = check_decode(cache, n_q_heads)) return rc;
    int n_cus = 0;
    Plan p;
    if (int rc = device_setup(&n_cus)) return rc;
    if (int rc = make_plan(*cache, n_q_heads, with_weights != 0, n_cus, &p)) return rc;
    return p.bytes;
}

extern "C" int bs_attn_decode(const bs_cache *cache, const bs_heads *q, const bs_heads *out, const int32_t *lens, int32_t window, float scale,
                              const bs_slots *slots, const bs_slots *slots_out, void *workspace, int64_t workspace_bytes, void *stream)
{
    using namespace bs;
    if (check_heads(q) || check_heads(out) || q->n_heads != out->n_heads || !lens || window < 0 || !(scale > 0.f) || !std::isfinite(scale)) return BS_EINVAL;
    if (int rc = check_decode(cache, q->n_heads)) return rc;
    if (!slots != !slots_out || !workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < 0) return BS_EINVAL;
    if (slots) {
        if (!slots->weights || !slots_out->weights || check_slots(*cache, slots) || check_slots(*cache, slots_out)) return BS_EINVAL;
        if (slots->weights == slots_out->weights && slots->row_stride != slots_out->row_stride) return BS_EINVAL;
        if (window > 0) return BS_EUNSUPPORTED;
    }
    if (!rows_aligned(*q, cache->dtype) || !rows_aligned(*out, cache->dtype)) return BS_EUNSUPPORTED;
    if (int rc = check_rows_apart(*out, cache->n_seqs, cache->head_dim)) return rc;
    if (q->head_stride * element_bytes(cache->dtype) * 32 > INT32_MAX) return BS_EUNSUPPORTED;   // rows of a group are addressed in 32 bits
    int n_cus = 0;
    Plan p;
    if (int rc = device_setup(&n_cus)) return rc;
    if (int rc = make_plan(*cache, q->n_heads, slots != nullptr, n_cus, &p)) return rc;
    if (workspace_bytes < p.bytes) return BS_EINVAL;
    DecodeArgs a{};
    a.cache = *cache;
    a.q = q->data; a.q_head = q->head_stride; a.q_seq = q->token_stride;
    a.out = out->data; a.out_head = out->head_stride; a.out_seq = out->token_stride;
    a.lens = lens;
    a.G = q->n_heads / cache->n_kv_heads;
    a.groups = p.groups;
    a.window = window;
    a.rows = p.rows;
    a.n_shares = p.n_shares;
    a.scale_log2e = scale * 1.4426950408889634f;
    char *ws = static_cast<char *>(workspace);
    a.part_o = reinterpret_cast<float *>(ws + p.part_o);
    a.part_ml = reinterpret_cast<float2 *>(ws + p.part_ml);
    a.cuts = reinterpret_cast<Cut *>(ws + p.cuts);
    a.by_item = p.n_cuts < p.n_shares;
    if (slots) {
        a.item_blocks = (int32_t)p.per_item;
        a.scores = reinterpret_cast<float *>(ws + p.scores);
        a.log_sums = reinterpret_cast<float *>(ws + p.log_sums);
        a.weights = slots->weights; a.in_stride = slots->row_stride;
        a.weights_out = slots_out->weights; a.out_stride = slots_out->row_stride;
    }
    hipStream_t st = (hipStream_t)stream;
    if (cache->dtype == BS_BF16) return cache->head_dim == 64 ? launch<__bf16, 64>(a, p, n_cus, st) : launch<__bf16, 128>(a, p, n_cus, st);
    return cache->head_dim == 64 ? launch<float, 64>(a, p, n_cus, st) : launch<float, 128>(a, p, n_cus, st);
}
