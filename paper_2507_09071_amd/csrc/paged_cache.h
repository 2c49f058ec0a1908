// Checks that the calls around the KV cache have in common (internal to the library).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "blindsight.h"

namespace bs {

inline int element_bytes(int32_t dtype) { return dtype == BS_BF16 ? 2 : 4; }
inline int64_t cache_slots(const bs_cache &c) { return (int64_t)c.max_pages * c.page_size; }   // slots that a sequence can have

// A kernel's loop over pages and slots keeps slot numbers in 32 bits.
constexpr int64_t kMaxSlots = INT32_MAX - 65536;
constexpr int64_t kMaxStride = (int64_t)1 << 40;

int check_cache(const bs_cache *c);
int check_heads(const bs_heads *h, bool none = false);   // data, sizes and strides; none: of no tokens, whose data may be null
// Rows that are written lie apart from each other.
int check_rows_apart(const bs_heads &h, int32_t n_tokens, int32_t head_dim);
int check_rows_apart(const bs_cache &c);
// Rows of the cache's sequences and KV heads; `row_stride` has to hold their slots.
int check_slots(const bs_cache &c, const bs_slots *s);
// 16-byte loads of whole rows: pointer and strides allow them.
bool rows_aligned(const bs_heads &h, int32_t dtype);

}  // namespace bs
