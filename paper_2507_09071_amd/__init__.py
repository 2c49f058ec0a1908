"""MI355X-native sparse prefill attention (BlindSight hot path): thin ctypes binding over
libblindsight.so.  Argument marshalling only — every step of the path runs in the library."""
from .binding import (  # noqa: F401
    BS_BF16, BS_F32, BS_MAP_BIDIR_IMAGES, BS_MAP_PACK_KEYS, BS_MAP_REGROUP_ROWS, DENSE, SINK, INTRA, INTRA_SINK, BlindsightError, TileMap,
    bs_build_tilemap, bs_attn_prefill, bs_attn_prefill_ex, bs_attn_prefill_static, bs_static_scratch_bytes, bs_characterize_prompt, bs_head_sq_error,
    bs_aggregate_head_type, bs_aggregate_layer, bs_alpha_layer, library_path, load_library,
    BS_ROPE_HALF, BS_ROPE_INTERLEAVED, BS_ROPE_PLAIN, BS_ROPE_LINEAR, BS_ROPE_BASE, BS_ROPE_PARTS, Rope, Heads, KVCache, CacheSlots,
    bs_rope_init, bs_rope_apply, bs_cache_append, bs_attn_decode, bs_attn_decode_workspace, bs_cache_evict, bs_cache_evict_workspace,
)
