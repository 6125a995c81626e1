"""Tile-sparse 3D attention (forward and gradients) for MI355X (gfx950).

The hot path of Efficient-vDiT (arXiv 2502.06155): softmax attention in which
each query latent frame only attends to the key frames its frame-tile mask
keeps (diagonal plus k global reference frames), computed by hand-written HIP
kernels behind a C ABI (include/tile_attn.h). This package is the thin Python
binding of that ABI.
"""
from .api import (  # noqa: F401
    MASK_FORMS,
    TileAttnError,
    dense_attn,
    dense_attn_fwd,
    tile_attn,
    tile_attn_bwd,
    tile_attn_bwd_mmdit,
    tile_attn_compact,
    tile_attn_fwd,
    tile_attn_fwd_heads,
    tile_attn_fwd_heads_noalloc,
    tile_attn_fwd_mmdit,
    tile_attn_make_mask,
    tile_attn_plan,
    tile_attn_plan_cache_stats,
)
from .blocks import (  # noqa: F401
    BLOCK_TOKENS,
    block_attn,
    block_attn_bwd,
    block_attn_bwd_workspace,
    block_attn_fwd,
    block_attn_fwd_workspace,
    block_attn_grad,
    block_attn_lists,
    block_attn_means,
    block_lists,
    block_means,
    cache_attn,
    cache_attn_fwd,
    cache_attn_fwd_workspace,
    cache_attn_write,
    cache_write,
)
from .cache4 import (  # noqa: F401
    CACHE4_GROUP,
    cache4_attn,
    cache4_attn_fwd,
    cache4_attn_fwd_workspace,
    cache4_attn_read,
    cache4_attn_write,
    cache4_new,
    cache4_read,
    cache4_write,
)
from .rope import (  # noqa: F401
    NORMS,
    ROPE_AXES,
    ROPE_LAYOUTS,
    HeadRopeSpec,
    Rows,
    grid_positions,
    head_rope,
    head_rope_bwd,
    head_rope_bwd_workspace,
    head_rope_fwd,
    head_rope_grad,
    rope_freqs,
)
