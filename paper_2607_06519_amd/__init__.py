"""FreqDepthKV compressed-KV path on AMD MI355X (gfx950).

The product is ``libfdkv.so`` (C ABI declared in ``include/fdkv.h``) with its
hand-written HIP kernels under ``csrc/``; ``binding`` marshals torch tensors
and numpy arrays into those calls.
"""
from . import binding  # noqa: F401
from .binding import (BF16, EXACT, F32, RESIDUAL, SHARED, Dims, FdkvError, block_select,  # noqa: F401
                      block_select_workspace, compress, decode_attn, decode_parts, decode_parts_workspace,
                      decode_workspace, dims, key_bounds, layout, page_read, page_write, paged_attn, paged_attn_workspace,
                      pages, part, probe, probe_workspace, prompt_attn, prompt_attn_workspace, rope, rope_append, route)
