"""MI355X (gfx950) implementation of MOPAR's sliced inference hot path.

The computation runs in libmopar.so (hand-written HIP); this package is its
Python binding.  See include/mopar.h for the C ABI.
"""
from ._lib import MoparError, lib  # noqa: F401
from .binding import (SlicedModel, boundary_to_canonical, make_codec, make_plan,  # noqa: F401
                      mopar_boundary_code_bytes, mopar_boundary_decode, mopar_boundary_encode,
                      mopar_plan_slices, mopar_subslice_range, tensor_desc)
from .decoder import (Rows8, alloc_linear8_workspace, alloc_rows8, alloc_token_logprobs_workspace, mopar_linear8,  # noqa: F401
                      mopar_linear8_workspace_bytes, mopar_quantize_rows, mopar_rms_norm, mopar_token_logprobs,
                      mopar_token_logprobs_workspace_bytes)
from .serving import (PagedCache, Rotary, alloc_attention_workspace, mopar_attention_cache,  # noqa: F401
                      mopar_attention_cache_workspace_bytes, mopar_attention_prompt, mopar_cache_append, mopar_cache_keep,
                      mopar_rotary_apply)
