"""Plain fp64 CPU oracle for block-diffusion masked attention, for the norms
and rotations in front of it, for decoding over a paged cache (also where sequences
share a prefix, or attend to chosen pages), and for the token log-probabilities and objectives that consume its output.

TEST INFRASTRUCTURE ONLY.  Only the test suite, the smoke check and the
benchmark's CPU-baseline leg may import this package; the product path
(the HIP library and its Python binding) never calls it.
"""
from .bd_attn_oracle import (  # noqa: F401
    block_index,
    visibility_mask,
    allowed_count,
    forward,
    backward,
    probabilities,
    sampled,
    varlen_visibility_mask,
    varlen_forward,
    varlen_backward,
    decode_forward,
)
from .lce_oracle import (  # noqa: F401
    lm_head_logprobs,
    lm_head_backward,
    masked_ce_objective,
    dipo_objective,
    lm_head_sampled,
)
from .rope_oracle import rope_table, norm_rope, norm_rope_backward  # noqa: F401
from .paged_oracle import paged_decode_forward, paged_plan  # noqa: F401
from .sparse_oracle import page_scores, select, shared_decode_forward, sparse_decode_forward, summarize  # noqa: F401
