"""CPU oracle (test infrastructure only; never imported by the product path)."""
from .lshmoe_oracle import (  # noqa: F401
    widen, narrow, hash_ref, sphere_hash_ref, gate_logits_ref, combine_codes, group_ref, centroid_ref, restore_ref, restore_backward_ref,
    compress_backward_ref, combine_backward_ref, row_rel_err,
)
from .experts_oracle import (  # noqa: F401
    gate_topk_ref, gate_topk_backward_ref, activation_ref, activation_slope_ref, expert_forward_ref,
    expert_backward_input_ref, expert_backward_weight_ref, mx4_quantize_ref, mx4_values_ref,
)
