"""MI355X-native emulated Trivance AllReduce (arXiv 2602.17254).

The native library (libtrivance.so, C ABI in include/trivance.h) holds the schedule generator, the
gfx950 kernels of the AllReduce and the operators of a data-parallel step around it (layer norm, a
router's balance loss, orthogonalised updates); `binding` marshals arguments to it; `inputs` produces seeded synthetic inputs.
"""

from .binding import (  # noqa: F401
    BANDWIDTH_OPT, BF16, BRUCK_REF, F16, F32, I32, I64, LATENCY_OPT, QUINTIC_5, Plan, TrivanceError, trivance_algorithmic_bytes,
    trivance_allreduce_emulated, trivance_allreduce_emulated_steps, trivance_allreduce_emulated_steps_ws,
    trivance_allreduce_emulated_ws, trivance_block_range, trivance_workspace_bytes,
    trivance_congestion, trivance_congestion_device, trivance_copy_device, trivance_cost_model,
    trivance_fill_hash_uniform,
    trivance_pass_bytes, trivance_plan, trivance_plan_step, trivance_plan_step_index,
    trivance_plan_with_dispatch_limit, trivance_layernorm_forward, trivance_layernorm_backward,
    trivance_layernorm_workspace_bytes, trivance_balance_counts, trivance_balance_loss,
    trivance_balance_backward, trivance_balance_workspace_bytes, trivance_orthogonalize,
    trivance_orthogonalize_workspace_bytes)
