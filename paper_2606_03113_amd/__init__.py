"""MI355X-native batch-1 self-speculative decoding with learned
(exit layer, draft length) control.  The compute path is liblede.so
(hand-written gfx950 HIP kernels behind the C ABI in include/lede.h);
``lede`` is its ctypes binding."""
from .lede import (Cache, CacheMoves, CachePlan, Dqn, Engine, HeadLoss, LedeError, Logprobs, QuantMatrix, load,  # noqa: F401
                   make_config,
                   op_cache_append, op_cache_attention, op_cache_compact, op_cache_copy, op_cache_fork, op_cache_free, op_cache_own,
                   op_cache_plan, op_cache_read, op_head_loss, op_head_loss_grad, op_linear, op_logprobs,
                   op_quant_linear, op_quantize, op_read_groups, op_read_probe, op_sample, op_sample_noalloc)
