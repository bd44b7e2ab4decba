"""MI355X-native batch-1 self-speculative decoding with learned
(exit layer, draft length) control.  The compute path is liblede.so
(hand-written gfx950 HIP kernels behind the C ABI in include/lede.h);
``lede`` is its ctypes binding."""
from .lede import (Cache, CachePlan, Dqn, Engine, LedeError, Logprobs, load, make_config,  # noqa: F401
                   op_cache_append, op_cache_attention, op_cache_plan, op_cache_read, op_linear, op_logprobs,
                   op_read_groups, op_read_probe, op_sample, op_sample_noalloc)
