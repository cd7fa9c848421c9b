"""ambptt: backpropagation through time under asynchronous multistage
checkpointing on one AMD Instinct MI355X (gfx950).

The compute path is libambptt.so (HIP kernels, checkpoint tiers, executor,
schedule generator, operators of a residual block) behind the C ABI in
include/ambptt.h and include/ambptt_ops.h; this package only marshals torch
tensors into it.
"""
from .api import (ProblemSpec, Runner, interval_from_timings, query, resident_program, revolve_advances, schedule_evals,
                  schedule_text, schedule_text_costs, schedule_text_online, schedule_text_sized, schedule_text_starts,
                  version)
from .ops import (add_norm, add_norm_backward, decay_attention, decay_attention_backward, decay_attention_step, dropout,
                  dropout_counters)
from ._lib import AmbpttError, LIB_PATH, load

__all__ = ["ProblemSpec", "Runner", "interval_from_timings", "query", "resident_program", "revolve_advances", "schedule_evals", "schedule_text",
           "schedule_text_costs", "schedule_text_online", "schedule_text_sized", "schedule_text_starts", "version", "add_norm", "add_norm_backward", "decay_attention",
           "decay_attention_backward", "decay_attention_step", "dropout", "dropout_counters", "AmbpttError", "LIB_PATH", "load"]
