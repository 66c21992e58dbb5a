"""GB300-native cache-aware MoE routing and expert residency.

The product is the CUDA library ``_build/libcrc.so`` (C ABI in
``include/crc.h``); :mod:`paper_2609_04895_gb300.crc` is its ctypes binding.
Build it with :func:`paper_2609_04895_gb300.build.build`.
"""
from . import crc  # noqa: F401
from .crc import (CrcError, MoeLayer, State, Trace, cache_loss, cache_scan,  # noqa: F401
                  expert_views, group_choices, group_matmul, group_matmul_grad, load_time,
                  matvec4, metrics, pinned_empty, problem, problem_of, quantize_rows,
                  quantize_rows4, rms_norm, rms_norm_grad, route_and_cache, route_and_cache_host,
                  route_scores, split_rows, sum_choices, sum_choices_grad, synth_hidden,
                  synth_weights, transfer_plan, transfer_replay)

__all__ = ["crc", "CrcError", "MoeLayer", "State", "Trace", "cache_loss", "cache_scan",
           "expert_views", "group_choices", "group_matmul", "group_matmul_grad", "load_time",
           "matvec4", "metrics", "pinned_empty", "problem", "problem_of", "quantize_rows",
           "quantize_rows4", "rms_norm", "rms_norm_grad", "route_and_cache",
           "route_and_cache_host", "route_scores", "split_rows", "sum_choices", "sum_choices_grad",
           "synth_hidden", "synth_weights", "transfer_plan", "transfer_replay"]
