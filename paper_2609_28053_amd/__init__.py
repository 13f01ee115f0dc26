"""MI355X-native routing + Exact Quantile Balancing statistics for one MoE layer.

The kernels live in libeqb.so (C ABI declared in include/eqb.h); ``eqb`` is its
thin Python binding; ``train`` holds the buffers of the operators that train a
layer around its routing (experts' rows, balance loss, AdamW).
"""
from . import eqb
from .eqb import Layer, run_layer, eqb_rank, qb_loop, rank_averaged_qb, histogram_qb
from .train import AdamW, BalanceLoss, ExpertRows

__all__ = ["eqb", "AdamW", "BalanceLoss", "ExpertRows", "Layer", "run_layer", "eqb_rank", "qb_loop", "rank_averaged_qb", "histogram_qb"]
