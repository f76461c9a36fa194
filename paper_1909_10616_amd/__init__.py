"""Tuned GEMM for MI355X (gfx950) with the G-BFS configuration search of
arxiv 1909.10616 (and its N-A2C and random-search tuners), and layer operators beside it: perceptron
layers with their gradients, the routing of tokens, and layers of experts. The compute path is
libgemmtune.so (HIP); this package only binds it."""
from .gemmtune import (A_KMAJOR, ADJACENT, ANY_PAIR, BF16, F32, GemmTuneError, Space,  # noqa: F401
                       gemm_run, gt_compare, gt_measure, gt_reference_gemm, lower, tflops,
                       tune_gbfs, tune_na2c, tune_random)
from .layers import (ExpertGrads, Route, gt_experts, gt_experts_backward, gt_linear,  # noqa: F401
                     gt_linear_backward, gt_route, gt_route_backward)
