"""What modules that keep data on the GPU between calls need to know of CUDA graphs and streams."""
from __future__ import annotations

import torch

from . import binding


def capturing(x: torch.Tensor) -> bool:
    """Whether what is done with x now goes into a CUDA graph."""
    return x.is_cuda and torch.cuda.is_current_stream_capturing()


def capture_id(x: torch.Tensor) -> int:
    """The number of the capture that what is done with x now goes into; every capture has another one.  (1 for what is not on a GPU.)"""
    return binding.b2_graph_capture_id(torch.cuda.current_stream(x.device).cuda_stream) if x.is_cuda else 1
