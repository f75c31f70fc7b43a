"""What modules that keep data on the GPU between calls need to know of CUDA graphs and streams."""
from __future__ import annotations

import weakref

import torch

from . import binding


def stream_of(x: torch.Tensor) -> int:
    """The handle of the current stream of x's device; 0 for what is not on a GPU."""
    if not x.is_cuda:
        return 0
    return binding._raw_stream(x.device.index) if binding._raw_stream is not None else torch.cuda.current_stream(x.device).cuda_stream


def capturing(x: torch.Tensor) -> bool:
    """Whether what is done with x now goes into a CUDA graph."""
    return x.is_cuda and torch.cuda.is_current_stream_capturing()


def capture_id(x: torch.Tensor) -> int:
    """The number of the capture that what is done with x now goes into; every capture has another one.  (1 for what is not on a GPU.)"""
    return binding.b2_graph_capture_id(stream_of(x)) if x.is_cuda else 1


class Made:
    """Tensors that one call leaves for later ones: who reads them on another stream waits for the work that makes them, and their memory is given away after him.

    capture: the number of the capture that they are made in, or 0."""

    __slots__ = ("tensors", "capture", "_event", "_streams")

    def __init__(self, tensors, capture: int):
        self.tensors, self.capture, self._event, self._streams = tensors, capture, None, set()
        if tensors[0].is_cuda:
            stream = torch.cuda.current_stream(tensors[0].device)
            self._event = stream.record_event()
            self._streams.add(stream.cuda_stream)

    def use(self, capture: int) -> None:
        """What is enqueued now on the current stream, in the capture of that number or in none, may read the tensors.  A graph that is captured has to keep them alive."""
        if self._event is None:
            return
        if capture and not self.capture:  # its graph may run on any stream
            binding.b2_event_finish(self._event.cuda_event)
            return
        if stream_of(self.tensors[0]) not in self._streams:
            stream = torch.cuda.current_stream(self.tensors[0].device)
            stream.wait_event(self._event)
            for t in self.tensors:
                t.record_stream(stream)
            self._streams.add(stream.cuda_stream)


class GraphWatch:
    """Tells when the graph that is being captured on x's current stream is gone, and with it who may read what was kept for it."""

    def __init__(self, x: torch.Tensor, capture: int):
        self.capture, self._watch = capture, None
        if x.is_cuda:
            try:
                self._watch = binding.b2_graph_watch(stream_of(x))
            except binding.B2Error as e:  # too many: what was kept for this one stays
                if e.status != binding.STATIC_LIMIT:
                    raise
                return
            weakref.finalize(self, binding.b2_graph_unwatch, self._watch).atexit = False

    def gone(self) -> bool:
        return self._watch is not None and binding.b2_graph_gone(self._watch)


DEFAULT_STREAM = 0


class AutogradGraphs(list):
    """The autograd graphs through a module that may be alive, each as a weak reference to its node and the stream that it was made on.

    What reaches a parameter's gradient goes to the stream where the oldest living graph met the parameter first.  A capture can take another stream in, but not the default one: there it ends
    with an error in the middle of the backward pass, or takes the process with it.  So such a pass is refused before it begins."""

    _most = 32  # entries before those that are gone are dropped

    def elsewhere(self, stream: int) -> list:
        """The nodes of those that were made on other streams."""
        return [node for node in (g() for g, s in self if s != stream) if node is not None]

    def add(self, node, stream: int) -> None:
        if len(self) >= self._most:  # a module that one pass calls a thousand times does not look through all of them every time
            self[:] = [g for g in self if g[0]() is not None]
            self._most = max(32, 2 * len(self))
        self.append((weakref.ref(node), stream))

    def refuse(self, node, stream: int) -> None:
        """In a captured backward pass through a node."""
        if stream != DEFAULT_STREAM and any(s == DEFAULT_STREAM and g() is not None for g, s in self) and any(_reached(n) for n, _ in node.next_functions):
            raise RuntimeError("an autograd graph of this module that was made on the default stream is alive: delete its results, or make it on the stream that captures")


def _reached(node) -> bool:
    """Whether the backward pass that runs now makes the gradient of the parameter whose node this is."""
    if node is None or not hasattr(node, "variable"):
        return False
    try:
        return torch._C._will_engine_execute_node(node)
    except RuntimeError:  # it does not say so of what torch.autograd.grad hands out
        return True
