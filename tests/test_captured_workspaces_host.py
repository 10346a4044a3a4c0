"""Which workspaces a context keeps for captured graphs, on a context without a device: what a captured graph refers to is never given back."""
import gc
import weakref

import pytest
import torch

from paper_2210_13149_b200 import binding as B


class Library:
    """The two calls that a change of workspace makes."""

    def __init__(self):
        self.attached = []

    def bigcn_set_workspace(self, handle, pointer, nbytes):
        self.attached.append(nbytes)
        return 0

    def bigcn_destroy(self, handle):
        pass


@pytest.fixture
def ctx(monkeypatch):
    c = object.__new__(B.BiGCN)
    c.lib, c.h, c.device, c.stream, c._raw_stream, c.workspace, c._captured = Library(), 1, torch.device("cpu"), None, 7, None, []
    c.capturing = False
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: c.capturing, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 7, raising=False)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: None)
    return c


def test_a_captured_workspace_outlives_an_eager_call_that_outgrows_it(ctx):
    ctx.capturing = True
    ctx.ensure_workspace(1000)                  # as layer_forward() and the others ask for theirs
    captured = weakref.ref(ctx.workspace)
    ctx.capturing = False
    ctx.ensure_workspace(5000)
    gc.collect()
    assert captured() is not None and ctx.workspace.numel() == 5000 and ctx.lib.attached == [1000, 5000]


def test_one_that_the_same_capture_replaces_stays_too(ctx):
    ctx.ensure_workspace(1000)                  # there before the capture
    first = weakref.ref(ctx.workspace)
    ctx.capturing = True
    ctx.ensure_workspace(800)
    ctx.ensure_workspace(3000)
    second = weakref.ref(ctx.workspace)
    ctx.ensure_workspace(9000)
    ctx.capturing = False
    ctx.ensure_workspace(20000)
    gc.collect()
    assert first() is not None and second() is not None and len(ctx._captured) == 3


def test_without_a_capture_nothing_is_kept(ctx):
    ctx.ensure_workspace(1000)
    first = weakref.ref(ctx.workspace)
    ctx.ensure_workspace(2000)
    gc.collect()
    assert first() is None and ctx._captured == []
