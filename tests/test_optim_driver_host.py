"""CPU: what the update's driver checks and in which order it calls, with the library's classes in place of a GPU's."""
import numpy as np
import pytest
import torch

from paper_2210_17357_amd import binding as B
from paper_2210_17357_amd import driver


class Plan:
    """Records the calls of a plan."""

    def __init__(self, layers, lr_scale=None, decay_scale=None):
        self.extent, self.L, self.blocks, self.calls = 100, len(layers), 3, CALLS

    def norms(self, *a, **k):
        self.calls.append("norms")

    def adamw(self, *a, **k):
        self.calls.append("adamw")


class Handle:
    def decompress(self, payload, offsets, layers, cands, choice, d_out, accumulate=False, stream=None):
        CALLS.append(("decompress", payload.numel(), accumulate))


CALLS = []
SENT = B.layer_table([0, 60], [50, 45], [0, 0], [0, 0])
OFFSETS = np.array([0, 64, 128], np.int64)
PAYLOADS = [torch.zeros(n, dtype=torch.uint8) for n in (128, 130, 144)]


@pytest.fixture
def run(monkeypatch):
    monkeypatch.setattr(B, "Optim", Plan)
    CALLS.clear()
    return driver.AdamW(B.layer_table([0], [100], [0], [0]), torch.zeros(105), B.adamw(lr=1e-3, max_norm=1.0))


def receive(run, payloads, d_grads, layers=SENT, offsets=OFFSETS):
    run.receive(Handle(), payloads, offsets, layers, None, np.zeros(2, np.int32), d_grads)


def test_receive_calls(run):
    receive(run, PAYLOADS, torch.zeros(105))
    assert CALLS == [("decompress", 128, False), ("decompress", 130, True), ("decompress", 144, True), "norms", "adamw"]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float64, torch.uint8])
def test_receive_refuses_sums_that_are_not_fp32(run, dtype):
    """The payloads are turned back to fp32: a buffer of 16-bit gradients, which the step itself takes, would be half as long."""
    with pytest.raises(ValueError):
        receive(run, PAYLOADS, torch.zeros(200, dtype=dtype))
    assert CALLS == []


def test_receive_refuses_short_buffers(run):
    for n in (0, 95, 99):                               # shorter than the plan's layers
        with pytest.raises(ValueError):
            receive(run, PAYLOADS, torch.zeros(n))
    with pytest.raises(ValueError):                     # and than those that travel
        receive(run, PAYLOADS, torch.zeros(105), layers=B.layer_table([0, 61], [50, 45], [0, 0], [0, 0]))
    with pytest.raises(ValueError):                     # a payload that ends before its last layer's does
        receive(run, PAYLOADS[:1] + [torch.zeros(127, dtype=torch.uint8)], torch.zeros(105))
    assert CALLS == []


@pytest.mark.parametrize("none", [[], (), iter(())])
def test_receive_refuses_no_payloads(run, none):
    """Without one there is nothing to turn back, and the step would take whatever the buffer holds."""
    with pytest.raises(ValueError):
        receive(run, none, torch.zeros(105))
    assert CALLS == []
