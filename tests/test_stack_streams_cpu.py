"""A stack's spans on a given stream: torch's own copies, reads and
allocations run on it as the library's calls do."""

import torch

from paper_2609_38823_amd import abi, inputs as I
from paper_2609_38823_amd.stack import MoEStack


class Handle:
    cuda_stream = 1234


class Current:
    """Stands for torch.cuda.stream."""

    def __init__(self):
        self.now = [None]

    def __call__(self, stream):
        self.given = stream
        return self

    def __enter__(self):
        self.now.append(self.given)

    def __exit__(self, *_):
        self.now.pop()


class Layer:
    one_call, packed, w_r_packed = True, True, 1

    def __init__(self, note):
        self.forward_rcep_chained = lambda *a, **k: note("layer", k.get("stream"))
        self.forward_dense = self.forward_rcep = self.forward_rcep_chained


def make(monkeypatch):
    current, seen = Current(), []

    def note(name, stream=None):
        seen.append((name, stream or current.now[-1]))

    monkeypatch.setattr(torch.cuda, "stream", current)
    for name in ("moe_combine_residual", "moe_savb_gate", "drop_visual_block_if", "drop_visual_block"):
        monkeypatch.setattr(abi, name, lambda *a, name=name, stream=None, **k: note(name, stream))
    monkeypatch.setattr(abi, "moe_savb_workspace_size", lambda *a: 16)
    s = MoEStack.__new__(MoEStack)
    s.sh, s.dt, s.device, s.L = I.WORKLOADS["small_stack_bf16"].shape, torch.bfloat16, "cpu", 2
    s.layers, s._bufs, s._h, s.K_trace = [Layer(note), Layer(note)], {}, {}, torch.zeros((2, 4), dtype=torch.int32)

    class Buffers:
        y_perm = row_of_slot = w = None

    monkeypatch.setattr(s, "buffers", lambda T: (note("buffers"), Buffers())[1])
    real = s.hidden
    monkeypatch.setattr(s, "hidden", lambda *a: (note("hidden"), real(*a))[1])
    for name in ("copy_", "item"):
        f = getattr(torch.Tensor, name)
        monkeypatch.setattr(torch.Tensor, name, lambda self, *a, f=f, name=name: (note(name), f(self, *a))[1])
    return s, seen


def test_a_decode_step_of_chained_layers(monkeypatch):
    s, seen = make(monkeypatch)
    stream = Handle()
    s.forward_decode(torch.zeros((3, s.sh.d), dtype=torch.bfloat16), 0.85, stream=stream)
    assert {"copy_", "layer", "moe_combine_residual", "hidden", "buffers"} <= {n for n, _ in seen}
    assert {at for _, at in seen} == {stream}
    seen.clear()
    s.forward_decode(torch.zeros((3, s.sh.d), dtype=torch.bfloat16), 0.85)
    assert {at for _, at in seen} == {None}


def test_a_gated_prefill(monkeypatch):
    s, seen = make(monkeypatch)
    stream = Handle()
    gate = dict(w1=torch.zeros((8, 2)), b1=torch.zeros(8), w2=torch.zeros((2, 8)), b2=torch.zeros(2))
    s.forward_gated(torch.zeros((6, s.sh.d), dtype=torch.bfloat16), 2, 0.85, {0: gate, 1: gate}, 0.5, stream=stream)
    assert {"item", "moe_savb_gate", "layer"} <= {n for n, _ in seen}
    assert {at for _, at in seen} == {stream}
