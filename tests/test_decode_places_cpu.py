"""Decode steps in which some places have no new token: host logic, with the
page tables' call replaced by the oracle on CPU tensors."""

import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2609_38823_amd import attention, inputs as I
from paper_2609_38823_amd.attention import PagedCache

HEADS = I.AttentionShape(n_q=8, n_kv=2, D=64)


@pytest.fixture
def tables(monkeypatch):
    """blk_kv_extend on CPU tensors, by the oracle."""
    calls = []

    def extend(len_in, add, n_free_in, table, free, page, len_out, n_free_out, offsets, slots, positions, accepted,
               status, stream=None):
        calls.append(add.tolist())
        got = O.kv_extend(len_in.tolist(), add.tolist(), int(n_free_in), table.numpy(), free.numpy(), page, slots.numel())
        for name, t in dict(len_out=len_out, n_free_out=n_free_out, block_table=table, free_pages=free, row_offsets=offsets,
                            slot_map=slots, positions=positions, accepted=accepted, status=status).items():
            t.copy_(torch.from_numpy(np.asarray(got[name])))

    monkeypatch.setattr(attention.B, "blk_kv_extend", extend)
    return calls


def test_a_step_of_every_place_is_the_extension(tables):
    cache = PagedCache(3, 1, HEADS, 40, page_size=4, device="cpu")
    slots, positions = cache.step()
    assert slots is cache.slots and positions is cache.positions and tables == [[1, 1, 1]]
    assert positions.tolist() == [0, 0, 0] and cache.lens.tolist() == [1, 1, 1]


def test_slots_of_a_step_belong_to_their_places(tables):
    """Row s of a step is place s's, whatever the places before it do."""
    cache = PagedCache(5, 1, HEADS, 40, page_size=4, n_pages=12, device="cpu")
    for add in ([1, 1, 1, 1, 1], [0, 1, 0, 1, 1], [1, 0, 1, 1, 0], [-1, 1, 0, 0, 7], [0, 0, 0, 0, 0], [1, 0, 0, 0, 1],
                [0, -3, 1, 1, 0]):
        before = cache.lens.tolist()
        slots, positions = cache.step(torch.tensor(add, dtype=torch.int32))
        for s, a in enumerate(add):
            if a > 0:  # one token a step, whatever is asked for
                assert cache.lens[s] == before[s] + 1 and positions[s] == before[s]
                assert slots[s] == cache.table[s, before[s] // 4] * 4 + before[s] % 4
            else:
                assert cache.lens[s] == (0 if a < 0 else before[s])
                assert slots[s] == -1 and positions[s] == 0
        held = sum(-(-n // 4) for n in cache.lens.tolist())
        assert cache.n_free.tolist() == [12 - held]


def test_idle_places_take_no_pages(tables):
    cache = PagedCache(4, 1, HEADS, 40, page_size=4, n_pages=6, device="cpu")
    cache.step()
    cache.release(torch.tensor([False, True, False, True]))
    add = torch.tensor([1, 0, 1, 0], dtype=torch.int32)
    for _ in range(11):  # to three pages each: all there are
        cache.step(add)
        assert cache.accepted.tolist() == [1, 1, 1, 1]
    assert cache.lens.tolist() == [12, 0, 12, 0] and cache.n_free.tolist() == [0]
    slots, _ = cache.step(add)  # and none is left: refused, not written
    assert cache.accepted.tolist() == [0, 1, 0, 1] and slots.tolist() == [-1] * 4 and cache.lens.tolist() == [12, 0, 12, 0]


def test_add_is_checked_before_anything_runs(tables):
    cache = PagedCache(3, 1, HEADS, 40, page_size=4, device="cpu")
    for add in (torch.ones(2, dtype=torch.int32), torch.ones(3), torch.ones((3, 1), dtype=torch.int32), [1, 1, 1]):
        with pytest.raises((TypeError, ValueError)):
            cache.step(add)
    assert not tables


class Recorder:
    """Stands for torch.cuda.stream: which stream is current."""

    def __init__(self):
        self.now = []

    def __call__(self, stream):
        self.stream = stream
        return self

    def __enter__(self):
        self.now.append(self.stream)

    def __exit__(self, *_):
        self.now.pop()


class Handle:
    cuda_stream = 1234


def test_release_forms_its_request_on_its_stream(monkeypatch):
    """torch's own work on the argument and the tables' call: one stream."""
    current, seen = Recorder(), []
    monkeypatch.setattr(torch.cuda, "stream", current)
    monkeypatch.setattr(attention.B, "blk_kv_extend", lambda *a, stream=None: seen.append(
        ("extend", a[1].tolist(), stream or (current.now or [None])[-1])))

    class Finished:
        def to(self, device):
            seen.append(("to", (current.now or [None])[-1]))
            return torch.tensor([True, False])

    cache, s = PagedCache(2, 1, HEADS, 8, page_size=4, device="cpu"), Handle()
    cache.release(Finished(), stream=s)
    assert seen == [("to", s), ("extend", [-1, 0], s)]
    seen.clear()
    cache.release(Finished())
    assert seen == [("to", None), ("extend", [-1, 0], None)]


def test_step_makes_its_buffers_on_its_stream(monkeypatch):
    """Buffers of a step's first call are allocated on the stream that uses
    them (memory that torch takes back from another one may still be in use)."""
    from paper_2609_38823_amd.stack import MoEStack
    current, seen = Recorder(), []
    monkeypatch.setattr(torch.cuda, "stream", current)
    stack = MoEStack.__new__(MoEStack)
    stack.sh, stack.dt, stack.device, stack.L = I.WORKLOADS["small_stack_bf16"].shape, torch.bfloat16, "cpu", 0
    stack.attn, stack.attention, stack.layers, stack._bufs, stack._h = HEADS, [], [], {}, {}
    for name in ("hidden", "buffers", "attention_buffers"):
        monkeypatch.setattr(stack, name, lambda *a, name=name: (seen.append((name, (current.now or [None])[-1])),
                                                               torch.zeros((2, 256)))[1])
    cache, s = stack.new_cache(2, 8), Handle()
    monkeypatch.setattr(cache, "step", lambda add=None, stream=None: (seen.append(
        ("step", stream or (current.now or [None])[-1])), (None, None))[1])
    stack.forward_decode_blocks(torch.zeros((2, 256)), 0.85, cache, stream=s)
    assert len(seen) == 4 and {at for _, at in seen} == {s}
