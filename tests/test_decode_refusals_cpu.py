"""What a decode step of whole blocks refuses, before anything advances."""

import pytest
import torch

from paper_2609_38823_amd import attention, inputs as I
from paper_2609_38823_amd.attention import PagedCache
from paper_2609_38823_amd.stack import MoEStack

HEADS = I.AttentionShape(n_q=8, n_kv=2, D=64)


@pytest.fixture
def stack(monkeypatch):
    def ran(*_, **__):
        raise AssertionError("a call ran")

    for name in ("blk_kv_extend", "blk_rms_norm", "blk_attn_workspace_size"):
        monkeypatch.setattr(attention.B, name, ran)
    s = MoEStack.__new__(MoEStack)
    s.sh, s.dt, s.device, s.L = I.WORKLOADS["small_stack_bf16"].shape, torch.bfloat16, "cpu", 2
    s.layers, s._bufs, s._h = [], {}, {}
    return s


def test_without_attention_sublayers(stack):
    with pytest.raises(ValueError, match="add_attention"):
        stack.new_cache(3, 16)
    cache = PagedCache(3, 2, HEADS, 16, device="cpu")
    x = torch.zeros((3, stack.sh.d), dtype=torch.bfloat16)
    for call in (stack.forward_decode_blocks, stack.capture_decode_blocks):
        with pytest.raises(ValueError, match="add_attention"):
            call(x, 0.85, cache)
    with pytest.raises(ValueError, match="add_attention"):
        stack.attention_buffers(cache)


def test_a_cache_of_another_stack(stack):
    stack.attn, stack.attention = HEADS, [None, None]
    x = torch.zeros((3, stack.sh.d), dtype=torch.bfloat16)
    assert stack.new_cache(3, 16).layers == 2
    for cache in (PagedCache(3, 1, HEADS, 16, device="cpu"), PagedCache(3, 3, HEADS, 16, device="cpu"),
                  PagedCache(3, 2, I.AttentionShape(n_q=8, n_kv=4, D=64), 16, device="cpu"),
                  PagedCache(3, 2, I.AttentionShape(n_q=8, n_kv=2, D=32), 16, device="cpu"),
                  PagedCache(3, 2, HEADS, 16, dtype=torch.float32, device="cpu")):
        for call in (stack.forward_decode_blocks, stack.capture_decode_blocks):
            with pytest.raises(ValueError, match="cache"):
                call(x, 0.85, cache)


@pytest.mark.parametrize("shape", [(2, None), (4, None), (3, 1), (3, 64), (1, None), (None,), (3, 1, None)])
def test_rows_of_another_shape(stack, shape):
    """Rows that torch would broadcast, too."""
    stack.attn, stack.attention = HEADS, [None, None]
    cache = stack.new_cache(3, 16)
    x = torch.zeros([stack.sh.d if n is None else n for n in shape], dtype=torch.bfloat16)
    for call in (stack.forward_decode_blocks, stack.capture_decode_blocks):
        with pytest.raises(ValueError, match="rows"):
            call(x, 0.85, cache)


def test_sizes_of_a_cache():
    for kw in (dict(max_tokens=0), dict(page_size=0), dict(n_pages=0), dict(n_seq=0)):
        args = dict(n_seq=2, layers=1, attn=HEADS, max_tokens=16, page_size=16, device="cpu")
        args.update(kw)
        with pytest.raises(ValueError):
            PagedCache(**args)
    with pytest.raises(ValueError):
        PagedCache(2, 1, HEADS, 16, dtype=torch.float32, mx=True, device="cpu")


def test_heads_that_no_call_takes():
    """Refused where the layers are made, not at their first step."""
    for attn in (I.AttentionShape(n_q=8, n_kv=3, D=64), I.AttentionShape(n_q=8, n_kv=2, D=80),
                 I.AttentionShape(n_q=8, n_kv=2, D=160), I.AttentionShape(n_q=0, n_kv=1, D=64)):
        with pytest.raises(ValueError):
            attention.check_heads(attn)
    for D in (32, 64, 96, 128, 192, 256):
        attention.check_heads(I.AttentionShape(n_q=8, n_kv=2, D=D))


def test_sizes_that_a_later_call_would_refuse(monkeypatch):
    """A step's buffers and cache are refused where they are made: their calls
    come after the tables have advanced."""
    def buffers(T, d=256, attn=HEADS, keys=64):
        return attention.AttentionBuffers(T, d, attn, torch.bfloat16, keys, device="cpu")

    assert buffers(4096).ws.numel() > 0
    for args in (dict(T=4097), dict(T=2, d=250), dict(T=2, keys=(1 << 30) + 64)):
        with pytest.raises(ValueError):
            buffers(**args)
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: pytest.fail("memory before the refusal"))
    for kw in (dict(page_size=16, n_pages=1 << 27), dict(page_size=64, n_pages=1 << 25),
               dict(max_tokens=(1 << 30) + 1, n_pages=1)):
        args = dict(n_seq=1, layers=1, attn=I.AttentionShape(n_q=8, n_kv=4, D=32), max_tokens=16, device="meta")
        args.update(kw)
        with pytest.raises(ValueError):
            PagedCache(**args)
