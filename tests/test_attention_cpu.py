"""Host logic of the attention layers that needs no GPU."""

import torch

from paper_2609_38823_amd import inputs as I
from paper_2609_38823_amd.attention import PagedCache
from paper_2609_38823_amd.stack import MoEStack


def test_buffers_follow_the_heads():
    """A stack whose heads are replaced makes buffers of the new sizes and
    keeps the ones of heads that come back."""
    stack = MoEStack.__new__(MoEStack)
    stack.sh, stack.dt, stack.device, stack.L, stack._bufs = I.WORKLOADS["small_stack_bf16"].shape, torch.bfloat16, "cpu", 1, {}
    made = []
    for attn in (I.AttentionShape(n_q=8, n_kv=2, D=64), I.AttentionShape(n_q=4, n_kv=4, D=32),
                 I.AttentionShape(n_q=8, n_kv=2, D=64)):
        stack.attn = attn
        b = stack.attention_buffers(stack.new_cache(3, 16))
        assert b.q.shape == (3, attn.n_q, attn.D) and b.qkv.shape == (3, (attn.n_q + 2 * attn.n_kv) * attn.D)
        made.append(b)
    assert made[0] is made[2]


def test_cache_holds_whole_pages():
    cache = PagedCache(3, 2, I.AttentionShape(n_q=8, n_kv=2, D=64), 33, page_size=16, mx=True, device="cpu")
    assert cache.max_pages == 3 and cache.n_pages == 9 and len(cache.k) == 2
    assert cache.k[0].shape == (9, 2, 16, 64) and cache.k_scale[0].shape == (9, 2, 16, 2)
    assert cache.k[0].dtype == torch.float8_e4m3fn and cache.free.tolist() == list(range(9))
