"""Decode steps of whole blocks in which some places have no new token: eager
and captured, with a pool of pages that only the live places may use."""

import pytest
import torch

from _util import ensure_built
from oracle import block as O

pytestmark = pytest.mark.gpu

from paper_2609_38823_amd import inputs as I  # noqa: E402
from paper_2609_38823_amd.stack import MoEStack  # noqa: E402
from test_gpu_block import attn_bound, host  # noqa: E402

HEADS = I.AttentionShape(n_q=8, n_kv=2, D=64)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()
    torch.cuda.init()


@pytest.fixture(scope="module", params=["small_stack_bf16", "tiny_stack_f32"])
def stack(request):
    s = MoEStack(I.WORKLOADS[request.param], n_layers=2, calib_rows=64)
    s.add_attention(HEADS)
    return s


def rows(stack, n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((n, stack.sh.d), generator=g, device="cuda").to(stack.dt)


def kinds(stack):
    return (False, True) if stack.sh.dtype == "bf16" else (False,)


def adds(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def test_a_released_place_stays_idle(stack):
    """A pool of pages for the live places alone: nobody is refused, the idle
    place takes nothing, eagerly and as replayed."""
    n = 4
    for mx in kinds(stack):
        eager, graphed = (stack.new_cache(n, 24, page_size=4, mx=mx, n_pages=13) for _ in range(2))
        x, add = rows(stack, n, 1), adds(1, 1, 1, 1)
        g, out = stack.capture_decode_blocks(x, 0.85, graphed, add=add)
        for step in range(16):
            if step == 3:  # place 1 ends in this step, and is idle from the next on
                add.copy_(adds(1, -1, 1, 1))
            elif step == 4:
                add.copy_(adds(1, 0, 1, 1))
            x.copy_(rows(stack, n, 10 + step))
            got = stack.forward_decode_blocks(x, 0.85, eager, add=add).clone()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, got), step
            for t, u in zip(eager.state(), graphed.state()):
                assert torch.equal(t, u)
            assert eager.accepted.tolist() == graphed.accepted.tolist() == [1] * n
            assert eager.lens.tolist() == [step + 1, min(step + 1, 3) if step < 3 else 0, step + 1, step + 1]
        assert eager.n_free.tolist() == [13 - 12]


def test_rows_go_to_their_own_places(stack):
    """Keys, values and attention of the places that have a token, with idle
    places between them, against the oracle."""
    n, a = 5, HEADS
    for mx in kinds(stack):
        cache = stack.new_cache(n, 24, page_size=4, mx=mx)
        for step, add in enumerate(((1, 1, 1, 1, 1), (0, 1, 0, 1, 1), (1, 0, 1, -1, 1), (0, 0, 1, 1, 0))):
            x = rows(stack, n, 40 + step)
            slots, positions = cache.step(adds(*add))
            h, b, lay = x.clone(), stack.attention_buffers(cache), stack.attention[0]
            before = [t.clone() for t in (cache.k[0], cache.v[0])]
            lay.forward(h, cache, 0, b, slots=slots, positions=positions)
            lens, table = cache.lens.tolist(), host(cache.table)
            vals = [(host(c) if s is None else O.dequantize_mx8(host(c), host(s)))
                    for c, s in ((cache.k[0], cache.k_scale[0]), (cache.v[0], cache.v_scale[0]))]
            written = [int(s) for s in slots.tolist() if s >= 0]
            assert len(written) == sum(v > 0 for v in add) and slots.tolist() == [
                int(table[s, (lens[s] - 1) // 4]) * 4 + (lens[s] - 1) % 4 if add[s] > 0 else -1 for s in range(n)]
            for t, u in zip((cache.k[0], cache.v[0]), before):  # nothing else was written
                flat = (t.view(torch.uint8) != u.view(torch.uint8)).any(-1).any(1).reshape(-1)
                assert set(flat.nonzero().flatten().tolist()) <= set(written)
            for s in range(n):
                k, v = (O.keys_of(c, table[s], lens[s], 4) for c in vals)
                q = host(b.q)[s]
                ref, w = O.attention(q, k, v, a.D ** -0.5)
                assert (abs(host(b.att)[s] - ref) <= attn_bound(q, k, v, w, ref, a.D ** -0.5, stack.sh.dtype, 4)).all()


def test_capture_leaves_the_cache_as_it_was(stack):
    """Everything of it: lengths, tables, free pages, what the last extension
    left, keys and values."""
    n = 3
    for mx in kinds(stack):
        for add in (None, adds(1, -1, 0)):
            cache = stack.new_cache(n, 24, page_size=4, mx=mx)
            for step in range(5):
                stack.forward_decode_blocks(rows(stack, n, step), 0.85, cache, add=adds(1, step % 2, 1))
            tensors = {k: t for k, t in vars(cache).items() if isinstance(t, torch.Tensor)}
            for name in ("k", "v", "k_scale", "v_scale"):
                tensors.update({(name, l): t for l, t in enumerate(getattr(cache, name)) if t is not None})
            assert len(tensors) >= 14
            torch.cuda.synchronize()
            before = {k: t.clone() for k, t in tensors.items()}
            stack.capture_decode_blocks(rows(stack, n, 9), 0.85, cache, add=add)
            torch.cuda.synchronize()
            for k, t in tensors.items():
                assert torch.equal(t.view(torch.uint8), before[k].view(torch.uint8)), k


def test_a_step_and_a_release_on_another_stream(stack):
    """A torch stream and a bare handle, against the current stream."""
    n, side = 3, torch.cuda.Stream()
    plain, on_side = (stack.new_cache(n, 24, page_size=4) for _ in range(2))
    torch.cuda.synchronize()
    for step in range(4):
        x = rows(stack, n, step)
        for stream in (side, side.cuda_stream):
            gone, add = torch.tensor([step % 2 == 0, False, step == 3], device="cuda"), adds(1, step % 2, 1)
            want = stack.forward_decode_blocks(x, 0.85, plain, add=add).clone()
            plain.release(gone)
            torch.cuda.synchronize()
            got = stack.forward_decode_blocks(x, 0.85, on_side, stream=stream, add=add)
            on_side.release(gone, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(got, want)
            for t, u in zip(plain.state() + plain.last(), on_side.state() + on_side.last()):
                assert torch.equal(t, u)
