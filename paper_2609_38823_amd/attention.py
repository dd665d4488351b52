"""The attention half of a decoder block in decode, composed from the calls of
``block_abi``: a paged key/value cache and a layer's attention sublayer.

Everything computed here runs in libdecomoe_block.so; this module only owns
device buffers and issues the calls in their order:

  once a step   blk_kv_extend         pages and slots of the new tokens
  per layer     blk_rms_norm          8-bit rows (bf16 layers)
                blk_linear_w4         queries, keys and values
                blk_qkv_cache         head norm, rotation, cache write
                blk_attn_decode
                blk_linear_w4         output projection
                blk_rms_norm          h <- h + output, and the rows of the MoE layer

All calls are asynchronous on one stream; lengths, tables and the stack of
free pages never leave the device.
"""

from __future__ import annotations

import contextlib

import torch

from . import block_abi as B
from . import inputs as I
from .layer import to_device


def on_stream(stream):
    """The context in which torch's own calls run on ``stream`` too (a torch
    stream or a handle; None: the current one)."""
    if stream is None:
        return contextlib.nullcontext()
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


def check_heads(attn: I.AttentionShape):
    """Heads that the calls of a step take."""
    if attn.n_q < 1 or attn.n_kv < 1 or attn.n_q % attn.n_kv or attn.D not in (32, 64, 96, 128, 192, 256):
        raise ValueError(f"{attn}: query heads in equal groups for the key/value heads, of 32, 64, 96, 128, 192 or 256")


class PagedCache:
    """Keys and values of ``n_seq`` sequences in ``layers`` layers, in pages of
    ``page_size`` tokens that the sequences share through one stack of free
    pages (one table for all layers).  ``mx``: 8-bit keys and values (bf16
    layers)."""

    def __init__(self, n_seq: int, layers: int, attn: I.AttentionShape, max_tokens: int, page_size: int = 16,
                 n_pages: int | None = None, dtype: torch.dtype = torch.bfloat16, mx: bool = False, device="cuda"):
        if mx and dtype != torch.bfloat16:
            raise ValueError("8-bit caches go with bf16 layers")
        if n_seq < 1 or max_tokens < 1 or page_size < 1 or (n_pages is not None and n_pages < 1):
            raise ValueError("a cache has sequences, tokens and pages")
        self.n_seq, self.layers, self.attn, self.dtype = n_seq, layers, attn, dtype
        self.page, self.mx = page_size, mx
        self.max_pages = -(-max_tokens // page_size)
        self.n_pages = n_seq * self.max_pages if n_pages is None else n_pages
        slots = self.n_pages * page_size  # the calls count them, and their rows, in 32 bits
        if slots > 2 ** 31 - 1 or slots * attn.n_kv >= 2 ** 32 - 1 or self.max_pages * page_size > 2 ** 30:
            raise ValueError(f"{self.n_pages} pages of {page_size} for up to {max_tokens} tokens: more than the calls take")
        shape = (self.n_pages, attn.n_kv, page_size, attn.D)
        store = torch.float8_e4m3fn if mx else dtype
        empty = lambda s, t: [torch.zeros(s, dtype=torch.uint8, device=device).view(t) if mx  # noqa: E731
                              else torch.zeros(s, dtype=t, device=device) for _ in range(layers)]
        self.k, self.v = empty(shape, store), empty(shape, store)
        scale = shape[:3] + (attn.D // B.BLOCK,)
        self.k_scale, self.v_scale = ([torch.zeros(scale, dtype=torch.uint8, device=device) for _ in range(layers)]
                                      if mx else [None] * layers for _ in range(2))
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)  # noqa: E731
        self.lens, self.n_free = i32(n_seq), torch.full((1,), self.n_pages, dtype=torch.int32, device=device)
        self.table = torch.full((n_seq, self.max_pages), -1, dtype=torch.int32, device=device)
        self.free = torch.arange(self.n_pages, dtype=torch.int32, device=device)
        # of the last extension
        self.row_offsets, self.slots, self.positions = i32(n_seq + 1), i32(n_seq), i32(n_seq)
        self.accepted, self.status = i32(n_seq), i32(4)
        self.ones = torch.ones((n_seq,), dtype=torch.int32, device=device)
        self.none = torch.full((n_seq,), -1, dtype=torch.int32, device=device)

    def extend(self, add=None, slots=None, positions=None, stream=None):
        """Room for ``add`` [n_seq] new tokens a sequence (default: one each;
        negative: the sequence is finished and its pages are free again).  The
        tables advance on the device; ``accepted`` and ``status`` say what was
        carried out.  slots, positions: arrays for more rows than sequences."""
        B.blk_kv_extend(self.lens, self.ones if add is None else add, self.n_free, self.table, self.free, self.page,
                        self.lens, self.n_free, self.row_offsets, self.slots if slots is None else slots,
                        self.positions if positions is None else positions, self.accepted, self.status, stream=stream)

    def step(self, add=None, stream=None):
        """Room for a decode step, whose row s is place s's one new token;
        returns its rows' (slots, positions).  add [n_seq] int32 on the device:
        a token where it is positive (one, whatever the number), none where it
        is 0 - an idle place keeps its length and takes no page -, and a
        negative one ends the sequence.  Default: a token each."""
        if add is None:
            self.extend(stream=stream)
            return self.slots, self.positions
        if not isinstance(add, torch.Tensor) or add.dtype != torch.int32:
            raise TypeError("add is an int32 tensor")
        if add.shape != self.ones.shape or add.device != self.ones.device:
            raise ValueError(f"add is {tuple(add.shape)} on {add.device}, expected ({self.n_seq},) on {self.ones.device}")
        with on_stream(stream):
            add = add.clamp(max=1)
            self.extend(add)
            # the extension's rows are those of the places with a token, one
            # behind the other: back to the places
            at, new = self.row_offsets[:-1].clamp(max=max(self.n_seq - 1, 0)), add > 0
            slots = torch.where(new, self.slots.index_select(0, at), self.none)
            return slots, self.positions.index_select(0, at) * new

    def release(self, finished, stream=None):
        """Give back the pages of the sequences where ``finished`` [n_seq]
        (bool) holds; their places start again at length 0."""
        with on_stream(stream):
            self.extend(-finished.to(self.lens.device).int())

    def state(self):
        """The tensors that an extension advances."""
        return self.lens, self.n_free, self.table, self.free

    def last(self):
        """The tensors that say what the last extension did."""
        return self.row_offsets, self.slots, self.positions, self.accepted, self.status


class AttentionBuffers:
    """Work buffers of one step of ``T`` sequences."""

    def __init__(self, T: int, d: int, attn: I.AttentionShape, dt: torch.dtype, max_keys: int, device="cuda"):
        ws = B.blk_attn_workspace_size(T, attn.n_q, attn.n_kv, attn.D, max_keys)
        if ws == 0 or d % B.BLOCK:
            raise ValueError(f"{T} rows of {d} over up to {max_keys} keys, {attn}: not taken")
        e = lambda *s: torch.empty(s, dtype=dt, device=device)  # noqa: E731
        u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device=device)  # noqa: E731
        self.x8 = self.x8_scale = self.x = None
        if dt == torch.bfloat16:
            self.x8, self.x8_scale = u8(T, d), u8(T, d // B.BLOCK)
        else:
            self.x = e(T, d)
        self.qkv = e(T, (attn.n_q + 2 * attn.n_kv) * attn.D)
        self.q, self.att = e(T, attn.n_q, attn.D), e(T, attn.n_q, attn.D)
        self.o, self.y = e(T, d), e(T, d)
        self.ws = u8(ws)


class AttentionLayer:
    """One layer's attention sublayer: norm weights in float32, projections in
    4 bits (quantised on the device when the layer is loaded)."""

    def __init__(self, params: dict, attn: I.AttentionShape, dtype: str, device="cuda"):
        check_heads(attn)
        self.attn = attn
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        f32 = lambda a: to_device(a, torch.float32, device)  # noqa: E731
        self.norm_in, self.norm_out = f32(params["norm_in"]), f32(params["norm_out"])
        self.q_norm, self.k_norm = f32(params["q_norm"]), f32(params["k_norm"])
        self.inv_freq = f32(attn.inv_freq())
        self.w_qkv, self.w_o = self._quantize(f32(params["w_qkv"])), self._quantize(f32(params["w_o"]))

    @staticmethod
    def _quantize(w: torch.Tensor):
        n, k = w.shape
        codes = torch.empty((n, k // 2), dtype=torch.uint8, device=w.device)
        scales = torch.empty((n, k // B.BLOCK), dtype=torch.uint8, device=w.device)
        B.blk_quantize_w4(w, codes, scales)
        return codes, scales

    def forward(self, h: torch.Tensor, cache: PagedCache, layer: int, b: AttentionBuffers, stream=None, slots=None,
                positions=None):
        """h [T, d] <- h + attention(norm(h)), in place, for the one new token
        of each sequence that cache.extend() has made room for (slots,
        positions: what cache.step() returned, where some places have none);
        returns the rows that the MoE layer reads (norm of the new h, b.y).
        A token's rotation position is its index in the cache."""
        a, s = self.attn, stream
        slots, positions = cache.slots if slots is None else slots, cache.positions if positions is None else positions
        B.blk_rms_norm(h, self.norm_in, a.eps, y=b.x, q=b.x8, q_scale=b.x8_scale, stream=s)
        B.blk_linear_w4(b.x if b.x8 is None else b.x8, *self.w_qkv, b.qkv, x_scale=b.x8_scale, stream=s)
        B.blk_qkv_cache(b.qkv, a.n_q, slots, cache.k[layer], cache.v[layer], b.q, positions=positions,
                        inv_freq=self.inv_freq, q_norm=self.q_norm, k_norm=self.k_norm, eps=a.eps,
                        k_scale=cache.k_scale[layer], v_scale=cache.v_scale[layer], stream=s)
        B.blk_attn_decode(b.q, cache.k[layer], cache.v[layer], cache.table, cache.lens, a.D ** -0.5, b.att, b.ws,
                          k_scale=cache.k_scale[layer], v_scale=cache.v_scale[layer], stream=s)
        B.blk_linear_w4(b.att.view(h.shape[0], -1), *self.w_o, b.o, stream=s)
        B.blk_rms_norm(b.o, self.norm_out, a.eps, residual=h, h_out=h, y=b.y, stream=s)
        return b.y


def random_layer(shape: I.LayerShape, attn: I.AttentionShape, seed: int, layer: int, device="cuda") -> AttentionLayer:
    """A layer of seeded random parameters (the workloads' recipe)."""
    return AttentionLayer(I.attention_params(shape, attn, seed, layer), attn, shape.dtype, device)


