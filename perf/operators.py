"""The attention half of a decode step, operator by operator, as cases that can be timed and checked.

A MoE block's step over a paged cache needs, next to the expert layers: the
norm with the residual (its output in 8 bits where a projection with 4-bit
weights reads it), the page tables and slot maps of the step's new tokens, the
heads' norm and rotation with the write into the cache, the attention of one
new token a sequence over its pages, and the projections themselves.  Each is
here in its plain form (elementary torch operations in 32 bits) and, with
``own``, as a call of ``paper_2609_38823_amd.block_abi``.

Sizes are those of the repository's workloads (the Qwen3-VL-MoE layer: d 2048,
32 query heads and 4 key/value heads of 128; the decode step of 64 sequences;
prefills of 4096 and 8192 rows) and generic ones.  8-bit values are e4m3 with
one power-of-two scale (e8m0) for every 32 along a row; 4-bit weights are e2m1
with the same scales.
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
BLOCK = 32
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HEADS = dict(n_q=32, n_kv=4, D=128)
#: the values of the 16 e2m1 codes
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def listed():
    return [
        # the norm before the attention of one user's next token, read by a projection in 8 bits
        dict(name="norm_1", op="norm", T=1, d=2048, dt="bf16", residual=True, out="mx"),
        # the norms of a prefill: the residual's sum, the rows and their 8-bit form
        dict(name="norm_4096", op="norm", T=4096, d=2048, dt="bf16", residual=True, out="both"),
        # one step of 64 sequences: a token each
        dict(name="extend_64", op="extend", n_seq=64, page=16, max_pages=512, longest=8000, most_new=1, release=0.0),
        # a mixed batch: prompts in part, single tokens, finished requests that give their pages back
        dict(name="extend_mixed_256", op="extend", n_seq=256, page=16, max_pages=640, longest=8000, most_new=2000,
             release=0.1),
        # a decode step's rows into an 8-bit cache
        dict(name="qkv_64", op="qkv", T=64, dt="bf16", cache="mx", page=16, norm=True, rot=128, far=8192, **HEADS),
        # a prompt's rows into a 16-bit cache
        dict(name="qkv_8192", op="qkv", T=8192, dt="bf16", cache="bf16", page=64, norm=True, rot=128, far=8192,
             **HEADS),
        # one short conversation
        dict(name="attn_1_short", op="attn", n_seq=1, longest=515, shortest=515, page=16, dt="bf16", cache="bf16",
             **HEADS),
        # a decode step of 64 sequences of all lengths
        dict(name="attn_64", op="attn", n_seq=64, longest=8192, shortest=1, page=16, dt="bf16", cache="bf16",
             **HEADS),
        # one long document, 8-bit cache
        dict(name="attn_1_long", op="attn", n_seq=1, longest=131072, shortest=131072, page=64, dt="bf16", cache="mx",
             **HEADS),
        # a small float32 model with a key/value head for every query head
        dict(name="attn_f32_7", op="attn", n_seq=7, longest=1000, shortest=0, page=8, dt="f32", cache="f32", n_q=8,
             n_kv=8, D=64),
        # the projection to queries, keys and values of one token, rows in 8 bits
        dict(name="linear_1", op="linear", T=1, n=5120, k=2048, x="mx"),
        # a large projection over a ragged step
        dict(name="linear_37", op="linear", T=37, n=8192, k=8192, x="bf16"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("norm", "extend", "qkv", "attn", "attn", "linear"))
    if op == "norm":
        d = log(64, 8192)
        d -= rng.choice((0, d % 32, d % 32, d % 256 if d > 256 else 0))
        return dict(op=op, T=max(1, min(log(1, 4096), 8192 * 1024 // d)), d=d, dt=rng.choice(("bf16", "bf16", "f32")),
                    residual=rng.random() < 0.75, out=rng.choice(("same", "mx", "both")))
    if op == "extend":
        page = rng.choice((1, 8, 16, 32, 64, 100))
        longest = log(16, 4000)
        most = rng.choice((1, 1, log(2, 2000)))
        return dict(op=op, n_seq=log(1, 256), page=page, max_pages=(longest + most) // page + 1, longest=longest,
                    most_new=most, release=rng.choice((0.0, 0.1)))
    D = rng.choice((32, 64, 96, 128, 128, 128, 192, 256))
    n_kv = rng.choice((1, 2, 4, 8))
    n_q = n_kv * rng.choice((1, 2, 4, 5, 8, 16))
    page = rng.choice((1, 8, 16, 16, 32, 64, 100))
    dt, cache = rng.choice((("bf16", "bf16"), ("bf16", "mx"), ("f32", "f32")))
    if op == "qkv":
        most = max(1, 8192 * 40 * 128 // ((n_q + 2 * n_kv) * D * (2 if dt == "f32" else 1)))
        return dict(op=op, T=log(1, min(8192, most)), dt=dt, cache=cache, page=page, norm=rng.random() < 0.5,
                    rot=rng.choice((0, D, D, D // 2)), far=log(100, 1000000), n_q=n_q, n_kv=n_kv, D=D)
    if op == "attn":
        n_seq = log(1, 128)
        # keys of all sequences, so that the cache takes at most 256 MB
        most = (1 << 28) // (2 * n_kv * D * {"bf16": 2, "mx": 1, "f32": 4}[cache])
        longest = log(1, max(2, min(131072, most // n_seq)))
        return dict(op=op, n_seq=n_seq, longest=longest, shortest=rng.choice((0, 1, longest)), page=page, dt=dt,
                    cache=cache, n_q=n_q, n_kv=n_kv, D=D)
    return dict(op=op, T=log(1, 64), n=log(100, 8192), k=32 * log(4, 256), x=rng.choice(("bf16", "mx", "mx", "f32")))


# --------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, shape, dt=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dt)


def _codes8(v):
    """e4m3 codes and e8m0 scales of random values [..., cols]: inputs only."""
    cols = v.shape[-1]
    m, e = torch.frexp(v.unflatten(-1, (cols // BLOCK, BLOCK)).abs().amax(-1))
    e = torch.where(m > 0.875, e - 8, e - 9)
    q = torch.ldexp(v, -e.repeat_interleave(BLOCK, -1)).to(torch.float8_e4m3fn)
    return q, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _lengths(g, n, lo, hi):
    return torch.randint(lo, hi + 1, (n,), generator=g, device=DEV, dtype=torch.int32)


def prepare(case, seed):
    c, g = case, _gen(seed)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    s = dict(case=c)
    if c["op"] == "norm":
        dt = DT[c["dt"]]
        T, d = c["T"], c["d"]
        s.update(x=_normal(g, (T, d), dt), r=_normal(g, (T, d), dt, 3.0) if c["residual"] else None,
                 w=1.0 + _normal(g, (d,), std=0.1))
        s["h"] = torch.empty((T, d), dtype=dt, device=DEV) if c["residual"] else None
        s["y"] = torch.empty((T, d), dtype=dt, device=DEV) if c["out"] != "mx" else None
        mx = c["out"] != "same"
        s["q"] = torch.empty((T, d), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) if mx else None
        s["qs"] = (torch.empty((T, -(-d // BLOCK)), dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
                   if mx else None)
    elif c["op"] == "extend":
        n, page, width = c["n_seq"], c["page"], c["max_pages"]
        lens = _lengths(g, n, 0, c["longest"])
        add = _lengths(g, n, 1, c["most_new"])
        add = torch.where(torch.rand(n, generator=g, device=DEV) < c["release"], -1, add).int()
        n_pages = n * width
        order = torch.randperm(n_pages, generator=g, device=DEV).int()
        have = (lens + page - 1) // page
        table = order.view(n, width)
        held = torch.arange(width, device=DEV)[None, :] < have[:, None]
        # the pages that no sequence holds, in some order, and what lies behind them
        free = table.reshape(-1)[torch.argsort(held.reshape(-1).int(), stable=True)].contiguous()
        rows = n * c["most_new"]
        s.update(lens=lens, add=add, table=torch.where(held, table, -1).int().contiguous(), free=free,
                 n_free=(~held).sum().int().view(1), len_out=i32(n), n_free_out=i32(1), offsets=i32(n + 1),
                 slots=i32(rows), positions=i32(rows), accepted=i32(n), status=i32(4))
    elif c["op"] == "qkv":
        dt = DT[c["dt"]]
        T, n_q, n_kv, D, page = c["T"], c["n_q"], c["n_kv"], c["D"], c["page"]
        n_pages = -(-T // page) + 8
        s.update(qkv=_normal(g, (T, (n_q + 2 * n_kv) * D), dt),
                 positions=torch.randint(0, c["far"], (T,), generator=g, device=DEV, dtype=torch.int32),
                 slots=torch.randperm(n_pages * page, generator=g, device=DEV)[:T].int(),
                 q=torch.empty((T, n_q, D), dtype=dt, device=DEV))
        rot = c["rot"]
        s["inv_freq"] = (1e6 ** (-torch.arange(0, rot, 2, device=DEV).double() / rot)).float() if rot else None
        s["q_norm"] = 1.0 + _normal(g, (D,), std=0.1) if c["norm"] else None
        s["k_norm"] = 1.0 + _normal(g, (D,), std=0.1) if c["norm"] else None
        shape = (n_pages, n_kv, page, D)
        s.update(k=torch.zeros(shape, dtype=dt, device=DEV), v=torch.zeros(shape, dtype=dt, device=DEV), ks=None,
                 vs=None)
        if c["cache"] == "mx":
            s["k"], s["ks"] = _codes8(_normal(g, shape))
            s["v"], s["vs"] = _codes8(_normal(g, shape))
    elif c["op"] == "attn":
        dt = DT[c["dt"]]
        n, n_q, n_kv, D, page = c["n_seq"], c["n_q"], c["n_kv"], c["D"], c["page"]
        lens = _lengths(g, n, c["shortest"], c["longest"])
        lens[0] = c["longest"]
        width = -(-c["longest"] // page)
        n_pages = n * width
        s.update(lens=lens, table=torch.randperm(n_pages, generator=g, device=DEV).int().view(n, width),
                 q=_normal(g, (n, n_q, D), dt), out=torch.empty((n, n_q, D), dtype=dt, device=DEV), ks=None, vs=None)
        shape = (n_pages, n_kv, page, D)
        if c["cache"] == "mx":
            s["k"], s["ks"] = _codes8(_normal(g, shape))
            s["v"], s["vs"] = _codes8(_normal(g, shape))
        else:
            s["k"], s["v"] = _normal(g, shape, dt), _normal(g, shape, dt)
        if own:
            from paper_2609_38823_amd import block_abi
            s["ws"] = torch.empty(block_abi.blk_attn_workspace_size(n, n_q, n_kv, D, width * page),
                                  dtype=torch.uint8, device=DEV)
    else:
        T, n, k = c["T"], c["n"], c["k"]
        x = _normal(g, (T, k))
        s["xs"] = None
        if c["x"] == "mx":
            s["x"], s["xs"] = _codes8(x)
        else:
            s["x"] = x.to(DT[c["x"]])
        s["codes"] = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
        # weights of about 0.02: scales of 2^-8 to 2^-6
        s["scales"] = torch.randint(119, 122, (n, k // BLOCK), generator=g, device=DEV,
                                    dtype=torch.uint8).view(torch.float8_e8m0fnu)
        s["y"] = torch.empty((T, n), dtype=torch.float32 if c["x"] == "f32" else torch.bfloat16, device=DEV)
    return s


# ----------------------------------------------------------- the plain forms
def _mx(v):
    """e4m3 values and power-of-two scales of v [..., cols], a scale for every 32 columns: the smallest
    2^E with max |v| <= 448 2^E."""
    cols = v.shape[-1]
    nb = -(-cols // BLOCK)
    b = torch.nn.functional.pad(v, (0, nb * BLOCK - cols)).unflatten(-1, (nb, BLOCK))
    m, e = torch.frexp(b.abs().amax(-1))
    e = torch.where(m == 0, -127, torch.where(m > 0.875, e - 8, e - 9)).clamp(min=-127)
    q = torch.ldexp(b, -e[..., None]).flatten(-2)[..., :cols].contiguous().to(torch.float8_e4m3fn)
    return q, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _of_mx(q, s):
    return q.float() * s.float().repeat_interleave(BLOCK, -1)[..., : q.shape[-1]]


def _norm(s):
    x, r = s["x"], s["r"]
    h = x.float() if r is None else x.float() + r.float()
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["w"]
    got = {}
    if r is not None:
        got["h"] = h.to(x.dtype)
    if s["y"] is not None:
        got["y"] = y.to(x.dtype)
    if s["q"] is not None:
        got["q"], got["scale"] = _mx(y)
    return got


def _extend(s):
    lens, add, table, free = s["lens"], s["add"], s["table"], s["free"]
    page, (n, width), rows, n_pages = s["case"]["page"], table.shape, s["slots"].numel(), free.numel()
    have = (lens + page - 1) // page
    gone = add < 0
    new = add.clamp(min=0)
    offsets = torch.cat([new.new_zeros(1), new.cumsum(0).int()]).clamp(max=rows)
    # pages that are given back go on top of the stack of free ones, in sequence order
    j = torch.arange(width, device=DEV)[None, :]
    back = torch.where(gone, have, 0)
    at = s["n_free"] + (back.cumsum(0) - back)[:, None] + j
    at = torch.where(gone[:, None] & (j < have[:, None]) & (at < n_pages), at, n_pages)
    stack = torch.cat([free, free.new_zeros(1)])
    stack[at.reshape(-1)] = table.reshape(-1)
    stack = stack[:n_pages].contiguous()
    top = (s["n_free"] + back.sum()).clamp(max=n_pages)
    # and pages are taken from its top, in sequence order, while they last
    pages = (lens + new + page - 1) // page
    fits = (pages <= width) & (new.cumsum(0) <= rows)
    need = torch.where(fits & ~gone, pages - have, 0)
    upto = need.cumsum(0)
    served = fits & ~gone & ((need == 0) | (upto <= top))
    taken = torch.where(served, need, 0)
    k = j - have[:, None]
    fresh = (k >= 0) & (k < taken[:, None])
    at = (top - 1 - ((upto - need)[:, None] + k)).clamp(0, n_pages - 1)
    table = torch.where(fresh, stack[at], table)
    row = torch.arange(rows, device=DEV, dtype=torch.int32)
    q = torch.searchsorted(offsets[1:].contiguous(), row, right=True).clamp(max=n - 1)
    pos = lens[q] + row - offsets[q]
    valid = served[q] & (row < offsets[-1])
    slot = table[q, (pos // page).clamp(0, width - 1)] * page + pos % page
    status = torch.stack([offsets[-1], taken.sum().int(), (~served & ~gone).sum().int(), (top - s["n_free"])[0].int()])
    return dict(lens=torch.where(gone, 0, torch.where(served, lens + new, lens)).int(),
                n_free=(top - taken.sum()).int(), table=table.int(), free=stack, offsets=offsets.int(),
                slots=torch.where(valid, slot, -1).int(), positions=torch.where(valid, pos, 0).int(),
                accepted=(served | gone).int(), status=status.int())


def _heads(v, w):
    return v if w is None else v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * w


def _rotate(v, cos, sin):
    half = cos.shape[-1]
    a, b = v[..., :half], v[..., half: 2 * half]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, v[..., 2 * half:]], -1)


def _qkv(s):
    c = s["case"]
    n_q, n_kv, D, page = c["n_q"], c["n_kv"], c["D"], c["page"]
    q, k, v = s["qkv"].float().view(-1, n_q + 2 * n_kv, D).split((n_q, n_kv, n_kv), 1)
    q, k = _heads(q, s["q_norm"]), _heads(k, s["k_norm"])
    if s["inv_freq"] is not None:
        a = s["positions"].double()[:, None, None] * s["inv_freq"].double()  # far positions: 64 bits
        cos, sin = a.cos().float(), a.sin().float()
        q, k = _rotate(q, cos, sin), _rotate(k, cos, sin)
    at, off = (s["slots"] // page).long(), (s["slots"] % page).long()
    got = dict(q=q.to(s["q"].dtype), k=s["k"], v=s["v"])
    if s["ks"] is None:
        s["k"][at, :, off] = k.to(s["k"].dtype)
        s["v"][at, :, off] = v.to(s["v"].dtype)
        return got
    for name, rows in (("k", k), ("v", v)):
        codes, scale = _mx(rows)
        s[name].view(torch.uint8)[at, :, off] = codes.view(torch.uint8)
        s[name + "s"].view(torch.uint8)[at, :, off] = scale.view(torch.uint8)
    return dict(got, ks=s["ks"], vs=s["vs"])


def _attn(s):
    c = s["case"]
    n, n_q, n_kv, D = c["n_seq"], c["n_q"], c["n_kv"], c["D"]

    def rows(cache, scale):  # [n, n_kv, keys, D]
        t = s["table"].long()
        v = cache[t].float() if scale is None else _of_mx(cache.view(torch.uint8)[t].view(cache.dtype),
                                                          scale.view(torch.uint8)[t].view(scale.dtype))
        return v.transpose(1, 2).reshape(n, n_kv, -1, D)

    k, v = rows(s["k"], s["ks"]), rows(s["v"], s["vs"])
    there = (torch.arange(k.shape[2], device=DEV)[None, :] < s["lens"][:, None])[:, None, None, :]
    q = s["q"].float().view(n, n_kv, n_q // n_kv, D)
    a = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(D))
    a = torch.where(there, a, -math.inf)
    top = a.amax(-1, keepdim=True)
    p = torch.exp(a - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, torch.where(there.transpose(2, 3), v, 0.0)) / torch.where(total == 0, 1.0, total)
    return dict(out=o.reshape(n, n_q, D).to(s["out"].dtype))


def _weights(codes, scales):
    table = torch.tensor(E2M1, device=DEV)
    v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1).flatten(-2)
    return v * scales.float().repeat_interleave(BLOCK, -1)


def _linear(s):
    x = s["x"].float() if s["xs"] is None else _of_mx(s["x"], s["xs"])
    return dict(y=torch.matmul(x, _weights(s["codes"], s["scales"]).t()).to(s["y"].dtype))


PLAIN = dict(norm=_norm, extend=_extend, qkv=_qkv, attn=_attn, linear=_linear)


# ---------------------------------------------------- the framework's calls
def _own(s):
    from paper_2609_38823_amd import block_abi as B
    c = s["case"]
    if c["op"] == "norm":
        B.blk_rms_norm(s["x"], s["w"], EPS, residual=s["r"], h_out=s["h"], y=s["y"], q=s["q"], q_scale=s["qs"])
        got = dict(h=s["h"], y=s["y"], q=s["q"], scale=s["qs"])
        return {k: v for k, v in got.items() if v is not None}
    if c["op"] == "extend":
        B.blk_kv_extend(s["lens"], s["add"], s["n_free"], s["table"], s["free"], c["page"], s["len_out"],
                        s["n_free_out"], s["offsets"], s["slots"], s["positions"], s["accepted"], s["status"])
        return dict(lens=s["len_out"], n_free=s["n_free_out"], table=s["table"], free=s["free"],
                    offsets=s["offsets"], slots=s["slots"], positions=s["positions"], accepted=s["accepted"],
                    status=s["status"])
    if c["op"] == "qkv":
        B.blk_qkv_cache(s["qkv"], c["n_q"], s["slots"], s["k"], s["v"], s["q"], positions=s["positions"],
                        inv_freq=s["inv_freq"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, k_scale=s["ks"],
                        v_scale=s["vs"])
        got = dict(q=s["q"], k=s["k"], v=s["v"], ks=s["ks"], vs=s["vs"])
        return {k: v for k, v in got.items() if v is not None}
    if c["op"] == "attn":
        B.blk_attn_decode(s["q"], s["k"], s["v"], s["table"], s["lens"], 1.0 / math.sqrt(c["D"]), s["out"], s["ws"],
                          k_scale=s["ks"], v_scale=s["vs"])
        return dict(out=s["out"])
    B.blk_linear_w4(s["x"], s["codes"], s["scales"], s["y"], x_scale=s["xs"])
    return dict(y=s["y"])


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------ the work
def work(case):
    c = case
    size = {"bf16": 2.0, "f32": 4.0, "mx": 1.0 + 1.0 / BLOCK}
    if c["op"] == "norm":
        per = size[c["dt"]] * (1 + 2 * c["residual"])
        per += size[c["dt"]] * (c["out"] != "mx") + size["mx"] * (c["out"] != "same")
        return dict(bytes=c["T"] * c["d"] * per + 4 * c["d"], flops=6 * c["T"] * c["d"])
    if c["op"] == "extend":
        n, new = c["n_seq"], (1 + c["most_new"]) / 2 * (1 - c["release"])
        moved = n * (new + c["release"] * c["longest"] / 2) / c["page"]
        return dict(bytes=20 * n + 8 * n * c["most_new"] + 8 * moved, flops=0)
    if c["op"] == "qkv":
        q, kv = c["T"] * c["n_q"] * c["D"], 2 * c["T"] * c["n_kv"] * c["D"]
        return dict(bytes=size[c["dt"]] * (2 * q + kv) + size[c["cache"]] * kv + 8 * c["T"], flops=9 * (q + kv))
    if c["op"] == "attn":
        n, q = c["n_seq"], c["n_seq"] * c["n_q"] * c["D"]
        keys = c["longest"] + (n - 1) * (c["longest"] + c["shortest"]) / 2  # on average over the seeds
        return dict(bytes=2 * keys * c["n_kv"] * c["D"] * size[c["cache"]] + 2 * q * size[c["dt"]]
                    + 4 * keys / c["page"], flops=4 * keys * c["n_q"] * c["D"])
    T, n, k = c["T"], c["n"], c["k"]
    return dict(bytes=n * k * (0.5 + 1.0 / BLOCK) + T * k * size[c["x"]] + T * n * (4 if c["x"] == "f32" else 2),
                flops=2.0 * T * n * k)


# ------------------------------------------------- the definitions in 64 bits
def _exact_mx(v):
    """The e4m3 values and the scales of v in 64 bits: steps of 2^max(e, -6) / 8 for values in [2^e, 2^(e+1))."""
    cols = v.shape[-1]
    short = -cols % BLOCK
    whole = torch.cat([v, v.new_zeros(v.shape[:-1] + (short,))], -1).reshape(v.shape[:-1] + (-1, BLOCK))
    most = whole.abs().max(-1).values
    E = torch.ceil(torch.log2(torch.where(most > 0, most, 2.0 ** -200) / 448.0))
    E = torch.where(most > 448.0 * 2.0 ** E, E + 1, E)  # the logarithm may be off by its rounding
    E = torch.where(most <= 448.0 * 2.0 ** (E - 1), E - 1, E).clamp(min=-127)
    u = (whole / 2.0 ** E[..., None]).reshape(v.shape[:-1] + (-1,))[..., :cols]
    step = 2.0 ** (torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(u / step) * step, 2.0 ** E


def exact(case, seed):
    if case["op"] == "extend":
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f64 = lambda t: t.to(torch.float64)  # noqa: E731
    c, got = case, {}
    if c["op"] == "norm":
        h = f64(s["x"]) if s["r"] is None else f64(s["x"]) + f64(s["r"])
        y = h / torch.sqrt(h.square().sum(-1, keepdim=True) / c["d"] + EPS) * f64(s["w"])
        if s["r"] is not None:
            got["h"] = h
        if c["out"] != "mx":
            got["y"] = y
        if c["out"] != "same":
            got["q"], got["scale"] = _exact_mx(y)
        return got
    if c["op"] == "qkv":
        n_q, n_kv, D, rot = c["n_q"], c["n_kv"], c["D"], c["rot"]
        rows = f64(s["qkv"]).view(c["T"], n_q + 2 * n_kv, D)
        parts = []
        for lo, hi, w in ((0, n_q, s["q_norm"]), (n_q, n_q + n_kv, s["k_norm"])):
            p = rows[:, lo:hi].clone()
            if w is not None:
                p = p / torch.sqrt(p.square().sum(-1, keepdim=True) / D + EPS) * f64(w)
            if rot:
                turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                                   f64(s["positions"])[:, None, None] * f64(s["inv_freq"]))
                z = torch.complex(p[..., : rot // 2].contiguous(), p[..., rot // 2: rot].contiguous()) * turn
                p = torch.cat([z.real, z.imag, p[..., rot:]], -1)
            parts.append(p)
        parts.append(rows[:, n_q + n_kv:])
        got["q"] = parts[0]
        at, off = (s["slots"] // c["page"]).long(), (s["slots"] % c["page"]).long()
        for name, part in (("k", parts[1]), ("v", parts[2])):
            got[name] = f64(s[name])
            if c["cache"] == "mx":
                got[name + "s"] = f64(s[name + "s"])
                part, scale = _exact_mx(part)
                got[name + "s"][at, :, off] = scale
            got[name][at, :, off] = part
        return got
    if c["op"] == "attn":
        out = torch.zeros((c["n_seq"], c["n_q"], c["D"]), dtype=torch.float64, device=DEV)
        group = c["n_q"] // c["n_kv"]
        for i, length in enumerate(s["lens"].tolist()):
            if length == 0:
                continue
            pages = s["table"][i, : -(-length // c["page"])].long()

            def keys(cache, scale):
                v = f64(cache.view(torch.uint8)[pages].view(cache.dtype)) if scale is not None else f64(cache[pages])
                if scale is not None:
                    v = v * f64(scale.view(torch.uint8)[pages].view(scale.dtype)).repeat_interleave(BLOCK, -1)
                return v.permute(1, 0, 2, 3).reshape(c["n_kv"], -1, c["D"])[:, :length]

            k, v = keys(s["k"], s["ks"]), keys(s["v"], s["vs"])
            for h in range(c["n_kv"]):
                a = f64(s["q"][i, h * group:(h + 1) * group]) @ k[h].t().contiguous() / math.sqrt(c["D"])
                out[i, h * group:(h + 1) * group] = torch.softmax(a, -1) @ v[h]
        return dict(out=out)
    w = torch.empty((c["n"], c["k"]), dtype=torch.float64, device=DEV)
    values = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
    w[:, 0::2] = values[(s["codes"] % 16).long()]
    w[:, 1::2] = values[(s["codes"] // 16).long()]
    w = (w.view(c["n"], -1, BLOCK) * f64(s["scales"])[..., None]).view(c["n"], c["k"])
    x = f64(s["x"])
    if s["xs"] is not None:
        x = (x.view(c["T"], -1, BLOCK) * f64(s["xs"])[..., None]).view(c["T"], c["k"])
    return dict(y=x @ w.t().contiguous())
