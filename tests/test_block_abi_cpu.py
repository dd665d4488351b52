"""Contract checks of the block library that need no GPU: it loads, exports
what include/decomoe_block.h declares, and refuses invalid arguments on the
host before anything is launched (only refused calls and empty ones are made
here)."""

import ctypes
import os
import re
import shutil
import subprocess

import pytest

from _util import ROOT
from paper_2609_38823_amd import block_abi, build

HEADER = os.path.join(ROOT, "include", "decomoe_block.h")
EINVAL, EALIAS, EWORKSPACE, EUNSUPPORTED = -1, -2, -3, -5
F32, BF16, MX = 0, 1, 2
NULL = None
# fake, never dereferenced, 16-byte aligned addresses, 16 MB apart
P = [ctypes.c_void_p(0x1000000 * i) for i in range(1, 20)]
ODD = ctypes.c_void_p(0x1000008)
BIG = 1 << 40


def declared():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"^[A-Za-z_][\w\s\*]*?\b(blk_[a-z0-9_]*)\s*\(", src, flags=re.M)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(block_abi.LIB_PATH):
        build.build()
    return block_abi.load()


def test_exports_are_the_declared_functions(lib):
    assert declared() == sorted(block_abi.EXPORTS)
    for name in declared():
        assert hasattr(lib, name) and callable(getattr(block_abi, name))
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("nm not available")
    out = subprocess.run([nm, "-D", "--defined-only", block_abi.LIB_PATH], capture_output=True, text=True,
                         check=True).stdout
    syms = {ln.split()[-1] for ln in out.splitlines() if " T " in ln and not ln.split()[-1].startswith("_Z")}
    assert sorted(syms) == declared()


@pytest.mark.parametrize("src", build.block_sources(), ids=[os.path.basename(s) for s in build.block_sources()])
def test_device_code(src, tmp_path):
    """No packed-fp32 instruction, no scratch traffic."""
    out = tmp_path / "dev.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    res = subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-S", "-I", os.path.join(ROOT, "include"), src,
                          "-o", str(out)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    asm = out.read_text()
    assert not re.search(r"\bv_pk_(fma|mul|add)_f32\b", asm)
    assert not re.search(r"\bscratch_(load|store)", asm)


def norm(lib, x=P[0], dt=BF16, r=P[1], w=P[2], T=4, d=64, eps=1e-6, h=P[3], y=P[4], q=P[5], qs=P[6]):
    return lib.blk_rms_norm(x, dt, r, w, T, d, eps, h, y, q, qs, NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), EINVAL), (dict(T=-1), EINVAL), (dict(d=0), EINVAL), (dict(d=32769), EUNSUPPORTED), (dict(T=(1 << 30) + 1), EUNSUPPORTED),
    (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL),
    (dict(x=NULL), EINVAL), (dict(qs=NULL), EINVAL), (dict(q=NULL), EINVAL),
    (dict(h=NULL, y=NULL, q=NULL, qs=NULL), EINVAL), (dict(x=ODD), EINVAL), (dict(qs=ODD), EINVAL),
    (dict(y=P[2]), EALIAS), (dict(h=P[4]), EALIAS), (dict(q=P[0]), EALIAS), (dict(qs=P[1]), EALIAS),
    (dict(h=P[0], y=P[0]), EALIAS),
    (dict(h=ctypes.c_void_p(0x1000000 + 128)), EALIAS),  # a part of x, not x itself
    (dict(T=0, x=NULL, r=NULL, h=NULL, y=NULL, q=NULL, qs=NULL), 0),
])
def test_rms_norm_refusals(lib, kw, status):
    assert norm(lib, **kw) == status


def extend(lib, len_in=P[0], add=P[1], n=4, page=16, width=8, n_pages=64, rows=32, nf=P[2], table=P[3], free=P[4],
           len_out=P[5], nfo=P[6], off=P[7], slots=P[8], pos=P[9], acc=P[10], st=P[11]):
    return lib.blk_kv_extend(len_in, add, n, page, width, n_pages, rows, nf, table, free, len_out, nfo, off, slots,
                             pos, acc, st, NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), EINVAL), (dict(page=0), EINVAL), (dict(width=0), EINVAL), (dict(n_pages=0), EINVAL),
    (dict(rows=-1), EINVAL), (dict(n_pages=1 << 28), EUNSUPPORTED), (dict(width=1 << 28), EUNSUPPORTED),
    (dict(page=1, n=1 << 20, width=1 << 12), EUNSUPPORTED), (dict(rows=(1 << 30) + 1), EUNSUPPORTED), (dict(add=NULL), EINVAL), (dict(table=NULL), EINVAL),
    (dict(acc=NULL), EINVAL), (dict(slots=NULL), EINVAL), (dict(st=NULL), EINVAL), (dict(off=ODD), EINVAL),
    (dict(len_out=P[1]), EALIAS), (dict(pos=P[8]), EALIAS), (dict(nfo=P[0]), EALIAS), (dict(acc=P[5]), EALIAS),
    (dict(len_out=ctypes.c_void_p(0x1000000 + 8), n=1), EINVAL),
])
def test_kv_extend_refusals(lib, kw, status):
    assert extend(lib, **kw) == status


def qkv(lib, x=P[0], dt=BF16, T=4, n_q=8, n_kv=2, D=64, qn=P[1], kn=P[2], eps=1e-6, pos=P[3], freq=P[4], rot=64,
        slots=P[5], cdt=BF16, n_pages=16, page=8, q=P[6], k=P[7], v=P[8], ks=NULL, vs=NULL):
    return lib.blk_qkv_cache(x, dt, T, n_q, n_kv, D, qn, kn, eps, pos, freq, rot, slots, cdt, n_pages, page, q, k, v,
                             ks, vs, NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), EINVAL), (dict(n_q=0), EINVAL), (dict(n_kv=0), EINVAL), (dict(rot=-16), EINVAL),
    (dict(rot=80), EINVAL), (dict(rot=40), EUNSUPPORTED), (dict(D=48, rot=0), EUNSUPPORTED),
    (dict(D=288, rot=0), EUNSUPPORTED), (dict(eps=-1.0), EINVAL), (dict(n_pages=0), EINVAL), (dict(page=0), EINVAL),
    (dict(n_pages=1 << 30), EUNSUPPORTED), (dict(cdt=F32), EINVAL), (dict(cdt=3), EINVAL),
    (dict(dt=F32, cdt=MX, ks=P[9], vs=P[10]), EUNSUPPORTED), (dict(cdt=MX), EINVAL), (dict(cdt=MX, ks=P[9]), EINVAL),
    (dict(ks=P[9], vs=P[10]), EINVAL), (dict(freq=NULL), EINVAL), (dict(pos=NULL), EINVAL), (dict(slots=NULL), EINVAL),
    (dict(k=NULL), EINVAL), (dict(q=ODD), EINVAL), (dict(k=P[8]), EALIAS), (dict(q=P[0]), EALIAS),
    (dict(v=P[5]), EALIAS), (dict(cdt=MX, ks=P[9], vs=P[9]), EALIAS),
    (dict(T=0, x=NULL, slots=NULL, q=NULL, pos=NULL), 0),
])
def test_qkv_cache_refusals(lib, kw, status):
    assert qkv(lib, **kw) == status


def attn(lib, q=P[0], dt=BF16, n=4, n_q=8, n_kv=2, D=64, k=P[1], v=P[2], ks=NULL, vs=NULL, cdt=BF16, n_pages=16,
         page=8, table=P[3], width=4, lens=P[4], scale=0.125, out=P[5], ws=ctypes.c_void_p(BIG), wsb=BIG):
    return lib.blk_attn_decode(q, dt, n, n_q, n_kv, D, k, v, ks, vs, cdt, n_pages, page, table, width, lens, scale,
                               out, ws, wsb, NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), EINVAL), (dict(n_q=0), EINVAL), (dict(n_q=9), EINVAL), (dict(n_kv=0), EINVAL),
    (dict(D=48), EUNSUPPORTED), (dict(D=160), EUNSUPPORTED), (dict(D=512), EUNSUPPORTED),
    (dict(n=4097), EUNSUPPORTED), (dict(width=0), EINVAL), (dict(width=1 << 29), EUNSUPPORTED),
    (dict(width=(1 << 27) + 1), EUNSUPPORTED),
    (dict(n_pages=1 << 29, n_kv=1), EUNSUPPORTED), (dict(n_pages=1 << 27, page=15, n_kv=4), EUNSUPPORTED),
    (dict(scale=float("nan")), EINVAL), (dict(cdt=F32), EINVAL), (dict(cdt=MX), EINVAL),
    (dict(dt=F32, cdt=MX, ks=P[9], vs=P[10]), EUNSUPPORTED), (dict(table=NULL), EINVAL), (dict(out=ODD), EINVAL),
    (dict(ws=NULL), EWORKSPACE), (dict(wsb=1024), EWORKSPACE), (dict(out=P[0]), EALIAS), (dict(out=P[2]), EALIAS),
    (dict(ws=P[0]), EALIAS), (dict(n=0, q=NULL, table=NULL, lens=NULL, out=NULL, ws=NULL, wsb=0), 0),
])
def test_attn_decode_refusals(lib, kw, status):
    assert attn(lib, **kw) == status


def test_attn_workspace_size(lib):
    size = lib.blk_attn_workspace_size
    assert size(64, 32, 4, 128, 8192) > 0 and size(0, 1, 1, 32, 1) > 0
    for bad in ((-1, 32, 4, 128, 64), (1, 33, 4, 128, 64), (1, 0, 1, 128, 64), (1, 4, 0, 128, 64), (1, 4, 4, 100, 64),
                (1, 4, 4, 128, 0), (4097, 4, 4, 128, 64), (4096, 64, 64, 128, (1 << 31) - 1)):
        assert size(*bad) == 0, bad


def linear(lib, x=P[0], dt=BF16, xs=NULL, T=4, k=64, codes=P[1], scales=P[2], n=40, y=P[3], ydt=BF16):
    return lib.blk_linear_w4(x, dt, xs, T, k, codes, scales, n, y, ydt, NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=3), EINVAL), (dict(ydt=2), EINVAL), (dict(T=-1), EINVAL), (dict(n=0), EINVAL), (dict(k=0), EINVAL),
    (dict(k=48), EUNSUPPORTED), (dict(k=(1 << 24) + 32), EUNSUPPORTED), (dict(T=(1 << 22) + 1), EUNSUPPORTED), (dict(dt=MX), EINVAL), (dict(xs=P[4]), EINVAL),
    (dict(codes=NULL), EINVAL), (dict(scales=NULL), EINVAL), (dict(y=NULL), EINVAL), (dict(x=ODD), EINVAL),
    (dict(y=P[0]), EALIAS), (dict(y=P[1]), EALIAS), (dict(dt=MX, xs=P[3]), EALIAS), (dict(T=0, x=NULL, y=NULL), 0),
])
def test_linear_w4_refusals(lib, kw, status):
    assert linear(lib, **kw) == status


@pytest.mark.parametrize("args,status", [
    ((P[0], 2, 4, 64, P[1], P[2]), EINVAL), ((P[0], BF16, 0, 64, P[1], P[2]), EINVAL),
    ((P[0], BF16, 4, 40, P[1], P[2]), EUNSUPPORTED), ((NULL, BF16, 4, 64, P[1], P[2]), EINVAL),
    ((P[0], BF16, 4, 64, P[1], NULL), EINVAL), ((P[0], BF16, 4, 64, ODD, P[2]), EINVAL),
    ((P[0], BF16, 4, 64, P[0], P[2]), EALIAS), ((P[0], BF16, 4, 64, P[1], P[1]), EALIAS),
])
def test_quantize_w4_refusals(lib, args, status):
    assert lib.blk_quantize_w4(*args, NULL) == status


# sizes whose launch would count its threads past 32 bits
@pytest.mark.parametrize("call", [
    lambda lib: norm(lib, T=(1 << 25) + 1, d=8), lambda lib: norm(lib, T=(1 << 23) + 1, d=520),
    lambda lib: norm(lib, T=(1 << 21) + 1, d=4097),
    lambda lib: qkv(lib, T=(1 << 25) + 1), lambda lib: qkv(lib, n_q=16385), lambda lib: qkv(lib, n_kv=16385),
    lambda lib: attn(lib, n=4096, n_q=2049, n_kv=2049, n_pages=1, page=1, width=1),
    lambda lib: attn(lib, n=4096, n_q=33 * 700, n_kv=700, n_pages=1, page=1, width=1),
    lambda lib: linear(lib, n=(1 << 26) + 1, k=32),
])
def test_launches_past_32_bits_are_refused(lib, call):
    assert call(lib) == EUNSUPPORTED


def test_attn_workspace_size_of_too_many_segments(lib):
    assert lib.blk_attn_workspace_size(4096, 2048, 2048, 64, 16) > 0
    assert lib.blk_attn_workspace_size(4096, 2049, 2049, 64, 16) == 0


@pytest.mark.parametrize("scale", [float("inf"), -float("inf"), 1e300, 3e38])
def test_attn_scale_beyond_float32_is_refused(lib, scale):
    assert attn(lib, scale=scale) == EINVAL
