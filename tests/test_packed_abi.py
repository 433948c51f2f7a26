"""Refusals of the packed cache's operators and of sampling, on the CPU: the C entry points reject bad
arguments before touching a device, and the binding checks its tensors.

Device pointers here are fake, so every call is built to stop at a host-side check.
"""

import ctypes
import math
import os

import numpy as np
import pytest
import torch
from torch._subclasses import FakeTensorMode

import paper_2608_00531_amd as pc
from paper_2608_00531_amd import build as pbuild
from test_binding_host import child, stub  # noqa: F401

E, U, OK, WS = pc.CURE_ERR_INVALID_ARG, pc.CURE_ERR_UNSUPPORTED, pc.CURE_OK, pc.CURE_ERR_WORKSPACE


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(pbuild.LIB_PATH):
        pbuild.build_library()
    return pc.lib()


def host(*v):
    a = np.array(v, np.int32)
    return a, a.ctypes.data_as(ctypes.c_void_p)


def pack(L, **kw):
    a = dict(k=4096, v=4096, dtype=1, n_layers=2, layer_stride=50 * 2 * 64, rows=50, hkv=2, d=64, batch=2, n_max=20, kv_off=4096,
             n_rows=4096, pk=4096, pv=4096, k_scale=4096, v_scale=4096, block_stride=9, blocks=9, blk_off=4096, packed_len=4096,
             row_status=4096, stream=None)
    assert not set(kw) - set(a)
    a.update(kw)
    return L.cure_kv_pack(*a.values())


def unpack(L, **kw):
    a = dict(pk=4096, pv=4096, k_scale=4096, v_scale=4096, block_stride=9, blocks=9, blk_off=4096, packed_len=4096, k=4096, v=4096,
             dtype=1, n_layers=2, layer_stride=50 * 2 * 64, rows=50, hkv=2, d=64, batch=2, n_max=20, kv_off=4096, n_rows=4096,
             row_status=4096, stream=None)
    assert not set(kw) - set(a)
    a.update(kw)
    return L.cure_kv_unpack(*a.values())


@pytest.mark.parametrize("call", [pack, unpack])
def test_pack_argument_errors(L, call):
    for name in ("k", "v", "pk", "pv", "k_scale", "v_scale", "kv_off", "n_rows", "blk_off", "packed_len", "row_status"):
        assert call(L, **{name: None}) == E, name
    assert call(L, dtype=2) == E
    for name in ("rows", "hkv", "d", "batch", "n_max", "blocks", "n_layers", "layer_stride", "block_stride"):
        assert call(L, **{name: -1}) == E, name
    assert call(L, hkv=0) == E and call(L, n_layers=0) == E
    for name in ("k", "v", "pk", "pv"):
        assert call(L, **{name: 4104}) == E, name           # not 16-byte aligned
    assert call(L, k_scale=4098) == E and call(L, v_scale=4098) == E
    assert call(L, layer_stride=50 * 2 * 64 + 4) == E       # layers 8 bytes off
    assert call(L, d=96) == U and call(L, d=256) == U
    assert call(L, batch=65536) == U and call(L, n_layers=65536) == U and call(L, n_max=1 << 29) == U
    assert call(L, hkv=(1 << 20) + 1, layer_stride=50 * ((1 << 20) + 1) * 64) == U
    assert call(L, batch=0) == OK and call(L, batch=0, kv_off=None) == OK


def attend(L, n=(3, 4), packed=(100, 7), ctx=(5, 0), **kw):
    hn, hp, hc = host(*n), host(*packed), host(*ctx)
    a = dict(q=4096, pk=4096, pv=4096, k_scale=4096, v_scale=4096, blocks=9, k=4096, v=4096, cache_rows=50, o=4096, lse=None, dtype=1,
             out_dtype=1, batch=2, rows=8, n_max=4, hq=4, hkv=2, d=64, scale=0.1, row_off=None, n_rows=4096, blk_off=4096,
             packed_len=4096, kv_off=4096, ctx_len=4096, parent=None, host_n_rows=hn[1], host_packed_len=hp[1],
             host_ctx_len=hc[1], kv_split=2, row_status=None, workspace=None, ws_bytes=0, stream=None)
    assert not set(kw) - set(a)
    a.update(kw)
    return L.cure_packed_attn(*a.values())


def test_attention_argument_errors(L):
    for name in ("q", "pk", "pv", "k_scale", "v_scale", "k", "v", "o", "n_rows", "blk_off", "packed_len", "kv_off", "ctx_len",
                 "host_n_rows", "host_packed_len", "host_ctx_len"):
        assert attend(L, **{name: None}) == E, name
    assert attend(L, dtype=2) == E and attend(L, out_dtype=7) == E
    for name in ("batch", "rows", "n_max", "blocks", "cache_rows", "hq", "hkv", "d", "kv_split"):
        assert attend(L, **{name: -1}) == E, name
    assert attend(L, hq=5) == E and attend(L, rows=7) == E
    for scale in (0.0, -0.1, math.inf, math.nan, 3e38):
        assert attend(L, scale=scale) == E, scale
    for name in ("q", "pk", "pv", "k", "v", "o"):
        assert attend(L, **{name: 4104}) == E, name
    assert attend(L, n=(5, 1)) == E and attend(L, n=(-1, 1)) == E and attend(L, packed=(-1, 1)) == E and attend(L, ctx=(1, -1)) == E
    assert attend(L, d=96) == U and attend(L, batch=65536) == U and attend(L, n_max=1 << 27, rows=1 << 28) == U
    assert attend(L, parent=4096, n_max=257, rows=514) == U and attend(L, packed=(2 ** 31 - 100, 0)) == U
    assert attend(L) == WS                                  # two splits and nowhere for them
    assert attend(L, workspace=4104, ws_bytes=1 << 30) == E and attend(L, workspace=4096, ws_bytes=8) == WS
    assert attend(L, batch=0) == OK and attend(L, batch=0, n_rows=None) == OK


def test_workspace_sizes(L):
    n, p, c = host(1, 1), host(8000, 8000), host(0, 9)
    size = lambda split, rows=2, hq=32, d=128: L.cure_packed_attn_workspace_size(2, rows, 1, hq, 8, d, n[1], p[1], c[1], split)  # noqa: E731
    parts = lambda slots, d=128: 2 * 32 * slots * (d + 1) * 4  # noqa: E731
    assert size(1) == 0 and size(2) == parts(2) and size(7) == parts(7) and size(4, d=64) == parts(4, 64)
    assert 0 < size(0) <= parts(64) and size(1000) == parts(64)
    assert size(3, rows=0) == 0 and size(3, hq=33) == 0 and size(-1) == 0
    bad = host(2, 1)
    assert L.cure_packed_attn_workspace_size(2, 2, 1, 32, 8, 128, bad[1], p[1], c[1], 2) == 0
    # Sizes at the ends of what is allowed are planned without overflow: 2^21 tiles over 2^26 steps each.
    many, long = host(1 << 20), host(2 ** 31 - 2 ** 21)
    got = L.cure_packed_attn_workspace_size(1, 1 << 20, 1 << 20, 256, 1, 128, many[1], long[1], host(0)[1], 0)
    assert got == 0                                         # parts would pass the limit


def sample(L, **kw):
    a = dict(logits=4096, dtype=1, batch=2, rows=3, vocab=100, ld=100, temperature=None, top_k=None, top_p=None, min_p=None,
             uniform=4096, n_rows=None, token=4096, logprob=None, kept=None, stream=None)
    assert not set(kw) - set(a)
    a.update(kw)
    return L.cure_sample(*a.values())


def test_sample_argument_errors(L):
    for name in ("logits", "uniform", "token"):
        assert sample(L, **{name: None}) == E, name
    assert sample(L, dtype=2) == E and sample(L, ld=99) == E and sample(L, vocab=0) == E
    for name in ("batch", "rows", "vocab"):
        assert sample(L, **{name: -1}) == E, name
    assert sample(L, logits=4097) == E and sample(L, dtype=0, logits=4098) == E
    assert sample(L, vocab=(1 << 20) + 1, ld=1 << 21) == U and sample(L, batch=1 << 20, rows=2) == U
    assert sample(L, batch=0) == OK and sample(L, rows=0, logits=None) == OK


def refused(fn, *args, **kw):
    try:
        fn(*args, **kw)
    except (pc.CureError, TypeError, ValueError) as e:
        return "data pointer" not in str(e)
    except RuntimeError:                                    # past the checks: no device, or no storage
        pass
    return False


@pytest.fixture
def f():
    """Tensors without a GPU."""
    with FakeTensorMode():
        yield lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")


def test_the_binding_checks_packing(f):
    i, l, b, g = (lambda *s, t=t: f(*s, dtype=t) for t in (torch.int32, torch.int64, torch.int8, torch.float32))
    good = dict(k=f(3, 50, 2, 64), v=f(3, 50, 2, 64), kv_off=l(2), n_rows=i(2), pk=b(3, 9, 2, 4096), pv=b(3, 9, 2, 4096),
                k_scale=g(3, 9, 2), v_scale=g(3, 9, 2), blk_off=l(2), packed_len=i(2))
    call = lambda **kw: refused(pc.cure_kv_pack, **{**good, **kw})  # noqa: E731
    assert not call()                                       # only the missing storage
    assert call(k=torch.zeros(3, 50, 2, 64, dtype=torch.bfloat16, device="cpu"))
    assert call(v=f(3, 51, 2, 64)) and call(v=f(3, 50, 2, 64, dtype=torch.float32)) and call(k=f(50, 2, 64), v=f(50, 2, 64))
    assert call(k=f(3, 50, 2, 64, dtype=torch.float16), v=f(3, 50, 2, 64, dtype=torch.float16))
    assert call(k=f(3, 50, 4, 64)[:, :, :2]) and call(pk=i(3, 9, 2, 4096)) and call(pv=b(3, 9, 2, 4097)) and call(pk=b(3, 8, 2, 4096))
    assert call(k_scale=l(3, 9, 2)) and call(v_scale=g(3, 9, 1)) and call(k_scale=g(3, 9, 4)[..., :2]) and call(pk=b(3, 18, 2, 4096)[:, ::2])
    assert call(kv_off=i(2)) and call(n_rows=l(2)) and call(blk_off=l(3)) and call(packed_len=i(1)) and call(n_rows=i(2, 1))
    assert call(k=f(6, 50, 2, 64)[::2]) and call(pk=b(3, 10, 2, 4096)[:, :9]) and call(n_max="x")
    assert call(k_scale=3)
    assert not call(k=f(6, 50, 2, 64)[::2], v=f(6, 50, 2, 64)[::2])        # layers of a larger cache
    good = dict(pk=b(9, 2, 4096), pv=b(9, 2, 4096), k_scale=g(9, 2), v_scale=g(9, 2), blk_off=l(2), first=i(2), k=f(50, 2, 64),
                v=f(50, 2, 64), kv_off=l(2), n_rows=i(2))
    call = lambda **kw: refused(pc.cure_kv_unpack, **{**good, **kw})  # noqa: E731
    assert not call()
    assert call(first=l(2)) and call(blk_off=i(2)) and call(v=f(50, 2, 32)) and call(pk=b(9, 2, 4096)[:, :1]) and call(n_max="x")


def test_the_binding_checks_attention(f):
    i, l, b, g = (lambda *s, t=t: f(*s, dtype=t) for t in (torch.int32, torch.int64, torch.int8, torch.float32))
    good = dict(q=f(2, 4, 4, 64), pk=b(9, 2, 4096), pv=b(9, 2, 4096), k_scale=g(9, 2), v_scale=g(9, 2), blk_off=l(2), packed_len=i(2),
                k=f(50, 2, 64), v=f(50, 2, 64), kv_off=l(2), ctx_len=i(2), n_rows=i(2), host_packed_len=[70, 3], host_ctx_len=[1, 2],
                host_n_rows=[4, 4], scale=0.1, parent=i(2, 4))
    call = lambda **kw: refused(pc.cure_packed_attn, **{**good, **kw})  # noqa: E731
    assert not call()
    assert call(q=f(8, 4, 64)) and call(q=f(2, 4, 8, 64)[:, :, ::2]) and call(k=f(50, 2, 32)) and call(v=f(51, 2, 64))
    assert call(pk=b(9, 2, 2048)) and call(pv=b(8, 2, 4096)) and call(pk=f(9, 2, 4096)) and call(k_scale=g(9, 1)) and call(v_scale=f(9, 2))
    assert call(k=f(1, 50, 2, 64), v=f(1, 50, 2, 64)) and call(q=f(2, 4, 4, 64, dtype=torch.float32))
    assert call(blk_off=i(2)) and call(packed_len=l(2)) and call(kv_off=l(3)) and call(ctx_len=l(2)) and call(n_rows=i(2, 1))
    assert call(parent=i(2, 5)) and call(parent=l(2, 4)) and call(host_packed_len=[1]) and call(host_ctx_len=[1])
    assert call(host_n_rows=[4]) and call(out=f(2, 4, 4, 32)) and call(out=f(2, 4, 4, 64), out_dtype=torch.float32)
    assert call(out_dtype=3) and call(scale="x") and call(kv_split="x") and call(row_off=l(2)) and call(k=None)
    good.update(q=f(8, 4, 64), parent=None, row_off=l(2))
    assert not call() and call(q=f(2, 4, 4, 64)) and call(row_off=i(2)) and call(row_off=l(3))


def test_the_binding_checks_sampling(f):
    i, g = (lambda *s, t=t: f(*s, dtype=t) for t in (torch.int32, torch.float32))
    good = dict(logits=f(2, 3, 100), uniform=g(2, 3), temperature=g(2), top_k=i(2), top_p=g(2), min_p=g(2), n_rows=i(2))
    call = lambda **kw: refused(pc.cure_sample, **{**good, **kw})  # noqa: E731
    assert not call()
    assert call(logits=f(2, 3, 100, dtype=torch.float16)) and call(logits=f(100))
    assert call(uniform=g(2, 4)) and call(uniform=f(2, 3)) and call(temperature=g(3)) and call(temperature=f(2)) and call(temperature=1.0)
    assert call(top_k=g(2)) and call(top_k=i(1)) and call(top_p=i(2)) and call(min_p=g(2, 1)) and call(n_rows=g(2)) and call(n_rows=i(3))


@pytest.mark.parametrize("name", ["pack", "unpack", "attend", "sample"])
def test_tensors_without_storage_raise(stub, name):  # noqa: F811
    """A tensor under vmap has no data pointer: every call says so and the process lives."""
    out = child(stub, """
        with FakeTensorMode():
            f = lambda *s: torch.zeros(3, *s, device="cuda")
            i = lambda *s: torch.zeros(3, *s, dtype=torch.int32, device="cuda")
            q, k, off, n = f(2, 4, 2, 64), f(40, 2, 64), torch.zeros(3, 2, dtype=torch.int64, device="cuda"), i(2)
            p, s, x, u = torch.zeros(3, 9, 2, 4096, dtype=torch.int8, device="cuda"), f(9, 2), f(2, 3, 100), f(2, 3)
            fn, args = {
                "pack": (lambda k, off, n, p, s: pc.cure_kv_pack(k, k, off, n, p, p, s, s, off, n), [k, off, n, p, s]),
                "unpack": (lambda k, off, n, p, s: pc.cure_kv_unpack(p, p, s, s, off, n, k, k, off, n), [k, off, n, p, s]),
                "attend": (lambda q, k, off, n, p, s: pc.cure_packed_attn(q, p, p, s, s, off, n, k, k, off, n, n, [8, 8], [8, 8], [4, 4], 1.0),
                           [q, k, off, n, p, s]),
                "sample": (lambda x, u: pc.cure_sample(x, u), [x, u]),
            }[sys.argv[2]]
            try:
                torch.vmap(fn)(*args)
            except RuntimeError as e:
                print("refused" if "data pointer" in str(e) else e)
        """, name)
    assert out == ["refused"]
