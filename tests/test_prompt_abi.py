"""Refusals of the operators around the verify step, on the CPU: the C entry points reject bad
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

E, U, OK = pc.CURE_ERR_INVALID_ARG, pc.CURE_ERR_UNSUPPORTED, pc.CURE_OK


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(pbuild.LIB_PATH):
        pbuild.build_library()
    return pc.lib()


def host(*v):
    a = np.array(v, np.int32)
    return a, a.ctypes.data_as(ctypes.c_void_p)


def append(L, **kw):
    a = dict(q=4096, q_ld=4 * 64, k=4096, k_ld=2 * 64, v=4096, v_ld=2 * 64, dtype=1, rows=8, batch=2, n_max=4,
             row_off=None, n_rows=1, parent=None, kv_off=1, ctx_len=1, pos_off=None, hq=4, hkv=2, d=64,
             q_weight=None, k_weight=None, eps=1e-6, inv_freq=1, rot=64, flags=0, mscale=1.0, q_out=8192, k_cache=4096,
             v_cache=4096, cache_rows=100, row_status=1, stream=None)
    assert not set(kw) - set(a)
    a.update(kw)
    return L.cure_rope_append(*a.values())


def test_append_argument_errors(L):
    for name in ("q", "k", "v", "n_rows", "kv_off", "ctx_len", "inv_freq", "q_out", "k_cache", "v_cache", "row_status"):
        assert append(L, **{name: None}) == E, name
    assert append(L, dtype=2) == E
    for name in ("batch", "n_max", "rows", "cache_rows", "hq", "hkv", "rot"):
        assert append(L, **{name: -1}) == E, name
    assert append(L, hq=0, hkv=0) == E
    assert append(L, d=0) == E
    assert append(L, rot=80) == E                           # more than the head has
    assert append(L, rows=7) == E                           # padded rows do not fit
    assert append(L, flags=2) == E
    assert append(L, q_ld=4 * 64 - 8) == E and append(L, k_ld=64) == E and append(L, v_ld=0) == E
    assert append(L, mscale=math.nan) == E and append(L, mscale=math.inf) == E
    assert append(L, q_weight=4096, eps=-1.0) == E and append(L, k_weight=4096, eps=math.nan) == E
    for name in ("q", "k", "v", "q_out", "k_cache", "v_cache"):
        assert append(L, **{name: 4104}) == E, name         # not 16-byte aligned
    assert append(L, q_weight=4104) == E
    assert append(L, q_ld=4 * 64 + 4) == E                  # rows 8 bytes off
    assert append(L, q_out=4096, q_ld=512) == E             # in place, rows of another distance
    assert append(L, d=72, q_ld=999 * 8, k_ld=999 * 8, v_ld=999 * 8) == U
    assert append(L, d=272, q_ld=9999 * 8, k_ld=9999 * 8, v_ld=9999 * 8) == U
    assert append(L, rot=8) == U
    assert append(L, n_max=257, rows=514, parent=1) == U
    assert append(L, batch=70000, rows=1 << 20) == U
    assert append(L, batch=0) == OK
    assert append(L, n_max=0, inv_freq=None) == E           # read whatever the rows are


def frequencies(L, rot=8, base=10000.0, scaling=0, factor=1.0, orig=0.0, p0=0.0, p1=0.0):
    out, m = (ctypes.c_float * max(1, rot // 2))(), ctypes.c_float(-1.0)
    st = L.cure_rope_frequencies(rot, base, scaling, factor, orig, p0, p1, out, ctypes.byref(m))
    return st, list(out)[:rot // 2], m.value


def test_frequencies_hand_worked(L):
    """rot 8, base 10^4: 1, 1/10, 1/100, 1/1000."""
    f32 = lambda *v: [float(np.float32(x)) for x in v]  # noqa: E731
    assert frequencies(L) == (OK, f32(1, 1e-1, 1e-2, 1e-3), 1.0)
    assert frequencies(L, scaling=1, factor=4.0)[1] == f32(0.25, 0.025, 0.0025, 0.00025)
    # base * factor^(8/6): the slowest pair turns `factor` times slower, the first as before.
    st, f, m = frequencies(L, scaling=2, factor=8.0)
    assert st == OK and f[0] == 1.0 and f[3] == pytest.approx(1e-3 / 8, rel=1e-6) and m == 1.0
    # Turns over 1000 tokens: 159.2, 15.9, 1.59, 0.159. Kept from 4 on, a quarter below 1, and
    # 1.59 blends (1.5915 - 1) / 3 = 0.19718 of the way.
    st, f, m = frequencies(L, scaling=3, factor=4.0, orig=1000.0, p0=1.0, p1=4.0)
    keep = (1000 * 1e-2 / (2 * math.pi) - 1) / 3
    assert st == OK and m == 1.0
    assert f == pytest.approx([1, 1e-1, 1e-2 * keep + 0.25e-2 * (1 - keep), 0.25e-3], rel=1e-6)
    # Pair index at 32 turns: 8 ln(1000 / (64 pi)) / (2 ln 10^4) = 0.697 -> 0; at one turn: 2.2 -> 3:
    # stretched 0, 1/3, 2/3 and all of the way.
    st, f, m = frequencies(L, scaling=4, factor=4.0, orig=1000.0, p0=32.0, p1=1.0)
    mix = lambda x, s: x / 4 * s + x * (1 - s)  # noqa: E731
    assert st == OK and m == pytest.approx(0.1 * math.log(4.0) + 1, rel=1e-6)
    assert f == pytest.approx([1, mix(1e-1, 1 / 3), mix(1e-2, 2 / 3), 0.25e-3], rel=1e-6)
    assert frequencies(L, rot=0) == (OK, [], 1.0)
    t, m = pc.cure_rope_frequencies(8, scaling="ramp", factor=4.0, orig_len=1000)
    assert t.tolist() == f and m == pytest.approx(0.1 * math.log(4.0) + 1, rel=1e-6)
    assert pc.cure_rope_frequencies(8, scaling="bands", factor=4.0, orig_len=1000)[0][0] == 1.0


def test_frequencies_argument_errors(L):
    for kw in (dict(rot=-2), dict(rot=7), dict(base=1.0), dict(base=math.inf), dict(scaling=5), dict(scaling=-1),
               dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.nan), dict(scaling=3, factor=2.0),
               dict(scaling=3, factor=2.0, orig=100.0, p0=4.0, p1=1.0), dict(scaling=4, factor=2.0, orig=100.0, p0=1.0, p1=32.0)):
        assert frequencies(L, **kw)[0] == E, kw
    assert L.cure_rope_frequencies(8, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None, None) == E
    with pytest.raises(pc.CureError):
        pc.cure_rope_frequencies(8, scaling="other")
    with pytest.raises(pc.CureError):
        pc.cure_rope_frequencies(-8)


def prompt(L, n=(4,), ctx=(10,), **kw):
    hn, hc = host(*n), host(*ctx)
    a = dict(q=4096, k=4096, v=4096, o=4096, lse=None, dtype=1, out_dtype=1, batch=len(n), rows=4, hq=4, hkv=2, d=64,
             scale=0.125, row_off=1, n_rows=1, kv_off=1, ctx_len=1, host_n_rows=hn[1], host_ctx_len=hc[1], kv_split=0,
             workspace=None, ws_bytes=0, stream=None)
    assert not set(kw) - set(a)
    a.update(kw)
    return L.cure_prompt_attn(*a.values())


def test_prompt_argument_errors(L):
    for name in ("q", "k", "v", "o", "row_off", "n_rows", "kv_off", "ctx_len", "host_n_rows", "host_ctx_len"):
        assert prompt(L, **{name: None}) == E, name
    assert prompt(L, dtype=2) == E and prompt(L, out_dtype=5) == E
    for name in ("batch", "rows", "kv_split"):
        assert prompt(L, **{name: -1}) == E, name
    assert prompt(L, hq=5) == E and prompt(L, hkv=0) == E
    assert prompt(L, d=96) == U and prompt(L, d=256) == U
    for scale in (0.0, -0.1, math.inf, math.nan, 3e38):
        assert prompt(L, scale=scale) == E, scale
    assert prompt(L, q=4104) == E and prompt(L, k=4104) == E and prompt(L, v=4100) == E and prompt(L, o=4100) == E
    assert prompt(L, o=4104, out_dtype=0) == E
    assert prompt(L, n=(5,)) == E                           # more tokens than rows
    assert prompt(L, n=(-1,)) == E and prompt(L, ctx=(-1,)) == E
    assert prompt(L, ctx=(2 ** 31 - 4,)) == U
    assert prompt(L, batch=0) == OK and prompt(L, rows=0) == OK and prompt(L, n=(0,)) == OK
    assert prompt(L, ctx=(1000,), kv_split=2) == pc.CURE_ERR_WORKSPACE
    assert prompt(L, ctx=(1000,), kv_split=2, workspace=4104, ws_bytes=1 << 30) == E


def prefix(L, nodes=(3, 4), ctx=(10, 0), **kw):
    hn, hc = host(*nodes), host(*ctx)
    a = dict(q=4096, k=4096, v=4096, o=4096, lse=None, dtype=1, out_dtype=1, batch=2, hq=4, hkv=2, d=64, scale=0.125,
             prefix_off=0, prefix_len=100, kv_off=1, ctx_len=1, n_nodes=1, parent=1, n_max=4, host_ctx_len=hc[1],
             host_n_nodes=hn[1], kv_split=0, tree_status=None, workspace=None, ws_bytes=0, stream=None)
    assert not set(kw) - set(a)
    a.update(kw)
    return L.cure_prefix_attn(*a.values())


def test_prefix_argument_errors(L):
    for name in ("q", "k", "v", "o", "kv_off", "ctx_len", "n_nodes", "parent", "host_ctx_len", "host_n_nodes"):
        assert prefix(L, **{name: None}) == E, name
        assert prefix(L, prefix_len=0, **{name: None}) == E, name
    assert prefix(L, dtype=2) == E and prefix(L, out_dtype=5) == E
    for name in ("batch", "n_max", "kv_split", "prefix_off", "prefix_len"):
        assert prefix(L, **{name: -1}) == E, name
    assert prefix(L, hq=5) == E and prefix(L, d=80) == U
    for scale in (0.0, -0.1, math.inf, math.nan, 3e38):
        assert prefix(L, scale=scale) == E, scale
    assert prefix(L, q=4104) == E and prefix(L, o=4100) == E
    assert prefix(L, n_max=257) == U and prefix(L, batch=1025) == U and prefix(L, prefix_len=2 ** 31 - 10) == U
    assert prefix(L, nodes=(3, 5)) == E and prefix(L, nodes=(-1, 2)) == E and prefix(L, ctx=(-1, 2)) == E
    assert prefix(L, nodes=(1,) * 1024, ctx=(0,) * 1024, batch=1024, n_max=256, hq=1 << 13, hkv=1) == U   # 2^31 rows
    assert prefix(L) == pc.CURE_ERR_WORKSPACE
    assert prefix(L, workspace=4104, ws_bytes=1 << 30) == E
    assert prefix(L, batch=0) == OK and prefix(L, n_max=0) == OK


def test_workspace_sizes(L):
    n, c = host(1, 1), host(8000, 8000)
    size = lambda split: L.cure_prompt_attn_workspace_size(2, 2, 32, 8, 128, n[1], c[1], split)  # noqa: E731
    assert size(1) == 0 and size(4) >= 2 * 32 * 4 * 129 * 4 and size(8) > size(4)
    assert L.cure_prompt_attn_workspace_size(0, 2, 32, 8, 128, n[1], c[1], 0) == 0
    tree = L.cure_tree_attn_workspace_size(2, 32, 8, 128, 1, c[1], n[1], 0)
    f = lambda length, split=0: L.cure_prefix_attn_workspace_size(2, 32, 8, 128, 1, length, c[1], n[1], split)  # noqa: E731
    parts = lambda slots: 2 * 32 * slots * 129 * 4  # noqa: E731
    assert f(0) == tree and f(100) >= parts(2) and f(1000, 8) >= parts(9) and f(1000, 8) > f(1000, 1)


@pytest.fixture
def t():
    """Tensors of a good call, without a GPU."""
    with FakeTensorMode():
        f = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
        yield dict(q=f(2, 4, 4, 64), k=f(2, 4, 2, 64), v=f(2, 4, 2, 64), k_cache=f(50, 2, 64), v_cache=f(50, 2, 64),
                   kv_off=f(2, dtype=torch.int64), ctx_len=f(2, dtype=torch.int32), n_rows=f(2, dtype=torch.int32),
                   inv_freq=f(32, dtype=torch.float32))


def refused(fn, *args, **kw):
    try:
        fn(*args, **kw)
    except (pc.CureError, TypeError, ValueError) as e:
        return "data pointer" not in str(e)
    return False


def test_the_binding_checks_append(t):
    f = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    call = lambda **kw: refused(pc.cure_rope_append, **{**t, **kw})  # noqa: E731
    assert call(q=torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16, device="cpu"))
    assert call(q=f(2, 4, 4, 32)) and call(q=f(2, 3, 4, 64)) and call(k=f(2, 4, 1, 64)) and call(q=f(8, 4, 64))
    assert call(q=f(2, 4, 4, 64, dtype=torch.float32)) and call(v=f(2, 4, 2, 64, dtype=torch.float16))
    assert call(k_cache=f(50, 2, 32)) and call(v_cache=f(49, 2, 64)) and call(k_cache=f(50, 3, 64), v_cache=f(50, 3, 64))
    assert call(k_cache=f(50, 4, 64)[:, :2]) and call(v_cache=f(50, 2, 64, dtype=torch.float32))
    assert call(kv_off=f(2, dtype=torch.int32)) and call(ctx_len=f(2, dtype=torch.int64)) and call(n_rows=f(3, dtype=torch.int32))
    assert call(parent=f(2, 5, dtype=torch.int32)) and call(pos_off=f(1, dtype=torch.int32))
    assert call(inv_freq=f(32)) and call(inv_freq=f(65, dtype=torch.float32)) and call(q_weight=f(32))
    assert call(k_weight=f(64, dtype=torch.float32)) and call(n_max=3) and call(row_off=f(2, dtype=torch.int64))
    assert call(out=f(2, 4, 4, 32)) and call(out=f(2, 4, 4, 64, dtype=torch.float32)) and call(q=None, out=f(2, 4, 4, 64))
    assert call(eps="x") and call(q=3)


def test_the_binding_checks_attention(t):
    f = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    i = lambda *s: f(*s, dtype=torch.int32)  # noqa: E731
    l = lambda *s: f(*s, dtype=torch.int64)  # noqa: E731
    good = dict(q=f(8, 4, 64), k=f(50, 2, 64), v=f(50, 2, 64), row_off=l(2), n_rows=i(2), kv_off=l(2), ctx_len=i(2),
                host_n_rows=[4, 4], host_ctx_len=[1, 2], scale=0.1)
    call = lambda **kw: refused(pc.cure_prompt_attn, **{**good, **kw})  # noqa: E731
    assert call(q=f(2, 4, 4, 64)) and call(q=f(8, 8, 64)[:, ::2]) and call(k=f(50, 2, 32)) and call(v=f(51, 2, 64))
    assert call(k=f(50, 2, 64, dtype=torch.float32)) and call(k=f(50, 4, 64)[:, :2]) and call(row_off=i(2))
    assert call(n_rows=i(2, 1)) and call(kv_off=l(3)) and call(ctx_len=l(2)) and call(host_n_rows=[4])
    assert call(host_ctx_len=[1]) and call(out=f(8, 4, 32)) and call(out=f(8, 4, 64), out_dtype=torch.float32)
    assert call(out_dtype=3) and call(scale="x")
    good = dict(q=f(2, 4, 4, 64), k=f(50, 2, 64), v=f(50, 2, 64), prefix_off=0, prefix_len=20, kv_off=l(2), ctx_len=i(2),
                n_nodes=i(2), parent=i(2, 4), host_ctx_len=[1, 2], host_n_nodes=[4, 4], scale=0.1)
    call = lambda **kw: refused(pc.cure_prefix_attn, **{**good, **kw})  # noqa: E731
    assert call(prefix_off=-1) and call(prefix_len=-1) and call(prefix_off=31) and call(prefix_len=2 ** 31)
    assert call(q=f(8, 4, 64)) and call(parent=i(2, 3)) and call(n_nodes=l(2)) and call(host_n_nodes=[4])
    assert call(k=f(50, 2, 32)) and call(kv_off=i(2)) and call(out=f(2, 4, 4, 32)) and call(prefix_len=1.5)
