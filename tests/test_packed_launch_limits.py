"""Launches of packing, unpacking and the packed attention at the ends of the sizes they support, on the CPU
through a stub of the HIP runtime (launch_stub.cpp), which takes any grid: none has 2^32 threads in a row, and calls
that would need one are refused."""

import json
import os
import subprocess
import sys

import pytest

import paper_2608_00531_amd as pc
from paper_2608_00531_amd import build as pbuild

HERE = os.path.dirname(os.path.abspath(__file__))

CHILD = """
import ctypes as c, json, sys
stub = c.CDLL(sys.argv[1], c.RTLD_GLOBAL)            # before the library's own HIP runtime
stub.stub_launches.restype = c.c_char_p
lib = c.CDLL(sys.argv[2])
p, i, l, f, z = c.c_void_p, c.c_int32, c.c_int64, c.c_float, c.c_size_t
lib.cure_kv_pack.argtypes = [p, p, i, i, l, l, i, i, i, i, p, p, p, p, p, p, l, l, p, p, p, p]
lib.cure_kv_unpack.argtypes = [p, p, p, p, l, l, p, p, p, p, i, i, l, l, i, i, i, i, p, p, p, p]
lib.cure_packed_attn.argtypes = [p] * 5 + [l, p, p, l, p, p, i, i, i, l, i, i, i, i, f] + [p] * 10 + [i, p, p, z, p]
big, t = 1 << 40, 4096
def call(name, n_max=0, hkv=1, d=128, rows=0, hq=1, dtype=1, split=0):
    stub.stub_reset(0)
    a = lambda v: (i * 1)(v)
    if name == "pack":
        status = lib.cure_kv_pack(t, t, dtype, 1, 0, big, hkv, d, 1, n_max, t, t, t, t, t, t, 0, big, t, t, t, None)
    elif name == "unpack":
        status = lib.cure_kv_unpack(t, t, t, t, 0, big, t, t, t, t, dtype, 1, 0, big, hkv, d, 1, n_max, t, t, t, None)
    else:
        status = lib.cure_packed_attn(t, t, t, t, t, big, t, t, big, t, t, dtype, dtype, 1, rows, n_max, hq, hkv, d, 0.125, t, t, t, t, t, t,
                                      None, a(rows), a(1 << 15), a(0), split, t, t, 1 << 60, None)
    return status, [[int(y) for y in x.split()[1:]] for x in stub.stub_launches().decode().splitlines()]
print(json.dumps([call(**kw) for kw in json.loads(sys.argv[3])]))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    stub = str(tmp_path_factory.mktemp("stub") / "launch_stub.so")
    res = subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", os.path.join(HERE, "launch_stub.cpp"), "-o", stub],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def run(*calls):
        res = subprocess.run([sys.executable, "-c", CHILD, stub, pbuild.LIB_PATH, json.dumps(calls)], capture_output=True, text=True,
                             timeout=300)
        assert res.returncode == 0, res.stdout + res.stderr
        out = json.loads(res.stdout)
        for status, grids in out:
            assert all(x * threads < 1 << 32 and y < 65536 and z < 65536 for x, y, z, threads in grids), (status, grids)
            assert bool(grids) == (status == 0)
        return out
    return run


# hkv, the largest n_max that packing holds, the largest that unpacking holds.
ENDS = [(1, (2 ** 24 - 1) * 64, (2 ** 24 - 2) * 64), (8, (2 ** 21 - 1) * 64, (2 ** 21 - 2) * 64), (1 << 20, 15 * 64, 14 * 64),
        (5, (2 ** 24 // 5) * 64, (2 ** 24 // 5 - 1) * 64)]


@pytest.mark.parametrize("hkv,pack,unpack", ENDS)
def test_packing(launches, hkv, pack, unpack):
    for name, most in (("pack", pack), ("unpack", unpack)):
        got = launches(*[dict(name=name, hkv=hkv, n_max=most + more, dtype=dtype, d=d) for dtype in (0, 1) for d in (64, 128) for more in (0, 1)])
        assert [status for status, _ in got] == [pc.CURE_OK, pc.CURE_ERR_UNSUPPORTED] * 4


def test_no_rows_at_all(launches):
    assert [s for s, _ in launches(dict(name="pack", hkv=1 << 20), dict(name="unpack", hkv=1 << 20))] == [0, 0]


@pytest.mark.parametrize("dtype,d", [(0, 64), (0, 128), (1, 64), (1, 128)])
def test_joined_splits(launches, dtype, d):
    """Splits are joined for the rows that there are, however many a sequence might have by n_max."""
    for hq, rows in ((256, 1000), (1, 1), (32, 9000), (1 << 20, 1)):
        n_max = (1 << 28) // hq
        (status, grids), (_, alike) = launches(dict(name="attend", n_max=n_max, hq=hq, hkv=1, d=d, rows=rows, dtype=dtype, split=2),
                                               dict(name="attend", n_max=rows, hq=hq, hkv=1, d=d, rows=rows, dtype=dtype, split=2))
        assert status == 0 and len(grids) in (1, 2) and grids == alike, (hq, rows, grids, alike)
        if len(grids) == 2:
            assert grids[1][0] == -(-rows * hq // (1024 // d))
    assert len(grids) == 1 or d == 64                       # 2^20 heads: no room for parts at d = 128
