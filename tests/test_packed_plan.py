"""Which kernels the attention over a packed context launches, on the CPU through a stub of the HIP
runtime (launch_stub.cpp): the form of the tiles and the splits. The shapes that the GPU tests take
for the form of many rows are kept here, so that they go on meeting it."""

import json
import os
import re
import subprocess
import sys

import pytest

from paper_2608_00531_amd import build as pbuild

HERE = os.path.dirname(os.path.abspath(__file__))

CHILD = """
import ctypes as c, json, sys
stub = c.CDLL(sys.argv[1], c.RTLD_GLOBAL)            # before the library's own HIP runtime
stub.stub_launches.restype = c.c_char_p
lib = c.CDLL(sys.argv[2])
p, i, l, f, z = c.c_void_p, c.c_int32, c.c_int64, c.c_float, c.c_size_t
lib.cure_packed_attn.argtypes = [p] * 5 + [l, p, p, l, p, p, i, i, i, l, i, i, i, i, f] + [p] * 10 + [i, p, p, z, p]
def call(rows, packed, ctx, hq, hkv, d, dtype="bf16", split=0, tree=True, n_max=None):
    a = lambda v: (i * len(v))(*v)
    t, b, n = 4096, len(rows), n_max or max(rows)
    stub.stub_reset(0)
    code = 0 if dtype == "f32" else 1
    status = lib.cure_packed_attn(t, t, t, t, t, 1 << 40, t, t, 1 << 40, t, t, code, code, b, b * n, n, hq, hkv, d, 0.125, None, t, t, t, t, t,
                                  t if tree else None, a(rows), a(packed), a(ctx), split, t, t, 1 << 60, None)
    return status, [x.split() for x in stub.stub_launches().decode().splitlines()]
print(json.dumps([call(**kw) for kw in json.loads(sys.argv[3])]))
"""

# Of the GPU tests: sequences of every length around a step's and a block's end, so many kv-heads that a form's
# throughput counts.
LENGTHS = [0, 1, 31, 32, 33, 63, 64, 65, 96, 97, 127, 128, 160, 193, 225]


def shape(rows, d, tree, hkv=64):
    return dict(rows=[rows // 4] * len(LENGTHS), packed=LENGTHS, ctx=[33] * len(LENGTHS), hq=4 * hkv, hkv=hkv, d=d, tree=tree)


MANY = [(rows, d, tree, 16 if d == 128 and 128 < rows <= 256 else 8) for rows in (68, 128, 132, 252, 260) for d in (64, 128)
        for tree in (True, False)]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    stub = str(tmp_path_factory.mktemp("stub") / "launch_stub.so")
    res = subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", os.path.join(HERE, "launch_stub.cpp"), "-o", stub],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def run(*calls):
        """Per call: its kernels as (form, workgroups, threads), forms as (name, d, waves of many rows)."""
        res = subprocess.run([sys.executable, "-c", CHILD, stub, pbuild.LIB_PATH, json.dumps(calls)], capture_output=True, text=True,
                             timeout=300)
        assert res.returncode == 0, res.stdout + res.stderr
        out = json.loads(res.stdout)
        assert all(status == 0 for status, _ in out), out
        form = lambda x: re.search(r"packed_(few|many|merge)I([ft]?)Li(\d+)E(?:Li(\d+)E)?(?:Lb(\d)E)?", x).groups()  # noqa: E731
        return [[(form(x[0]), int(x[1]), int(x[4])) for x in got] for _, got in out]
    return run


def test_the_gpu_tests_shapes_of_many_rows(kernels):
    got = kernels(*[shape(rows, d, tree) for rows, d, tree, _ in MANY])
    for (rows, d, tree, waves), launches in zip(MANY, got):
        (name, _, dim, groups, _), wgs, threads = launches[0]
        assert (name, int(dim)) == ("many", d) and int(groups) in (8, waves), (rows, d, tree, launches)
        assert threads == 64 * int(groups)
    assert {int(x[0][0][3]) for x in got} == {8, 16}


def test_forms(kernels):
    trees = dict(rows=[32], packed=[2048], ctx=[21], hq=32, hkv=8, d=128)
    batch = dict(rows=[20, 48, 33, 40] * 4, packed=[1024, 4096, 2000, 3000] * 4, ctx=[9] * 16, hq=32, hkv=8, d=128)
    long = dict(rows=[32] * 4, packed=[32768] * 4, ctx=[5] * 4, hq=32, hkv=8, d=128)
    token = dict(rows=[1] * 8, packed=[4096 * (b + 1) for b in range(8)], ctx=[5] * 8, hq=32, hkv=8, d=128, tree=False)
    f32 = dict(long, dtype="f32")
    few = [dict(long, rows=[16] * 4), dict(token, d=64)]
    got = kernels(trees, batch, long, token, f32, *few)
    assert [x[0][0][0] for x in got] == ["few", "few", "many", "few", "few", "few", "few"]
    assert [x[0][0][1] for x in got] == ["t", "t", "", "t", "f", "t", "t"]
    # One tile's keys are read once, past the caches; several share them.
    assert [x[0][0][4] for x in got] == ["0", "0", None, "1", "0", "0", "1"]
    assert all(x[1][0][0] == "merge" for x in got if len(x) > 1) and len(got[2]) == 2 and len(got[3]) == 2


def test_splits_as_asked_and_room_for_more_rows(kernels):
    call = dict(rows=[5, 2], packed=[9000, 64], ctx=[1, 1], hq=8, hkv=2, d=128)
    one, seven, wide = kernels(dict(call, split=1), dict(call, split=7), dict(call, split=7, n_max=200))
    assert len(one) == 1 and len(seven) == 2
    assert one[0][1] == 2 and seven[0][1] == 7 * one[0][1]
    assert wide[0][1] == 25 * seven[0][1]                   # tiles for 800 rows of a kv-head in place of 20
