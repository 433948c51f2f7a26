"""The binding's calls of the prompt and rotary operators, on the CPU: tensors without storage raise, and
their scratch memory is each call's own."""

import pytest

from test_binding_host import child, stub  # noqa: F401


@pytest.mark.parametrize("name", ["rope_append", "prompt_attn", "prefix_attn"])
def test_tensors_without_storage_raise(stub, name):  # noqa: F811
    """A tensor under vmap has no data pointer: every call says so and the process lives."""
    out = child(stub, """
        with FakeTensorMode():
            f = lambda *s: torch.zeros(3, *s, device="cuda")
            i = lambda *s: torch.zeros(3, *s, dtype=torch.int32, device="cuda")
            q, p, k, off, n, t = f(2, 4, 2, 64), f(8, 2, 64), f(40, 2, 64), torch.zeros(3, 2, dtype=torch.int64, device="cuda"), i(2), i(2, 4)
            w = torch.zeros(32, device="cuda")
            fn, args = {
                "rope_append": (lambda q, k, off, n, t: pc.cure_rope_append(q, q, q, k, k, off, n, n, w, parent=t), [q, k, off, n, t]),
                "prompt_attn": (lambda p, k, off, n: pc.cure_prompt_attn(p, k, k, off, n, off, n, [4, 4], [8, 8], 1.0), [p, k, off, n]),
                "prefix_attn": (lambda q, k, off, n, t: pc.cure_prefix_attn(q, k, k, 0, 9, off, n, n, t, [8, 8], [4, 4], 1.0),
                                [q, k, off, n, t]),
            }[sys.argv[2]]
            try:
                torch.vmap(fn)(*args)
            except RuntimeError as e:
                print("refused" if "data pointer" in str(e) else e)
        """, name)
    assert out == ["refused"]
