"""csrc/binding.cpp on the host: it declines whatever is not a call on GPU tensors, and Python then says what is wrong."""
import os

import pytest
import torch

from paper_2504_15930_amd import sl


@pytest.fixture(scope="module")
def fast():
    from paper_2504_15930_amd import build
    if not (os.path.exists(build.LIBRARY) and os.path.exists(build.BINDING)):
        build.build()
    return sl._binding()


def test_declines_host_tensors_and_other_objects(fast):
    q, pool = torch.zeros((2, 8, 64), dtype=torch.bfloat16), torch.zeros((4, 2, 17 * 64), dtype=torch.uint8)
    table, lens = torch.zeros((2, 3), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    rows, one = torch.zeros((2, 2, 64), dtype=torch.bfloat16), torch.ones(1, dtype=torch.int32)
    calls = {"attn": (q, pool, table, lens, 0.125, None, None, None, 0), "append": (rows, rows, table, lens, pool),
             "write": (rows, rows, lens, pool), "read": (lens, pool, None, None),
             "extend": (lens, lens, table, lens, one, 8, None, None, None, None),
             "release": (lens, lens, table, lens, one, None, None)}
    for name, args in calls.items():
        f = getattr(fast, name)
        assert f(*args) is None, name
        for i in range(len(args)):
            for x in (None, 3, "x", object(), torch.zeros(0)):
                assert f(*args[:i], x, *args[i + 1:]) is None, (name, i, x)
        assert f(*args[:-1]) is None and f(*args, None) is None and f() is None, name


def test_binding_needs_every_function(fast):
    with pytest.raises(KeyError):
        fast.bind({}, {}, print, print)
    with pytest.raises(TypeError):
        fast.bind(None, {}, print, print)
    # the functions that were bound before are still there
    with pytest.raises(TypeError):
        sl.decode_attn_fp4(torch.zeros(2, 8, 64), None, None, None, 1.0)


@pytest.mark.parametrize("call", [
    lambda t: sl.decode_attn_fp4(t.bfloat16(), t.to(torch.uint8), t[0].int(), t[0, 0].int(), 1.0),
    lambda t: sl.kv_append_fp4(t.bfloat16(), t.bfloat16(), t[0].int(), t[0, 0].int(), t.to(torch.uint8)),
    lambda t: sl.kv_write_fp4(t.bfloat16(), t.bfloat16(), t[0, 0].int(), t.to(torch.uint8)),
    lambda t: sl.kv_read_fp4(t[0, 0].int(), t.to(torch.uint8)),
    lambda t: sl.pages_extend(t[0, 0].int(), t[0, 0].int(), t[0].int(), t[0, 0].int(), t[0, 0, :1].int(), 8),
    lambda t: sl.pages_release(t[0, 0].int(), t[0, 0].int(), t[0].int(), t[0, 0].int(), t[0, 0, :1].int()),
])
def test_host_tensors_are_refused(fast, call):
    with pytest.raises(ValueError):
        call(torch.zeros(2, 2, 64))
