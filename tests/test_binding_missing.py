"""Without csrc/binding.cpp's module the calls that it makes are made by Python alone, with one warning."""
import sys
import warnings

import pytest
import torch

import paper_2504_15930_amd
from paper_2504_15930_amd import sl


def test_calls_without_the_binding(monkeypatch):
    name = "paper_2504_15930_amd._binding"
    monkeypatch.setattr(sl, "_fast", None)
    monkeypatch.delattr(paper_2504_15930_amd, "_binding", raising=False)
    monkeypatch.setitem(sys.modules, name, None)      # an import raises ImportError
    t = torch.zeros(2, 2, 64)
    calls = [lambda: sl.decode_attn_fp4(t.bfloat16(), t.to(torch.uint8), t[0].int(), t[0, 0].int(), 1.0),
             lambda: sl.kv_read_fp4(t[0, 0].int(), t.to(torch.uint8)),
             lambda: sl.pages_release(t[0, 0].int(), t[0, 0].int(), t[0].int(), t[0, 0].int(), t[0, 0, :1].int())]
    with pytest.warns(RuntimeWarning, match="_binding.so"), pytest.raises(ValueError, match="GPU"):
        calls[0]()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        for call in calls:
            with pytest.raises(ValueError):           # Python's own check of the arguments
                call()
