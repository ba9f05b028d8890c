"""The decode engine takes a workspace that is large enough for its own caches (bf16 and E4M3), also where a 4-bit cache's
default, which sl_decode_attn_workspace_size covers too, has more workers."""
import numpy as np
import pytest
import torch

from paper_2504_15930_amd import engine as E
from paper_2504_15930_amd import sl

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs an MI355X")]


@pytest.mark.parametrize("fp8", [False, True])
def test_engine_asks_for_its_own_caches_workspace(monkeypatch, fp8):
    args = dict(batch_slots=40, num_q_heads=32, num_kv_heads=8, head_dim=64, kv_fp8=fp8, two_launch=True)
    lens = np.full(50, 40, np.int32)
    sizes = (40, 32, 8, 64, 16, 5, 200)
    desc = sl.make_desc(*sizes)
    own = sl.make_desc(*sizes, num_workers=max(sl.num_workers(desc, f) for f in (False, True)))
    need = sl.workspace_size(own)
    assert need < sl.workspace_size(desc)
    want = E.Engine(lens, lens, **args)
    for size in (need, need - 1):
        monkeypatch.setattr(E.sl, "workspace_size", lambda d: size)
        if size < need:
            with pytest.raises(sl.SlError) as e:
                E.Engine(lens, lens, **args)
            assert e.value.status == -4
            continue
        eng = E.Engine(lens, lens, **args)
        assert eng.workspace.numel() == need
        assert eng.run(30) == want.run(30) == 30
        torch.cuda.synchronize()
        assert torch.equal(eng.out.view(torch.int16), want.out.view(torch.int16)) and torch.isfinite(eng.out).all()
