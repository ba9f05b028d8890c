"""Which scratch buffer a Python call gets (on the host: torch's allocation and capture state are stood in for)."""
import threading

import pytest
import torch

from paper_2504_15930_amd import sl


@pytest.fixture
def capturing(monkeypatch):
    """A list whose first entry says whether the current stream is being captured; host buffers for device ones."""
    state = [False]
    empty = torch.empty
    monkeypatch.setattr(sl.torch, "empty", lambda n, dtype, device: empty(n, dtype=dtype))
    monkeypatch.setattr(sl.torch.cuda, "is_current_stream_capturing", lambda: state[0])
    monkeypatch.setattr(sl, "_workspaces", {})
    return state


def test_a_stream_keeps_its_buffer_until_a_larger_one(capturing):
    a = sl._workspace(0, 5, 1000)
    assert sl._workspace(0, 5, 10) is a and sl._workspace(0, 5, 1000) is a
    assert sl._workspace(0, 6, 1000) is not a and sl._workspace(1, 5, 1000) is not a
    b = sl._workspace(0, 5, 1001)
    assert b is not a and b.numel() >= 1001 and sl._workspace(0, 5, 1) is b


def test_a_captured_call_gets_a_buffer_that_no_other_call_has(capturing):
    """A graph holds its address: it is neither what eager calls on the stream use, nor dropped by them for a larger one,
    nor another graph's."""
    a = sl._workspace(0, 5, 1000)
    capturing[0] = True
    x, y = sl._workspace(0, 5, 1000), sl._workspace(0, 5, 10)
    assert len({t.data_ptr() for t in (a, x, y)}) == 3 and x.numel() >= 1000 and y.numel() >= 10
    sl._workspace(0, 7, 1000)
    assert list(sl._workspaces.values()) == [a]     # nothing of a capture is kept for later calls
    capturing[0] = False
    assert sl._workspace(0, 5, 1000) is a


def test_threads_on_one_stream_have_their_own(capturing):
    """A call is two kernels, which another thread's could come between."""
    mine, theirs = sl._workspace(0, 5, 1000), []
    t = threading.Thread(target=lambda: theirs.extend(sl._workspace(0, 5, n) for n in (1000, 10, 2000)))
    t.start()
    t.join()
    assert theirs[0] is theirs[1] and theirs[2] is not theirs[0] and all(x is not mine for x in theirs)
    assert sl._workspace(0, 5, 1000) is mine


def test_an_ended_threads_buffers_go(capturing):
    """Not at once: with the next buffer that is made."""
    mine = sl._workspace(0, 5, 1000)
    inside, done = threading.Event(), threading.Event()
    alive = threading.Thread(target=lambda: (sl._workspace(0, 5, 1000), inside.set(), done.wait(30)))
    ended = threading.Thread(target=lambda: [sl._workspace(0, s, 1000) for s in (5, 6, 7)])
    alive.start()                 # (before the other ends, whose number it could be given)
    assert inside.wait(30)
    ended.start()
    ended.join()
    assert len(sl._workspaces) == 5
    sl._workspace(1, 5, 1000)
    threads = {k[2] for k in sl._workspaces}
    assert threads == {threading.get_ident(), alive.ident} and len(sl._workspaces) == 3
    assert sl._workspace(0, 5, 1000) is mine
    done.set()
    alive.join()
