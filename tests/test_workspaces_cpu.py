"""The workspaces that the Python calls keep for each device and stream, without a GPU: memory is made on the host in their place."""
import threading
import time

import pytest

from paper_2509_01229_amd import api


@pytest.fixture
def made(monkeypatch):
    """Every buffer that is made from here on."""
    import torch

    buffers = []

    class Sized:  # stands for a buffer of n bytes
        def __init__(self, n):
            self.n = int(n)

        def numel(self):
            return self.n

    def make(n, dtype=None, device=None):
        time.sleep(0.02)
        buffers.append(Sized(n))
        return buffers[-1]

    monkeypatch.setattr(torch, "zeros", make)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    monkeypatch.setattr(api, "_dev", lambda t, *a, **k: t)
    monkeypatch.setattr(api, "_ws_cache", {})
    monkeypatch.setattr(api, "_ws_retired", [])
    return buffers


def _ask(need, stream):
    import torch

    return api._ws(None, device=torch.device("cuda", 0), stream=stream, need=need)


def test_threads_that_need_one_at_once(made):
    """A buffer that a call has been given is kept: work that uses it may still be in the stream's queue when the call returns."""
    given, start = [], threading.Barrier(8)

    def work(i):
        start.wait()
        given.append(_ask(1 << (16 + i // 2), 5))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(8)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    kept = [*api._ws_cache.values(), *api._ws_retired]
    assert len(given) == 8 and all(any(b is k for k in kept) for b, _ in given)
    assert all(any(b is k for k in kept) for b in made)
    assert api._ws_cache[(0, 5)].numel() >= 1 << 19
