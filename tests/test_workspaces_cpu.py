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


def _needs():
    """What the calls of serving loops ask for, one after another."""
    L = api.lib()
    batches = [L.kv4_attention_workspace_size(n, 1, 32, 8, 128) for n in range(1, 600)]
    prompts = [L.attn_prompt_workspace_size(2, 40 * n, 40 * n + 100 * n, 32, 8, 128) for n in range(1, 200)]
    products = [api.w4a8_gemm_workspace_size(m, 4096, 14336, 64) for m in range(1, 300)]
    return {"batches": batches, "prompts": prompts, "products": products}


@pytest.mark.parametrize("kind", ["batches", "prompts", "products"])
def test_needs_that_grow_step_by_step(made, kind):
    """A larger buffer waits for the device and leaves the old one behind: as the needs grow, few are made, and what is left behind
    stays below what is in use."""
    needs = [n for n in _needs()[kind] if n]
    assert len(set(needs)) >= 5
    for need in needs:
        assert _ask(need, 5)[1] >= need
    kept = api._ws_cache[(0, 5)].numel()
    assert len(made) <= 12 and sum(b.numel() for b in api._ws_retired) <= kept <= 2 * max(needs)
