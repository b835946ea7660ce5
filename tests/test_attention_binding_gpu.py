"""The attention calls through the native module against the ctypes path behind it: the same results, and the native module leaves
to the general path what is not the plain case."""
import numpy as np
import pytest

from paper_2509_01229_amd import api

pytestmark = pytest.mark.gpu


class _Nothing:
    rope = write = append = read = decode = prompt = staticmethod(lambda *a: None)


def _both(monkeypatch, call):
    import torch

    answers, native = [], api._native

    class Watched:
        def __getattr__(self, name):
            def run(*a):
                answers.append(getattr(native, name)(*a))
                return answers[-1]
            return run

    monkeypatch.setattr(api, "_native", Watched())
    fast = call()
    assert answers and all(a is not None for a in answers)
    monkeypatch.setattr(api, "_native", _Nothing)
    general = call()
    monkeypatch.setattr(api, "_native", native)
    flat = lambda r: list(r) if isinstance(r, tuple) else [r]
    assert len(flat(fast)) == len(flat(general))
    for f, g in zip(flat(fast), flat(general)):
        assert type(f) is type(g) and f.dtype == g.dtype and f.shape == g.shape and f.device == g.device and f.stride() == g.stride()
        assert torch.equal(f.view(torch.uint8), g.view(torch.uint8))
    return fast


def _inputs(dtype, T=5, Hq=8, Hkv=2, D=128):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(T)
    qkv = torch.randn((T, Hq + 2 * Hkv, D), generator=gen, device="cuda").to(dtype)
    return *qkv.split((Hq, Hkv, Hkv), 1), torch.arange(T, dtype=torch.int32, device="cuda"), torch.rand((16, D), generator=gen, device="cuda")


@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
def test_calls(monkeypatch, kind):
    import torch

    dtype = getattr(torch, kind)
    api.lib()
    q, k, v, pos, table = _inputs(dtype)
    w = torch.rand(128, device="cuda")
    cache = api.kv4_cache(4, 16, 2, 128)
    _both(monkeypatch, lambda: api.attn_qk_norm_rope(q, k, pos, table))
    out = torch.empty_like(q), torch.empty_like(k)
    r = _both(monkeypatch, lambda: api.attn_qk_norm_rope(q, k, pos, table, interleaved=True, q_norm=w, k_norm=w, eps=1e-5, out_q=out[0], out_k=out[1],
                                                        stream=torch.cuda.current_stream().cuda_stream))
    assert r[0] is out[0] and r[1] is out[1]
    assert _both(monkeypatch, lambda: api.kv4_write(k, v, pos, cache)) is cache
    _both(monkeypatch, lambda: api.kv4_append(q, k, v, pos, table, pos, cache))
    assert _both(monkeypatch, lambda: api.kv4_append(q, k, v, pos, table, pos, cache, q_norm=w, out_q=out[0])) is out[0]
    _both(monkeypatch, lambda: api.kv4_read(cache, pos, dtype=dtype))
    pages = torch.arange(4, dtype=torch.int32, device="cuda").repeat(5, 1)
    context = torch.full((5,), 5, dtype=torch.int32, device="cuda")
    api.kv4_attention(q, cache, pages, context)  # (makes this stream's workspace)
    _both(monkeypatch, lambda: api.kv4_attention(q, cache, pages, context))
    four, got = q.unsqueeze(1), torch.empty((5, 1, 8, 128), dtype=dtype, device="cuda")
    assert _both(monkeypatch, lambda: api.kv4_attention(four, cache, pages, context, scale=0.2, out=got)) is got
    ws = torch.zeros(max(16, int(api.lib().kv4_attention_workspace_size(5, 1, 8, 2, 128))), dtype=torch.uint8, device="cuda")
    _both(monkeypatch, lambda: api.kv4_attention(q, cache, pages, context, workspace=ws))
    _both(monkeypatch, lambda: api.kv4_attention(q, cache, pages, context, workspace=ws[:16]))
    starts = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    _both(monkeypatch, lambda: api.attn_prompt(q, k, v, starts))
    got = torch.empty((5, 8, 128), dtype=dtype, device="cuda")
    assert _both(monkeypatch, lambda: api.attn_prompt(q, k, v, starts, starts, scale=0.3, causal=False, out=got)) is got


def test_errors_of_the_library_are_raised(monkeypatch):
    import torch

    q, k, v, pos, table = _inputs(torch.float16, Hq=8, Hkv=3)
    starts = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    with pytest.raises(api.LiquidGemmError) as e:
        api.attn_prompt(q, k, v, starts)
    assert e.value.code == api.LQ_ERR_INVALID and "multiple" in str(e.value)
    with pytest.raises(api.LiquidGemmError):
        api.attn_qk_norm_rope(q, k, pos, table[:, :24].contiguous())


def test_what_is_not_plain_is_left_to_the_general_path():
    import torch

    api.lib()
    native = api._native
    q, k, v, pos, table = _inputs(torch.float16)
    cache = api.kv4_cache(4, 16, 2, 128)
    sub = type("Sub", (torch.Tensor,), {})
    for a in [(q.float(), k, pos, table), (q, k.bfloat16(), pos, table), (q[:, :, ::2], k, pos, table), (q, k[:4], pos, table), (q, k, pos.long(), table),
              (q, k, pos, table.T), (q.as_subclass(sub), k, pos, table), (q.cpu(), k, pos, table), (None, k, pos, table)]:
        assert native.rope(*a, False, None, None, 1e-6, None, None, None) is None
    assert native.rope(q, k, pos, table, 1, None, None, 1e-6, None, None, None) is None
    assert native.rope(q, k, pos, table, False, None, None, 1, None, None, None) is None
    assert native.write(k, v, pos, cache[:, :, :-8], None) is None and native.write(k, v, pos, cache[:, :1].contiguous(), None) is None
    assert native.read(cache, pos, None, None) is None
    pages = torch.zeros((5, 4), dtype=torch.int32, device="cuda")
    assert native.decode(q, cache, pages, pos, 1, None, None, None, {}) is None
    assert native.decode(q, cache, pages[:4], pos, None, None, None, None, {}) is None
    assert native.prompt(q, k, v, pos, pos, None, 1, None, None, None, {}) is None
