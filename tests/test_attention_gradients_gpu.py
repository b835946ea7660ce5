"""The attention calls compute no gradients: tensors that ask for one are refused instead of coming back without it."""
import pytest

from paper_2509_01229_amd import api

pytestmark = pytest.mark.gpu


def _calls():
    import torch

    T, Hq, Hkv, D = 4, 8, 2, 128
    made = {n: torch.randn((T, h, D), device="cuda").half() for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
    made |= {n: torch.rand(D, device="cuda") for n in ("q_norm", "k_norm")}
    made |= {"table": torch.rand((16, D), device="cuda"), "out_q": torch.empty((T, Hq, D), dtype=torch.float16, device="cuda"),
             "out_k": torch.empty((T, Hkv, D), dtype=torch.float16, device="cuda"), "out": torch.empty((T, Hq, D), dtype=torch.float16, device="cuda")}
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    cache, pages = api.kv4_cache(4, 16, Hkv, D), torch.zeros((T, 4), dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    calls = [
        (lambda q, k, table, q_norm, k_norm, out_q, out_k: api.attn_qk_norm_rope(q, k, pos, table, q_norm=q_norm, k_norm=k_norm, out_q=out_q, out_k=out_k),
         ("q", "k", "table", "q_norm", "k_norm", "out_q", "out_k")),
        (lambda k, v: api.kv4_write(k, v, pos, cache), ("k", "v")),
        (lambda q, k, v, table, q_norm, k_norm, out_q: api.kv4_append(q, k, v, pos, table, pos, cache, q_norm=q_norm, k_norm=k_norm, out_q=out_q),
         ("q", "k", "v", "table", "q_norm", "k_norm", "out_q")),
        (lambda q, out: api.kv4_attention(q, cache, pages, pos, out=out), ("q", "out")),
        (lambda q, k, v, out: api.attn_prompt(q, k, v, starts, out=out), ("q", "k", "v", "out")),
    ]
    return made, calls


@pytest.mark.parametrize("which", range(5))
@pytest.mark.parametrize("parameter", [False, True])
def test_what_asks_for_a_gradient_is_refused(which, parameter):
    import torch

    made, calls = _calls()
    call, names = calls[which]
    call(*(made[n] for n in names))
    for name in names:
        wanting = torch.nn.Parameter(made[name].clone()) if parameter else made[name].clone().requires_grad_()
        args = [wanting if n == name else made[n] for n in names]
        with pytest.raises(ValueError, match=name):
            call(*args)
        with torch.no_grad():
            call(*args)
        with torch.inference_mode():
            call(*args)
        call(*(a.detach() for a in args))
